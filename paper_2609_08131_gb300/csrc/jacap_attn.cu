// jacap_attn.cu - host side of the entry points around the cached tokens' attention
// (declared in include/jacap.h): rotary positions, attention of drafted tokens, and the
// weights that the cached tokens received. Arguments are checked before anything is
// enqueued; nothing is allocated.
#include <algorithm>
#include <math.h>
#include <string.h>

#include "jacap.h"
#include "jacap_dev.cuh"
#include "jacap_internal.h"

using namespace jacap;

namespace {

constexpr size_t ALIGN = 1024;
inline size_t align_up(size_t x) { return (x + ALIGN - 1) & ~(ALIGN - 1); }

// The tensor cores' float32 sums truncate: of the eight K-steps of a dot product of 128 channels the j-th
// loses 2^-24 / (2 ln 2) of a sum of about j / 8 of the whole on average over a mantissa, together 9 2^-23 /
// (8 ln 2) of it, by which logits are too small; the scale makes up for that.
constexpr double TRUNCATION = 9.0 * 1.1920928955078125e-07 * 0.18033688011112042;

// ------------------------------------------------------------- attention ----
constexpr int AT_DRAFTS_MAX = 64;

// How a call is split: `chunk` tokens per CTA, `nsplit` splits of the longest request,
// `nrb` row blocks. Depends on the layout alone (a GB300 has 152 SMs), so that the
// workspace does.
struct AttendPlan {
  int chunk, nsplit, nrb, block, edge, slots, srows;
  size_t status, counts, nsps, opart, mlpart, total;
};
constexpr int64_t F32_EXTRA = 128;
AttendPlan attend_plan(const jacap_layout* L) {
  AttendPlan p;
  const int bf = L->dtype == JACAP_BF16 ? 1 : 0, rows = L->num_q_heads / L->num_kv_heads * L->window;
  const int block = attend_row_block(bf, rows);
  p.nrb = (rows + block - 1) / block;
  const int64_t units = (int64_t)L->num_seqs * L->num_layers * L->num_kv_heads, ctas = units * p.nrb;
  const int64_t most = L->max_seqlen;
  // bf16: the least that a CTA's share may have (the kernel shares out the live tokens); a split's sums,
  // written and read by the join, stay an eighth of its K and V on the average. float32: of the splits of 128
  // tokens or more that fill one to four rounds of CTAs (three, two or one on an SM), or none, those whose last
  // round ends first, with F32_EXTRA tokens' time for a CTA's start and end (64 to 512 measured alike).
  int64_t chunk = std::max<int64_t>(256, std::min(rows, block) * 16);
  if (!bf) {
    const int64_t places = 152 * (block <= 8 ? 3 : (block == 16 ? 2 : 1));
    int64_t best = INT64_MAX;
    for (int64_t rounds = 0; rounds <= 4; ++rounds) {
      const int64_t k = std::max<int64_t>(1, rounds * places / ctas);
      const int64_t c = std::max<int64_t>(128, ((most + k - 1) / k + 63) / 64 * 64), items = (most + c - 1) / c * ctas;
      const int64_t time = (items + places - 1) / places * (c + F32_EXTRA);
      if (time < best) best = time, chunk = c;
    }
  }
  chunk = std::min<int64_t>((chunk + 63) / 64 * 64, (most + 63) / 64 * 64);
  p.chunk = (int)chunk;
  p.nsplit = (int)((most + chunk - 1) / chunk);
  p.block = block;
  p.edge = std::max(4, std::min(rows, block) / 16);
  if (bf) p.nsplit = (most + 63) / 64 + 1 < 2 * p.edge ? 1 : p.nsplit + 2;  // a share's borders are anywhere in a unit
  size_t o = 0;
  p.status = o; o += 64;
  // (whatever the layout, so that calls of several layouts may use a workspace one after the other)
  p.counts = o; o = align_up(o + (size_t)ATTEND_CTAS * 4);
  static_assert(64 + (size_t)ATTEND_CTAS * 4 <= JACAP_ATTEND_ZERO_BYTES, "what starts at zero");
  p.nsps = o; o = align_up(o + (bf ? (size_t)ctas * 4 : 0));
  // bf16: two slots for each border between CTAs, whatever the units' number: the split before and the one after
  const int64_t most_ctas = ATTEND_CTAS * 128 / block;
  const int64_t slots = bf ? 2 * (std::min<int64_t>(ctas * p.nsplit, most_ctas) - 1) : units * p.nsplit;
  const size_t parts = p.nsplit > 1 ? (size_t)slots : 0, prows = attend_part_rows(rows);
  p.slots = bf ? (int)slots : 0;
  p.srows = bf ? std::min(rows, block) : rows;
  p.opart = o; o = align_up(o + parts * ((p.srows + prows - 1) / prows * prows) * D * 4);
  p.mlpart = o; o = align_up(o + parts * p.srows * 8);
  p.total = o;
  return p;
}

jacap_status check_attend_layout(const jacap_layout* L) {
  const jacap_status st = check_layout(L);
  if (st != JACAP_OK) return st;
  const int64_t planes = (int64_t)L->num_layers * L->num_kv_heads, units = layout_units(L);
  const int64_t rows = (int64_t)L->num_q_heads / L->num_kv_heads * L->window;
  if (L->window > AT_DRAFTS_MAX || units * rows > INT32_MAX / 8) return JACAP_ERR_UNSUPPORTED;
  const AttendPlan p = attend_plan(L);
  if (units * p.nsplit * p.nrb > INT32_MAX) return JACAP_ERR_UNSUPPORTED;
  // the positions on the line of tiles (k_attend.cu): at most 4 for each of a request's tiles, and of AT_START more
  if (L->total_tokens / 64 + 8 * (int64_t)L->num_seqs > INT32_MAX / 4 / (planes * p.nrb)) return JACAP_ERR_UNSUPPORTED;
  return JACAP_OK;
}

// ----------------------------------------------------------------- weights ----
struct WeighCarve {
  size_t status, plan, chunks, counters, runs, sched, lse, stat, norm, total;
};
WeighCarve carve_weigh(const Dims& dm) {
  WeighCarve c;
  const size_t planes = (size_t)dm.L * dm.Hkv, rows = ((size_t)dm.G * dm.window + 127) / 128 * 128;
  size_t o = 0;
  c.status = o; o = align_up(o + 64);
  c.plan = o; o = align_up(o + ((size_t)dm.S + 2) * 4);
  c.chunks = o; o = align_up(o + (size_t)dm.c_cap * 16);
  c.counters = o; o = align_up(o + planes * dm.S * 8);
  c.runs = o; o = align_up(o + 2 * (size_t)dm.c_cap * 16);
  c.sched = o; o = align_up(o + 32 + (2 * ((size_t)dm.S + 2) + dm.S + 1 + 1) * 4);
  c.lse = o; o = align_up(o + (size_t)dm.S * dm.L * dm.Hq * dm.window * 4);
  c.stat = o; o = align_up(o + planes * (size_t)dm.c_cap * 2 * rows * 8);
  c.norm = o; o = align_up(o + planes * dm.S * rows * 8);
  c.total = o;
  return c;
}
Ws make_weigh_ws(void* base, const WeighCarve& c, const Dims& dm) {
  uint8_t* b = (uint8_t*)base;
  Ws ws;
  memset(&ws, 0, sizeof(ws));
  ws.status = (uint32_t*)(b + c.status);
  ws.plan = (int32_t*)(b + c.plan);
  ws.chunks = (int4*)(b + c.chunks);
  ws.gcount = (int32_t*)(b + c.counters);
  ws.fdone = ws.gcount + (size_t)dm.L * dm.Hkv * dm.S;
  ws.runs = (int4*)(b + c.runs);
  ws.sched = (int32_t*)(b + c.sched);
  ws.rplan = ws.sched + 8;
  ws.tpre = ws.rplan + 2 * ((size_t)dm.S + 2);
  ws.starts = ws.tpre + dm.S + 1;
  return ws;
}
jacap_status check_weigh_layout(const jacap_layout* L) {
  const jacap_status st = check_layout(L);
  if (st != JACAP_OK) return st;
  const int64_t rows = (int64_t)L->num_q_heads / L->num_kv_heads * L->window;
  if (rows > WEIGH_ROWS_MAX || layout_units(L) * ((rows + 31) / 32) > INT32_MAX) return JACAP_ERR_UNSUPPORTED;
  Dims dm;
  make_dims(L, nullptr, dm);
  return plan_items(L, dm) > INT32_MAX ? JACAP_ERR_UNSUPPORTED : JACAP_OK;
}

// far enough from the ends of float32 for the scale times log2 e and what is divided by it
bool scale_ok(float s) { return s >= 1e-30f && s <= 1e30f; }
bool aligned4(const void* p) { return ((uintptr_t)p & 3u) == 0; }
bool aligned8(const void* p) { return ((uintptr_t)p & 7u) == 0; }

}  // namespace

extern "C" {

jacap_status jacap_rotate(const jacap_rope* rope, jacap_dtype dtype, int32_t num_seqs, int32_t tokens,
                          const int32_t* positions, const int64_t* position_strides, int32_t inverse,
                          const jacap_rope_tensor* q, const jacap_rope_tensor* k, void* stream) {
  if (rope == nullptr || positions == nullptr || position_strides == nullptr || (q == nullptr && k == nullptr))
    return JACAP_ERR_INVALID_ARG;
  if ((dtype != JACAP_F32 && dtype != JACAP_BF16) || num_seqs < 0 || tokens < 0 ||
      (int64_t)num_seqs * tokens > INT32_MAX - 4 || (inverse != 0 && inverse != 1))
    return JACAP_ERR_INVALID_ARG;
  if (rope->head_dim != D) return JACAP_ERR_UNSUPPORTED;
  if (rope->rot_dim < 2 || rope->rot_dim > D || rope->rot_dim % 2 != 0 || rope->turns == nullptr ||
      (rope->interleaved != 0 && rope->interleaved != 1) || !isfinite(rope->amplitude))
    return JACAP_ERR_INVALID_ARG;
  if (!aligned4(positions) || !aligned8(rope->turns) || position_strides[0] < 0 || position_strides[1] < 0)
    return JACAP_ERR_INVALID_ARG;
  const int es = dtype == JACAP_BF16 ? 2 : 4, V = 16 / es;
  bool vec = (rope->interleaved ? rope->rot_dim : rope->rot_dim / 2) % V == 0 && rope->rot_dim % V == 0;
  RopeArgs a;
  memset(&a, 0, sizeof(a));
  const jacap_rope_tensor* in[2] = {q, k};
  RopeTensor* out[2] = {&a.q, &a.k};
  for (int i = 0; i < 2; ++i) {
    if (in[i] == nullptr) continue;
    const jacap_rope_tensor& t = *in[i];
    if (t.x == nullptr || t.y == nullptr || t.heads < 1 || t.heads > (1 << 20)) return JACAP_ERR_INVALID_ARG;
    if ((uintptr_t)t.x % es != 0 || (uintptr_t)t.y % es != 0) return JACAP_ERR_INVALID_ARG;
    const int64_t count[3] = {num_seqs, tokens, t.heads};
    for (int d = 0; d < 3; ++d) {
      // rows of the result do not overlap; in place the two are laid out alike
      if (t.x_strides[d] < 0 || t.y_strides[d] < 0 || (count[d] > 1 && t.y_strides[d] < D))
        return JACAP_ERR_INVALID_ARG;
      if (t.x == t.y && count[d] > 1 && t.x_strides[d] != t.y_strides[d]) return JACAP_ERR_INVALID_ARG;
      if (count[d] > 1) vec = vec && t.x_strides[d] % V == 0 && t.y_strides[d] % V == 0;
      out[i]->xs[d] = t.x_strides[d];
      out[i]->ys[d] = t.y_strides[d];
    }
    vec = vec && aligned16(t.x) && aligned16(t.y);
    out[i]->x = t.x;
    out[i]->y = t.y;
    out[i]->heads = t.heads;
  }
  int sms = 0;
  const jacap_status st = check_device(&sms);
  if (st != JACAP_OK) return st;
  if (num_seqs == 0 || tokens == 0) return JACAP_OK;
  a.pos = positions;
  a.ps[0] = position_strides[0];
  a.ps[1] = position_strides[1];
  a.turns = rope->turns;
  a.seqs = num_seqs;
  a.tokens = tokens;
  a.rot = rope->rot_dim;
  a.interleaved = rope->interleaved;
  a.inverse = inverse;
  a.amplitude = rope->amplitude;
  const TraceRange trace("jacap/rotate");
  return map_cuda(launch_rope(a, dtype == JACAP_BF16 ? 1 : 0, vec, sms, (cudaStream_t)stream));
}

size_t jacap_attend_workspace(const jacap_layout* layout) {
  return check_attend_layout(layout) == JACAP_OK ? attend_plan(layout).total : 0;
}

jacap_status jacap_attend(const jacap_layout* layout, const jacap_attention* attn, const void* q, const void* k,
                          const void* v, void* o, float* lse, void* ws, size_t ws_bytes, void* stream) {
  jacap_status st = check_attend_layout(layout);
  if (st != JACAP_OK) return st;
  if (attn == nullptr || q == nullptr || k == nullptr || v == nullptr || o == nullptr || ws == nullptr)
    return JACAP_ERR_INVALID_ARG;
  if (!scale_ok(attn->scale)) return JACAP_ERR_INVALID_ARG;
  if ((attn->k_draft == nullptr) != (attn->v_draft == nullptr) || (attn->tree != nullptr && attn->k_draft == nullptr))
    return JACAP_ERR_INVALID_ARG;
  if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(o) || !aligned4(lse) || !aligned4(attn->lengths) ||
      !aligned4(attn->draft_lens) || !aligned8(attn->tree) || !aligned16(attn->k_draft) || !aligned16(attn->v_draft))
    return JACAP_ERR_INVALID_ARG;
  const bool bf = layout->dtype == JACAP_BF16;
  const int64_t el16 = bf ? 8 : 4;
  const int64_t count[4] = {layout->num_seqs, layout->num_layers, layout->num_q_heads, layout->window};
  for (int i = 0; i < 4; ++i) {
    if (attn->o_strides[i] % el16 != 0 || attn->o_strides[i] < (count[i] > 1 ? D : 0)) return JACAP_ERR_INVALID_ARG;
  }
  for (int i = 0; lse != nullptr && i < 3; ++i)
    if (attn->lse_strides[i] < (count[i] > 1 ? layout->window : 0)) return JACAP_ERR_INVALID_ARG;
  for (int i = 0; attn->k_draft != nullptr && i < 8; ++i)
    if (attn->draft_strides[i] % el16 != 0 || attn->draft_strides[i] < D || attn->draft_strides[i] >= (1ll << 38))
      return JACAP_ERR_INVALID_ARG;
  const AttendPlan p = attend_plan(layout);
  if (((uintptr_t)ws & 255u) != 0 || ws_bytes < p.total) return JACAP_ERR_WORKSPACE;
  int sms = 0;
  if ((st = check_device(&sms)) != JACAP_OK) return st;
  Dims dm;
  make_dims(layout, nullptr, dm);
  AttendArgs a;
  memset(&a, 0, sizeof(a));
  a.q = q, a.k = k, a.v = v, a.kd = attn->k_draft, a.vd = attn->v_draft, a.o = o, a.lse = lse;
  a.lengths = attn->lengths;
  a.draft_lens = attn->draft_lens;
  a.tree = attn->tree;
  for (int i = 0; i < 4; ++i) {
    a.os[i] = attn->o_strides[i];
    a.kds[i] = attn->k_draft != nullptr ? attn->draft_strides[i] : 0;
    a.vds[i] = attn->k_draft != nullptr ? attn->draft_strides[4 + i] : 0;
  }
  for (int i = 0; i < 3; ++i) a.ls[i] = attn->lse_strides[i];
  a.scale2 = (float)((double)attn->scale * 1.4426950408889634 * (bf ? 1.0 + TRUNCATION : 1.0));
  a.slots = p.slots, a.srows = p.srows, a.prows = attend_part_rows(dm.G * dm.window);
  a.tdiv = dm.window > 1 ? 0xffffffffu / (uint32_t)dm.window + 1u : 0u;
  a.chunk = p.chunk, a.nsplit = p.nsplit, a.nrb = p.nrb, a.max_seqlen = layout->max_seqlen;
  a.block = p.block, a.least = p.chunk / 64, a.edge = p.edge;
  uint8_t* b = (uint8_t*)ws;
  a.status = (uint32_t*)(b + p.status);
  a.counts = (int32_t*)(b + p.counts);
  a.nsps = (int32_t*)(b + p.nsps);
  a.opart = (float*)(b + p.opart);
  a.mlpart = (float*)(b + p.mlpart);
  CUtensorMap maps[4];
  memset(maps, 0, sizeof(maps));
  if (bf) {
    if (!encode_kv_map(&maps[0], layout, k, 64) || !encode_kv_map(&maps[1], layout, v, 64)) return JACAP_ERR_CUDA;
    if (a.kd != nullptr && (!encode_draft_map(&maps[2], layout, a.kd, a.kds, layout->window) ||
                            !encode_draft_map(&maps[3], layout, a.vd, a.vds, layout->window)))
      return JACAP_ERR_CUDA;
  }
  const TraceRange trace("jacap/attend");
  return map_cuda(launch_attend(maps, dm, bf ? 1 : 0, a, layout->cu_seqlens, sms, (cudaStream_t)stream));
}

size_t jacap_weigh_workspace(const jacap_layout* layout) {
  if (check_weigh_layout(layout) != JACAP_OK) return 0;
  Dims dm;
  make_dims(layout, nullptr, dm);
  return carve_weigh(dm).total;
}

jacap_status jacap_weigh(const jacap_layout* layout, const jacap_weighing* how, const void* q_win, const void* k,
                         float* lse, const float* before, float* weights, void* ws, size_t ws_bytes, void* stream) {
  jacap_status st = check_weigh_layout(layout);
  if (st != JACAP_OK) return st;
  if (how == nullptr || q_win == nullptr || k == nullptr || weights == nullptr || ws == nullptr)
    return JACAP_ERR_INVALID_ARG;
  if (!scale_ok(how->scale) || (how->lse_given != 0 && how->lse_given != 1) || (how->lse_given == 1 && lse == nullptr))
    return JACAP_ERR_INVALID_ARG;
  if (!aligned16(q_win) || !aligned16(k) || !aligned4(lse) || !aligned4(before) || !aligned4(weights) ||
      !aligned4(how->lengths) || !aligned4(how->q_lens) || !aligned4(how->q_rows))
    return JACAP_ERR_INVALID_ARG;
  Dims dm;
  make_dims(layout, nullptr, dm);
  const WeighCarve c = carve_weigh(dm);
  if (((uintptr_t)ws & 255u) != 0 || ws_bytes < c.total) return JACAP_ERR_WORKSPACE;
  int sms = 0;
  if ((st = check_device(&sms)) != JACAP_OK) return st;
  const bool bf = layout->dtype == JACAP_BF16;
  CUtensorMap kmap;
  memset(&kmap, 0, sizeof(kmap));
  if (bf && !encode_kv_map(&kmap, layout, k)) return JACAP_ERR_CUDA;
  const int64_t items = plan_items(layout, dm);
  plan_runs(dm, items, sms);
  dm.gram_parts = 0;
  const Ws w = make_weigh_ws(ws, c, dm);
  uint8_t* b = (uint8_t*)ws;
  WeighArgs a;
  memset(&a, 0, sizeof(a));
  a.q = q_win, a.k = k;
  a.lengths = how->lengths, a.q_lens = how->q_lens, a.q_rows = how->q_rows;
  a.lse = lse != nullptr ? lse : (float*)(b + c.lse);
  a.given = how->lse_given;
  a.before = before;
  a.weights = weights;
  a.scale2 = (float)((double)how->scale * 1.4426950408889634 * (bf ? 1.0 + TRUNCATION : 1.0));
  a.tdiv = dm.window > 1 ? 0xffffffffu / (uint32_t)dm.window + 1u : 0u;
  a.stat = (float2*)(b + c.stat);
  a.norm = (float2*)(b + c.norm);
  const cudaStream_t s = (cudaStream_t)stream;
  const TraceRange trace("jacap/weigh");
  if ((st = map_cuda(launch_plan(dm, w, layout->cu_seqlens, s, how->lengths))) != JACAP_OK) return st;
  return map_cuda(launch_weigh(kmap, dm, w, bf ? 1 : 0, a, layout->cu_seqlens, plan_grid(items, sms), s));
}

}  // extern "C"
