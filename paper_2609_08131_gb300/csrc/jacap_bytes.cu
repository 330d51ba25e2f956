// jacap_bytes.cu - host side of the entry points of a cache held in 8 bits and of the
// verification of drafted tokens (declared in include/jacap.h). Arguments are checked before
// anything is enqueued; nothing is allocated.
#include <algorithm>
#include <string.h>

#include "jacap.h"
#include "jacap_dev.cuh"
#include "jacap_internal.h"

using namespace jacap;

namespace {

constexpr int DRAFTS_MAX = 64;
inline size_t align_up(size_t x) { return (x + 1023) & ~(size_t)1023; }
bool aligned4(const void* p) { return ((uintptr_t)p & 3u) == 0; }
bool aligned8(const void* p) { return ((uintptr_t)p & 7u) == 0; }

jacap_status check_cache(const jacap_byte_cache* c) {
  if (c == nullptr || c->k == nullptr || c->v == nullptr || c->k_scales == nullptr || c->v_scales == nullptr)
    return JACAP_ERR_INVALID_ARG;
  if (c->num_seqs < 1 || c->num_layers < 1 || c->num_q_heads < 1 || c->num_kv_heads < 1 || c->slot_tokens < 1 ||
      c->slot_tokens % 64 != 0 || c->num_q_heads % c->num_kv_heads != 0)
    return JACAP_ERR_INVALID_ARG;
  if (!aligned16(c->k) || !aligned16(c->v) || !aligned4(c->k_scales) || !aligned4(c->v_scales))
    return JACAP_ERR_INVALID_ARG;
  const int64_t count[3] = {c->num_layers, c->num_kv_heads, c->num_seqs};
  for (int i = 0; i < 3; ++i) {
    if (count[i] == 1) continue;
    if (c->strides[i] % 16 != 0 || c->strides[i] < (int64_t)c->slot_tokens * D || c->strides[i] >= (1ll << 40) ||
        c->scale_strides[i] < c->slot_tokens / 64)
      return JACAP_ERR_INVALID_ARG;
  }
  if (c->head_dim != D || c->num_q_heads / c->num_kv_heads > G_MAX) return JACAP_ERR_UNSUPPORTED;
  // positions on the line of tiles (k_attend_body.cuh), and items of a call: both tensors' blocks of 64 tokens in all units
  const int64_t planes = (int64_t)c->num_layers * c->num_kv_heads, blocks = c->slot_tokens / 64;
  const int64_t rb = c->num_q_heads / c->num_kv_heads;  // (row blocks at most)
  if (planes > INT32_MAX / (blocks + 8) / c->num_seqs / std::max<int64_t>(2, rb) || c->num_seqs > INT32_MAX / 64)
    return JACAP_ERR_UNSUPPORTED;
  return JACAP_OK;
}

// How attention of `tokens` queries is split: `least` tiles of 128 tokens of a CTA's share at least, `nsplit` splits
// of a unit and row block at most, `edge` tiles between a split's border and a unit's start or end.
struct BytesPlan {
  int rows, block, nrb, least, nsplit, edge, srows, slots;
};
BytesPlan plan_of(const jacap_byte_cache* c, int tokens) {
  BytesPlan p;
  p.rows = c->num_q_heads / c->num_kv_heads * tokens;
  p.block = attend_bytes_block(p.rows);
  p.nrb = (p.rows - 1) / p.block + 1;
  // a split's sums, written and read by the join, are at most half of its K and V
  p.least = p.edge = std::max(2, std::min(p.rows, p.block) / 32);
  const int64_t tiles = (c->slot_tokens - 1) / 128 + 2, units = (int64_t)c->num_seqs * c->num_layers * c->num_kv_heads;
  p.nsplit = tiles < 2 * p.edge ? 1 : (int)((tiles - 1) / p.least + 2);  // a share's borders are anywhere in a unit
  // two slots for each border between CTAs: the split before and the one after
  p.slots = (int)(2 * (std::min<int64_t>(units * p.nrb * p.nsplit, attend_bytes_ctas(p.block)) - 1));
  p.srows = std::min(p.rows, p.block);
  return p;
}

// The workspace: the status word and the counters of the attention's splits (at the places of jacap_attend's), a counter
// per request, then what need not be zero.
struct BytesCarve {
  size_t counts, opart, mlpart, total;
};
BytesCarve carve(const jacap_byte_cache* c, int tokens) {
  BytesCarve b;
  size_t o = JACAP_ATTEND_ZERO_BYTES;
  b.counts = o; o = align_up(o + (size_t)c->num_seqs * 4);
  b.opart = b.mlpart = o;
  size_t most = o;
  for (int t = 1; t <= tokens; ++t) {  // (calls of fewer tokens too)
    const BytesPlan p = plan_of(c, t);
    size_t at = o;
    const size_t parts = p.nsplit > 1 ? (size_t)p.slots : 0;
    b.opart = at; at = align_up(at + parts * p.srows * D * 4);
    b.mlpart = at; at += parts * p.srows * 8;
    most = std::max(most, align_up(at));
  }
  b.total = most;
  return b;
}

// Checks shared by store and append; `tokens` rows of K and V per request, and the arguments of both.
jacap_status byte_args(const jacap_byte_cache* c, jacap_dtype dtype, const void* k, const void* v,
                       const int64_t* strides, int tokens, void* ws, size_t ws_bytes, ByteArgs& a) {
  if (dtype != JACAP_F32 && dtype != JACAP_BF16) return JACAP_ERR_INVALID_ARG;
  if (strides == nullptr || !aligned16(k) || !aligned16(v)) return JACAP_ERR_INVALID_ARG;
  if (tokens > 0 && (k == nullptr || v == nullptr)) return JACAP_ERR_INVALID_ARG;  // (no rows have no address)
  const int64_t el16 = dtype == JACAP_BF16 ? 8 : 4;
  const int64_t count[4] = {c->num_seqs, c->num_layers, c->num_kv_heads, tokens};
  memset(&a, 0, sizeof(a));
  for (int i = 0; i < 8; ++i) {
    if (count[i & 3] <= 1) continue;  // (the stride of an axis of one entry means nothing)
    if (strides[i] < 0 || strides[i] % el16 != 0 || strides[i] >= (1ll << 40)) return JACAP_ERR_INVALID_ARG;
    a.row_strides[i] = strides[i];
  }
  const size_t counts = JACAP_ATTEND_ZERO_BYTES;
  if (ws == nullptr || ((uintptr_t)ws & 255u) != 0 || ws_bytes < counts + (size_t)c->num_seqs * 4)
    return JACAP_ERR_WORKSPACE;
  a.rows_in[0] = k, a.rows_in[1] = v;
  a.bytes[0] = (uint8_t*)c->k, a.bytes[1] = (uint8_t*)c->v;
  a.scales[0] = c->k_scales, a.scales[1] = c->v_scales;
  for (int i = 0; i < 3; ++i) {
    a.strides[i] = c->strides[i];
    a.scale_strides[i] = c->scale_strides[i];
  }
  a.S = c->num_seqs, a.L = c->num_layers, a.Hkv = c->num_kv_heads;
  a.status = (uint32_t*)ws;
  a.counts = (int32_t*)((uint8_t*)ws + counts);
  int sms = 0;
  return check_device(&sms);
}

}  // namespace

extern "C" {

size_t jacap_bytes_workspace(const jacap_byte_cache* cache, int32_t tokens) {
  if (check_cache(cache) != JACAP_OK || tokens < 1 || tokens > DRAFTS_MAX) return 0;
  return carve(cache, tokens).total;
}

jacap_status jacap_bytes_store(const jacap_byte_cache* cache, jacap_dtype dtype, const void* k_rows,
                               const void* v_rows, const int64_t* row_strides, int32_t rows, const int32_t* lengths,
                               int32_t* lengths_out, void* ws, size_t ws_bytes, void* stream) {
  jacap_status st = check_cache(cache);
  if (st != JACAP_OK) return st;
  if (rows < 0 || rows > cache->slot_tokens || !aligned4(lengths) || !aligned4(lengths_out)) return JACAP_ERR_INVALID_ARG;
  ByteArgs a;
  if ((st = byte_args(cache, dtype, k_rows, v_rows, row_strides, rows, ws, ws_bytes, a)) != JACAP_OK) return st;
  a.rows = rows;
  a.blocks = rows > 0 ? (rows - 1) / 64 + 1 : 1;
  a.lengths = lengths, a.lengths_out = lengths_out;
  const TraceRange trace("jacap/bytes_store");
  return map_cuda(launch_bytes_store(a, dtype == JACAP_BF16 ? 1 : 0, (cudaStream_t)stream));
}

jacap_status jacap_bytes_append(const jacap_byte_cache* cache, jacap_dtype dtype, const void* k_new,
                                const void* v_new, const int64_t* new_strides, int32_t tokens, const int32_t* path,
                                const int32_t* taken, const int32_t* lengths, int32_t* lengths_out, void* ws,
                                size_t ws_bytes, void* stream) {
  jacap_status st = check_cache(cache);
  if (st != JACAP_OK) return st;
  if (tokens < 1 || lengths == nullptr || !aligned4(lengths) || !aligned4(lengths_out) || !aligned4(path) ||
      !aligned4(taken))
    return JACAP_ERR_INVALID_ARG;
  if (tokens > DRAFTS_MAX) return JACAP_ERR_UNSUPPORTED;
  ByteArgs a;
  if ((st = byte_args(cache, dtype, k_new, v_new, new_strides, tokens, ws, ws_bytes, a)) != JACAP_OK) return st;
  a.rows = cache->slot_tokens;
  a.tokens = tokens;
  a.lengths = lengths, a.lengths_out = lengths_out;
  a.path = path, a.taken = taken;
  const TraceRange trace("jacap/bytes_append");
  return map_cuda(launch_bytes_append(a, dtype == JACAP_BF16 ? 1 : 0, (cudaStream_t)stream));
}

jacap_status jacap_bytes_attend(const jacap_byte_cache* cache, const jacap_attention* attn, int32_t tokens,
                                const void* q, const int64_t* q_strides, void* o, float* lse, void* ws,
                                size_t ws_bytes, void* stream) {
  jacap_status st = check_cache(cache);
  if (st != JACAP_OK) return st;
  if (attn == nullptr || q == nullptr || q_strides == nullptr || o == nullptr || tokens < 1) return JACAP_ERR_INVALID_ARG;
  if (tokens > DRAFTS_MAX) return JACAP_ERR_UNSUPPORTED;
  if (!(attn->scale >= 1e-30f && attn->scale <= 1e30f) || attn->lengths == nullptr) return JACAP_ERR_INVALID_ARG;
  if ((attn->k_draft == nullptr) != (attn->v_draft == nullptr) || (attn->tree != nullptr && attn->k_draft == nullptr))
    return JACAP_ERR_INVALID_ARG;
  if (!aligned16(q) || !aligned16(o) || !aligned4(lse) || !aligned4(attn->lengths) || !aligned4(attn->draft_lens) ||
      !aligned8(attn->tree) || !aligned16(attn->k_draft) || !aligned16(attn->v_draft))
    return JACAP_ERR_INVALID_ARG;
  const int64_t count[4] = {cache->num_seqs, cache->num_layers, cache->num_q_heads, tokens};
  for (int i = 0; i < 4; ++i) {
    if (attn->o_strides[i] % 8 != 0 || attn->o_strides[i] < (count[i] > 1 ? D : 0)) return JACAP_ERR_INVALID_ARG;
    if (count[i] > 1 && (q_strides[i] % 8 != 0 || q_strides[i] < 0 || q_strides[i] >= (1ll << 40)))
      return JACAP_ERR_INVALID_ARG;
  }
  for (int i = 0; lse != nullptr && i < 3; ++i)
    if (attn->lse_strides[i] < (count[i] > 1 ? tokens : 0)) return JACAP_ERR_INVALID_ARG;
  for (int i = 0; attn->k_draft != nullptr && i < 8; ++i)
    if (attn->draft_strides[i] % 8 != 0 || attn->draft_strides[i] < D || attn->draft_strides[i] >= (1ll << 38))
      return JACAP_ERR_INVALID_ARG;
  const BytesCarve c = carve(cache, tokens);
  if (ws == nullptr || ((uintptr_t)ws & 255u) != 0 || ws_bytes < c.total) return JACAP_ERR_WORKSPACE;
  int sms = 0;
  if ((st = check_device(&sms)) != JACAP_OK) return st;
  const BytesPlan p = plan_of(cache, tokens);
  Dims dm;
  memset(&dm, 0, sizeof(dm));
  dm.S = cache->num_seqs, dm.L = cache->num_layers, dm.Hq = cache->num_q_heads, dm.Hkv = cache->num_kv_heads;
  dm.G = dm.Hq / dm.Hkv;
  dm.window = tokens;
  dm.Ntot = cache->slot_tokens;
  dm.q_ss = q_strides[0], dm.q_sl = q_strides[1], dm.q_sh = q_strides[2], dm.q_sp = q_strides[3];
  AttendArgs a;
  memset(&a, 0, sizeof(a));
  a.q = q, a.kd = attn->k_draft, a.vd = attn->v_draft, a.o = o, a.lse = lse;
  a.lengths = attn->lengths;
  a.draft_lens = attn->draft_lens;
  a.tree = attn->tree;
  for (int i = 0; i < 4; ++i) {
    a.os[i] = attn->o_strides[i];
    a.kds[i] = attn->k_draft != nullptr ? attn->draft_strides[i] : 0;
    a.vds[i] = attn->k_draft != nullptr ? attn->draft_strides[4 + i] : 0;
  }
  for (int i = 0; i < 3; ++i) a.ls[i] = attn->lse_strides[i];
  a.scale2 = 1.f;
  a.nsplit = p.nsplit, a.nrb = p.nrb, a.max_seqlen = cache->slot_tokens;
  a.chunk = p.least * 128, a.block = p.block, a.least = p.least, a.edge = p.edge;
  a.slots = p.slots, a.srows = p.srows;
  a.tdiv = tokens > 1 ? 0xffffffffu / (uint32_t)tokens + 1u : 0u;
  uint8_t* b = (uint8_t*)ws;
  a.status = (uint32_t*)b;
  a.counts = (int32_t*)(b + 64);
  a.opart = (float*)(b + c.opart);
  a.mlpart = (float*)(b + c.mlpart);
  ByteScales sc;
  sc.ks = cache->k_scales, sc.vs = cache->v_scales;
  sc.k = (const uint8_t*)cache->k, sc.v = (const uint8_t*)cache->v;
  for (int i = 0; i < 3; ++i) sc.strides[i] = cache->scale_strides[i], sc.row_strides[i] = cache->strides[i];
  sc.scale2 = (float)((double)attn->scale * 1.4426950408889634);
  CUtensorMap maps[4];
  memset(maps, 0, sizeof(maps));
  jacap_layout lay;  // (the axes of the drafted rows)
  memset(&lay, 0, sizeof(lay));
  lay.num_seqs = dm.S, lay.num_layers = dm.L, lay.num_kv_heads = dm.Hkv;
  if (!encode_byte_map(&maps[0], cache, cache->k) || !encode_byte_map(&maps[1], cache, cache->v)) return JACAP_ERR_CUDA;
  if (a.kd != nullptr && (!encode_draft_map(&maps[2], &lay, a.kd, a.kds, tokens) ||
                          !encode_draft_map(&maps[3], &lay, a.vd, a.vds, tokens)))
    return JACAP_ERR_CUDA;
  const TraceRange trace("jacap/bytes_attend");
  return map_cuda(launch_attend_bytes(maps, dm, a, sc, sms, (cudaStream_t)stream));
}

jacap_status jacap_verify(const jacap_verification* how, void* status, void* stream) {
  if (how == nullptr || how->tokens_in == nullptr || how->p == nullptr || how->u == nullptr || how->path == nullptr ||
      how->taken == nullptr || how->next == nullptr)
    return JACAP_ERR_INVALID_ARG;
  if ((how->dtype != JACAP_F32 && how->dtype != JACAP_BF16) || how->num_seqs < 0 || how->tokens < 1 || how->vocab < 1)
    return JACAP_ERR_INVALID_ARG;
  const uintptr_t es = how->dtype == JACAP_BF16 ? 2 : 4;
  if (!aligned4(how->tokens_in) || !aligned8(how->tree) || !aligned4(how->draft_lens) || (uintptr_t)how->p % es != 0 ||
      (uintptr_t)how->q % es != 0 || !aligned4(how->u) || !aligned4(how->path) || !aligned4(how->taken) ||
      !aligned4(how->next))
    return JACAP_ERR_INVALID_ARG;
  for (int i = 0; i < 2; ++i)
    if (how->p_strides[i] < 0 || (how->q != nullptr && how->q_strides[i] < 0)) return JACAP_ERR_INVALID_ARG;
  // (a cluster of eight CTAs per request; the warps' parts are counted in 32 bits)
  if (how->tokens > DRAFTS_MAX || how->vocab > INT32_MAX / 2 || how->num_seqs > INT32_MAX / 64)
    return JACAP_ERR_UNSUPPORTED;
  if (status == nullptr || ((uintptr_t)status & 255u) != 0) return JACAP_ERR_WORKSPACE;
  int sms = 0;
  const jacap_status st = check_device(&sms);
  if (st != JACAP_OK) return st;
  if (how->num_seqs == 0) return JACAP_OK;
  const TraceRange trace("jacap/verify");
  return map_cuda(launch_verify(*how, (uint32_t*)status, (cudaStream_t)stream));
}

}  // extern "C"
