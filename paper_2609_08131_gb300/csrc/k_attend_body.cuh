// k_attend_body.cuh - what the attention kernels over cached and drafted tokens share
// (k_attend.cu, k_attend_bytes.cu): a call's units, the drafted tokens' masks, where splits' sums lie and how
// they are joined, and how the work is shared out.
#pragma once

#include "jacap_dev.cuh"
#include "jacap_internal.h"

namespace jacap {

constexpr int AT_QUEUE = 3;            // items published and not yet taken by all
// Two values at once: the same arithmetic in half the issue slots.
__device__ __forceinline__ float2 fma2(float2 x, float2 y, float2 z) {
  float2 r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;"
      : "=l"(*(uint64_t*)&r)
      : "l"(*(uint64_t*)&x), "l"(*(uint64_t*)&y), "l"(*(uint64_t*)&z));
  return r;
}
__device__ __forceinline__ float2 add2(float2 x, float2 y) {
  float2 r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(*(uint64_t*)&r) : "l"(*(uint64_t*)&x), "l"(*(uint64_t*)&y));
  return r;
}

__device__ __forceinline__ void tma_load_5d(uint32_t dst, const CUtensorMap* map, int c0, int c1, int c2, int c3,
                                            int c4, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.5d.shared::cta.global.tile.mbarrier::complete_tx::bytes"
      " [%0], [%1, {%2, %3, %4, %5, %6}], [%7];" ::"r"(dst),
      "l"(map), "r"(c0), "r"(c1), "r"(c2), "r"(c3), "r"(c4), "r"(bar)
      : "memory");
}

// What a CTA works on. `n` live cached tokens of the request, `rows` of its T queries
// (those behind are left alone), `nd` drafted tokens, `nsp` splits.
struct AtUnit {
  int s, l, g, split;
  int64_t u, t0;
  int n, rows, nd, nsp;
  int first;                   // bf16: the CTA that has the unit's first split
  int tok0, tok1, ncache, nt;  // this split's tokens, its tiles of cached tokens and in all (`tile` tokens each)
  int r0;                      // bf16: the CTA's first row (float32: 0)
};
// A request's live cached tokens and queries, clamped to what there can be (`ok`: nothing had to be). Without cu a
// request has a slot of max_seqlen tokens.
struct AtLive {
  int64_t start;
  int n, rows;
  bool ok;
};
__device__ __forceinline__ AtLive at_live(const Dims& dm, const AttendArgs& a, const int32_t* cu, int s) {
  AtLive x;
  const int64_t start = cu != nullptr ? cu[s] : 0, end = cu != nullptr ? cu[s + 1] : a.max_seqlen;
  const int given = a.lengths != nullptr ? a.lengths[s] : 0;
  const int want = a.draft_lens != nullptr ? a.draft_lens[s] : dm.window;
  const bool ok = start >= 0 && end >= start && end <= dm.Ntot;
  const int64_t room = ok ? (end - start < a.max_seqlen ? end - start : a.max_seqlen) : 0;
  const int64_t live = a.lengths != nullptr ? (int64_t)given : end - start;
  x.start = ok ? start : 0;
  x.n = (int)(live < 0 ? 0 : (live < room ? live : room));
  x.rows = want < 0 ? 0 : (want < dm.window ? want : dm.window);
  x.ok = ok && live == x.n && want == x.rows;
  return x;
}
__device__ __forceinline__ AtUnit at_unit(const Dims& dm, const AttendArgs& a, const int32_t* cu, int l, int g, int s,
                                          int split, int tile, int chunk) {
  AtUnit x;
  x.s = s, x.l = l, x.g = g;
  x.u = (uint32_t)(l * dm.Hkv + g) * dm.S + s;
  x.split = split;
  x.first = x.r0 = 0;
  const AtLive live = at_live(dm, a, cu, x.s);
  if (!live.ok) atomicOr(a.status, (uint32_t)ST_INVALID);
  x.t0 = live.start;
  x.n = live.n;
  x.rows = live.rows;
  x.nd = a.kd != nullptr ? x.rows : 0;
  x.nsp = x.n > chunk ? (x.n - 1) / chunk + 1 : 1;
  x.tok0 = split * chunk;
  x.tok1 = x.tok0 + chunk < x.n ? x.tok0 + chunk : x.n;
  x.ncache = x.tok1 > x.tok0 ? (x.tok1 - x.tok0 - 1) / tile + 1 : 0;
  x.nt = x.ncache + (split == x.nsp - 1 && x.nd > 0 ? (x.nd - 1) / tile + 1 : 0);
  return x;
}

__device__ __forceinline__ AtUnit at_unit(const Dims& dm, const AttendArgs& a, const int32_t* cu, uint32_t u, int split,
                                          int tile, int chunk) {  // (32-bit divisions: a 64-bit one takes ~300 cycles)
  const uint32_t plane = u / (uint32_t)dm.S, l = plane / (uint32_t)dm.Hkv;
  return at_unit(dm, a, cu, (int)l, (int)(plane - l * dm.Hkv), (int)(u - plane * dm.S), split, tile, chunk);
}

// Where a split's sums lie. bf16: a border between two CTAs divides one unit (and row block) at most, so the first
// split of a unit of several has slot 2 k, of the CTA k that has it, and each further one 2 k - 1. float32: by unit
// and split.
template <typename T>
__device__ __forceinline__ int64_t at_slot(const AttendArgs& a, const AtUnit& x, int split) {
  if constexpr (sizeof(T) == 2) return 2 * (x.first + split) - (split > 0 ? 1 : 0);
  return x.u * a.nsplit + split;
}
// A slot's unnormalised sums of row r: channels 4 c .. + 3 at [c prows] (the rows of a block lie
// next to each other, as a warp's lanes have them).
__device__ __forceinline__ float4* at_part(const AttendArgs& a, const AtUnit& x, int64_t slot, int r) {
  const int rows = a.prows, blocks = (a.srows - 1) / rows + 1, b = (r - x.r0) / rows;
  return (float4*)a.opart + (slot * blocks + b) * (32 * rows) + (r - x.r0 - b * rows);
}
// A slot's (maximum, sum) of row r.
__device__ __forceinline__ float2* at_ml(const AttendArgs& a, const AtUnit& x, int64_t slot, int r) {
  return (float2*)a.mlpart + slot * a.srows + (r - x.r0);
}

// Drafted tokens that drafted token t of request s sees (bit j: token j).
__device__ __forceinline__ uint64_t at_mask(const Dims& dm, const AttendArgs& a, const AtUnit& x, int t) {
  const uint64_t all = x.nd >= 64 ? ~0ull : (1ull << x.nd) - 1;
  if (t >= x.rows) return 0;
  return (a.tree != nullptr ? a.tree[(int64_t)x.s * dm.window + t] : (t >= 63 ? ~0ull : (2ull << t) - 1)) & all;
}

// Row r of a unit (unnormalised sums acc of channels 4 lane .. + 3, maximum m in logit
// units before the scale, sum z) to the output, or to the split's partial.
template <typename T>
__device__ __forceinline__ void at_put(const Dims& dm, const AttendArgs& a, const AtUnit& x, int r, float4 acc, float m,
                                       float z, int lane) {
  const int h = row_head(dm.window, a.tdiv, r), t = r - h * dm.window;
  if (t >= x.rows) return;
  if (x.nsp > 1) {
    const int64_t slot = at_slot<T>(a, x, x.split);
    at_part(a, x, slot, r)[lane * a.prows] = acc;
    if (lane == 0) *at_ml(a, x, slot, r) = make_float2(m, z);
    return;
  }
  const float inv = z == 0.f ? 0.f : 1.f / z;
  T* o = (T*)a.o + x.s * a.os[0] + x.l * a.os[1] + (int64_t)(x.g * dm.G + h) * a.os[2] + t * a.os[3] + 4 * lane;
  if constexpr (sizeof(T) == 2)
    *(uint2*)o = make_uint2(pack_bf16x2(acc.x * inv, acc.y * inv), pack_bf16x2(acc.z * inv, acc.w * inv));
  else
    *(float4*)o = make_float4(acc.x * inv, acc.y * inv, acc.z * inv, acc.w * inv);
  if (lane == 0 && a.lse != nullptr)
    a.lse[x.s * a.ls[0] + x.l * a.ls[1] + (x.g * dm.G + h) * a.ls[2] + t] =
        z == 0.f ? -INFINITY : m * (a.scale2 * 0.6931471805599453f) + logf(z);
}

// Few rows in few splits (bf16) are joined by the CTA that finishes the unit's last split; the others by a
// kernel of their own, which has more reads in flight.
__host__ __device__ __forceinline__ bool at_joins_inside(int nsp, int R) { return R <= 32 && nsp <= 16; }

// Rows r0 .. r0 + NR - 1 (4 or 8) of unit x from its splits' sums, scaled to the largest maximum and added in the
// splits' order. W warps share the work (warp `part` takes every W-th split, and part 0 adds the
// others' sums in order, from s_o and s_z, the warp's own shared memory, the warps' next to each
// other; with a barrier of the whole block, which all its warps reach); one warp needs none. A lane
// has channels 4 lane .. + 3 of all the rows.
template <typename T, int W, int NR>
__device__ __forceinline__ void at_join(const Dims& dm, const AttendArgs& a, const AtUnit& x, int r0, int part,
                                        float4* s_o, float* s_z) {
  const int R = dm.G * dm.window, lane = threadIdx.x & 31, rl = lane % NR;
  const float scale2 = a.scale2;
  const bool on = r0 < R && x.nsp > 1;
  float m = -INFINITY, z = 0.f;  // of row r0 + rl
  float4 s[NR];
#pragma unroll
  for (int i = 0; i < NR; ++i) s[i] = make_float4(0.f, 0.f, 0.f, 0.f);
  if (on) {
    const int r = r0 + rl < R ? r0 + rl : R - 1;
    const float2* ml = at_ml(a, x, 0, r);
    const float4* o = at_part(a, x, 0, r0) + lane * a.prows;
    const int64_t step = at_part(a, x, 1, r0) - at_part(a, x, 0, r0);
    for (int j = lane / NR; j < x.nsp; j += 32 / NR) m = fmaxf(m, ml[at_slot<T>(a, x, j) * a.srows].x);
#pragma unroll
    for (int off = NR; off < 32; off <<= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, off));
#pragma unroll (NR == 8 ? 2 : 4)
    for (int j = part; j < x.nsp; j += W) {
      const int64_t slot = at_slot<T>(a, x, j);
      const float2 w = ml[slot * a.srows];
      float4 v[NR];
#pragma unroll
      for (int i = 0; i < NR; ++i) v[i] = o[slot * step + i];  // (rows behind the last lie in the block too)
      // (a split that saw nothing has the maximum -inf and the sum 0, one of NaN only -inf and NaN)
      const float f = w.x == m ? 1.f : ex2((w.x - m) * scale2);
      const bool none = w.x == -INFINITY && w.y == 0.f;
      z += none ? 0.f : w.y * f;
#pragma unroll
      for (int i = 0; i < NR; ++i) {
        const float fi = __shfl_sync(0xffffffffu, none ? 0.f : f, i);
        const bool skip = __shfl_sync(0xffffffffu, none ? 1 : 0, i);
        s[i].x += skip ? 0.f : v[i].x * fi;
        s[i].y += skip ? 0.f : v[i].y * fi;
        s[i].z += skip ? 0.f : v[i].z * fi;
        s[i].w += skip ? 0.f : v[i].w * fi;
      }
    }
  }
  if constexpr (W > 1) {
#pragma unroll
    for (int i = 0; i < NR; ++i) s_o[i * 32 + lane] = s[i];
    if (lane < NR) s_z[lane] = z;
    __syncthreads();
    if (part != 0) return;
    for (int k = 1; k < W; ++k) {
#pragma unroll
      for (int i = 0; i < NR; ++i) {
        const float4 v = s_o[(k * NR + i) * 32 + lane];
        s[i].x += v.x, s[i].y += v.y, s[i].z += v.z, s[i].w += v.w;
      }
      z += s_z[k * NR + rl];
    }
  }
  if (!on) return;
  AtUnit whole = x;
  whole.nsp = 1;  // straight to the output
#pragma unroll
  for (int i = 0; i < NR; ++i) {
    const float mi = __shfl_sync(0xffffffffu, m, i), zi = __shfl_sync(0xffffffffu, z, i);
    if (r0 + i < R) at_put<T>(dm, a, whole, r0 + i, s[i], mi, zi, lane);
  }
}

// acc, the sums of channels c .. c + 3 of drafted token t's row, with the drafted values that are
// not finite (of the tokens `bad`, zeroed in the product) added where the row sees them.
__device__ __forceinline__ void at_bad(const Dims& dm, const AttendArgs& a, const AtUnit& x, uint64_t bad, int t, int c,
                                       float* acc) {
  uint64_t seen = bad & at_mask(dm, a, x, t);
  const __nv_bfloat16* vd = (const __nv_bfloat16*)a.vd + x.s * a.vds[0] + x.l * a.vds[1] + x.g * a.vds[2] + c;
  for (; seen != 0; seen &= seen - 1) {
    const uint2 w = *(const uint2*)(vd + (__ffsll((long long)seen) - 1) * a.vds[3]);
    const float e[4] = {bf16lo(w.x), bf16hi(w.x), bf16lo(w.y), bf16hi(w.y)};
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (!isfinite(e[i])) acc[i] += e[i];
  }
}

// How the work is shared out (bf16): all tiles of all units lie on a line, plane by plane, row block by row block and
// request by request, each with its cost (START more tiles for a unit's start), and CTA k takes positions
// [k per, (k + 1) per). A border that is fewer than `edge` tiles from a unit's start or end moves there, so that short
// units stay whole and no split is a sliver. A unit whose first tile is at p0 then has its
// first split in CTA floor((p0 + (edge - 1) cost) / per), and a further one in each CTA up to the one of position
// p0 + (tiles - edge) cost. (Items dealt one by one as CTAs became free, of a size chosen by an account of their
// number: 37 and 216 us where this takes 36 and 173, with one token in 16 slots and 16 trees; one
// token over 16 requests of 46 to 16383 97 and 82.)
// Cost: cost(row block) of a tile, and UNIT, the least tile's.
struct AtDivisor {  // x / d by a multiplication with floor((2^32 - 1) / d): at most 2 below, which is made up for
  uint32_t d, inv;
  __device__ __forceinline__ uint32_t of(uint32_t x) const {
    uint32_t q = __umulhi(x, inv);
    for (uint32_t r = x - q * d; r >= d; r -= d) ++q;
    return q;
  }
};
template <int TOK, uint32_t START, typename Cost>
struct AtShares {
  const Dims& dm;
  const AttendArgs& a;
  const int32_t* cu;
  const Cost cost;
  uint32_t per, w0, w1, pos;  // pos: where the unit (plane (l, g), row block rb, request s) starts
  AtDivisor by;               // per
  int l, g, rb, s;

  // Virtual tiles of request s0 + lane (as at_unit counts them, at least one, and its start), and of requests s0 ..
  // s0 + lane. (Inlined at both places: as a function 16 slots took 37.5 us instead of 36.8, in bytes 24.5, not 24.2.)
  static __device__ __forceinline__ uint2 count(const Dims& dm, const AttendArgs& a, const int32_t* cu, int s0, int lane) {
    uint32_t own = 0;
    if (s0 + lane < dm.S) {
      const AtLive x = at_live(dm, a, cu, s0 + lane);
      own = max(1, (x.n > 0 ? (x.n - 1) / TOK + 1 : 0) + (a.kd != nullptr && x.rows > 0 ? 1 : 0)) + START;
    }
    uint32_t sum = own;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const uint32_t x = __shfl_up_sync(0xffffffffu, sum, o);
      if (lane >= o) sum += x;
    }
    return make_uint2(own, sum);
  }

  // The CTA's share, and the unit at its start. A whole warp.
  __device__ __forceinline__ AtShares(const Dims& dm_, const AttendArgs& a_, const int32_t* cu_, Cost cost_, int lane)
      : dm(dm_), a(a_), cu(cu_), cost(cost_) {
    const uint32_t planes = (uint32_t)dm.L * dm.Hkv;
    uint32_t csum = 0;   // cost of a tile of a plane
    uint64_t tiles = 0;  // virtual tiles of a plane
    uint2 own;           // count()
    for (int s0 = 0; s0 < dm.S; s0 += 32) {
      own = count(dm, a, cu, s0, lane);
      tiles += __shfl_sync(0xffffffffu, own.y, 31);
    }
    for (int b = 0; b < a.nrb; ++b) csum += cost(b);
    // below 2^31 (checked by the host), unless ranges of cu_seqlens overlap: nothing is done then
    const bool fits = tiles * planes * csum <= (uint64_t)INT32_MAX;
    if (!fits && lane == 0) atomicOr(a.status, (uint32_t)ST_INVALID);
    const uint32_t tp = fits ? (uint32_t)tiles : 1u, total = fits ? planes * tp * csum : 0u;
    per = max((total + gridDim.x - 1) / gridDim.x, (uint32_t)a.least * Cost::UNIT);
    by = {per, 0xffffffffu / per};
    w0 = blockIdx.x * per, w1 = min(w0 + per, total);
    l = g = rb = s = 0, pos = total;
    if (w0 >= total) return;
    const uint32_t plane = w0 / (tp * csum);
    pos = plane * tp * csum;
    l = (int)(plane / (uint32_t)dm.Hkv), g = (int)(plane - l * dm.Hkv);
    for (; w0 - pos >= tp * cost(rb); ++rb) pos += tp * cost(rb);
    const uint32_t c = cost(rb), v = (w0 - pos) / c;
    uint32_t before = 0;
    for (int s0 = 0; s0 < dm.S; s0 += 32) {
      if (dm.S > 32) own = count(dm, a, cu, s0, lane);
      const uint32_t past = __ballot_sync(0xffffffffu, before + own.y > v);
      if (past != 0) {
        const int at = __ffs((int)past) - 1;
        s = s0 + at;
        before += __shfl_sync(0xffffffffu, own.y - own.x, at);
        break;
      }
      before += __shfl_sync(0xffffffffu, own.y, 31);
    }
    pos += before * c;
  }

  // This CTA's next item (nt = -1: none), with the first row `rows` times the row block. One thread.
  __device__ __forceinline__ void next(AtUnit& next, int rows) {
    for (;;) {
      if (pos >= w1) {
        next.nt = -1;
        return;
      }
      next = at_unit(dm, a, cu, l, g, s, 0, TOK, INT32_MAX);
      next.r0 = rb * rows;
      const uint32_t nt = max(next.nt, 1), c = cost(rb), p0 = pos + START * c, edge = a.edge;
      const uint32_t first = by.of(p0 + (min(edge, nt) - 1) * c);
      const uint32_t last = nt >= edge ? by.of(p0 + (nt - edge) * c) : 0;
      const int at = rb + a.nrb * (int)next.u, split = (int)blockIdx.x - (int)first;
      pos = p0 + nt * c;
      if (++s == dm.S) {
        s = 0;
        if (++rb == a.nrb) {
          rb = 0;
          if (++g == dm.Hkv) g = 0, ++l;
        }
      }
      next.nsp = last > first ? (int)(last - first) + 1 : 1;
      if (split < 0 || split >= next.nsp) continue;
      next.split = split;
      next.first = (int)first;
      if (split == 0 && a.nsps != nullptr) a.nsps[at] = next.nsp << 16 | (int)first;
      if (next.nt > 0) {
        const int ta = split == 0 ? 0 : (int)((w0 - p0 + c - 1) / c);
        const int tb = split == next.nsp - 1 ? (int)nt : (int)((w0 + per - p0 + c - 1) / c);
        const int cached = next.ncache;
        next.tok0 = ta * TOK;
        next.tok1 = min(next.n, tb * TOK);
        next.ncache = max(0, min(tb, cached) - ta);
        next.nt = tb - ta;
      }
      return;
    }
  }
};

}  // namespace jacap
