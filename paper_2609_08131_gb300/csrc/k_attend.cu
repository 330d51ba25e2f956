// k_attend.cu - attention of a few queries per request over its cached tokens and,
// where a draft model proposed them, over the drafted tokens themselves: one token (an
// ordinary decode step), a chain, or a tree whose tokens see their ancestors. For the
// rows r = (head h of the group, drafted token t) of a unit (request, layer, KV head)
//   l_i = scale q_r . k_i,   o_r = sum_i exp(l_i - M) v_i / Z,   Z = sum_i exp(l_i - M),
//   lse_r = M + ln Z,
// over the cached tokens i and the drafted tokens j with bit j of token t's mask set. A
// row that sees nothing has o = 0 and lse = -inf.
//
// K and V are read once, in one pass with a running maximum and sum. A unit's tokens are
// split into items (the drafted ones with the last), which leave unnormalised sums to be
// joined where a request has several splits.
//
// bf16: persistent CTAs with even shares of the tiles, which each works out from the live
// lengths, so that the host need not know them and a CTA's ring of tiles never runs dry
// between two items (one CTA per item: 158 us instead of 92 for the long chain below). A CTA's
// roles: a TMA producer, an MMA issuer, softmax warps with a row per lane, and warps that
// fetch the next item's rows. R = G T rows are an M = 128 operand whatever R is: the
// memory's time for a tile (64 tokens, 32 KB of K and V: ~700 SM cycles at the copy rate
// with two CTAs per SM) covers its products even where only a few rows are real, and the
// softmax warps work on real rows only: with R <= 32 every tensor-memory lane quarter
// holds a copy of the rows and takes a quarter of each tile's tokens (R <= 64: two
// copies, halves), each with a maximum and a sum of its own; the other tokens' weights are
// zero in its lanes, and the copies are joined at the item's end. So a warp has 16 columns
// per tile instead of 64, and no two warps ever wait for each other. Up to 256 rows share a
// CTA's tiles as two blocks of 128 (one CTA per SM); beyond that K and V are read again.
// The weights p are rounded to bf16 for the second product (the sums Z are not): of an
// output of many comparable terms that is an error of about the output's own rounding.
// The maximum is only raised when a logit passes it by 2^8, which a rescaling of the
// accumulators then follows: rare after the first tiles, and harmless to the sums (p <= 256).
// The tensor cores truncate each of a logit's partial sums, which shrinks logits by some
// 2^-23; the scale makes up for the mean of it.
// Rows of V past the live tokens, and drafted rows past the request's, are zeroed in
// shared memory before the product, as 0 times what an unwritten row holds may be NaN;
// a drafted value that is not finite is zeroed too and added to the rows that see it.
//
// Measured (32 query heads on 8, 92 us = 5.8 TB/s of K and V for 8 drafted tokens over 131011
// cached ones; 37 us = 3.7 TB/s for one token in 16 slots of 2100, of which ~8 us are the
// launch and the first tiles' way; 9 us for one token over 37): bound by memory up to 128 rows.
// 64 drafted tokens of 5 heads a group, 320 rows, over 110000 tokens in 16 requests: 173 us, 157 of them this
// kernel, for 138 GFLOP and 842 MB (K and V twice, 5.4 TB/s). A tile of 256 rows takes ~1500 cycles: the products ~1280
// (S reads its rows from shared memory again for every 64 tokens, 48 cycles for each 128 x 64 x 16), and the softmax
// ~1150 with two warps per scheduler, which overlap but for the waits between them. Tried and
// left out, of 216 us at the time: an MMA issuer per block (218), the barriers asked ahead of the
// issue (226).
//
// float32: CUDA cores, as the tensor cores would round the inputs. Up to 16 rows a warp takes
// 8 of a tile's tokens for all rows of the CTA (4, 8 or 16), four lanes to a token's dot
// products, and keeps a maximum, sums and accumulators of its own, so that tiles need no
// barrier but the one that says they have landed; the warps are joined at the end. More rows
// are a product of tiles (attend_f32_rows_kernel). Measured, 8 KV heads: 5 rows over 5473 tokens
// in two requests 32 us (45 MB: 7 us at the copy rate; the splits' start and end and the join are
// the rest), one row over 32768 tokens 57 us (268 MB: 40 us; with eight rows to a block 76 us); 4 requests of
// 4096 tokens with 12 rows 84 us, 25 rows 157 us; 2 requests with 64 rows 94 us, 256 rows 275 us (8.6 GFLOP: 115 us
// at 75 TFLOP/s; 574 us with 32 rows to a block, which read shared memory four times for as many multiply-adds).
#include "jacap_dev.cuh"
#include "jacap_internal.h"

namespace jacap {

constexpr int AT_TOK = 64;             // tokens per tile
constexpr int AT_BOX = AT_TOK * 128;   // {64 channels, 64 tokens} bf16
constexpr int AT_TILE = 2 * AT_BOX;
// A CTA of NB blocks of 128 rows (that share its tiles): warps 0 TMA producer, 1 MMA, then 4 NB
// softmax and 2 NB row warps. Two CTAs of one block share an SM, a CTA of two blocks has one.
constexpr int AT_QUEUE = 3;            // items published and not yet taken by all
template <int NB>
struct AtCfg {
  static constexpr int RING = 5 * NB;  // tiles of K and of V in flight, in the order K0 V0 K1 V1 ...
  static constexpr int Q_BYTES = NB * 128 * D * 2;
  static constexpr int LOADERS = 2 * NB, LOAD0 = 2 + 4 * NB, THREADS = 32 * (LOAD0 + LOADERS);
  static constexpr uint32_t COLS = 256 * NB;  // tensor memory: per block S (and P over it) 2 x 64, O 128
};
constexpr float AT_LAZY = 8.f;         // log2 of how far a logit may pass the maximum

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
// A request's live cached tokens and queries, clamped to what there can be (`ok`: nothing had to be).
struct AtLive {
  int64_t start;
  int n, rows;
  bool ok;
};
__device__ __forceinline__ AtLive at_live(const Dims& dm, const AttendArgs& a, const int32_t* cu, int s) {
  AtLive x;
  const int64_t start = cu[s], end = cu[s + 1];
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
__device__ __forceinline__ AtUnit at_unit(const Dims& dm, const AttendArgs& a, const int32_t* cu, uint32_t u, int split,
                                          int tile, int chunk) {  // (32-bit divisions: a 64-bit one takes ~300 cycles)
  AtUnit x;
  x.u = u;
  x.split = split;
  x.first = x.r0 = 0;
  const uint32_t plane = u / (uint32_t)dm.S;
  x.s = (int)(u - plane * dm.S);
  x.l = (int)(plane / (uint32_t)dm.Hkv);
  x.g = (int)(plane - x.l * dm.Hkv);
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

// Two CTAs share an SM's 228 KB (1 KB of each is the system's). There are no static
// variables, so the dynamic ones start on the 1024 bytes that the swizzle needs; the rest up
// to AT_SMEM makes up for a start that does not.
template <int NB>
struct AtSmem {
  uint64_t full[AtCfg<NB>::RING], empty[AtCfg<NB>::RING], sfull[2], pready[2];
  uint64_t pvdone[2];  // by a tile's parity: a wait for tile i knows that tile i - 2's product is done (S of tile i
                       // follows it)
  uint64_t qfull[AT_QUEUE], qempty[AT_QUEUE];
  uint64_t rowsready, rowsfree, rowsasked, ofree;
  AtUnit queue[AT_QUEUE];
  uint32_t tmem, bad[2];
  int abort, last;
};
template <int NB>
constexpr size_t at_used() { return AtCfg<NB>::Q_BYTES + AtCfg<NB>::RING * AT_TILE + sizeof(AtSmem<NB>); }
template <int NB>
constexpr size_t at_smem() { return 233472 / (3 - NB) - 1024; }
static_assert(at_used<1>() <= at_smem<1>() && at_used<2>() <= at_smem<2>(), "shared memory");
static_assert(128 * D * 2 >= 128 * 64 * 4, "the rows' space holds half the channels of the accumulators (copies)");

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
// request by request, each with its cost (AT_START more tiles for a unit's start), and CTA k takes positions
// [k per, (k + 1) per). A border that is fewer than `edge` tiles from a unit's start or end moves there, so that short
// units stay whole and no split is a sliver. A unit whose first tile is at p0 then has its
// first split in CTA floor((p0 + (edge - 1) cost) / per), and a further one in each CTA up to the one of position
// p0 + (tiles - edge) cost. (Items dealt one by one as CTAs became free, of a size chosen by an account of their
// number: 37 and 216 us where this takes 36 and 173, with one token in 16 slots and 16 trees; one
// token over 16 requests of 46 to 16383 97 and 82.)
template <int NB>
__device__ __forceinline__ uint32_t at_cost(const Dims& dm, int rb) {  // of a tile; measured 0.86 and 0.63 us
  return NB == 1 ? 1u : (dm.G * dm.window - rb * 256 > 128 ? 4u : 3u);
}
template <int NB>
constexpr uint32_t AT_START = NB == 1 ? 3 : 4;

template <int REP, int NB>
__global__ void __launch_bounds__(AtCfg<NB>::THREADS, 3 - NB)
    attend_bf16_kernel(const __grid_constant__ CUtensorMap kmap, const __grid_constant__ CUtensorMap vmap,
                       const __grid_constant__ CUtensorMap kdmap, const __grid_constant__ CUtensorMap vdmap, Dims dm,
                       const __grid_constant__ AttendArgs a, const int32_t* __restrict__ cu) {
  using C = AtCfg<NB>;
  static_assert(NB == 1 || REP == 1, "copies are for few rows");
  constexpr int AT_RING = C::RING, AT_LOAD0 = C::LOAD0, AT_LOADERS = C::LOADERS;
  // columns [0, AT_O): S of block j at 128 j + 64 (tile % 2); O of block j at AT_O + 128 j
  constexpr uint32_t AT_O = 128 * NB;
  constexpr int ROWS = 128 / REP;      // rows per copy (and block)
  constexpr int NC = AT_TOK / REP;     // columns per softmax warp
  extern __shared__ __align__(1024) uint8_t smem_raw[];
  uint8_t* smem = (uint8_t*)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
  uint8_t* qs = smem;
  uint8_t* ring = qs + C::Q_BYTES;
  AtSmem<NB>& sh = *(AtSmem<NB>*)(ring + AT_RING * AT_TILE);

  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int R = dm.G * dm.window;
  if (smem + at_used<NB>() > smem_raw + at_smem<NB>()) {  // (the start was not on 1024 bytes)
    pdl_wait();
    if (tid == 0) atomicOr(a.status, (uint32_t)ST_INVALID);
    return;
  }
  if (tid == 0) {
    sh.abort = 0;
    sh.bad[0] = sh.bad[1] = 0;
    for (int i = 0; i < AT_RING; ++i) {
      mbar_init(smem_u32(&sh.full[i]), 1);
      mbar_init(smem_u32(&sh.empty[i]), 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(smem_u32(&sh.sfull[i]), 1);
      mbar_init(smem_u32(&sh.pready[i]), 4 * NB);
      mbar_init(smem_u32(&sh.pvdone[i]), 1);
    }
    for (int i = 0; i < AT_QUEUE; ++i) {
      mbar_init(smem_u32(&sh.qfull[i]), 1);
      mbar_init(smem_u32(&sh.qempty[i]), 1 + 4 * NB + AT_LOADERS);  // MMA, softmax and row warps
    }
    mbar_init(smem_u32(&sh.rowsready), AT_LOADERS);
    mbar_init(smem_u32(&sh.rowsasked), AT_LOADERS);
    mbar_init(smem_u32(&sh.rowsfree), REP == 1 ? 1 : 4);
    mbar_init(smem_u32(&sh.ofree), 4 * NB);
    fence_mbar_init();
  }
  if (warp == 1) {
    tmem_alloc(smem_u32(&sh.tmem), C::COLS);
    tmem_relinquish();
  }
  if (tid == 0) {
    prefetch_tmap(&kmap);
    prefetch_tmap(&vmap);
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  pdl_wait();  // nothing before it touches global memory
  const uint32_t tmem = sh.tmem;
  Ws ws;
  ws.status = a.status;
  volatile int* abort = &sh.abort;
  // item `k` of this CTA, as the producer published it; the caller's warp (or thread) takes it once
  auto take = [&](uint32_t k, AtUnit& x, bool whole) {
    const int q = k % AT_QUEUE;
    if (!mbar_wait(smem_u32(&sh.qfull[q]), (k / AT_QUEUE) & 1, ws, abort)) return false;
    x = sh.queue[q];
    if (whole) __syncwarp();
    if (!whole || lane == 0) mbar_arrive(smem_u32(&sh.qempty[q]));
    return x.nt >= 0;
  };

  if (warp == 0) {
    // ------------------------------------------------ TMA producer --------
    const auto tiles_of = [&](int s) {  // as at_unit counts them, at least one
      const AtLive x = at_live(dm, a, cu, s);
      return (uint32_t)max(1, (x.n > 0 ? (x.n - 1) / AT_TOK + 1 : 0) + (a.kd != nullptr && x.rows > 0 ? 1 : 0));
    };
    const uint32_t planes = (uint32_t)dm.L * dm.Hkv;
    uint32_t mine = 0, csum = 0;  // virtual tiles of request `lane`, cost of a tile of a plane
    uint64_t tiles = 0;           // virtual tiles of a plane
    for (int s0 = 0; s0 < dm.S; s0 += 32) {
      const uint32_t v = s0 + lane < dm.S ? tiles_of(s0 + lane) + AT_START<NB> : 0u;
      if (s0 == 0) mine = v;
      tiles += __reduce_add_sync(0xffffffffu, v);
    }
    for (int rb = 0; rb < a.nrb; ++rb) csum += at_cost<NB>(dm, rb);
    // below 2^31 (checked by the host), unless ranges of cu_seqlens overlap: nothing is done then
    const bool fits = tiles * planes * csum <= (uint64_t)INT32_MAX;
    if (!fits && lane == 0) atomicOr(a.status, (uint32_t)ST_INVALID);
    const uint32_t tp = fits ? (uint32_t)tiles : 1u, total = fits ? planes * tp * csum : 0u;
    const uint32_t per = max((total + gridDim.x - 1) / gridDim.x, (uint32_t)a.least * (NB == 1 ? 1u : 4u));
    const uint32_t w0 = blockIdx.x * per, w1 = min(w0 + per, total);
    // the unit at w0: plane, row block, request, and the position where it starts
    uint32_t plane = w0 / (tp * csum), pos = plane * tp * csum;
    int rb = 0, s = 0;
    if (w0 < total) {
      for (; w0 - pos >= tp * at_cost<NB>(dm, rb); ++rb) pos += tp * at_cost<NB>(dm, rb);
      const uint32_t c = at_cost<NB>(dm, rb), v = (w0 - pos) / c;
      uint32_t before = 0;
      for (int s0 = 0; s0 < dm.S; s0 += 32) {
        const uint32_t own = s0 == 0 ? mine : (s0 + lane < dm.S ? tiles_of(s0 + lane) + AT_START<NB> : 0u);
        uint32_t sum = own;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
          const uint32_t x = __shfl_up_sync(0xffffffffu, sum, o);
          if (lane >= o) sum += x;
        }
        const uint32_t past = __ballot_sync(0xffffffffu, before + sum > v);
        if (past != 0) {
          const int at = __ffs((int)past) - 1;
          s = s0 + at;
          before += __shfl_sync(0xffffffffu, sum - own, at);
          break;
        }
        before += __shfl_sync(0xffffffffu, sum, 31);
      }
      pos += before * c;
    }
    if (lane == 0) {
      uint32_t n = 0, published = 0;  // loads, items
      bool ok = true;
      AtUnit next;
      // This CTA's next item, into `next` and the queue.
      auto publish = [&]() {
        for (;;) {
          if (pos >= w1) {
            next.nt = -1;
            break;
          }
          next = at_unit(dm, a, cu, plane * dm.S + s, 0, AT_TOK, INT32_MAX);
          next.r0 = rb * (128 * NB);
          const uint32_t nt = max(next.nt, 1), c = at_cost<NB>(dm, rb), p0 = pos + AT_START<NB> * c, edge = a.edge;
          const uint32_t first = (p0 + (min(edge, nt) - 1) * c) / per;
          const uint32_t last = nt >= edge ? (p0 + (nt - edge) * c) / per : 0;
          const int at = rb + a.nrb * (int)next.u, split = (int)blockIdx.x - (int)first;
          pos = p0 + nt * c;
          if (++s == dm.S) {
            s = 0;
            if (++rb == a.nrb) rb = 0, ++plane;
          }
          next.nsp = last > first ? (int)(last - first) + 1 : 1;
          if (split < 0 || split >= next.nsp) continue;
          next.split = split;
          next.first = (int)first;
          if (split == 0) a.nsps[at] = next.nsp << 16 | (int)first;
          if (next.nt > 0) {
            const int ta = split == 0 ? 0 : (int)((w0 - p0 + c - 1) / c);
            const int tb = split == next.nsp - 1 ? (int)nt : (int)((w0 + per - p0 + c - 1) / c);
            const int cached = next.ncache;
            next.tok0 = ta * AT_TOK;
            next.tok1 = min(next.n, tb * AT_TOK);
            next.ncache = max(0, min(tb, cached) - ta);
            next.nt = tb - ta;
          }
          break;
        }
        const int q = published % AT_QUEUE;
        if (published >= AT_QUEUE && !mbar_wait(smem_u32(&sh.qempty[q]), ((published / AT_QUEUE) & 1) ^ 1, ws, abort))
          return false;
        sh.queue[q] = next;
        mbar_arrive(smem_u32(&sh.qfull[q]));
        ++published;
        return true;
      };
      ok = publish();
      // the first rows are asked for before the tiles, which would be ahead of them in memory's queues
      if (ok && next.nt > 0) ok = mbar_wait(smem_u32(&sh.rowsasked), 0, ws, abort);
      while (ok && next.nt >= 0) {
        const AtUnit x = next;
        // the item after it, a few loads later: its rows are on their way long before they are needed
        const int when = 2 * x.nt < 4 ? 2 * x.nt : 4;
        for (int i = 0; ok && i < 2 * x.nt; ++i, ++n) {  // K and V of each tile
          if (i == when && !(ok = publish())) break;
          const int st = n % AT_RING;
          if (n >= AT_RING && !mbar_wait(smem_u32(&sh.empty[st]), ((n / AT_RING) & 1) ^ 1, ws, abort)) {
            ok = false;
            break;
          }
          const uint32_t dst = smem_u32(ring + st * AT_TILE), bar = smem_u32(&sh.full[st]);
          mbar_arrive_expect_tx(bar, AT_TILE);
          if ((i >> 1) < x.ncache) {
            const CUtensorMap* map = i & 1 ? &vmap : &kmap;
            const int t = (int)x.t0 + x.tok0 + (i >> 1) * AT_TOK;
            tma_load_4d(dst, map, 0, t, x.g, x.l, bar);
            tma_load_4d(dst + AT_BOX, map, 64, t, x.g, x.l, bar);
          } else {
            const CUtensorMap* map = i & 1 ? &vdmap : &kdmap;
            tma_load_5d(dst, map, 0, 0, x.g, x.l, x.s, bar);
            tma_load_5d(dst + AT_BOX, map, 64, 0, x.g, x.l, x.s, bar);
          }
        }
        if (ok && when == 2 * x.nt) ok = publish();
      }
      // what is under way lands before the CTA leaves
      for (uint32_t k = n > AT_RING ? n - AT_RING : 0; k < n; ++k)
        mbar_wait(smem_u32(&sh.full[k % AT_RING]), (k / AT_RING) & 1, ws, nullptr);
    }
  } else if (warp == 1) {
    // ------------------------------------------------ MMA issuer ----------
    if (elect_one()) {
      constexpr uint32_t IDESC_S = idesc_bf16_f32(128, AT_TOK, 0, 0), IDESC_O = idesc_bf16_f32(128, D, 0, 1);
      const uint64_t qd = smem_desc_sw128(smem_u32(qs), 16, 1024);
      uint32_t it = 0, n = 0, busy = 0;  // tiles whose S was issued, loads, items with tiles
      uint32_t issued = 0;               // second products
      bool ok = true;
      int nb = NB;                       // blocks that hold rows
      AtUnit x;
      auto second = [&](uint32_t t, uint32_t load, bool first) {  // O (+)= P V of tile t
        const uint32_t b = t & 1, st = load % AT_RING;
        // the first of an item: the accumulators of the item before are read out
        if (first && busy > 1 && !mbar_wait(smem_u32(&sh.ofree), busy & 1, ws, abort)) return false;
        if (!mbar_wait(smem_u32(&sh.pready[b]), (t >> 1) & 1, ws, abort) ||
            !mbar_wait(smem_u32(&sh.full[st]), (load / AT_RING) & 1, ws, abort))
          return false;
        tc_fence_after();
        const uint64_t vd = smem_desc_sw128(smem_u32(ring + st * AT_TILE), AT_BOX, 1024);
#pragma unroll
        for (int j = 0; j < NB; ++j) {
          if (j >= nb) break;
#pragma unroll
          for (int k = 0; k < AT_TOK / 16; ++k)
            umma_f16_ts(tmem + AT_O + 128 * j, tmem + 128 * j + 64 * b + 8 * k, vd + (uint64_t)((k * 2048) >> 4),
                        IDESC_O, !first || k > 0 ? 1u : 0u);
        }
        umma_commit(smem_u32(&sh.empty[st]));
        umma_commit(smem_u32(&sh.pvdone[b]));
        ++issued;
        return true;
      };
      for (uint32_t k = 0; ok && take(k, x, false); ++k) {
        if (x.nt == 0) continue;
        nb = (min(R - x.r0, NB * 128) + 127) / 128;
        // the rows are there, which the row warps put down when the item before no longer needed the space
        if (!mbar_wait(smem_u32(&sh.rowsready), busy & 1, ws, abort)) break;
        ++busy;
        for (int i = 0; ok && i < x.nt; ++i, ++it, n += 2) {
          const uint32_t b = it & 1, st = n % AT_RING;
          if (!mbar_wait(smem_u32(&sh.full[st]), (n / AT_RING) & 1, ws, abort)) {
            ok = false;
            break;
          }
          tc_fence_after();
          // S of tile it goes where P of tile it - 2 was: its product, issued before, has read it
          const uint64_t kd = smem_desc_sw128(smem_u32(ring + st * AT_TILE), 16, 1024);
#pragma unroll
          for (int j = 0; j < NB; ++j) {
            if (j >= nb) break;
#pragma unroll
            for (int c = 0; c < D / 16; ++c)
              umma_f16_ss(tmem + 128 * j + 64 * b,
                          qd + (uint64_t)((j * 32768 + ((c >> 2) * 16384) + (c & 3) * 32) >> 4),
                          kd + (uint64_t)((((c >> 2) * AT_BOX) + (c & 3) * 32) >> 4), IDESC_S, c > 0 ? 1u : 0u);
          }
          umma_commit(smem_u32(&sh.empty[st]));
          umma_commit(smem_u32(&sh.sfull[b]));
          if (REP == 1 && i == x.nt - 1) umma_commit(smem_u32(&sh.rowsfree));  // the item's last use of its rows
          if (i > 0) ok = second(it - 1, n - 1, i == 1);
        }
        if (ok) ok = second(it - 1, n - 1, x.nt == 1);
      }
      // every MMA issued here completes before the CTA tears down tensor memory
      if (it > 0) mbar_wait(smem_u32(&sh.sfull[(it - 1) & 1]), ((it - 1) >> 1) & 1, ws, nullptr);
      if (issued > 0) mbar_wait(smem_u32(&sh.pvdone[(issued - 1) & 1]), ((issued - 1) >> 1) & 1, ws, nullptr);
    }
  } else if (warp >= AT_LOAD0) {
    // ------------------ the rows, K-major with the 128-byte swizzle; a copy per group of lane quarters
    const int e0 = (warp - AT_LOAD0) * 32 + lane;
    uint32_t busy = 0;
    AtUnit x;
    for (uint32_t k = 0; take(k, x, true); ++k) {
      if (x.nt == 0) continue;
      const int nrow = min(R - x.r0, NB * ROWS);
      const __nv_bfloat16* q =
          (const __nv_bfloat16*)a.q + x.s * dm.q_ss + x.l * dm.q_sl + (int64_t)x.g * dm.G * dm.q_sh;
      auto row = [&](int r) {
        const int h = row_head(dm.window, a.tdiv, x.r0 + r), t = x.r0 + r - h * dm.window;
        return q + h * dm.q_sh + t * dm.q_sp;
      };
      // into L2 while the item before is at work: two 128-byte lines per row
      for (int e = e0; busy > 0 && e < 2 * nrow; e += 32 * AT_LOADERS)
        asm volatile("prefetch.global.L2 [%0];" ::"l"(row(e >> 1) + (e & 1) * 64));
      // the item before's last tile has met its rows (with copies of them: and the space carried its sums out)
      if (busy > 0 && !mbar_wait(smem_u32(&sh.rowsfree), (busy - 1) & 1, ws, abort)) break;
      const int c = e0 & 15;
#pragma unroll 8
      for (int k2 = 0; k2 < 32; ++k2) {
        const int y = (e0 >> 4) + k2 * 2 * AT_LOADERS, r = y % (NB * ROWS);
        const bool on = r < nrow;
        cp_async16(smem_u32(qs + (y >> 7) * 32768 + (c >> 3) * 16384 + sw128_off(y & 127, c & 7)),
                   (const uint4*)row(on ? r : 0) + c, on);
      }
      cp_async_commit();
      if (busy == 0) {
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&sh.rowsasked));
      }
      cp_async_wait<0>();
      fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) mbar_arrive(smem_u32(&sh.rowsready));
      ++busy;
    }
  } else {
    // ------------------------------------------------ softmax -------------
    const int blk = (warp - 2) >> 2, quarter = warp & 3, y = quarter * 32 + lane, tsm = tid - 64;
    constexpr int SM_THREADS = 128 * NB;
    const uint32_t scol = tmem + 128 * blk, ocol = tmem + AT_O + 128 * blk;
    uint8_t* stage = qs + 32768 * blk;
    const int rep = y / ROWS;  // the copy (uniform in a warp)
    const uint32_t lanes = (uint32_t)(quarter * 32) << 16;
    const float scale2 = a.scale2, lazy = AT_LAZY / scale2;
    uint32_t it = 0, n = 1;  // tiles, loads (of V)
    bool ok = true;
    AtUnit x;
    for (uint32_t k = 0; ok; ++k) {
      const bool more = take(k, x, true);
      // (all warps decide together whether to go on: a wait may fail in one of them)
      if (named_barrier_any(1, SM_THREADS, !more && *abort != 0) || !more) break;
      const int b0 = x.r0 + 128 * blk, nrow = min(R - b0, ROWS);  // the block's first row, and rows
      if (x.nt == 0) {  // nothing to see
        for (int r = warp - 2 - 4 * blk; r < nrow; r += 4)
          at_put<__nv_bfloat16>(dm, a, x, b0 + r, make_float4(0.f, 0.f, 0.f, 0.f), -INFINITY, 0.f, lane);
        continue;
      }
      const int row = b0 + y % ROWS;
      const uint64_t mask = row < R && x.nt > x.ncache ? at_mask(dm, a, x, row % dm.window) : 0;
      float m = -INFINITY, z = 0.f;
      for (int i = 0; i < x.nt; ++i, ++it, n += 2) {
        const uint32_t b = it & 1;
        if (!mbar_wait(smem_u32(&sh.sfull[b]), (it >> 1) & 1, ws, abort)) {
          ok = false;
          break;
        }
        tc_fence_after();
        const bool drafted = i >= x.ncache;
        const int nv = drafted ? x.nd : x.tok1 - x.tok0 - i * AT_TOK;  // rows of the tile that hold tokens
        if (nrow > 0) {  // (of two blocks the second may have no rows)
        float v[NC];
        if constexpr (NC == 64) {
          tmem_ld32x2(scol + 64 * b + lanes, scol + 64 * b + 32 + lanes, (uint32_t*)v, (uint32_t*)(v + 32));
        } else if constexpr (NC == 32) {
          tmem_ld32(scol + 64 * b + 32 * rep + lanes, v);
        } else {
          tmem_ld16(scol + 64 * b + 16 * rep + lanes, v);
        }
        if (drafted) {
          const uint64_t mine = mask >> (NC * rep);
#pragma unroll
          for (int e = 0; e < NC; ++e) v[e] = mine >> e & 1 ? v[e] : -INFINITY;
        } else if (nv < AT_TOK) {
#pragma unroll
          for (int e = 0; e < NC; ++e) v[e] = NC * rep + e < nv ? v[e] : -INFINITY;
        }
        float mx[4] = {v[0], v[1], v[2], v[3]};
#pragma unroll
        for (int e = 4; e < NC; ++e) mx[e & 3] = fmaxf(mx[e & 3], v[e]);
        const float top = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3]));
        const bool up = top > m + lazy;
        if (__any_sync(0xffffffffu, up)) {
          const float f = up ? (m == -INFINITY ? 0.f : ex2((m - top) * scale2)) : 1.f;
          if (up) m = top;
          z *= f;
          if (i > 0) {
            if (!mbar_wait(smem_u32(&sh.pvdone[b ^ 1]), ((it - 1) >> 1) & 1, ws, abort)) {
              ok = false;
              break;
            }
            tc_fence_after();
#pragma unroll 1
            for (int c = 0; c < D; c += 32) {
              float w[32];
              tmem_ld32(ocol + c + lanes, w);
#pragma unroll
              for (int e = 0; e < 32; ++e) w[e] *= f;
              tmem_st_32x32b_x32(ocol + c + lanes, *(const uint32_t(*)[32])w);
            }
            tmem_wait_st();
          }
        }
        const float base = m == -INFINITY ? 0.f : m * scale2;
        const float2 by = make_float2(scale2, scale2), less = make_float2(-base, -base);
        float2 sum[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
#pragma unroll
        for (int e = 0; e < NC; e += 2) {
          const float2 w = fma2(make_float2(v[e], v[e + 1]), by, less);
          v[e] = ex2(w.x), v[e + 1] = ex2(w.y);
          sum[e >> 1 & 1] = add2(sum[e >> 1 & 1], make_float2(v[e], v[e + 1]));
        }
        sum[0] = add2(sum[0], sum[1]);
        z += sum[0].x + sum[0].y;
        uint32_t p[32];
#pragma unroll
        for (int c = 0; c < 32; ++c) {
          const int cc = c % (NC / 2);
          const uint32_t pk = pack_bf16x2(v[2 * cc], v[2 * cc + 1]);
          p[c] = REP == 1 || c / (NC / 2) == rep ? pk : 0u;
        }
        tmem_st_32x32b_x32(scol + 64 * b + lanes, p);
        }
        if (drafted || nv < AT_TOK) {
          if (!mbar_wait(smem_u32(&sh.full[n % AT_RING]), (n / AT_RING) & 1, ws, abort)) {
            ok = false;
            break;
          }
          uint8_t* vt = ring + n % AT_RING * AT_TILE;
          for (int e = tsm + (drafted ? 0 : nv * 16); e < AT_TOK * 16; e += SM_THREADS) {
            const int tok = e >> 4, c = e & 15;
            uint4* at = (uint4*)(vt + (c >> 3) * AT_BOX + sw128_off(tok, c & 7));
            if (tok >= nv) {
              *at = make_uint4(0, 0, 0, 0);
              continue;
            }
            uint4 w = *at;
            uint32_t* ww = (uint32_t*)&w;
            bool bad = false;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              if ((ww[j] & 0x7f80u) == 0x7f80u) bad = true, ww[j] &= 0xffff0000u;
              if ((ww[j] & 0x7f800000u) == 0x7f800000u) bad = true, ww[j] &= 0xffffu;
            }
            if (bad) {
              *at = w;
              atomicOr(&sh.bad[tok >> 5], 1u << (tok & 31));
            }
          }
          fence_proxy_async_smem();
        }
        tmem_wait_st();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&sh.pready[b]));
      }
      if (ok) ok = mbar_wait(smem_u32(&sh.pvdone[(it - 1) & 1]), ((it - 1) >> 1) & 1, ws, abort);
      // all warps meet here whether or not a wait failed, and leave together if one did
      if (named_barrier_any(1, SM_THREADS, !ok)) break;
      tc_fence_after();
      const uint64_t bad = (uint64_t)sh.bad[1] << 32 | sh.bad[0];
      if constexpr (REP == 1) {
        // a lane has a whole row: 32 channels at a time, partial sums with the rows of a block next to each other
        const int h = row_head(dm.window, a.tdiv, row), t = row - h * dm.window;
        const bool on = y < nrow && t < x.rows;
        const float f = x.nsp > 1 ? 1.f : (z == 0.f ? 0.f : 1.f / z);
        float4* part = nullptr;
        __nv_bfloat16* o = nullptr;
        if (on && x.nsp > 1) {
          const int64_t slot = at_slot<__nv_bfloat16>(a, x, x.split);
          part = at_part(a, x, slot, row);
          *at_ml(a, x, slot, row) = make_float2(m, z);
        } else if (on) {
          o = (__nv_bfloat16*)a.o + x.s * a.os[0] + x.l * a.os[1] + (int64_t)(x.g * dm.G + h) * a.os[2] + t * a.os[3];
          if (a.lse != nullptr)
            a.lse[x.s * a.ls[0] + x.l * a.ls[1] + (x.g * dm.G + h) * a.ls[2] + t] =
                z == 0.f ? -INFINITY : m * (a.scale2 * 0.6931471805599453f) + logf(z);
        }
        if (nrow > 0) {
#pragma unroll 1
          for (int c = 0; c < D; c += 32) {
            float w[32];
            tmem_ld32(ocol + c + lanes, w);
            if (part != nullptr) {
#pragma unroll
              for (int e = 0; e < 8; ++e)
                part[(c / 4 + e) * a.prows] = make_float4(w[4 * e], w[4 * e + 1], w[4 * e + 2], w[4 * e + 3]);
            } else if (o != nullptr) {
#pragma unroll
              for (int e = 0; e < 32; e += 8)
                *(uint4*)(o + c + e) =
                    make_uint4(pack_bf16x2(w[e] * f, w[e + 1] * f), pack_bf16x2(w[e + 2] * f, w[e + 3] * f),
                               pack_bf16x2(w[e + 4] * f, w[e + 5] * f), pack_bf16x2(w[e + 6] * f, w[e + 7] * f));
            }
          }
          if (bad != 0 && on) {  // added to what this lane has just written
#pragma unroll 1
            for (int c = 0; c < D; c += 4) {
              float acc[4] = {0.f, 0.f, 0.f, 0.f};
              at_bad(dm, a, x, bad, t, c, acc);
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                if (acc[e] == 0.f) continue;
                if (part != nullptr) ((float*)(part + c / 4 * a.prows))[e] += acc[e];
                else o[c + e] = __float2bfloat16(__bfloat162float(o[c + e]) + acc[e]);
              }
            }
          }
        }
      } else {
        // A row's copies scaled to their common maximum (and by 1 / Z where there is one split) meet in the space
        // of the query rows, which the item's last tile has met, half the channels at a time.
        constexpr int RL = ROWS / 32;  // rows per lane: lane + 32 j
        float mr[RL], zr[RL];
        float2* ex = (float2*)stage;  // [128] (maximum, sum)
        ex[y] = make_float2(m, z);
        named_barrier_sync(1, SM_THREADS);
        // (a copy whose logits are all NaN has the maximum -inf and a sum that is not 0)
        const auto share = [&](float2 mz, float t) {
          return mz.x == -INFINITY ? (mz.y == 0.f ? 0.f : 1.f) : ex2((mz.x - t) * scale2);
        };
        float4* part[RL];
        __nv_bfloat16* o[RL];
#pragma unroll
        for (int j = 0; j < RL; ++j) {
          mr[j] = -INFINITY, zr[j] = 0.f;
#pragma unroll
          for (int c = 0; c < REP; ++c) mr[j] = fmaxf(mr[j], ex[c * ROWS + 32 * j + lane].x);
#pragma unroll
          for (int c = 0; c < REP; ++c)
            zr[j] += ex[c * ROWS + 32 * j + lane].y * share(ex[c * ROWS + 32 * j + lane], mr[j]);
          const int rr = lane + 32 * j, h = row_head(dm.window, a.tdiv, rr), t = rr - h * dm.window;
          part[j] = nullptr, o[j] = nullptr;
          if (rr >= nrow || t >= x.rows) continue;
          if (x.nsp > 1) {
            const int64_t slot = at_slot<__nv_bfloat16>(a, x, x.split);
            part[j] = at_part(a, x, slot, rr);
            if (warp == 2) *at_ml(a, x, slot, rr) = make_float2(mr[j], zr[j]);
          } else {
            o[j] = (__nv_bfloat16*)a.o + x.s * a.os[0] + x.l * a.os[1] + (int64_t)(x.g * dm.G + h) * a.os[2] +
                   t * a.os[3];
            if (warp == 2 && a.lse != nullptr)
              a.lse[x.s * a.ls[0] + x.l * a.ls[1] + (x.g * dm.G + h) * a.ls[2] + t] =
                  zr[j] == 0.f ? -INFINITY : mr[j] * (a.scale2 * 0.6931471805599453f) + logf(zr[j]);
          }
        }
        float f = share(make_float2(m, z), mr[y % ROWS / 32]);
        if (x.nsp == 1) f *= zr[y % ROWS / 32] == 0.f ? 0.f : 1.f / zr[y % ROWS / 32];
        named_barrier_sync(1, SM_THREADS);
        float4* out = (float4*)stage;  // [128][16], 16-byte pieces swizzled by the row
#pragma unroll 1
        for (int half = 0; half < 2; ++half) {
#pragma unroll
          for (int c = 0; c < 64; c += 32) {
            float w[32];
            tmem_ld32(ocol + 64 * half + c + lanes, w);
#pragma unroll
            for (int e = 0; e < 8; ++e)
              out[y * 16 + ((c / 4 + e) ^ (y & 7))] =
                  make_float4(w[4 * e] * f, w[4 * e + 1] * f, w[4 * e + 2] * f, w[4 * e + 3] * f);
          }
          named_barrier_sync(1, SM_THREADS);
          // a lane per row, a warp per four of the 16 pieces
#pragma unroll
          for (int j = 0; j < RL; ++j) {
            const int r = lane + 32 * j;
#pragma unroll
            for (int k4 = 0; k4 < 4; ++k4) {
              const int c = 4 * (warp - 2) + k4;
              float acc[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
              for (int q = 0; q < REP; ++q) {
                const float4 w = out[(q * ROWS + r) * 16 + (c ^ (r & 7))];
                acc[0] += w.x, acc[1] += w.y, acc[2] += w.z, acc[3] += w.w;
              }
              if (bad != 0 && (part[j] != nullptr || o[j] != nullptr))
                at_bad(dm, a, x, bad, r - row_head(dm.window, a.tdiv, r) * dm.window, 64 * half + 4 * c, acc);
              if (part[j] != nullptr)
                part[j][(16 * half + c) * a.prows] = make_float4(acc[0], acc[1], acc[2], acc[3]);
              else if (o[j] != nullptr)
                *(uint2*)(o[j] + 64 * half + 4 * c) =
                    make_uint2(pack_bf16x2(acc[0], acc[1]), pack_bf16x2(acc[2], acc[3]));
            }
          }
          named_barrier_sync(1, SM_THREADS);
        }
      }
      if (bad != 0) {
        named_barrier_sync(1, SM_THREADS);  // (the same for all: the bits were set before the barriers above)
        if (tsm == 0) sh.bad[0] = sh.bad[1] = 0;
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) {
        mbar_arrive(smem_u32(&sh.ofree));
        if (REP > 1) mbar_arrive(smem_u32(&sh.rowsfree));
      }
      if (REP == 4 && x.nsp > 1 && at_joins_inside(x.nsp, R)) {
        __threadfence();
        named_barrier_sync(1, SM_THREADS);
        if (tsm == 0) {
          // (a CTA has the first split of one unit of several at most: the one that its end divides)
          sh.last = atomicAdd(a.counts + x.first, 1) == x.nsp - 1;
          if (sh.last) a.counts[x.first] = 0;  // (zero between calls)
          __threadfence();
        }
        named_barrier_sync(1, SM_THREADS);
        if (sh.last) at_join<__nv_bfloat16, 1, 8>(dm, a, x, 8 * (warp - 2), 0, nullptr, nullptr);
      }
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc(tmem, C::COLS);
  }
}

// ------------------------------------------------------------- float32 ----
// Up to 4 or 8 rows: K and V's arrival bounds it; four warps and tiles of 32 tokens, three CTAs per SM. More: the reads
// of shared memory that feed the multiply-adds; up to 16 rows two such CTAs (12 rows: 84 us, with 32 rows to a block
// 152).
template <int RB>
struct AfCfg {
  static constexpr int WARPS = 4, THREADS = 32 * WARPS, TOK = 8 * WARPS, LDK = D + 4;
  static constexpr int KF = TOK * LDK, VF = TOK * D;  // floats per stage
  static constexpr size_t SMEM = (size_t)(RB * D + 2 * (KF + VF) + WARPS * 8 * RB + 2 * WARPS * RB) * 4;
  static constexpr int PER_SM = RB <= 8 ? 3 : 2;
};

template <int RB>
__global__ void __launch_bounds__(AfCfg<RB>::THREADS, AfCfg<RB>::PER_SM)
    attend_f32_kernel(Dims dm, const __grid_constant__ AttendArgs a, const int32_t* __restrict__ cu) {
  using C = AfCfg<RB>;
  constexpr int AF_THREADS = C::THREADS, AF_WARPS = C::WARPS, AF_TOK = C::TOK, AF_LDK = C::LDK;
  constexpr int AF_KF = C::KF, AF_VF = C::VF;
  extern __shared__ __align__(16) float sf[];
  float* qs = sf;                          // [RB][D]
  float* ks = qs + RB * D;                 // [2][TOK][LDK]
  float* vs = ks + 2 * AF_KF;              // [2][TOK][D]
  float* ps = vs + 2 * AF_VF;              // [warp][8 tokens][RB]
  float* sm = ps + AF_WARPS * 8 * RB;      // [warp][RB] maxima, then sums
  float* sz = sm + AF_WARPS * RB;
  static_assert(2 * (AF_KF + AF_VF) >= AF_WARPS * RB * D, "the tiles' space holds the warps' accumulators at the end");
  pdl_wait();
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int rb = blockIdx.x % a.nrb, rest = blockIdx.x / a.nrb;
  const AtUnit x = at_unit(dm, a, cu, rest / a.nsplit, rest % a.nsplit, AF_TOK, a.chunk);
  if (x.split >= x.nsp) return;
  const int R = dm.G * dm.window, r0 = rb * RB, nrow = R - r0 < RB ? R - r0 : RB;
  if (x.nt == 0) {
    for (int r = warp; r < nrow; r += AF_WARPS)
      at_put<float>(dm, a, x, r0 + r, make_float4(0.f, 0.f, 0.f, 0.f), -INFINITY, 0.f, lane);
    return;
  }
  const int64_t plane = (int64_t)x.l * dm.kv_sl + (int64_t)x.g * dm.kv_sh;
  const int64_t kd0 = x.s * a.kds[0] + x.l * a.kds[1] + x.g * a.kds[2];
  const int64_t vd0 = x.s * a.vds[0] + x.l * a.vds[1] + x.g * a.vds[2];
  auto fetch = [&](int i) {
    float *kt = ks + (i & 1) * AF_KF, *vt = vs + (i & 1) * AF_VF;
    const bool drafted = i >= x.ncache;
    const int first = drafted ? (i - x.ncache) * AF_TOK : x.tok0 + i * AF_TOK;
    const int nv = (drafted ? x.nd : x.tok1) - first;
    const float* kb = drafted ? (const float*)a.kd + kd0 + first * a.kds[3]
                              : (const float*)a.k + plane + (x.t0 + first) * dm.kv_st;
    const float* vb = drafted ? (const float*)a.vd + vd0 + first * a.vds[3]
                              : (const float*)a.v + plane + (x.t0 + first) * dm.kv_st;
    const int64_t kst = drafted ? a.kds[3] : dm.kv_st, vst = drafted ? a.vds[3] : dm.kv_st;
#pragma unroll 4
    for (int e = tid; e < AF_TOK * 32; e += AF_THREADS) {
      const int tok = e >> 5, c = (e & 31) * 4;
      const bool on = tok < nv;
      cp_async16(smem_u32(kt + tok * AF_LDK + c), kb + (on ? tok * kst : 0) + c, on);
      cp_async16(smem_u32(vt + tok * D + c), vb + (on ? tok * vst : 0) + c, on);
    }
  };
  fetch(0);
  {
    const float* q = (const float*)a.q + x.s * dm.q_ss + x.l * dm.q_sl + (int64_t)x.g * dm.G * dm.q_sh;
    for (int e = tid; e < RB * 32; e += AF_THREADS) {
      const int r = e >> 5, c = (e & 31) * 4;
      const int h = (r0 + r) / dm.window, t = r0 + r - h * dm.window;
      const bool on = r < nrow;
      cp_async16(smem_u32(qs + r * D + c), q + (on ? h * dm.q_sh + t * dm.q_sp : 0) + c, on);
    }
  }
  cp_async_commit();
  const float scale2 = a.scale2, lazy = AT_LAZY / scale2;
  const int tok = lane >> 2, kq = lane & 3;
  // lane r: row r's maximum (all tokens of the warp) and sum; every lane: channels 4 lane .. + 3 of all rows
  float m = -INFINITY, z = 0.f;
  float4 acc[RB];
#pragma unroll
  for (int r = 0; r < RB; ++r) acc[r] = make_float4(0.f, 0.f, 0.f, 0.f);
  float* pw = ps + warp * 8 * RB;  // [8 tokens][RB]
  const int myrow = lane % RB;
  const int myt = r0 + myrow - row_head(dm.window, a.tdiv, r0 + myrow) * dm.window;
  const uint64_t mask = x.nt > x.ncache && r0 + myrow < R ? at_mask(dm, a, x, myt) : 0;
  for (int i = 0; i < x.nt; ++i) {
    if (i + 1 < x.nt) fetch(i + 1);
    cp_async_commit();
    cp_async_wait<1>();
    __syncthreads();
    const bool drafted = i >= x.ncache;
    const int first = drafted ? (i - x.ncache) * AF_TOK : x.tok0 + i * AF_TOK;
    const int left = (drafted ? x.nd : x.tok1) - first - 8 * warp;  // tokens of this warp's eight
    if (left > 0) {
      const float* kt = ks + (i & 1) * AF_KF + (8 * warp + tok) * AF_LDK + 4 * kq;
      float s[RB];
#pragma unroll
      for (int r = 0; r < RB; ++r) s[r] = 0.f;
#pragma unroll 2
      for (int k = 0; k < D; k += 16) {
        const float4 kk = *(const float4*)(kt + k);
#pragma unroll
        for (int r = 0; r < RB; ++r) {
          const float4 qq = *(const float4*)(qs + r * D + k + 4 * kq);
          s[r] = fmaf(qq.x, kk.x, fmaf(qq.y, kk.y, fmaf(qq.z, kk.z, fmaf(qq.w, kk.w, s[r]))));
        }
      }
      // the logits to shared memory, four rows by each lane of a token, so that lane r has row r's eight
      __syncwarp();  // the previous tile's weights are read
#pragma unroll
      for (int r = 0; r < RB; ++r) {
        s[r] += __shfl_xor_sync(0xffffffffu, s[r], 1);
        s[r] += __shfl_xor_sync(0xffffffffu, s[r], 2);
        if ((r & 3) == kq) pw[tok * RB + r] = s[r];
      }
      __syncwarp();
      float l[8], top = -INFINITY;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        l[j] = pw[j * RB + myrow];
        if (j >= left || (drafted && !(mask >> (first + 8 * warp + j & 63) & 1))) l[j] = -INFINITY;
        top = fmaxf(top, l[j]);
      }
      const bool up = top > m + lazy;
      const uint32_t who = __ballot_sync(0xffffffffu, up);
      if (who != 0) {
        const float f = up ? (m == -INFINITY ? 0.f : ex2((m - top) * scale2)) : 1.f;
        if (up) m = top;
        z *= f;
#pragma unroll
        for (int r = 0; r < RB; ++r) {
          if (!(who >> r & 1)) continue;
          const float fr = __shfl_sync(0xffffffffu, f, r);
          acc[r].x *= fr, acc[r].y *= fr, acc[r].z *= fr, acc[r].w *= fr;
        }
      }
      const float base = m == -INFINITY ? 0.f : m * scale2;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        l[j] = ex2(fmaf(l[j], scale2, -base));
        z += l[j];
        if (lane < RB) pw[j * RB + lane] = l[j];
      }
      __syncwarp();
      const float* vt = vs + (i & 1) * AF_VF + 8 * warp * D + 4 * lane;
      const int nt8 = left < 8 ? left : 8;
#pragma unroll 4
      for (int j = 0; j < nt8; ++j) {
        const float4 vv = *(const float4*)(vt + j * D);
#pragma unroll
        for (int r = 0; r < RB; r += 4) {
          const float4 p4 = *(const float4*)(pw + j * RB + r);
          const float p[4] = {p4.x, p4.y, p4.z, p4.w};
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            if (drafted && p[e] == 0.f) continue;  // a masked value may be anything
            acc[r + e].x = fmaf(p[e], vv.x, acc[r + e].x);
            acc[r + e].y = fmaf(p[e], vv.y, acc[r + e].y);
            acc[r + e].z = fmaf(p[e], vv.z, acc[r + e].z);
            acc[r + e].w = fmaf(p[e], vv.w, acc[r + e].w);
          }
        }
      }
    }
    __syncthreads();  // the tile's stage is free
  }
  cp_async_wait<0>();
  // the warps joined: accumulators through the tiles' space
  float4* out = (float4*)ks;  // [warp][RB][32]
  if (lane < RB) sm[warp * RB + lane] = m, sz[warp * RB + lane] = z;
#pragma unroll
  for (int r = 0; r < RB; ++r) out[(warp * RB + r) * 32 + lane] = acc[r];
  __syncthreads();
  for (int r = warp; r < nrow; r += AF_WARPS) {
    float mr = -INFINITY, zr = 0.f;
    float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int w = 0; w < AF_WARPS; ++w) mr = fmaxf(mr, sm[w * RB + r]);
    for (int w = 0; w < AF_WARPS; ++w) {
      const float mw = sm[w * RB + r];
      if (mw == -INFINITY && !(sz[w * RB + r] != 0.f)) continue;  // that warp saw nothing
      const float f = mw == mr ? 1.f : ex2((mw - mr) * scale2);
      const float4 v = out[(w * RB + r) * 32 + lane];
      zr = fmaf(sz[w * RB + r], f, zr);
      s.x = fmaf(v.x, f, s.x), s.y = fmaf(v.y, f, s.y), s.z = fmaf(v.z, f, s.z), s.w = fmaf(v.w, f, s.w);
    }
    at_put<float>(dm, a, x, r0 + r, s, mr, zr, lane);
  }
}

// More than 16 rows (25 rows: 157 us, 154 with 32 rows to a block of the kernel above): bound by the latency
// between reads of shared memory and the multiply-adds that they feed. A block of NT threads takes NT / 4
// rows (64 or 128): in both products a thread has the same four rows, of 4 tokens (tx, tx + 16, ...) and
// then of 8 channels (4 tx .. and 64 + 4 tx ..), so that a 16-byte read feeds 8 to 11 of them, a row's
// maximum and sum stay with its 16 lanes, and its weights go from one product to the other within a warp,
// 32 tokens at a time. (256 rows: 275 us; with eight rows to a thread and half the threads 337 us.)
template <int NT>
struct AgCfg {
  static constexpr int MR = 4, ROWS = NT / 16 * MR, THREADS = NT, TOK = 64, LDK = D + 4, LDP = ROWS + 4, HALF = TOK / 2;
  static constexpr int KF = TOK * LDK, VF = TOK * D;  // floats per stage
  static constexpr size_t SMEM = (size_t)(ROWS * D + 2 * (KF + VF) + HALF * LDP) * 4;
};

template <int NT>
__global__ void __launch_bounds__(NT, 1)
    attend_f32_rows_kernel(Dims dm, const __grid_constant__ AttendArgs a, const int32_t* __restrict__ cu) {
  using C = AgCfg<NT>;
  constexpr int MR = C::MR, TOK = C::TOK, LDK = C::LDK, LDP = C::LDP;
  extern __shared__ __align__(16) float sf[];
  float* qs = sf;                  // [ROWS][D]
  float* ks = qs + C::ROWS * D;    // [2][TOK][LDK]
  float* vs = ks + 2 * C::KF;      // [2][TOK][D]
  float* ps = vs + 2 * C::VF;      // [HALF tokens][LDP]
  pdl_wait();
  const int tid = threadIdx.x, tx = tid & 15, ty = tid >> 4;
  const int rb = blockIdx.x % a.nrb, rest = blockIdx.x / a.nrb;
  const AtUnit x = at_unit(dm, a, cu, rest / a.nsplit, rest % a.nsplit, TOK, a.chunk);
  if (x.split >= x.nsp) return;
  const int R = dm.G * dm.window, r0 = rb * C::ROWS, nrow = R - r0 < C::ROWS ? R - r0 : C::ROWS;
  const int64_t plane = (int64_t)x.l * dm.kv_sl + (int64_t)x.g * dm.kv_sh;
  const int64_t kd0 = x.s * a.kds[0] + x.l * a.kds[1] + x.g * a.kds[2];
  const int64_t vd0 = x.s * a.vds[0] + x.l * a.vds[1] + x.g * a.vds[2];
  auto fetch = [&](int i) {
    float *kt = ks + (i & 1) * C::KF, *vt = vs + (i & 1) * C::VF;
    const bool drafted = i >= x.ncache;
    const int first = drafted ? 0 : x.tok0 + i * TOK;  // (the drafted tokens are one tile)
    const int nv = (drafted ? x.nd : x.tok1) - first;
    const float* kb = drafted ? (const float*)a.kd + kd0 : (const float*)a.k + plane + (x.t0 + first) * dm.kv_st;
    const float* vb = drafted ? (const float*)a.vd + vd0 : (const float*)a.v + plane + (x.t0 + first) * dm.kv_st;
    const int64_t kst = drafted ? a.kds[3] : dm.kv_st, vst = drafted ? a.vds[3] : dm.kv_st;
#pragma unroll 4
    for (int e = tid; e < TOK * 32; e += C::THREADS) {
      const int tok = e >> 5, c = (e & 31) * 4;
      const bool on = tok < nv;
      cp_async16(smem_u32(kt + tok * LDK + c), kb + (on ? tok * kst : 0) + c, on);
      cp_async16(smem_u32(vt + tok * D + c), vb + (on ? tok * vst : 0) + c, on);
    }
  };
  if (x.nt > 0) fetch(0);
  {
    const float* q = (const float*)a.q + x.s * dm.q_ss + x.l * dm.q_sl + (int64_t)x.g * dm.G * dm.q_sh;
    for (int e = tid; e < C::ROWS * 32; e += C::THREADS) {
      const int r = e >> 5, c = (e & 31) * 4, h = row_head(dm.window, a.tdiv, r0 + r), t = r0 + r - h * dm.window;
      const bool on = r < nrow;
      cp_async16(smem_u32(qs + r * D + c), q + (on ? h * dm.q_sh + t * dm.q_sp : 0) + c, on);
    }
  }
  cp_async_commit();
  const float scale2 = a.scale2, lazy = AT_LAZY / scale2;
  float m[MR], z[MR];      // of row ty MR + i: the maximum, and the sum over this thread's tokens
  float4 o[MR][2];
#pragma unroll
  for (int i = 0; i < MR; ++i) {
    m[i] = -INFINITY, z[i] = 0.f;
    o[i][0] = o[i][1] = make_float4(0.f, 0.f, 0.f, 0.f);
  }
  for (int i = 0; i < x.nt; ++i) {
    if (i + 1 < x.nt) fetch(i + 1);
    cp_async_commit();
    cp_async_wait<1>();
    __syncthreads();
    const bool drafted = i >= x.ncache;
    const int left = drafted ? x.nd : x.tok1 - x.tok0 - i * TOK;  // tokens of the tile
    const float* kt = ks + (i & 1) * C::KF + tx * LDK;
    const float* qt = qs + ty * MR * D;
    float s[MR][4];
#pragma unroll
    for (int r = 0; r < MR; ++r) s[r][0] = s[r][1] = s[r][2] = s[r][3] = 0.f;
#pragma unroll(NT == 512 ? 2 : 1)
    for (int k = 0; k < D; k += 4) {
      float4 kk[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) kk[j] = *(const float4*)(kt + 16 * j * LDK + k);
#pragma unroll
      for (int r = 0; r < MR; ++r) {
        const float4 q = *(const float4*)(qt + r * D + k);
#pragma unroll
        for (int j = 0; j < 4; ++j)
          s[r][j] = fmaf(q.x, kk[j].x, fmaf(q.y, kk[j].y, fmaf(q.z, kk[j].z, fmaf(q.w, kk[j].w, s[r][j]))));
      }
    }
#pragma unroll
    for (int r = 0; r < MR; ++r) {
      if (drafted) {
        const int row = r0 + ty * MR + r, t = row - row_head(dm.window, a.tdiv, row) * dm.window;
        const uint64_t mask = row < R ? at_mask(dm, a, x, t) : 0;
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (!(mask >> (tx + 16 * j) & 1)) s[r][j] = -INFINITY;
      } else if (left < TOK) {
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (tx + 16 * j >= left) s[r][j] = -INFINITY;
      }
      float top = fmaxf(fmaxf(s[r][0], s[r][1]), fmaxf(s[r][2], s[r][3]));
#pragma unroll
      for (int off = 8; off >= 1; off >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, off));
      if (top > m[r] + lazy) {
        const float f = m[r] == -INFINITY ? 0.f : ex2((m[r] - top) * scale2);
        m[r] = top;
        z[r] *= f;
#pragma unroll
        for (int c = 0; c < 2; ++c) o[r][c].x *= f, o[r][c].y *= f, o[r][c].z *= f, o[r][c].w *= f;
      }
      const float base = m[r] == -INFINITY ? 0.f : m[r] * scale2;
#pragma unroll
      for (int j = 0; j < 4; ++j) s[r][j] = ex2(fmaf(s[r][j], scale2, -base));
      z[r] += (s[r][0] + s[r][1]) + (s[r][2] + s[r][3]);
    }
    // the weights of tokens tx + 16 j at [tx + 16 (j % 2)]: read by the lanes of the same rows alone
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      __syncwarp();  // the half before is read
#pragma unroll
      for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int r = 0; r < MR; r += 4)
          *(float4*)(ps + (tx + 16 * j) * LDP + ty * MR + r) =
              make_float4(s[r][2 * half + j], s[r + 1][2 * half + j], s[r + 2][2 * half + j], s[r + 3][2 * half + j]);
      __syncwarp();
      const float* vt = vs + (i & 1) * C::VF + half * C::HALF * D + 4 * tx;
      const int n = left - half * C::HALF < C::HALF ? left - half * C::HALF : C::HALF;
#pragma unroll 2
      for (int j = 0; j < n; ++j) {
        const float4 v0 = *(const float4*)(vt + j * D), v1 = *(const float4*)(vt + j * D + 64);
#pragma unroll
        for (int r = 0; r < MR; r += 4) {
          const float4 p4 = *(const float4*)(ps + j * LDP + ty * MR + r);
          const float p[4] = {p4.x, p4.y, p4.z, p4.w};
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            if (drafted && p[e] == 0.f) continue;  // a masked value may be anything
            float4 &u = o[r + e][0], &w = o[r + e][1];
            u.x = fmaf(p[e], v0.x, u.x), u.y = fmaf(p[e], v0.y, u.y);
            u.z = fmaf(p[e], v0.z, u.z), u.w = fmaf(p[e], v0.w, u.w);
            w.x = fmaf(p[e], v1.x, w.x), w.y = fmaf(p[e], v1.y, w.y);
            w.z = fmaf(p[e], v1.z, w.z), w.w = fmaf(p[e], v1.w, w.w);
          }
        }
      }
    }
    __syncthreads();  // the tile's stage is free
  }
  cp_async_wait<0>();
#pragma unroll
  for (int i = 0; i < MR; ++i) {
#pragma unroll
    for (int off = 8; off >= 1; off >>= 1) z[i] += __shfl_xor_sync(0xffffffffu, z[i], off);
    const int r = r0 + ty * MR + i;
    if (ty * MR + i < nrow) {
      at_put<float>(dm, a, x, r, o[i][0], m[i], z[i], tx);
      at_put<float>(dm, a, x, r, o[i][1], m[i], z[i], tx + 16);
    }
  }
}

// Joins the splits of units that have several: NR rows to W warps.
constexpr int AJ_THREADS = 256, AJ_WARPS = AJ_THREADS / 32;
template <typename T, int W, int NR>
__global__ void __launch_bounds__(AJ_THREADS)
    attend_join_kernel(Dims dm, const __grid_constant__ AttendArgs a, const int32_t* __restrict__ cu) {
  __shared__ float4 s_o[W > 1 ? AJ_WARPS * NR * 32 : 1];
  __shared__ float s_z[AJ_WARPS][NR];
  pdl_wait();
  const int R = dm.G * dm.window, groups = (R + NR - 1) / NR, warp = threadIdx.x >> 5;
  const int w = blockIdx.x * (AJ_WARPS / W) + warp / W, units = dm.L * dm.Hkv * dm.S;
  const bool real = w < units * groups;
  const int u = real ? w / groups : 0;
  AtUnit x = at_unit(dm, a, cu, u, 0, AT_TOK, a.chunk);
  if constexpr (sizeof(T) == 2) {
    const int rb = (w - u * groups) * NR / a.block, shares = a.nsps[a.nrb * u + rb];
    x.nsp = shares >> 16;
    x.first = shares & 0xffff;
    x.r0 = rb * a.block;
    // (a call that failed may not have written them)
    if (x.nsp < 0 || x.nsp > a.nsplit || at_slot<T>(a, x, x.nsp) > a.slots + 1) x.nsp = 0;
  }
  const bool inside = sizeof(T) == 2 && at_joins_inside(x.nsp, R);  // that unit is done
  at_join<T, W, NR>(dm, a, x, real && !inside ? (w - u * groups) * NR : R, warp % W,
                    s_o + (W > 1 ? warp * NR * 32 : 0), s_z[warp]);
}

template <typename T, int W, int NR>
static cudaError_t launch_join(const Dims& dm, const AttendArgs& a, const int32_t* cu, cudaStream_t st) {
  const int64_t groups = (int64_t)dm.L * dm.Hkv * dm.S * ((dm.G * dm.window + NR - 1) / NR);
  const dim3 grid((unsigned)((groups * W + AJ_WARPS - 1) / AJ_WARPS));
  return launch_pdl(true, attend_join_kernel<T, W, NR>, grid, AJ_THREADS, 0, st, dm, a, cu);
}
template <typename T>
static cudaError_t launch_join(const Dims& dm, const AttendArgs& a, const int32_t* cu, cudaStream_t st) {
  return a.nsplit <= 16 ? launch_join<T, 1, 8>(dm, a, cu, st) : launch_join<T, 8, 4>(dm, a, cu, st);
}

// ------------------------------------------------------------- launchers ----
template <int REP, int NB>
static cudaError_t launch_bf16(const CUtensorMap* maps, const Dims& dm, const AttendArgs& a, const int32_t* cu,
                               int64_t items, int sms, cudaStream_t st) {
  auto kern = attend_bf16_kernel<REP, NB>;
  JACAP_TRY(cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)at_smem<NB>()));
  const int places = sms * (3 - NB) < ATTEND_CTAS / NB ? sms * (3 - NB) : ATTEND_CTAS / NB;
  return launch_pdl(true, kern, (int)(items < places ? items : places), AtCfg<NB>::THREADS, at_smem<NB>(), st, maps[0],
                    maps[1], maps[2], maps[3], dm, a, cu);
}
template <int NT>
static cudaError_t launch_f32_rows(const Dims& dm, const AttendArgs& a, const int32_t* cu, int grid, cudaStream_t st) {
  using C = AgCfg<NT>;
  static_assert(C::SMEM <= 232448, "shared memory");
  auto kern = attend_f32_rows_kernel<NT>;
  JACAP_TRY(cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)C::SMEM));
  return launch_pdl(true, kern, grid, C::THREADS, C::SMEM, st, dm, a, cu);
}
template <int RB>
static cudaError_t launch_f32(const Dims& dm, const AttendArgs& a, const int32_t* cu, int grid, cudaStream_t st) {
  using C = AfCfg<RB>;
  static_assert((C::SMEM + 1024) * C::PER_SM <= 233472, "shared memory");
  JACAP_TRY(cudaFuncSetAttribute(attend_f32_kernel<RB>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)C::SMEM));
  return launch_pdl(true, attend_f32_kernel<RB>, grid, C::THREADS, C::SMEM, st, dm, a, cu);
}

static int attend_f32_rows(int rows) {
  return rows <= 4 ? 4 : rows <= 8 ? 8 : (rows <= 16 ? 16 : (rows <= 64 ? 64 : 128));
}
int attend_row_block(int dtype, int rows) { return dtype == 1 ? (rows <= 128 ? 128 : 256) : attend_f32_rows(rows); }

int attend_part_rows(int rows) { return rows <= 32 ? 32 : (rows <= 64 ? 64 : 128); }

cudaError_t launch_attend(const CUtensorMap* maps, const Dims& dm, int dtype, const AttendArgs& a, const int32_t* cu,
                          int sms, cudaStream_t st) {
  const int R = dm.G * dm.window;
  const int64_t units = (int64_t)dm.L * dm.Hkv * dm.S, blocks = units * a.nsplit * a.nrb;
  if (dtype == 1) {
    if (R <= 32) JACAP_TRY((launch_bf16<4, 1>(maps, dm, a, cu, blocks, sms, st)));
    else if (R <= 64) JACAP_TRY((launch_bf16<2, 1>(maps, dm, a, cu, blocks, sms, st)));
    else if (R <= 128) JACAP_TRY((launch_bf16<1, 1>(maps, dm, a, cu, blocks, sms, st)));
    else JACAP_TRY((launch_bf16<1, 2>(maps, dm, a, cu, blocks, sms, st)));
  } else {
    if (R <= 4) JACAP_TRY(launch_f32<4>(dm, a, cu, (int)blocks, st));
    else if (R <= 8) JACAP_TRY(launch_f32<8>(dm, a, cu, (int)blocks, st));
    else if (R <= 16) JACAP_TRY(launch_f32<16>(dm, a, cu, (int)blocks, st));
    else if (R <= 64) JACAP_TRY(launch_f32_rows<256>(dm, a, cu, (int)blocks, st));
    else JACAP_TRY(launch_f32_rows<512>(dm, a, cu, (int)blocks, st));
  }
  if (a.nsplit == 1 || (dtype == 1 && at_joins_inside(a.nsplit, R))) return cudaSuccess;
  return dtype == 1 ? launch_join<__nv_bfloat16>(dm, a, cu, st) : launch_join<float>(dm, a, cu, st);
}

}  // namespace jacap
