// k_weigh.cu - the attention weight that every cached token received from a window of
// queries: for the rows r = (head h of the group, query j) of a unit,
//   l_r,i = scale q_r . k_i over the tokens i <= n - w + j (query j is at position n - w + j),
//   lse_r = ln sum_i exp(l_r,i),   weights_i = [before_i +] sum_r exp(l_r,i - lse_r).
// Two passes over K (the second only, where lse is known), each 128 x 128 x 128
// products per 128-token tile and block of 128 rows. The passes differ in which operand
// is which, so that neither needs a sum across threads for every tile:
//  - statistics: A = the rows, B = the tile: a thread has a row, its running maximum and
//    sum; the runs' results meet in a small kernel that writes lse;
//  - weights: A = the tile, B = the rows: a thread has a token and adds its weights.
// Runs of chunks are dealt to persistent CTAs as they become free (RunStream), from the
// work plan of the eviction pass.
//
// Measured, 32 queries of 32 heads on 8: one layer of 4099 tokens 24 us (plan, statistics,
// their join and weights: four dependent launches of 5 to 7 us each bound it), 8 layers of
// 32768 tokens 188 us: K twice is 1.07 GB, 5.7 TB/s. 28 layers of 8 slots of 2100 tokens, 4
// queries of 28 heads on 4 with lse given: 83 us, 6.3 TB/s. 64 queries a head (256 rows) 230 us
// for 4 layers: the second row block doubles the products and exponentials. Bound by memory up
// to 128 rows, by the exponentials beyond. Tried and left out: both passes in one launch so that
// the second finds K in L2 (480 us and more: a batch of planes small enough for L2 has each CTA
// wait for the others' statistics); the runs' join by the last run's own warp (n = 131072: 126
// -> 210 us, one warp's chain over hundreds of runs; 8 layers 226 us); two tiles at a time to each
// reader, so that a read of a row's constants serves both (8 layers 184 us, the slots 88).
//
// A row's sum takes exp over thousands of tokens: 32 at a time are added plainly and
// those sums with compensation (Kahan), so that the order of magnitude of the rounding
// does not grow with the run. Queries that a request does not have, and rows that see
// nothing (lse = -inf), give no weight: their constant is +inf, and they see no token (a token
// whose K is not finite and that no row sees has no weight either; one that a row sees, NaN).
//
// float32: CUDA cores; a warp takes 8 rows and two tokens per lane, so that 16-byte reads
// of K and (one address per warp) of Q feed 64 multiply-adds.
#include "jacap_dev.cuh"
#include "jacap_internal.h"

namespace jacap {

constexpr int WG_TILE_BYTES = TILE * D * 2;
constexpr int WG_BOX = WG_TILE_BYTES / 2;
constexpr int WG_IMG = 128 * D * 2;
constexpr int WG_BUILD0 = 2, WG_READ0 = 4;
constexpr float WG_LAZY = 8.f;  // log2 of how far a logit may pass the running maximum
constexpr int WG_NONE = -(1 << 30);  // j of a row that gives no weight: it sees no token
constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;

// Query rows of a request: `ql` queries, the first of them at position `p0` (it may be
// negative) of `n` live tokens that start at `start`.
struct WgReq {
  int64_t start;
  int n, ql, p0;
};
__device__ __forceinline__ WgReq wg_req(const Dims& dm, const WeighArgs& a, const int32_t* cu, int s) {
  WgReq x;
  x.start = cu[s];
  x.n = a.lengths != nullptr ? a.lengths[s] : cu[s + 1] - cu[s];
  const int ql = a.q_lens != nullptr ? a.q_lens[s] : dm.window;
  x.ql = ql < 0 ? 0 : (ql < dm.window ? ql : dm.window);
  x.p0 = x.n - x.ql;
  return x;
}
// Which query the j-th of request s is (-1: none).
__device__ __forceinline__ int wg_query(const Dims& dm, const WeighArgs& a, const WgReq& x, int s, int j) {
  if (j >= x.ql) return -1;
  const int q = a.q_rows != nullptr ? a.q_rows[(int64_t)s * dm.window + j] : j;
  return q >= 0 && q < dm.window ? q : -1;
}

// What a row's weights take: weight = f 2^(l scale2 - b), with b = M scale2 and f = 1 / Z for the row's maximum
// and sum (b is the rounded product that the sum's terms used too, so that its rounding cancels), or, where lse is
// given, b = lse log2 e and f = 1. No query, or nothing seen: b = inf and f = 0.
__device__ __forceinline__ float2 wg_const(const Dims& dm, const WeighArgs& a, const Item& item, int l, int g, int h,
                                           int qi, int r, int rows) {
  const float2 none = make_float2(INFINITY, 0.f);
  if (qi < 0) return none;
  if (a.given) {
    const float e = a.lse[(((int64_t)item.seq * dm.L + l) * dm.Hq + g * dm.G + h) * dm.window + qi];
    return e == -INFINITY ? none : make_float2(e * LOG2E, 1.f);
  }
  const float2 mz = a.norm[((int64_t)item.plane * dm.S + item.seq) * rows + r];
  return mz.y == 0.f ? none : make_float2(mz.x * a.scale2, 1.f / mz.y);
}

// Adds a (maximum, sum of exponentials from it) pair to (m, z). Nothing seen is (-inf, 0); NaN only, (-inf, NaN).
__device__ __forceinline__ void wg_merge(float& m, float& z, float2 x, float scale2) {
  if (x.x == -INFINITY && x.y == 0.f) return;
  const float top = fmaxf(m, x.x);
  z = (m == -INFINITY ? z : z * ex2((m - top) * scale2)) + (x.x == -INFINITY ? x.y : x.y * ex2((x.x - top) * scale2));
  m = top;
}

template <int NRB, bool SUM>
struct WgCfg {
  // groups of four read warps, that take the tiles in turn. The weights of one row block have four (an
  // accumulator each: with two, the latency of a group's chain through a tile bounds the pass, 114 us for
  // 64 planes of 32768 tokens of which K takes 79).
  static constexpr int GROUPS = SUM && NRB == 1 ? 4 : 2;
  static constexpr int THREADS = 32 * (WG_READ0 + 4 * GROUPS);
  static constexpr int IMGS = NRB == 1 ? 2 : 1;  // images: the next run's is built ahead
  static constexpr int STAGES = NRB <= 2 ? 4 : (NRB == 3 ? 3 : 2);
  static constexpr int ROWS = NRB * 128;
  static constexpr size_t SMEM = 1024 + (size_t)STAGES * WG_TILE_BYTES + (size_t)IMGS * NRB * WG_IMG + IMGS * ROWS * 12;
};

template <int NRB, bool SUM>
__global__ void __launch_bounds__(WgCfg<NRB, SUM>::THREADS, 1)
    weigh_bf16_kernel(const __grid_constant__ CUtensorMap kmap, Dims dm, Ws ws, const __grid_constant__ WeighArgs a,
                      const int32_t* __restrict__ cu) {
  using C = WgCfg<NRB, SUM>;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = (uint8_t*)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
  uint8_t* tiles = smem;
  uint8_t* img = tiles + C::STAGES * WG_TILE_BYTES;            // [IMGS][NRB][128 rows]
  float2* cst = (float2*)(img + C::IMGS * NRB * WG_IMG);       // [IMGS][ROWS] (b, f): weight = f 2^(l scale2 - b)
  int* jrow = (int*)(cst + C::IMGS * C::ROWS);                 // [IMGS][ROWS] j of the row
  __shared__ uint64_t full[C::STAGES], empty[C::STAGES], accfull[4], accempty[4], imgready[2], imgfree[2];
  __shared__ uint32_t s_tmem;
  __shared__ int s_abort;
  __shared__ RunQueue s_queue;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int R = dm.G * dm.window;
  if (tid == 0) {
    s_abort = 0;
    run_queue_init(&s_queue, 1 + 2 + 4 * C::GROUPS);  // MMA, build and read warps
    for (int i = 0; i < C::STAGES; ++i) {
      mbar_init(smem_u32(&full[i]), 1);
      mbar_init(smem_u32(&empty[i]), 1);
    }
    for (int i = 0; i < 4; ++i) {
      mbar_init(smem_u32(&accfull[i]), 1);
      mbar_init(smem_u32(&accempty[i]), 4);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(smem_u32(&imgready[i]), 2);
      mbar_init(smem_u32(&imgfree[i]), 1 + (SUM ? 4 * C::GROUPS : 0));  // the MMAs, and the readers of the constants
    }
    fence_mbar_init();
    prefetch_tmap(&kmap);
  }
  if (warp == 1) {
    tmem_alloc(smem_u32(&s_tmem), 512);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  pdl_wait();  // nothing before it touches global memory (a plan that failed has no runs)
  const uint32_t tmem = s_tmem;
  volatile int* abort = &s_abort;

  if (warp == 0) {
    // ------------------------------------------------ TMA producer --------
    if (lane == 0) {
      prefetch_tmap(&kmap);
      uint32_t it = 0;
      bool ok = true;
      Item item;
      for (RunStream<true> is(dm, ws, &s_queue, abort, true, SUM ? SCHED_SCORE : SCHED_KPASS); ok && is.next(item);) {
        const int l = item.plane / dm.Hkv, g = item.plane % dm.Hkv;
        for (int64_t t = item.t0; t < item.t1; t += TILE, ++it) {
          const int st = it % C::STAGES;
          if (it >= (uint32_t)C::STAGES &&
              !mbar_wait(smem_u32(&empty[st]), ((it / C::STAGES) & 1) ^ 1, ws, abort)) {
            ok = false;
            break;
          }
          const uint32_t kt = smem_u32(tiles + st * WG_TILE_BYTES), fb = smem_u32(&full[st]);
          mbar_arrive_expect_tx(fb, WG_TILE_BYTES);
          tma_load_4d(kt, &kmap, 0, (int)t, g, l, fb);
          tma_load_4d(kt + WG_BOX, &kmap, 64, (int)t, g, l, fb);
        }
      }
      for (uint32_t k = (it > (uint32_t)C::STAGES ? it - C::STAGES : 0); k < it; ++k)
        mbar_wait(smem_u32(&full[k % C::STAGES]), (k / C::STAGES) & 1, ws, nullptr);
    }
  } else if (warp == 1) {
    // ------------------------------------------------ MMA issuer ----------
    if (elect_one()) {
      uint32_t it = 0, e = 0, nrun = 0;
      bool ok = true, cont = false;
      Item item;
      for (RunStream<false> is(dm, ws, &s_queue, abort, true); ok && is.next(item);) {
        const int p = nrun % C::IMGS;
        if (!cont) {
          if (!mbar_wait(smem_u32(&imgready[p]), (nrun / C::IMGS) & 1, ws, abort)) break;
          tc_fence_after();
        }
        for (int64_t t = item.t0; ok && t < item.t1; t += TILE, ++it) {
          const int st = it % C::STAGES;
          if (!mbar_wait(smem_u32(&full[st]), (it / C::STAGES) & 1, ws, abort)) {
            ok = false;
            break;
          }
          const uint64_t kd = smem_desc_sw128(smem_u32(tiles + st * WG_TILE_BYTES), 16, 1024);
#pragma unroll
          for (int rb = 0; rb < NRB; ++rb) {
            const int slot = e & 3;
            if (e >= 4 && !mbar_wait(smem_u32(&accempty[slot]), ((e >> 2) & 1) ^ 1, ws, abort)) {
              ok = false;
              break;
            }
            tc_fence_after();
            const uint64_t rd = smem_desc_sw128(smem_u32(img + (p * NRB + rb) * WG_IMG), 16, 1024);
            const int left = R - rb * 128, n = SUM ? (left < 128 ? (left + 31) & ~31 : 128) : 128;
            const uint32_t idesc = idesc_bf16_f32(128, n, 0, 0);
#pragma unroll
            for (int k = 0; k < D / 16; ++k) {
              const uint64_t off = (uint64_t)((((k >> 2) * 16384) + (k & 3) * 32) >> 4);
              umma_f16_ss(tmem + 128 * slot, (SUM ? kd : rd) + off, (SUM ? rd : kd) + off, idesc, k > 0 ? 1u : 0u);
            }
            umma_commit(smem_u32(&accfull[slot]));
            ++e;
          }
          if (ok) umma_commit(smem_u32(&empty[st]));
        }
        if (!ok) break;
        cont = is.next_same_unit(item);
        if (!cont) {
          umma_commit(smem_u32(&imgfree[p]));
          ++nrun;
        }
      }
      // every MMA issued here completes before the CTA tears down tensor memory
      if (e > 0) mbar_wait(smem_u32(&accfull[(e - 1) & 3]), ((e - 1) >> 2) & 1, ws, nullptr);
    }
  } else if (warp < WG_READ0) {
    // ------------------ the rows of a run's unit, K-major with the 128-byte swizzle
    uint32_t nrun = 0;
    bool cont = false;
    Item item;
    for (RunStream<false> is(dm, ws, &s_queue, abort, false); is.next(item);) {
      const bool same = cont;
      cont = is.next_same_unit(item);
      if (same) continue;
      const int p = nrun % C::IMGS, l = item.plane / dm.Hkv, g = item.plane % dm.Hkv, b = warp - WG_BUILD0;
      const WgReq x = wg_req(dm, a, cu, item.seq);
      if (nrun >= (uint32_t)C::IMGS && !mbar_wait(smem_u32(&imgfree[p]), ((nrun / C::IMGS) & 1) ^ 1, ws, abort)) break;
      const __nv_bfloat16* q =
          (const __nv_bfloat16*)a.q + item.seq * dm.q_ss + l * dm.q_sl + (int64_t)g * dm.G * dm.q_sh;
      uint8_t* im = img + p * NRB * WG_IMG;
      for (int r0 = 32 * b; r0 < C::ROWS; r0 += 64) {  // 32 rows at a time, one per lane to look up
        const int r = r0 + lane, h = row_head(dm.window, a.tdiv, r), j = r - h * dm.window;
        const int qi = r < R ? wg_query(dm, a, x, item.seq, j) : -1;
        const int64_t off = qi >= 0 ? h * dm.q_sh + qi * dm.q_sp : 0;
        if constexpr (SUM) {
          const float2 k = wg_const(dm, a, item, l, g, h, qi, r, C::ROWS);
          cst[p * C::ROWS + r] = k;
          jrow[p * C::ROWS + r] = k.y != 0.f ? j : WG_NONE;
        }
#pragma unroll 8
        for (int k = 0; k < 16; ++k) {  // lanes 0-15 and 16-31: the 16-byte pieces of two rows
          const int rr = 2 * k + (lane >> 4), c = lane & 15;
          const int64_t o = __shfl_sync(0xffffffffu, off, rr);
          const int on = __shfl_sync(0xffffffffu, qi, rr);
          cp_async16(smem_u32(im + ((r0 + rr) >> 7) * WG_IMG + (c >> 3) * 16384 + sw128_off((r0 + rr) & 127, c & 7)),
                     (const uint4*)(q + o) + c, on >= 0);
        }
      }
      cp_async_commit();
      cp_async_wait<0>();
      fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) mbar_arrive(smem_u32(&imgready[p]));
      ++nrun;
    }
  } else {
    // ------------------------------------------------ readers -------------
    const int quarter = warp & 3, grp = (warp - WG_READ0) >> 2, y = quarter * 32 + lane;
    const uint32_t lanes = (uint32_t)(quarter * 32) << 16;
    const float scale2 = a.scale2, lazy = WG_LAZY / scale2;
    uint32_t it = 0, nrun = 0;
    bool cont = false, bad = false, live = false;
    int c0 = 0;
    WgReq x = {};
    float m[NRB], z[NRB], zc[NRB];  // statistics: running maximum, sum and its compensation
    int lim[NRB];                   // the last token that a row sees
    Item item;
    for (RunStream<false> is(dm, ws, &s_queue, abort, false); is.next(item);) {
      const int p = nrun % C::IMGS;
      if (!cont) {
        x = wg_req(dm, a, cu, item.seq);
        c0 = item.cidx;
#pragma unroll
        for (int rb = 0; rb < NRB; ++rb) {
          m[rb] = -INFINITY, z[rb] = 0.f, zc[rb] = 0.f;
          lim[rb] = x.p0 + (rb * 128 + y) - row_head(dm.window, a.tdiv, rb * 128 + y) * dm.window;
        }
        // (the constants are the builders' work: the tile's accumulators follow them)
        if (SUM && !mbar_wait(smem_u32(&imgready[p]), (nrun / C::IMGS) & 1, ws, abort)) goto done;
        if constexpr (SUM) {
          live = false;
#pragma unroll
          for (int r = 0; r < C::ROWS; r += 32) live |= jrow[p * C::ROWS + r + lane] != WG_NONE;
          live = __any_sync(0xffffffffu, live);
        }
      }
      for (int64_t t = item.t0; t < item.t1; t += TILE, ++it) {
        const int rel = (int)(t - x.start);  // the tile's first token
        const int nv = (int)(item.t1 - t < TILE ? item.t1 - t : TILE);
        float w = 0.f;
        const bool late = rel + TILE - 1 > x.p0;  // some row does not see all of the tile
#pragma unroll
        for (int rb = 0; rb < NRB; ++rb) {
          const uint32_t e = it * NRB + rb;
          // which group: its accumulators are its own, so that no barrier's phase passes it by
          // (four row blocks use all accumulators for every tile: one group sums them all)
          if ((SUM && NRB == 4 ? 0 : (int)((SUM ? it : e) % C::GROUPS)) != grp) continue;
          const int slot = e & 3;
          if (!mbar_wait(smem_u32(&accfull[slot]), (e >> 2) & 1, ws, abort)) goto done;
          tc_fence_after();
          const uint32_t acc = tmem + 128 * slot + lanes;
          if constexpr (SUM) {
            const int left = R - rb * 128, cols = left < 128 ? (left + 31) & ~31 : 128;
            const float2* cp = cst + p * C::ROWS + rb * 128;
            const int* jp = jrow + p * C::ROWS + rb * 128;
            float s[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 1
            for (int c = 0; c < cols; c += 32) {
              float v[32];
              tmem_ld32(acc + c, v);
              if (late) {
                const int need = rel + y - x.p0;  // queries j >= need see token rel + y
#pragma unroll
                for (int q = 0; q < 32; ++q) v[q] = jp[c + q] >= need ? v[q] : -INFINITY;
              }
#pragma unroll
              for (int q = 0; q < 32; q += 2) {
                const float4 k = *(const float4*)(cp + c + q);  // (no weight: f = 0)
                s[q & 3] = fmaf(ex2(fmaf(v[q], scale2, -k.x)), k.y, s[q & 3]);
                s[(q + 1) & 3] = fmaf(ex2(fmaf(v[q + 1], scale2, -k.z)), k.w, s[(q + 1) & 3]);
              }
            }
            w += (s[0] + s[1]) + (s[2] + s[3]);
          } else {
            const int last = lim[rb] - rel < nv - 1 ? lim[rb] - rel : nv - 1;  // columns that the row sees
            const bool masked = __any_sync(0xffffffffu, last < TILE - 1);
            float mm = m[rb], zz = z[rb], cc = zc[rb];
#pragma unroll 1
            for (int c = 0; c < 128; c += 32) {
              float v[32];
              tmem_ld32(acc + c, v);
              if (masked) {
#pragma unroll
                for (int q = 0; q < 32; ++q) v[q] = c + q <= last ? v[q] : -INFINITY;
              }
              float mx[4] = {v[0], v[1], v[2], v[3]};
#pragma unroll
              for (int q = 4; q < 32; ++q) mx[q & 3] = fmaxf(mx[q & 3], v[q]);
              const float top = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3]));
              const bool up = top > mm + lazy;
              if (__any_sync(0xffffffffu, up)) {
                const float f = up ? (mm == -INFINITY ? 0.f : ex2((mm - top) * scale2)) : 1.f;
                zz *= f, cc *= f;
                mm = up ? top : mm;
              }
              const float base = mm == -INFINITY ? 0.f : mm * scale2;
              float s[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
              for (int q = 0; q < 32; ++q) s[q & 3] += ex2(fmaf(v[q], scale2, -base));
              const float add = ((s[0] + s[1]) + (s[2] + s[3])) - cc, sum = zz + add;
              cc = (sum - zz) - add;
              zz = sum;
            }
            m[rb] = mm, z[rb] = zz, zc[rb] = cc;
          }
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(smem_u32(&accempty[slot]));
        }
        if (SUM && (NRB == 4 ? 0 : (int)(it % C::GROUPS)) == grp && y < nv) {
          const int64_t at = (int64_t)item.plane * dm.Ntot + t + y;
          if (!live) w = 0.f;  // (no row: what K holds is nobody's, NaN included)
          if (a.before != nullptr && rel + y < x.p0) w += a.before[at];
          bad |= !isfinite(w);
          a.weights[at] = w;
        }
      }
      cont = is.next_same_unit(item);
      if (cont) continue;
      if constexpr (SUM) {
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&imgfree[p]));
      } else {
        float2* to = a.stat + (((int64_t)item.plane * dm.c_cap + c0) * 2 + grp) * C::ROWS + y;
#pragma unroll
        for (int rb = 0; rb < NRB; ++rb) to[rb * 128] = make_float2(m[rb], z[rb]);
      }
      ++nrun;
    }
  done:
    if (bad) flag(ws, ST_NONFINITE);
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc(tmem, 512);
  }
}

// lse of every row from its unit's runs (bf16) or chunks: a block per 32 rows of a unit,
// eight threads to a row.
constexpr int WM_THREADS = 256;
__global__ void __launch_bounds__(WM_THREADS)
    weigh_lse_kernel(Dims dm, Ws ws, const __grid_constant__ WeighArgs a, const int32_t* __restrict__ cu, int rows,
                     int by_chunk) {
  pdl_wait();
  __shared__ float sm[8][32], sz[8][32];
  if (__syncthreads_or(status_failed(ws) ? 1 : 0)) return;
  const int R = dm.G * dm.window, blocks = (R + 31) / 32;
  const int u = blockIdx.x / blocks, lane = threadIdx.x & 31, part = threadIdx.x >> 5;
  const int s = u % dm.S, plane = u / dm.S, r = blockIdx.x % blocks * 32 + lane;
  const int list = plane < dm.big_planes ? 0 : 1;
  const int32_t* rpre = ws.rplan + list * (dm.S + 2) + 1;
  const int32_t* cpre = ws.plan + 1;
  const int first = by_chunk ? cpre[s] : rpre[s], count = (by_chunk ? cpre[s + 1] : rpre[s + 1]) - first;
  const int groups = by_chunk ? 1 : 2;
  float m = -INFINITY, z = 0.f;
  if (r < R)
    for (int i0 = part; i0 < count; i0 += 32) {  // four runs' (chunks') reads in flight (n = 131072: 126 -> 115 us)
      int c[4];
      float2 x[4][2];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int i = i0 + 8 * k < count ? i0 + 8 * k : i0;
        c[k] = by_chunk ? first + i : ws.runs[list * dm.c_cap + first + i].w;
      }
#pragma unroll
      for (int k = 0; k < 4; ++k)
#pragma unroll
        for (int g = 0; g < 2; ++g)
          x[k][g] = i0 + 8 * k < count && g < groups
                        ? a.stat[(((int64_t)plane * dm.c_cap + c[k]) * groups + g) * rows + r]
                        : make_float2(-INFINITY, 0.f);
#pragma unroll
      for (int k = 0; k < 4; ++k)
#pragma unroll
        for (int g = 0; g < 2; ++g) wg_merge(m, z, x[k][g], a.scale2);
    }
  sm[part][lane] = m;
  sz[part][lane] = z;
  __syncthreads();
  if (part != 0 || r >= R) return;
  m = -INFINITY, z = 0.f;
  for (int p = 0; p < 8; ++p) wg_merge(m, z, make_float2(sm[p][lane], sz[p][lane]), a.scale2);
  a.norm[(int64_t)u * rows + r] = make_float2(m, z);
  const int h = r / dm.window, j = r - h * dm.window;
  const WgReq x = wg_req(dm, a, cu, s);
  const int q = wg_query(dm, a, x, s, j);
  if (q >= 0)
    a.lse[(((int64_t)s * dm.L + plane / dm.Hkv) * dm.Hq + plane % dm.Hkv * dm.G + h) * dm.window + q] =
        z == 0.f ? -INFINITY : fmaf(m == -INFINITY ? 0.f : m, a.scale2 * LN2, logf(z));
}

// ------------------------------------------------------------- float32 ----
// A block takes a chunk at a time, 32 rows (four warps) or 64 of its unit at a time, in tiles of 64 tokens.
constexpr int WF_TOK = 64, WF_LD = D + 4;
template <int WARPS>
constexpr size_t wf_smem() { return ((size_t)8 * WARPS * D + 2 * WF_TOK * WF_LD + WARPS * WF_TOK + 3 * 8 * WARPS) * 4; }

template <bool SUM, int WARPS>
__global__ void __launch_bounds__(32 * WARPS, 2)
    weigh_f32_kernel(Dims dm, Ws ws, const __grid_constant__ WeighArgs a, const int32_t* __restrict__ cu, int rows) {
  constexpr int WF_THREADS = 32 * WARPS, WF_ROWS = 8 * WARPS;
  extern __shared__ __align__(16) float sf[];
  float* qs = sf;                        // [ROWS][D]
  float* ks = qs + WF_ROWS * D;          // [2][64][LD]
  float* red = ks + 2 * WF_TOK * WF_LD;  // [warp][64]
  float2* cst = (float2*)(red + WARPS * WF_TOK);  // [ROWS] (b, f)
  int* jrow = (int*)(cst + WF_ROWS);     // [ROWS]
  pdl_wait();
  if (__syncthreads_or(status_failed(ws) ? 1 : 0)) return;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int R = dm.G * dm.window;
  const float scale2 = a.scale2, lazy = WG_LAZY / scale2;
  bool bad = false;
  Item item;
  for (ItemStream is(dm, ws, blockIdx.x, gridDim.x); is.next(item);) {
    const int l = item.plane / dm.Hkv, g = item.plane % dm.Hkv;
    const WgReq x = wg_req(dm, a, cu, item.seq);
    const float* q = (const float*)a.q + item.seq * dm.q_ss + l * dm.q_sl + (int64_t)g * dm.G * dm.q_sh;
    const float* kb = (const float*)a.k + (int64_t)l * dm.kv_sl + (int64_t)g * dm.kv_sh;
    auto fetch = [&](int64_t t, int buf) {
      float* kt = ks + buf * WF_TOK * WF_LD;
#pragma unroll 4
      for (int e = tid; e < WF_TOK * 32; e += WF_THREADS) {
        const int tok = e >> 5, c = (e & 31) * 4;
        const bool on = t + tok < item.t1;
        cp_async16(smem_u32(kt + tok * WF_LD + c), kb + (t + (on ? tok : 0)) * dm.kv_st + c, on);
      }
    };
    for (int r0 = 0; r0 < R; r0 += WF_ROWS) {
      __syncthreads();  // the rows and the tiles before are read
      fetch(item.t0, 0);
      for (int e = tid; e < WF_ROWS * 32; e += WF_THREADS) {
        const int r = r0 + (e >> 5), c = (e & 31) * 4, h = row_head(dm.window, a.tdiv, r), j = r - h * dm.window;
        const int qi = r < R ? wg_query(dm, a, x, item.seq, j) : -1;
        cp_async16(smem_u32(qs + (e >> 5) * D + c), q + (qi >= 0 ? h * dm.q_sh + qi * dm.q_sp : 0) + c, qi >= 0);
        if (c == 0) {
          jrow[e >> 5] = j;
          if constexpr (SUM) {
            const float2 k = wg_const(dm, a, item, l, g, h, qi, r, rows);
            cst[e >> 5] = k;
            if (k.y == 0.f) jrow[e >> 5] = WG_NONE;
          }
        }
      }
      cp_async_commit();
      float m[8], z[8], zc[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) m[i] = -INFINITY, z[i] = 0.f, zc[i] = 0.f;
      int buf = 0;
      for (int64_t t = item.t0; t < item.t1; t += WF_TOK, buf ^= 1) {
        if (t + WF_TOK < item.t1) fetch(t + WF_TOK, buf ^ 1);
        cp_async_commit();
        cp_async_wait<1>();
        __syncthreads();
        const float *k0 = ks + buf * WF_TOK * WF_LD + lane * WF_LD, *k1 = k0 + 32 * WF_LD;
        float s[8][2];
#pragma unroll
        for (int i = 0; i < 8; ++i) s[i][0] = s[i][1] = 0.f;
#pragma unroll 2
        for (int c = 0; c < D; c += 4) {
          const float4 u = *(const float4*)(k0 + c), v = *(const float4*)(k1 + c);
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const float4 w = *(const float4*)(qs + (8 * warp + i) * D + c);
            s[i][0] = fmaf(w.x, u.x, fmaf(w.y, u.y, fmaf(w.z, u.z, fmaf(w.w, u.w, s[i][0]))));
            s[i][1] = fmaf(w.x, v.x, fmaf(w.y, v.y, fmaf(w.z, v.z, fmaf(w.w, v.w, s[i][1]))));
          }
        }
        const int rel = (int)(t - x.start);
        float w[2] = {0.f, 0.f};
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const int j = jrow[8 * warp + i];
#pragma unroll
          for (int b = 0; b < 2; ++b) {
            const int tok = lane + 32 * b;
            const bool see = t + tok < item.t1 && rel + tok <= x.p0 + j;
            if constexpr (SUM) {
              const float2 k = cst[8 * warp + i];
              if (see) w[b] = fmaf(ex2(fmaf(s[i][b], scale2, -k.x)), k.y, w[b]);
            } else if (see) {
              const float v = s[i][b];
              if (v > m[i] + lazy) {
                const float f = m[i] == -INFINITY ? 0.f : ex2((m[i] - v) * scale2);
                z[i] *= f, zc[i] *= f;
                m[i] = v;
              }
              const float add = ex2(fmaf(v, scale2, m[i] == -INFINITY ? 0.f : -m[i] * scale2)) - zc[i];
              const float sum = z[i] + add;
              zc[i] = (sum - z[i]) - add;
              z[i] = sum;
            }
          }
        }
        if constexpr (SUM) {
          red[warp * WF_TOK + lane] = w[0];
          red[warp * WF_TOK + lane + 32] = w[1];
        }
        __syncthreads();  // the stage is free, the sums are there
        if (SUM && tid < WF_TOK && t + tid < item.t1) {
          float v = 0.f;
#pragma unroll
          for (int k = 0; k < WARPS; ++k) v += red[k * WF_TOK + tid];
          const int64_t at = (int64_t)item.plane * dm.Ntot + t + tid;
          if (r0 > 0) v += a.weights[at];  // the rows before, by this thread
          else if (a.before != nullptr && rel + tid < x.p0) v += a.before[at];
          bad |= !isfinite(v);
          a.weights[at] = v;
        }
      }
      cp_async_wait<0>();
      if constexpr (!SUM) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          float mm = m[i], zz = z[i];
          float top = mm;
#pragma unroll
          for (int off = 16; off >= 1; off >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, off));
          zz = mm == -INFINITY ? zz : zz * ex2((mm - top) * scale2);
#pragma unroll
          for (int off = 16; off >= 1; off >>= 1) zz += __shfl_xor_sync(0xffffffffu, zz, off);
          const int r = r0 + 8 * warp + i;
          if (lane == 0 && r < R)
            a.stat[((int64_t)item.plane * dm.c_cap + item.cidx) * rows + r] = make_float2(top, zz);
        }
      }
    }
  }
  if (bad) flag(ws, ST_NONFINITE);
}

template <int NRB, bool SUM>
static cudaError_t launch_bf16(const CUtensorMap& kmap, const Dims& dm, const Ws& ws, const WeighArgs& a,
                               const int32_t* cu, int grid, cudaStream_t st) {
  constexpr size_t smem = WgCfg<NRB, SUM>::SMEM;
  static_assert(smem + 1024 <= 232448, "shared memory");  // 1024: the static variables
  JACAP_TRY(cudaFuncSetAttribute(weigh_bf16_kernel<NRB, SUM>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem));
  return launch_pdl(true, weigh_bf16_kernel<NRB, SUM>, grid, WgCfg<NRB, SUM>::THREADS, smem, st, kmap, dm, ws, a, cu);
}
template <bool SUM, int WARPS>
static cudaError_t launch_f32(const Dims& dm, const Ws& ws, const WeighArgs& a, const int32_t* cu, int grid, int rows,
                              cudaStream_t st) {
  auto kern = weigh_f32_kernel<SUM, WARPS>;
  JACAP_TRY(cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)wf_smem<WARPS>()));
  return launch_pdl(true, kern, grid, 32 * WARPS, wf_smem<WARPS>(), st, dm, ws, a, cu, rows);
}
template <bool SUM>
static cudaError_t launch_pass(const CUtensorMap& kmap, const Dims& dm, const Ws& ws, int dtype, const WeighArgs& a,
                               const int32_t* cu, int grid, int nrb, cudaStream_t st) {
  if (dtype != 1)
    return dm.G * dm.window <= 32 ? launch_f32<SUM, 4>(dm, ws, a, cu, 2 * grid, 128 * nrb, st)
                                  : launch_f32<SUM, 8>(dm, ws, a, cu, 2 * grid, 128 * nrb, st);
  switch (nrb) {
    case 1: return launch_bf16<1, SUM>(kmap, dm, ws, a, cu, grid, st);
    case 2: return launch_bf16<2, SUM>(kmap, dm, ws, a, cu, grid, st);
    case 3: return launch_bf16<3, SUM>(kmap, dm, ws, a, cu, grid, st);
    case 4: return launch_bf16<4, SUM>(kmap, dm, ws, a, cu, grid, st);
    default: return cudaErrorInvalidValue;
  }
}

cudaError_t launch_weigh(const CUtensorMap& kmap, const Dims& dm, const Ws& ws, int dtype, const WeighArgs& a,
                         const int32_t* cu, int grid, cudaStream_t st) {
  const int R = dm.G * dm.window, nrb = (R + 127) / 128;
  const int64_t blocks = (int64_t)dm.L * dm.Hkv * dm.S * ((R + 31) / 32);
  if (!a.given) {
    JACAP_TRY(launch_pass<false>(kmap, dm, ws, dtype, a, cu, grid, nrb, st));
    JACAP_TRY(launch_pdl(true, weigh_lse_kernel, (int)blocks, WM_THREADS, 0, st, dm, ws, a, cu, 128 * nrb,
                         dtype == 1 ? 0 : 1));
  }
  return launch_pass<true>(kmap, dm, ws, dtype, a, cu, grid, nrb, st);
}

}  // namespace jacap
