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
// split over CTAs (`chunk` tokens each, the drafted ones with the last), which leave
// unnormalised sums for a second launch to join where a request has several splits.
//
// bf16: R = G T rows are an M = 128 operand whatever R is: the memory's time for a tile
// (64 tokens, 32 KB of K and V: ~700 SM cycles at the copy rate with two CTAs per SM)
// covers its MMAs (N = 64 and N = 128: ~260 cycles) even where only a few rows are real,
// and the softmax warps work on real rows only: with R <= 32 every tensor-memory lane
// quarter holds a copy of the rows and takes a quarter of each tile's tokens (R <= 64: two
// copies, halves), each with a maximum and a sum of its own; the other tokens' weights are
// zero in its lanes, and the copies are joined at the end. So a warp has 16 columns
// per tile instead of 64, and no two warps ever wait for each other. More than 128 rows
// take several CTAs, neighbours that share K and V through L2.
// The weights p are rounded to bf16 for the second product (the sums Z are not): of an
// output of many comparable terms that is an error of about the output's own rounding.
// The maximum is only raised when a logit passes it by 2^8, which a rescaling of the
// accumulators then follows: rare after the first tiles, and harmless to the sums (p <= 256).
// Rows of V past the live tokens, and drafted rows past the request's, are zeroed in
// shared memory before the product, as 0 times what an unwritten row holds may be NaN;
// a drafted value that is not finite is zeroed too and added to the rows that see it.
//
// float32: CUDA cores, as the tensor cores would round the inputs. A warp takes 8 of a
// tile's 64 tokens for all rows of the CTA (8 or 32), four lanes to a token's dot
// products, and keeps a maximum, sums and accumulators of its own, so that tiles need no
// barrier but the one that says they have landed; the warps are joined at the end.
#include "jacap_dev.cuh"
#include "jacap_internal.h"

namespace jacap {

constexpr int AT_TOK = 64;             // tokens per tile
constexpr int AT_BOX = AT_TOK * 128;   // {64 channels, 64 tokens} bf16
constexpr int AT_TILE = 2 * AT_BOX;
constexpr int AT_STAGES = 2;
constexpr int AT_Q_BYTES = 128 * D * 2;
constexpr int AT_THREADS = 192;
constexpr uint32_t AT_COLS = 256;      // S (and P over it): 2 x 64, O: 128
constexpr uint32_t AT_O = 128;
constexpr size_t AT_SMEM = 1024 + AT_Q_BYTES + 2 * AT_STAGES * AT_TILE;
static_assert(2 * AT_STAGES * AT_TILE >= 128 * D * 4, "the ring holds the accumulators on their way out");
constexpr float AT_LAZY = 8.f;         // log2 of how far a logit may pass the maximum

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

__device__ __forceinline__ void tma_load_5d(uint32_t dst, const CUtensorMap* map, int c0, int c1, int c2, int c3, int c4,
                                            uint32_t bar) {
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
  int tok0, tok1, ncache, nt;  // this split's tokens, its tiles of cached tokens and in all (`tile` tokens each)
};
__device__ __forceinline__ AtUnit at_unit(const Dims& dm, const AttendArgs& a, const int32_t* cu, int64_t u, int split,
                                          int tile) {
  AtUnit x;
  x.u = u;
  x.split = split;
  x.s = (int)(u % dm.S);
  const int plane = (int)(u / dm.S);
  x.l = plane / dm.Hkv;
  x.g = plane % dm.Hkv;
  const int64_t start = cu[x.s], end = cu[x.s + 1];
  const bool ok = start >= 0 && end >= start && end <= dm.Ntot;
  const int64_t room = ok ? (end - start < a.max_seqlen ? end - start : a.max_seqlen) : 0;
  const int64_t live = a.lengths != nullptr ? a.lengths[x.s] : end - start;
  const int want = a.draft_lens != nullptr ? a.draft_lens[x.s] : dm.window;
  x.t0 = ok ? start : 0;
  x.n = (int)(live < 0 ? 0 : (live < room ? live : room));
  x.rows = want < 0 ? 0 : (want < dm.window ? want : dm.window);
  if (!ok || live != x.n || want != x.rows) atomicOr(a.status, (uint32_t)ST_INVALID);
  x.nd = a.kd != nullptr ? x.rows : 0;
  x.nsp = x.n > a.chunk ? (x.n - 1) / a.chunk + 1 : 1;
  x.tok0 = split * a.chunk;
  x.tok1 = x.tok0 + a.chunk < x.n ? x.tok0 + a.chunk : x.n;
  x.ncache = x.tok1 > x.tok0 ? (x.tok1 - x.tok0 - 1) / tile + 1 : 0;
  x.nt = x.ncache + (split == x.nsp - 1 && x.nd > 0 ? (x.nd - 1) / tile + 1 : 0);
  return x;
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
  const int h = r / dm.window, t = r - h * dm.window;
  if (t >= x.rows) return;
  if (x.nsp > 1) {
    const int64_t p = (x.u * a.nsplit + x.split) * ((int64_t)dm.G * dm.window) + r;
    *(float4*)(a.opart + p * D + 4 * lane) = acc;
    if (lane == 0) *(float2*)(a.mlpart + 2 * p) = make_float2(m, z);
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
        z == 0.f ? -INFINITY : m * a.scale + logf(z);
}

template <int REP>
__global__ void __launch_bounds__(AT_THREADS, 2)
    attend_bf16_kernel(const __grid_constant__ CUtensorMap kmap, const __grid_constant__ CUtensorMap vmap,
                       const __grid_constant__ CUtensorMap kdmap, const __grid_constant__ CUtensorMap vdmap, Dims dm,
                       const __grid_constant__ AttendArgs a, const int32_t* __restrict__ cu) {
  constexpr int ROWS = 128 / REP;      // rows per copy
  constexpr int NC = AT_TOK / REP;     // columns per softmax warp
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = (uint8_t*)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
  uint8_t* qs = smem;
  uint8_t* ks = qs + AT_Q_BYTES;
  uint8_t* vs = ks + AT_STAGES * AT_TILE;
  __shared__ uint64_t kfull[AT_STAGES], kempty[AT_STAGES], vfull[AT_STAGES], vempty[AT_STAGES], sfull[2], pready[2],
      pvdone[2];  // by a tile's parity: a wait for tile i knows that tile i - 2's product is done (S of tile i follows it)
  __shared__ uint32_t s_tmem, s_bad[2];
  __shared__ int s_abort;
  __shared__ float s_m[128], s_z[128];

  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  pdl_wait();
  const int rb = blockIdx.x % a.nrb, rest = blockIdx.x / a.nrb;
  const AtUnit x = at_unit(dm, a, cu, rest / a.nsplit, rest % a.nsplit, AT_TOK);
  if (x.split >= x.nsp) return;
  const int R = dm.G * dm.window, r0 = rb * 128;
  const int nrow = R - r0 < ROWS ? R - r0 : ROWS;
  if (x.nt == 0) {  // nothing to see
    for (int r = warp; r < nrow; r += AT_THREADS / 32)
      at_put<__nv_bfloat16>(dm, a, x, r0 + r, make_float4(0.f, 0.f, 0.f, 0.f), -INFINITY, 0.f, lane);
    return;
  }
  if (tid == 0) {
    s_abort = 0;
    s_bad[0] = s_bad[1] = 0;
    for (int i = 0; i < AT_STAGES; ++i) {
      mbar_init(smem_u32(&kfull[i]), 1);
      mbar_init(smem_u32(&kempty[i]), 1);
      mbar_init(smem_u32(&vfull[i]), 1);
      mbar_init(smem_u32(&vempty[i]), 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(smem_u32(&sfull[i]), 1);
      mbar_init(smem_u32(&pready[i]), 4);
      mbar_init(smem_u32(&pvdone[i]), 1);
    }
    fence_mbar_init();
  }
  if (warp == 1) {
    tmem_alloc(smem_u32(&s_tmem), AT_COLS);
    tmem_relinquish();
  }
  __syncthreads();
  Ws ws;
  ws.status = a.status;
  volatile int* abort = &s_abort;

  auto load = [&](int i, bool values) {  // tile i of K or V into its stage
    const int st = i % AT_STAGES;
    const uint32_t dst = smem_u32((values ? vs : ks) + st * AT_TILE), bar = smem_u32(&(values ? vfull : kfull)[st]);
    mbar_arrive_expect_tx(bar, AT_TILE);
    if (i < x.ncache) {
      const CUtensorMap* map = values ? &vmap : &kmap;
      const int t = (int)x.t0 + x.tok0 + i * AT_TOK;
      tma_load_4d(dst, map, 0, t, x.g, x.l, bar);
      tma_load_4d(dst + AT_BOX, map, 64, t, x.g, x.l, bar);
    } else {
      const CUtensorMap* map = values ? &vdmap : &kdmap;
      tma_load_5d(dst, map, 0, 0, x.g, x.l, x.s, bar);
      tma_load_5d(dst + AT_BOX, map, 64, 0, x.g, x.l, x.s, bar);
    }
  };
  if (tid == 0) {
    for (int i = 0; i < AT_STAGES && i < x.nt; ++i) {
      load(i, false);
      load(i, true);
    }
  }
  // the rows, K-major with the 128-byte swizzle; a copy for each group of lane quarters
  {
    const __nv_bfloat16* q = (const __nv_bfloat16*)a.q + x.s * dm.q_ss + x.l * dm.q_sl + (int64_t)x.g * dm.G * dm.q_sh;
#pragma unroll 4
    for (int e = tid; e < 128 * 16; e += AT_THREADS) {
      const int y = e >> 4, c = e & 15, r = y % ROWS;
      uint4 v = make_uint4(0, 0, 0, 0);
      if (r < nrow) {
        const int h = (r0 + r) / dm.window, t = r0 + r - h * dm.window;
        v = *((const uint4*)(q + h * dm.q_sh + t * dm.q_sp) + c);
      }
      *(uint4*)(qs + (c >> 3) * 16384 + sw128_off(y, c & 7)) = v;
    }
  }
  fence_proxy_async_smem();
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = s_tmem;

  if (warp == 0) {
    // ------------------------------------------------ TMA producer --------
    if (lane == 0) {
      int i = AT_STAGES;
      for (; i < x.nt; ++i) {
        const int st = i % AT_STAGES;
        const uint32_t par = ((i / AT_STAGES) & 1) ^ 1;
        if (!mbar_wait(smem_u32(&kempty[st]), par, ws, abort)) break;
        load(i, false);
        if (!mbar_wait(smem_u32(&vempty[st]), par, ws, abort)) {  // K of this tile is under way alone
          mbar_wait(smem_u32(&kfull[st]), (i / AT_STAGES) & 1, ws, nullptr);
          break;
        }
        load(i, true);
      }
      const int loaded = i < x.nt ? i : x.nt;  // what is under way lands before the CTA leaves
      for (int k = loaded > AT_STAGES ? loaded - AT_STAGES : 0; k < loaded; ++k) {
        mbar_wait(smem_u32(&kfull[k % AT_STAGES]), (k / AT_STAGES) & 1, ws, nullptr);
        mbar_wait(smem_u32(&vfull[k % AT_STAGES]), (k / AT_STAGES) & 1, ws, nullptr);
      }
    }
  } else if (warp == 1) {
    // ------------------------------------------------ MMA issuer ----------
    if (elect_one()) {
      constexpr uint32_t IDESC_S = idesc_bf16_f32(128, AT_TOK, 0, 0), IDESC_O = idesc_bf16_f32(128, D, 0, 1);
      const uint64_t qd = smem_desc_sw128(smem_u32(qs), 16, 1024);
      int issued = 0;  // second products
      auto second = [&](int i) {  // O += P V of tile i
        const int b = i & 1, st = i % AT_STAGES;
        if (!mbar_wait(smem_u32(&pready[b]), (i >> 1) & 1, ws, abort) ||
            !mbar_wait(smem_u32(&vfull[st]), (i / AT_STAGES) & 1, ws, abort))
          return false;
        tc_fence_after();
        const uint64_t vd = smem_desc_sw128(smem_u32(vs + st * AT_TILE), AT_BOX, 1024);
#pragma unroll
        for (int k = 0; k < AT_TOK / 16; ++k)
          umma_f16_ts(tmem + AT_O, tmem + 64 * b + 8 * k, vd + (uint64_t)((k * 2048) >> 4), IDESC_O,
                      i > 0 || k > 0 ? 1u : 0u);
        umma_commit(smem_u32(&vempty[st]));
        umma_commit(smem_u32(&pvdone[b]));
        ++issued;
        return true;
      };
      bool ok = true;
      int firsts = 0;
      for (int i = 0; ok && i < x.nt; ++i) {
        const int b = i & 1, st = i % AT_STAGES;
        if (!mbar_wait(smem_u32(&kfull[st]), (i / AT_STAGES) & 1, ws, abort)) {
          ok = false;
          break;
        }
        tc_fence_after();
        // S of tile i goes where P of tile i - 2 was: its product, issued before, has read it
        const uint64_t kd = smem_desc_sw128(smem_u32(ks + st * AT_TILE), 16, 1024);
#pragma unroll
        for (int k = 0; k < D / 16; ++k)
          umma_f16_ss(tmem + 64 * b, qd + (uint64_t)((((k >> 2) * 16384) + (k & 3) * 32) >> 4),
                      kd + (uint64_t)((((k >> 2) * AT_BOX) + (k & 3) * 32) >> 4), IDESC_S, k > 0 ? 1u : 0u);
        umma_commit(smem_u32(&kempty[st]));
        umma_commit(smem_u32(&sfull[b]));
        ++firsts;
        if (i > 0) ok = second(i - 1);
      }
      if (ok) ok = second(x.nt - 1);
      // every MMA issued here completes before the CTA tears down tensor memory
      if (firsts > 0) mbar_wait(smem_u32(&sfull[(firsts - 1) & 1]), ((firsts - 1) >> 1) & 1, ws, nullptr);
      if (issued > 0) mbar_wait(smem_u32(&pvdone[(issued - 1) & 1]), ((issued - 1) >> 1) & 1, ws, nullptr);
    }
  } else {
    // ------------------------------------------------ softmax -------------
    const int quarter = warp & 3, y = quarter * 32 + lane, t128 = tid - 64;
    const int rep = y / ROWS;  // the copy (uniform in a warp)
    const uint32_t lanes = (uint32_t)(quarter * 32) << 16;
    const float scale2 = a.scale * 1.4426950408889634f, lazy = AT_LAZY / scale2;
    const int row = r0 + y % ROWS;
    const uint64_t mask = row < R ? at_mask(dm, a, x, row % dm.window) : 0;
    float m = -INFINITY, z = 0.f;
    bool ok = true;
    for (int i = 0; i < x.nt; ++i) {
      const int b = i & 1, st = i % AT_STAGES;
      if (!mbar_wait(smem_u32(&sfull[b]), (i >> 1) & 1, ws, abort)) {
        ok = false;
        break;
      }
      tc_fence_after();
      float v[NC];
      if constexpr (NC == 64) {
        tmem_ld32x2(tmem + 64 * b + lanes, tmem + 64 * b + 32 + lanes, (uint32_t*)v, (uint32_t*)(v + 32));
      } else if constexpr (NC == 32) {
        tmem_ld32(tmem + 64 * b + 32 * rep + lanes, v);
      } else {
        tmem_ld16(tmem + 64 * b + 16 * rep + lanes, v);
      }
      const bool drafted = i >= x.ncache;
      const int nv = drafted ? x.nd : x.tok1 - x.tok0 - i * AT_TOK;  // rows of the tile that hold tokens
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
          if (!mbar_wait(smem_u32(&pvdone[(i - 1) & 1]), ((i - 1) >> 1) & 1, ws, abort)) {
            ok = false;
            break;
          }
          tc_fence_after();
#pragma unroll 1
          for (int c = 0; c < D; c += 32) {
            float w[32];
            tmem_ld32(tmem + AT_O + c + lanes, w);
#pragma unroll
            for (int e = 0; e < 32; ++e) w[e] *= f;
            tmem_st_32x32b_x32(tmem + AT_O + c + lanes, *(const uint32_t(*)[32])w);
          }
          tmem_wait_st();
        }
      }
      const float base = m == -INFINITY ? 0.f : m * scale2;
      float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int e = 0; e < NC; ++e) {
        v[e] = ex2(fmaf(v[e], scale2, -base));
        sum[e & 3] += v[e];
      }
      z += (sum[0] + sum[1]) + (sum[2] + sum[3]);
      uint32_t p[32];
#pragma unroll
      for (int c = 0; c < 32; ++c) {
        const int cc = c % (NC / 2);
        const uint32_t pk = pack_bf16x2(v[2 * cc], v[2 * cc + 1]);
        p[c] = REP == 1 || c / (NC / 2) == rep ? pk : 0u;
      }
      tmem_st_32x32b_x32(tmem + 64 * b + lanes, p);
      if (drafted || nv < AT_TOK) {
        if (!mbar_wait(smem_u32(&vfull[st]), (i / AT_STAGES) & 1, ws, abort)) {
          ok = false;
          break;
        }
        uint8_t* vt = vs + st * AT_TILE;
        for (int e = t128 + (drafted ? 0 : nv * 16); e < AT_TOK * 16; e += 128) {
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
            atomicOr(&s_bad[tok >> 5], 1u << (tok & 31));
          }
        }
        fence_proxy_async_smem();
      }
      tmem_wait_st();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(smem_u32(&pready[b]));
    }
    if (ok) ok = mbar_wait(smem_u32(&pvdone[(x.nt - 1) & 1]), ((x.nt - 1) >> 1) & 1, ws, abort);
    tc_fence_after();
    s_m[y] = m;
    s_z[y] = z;
    // all four warps meet here whether or not a wait failed, and leave together if one did
    if (!named_barrier_any(1, 128, !ok)) {
      // a row's copies scaled to their common maximum, through the ring (its last reader
      // was the last product) so that whole rows leave in one piece
      float top = -INFINITY;
#pragma unroll
      for (int c = 0; c < REP; ++c) top = fmaxf(top, s_m[c * ROWS + y % ROWS]);
      // (a copy whose logits are all NaN has the maximum -inf and a sum that is not 0)
      const auto share = [&](float mc, float zc) {
        return REP == 1 ? 1.f : (mc == -INFINITY ? (zc == 0.f ? 0.f : 1.f) : ex2((mc - top) * scale2));
      };
      const float f = share(m, z);
      float4* out = (float4*)ks;  // [128][32], 16-byte pieces swizzled by the row
#pragma unroll 1
      for (int c = 0; c < D; c += 32) {
        float w[32];
        tmem_ld32(tmem + AT_O + c + lanes, w);
#pragma unroll
        for (int e = 0; e < 8; ++e)
          out[y * 32 + ((c / 4 + e) ^ (lane & 7))] =
              make_float4(w[4 * e] * f, w[4 * e + 1] * f, w[4 * e + 2] * f, w[4 * e + 3] * f);
      }
      named_barrier_sync(1, 128);
      for (int r = warp - 2; r < nrow; r += 4) {
        float mr = -INFINITY, zr = 0.f;
        float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int c = 0; c < REP; ++c) mr = fmaxf(mr, s_m[c * ROWS + r]);
#pragma unroll
        for (int c = 0; c < REP; ++c) {
          const int yy = c * ROWS + r;
          const float mc = s_m[yy];
          top = mr;
          zr += s_z[yy] * share(mc, s_z[yy]);
          const float4 w = out[yy * 32 + (lane ^ (yy & 7))];
          acc.x += w.x, acc.y += w.y, acc.z += w.z, acc.w += w.w;
        }
        const uint64_t bad = (uint64_t)s_bad[1] << 32 | s_bad[0];
        if (bad != 0) {  // drafted values that are not finite, for the rows that see them
          uint64_t seen = bad & at_mask(dm, a, x, (r0 + r) % dm.window);
          const __nv_bfloat16* vd = (const __nv_bfloat16*)a.vd + x.s * a.vds[0] + x.l * a.vds[1] + x.g * a.vds[2] + 4 * lane;
          for (; seen != 0; seen &= seen - 1) {
            const uint2 w = *(const uint2*)(vd + (__ffsll((long long)seen) - 1) * a.vds[3]);
            const float e[4] = {bf16lo(w.x), bf16hi(w.x), bf16lo(w.y), bf16hi(w.y)};
            if (!isfinite(e[0])) acc.x += e[0];
            if (!isfinite(e[1])) acc.y += e[1];
            if (!isfinite(e[2])) acc.z += e[2];
            if (!isfinite(e[3])) acc.w += e[3];
          }
        }
        at_put<__nv_bfloat16>(dm, a, x, r0 + r, acc, mr, zr, lane);
      }
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc(tmem, AT_COLS);
  }
}

// ------------------------------------------------------------- float32 ----
constexpr int AF_THREADS = 256, AF_WARPS = 8, AF_TOK = 64, AF_LDK = D + 4;
constexpr int AF_KF = AF_TOK * AF_LDK, AF_VF = AF_TOK * D;  // floats per stage
template <int RB>
constexpr size_t af_smem() {
  return (size_t)(RB * D + 2 * (AF_KF + AF_VF) + AF_WARPS * 8 * RB + 2 * AF_WARPS * RB) * 4;
}

template <int RB>
__global__ void __launch_bounds__(AF_THREADS, 1)
    attend_f32_kernel(Dims dm, const __grid_constant__ AttendArgs a, const int32_t* __restrict__ cu) {
  extern __shared__ __align__(16) float sf[];
  float* qs = sf;                          // [RB][D]
  float* ks = qs + RB * D;                 // [2][64][LDK]
  float* vs = ks + 2 * AF_KF;              // [2][64][D]
  float* ps = vs + 2 * AF_VF;              // [warp][8 tokens][RB]
  float* sm = ps + AF_WARPS * 8 * RB;      // [warp][RB] maxima, then sums
  float* sz = sm + AF_WARPS * RB;
  static_assert(2 * (AF_KF + AF_VF) >= AF_WARPS * RB * D, "the tiles' space holds the warps' accumulators at the end");
  pdl_wait();
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int rb = blockIdx.x % a.nrb, rest = blockIdx.x / a.nrb;
  const AtUnit x = at_unit(dm, a, cu, rest / a.nsplit, rest % a.nsplit, AF_TOK);
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
  const float scale2 = a.scale * 1.4426950408889634f, lazy = AT_LAZY / scale2;
  const int tok = lane >> 2, kq = lane & 3;
  float m[RB], z[RB];       // z: this lane's token's share
  float4 acc[RB];           // channels 4 lane .. + 3
#pragma unroll
  for (int r = 0; r < RB; ++r) m[r] = -INFINITY, z[r] = 0.f, acc[r] = make_float4(0.f, 0.f, 0.f, 0.f);
  float* pw = ps + warp * 8 * RB;
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
#pragma unroll 1
      for (int k = 0; k < D; k += 16) {
        const float4 kk = *(const float4*)(kt + k);
#pragma unroll
        for (int r = 0; r < RB; ++r) {
          const float4 qq = *(const float4*)(qs + r * D + k + 4 * kq);
          s[r] = fmaf(qq.x, kk.x, fmaf(qq.y, kk.y, fmaf(qq.z, kk.z, fmaf(qq.w, kk.w, s[r]))));
        }
      }
      bool up = false;
#pragma unroll
      for (int r = 0; r < RB; ++r) {
        s[r] += __shfl_xor_sync(0xffffffffu, s[r], 1);
        s[r] += __shfl_xor_sync(0xffffffffu, s[r], 2);
        bool see = tok < left;
        if (drafted)
          see = r < nrow && at_mask(dm, a, x, (r0 + r) % dm.window) >> (first + 8 * warp + tok & 63) & 1 && see;
        if (!see) s[r] = -INFINITY;
        up |= s[r] > m[r] + lazy;
      }
      if (__any_sync(0xffffffffu, up)) {
#pragma unroll
        for (int r = 0; r < RB; ++r) {
          float top = s[r];
#pragma unroll
          for (int off = 4; off <= 16; off <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, off));
          if (top > m[r] + lazy) {  // the same on every lane
            const float f = m[r] == -INFINITY ? 0.f : ex2((m[r] - top) * scale2);
            m[r] = top;
            z[r] *= f;
            acc[r].x *= f, acc[r].y *= f, acc[r].z *= f, acc[r].w *= f;
          }
        }
      }
      __syncwarp();  // the previous tile's weights are read
#pragma unroll
      for (int r = 0; r < RB; ++r) {
        const float p = ex2(fmaf(s[r], scale2, m[r] == -INFINITY ? 0.f : -m[r] * scale2));
        z[r] += p;
        if ((r & 3) == kq) pw[tok * RB + r] = p;
      }
      __syncwarp();
      const float* vt = vs + (i & 1) * AF_VF + 8 * warp * D + 4 * lane;
      const int nt8 = left < 8 ? left : 8;
#pragma unroll 1
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
#pragma unroll
  for (int r = 0; r < RB; ++r) {
    float zz = z[r];
#pragma unroll
    for (int off = 4; off <= 16; off <<= 1) zz += __shfl_xor_sync(0xffffffffu, zz, off);
    if (lane == 0) sm[warp * RB + r] = m[r], sz[warp * RB + r] = zz;
    out[(warp * RB + r) * 32 + lane] = acc[r];
  }
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

// --------------------------------------------------------- joined splits ----
// A warp per row of a unit with several splits: their sums scaled to the largest
// maximum, added in the splits' order.
constexpr int AJ_THREADS = 128;
template <typename T>
__global__ void __launch_bounds__(AJ_THREADS)
    attend_join_kernel(Dims dm, const __grid_constant__ AttendArgs a, const int32_t* __restrict__ cu) {
  pdl_wait();
  const int R = dm.G * dm.window, lane = threadIdx.x & 31;
  const int64_t w = (int64_t)blockIdx.x * (AJ_THREADS / 32) + (threadIdx.x >> 5);
  if (w >= (int64_t)dm.L * dm.Hkv * dm.S * R) return;
  const int r = (int)(w % R);
  AtUnit x = at_unit(dm, a, cu, w / R, 0, AT_TOK);
  if (x.nsp == 1 || r % dm.window >= x.rows) return;
  const int64_t p0 = x.u * a.nsplit * R + r;
  const float scale2 = a.scale * 1.4426950408889634f;
  float m = -INFINITY;
  for (int j = lane; j < x.nsp; j += 32) m = fmaxf(m, a.mlpart[2 * (p0 + (int64_t)j * R)]);
#pragma unroll
  for (int off = 16; off >= 1; off >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, off));
  float z = 0.f;
  float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
  for (int j = 0; j < x.nsp; ++j) {
    const int64_t p = p0 + (int64_t)j * R;
    const float2 ml = *(const float2*)(a.mlpart + 2 * p);
    const float4 v = *(const float4*)(a.opart + p * D + 4 * lane);
    const float f = ml.x == m ? 1.f : ex2((ml.x - m) * scale2);
    const bool none = ml.x == -INFINITY && ml.y == 0.f;  // that split saw nothing
    z += none ? 0.f : ml.y * f;
    s.x += none ? 0.f : v.x * f;
    s.y += none ? 0.f : v.y * f;
    s.z += none ? 0.f : v.z * f;
    s.w += none ? 0.f : v.w * f;
  }
  x.nsp = 1;  // straight to the output
  at_put<T>(dm, a, x, r, s, m, z, lane);
}

// ------------------------------------------------------------- launchers ----
template <int REP>
static cudaError_t launch_bf16(const CUtensorMap* maps, const Dims& dm, const AttendArgs& a, const int32_t* cu,
                               int grid, cudaStream_t st) {
  static_assert(AT_SMEM + 2048 <= 116736, "two CTAs per SM");
  JACAP_TRY(cudaFuncSetAttribute(attend_bf16_kernel<REP>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)AT_SMEM));
  return launch_pdl(true, attend_bf16_kernel<REP>, grid, AT_THREADS, AT_SMEM, st, maps[0], maps[1], maps[2], maps[3], dm,
                    a, cu);
}
template <int RB>
static cudaError_t launch_f32(const Dims& dm, const AttendArgs& a, const int32_t* cu, int grid, cudaStream_t st) {
  static_assert(af_smem<RB>() <= 232448 - 1024, "shared memory");
  JACAP_TRY(cudaFuncSetAttribute(attend_f32_kernel<RB>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)af_smem<RB>()));
  return launch_pdl(true, attend_f32_kernel<RB>, grid, AF_THREADS, af_smem<RB>(), st, dm, a, cu);
}

int attend_row_block(int dtype, int rows) { return dtype == 1 ? 128 : (rows <= 8 ? 8 : 32); }

cudaError_t launch_attend(const CUtensorMap* maps, const Dims& dm, int dtype, const AttendArgs& a, const int32_t* cu,
                          cudaStream_t st) {
  const int R = dm.G * dm.window;
  const int64_t units = (int64_t)dm.L * dm.Hkv * dm.S, blocks = units * a.nsplit * a.nrb;
  if (blocks > INT32_MAX || units * R / 4 + 1 > INT32_MAX) return cudaErrorInvalidValue;
  if (dtype == 1) {
    if (R <= 32) JACAP_TRY(launch_bf16<4>(maps, dm, a, cu, (int)blocks, st));
    else if (R <= 64) JACAP_TRY(launch_bf16<2>(maps, dm, a, cu, (int)blocks, st));
    else JACAP_TRY(launch_bf16<1>(maps, dm, a, cu, (int)blocks, st));
  } else {
    if (R <= 8) JACAP_TRY(launch_f32<8>(dm, a, cu, (int)blocks, st));
    else JACAP_TRY(launch_f32<32>(dm, a, cu, (int)blocks, st));
  }
  if (a.nsplit == 1) return cudaSuccess;
  const int grid = (int)((units * R + AJ_THREADS / 32 - 1) / (AJ_THREADS / 32));
  return dtype == 1 ? launch_pdl(true, attend_join_kernel<__nv_bfloat16>, grid, AJ_THREADS, 0, st, dm, a, cu)
                    : launch_pdl(true, attend_join_kernel<float>, grid, AJ_THREADS, 0, st, dm, a, cu);
}

}  // namespace jacap
