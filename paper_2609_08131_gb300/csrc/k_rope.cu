// k_rope.cu - rotary positions: the first `rot` channels of every query and key
// head, taken as rot / 2 pairs (a, b), are turned by the angle of the token's
// position p,
//   (a, b) -> m (a cos t - b sin t, b cos t + a sin t),   t = p f_i for pair i
// (with the sine's sign changed for the inverse, which is the gradient too); m
// scales both. Pair i is channels (i, i + rot / 2), or (2 i, 2 i + 1) interleaved.
//
// Angles: f_i is given as a 64-bit fraction of a turn, so p f_i modulo one turn is
// the low 64 bits of an integer product, exact for every position (in float32 the
// angle of position 2^17 would be off by 0.008). Its nearest quarter turn is taken
// off as an integer and sincospif sees at most an eighth, rounded to 24 bits: the
// sine and cosine are within 6e-8 of those of 64-bit angles.
//
// A block takes TB tokens: their sines and cosines go to shared memory once, for all
// heads (they cost ~60 instructions each), then GS threads take a row (a head of a
// token) and four rows each are in flight at a time, the first of them asked for before
// the angles are worked out. 16-byte loads where the rows' addresses and strides allow them
// and no pair is split by a piece's end; otherwise a thread takes a pair of single elements.
//
// Bound by memory, and for few tokens by the launch. Measured, 32 + 8 heads in bf16: 32768
// tokens 125 us = 5.4 TB/s (1, 2, 3, 6 and 8 tokens per block: 193, 140, 124, 137, 134 us; five
// rows in flight 143 us; streaming loads and stores 125 us); 4 tokens 2.9 us.
#include <type_traits>

#include "jacap_dev.cuh"
#include "jacap_internal.h"

namespace jacap {

constexpr int RP_THREADS = 256, RP_UNROLL = 4, RP_TB = 4;

template <typename T>
__device__ __forceinline__ float rp_load(const T* p);
template <>
__device__ __forceinline__ float rp_load<float>(const float* p) { return *p; }
template <>
__device__ __forceinline__ float rp_load<__nv_bfloat16>(const __nv_bfloat16* p) { return __bfloat162float(*p); }
__device__ __forceinline__ void rp_store(float* p, float x) { *p = x; }
__device__ __forceinline__ void rp_store(__nv_bfloat16* p, float x) { *p = __float2bfloat16(x); }

// the 16 bytes of v as floats, and back (bf16: one rounding to nearest)
template <typename T>
__device__ __forceinline__ void rp_unpack(const uint4 v, float* x) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (sizeof(T) == 2) x[2 * i] = bf16lo(w[i]), x[2 * i + 1] = bf16hi(w[i]);
    else x[i] = __uint_as_float(w[i]);
  }
}
template <typename T>
__device__ __forceinline__ uint4 rp_pack(const float* x) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (sizeof(T) == 2) w[i] = pack_bf16x2(x[2 * i], x[2 * i + 1]);
    else w[i] = __float_as_uint(x[i]);
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}

__device__ __forceinline__ float2 rp_turn(float a, float b, float2 cs) {
  return make_float2(fmaf(a, cs.x, -(b * cs.y)), fmaf(b, cs.x, a * cs.y));
}

// lgs: log2 of the threads per row. A row's items: first its pairs (VEC: 16-byte
// pieces of them), then, where y is not x, the channels from `rot` on.
template <typename T, bool VEC>
__global__ void __launch_bounds__(RP_THREADS) rope_kernel(const __grid_constant__ RopeArgs a, int tb, int lgs) {
  constexpr int V = 16 / (int)sizeof(T);
  pdl_wait();
  __shared__ float2 cs[RP_TB][D / 2];
  const int tid = threadIdx.x, half = a.rot / 2;
  const int tok0 = blockIdx.x * tb, ntok = a.seqs * a.tokens;  // (fewer than 2^31)
  const int nt = ntok - tok0 < tb ? ntok - tok0 : tb;
  const int first_s = tok0 / a.tokens, first_j = tok0 - first_s * a.tokens;
  const int item = tid & ((1 << lgs) - 1), rpb = RP_THREADS >> lgs;
  const int heads = a.q.heads + a.k.heads;
  const int pairs = VEC ? (a.interleaved ? a.rot / V : half / V) : half;
  const int rest = VEC ? (D - a.rot) / V : D - a.rot;
  int t = 0, h = tid >> lgs, rs = first_s, rj = first_j;  // the row: token t of the block, its request and number
  auto settle = [&]() {
    while (h >= heads) {
      h -= heads;
      ++t;
      if (++rj == a.tokens) rj = 0, ++rs;
    }
  };
  settle();
  const bool two = VEC && !a.interleaved && item < pairs;  // (a, b) are half a rotation apart
  const int c0 = VEC ? (item < pairs ? item * V : a.rot + (item - pairs) * V)
                     : (item < pairs ? (a.interleaved ? 2 * item : item) : a.rot + item - pairs);
  const int c1 = VEC ? c0 + half : (a.interleaved ? c0 + 1 : c0 + half);
  const bool second = VEC ? two : item < pairs;
  using P = typename std::conditional<VEC, uint4, T>::type;  // a piece
  P va[RP_UNROLL], vb[RP_UNROLL];
  T* dst[RP_UNROLL];  // null: no row
  int tk[RP_UNROLL];
  auto load = [&]() {  // the next rows
#pragma unroll
    for (int u = 0; u < RP_UNROLL; ++u) {
      dst[u] = nullptr;
      tk[u] = t;
      if (t < nt) {
        const bool isq = h < a.q.heads;
        const RopeTensor& x = isq ? a.q : a.k;
        const int hh = isq ? h : h - a.q.heads;
        const T* src = (const T*)x.x + rs * x.xs[0] + rj * x.xs[1] + hh * x.xs[2];
        T* to = (T*)x.y + rs * x.ys[0] + rj * x.ys[1] + hh * x.ys[2];
        if (item < pairs || (item < pairs + rest && (const void*)src != (const void*)to)) {
          dst[u] = to;
          va[u] = *(const P*)(src + c0);
          if (second) vb[u] = *(const P*)(src + c1);
        }
      }
      h += rpb;
      settle();
    }
  };
  load();  // under way while the angles are worked out
  for (int e = tid; e < nt * half; e += RP_THREADS) {
    const int t = e / half, i = e - t * half;
    int s = first_s, j = first_j + t;
    while (j >= a.tokens) j -= a.tokens, ++s;
    const int64_t p = a.pos[s * a.ps[0] + j * a.ps[1]];
    const uint64_t turn = (uint64_t)p * a.turns[i];
    const uint32_t quarter = (uint32_t)((turn + (1ull << 61)) >> 62);  // 0 .. 3, 4 wraps to 0
    const int64_t left = (int64_t)(turn - ((uint64_t)quarter << 62));  // in [-2^61, 2^61)
    float sn, c;
    sincospif((float)left * 1.0842021724855044e-19f, &sn, &c);  // 2^-63: left in half turns
    if (quarter & 1) {
      const float x = c;
      c = -sn;
      sn = x;
    }
    if (quarter & 2) c = -c, sn = -sn;
    cs[t][i] = make_float2(a.amplitude * c, a.inverse ? -a.amplitude * sn : a.amplitude * sn);
  }
  __syncthreads();
  for (bool more = true; more;) {
#pragma unroll
    for (int u = 0; u < RP_UNROLL; ++u) {
      if (dst[u] == nullptr) continue;
      if constexpr (VEC) {
        if (item < pairs) {
          float x[V], y[V];
          rp_unpack<T>(va[u], x);
          if (two) {
            rp_unpack<T>(vb[u], y);
#pragma unroll
            for (int i = 0; i < V; ++i) {
              const float2 r = rp_turn(x[i], y[i], cs[tk[u]][c0 + i]);
              x[i] = r.x, y[i] = r.y;
            }
            *(uint4*)(dst[u] + c1) = rp_pack<T>(y);
          } else {
#pragma unroll
            for (int i = 0; i < V; i += 2) {
              const float2 r = rp_turn(x[i], x[i + 1], cs[tk[u]][(c0 + i) / 2]);
              x[i] = r.x, x[i + 1] = r.y;
            }
          }
          va[u] = rp_pack<T>(x);
        }
        *(uint4*)(dst[u] + c0) = va[u];
      } else if (item < pairs) {
        const float2 r = rp_turn(rp_load<T>(&va[u]), rp_load<T>(&vb[u]), cs[tk[u]][item]);
        rp_store(dst[u] + c0, r.x);
        rp_store(dst[u] + c1, r.y);
      } else {
        dst[u][c0] = va[u];
      }
    }
    more = t < nt;
    if (more) load();
  }
}

cudaError_t launch_rope(const RopeArgs& a, int dtype, bool vec, int sms, cudaStream_t st) {
  const int V = dtype == 1 ? 8 : 4;
  const int items = vec ? (a.interleaved ? a.rot / V : a.rot / 2 / V) + (D - a.rot) / V : D - a.rot / 2;
  int lgs = 0;
  while ((1 << lgs) < items) ++lgs;
  const int64_t ntok = (int64_t)a.seqs * a.tokens;
  if (ntok > INT32_MAX - RP_TB) return cudaErrorInvalidValue;
  // a token per block until that fills the SMs with eight blocks each
  const int tb = ntok >= (int64_t)sms * 8 * RP_TB ? RP_TB : 1;
  const int64_t blocks = (ntok + tb - 1) / tb;
  if (blocks > INT32_MAX) return cudaErrorInvalidValue;
  const dim3 grid((unsigned)blocks);
  if (dtype == 1)
    return vec ? launch_pdl(true, rope_kernel<__nv_bfloat16, true>, grid, RP_THREADS, 0, st, a, tb, lgs)
               : launch_pdl(true, rope_kernel<__nv_bfloat16, false>, grid, RP_THREADS, 0, st, a, tb, lgs);
  return vec ? launch_pdl(true, rope_kernel<float, true>, grid, RP_THREADS, 0, st, a, tb, lgs)
             : launch_pdl(true, rope_kernel<float, false>, grid, RP_THREADS, 0, st, a, tb, lgs);
}

}  // namespace jacap
