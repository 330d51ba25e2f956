// k_bytes.cu - rows of K and V into a cache held in 8 bits: e4m3 bytes with a power-of-two
// scale for each block of 64 tokens of a slot,
//   scale = least 2^e with max |x| <= 448 2^e,   byte = e4m3(x / scale), to nearest even.
// The division is exact, so that a byte is one rounding of its value; a scale that is raised later
// (append) multiplies the bytes' values by a power of two, which is exact but for the lowest of them.
#include "jacap_dev.cuh"
#include "jacap_internal.h"

namespace jacap {

constexpr int BY_BLOCK = 64;  // tokens per scale

// The scale of values up to `top` (not negative, not NaN): 2^e with 448 2^e >= top, from top's exponent and whether
// its mantissa passes that of 448 = 1.75 2^8.
__device__ __forceinline__ float by_scale(float top) {
  const uint32_t b = __float_as_uint(top);
  if (b == 0) return 0.f;
  const int e = (int)(b >> 23) - 8 + ((b & 0x7fffffu) > 0x600000u ? 1 : 0);
  return __uint_as_float((uint32_t)(e < 1 ? 1 : e) << 23);
}
// 1 / scale, exact for these (2^-126 to 2^120); 0 for 0.
__device__ __forceinline__ float by_inverse(float scale) { return scale == 0.f ? 0.f : 1.f / scale; }
// Two values to e4m3 bytes (a in the low one): to the nearest even, infinities to 448, NaN kept.
__device__ __forceinline__ uint32_t e4m3x2(float a, float b) {
  uint16_t r;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(b), "f"(a));
  return r;
}
__device__ __forceinline__ uint32_t e4m3x4(const float* x, float by) {
  return e4m3x2(x[0] * by, x[1] * by) | e4m3x2(x[2] * by, x[3] * by) << 16;
}

template <typename T>
struct ByPiece {  // 16 bytes of a row
  static constexpr int N = 16 / sizeof(T);
  float x[N];
  __device__ __forceinline__ void unpack(const uint4& w) {
    const uint32_t a[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (sizeof(T) == 2) {
        x[2 * i] = bf16lo(a[i]), x[2 * i + 1] = bf16hi(a[i]);
      } else {
        x[i] = __uint_as_float(a[i]);
      }
    }
  }
};

// A CTA per block of 64 tokens: the rows stay in registers between the block's maximum and their bytes, so that they are
// read once. Bound by memory: 32 layers of 8 heads, 4 prompts of 1638 to 4096 tokens in bf16 take 353 us, 2.17 GB at
// 6.1 TB/s (a plain copy reaches 6.8).
constexpr int BS_THREADS = 256;
template <typename T>
__global__ void __launch_bounds__(BS_THREADS) bytes_store_kernel(const __grid_constant__ ByteArgs a) {
  constexpr int N = ByPiece<T>::N, PER_ROW = D / N, STEP = BS_THREADS / PER_ROW, PIECES = BY_BLOCK / STEP;
  __shared__ float tops[BS_THREADS / 32];
  pdl_wait();
  const int tid = threadIdx.x;
  const uint32_t item = blockIdx.x / (uint32_t)a.blocks, b = blockIdx.x - item * a.blocks;
  const uint32_t unit = item >> 1, plane = unit / (uint32_t)a.S;
  const int kv = item & 1, s = (int)(unit - plane * a.S), l = (int)(plane / (uint32_t)a.Hkv), g = (int)(plane - l * a.Hkv);
  const int want = a.lengths != nullptr ? a.lengths[s] : a.rows;
  const int n = want < 0 ? 0 : (want < a.rows ? want : a.rows);
  if (b == 0 && plane == 0 && kv == 0 && tid == 0) {
    if (n != want) atomicOr(a.status, (uint32_t)ST_INVALID);
    if (a.lengths_out != nullptr) a.lengths_out[s] = n;
  }
  const int row0 = b * BY_BLOCK, live = n - row0 < BY_BLOCK ? n - row0 : BY_BLOCK;
  if (live <= 0) return;  // (the whole CTA: no barrier is met)
  const int64_t* st = a.row_strides + 4 * kv;
  const T* x = (const T*)a.rows_in[kv] + s * st[0] + l * st[1] + g * st[2];
  const int r0 = tid / PER_ROW, c = tid % PER_ROW;
  uint4 w[PIECES];
#pragma unroll
  for (int i = 0; i < PIECES; ++i) {
    const int r = r0 + i * STEP;
    w[i] = r < live ? __ldcs((const uint4*)(x + (row0 + r) * st[3]) + c) : make_uint4(0, 0, 0, 0);
  }
  float top = 0.f;
  ByPiece<T> p;
#pragma unroll
  for (int i = 0; i < PIECES; ++i) {
    p.unpack(w[i]);
#pragma unroll
    for (int e = 0; e < N; ++e) top = fmaxf(top, fabsf(p.x[e]));  // (without the NaN)
  }
#pragma unroll
  for (int off = 16; off >= 1; off >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, off));
  if ((tid & 31) == 0) tops[tid >> 5] = top;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < BS_THREADS / 32; ++i) top = fmaxf(top, tops[i]);
  const float scale = by_scale(top), by = by_inverse(scale);
  uint8_t* y = a.bytes[kv] + l * a.strides[0] + g * a.strides[1] + s * a.strides[2] + (int64_t)row0 * D + c * N;
#pragma unroll
  for (int i = 0; i < PIECES; ++i) {
    const int r = r0 + i * STEP;
    if (r >= live) continue;
    p.unpack(w[i]);
    if constexpr (N == 8) {
      *(uint2*)(y + r * D) = make_uint2(e4m3x4(p.x, by), e4m3x4(p.x + 4, by));
    } else {
      *(uint32_t*)(y + r * D) = e4m3x4(p.x, by);
    }
  }
  if (tid == 0) a.scales[kv][l * a.scale_strides[0] + g * a.scale_strides[1] + s * a.scale_strides[2] + b] = scale;
}

// W warps per unit and tensor (K or V): one where a few tokens come, so that all units are in one round of CTAs. A
// lane has four channels of a row. The new rows are read twice (the second time from the caches). Bound by the launch
// and three dependent reads: the length, the path, the row (28 layers of 4 heads, 16 slots, a token each: 3.2 us;
// 32 layers of 8 heads, 8 slots, up to 8 of 8 tokens: 4.1 us).
constexpr int BA_THREADS = 128;
template <typename T, int W>
__global__ void __launch_bounds__(BA_THREADS) bytes_append_kernel(const __grid_constant__ ByteArgs a) {
  constexpr int PER = BA_THREADS / 32 / W;  // items per CTA
  __shared__ float tops[2][BA_THREADS / 32];
  pdl_wait();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, part = warp % W;
  const uint32_t items = 2u * a.L * a.Hkv, ctas = (items + PER - 1) / PER;  // of a request
  const int s = (int)(blockIdx.x / ctas);
  const uint32_t item = (blockIdx.x - s * ctas) * PER + warp / W;
  const int given = a.lengths[s], want = a.taken != nullptr ? a.taken[s] : a.tokens;
  const int n = given < 0 ? 0 : (given < a.rows ? given : a.rows);
  const int most = a.rows - n < a.tokens ? a.rows - n : a.tokens;
  const int taken = want < 0 ? 0 : (want < most ? want : most);
  if (a.lengths_out != nullptr) {  // by the last of the request's CTAs, as `lengths` may be the same array
    __syncthreads();  // all of this CTA have read it
    if (tid == 0) {
      __threadfence();
      if (atomicAdd(a.counts + s, 1) == (int)ctas - 1) {
        a.counts[s] = 0;
        a.lengths_out[s] = n + taken;
      }
    }
  }
  bool bad = given != n || want != taken;
  const bool on = item < items && taken > 0;
  const int kv = item & 1, plane = on ? (int)(item >> 1) : 0, l = plane / a.Hkv, g = plane - l * a.Hkv;
  const int64_t* st = a.row_strides + 4 * kv;
  const T* x = (const T*)a.rows_in[kv] + s * st[0] + l * st[1] + g * st[2] + 4 * lane;
  // the new token that comes to row n + j
  const auto row = [&](int j, float* v) {
    int t = a.path != nullptr ? a.path[(int64_t)s * a.tokens + j] : j;
    if (t < 0 || t >= a.tokens) bad = true, t = 0;
    if constexpr (sizeof(T) == 2) {
      const uint2 w = *(const uint2*)(x + t * st[3]);
      v[0] = bf16lo(w.x), v[1] = bf16hi(w.x), v[2] = bf16lo(w.y), v[3] = bf16hi(w.y);
    } else {
      *(float4*)v = *(const float4*)(x + t * st[3]);
    }
  };
  const int b0 = n / BY_BLOCK, split = (b0 + 1) * BY_BLOCK - n;  // new tokens from `split` on are in the block after b0
  float* scales = a.scales[kv] + l * a.scale_strides[0] + g * a.scale_strides[1] + s * a.scale_strides[2];
  const float before = on && n > b0 * BY_BLOCK ? scales[b0] : 0.f;  // of the live tokens in b0
  float top[2] = {0.f, 0.f};
  if (on) {
#pragma unroll 4
    for (int j = part; j < taken; j += W) {
      float v[4];
      row(j, v);
      const float t = fmaxf(fmaxf(fabsf(v[0]), fabsf(v[1])), fmaxf(fabsf(v[2]), fabsf(v[3])));
      if (j < split) top[0] = fmaxf(top[0], t);
      else top[1] = fmaxf(top[1], t);
    }
  }
#pragma unroll
  for (int i = 0; i < 2; ++i) {
#pragma unroll
    for (int off = 16; off >= 1; off >>= 1) top[i] = fmaxf(top[i], __shfl_xor_sync(0xffffffffu, top[i], off));
    if constexpr (W > 1) {
      if (lane == 0) tops[i][warp] = top[i];
    }
  }
  if constexpr (W > 1) {
    __syncthreads();  // (also: the block's old scale is read)
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int k = 0; k < W; ++k) top[i] = fmaxf(top[i], tops[i][warp - part + k]);
  }
  if (bad && lane == 0) atomicOr(a.status, (uint32_t)ST_INVALID);
  if (!on) return;
  const float scale[2] = {fmaxf(before, by_scale(top[0])), by_scale(top[1])};
  const float by[2] = {by_inverse(scale[0]), by_inverse(scale[1])};
  uint8_t* y = a.bytes[kv] + l * a.strides[0] + g * a.strides[1] + s * a.strides[2] + 4 * lane;
  if (before > 0.f && scale[0] > before) {  // the live tokens' bytes at the raised scale
    const float f = before * by[0];
#pragma unroll 4
    for (int i = b0 * BY_BLOCK + part; i < n; i += W) {
      uint32_t* at = (uint32_t*)(y + (int64_t)i * D);
      const uint32_t w = *at;
      const float2 lo = e4m3_values(w & 0xffffu), hi = e4m3_values(w >> 16);
      const float v[4] = {lo.x, lo.y, hi.x, hi.y};
      *at = e4m3x4(v, f);
    }
  }
#pragma unroll 4
  for (int j = part; j < taken; j += W) {
    float v[4];
    row(j, v);
    *(uint32_t*)(y + (int64_t)(n + j) * D) = e4m3x4(v, j < split ? by[0] : by[1]);
  }
  if (part == 0 && lane == 0) {
    scales[b0] = scale[0];
    if (taken > split) scales[b0 + 1] = scale[1];
  }
}

cudaError_t launch_bytes_store(const ByteArgs& a, int dtype, cudaStream_t st) {
  const dim3 grid((unsigned)((int64_t)2 * a.L * a.Hkv * a.S * a.blocks));
  return dtype == 1 ? launch_pdl(true, bytes_store_kernel<__nv_bfloat16>, grid, BS_THREADS, 0, st, a)
                    : launch_pdl(true, bytes_store_kernel<float>, grid, BS_THREADS, 0, st, a);
}

template <typename T, int W>
static cudaError_t launch_append(const ByteArgs& a, cudaStream_t st) {
  const int64_t per = BA_THREADS / 32 / W, ctas = ((int64_t)2 * a.L * a.Hkv + per - 1) / per;
  return launch_pdl(true, bytes_append_kernel<T, W>, dim3((unsigned)(ctas * a.S)), BA_THREADS, 0, st, a);
}
cudaError_t launch_bytes_append(const ByteArgs& a, int dtype, cudaStream_t st) {
  if (a.tokens <= 8) return dtype == 1 ? launch_append<__nv_bfloat16, 1>(a, st) : launch_append<float, 1>(a, st);
  return dtype == 1 ? launch_append<__nv_bfloat16, 4>(a, st) : launch_append<float, 4>(a, st);
}

}  // namespace jacap
