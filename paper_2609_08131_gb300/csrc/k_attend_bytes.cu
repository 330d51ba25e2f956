// k_attend_bytes.cu - attention of a few queries per request over its tokens in a cache held
// in 8 bits (e4m3 bytes k8, v8 and a scale for each block of 64 tokens) and over drafted tokens in bf16. For
// the rows r = (head h of the group, drafted token t) of a unit (request, layer, KV head)
//   l_i = scale ks_b q_r . k8_i,   o_r = sum_i exp(l_i - M) vs_b v8_i / Z,   Z = sum_i exp(l_i - M),
// b being token i's block; drafted tokens as in k_attend.cu.
//
// The tensor cores multiply the cache's bytes as they lie in memory, so that nothing is converted per token: what
// meets them is split into two parts of 8 bits instead, hi = e4m3(x) and lo = e5m2(x - hi). A bf16 value has eight
// significant bits: e4m3 keeps four, what is left is at most half of their last step and three bits of it remain, as
// many as e5m2 has, so that x = hi + lo exactly (from e4m3's lowest normal value, 2^-6, on; below that to 2^-14), and
//   q . k8 = hi . k8 + lo . k8
// are two products into one accumulator. The softmax weights are split alike, which rounds them to eight bits, as
// they would be for a product in bf16. (e5m2, not e4m3 again, because of its lowest step, 2^-16: with e4m3 weights
// below 2^-10 would be lost, and with them the output of rows whose largest weight meets a value near zero.)
//
// S is computed transposed, S^T = K8 Q^T: tokens are the 128 lanes of tensor memory and rows its columns (16, 32 or
// 64 per CTA, padded), so that one query row costs a small product, not one of 128 rows. A softmax warp has 32
// tokens, a lane one token of all rows: the maximum over a tile is a warp's reduction and an exchange of 4 values per
// row; the sums stay with the lanes until the item's end. O^T = V8^T P^T accumulates with channels as lanes.
//
// A weight is w = exp2(l log2 e + log2 vs_b - ref_r), which takes in V's scale, and fits e4m3 (448) as ref_r follows
// the rows' maxima: a tile whose largest weight would pass 2^8.75, or not reach 2^0.25, moves ref_r so that it is
// 2^4.5, and the accumulators are rescaled. (Downwards too, so that weights that are small beside one seen before,
// but not beside their neighbours, keep their bits; 2^-40 below the largest one seen it stops.) Where one of a tile's
// four quarters has none above 2^-6 of the largest (a prompt's first token may have nearly all of the weight, and a
// value near zero), the largest is put to 2^8.5 instead, so that the others keep eight bits down to 2^-14.5 of it. Z
// takes w / vs_b.
//
// That holds while V's scales are of ordinary size. Beside a block of 2^120 (of a value that is infinite) or 2^-126
// the other blocks' weights, or its own part of Z, would leave float32's range, and eight bits long before. So a
// block whose scale is outside 2^-32 .. 2^16 (values all below 1e-7, or one above 2.9e7) counts in Z with the scale
// of an ordinary one, and its part of the output is not left to the tensor cores but added at the item's end, one by
// one (add_far): one such block in every slot and head makes 16 slots' 24 us 35, a chain's 64 us 109 and the trees'
// 322 us 796.
//
// CTAs and splits are those of k_attend.cu: persistent CTAs with even shares of all tiles (128 tokens: 16 KB of K, 16
// of V); a split's sums are joined by the CTA that finishes its unit's last one. More than 64 rows: K and V are read
// again for each 64. (Turning the tiles to bf16 in shared memory for products of 128 rows and more takes 151 us for
// 128 rows of 8 heads over 31290 tokens, this 58 us; 256 rows 123 and 87 us; only 512 rows gain, 134 and 149 us.)
//
// Measured, 32 query heads of 8 KV heads: 16 slots of about 2100 tokens 24.4 us (69 MB, 10 us at a copy's rate;
// start, end and join take some 9 us), a chain of 8 over 131011 tokens 63.6 us (268 MB, 4.2 TB/s, floor 39.5 us), 48
// slots of 28 / 4 heads 57 us (278 MB, 4.9 TB/s, floor 41 us). With 16 and 32 rows the loads' latency and the softmax
// chain bound it, with 64 the chain: 16 trees of 64 over 46 to 16383 tokens, 40 / 8 heads, 321 us, 55 % of the issue
// slots, tensor pipe 20 %.
#include "k_attend_body.cuh"

namespace jacap {

constexpr int AB_TOK = 128, AB_TILE = AB_TOK * D;  // bytes of a tile of K or V; a drafted one: 64 tokens of bf16
constexpr int AB_QUEUE = 5;  // items published and not yet done with by all
// A CTA of N rows. Warps: 0 TMA producer, 1 MMA, then two teams of CG softmax groups (four warps, GR rows each), then
// those that fetch rows. A softmax is a chain of some 2000 to 4600 cycles, of which a warp waits most: the teams take
// turns at the tiles, each with accumulators and references of its own, which meet at an item's end.
constexpr int AB_TURNS = 2, AB_SBUF = 4;  // teams, and tiles' S at a time
template <int N>
struct AbCfg {
  static constexpr int GR = N == 64 ? 32 : 16, CG = N / GR, GROUPS = AB_TURNS * CG;
  static constexpr int PER_SM = N == 16 ? 2 : 1;                   // CTAs
  static constexpr int RING = N == 16 ? 5 : (N == 32 ? 10 : 8);    // tiles in flight
  static constexpr int LOADERS = 2, LOAD0 = 2 + 4 * GROUPS, THREADS = 32 * (LOAD0 + LOADERS);
  static constexpr int PART = N * D;                               // bytes of the rows' hi or lo part
  static constexpr int WBUF = 2 * N * D;                           // bytes of a team's weights
  static constexpr uint32_t COLS = N == 16 ? 128 : (N == 32 ? 256 : 512);  // S N AB_SBUF, O N AB_TURNS
};
constexpr float AB_HIGH = 8.75f, AB_LOW = 0.25f, AB_TOP = 4.5f, AB_DEEP = 40.f;  // log2 of the weights' bounds, see above
constexpr float AB_WIDE = 6.f, AB_WIDE_LOW = 7.f, AB_WIDE_TOP = 8.5f;            // where a tile's quarters are that far apart
constexpr float AB_UNIT = -8.f;  // log2 of V's unit in the sums: about the scale of a block of ordinary values

template <int N>
struct AbSmem {
  using C = AbCfg<N>;
  uint64_t full[C::RING], empty[C::RING];
  uint64_t sfull[AB_SBUF], pready[2], pvdone[2];  // by a tile's buffer, and its team
  uint64_t qfull[AB_QUEUE], qempty[AB_QUEUE];
  uint64_t rowsready, rowsfree, rowsasked, ofree, drained;
  AtUnit queue[AB_QUEUE];
  uint64_t rowmask[N];                     // drafted tokens that a row sees
  __align__(16) float4 top[2][N];                  // by a tile's parity: the four quarters' maxima of a row
  __align__(16) float base[4 * C::GROUPS][C::GR];  // a warp's own: its rows' maxima, then log2 vs - ref
  __align__(16) float coef[4 * C::GROUPS][C::GR];  // and what their products are multiplied with
  float sum[2][4][N], ref[2][N], inv[2][N];        // by team
  float qfac[AB_QUEUE][N];                 // scale log2(e) 2^e of a row
  uint32_t tmem, bad[2];
  float2 norm[N];                          // a row's reference, and what exp2(logit - reference) is multiplied with
  float far[C::GROUPS][4][64];             // add_far's weights
  int abort, last, any_far;
};
template <int N>
constexpr size_t ab_used() {
  return (size_t)AbCfg<N>::RING * AB_TILE + 4 * AbCfg<N>::PART + 2 * AbCfg<N>::WBUF + sizeof(AbSmem<N>);
}
template <int N>
constexpr size_t ab_smem() { return 233472 / AbCfg<N>::PER_SM - 1024; }
static_assert(ab_used<16>() <= ab_smem<16>() && ab_used<32>() <= ab_smem<32>() && ab_used<64>() <= ab_smem<64>(), "shared memory");

// Instruction descriptor of kind::f8f6f4: A of e4m3, B of e4m3 or e5m2, f32 D (the fields of kind::f16's).
__host__ __device__ constexpr uint32_t idesc_e4m3_f32(int M, int N, int a_mn, int b_mn, bool b_e5m2) {
  return (1u << 4) | (b_e5m2 ? 1u << 10 : 0u) | ((uint32_t)a_mn << 15) | ((uint32_t)b_mn << 16) | ((uint32_t)(N >> 3) << 17) |
         ((uint32_t)(M >> 4) << 24);
}
// D[tmem] (+)= A[smem] B[smem], 8 bits, K = 32.
__device__ __forceinline__ void umma_f8_ss(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc,
                                           uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}" ::"r"(d_tmem),
      "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate)
      : "memory");
}
__device__ __forceinline__ float warp_max(float x) {  // (without NaN)
  float r;
  asm volatile("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(x));
  return r;
}
// Four values' parts, hi = e4m3(x) and lo = e5m2(x - hi), packed (a's in the low bytes). The difference is taken in
// 16 bits (eleven significant ones, exact from there on), two at a time.
__device__ __forceinline__ void split_f8(float a, float b, float c, float d, uint32_t& hi, uint32_t& lo) {
  asm("{\n\t.reg .b16 h0, h1, l0, l1;\n\t.reg .b32 v0, v1, x0, x1;\n\t"
      "cvt.rn.satfinite.e4m3x2.f32 h0, %3, %2;\n\tcvt.rn.satfinite.e4m3x2.f32 h1, %5, %4;\n\t"
      "cvt.rn.f16x2.e4m3x2 v0, h0;\n\tcvt.rn.f16x2.e4m3x2 v1, h1;\n\t"
      "cvt.rn.f16x2.f32 x0, %3, %2;\n\tcvt.rn.f16x2.f32 x1, %5, %4;\n\t"
      "sub.rn.f16x2 x0, x0, v0;\n\tsub.rn.f16x2 x1, x1, v1;\n\t"
      "cvt.rn.satfinite.e5m2x2.f16x2 l0, x0;\n\tcvt.rn.satfinite.e5m2x2.f16x2 l1, x1;\n\t"
      "mov.b32 %0, {h0, h1};\n\tmov.b32 %1, {l0, l1};\n\t}"
      : "=r"(hi), "=r"(lo)
      : "f"(a), "f"(b), "f"(c), "f"(d));
}
__device__ __forceinline__ void sts_u32s(uint32_t at, const uint32_t (&v)[2]) {
  asm volatile("st.shared.v2.u32 [%0], {%1, %2};" ::"r"(at), "r"(v[0]), "r"(v[1]) : "memory");
}
__device__ __forceinline__ void sts_u32s(uint32_t at, const uint32_t (&v)[4]) {
  asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]) : "memory");
}
__device__ __forceinline__ void sts_f32(uint32_t at, float x) { asm volatile("st.shared.f32 [%0], %1;" ::"r"(at), "f"(x) : "memory"); }
__device__ __forceinline__ float lds_f32(uint32_t at) {
  float x;
  asm volatile("ld.shared.f32 %0, [%1];" : "=f"(x) : "r"(at) : "memory");
  return x;
}
__device__ __forceinline__ float4 lds_f32x4(uint32_t at) {
  float4 x;
  asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(x.x), "=f"(x.y), "=f"(x.z), "=f"(x.w) : "r"(at) : "memory");
  return x;
}

// The weights' bytes of N rows: a line of 2 N bytes per token, the rows' hi parts and then their lo parts, MN-major
// with the swizzle of as many bytes (16-byte pieces, by bits of the byte offset from 7 on).
// Shared-memory descriptor of that, from byte `saddr` on: 8 tokens every 16 N bytes.
template <int N>
__device__ __forceinline__ uint64_t weight_desc(uint32_t saddr) {
  const uint64_t swizzle = N == 64 ? 2 : (N == 32 ? 4 : 6);  // 128, 64, 32 bytes
  return (uint64_t)((saddr & 0x3FFFFu) >> 4) | (uint64_t)1 << 16 | (uint64_t)(16 * N >> 4) << 32 | (uint64_t)1 << 46 |
         swizzle << 61;
}

// 4, 8, 16 or 32 columns of this thread's lane, and back.
__device__ __forceinline__ void tmem_ld_cols(uint32_t at, float (&v)[32]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,"
      "%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];\n\ttcgen05.wait::ld.sync.aligned;"
      : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7]), "=f"(v[8]),
        "=f"(v[9]), "=f"(v[10]), "=f"(v[11]), "=f"(v[12]), "=f"(v[13]), "=f"(v[14]), "=f"(v[15]), "=f"(v[16]),
        "=f"(v[17]), "=f"(v[18]), "=f"(v[19]), "=f"(v[20]), "=f"(v[21]), "=f"(v[22]), "=f"(v[23]), "=f"(v[24]),
        "=f"(v[25]), "=f"(v[26]), "=f"(v[27]), "=f"(v[28]), "=f"(v[29]), "=f"(v[30]), "=f"(v[31])
      : "r"(at)
      : "memory");
}
__device__ __forceinline__ void tmem_ld_cols(uint32_t at, float (&v)[8]) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];\n\ttcgen05.wait::ld.sync.aligned;"
               : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7])
               : "r"(at)
               : "memory");
}
__device__ __forceinline__ void tmem_st_cols(uint32_t at, const float (&v)[4]) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x4.b32 [%0], {%1,%2,%3,%4};" ::"r"(at), "f"(v[0]), "f"(v[1]), "f"(v[2]),
               "f"(v[3])
               : "memory");
}
__device__ __forceinline__ void tmem_st_cols(uint32_t at, const float (&v)[8]) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"r"(at), "f"(v[0]),
               "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7])
               : "memory");
}
__device__ __forceinline__ void tmem_ld_cols(uint32_t at, float (&v)[4]) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x4.b32 {%0,%1,%2,%3}, [%4];\n\ttcgen05.wait::ld.sync.aligned;"
               : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3])
               : "r"(at)
               : "memory");
}
__device__ __forceinline__ void tmem_ld_cols(uint32_t at, float (&v)[16]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];\n\t"
      "tcgen05.wait::ld.sync.aligned;"
      : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7]), "=f"(v[8]),
        "=f"(v[9]), "=f"(v[10]), "=f"(v[11]), "=f"(v[12]), "=f"(v[13]), "=f"(v[14]), "=f"(v[15])
      : "r"(at)
      : "memory");
}
__device__ __forceinline__ void tmem_st_cols(uint32_t at, const float (&v)[16]) {
  tmem_st_32x32b_x16(at, *(const uint32_t(*)[16])v);
}

// The sums over a warp's lanes of x[0 .. N): lane l gets that of l % N (N = 8, 16, 32).
template <int N>
__device__ __forceinline__ float lane_sums(float* x, int lane) {
#pragma unroll
  for (int half = N / 2; half >= 1; half >>= 1) {
    const bool upper = (lane & half) != 0;
#pragma unroll
    for (int i = 0; i < half; ++i) {
      const float mine = upper ? x[i + half] : x[i], other = upper ? x[i] : x[i + half];
      x[i] = mine + __shfl_xor_sync(0xffffffffu, other, half);
    }
  }
#pragma unroll
  for (int off = N; off < 32; off <<= 1) x[0] += __shfl_xor_sync(0xffffffffu, x[0], off);
  return x[0];
}

// log2 of a block's scale, exact for a power of two.
__device__ __forceinline__ float log2_scale(float x) {
  const uint32_t b = __float_as_uint(x), m = b & 0x7fffffu;
  return (float)((int)(b >> 23) - 127) + (m == 0 ? 0.f : __log2f(__uint_as_float(m | 0x3f800000u)));
}

// Whether a block's values go past the tensor cores (see above).
__device__ __forceinline__ bool is_far(float vs) { return vs > 0.f && (vs < 0x1p-32f || vs > 0x1p16f); }

// Drafted values that are not finite (of the tokens `seen`, zeroed in the product), one channel, added up.
__device__ __noinline__ float bad_values(const __nv_bfloat16* vd, int64_t stride, uint64_t seen) {
  float y = 0.f;
  for (; seen != 0; seen &= seen - 1) {
    const float d = __bfloat162float(vd[(__ffsll((long long)seen) - 1) * stride]);
    if (!isfinite(d)) y += d;
  }
  return y;
}

// A row's logarithm of the sum of exponentials, of the reference m (log2) and the sum.
__device__ __forceinline__ float row_lse(float m, float sum) {
  return sum == 0.f ? -INFINITY : m * 0.6931471805599453f + logf(sum);
}
// A row to the output: channels 4 lane .. + 3 of its sums, its reference and sum of weights.
__device__ __forceinline__ void put_row(const Dims& dm, const AttendArgs& a, int s, int l, int head, int t, bool real,
                                        float4 y, float m, float sum, int lane) {
  if (!real) return;
  const float inv = sum == 0.f ? 0.f : 1.f / sum;
  __nv_bfloat16* o = (__nv_bfloat16*)a.o + s * a.os[0] + l * a.os[1] + head * a.os[2] + t * a.os[3] + 4 * lane;
  *(uint2*)o = make_uint2(pack_bf16x2(y.x * inv, y.y * inv), pack_bf16x2(y.z * inv, y.w * inv));
  if (lane == 0 && a.lse != nullptr) a.lse[s * a.ls[0] + l * a.ls[1] + head * a.ls[2] + t] = row_lse(m, sum);
}
// Rows r, r + step, .. of a unit from its splits' sums, [slot][row][128], scaled to the largest reference and added in
// the splits' order (a lane has the weights of splits lane, lane + 32, ..; the next row's are asked for ahead). A warp.
__device__ __noinline__ void join_rows(const Dims& dm, const AttendArgs& a, const AtUnit& x, int r, int step, int nrow) {
  const int lane = threadIdx.x & 31, nsp = x.nsp;
  const uint32_t s0 = 2 * x.first;
  const auto at = [&](int j) { return (int64_t)((s0 + 2 * j - (j > 0 ? 1 : 0)) * a.srows); };
  const auto ml = [&](int j, int row) {
    return j < nsp && row < nrow ? __ldcg((const float2*)a.mlpart + at(j) + row) : make_float2(-INFINITY, 0.f);
  };
  float2 next = ml(lane, r);
#pragma unroll 1
  for (; r < nrow; r += step) {
    float2 w = next;
    next = ml(lane, r + step);
    float m = w.x;
    for (int j = lane + 32; j < nsp; j += 32) m = fmaxf(m, ml(j, r).x);
    m = warp_max(m);
    float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
    float sum = 0.f;
#pragma unroll 1
    for (int j0 = 0; j0 < nsp; j0 += 32) {
      if (j0 > 0) w = ml(j0 + lane, r);
      // (a split that saw nothing has the reference -inf and the sum 0, one of NaN only -inf and NaN)
      const float f = w.x == m ? (w.x == -INFINITY && w.y == 0.f ? 0.f : 1.f) : ex2(w.x - m);
      const float fo = fmaxf(f, 0x1p-149f);  // (what is not finite stays so, whatever its split's weight)
      float z = w.y * f;
#pragma unroll
      for (int off = 16; off >= 1; off >>= 1) z += __shfl_xor_sync(0xffffffffu, z, off);
      sum += z;
      const int n = nsp - j0 < 32 ? nsp - j0 : 32;
#pragma unroll 4
      for (int j = 0; j < n; ++j) {
        const float4 v = __ldcg((const float4*)(a.opart + (at(j0 + j) + r) * D) + lane);
        const float fj = __shfl_sync(0xffffffffu, fo, j);
        y.x = fmaf(v.x, fj, y.x), y.y = fmaf(v.y, fj, y.y), y.z = fmaf(v.z, fj, y.z), y.w = fmaf(v.w, fj, y.w);
      }
    }
    const int row = x.r0 + r, h = row_head(dm.window, a.tdiv, row), t = row - h * dm.window;
    put_row(dm, a, x.s, x.l, x.g * dm.G + h, t, t < x.rows, y, m, sum, lane);
  }
}

// mbar_wait with few instructions between two looks (which the hardware holds back for a while by itself): the warps
// that wait share the issue slots with those that do not.
__device__ __forceinline__ bool wait_for(uint32_t bar, uint32_t parity, uint32_t* status, volatile int* abort) {
  if (mbar_try_wait(bar, parity)) return true;
  const unsigned long long t0 = globaltimer();
  for (;;) {
#pragma unroll 1
    for (int i = 0; i < 64; ++i)
      if (mbar_try_wait(bar, parity)) return true;
    if (abort != nullptr && *abort) return false;
    if (globaltimer() - t0 > WAIT_LIMIT_NS) {
      atomicOr(status, (uint32_t)ST_TIMEOUT);
      if (abort != nullptr) *abort = 1;
      return false;
    }
  }
}

// What such blocks of the item add to rows c0 .. c0 + 3 (of `nrow`), one channel (that of the thread) each. All of
// the group's 128 threads: two rows' logits of a token each, then the sums over the block's tokens. An infinite value
// is added as it is, whatever its weight.
__device__ __forceinline__ float4 far_values(const Dims& dm, const AttendArgs& a, const ByteScales& sc, const AtUnit& x,
                                          int c0, int nrow, const float2* norm, float (*w)[64], int bar, int tok) {
  const int64_t scales = x.l * sc.strides[0] + x.g * sc.strides[1] + x.s * sc.strides[2];
  const int64_t slot = x.l * sc.row_strides[0] + x.g * sc.row_strides[1] + x.s * sc.row_strides[2];
  float y[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 1
  for (int b = x.tok0 / 64; b * 64 < x.tok1; ++b) {
    const float vs = __ldg(sc.vs + scales + b);
    if (!is_far(vs)) continue;
    const float scale = sc.scale2 * __ldg(sc.ks + scales + b);
    const int live = min(64, x.tok1 - b * 64), j = tok & 63;
    const int64_t at = slot + (int64_t)b * 64 * D;
#pragma unroll 1
    for (int e = (tok >> 6) * 2; e < (tok >> 6) * 2 + 2; ++e) {
      const int row = x.r0 + c0 + e, h = row_head(dm.window, a.tdiv, row), t = row - h * dm.window;
      float p = 0.f;
      if (j < live && c0 + e < nrow && t < x.rows) {
        const uint4* k = (const uint4*)(sc.k + at + j * D);
        const uint4* q = (const uint4*)((const __nv_bfloat16*)a.q + x.s * dm.q_ss + x.l * dm.q_sl +
                                        (int64_t)(x.g * dm.G + h) * dm.q_sh + t * dm.q_sp);
        float dot = 0.f;
#pragma unroll 1
        for (int c = 0; c < D / 16; ++c) {
          const uint4 kw = __ldg(k + c), q0 = __ldg(q + 2 * c), q1 = __ldg(q + 2 * c + 1);
          const uint32_t kk[4] = {kw.x, kw.y, kw.z, kw.w}, qq[8] = {q0.x, q0.y, q0.z, q0.w, q1.x, q1.y, q1.z, q1.w};
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const float2 two = e4m3_values(kk[i >> 1] >> (16 * (i & 1)) & 0xffffu);
            dot = fmaf(bf16hi(qq[i]), two.y, fmaf(bf16lo(qq[i]), two.x, dot));
          }
        }
        p = ex2(fmaf(dot, scale, -norm[c0 + e].x)) * norm[c0 + e].y;
      }
      w[e][j] = p;
    }
    named_barrier_sync(bar, 128);
#pragma unroll 4
    for (int i = 0; i < live; ++i) {
      const float v = vs * e4m3_values(__ldg(sc.v + at + i * D + tok)).x;
#pragma unroll
      for (int e = 0; e < 4; ++e) y[e] += isinf(v) ? v : w[e][i] * v;
    }
    named_barrier_sync(bar, 128);
  }
  return make_float4(y[0], y[1], y[2], y[3]);
}

// Such a block's rows of V's tile (place n of the ring) are zeros to the tensor cores: a warp's 32. False: the wait
// failed.
template <int N>
__device__ __noinline__ bool drop_far(AbSmem<N>& sh, uint8_t* ring, uint32_t n, int quarter, int lane, uint32_t* status) {
  constexpr int RING = AbCfg<N>::RING;
  if (lane == 0) sh.any_far = 1;
  const bool ok = wait_for(smem_u32(&sh.full[n % RING]), (n / RING) & 1, status, &sh.abort);
#pragma unroll 1
  for (int e = lane; e < 32 * 8; e += 32)
    ((uint4*)(ring + n % RING * AB_TILE))[quarter * 32 * 8 + e] = make_uint4(0, 0, 0, 0);
  return ok;
}

// An item with such blocks, whose first tile was team `one`'s: what both teams have of a row, normalised, and the far
// values come to be that team's sums, with a factor of 1, and the other's have one of 0. All threads of the softmax
// groups.
template <int N>
__device__ __noinline__ void add_far(const Dims& dm, const AttendArgs& a, const ByteScales& sc, AbSmem<N>& sh, uint32_t k,
                                     int one) {
  const int warp = threadIdx.x >> 5, gi = (warp - 2) >> 2, tok = (warp & 3) * 32 + (threadIdx.x & 31);
  const AtUnit& x = sh.queue[k % AB_QUEUE];
  const int nrow = min(dm.G * dm.window - x.r0, N), r = threadIdx.x - 64;
  if (x.nsp > 1) {
    // A split's reference may be 2^40 below a weight of an earlier tile: the large values want its sum between 1 and 2.
    if (r < nrow) {  // (the thread has written them)
      float2* ml = (float2*)a.mlpart + (int64_t)at_slot<__nv_bfloat16>(a, x, x.split) * a.srows + r;
      const float2 z = *ml;
      if (z.y > 0.f && z.y < INFINITY) {
        const int e = min((int)(__float_as_uint(z.y) >> 23) - 127, 126);
        const float by = __uint_as_float((uint32_t)(127 - e) << 23);
        *ml = make_float2(z.x + (float)e, z.y * by);
        sh.norm[r].x = z.x + (float)e;
        sh.inv[0][r] *= by, sh.inv[1][r] *= by;
      }
    }
    named_barrier_sync(1, 128 * AbCfg<N>::GROUPS);
  }
  const uint32_t o0 = sh.tmem + AB_SBUF * N + ((uint32_t)((warp & 3) * 32) << 16);
#pragma unroll 1
  for (int c0 = 4 * gi; c0 < nrow; c0 += 4 * AbCfg<N>::GROUPS) {
    const float4 far = far_values(dm, a, sc, x, c0, nrow, sh.norm, sh.far[gi], 3 + gi, tok);
    float v[4], w[4] = {0.f, 0.f, 0.f, 0.f};
    tmem_ld_cols(o0 + N * one + c0, v);
    if (x.nt > 1) tmem_ld_cols(o0 + N * (one ^ 1) + c0, w);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      v[e] = fmaf(w[e], sh.inv[one ^ 1][c0 + e], v[e] * sh.inv[one][c0 + e]);
      v[e] += e == 0 ? far.x : (e == 1 ? far.y : (e == 2 ? far.z : far.w));
      w[e] = 0.f;
    }
    tmem_st_cols(o0 + N * one + c0, v);
    if (x.nt > 1) tmem_st_cols(o0 + N * (one ^ 1) + c0, w);
    named_barrier_sync(3 + gi, 128);  // the factors are read
    if (tok < 4) sh.inv[one][c0 + tok] = 1.f, sh.inv[one ^ 1][c0 + tok] = 0.f;
  }
  tmem_wait_st();
  named_barrier_sync(3 + gi, 128);
}

struct AbCost {
  static constexpr uint32_t UNIT = 1;
  __device__ __forceinline__ uint32_t operator()(int) const { return 1u; }
};
constexpr uint32_t AB_START = 2;  // tiles' time of a unit's start

template <int N>
__global__ void __launch_bounds__(AbCfg<N>::THREADS, AbCfg<N>::PER_SM)
    attend_bytes_kernel(const __grid_constant__ CUtensorMap kmap, const __grid_constant__ CUtensorMap vmap,
                        const __grid_constant__ CUtensorMap kdmap, const __grid_constant__ CUtensorMap vdmap,
                        const __grid_constant__ Dims dm,
                        const __grid_constant__ AttendArgs a, const __grid_constant__ ByteScales sc) {
  using C = AbCfg<N>;
  constexpr int RING = C::RING, PART = C::PART;
  constexpr int TURNS = AB_TURNS, SBUF = AB_SBUF, GR = C::GR, CG = C::CG;
  constexpr int LOAD0 = C::LOAD0, LOADERS = C::LOADERS, WBUF = C::WBUF;
  constexpr uint32_t AB_O = SBUF * N;  // columns: S of tile i at N (i % SBUF), O from here on (N for each turn)
  constexpr int SM_THREADS = 128 * C::GROUPS;
  // (there are no static variables, so that it starts on the 1024 bytes that the swizzle needs)
  extern __shared__ __align__(1024) uint8_t smem[];
  uint8_t* ring = smem;                // (a drafted tile's product reads 8 KB on: the rows' space behind the last)
  uint8_t* q8 = ring + RING * AB_TILE;  // rows: hi, lo [N][128] bytes, K-major with the 128-byte swizzle
  uint8_t* qb = q8 + 2 * PART;          // and bf16, for drafted tokens: [2][N][64]
  uint8_t* ps = qb + 2 * PART;          // a team's weights: [128 tokens][hi, lo][N] bytes; drafted: bf16 [N][64 tokens]
  AbSmem<N>& sh = *(AbSmem<N>*)(ps + 2 * WBUF);
  static_assert(4 * PART + 2 * WBUF + sizeof(AbSmem<N>) >= 8192, "what a drafted tile's product reads behind the ring");

  // (numbers that are a warp's own, and known to be: the tensor instructions take their operands from uniform
  // registers)
  const auto uniform = [](int x) { return __reduce_max_sync(0xffffffffu, x); };
  const int tid = threadIdx.x, warp = uniform(tid >> 5), lane = tid & 31;
  const int R = dm.G * dm.window;
  if ((smem_u32(smem) & 1023u) != 0) {
    pdl_wait();
    if (tid == 0) atomicOr(a.status, (uint32_t)ST_INVALID);
    return;
  }
  if (tid == 0) {
    sh.abort = sh.any_far = 0;
    sh.bad[0] = sh.bad[1] = 0;
    for (int i = 0; i < RING; ++i) {
      mbar_init(smem_u32(&sh.full[i]), 1);
      mbar_init(smem_u32(&sh.empty[i]), 1);
    }
    for (int i = 0; i < SBUF; ++i) mbar_init(smem_u32(&sh.sfull[i]), 1);
    for (int i = 0; i < 2; ++i) {
      mbar_init(smem_u32(&sh.pready[i]), 4 * CG);
      mbar_init(smem_u32(&sh.pvdone[i]), 1);
    }
    for (int i = 0; i < AB_QUEUE; ++i) {
      mbar_init(smem_u32(&sh.qfull[i]), 1);
      mbar_init(smem_u32(&sh.qempty[i]), 1 + 4 * C::GROUPS + LOADERS);  // MMA, softmax and row warps
    }
    mbar_init(smem_u32(&sh.rowsready), LOADERS);
    mbar_init(smem_u32(&sh.rowsasked), LOADERS);
    mbar_init(smem_u32(&sh.rowsfree), 1);
    mbar_init(smem_u32(&sh.ofree), 4 * C::GROUPS);
    mbar_init(smem_u32(&sh.drained), 1);
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
  const uint32_t tmem = (uint32_t)uniform((int)sh.tmem);
  volatile int* abort = &sh.abort;
  // Item `k` of this CTA is there, as the producer published it, and is not the end. The warp (or thread) is done with
  // it when it says so.
  auto ready = [&](uint32_t k) {
    const uint32_t bar = smem_u32(&sh.qfull[k % AB_QUEUE]), parity = (k / AB_QUEUE) & 1;
    return wait_for(bar, parity, a.status, abort) &&
           sh.queue[k % AB_QUEUE].nt >= 0;
  };
  auto done = [&](uint32_t k) { mbar_arrive(smem_u32(&sh.qempty[k % AB_QUEUE])); };

  // An item's loads come as they are used: K of its first two tiles, then K of tile i + 2 and V of tile i. The place of
  // V of tile i of nt among them:
  const auto place_v = [&](int i, int nt) { return i < nt - TURNS ? TURNS + 2 * i + 1 : nt + i; };

  if (warp == 0) {
    // ------------------------------------------------ TMA producer --------
    AtShares<AB_TOK, AB_START, AbCost> share(dm, a, nullptr, AbCost{}, lane);
    if (lane == 0) {
      uint32_t published = 0, st = 0, pass = 0;  // items; the ring's place, and how often it was filled
      AtUnit x, next;
      bool ok = true, first = true;
      // Item x; the item after it is published a few loads later, so that its rows are on their way long before they
      // are needed. (One place for each step, as a CTA runs most of its instructions for the first time.)
      for (int tk = 0, tv = 0, end = 0, when = 0; ok;) {  // next tile of K and of V, tiles
        if (tk + tv == when) {
          share.next(next, N);
          const int q = published % AB_QUEUE;
          if (published >= AB_QUEUE && !wait_for(smem_u32(&sh.qempty[q]), ((published / AB_QUEUE) & 1) ^ 1, a.status, abort))
            break;
          sh.queue[q] = next;
          mbar_arrive(smem_u32(&sh.qfull[q]));
          ++published;
          when = -1;
        }
        if (tv == end) {
          x = next;
          if (x.nt < 0) break;
          tk = tv = 0, end = x.nt, when = end < 2 ? 2 * end : 4;
          continue;
        }
        if (pass > 0) ok = wait_for(smem_u32(&sh.empty[st]), (pass & 1) ^ 1, a.status, abort);
        // the first rows are asked for before all but a first tile, which would be ahead of them in memory's queues
        else if (st == 1) ok = wait_for(smem_u32(&sh.rowsasked), 0, a.status, abort);
        if (!ok) break;
        const bool of_k = tk < end && tk <= tv + TURNS;
        const int tile = of_k ? tk++ : tv++;
        const uint32_t dst = smem_u32(ring) + st * AB_TILE, bar = smem_u32(&sh.full[st]);
        mbar_arrive_expect_tx(bar, AB_TILE);
        if (tile < x.ncache) {
          tma_load_5d(dst, of_k ? &kmap : &vmap, 0, x.tok0 + tile * AB_TOK, x.s, x.g, x.l, bar);
        } else {
          const CUtensorMap* map = of_k ? &kdmap : &vdmap;
          tma_load_5d(dst, map, 0, 0, x.g, x.l, x.s, bar);
          tma_load_5d(dst + AB_TILE / 2, map, 64, 0, x.g, x.l, x.s, bar);
        }
        first = false;
        if (++st == RING) st = 0, ++pass;
      }
      // what is under way lands before the CTA leaves
      for (int k = 0; !first && k < RING; ++k) {
        if (st == 0) st = RING, --pass;
        --st;
        wait_for(smem_u32(&sh.full[st]), pass & 1, a.status, nullptr);
        if (st == 0 && pass == 0) break;
      }
    }
  } else if (warp == 1) {
    // ------------------------------------------------ MMA issuer ---------- (All lanes go through it, so that what
    // they compute is uniform; one issues, some 70 cycles a product whatever N is. Both parts of the weights in one
    // product of twice the columns, and of the rows with 32, gained nothing: an issue that ends sooner waits longer
    // for the weights.)
    const bool leader = elect_one();
    constexpr uint32_t IDESC_S[2] = {idesc_e4m3_f32(128, N, 0, 0, false), idesc_e4m3_f32(128, N, 0, 0, true)};  // hi, lo
    constexpr uint32_t IDESC_O[2] = {idesc_e4m3_f32(128, N, 1, 1, false), idesc_e4m3_f32(128, N, 1, 1, true)};
    constexpr uint32_t IDESC_SD = idesc_bf16_f32(128, N, 0, 0), IDESC_OD = idesc_bf16_f32(128, N, 1, 0);
    const uint64_t qd = smem_desc_sw128(smem_u32(q8), 16, 1024), qbd = smem_desc_sw128(smem_u32(qb), 16, 1024);
    const uint64_t pd = weight_desc<N>(smem_u32(ps)), pbd = smem_desc_sw128(smem_u32(ps), 16, 1024);
    const uint64_t kd0 = smem_desc_sw128(smem_u32(ring), 16, 1024), vd0 = smem_desc_sw128(smem_u32(ring), AB_TILE / 2, 1024);
    uint32_t it = 0, busy = 0, st = 0, pass = 0;  // tiles before the item, items with tiles; the ring's place and filling
    bool ok = true;
    const auto landed = [&]() {
      const bool there = wait_for(smem_u32(&sh.full[st]), pass & 1, a.status, abort);
      tc_fence_after();
      return there;
    };
    const auto used = [&]() {
      if (leader) umma_commit(smem_u32(&sh.empty[st]));
      if (++st == RING) st = 0, ++pass;
    };
    for (uint32_t k = 0; ok && ready(k); ++k) {
      const AtUnit& x = sh.queue[k % AB_QUEUE];
      const int nt = uniform(x.nt), ncache = uniform(x.ncache);
      __syncwarp();
      if (leader) done(k);
      if (nt == 0) continue;
      // the rows are there, which the row warps put down when the item before no longer needed the space
      if (!wait_for(smem_u32(&sh.rowsready), busy & 1, a.status, abort)) break;
      ++busy;
#pragma unroll 1
      for (int i = 0; ok && i < nt + TURNS; ++i) {
        if (i < nt) {
          // S^T = K Q^T of tile i goes where that of the tile SBUF before was, which was read before its product was
          // issued
          if (!(ok = landed())) break;
          const uint32_t b = (it + i) % SBUF, d = tmem + N * b;
          const uint64_t kd = kd0 + (uint64_t)(st * (AB_TILE >> 4));
          if (leader) {
            if (i >= ncache) {
#pragma unroll
              for (int c = 0; c < 8; ++c)
                umma_f16_ss(d, kd + (uint64_t)((c >> 2) * (AB_TILE / 2) + (c & 3) * 32 >> 4),
                            qbd + (uint64_t)((c >> 2) * PART + (c & 3) * 32 >> 4), IDESC_SD, c > 0 ? 1u : 0u);
            } else {
#pragma unroll
              for (int c = 0; c < 8; ++c)  // the rows' hi parts, then their lo parts
                umma_f8_ss(d, kd + (uint64_t)((c & 3) * 32 >> 4), qd + (uint64_t)((c >> 2) * PART + (c & 3) * 32 >> 4),
                           IDESC_S[c >> 2], c > 0 ? 1u : 0u);
            }
          }
          used();
          if (leader) {
            umma_commit(smem_u32(&sh.sfull[b]));
            if (i == nt - 1) umma_commit(smem_u32(&sh.rowsfree));  // the item's last use of its rows
          }
        }
        if (i >= TURNS) {
          // O^T (+)= V^T P^T of tile j
          const int j = i - TURNS;
          if (j >= nt) continue;
          const uint32_t t = it + j, b = t & 1, o = tmem + AB_O + N * b, w = b * WBUF;
          // (before the first one: the accumulators of the item before are read out)
          ok = (j > 0 || busy == 1 || wait_for(smem_u32(&sh.ofree), busy & 1, a.status, abort)) && landed() &&
               wait_for(smem_u32(&sh.pready[b]), (t >> 1) & 1, a.status, abort);
          if (!ok) break;
          tc_fence_after();
          const uint64_t vd = vd0 + (uint64_t)(st * (AB_TILE >> 4));
          const uint32_t more = j < TURNS ? 0u : 1u;
          if (leader) {
            if (j >= ncache) {
#pragma unroll
              for (int c = 0; c < 4; ++c)
                umma_f16_ss(o, vd + (uint64_t)(c * 2048 >> 4), pbd + (uint64_t)(w + c * 32 >> 4), IDESC_OD,
                            c > 0 ? 1u : more);
            } else {
#pragma unroll
              for (int c = 0; c < 8; ++c)  // the weights' hi parts, then their lo parts: 32 tokens each
                umma_f8_ss(o, vd + (uint64_t)((c & 3) * 4096 >> 4),
                           pd + (uint64_t)(w + (c >> 2) * N + (c & 3) * 64 * N >> 4), IDESC_O[c >> 2], c > 0 ? 1u : more);
            }
          }
          used();
          if (leader) umma_commit(smem_u32(&sh.pvdone[b]));
        }
      }
      it += nt;
    }
    // every MMA issued here completes before the CTA tears down tensor memory
    __syncwarp();
    if (leader) umma_commit(smem_u32(&sh.drained));
    wait_for(smem_u32(&sh.drained), 0, a.status, nullptr);
  } else if (warp >= LOAD0) {
    // ------------------ the rows as they are (for drafted tokens), then each scaled to e4m3's range and split
    const int e0 = (warp - LOAD0) * 32 + lane, c = e0 & 15;  // 16 bytes: channels 8 c .. + 7
    constexpr int STEP = 2 * LOADERS, PIECES = N / STEP;
    const uint32_t mine = smem_u32(qb) + (c >> 3) * PART;
    uint32_t busy = 0;
    for (uint32_t k = 0;; ++k) {
      const bool more = ready(k);
      if (named_barrier_any(2, 32 * LOADERS, !more && *abort != 0) || !more) break;  // (together; qmax is read)
      const AtUnit x = sh.queue[k % AB_QUEUE];
      __syncwarp();
      if (lane == 0) done(k);
      if (x.nt == 0) continue;
      const __nv_bfloat16* q =
          (const __nv_bfloat16*)a.q + x.s * dm.q_ss + x.l * dm.q_sl + (int64_t)x.g * dm.G * dm.q_sh;
      const auto piece = [&](int r, bool& on) {
        const int row = x.r0 + r, h = row_head(dm.window, a.tdiv, row), t = row - h * dm.window;
        on = row < R && t < x.rows;  // (a row behind the request's last may hold anything)
        return (const uint4*)(on ? q + h * dm.q_sh + t * dm.q_sp : q) + c;
      };
      bool on;
      // into L2 while the item before is at work
      for (int r = e0 >> 4; busy > 0 && r < min(N, R - x.r0); r += STEP) {
        const uint4* at = piece(r, on);
        if (on && (c & 7) == 0) asm volatile("prefetch.global.L2 [%0];" ::"l"(at));
      }
      // the item before's last tile has met its rows
      const bool ok = busy == 0 || wait_for(smem_u32(&sh.rowsfree), (busy - 1) & 1, a.status, abort);
      // (zeros behind the last row, as far as the softmax looks: CH rows at a time)
      constexpr int CH = N == 16 ? 8 : 16;
      const int pieces = min(PIECES, (R - x.r0 + CH - 1) / CH * (CH / STEP));
#pragma unroll 4
      for (int i = 0; i < pieces; ++i) {
        const int r = (e0 >> 4) + STEP * i;
        const uint4* at = piece(r, on);
        cp_async16(mine + sw128_off(r, c & 7), at, on);
      }
      cp_async_commit();
      if (busy == 0) {
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&sh.rowsasked));
      }
      cp_async_wait<0>();  // (a thread reads what it has copied itself)
      if (named_barrier_any(2, 32 * LOADERS, !ok)) break;
#pragma unroll 2
      for (int i = 0; i < pieces; ++i) {
        const int r = (e0 >> 4) + STEP * i;
        const uint4 w = lds_u128(mine + sw128_off(r, c & 7));
        const uint32_t u[4] = {w.x, w.y, w.z, w.w};
        float top = 0.f;  // the row's largest finite one: 16 lanes have it
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float lo = fabsf(bf16lo(u[j])), hi = fabsf(bf16hi(u[j]));
          if (lo < INFINITY) top = fmaxf(top, lo);
          if (hi < INFINITY) top = fmaxf(top, hi);
        }
#pragma unroll
        for (int off = 8; off >= 1; off >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, off));
        // the power of two that brings it to 224 .. 448
        int e = top == 0.f ? 127 : (int)(__float_as_uint(top) >> 23) - 8 + ((__float_as_uint(top) & 0x7fffffu) > 0x600000u);
        e = e < 1 ? 1 : e;
        const float by = __uint_as_float((uint32_t)(254 - e) << 23);
        if (c == 0) sh.qfac[k % AB_QUEUE][r] = sc.scale2 * __uint_as_float((uint32_t)e << 23);
        uint32_t hi[2], lo[2];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          float y[4] = {bf16lo(u[2 * j]) * by, bf16hi(u[2 * j]) * by, bf16lo(u[2 * j + 1]) * by, bf16hi(u[2 * j + 1]) * by};
#pragma unroll
          for (int k2 = 0; k2 < 4; ++k2) y[k2] = fabsf(y[k2]) < INFINITY ? y[k2] : NAN;
          split_f8(y[0], y[1], y[2], y[3], hi[j], lo[j]);
        }
        const uint32_t at = r * 128 + ((((uint32_t)c >> 1) ^ (r & 7)) << 4) + (c & 1) * 8;
        sts_u32s(smem_u32(q8) + at, hi);
        sts_u32s(smem_u32(q8) + PART + at, lo);
      }
      fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) mbar_arrive(smem_u32(&sh.rowsready));
      ++busy;
    }
  } else {
    // ------------------------------------------------ softmax -------------
    // group: four warps, which have the tensor memory's four quarters of lanes
    const int gi = (warp - 2) >> 2, team = gi / CG, cg = gi % CG, quarter = warp & 3, tok = quarter * 32 + lane;
    const int first = GR * cg, tsm = tid - 64;  // the group's first row
    const uint32_t bases = smem_u32(sh.base[warp - 2]), coefs = smem_u32(sh.coef[warp - 2]);
    // where the token's line of weights is, and its swizzle of the group's bytes in it (weight_off)
    const uint32_t line = smem_u32(ps) + team * WBUF + tok * (2 * N);
    const uint32_t swizzle = ((uint32_t)(tok * (2 * N)) >> 3 & (uint32_t)(2 * N - 16)) ^ (uint32_t)first;
    const uint32_t lanes = (uint32_t)(quarter * 32) << 16, ocol = tmem + AB_O + N * team + first + lanes;
    constexpr int CH = N == 16 ? 8 : 16;  // rows at a time
    constexpr bool KEEP = GR == 16;       // S stays in registers from the maxima to the weights
    const int mine = lane % GR;  // a lane keeps the reference of one of the group's rows
    uint32_t it0 = 0;  // tiles before this item
    bool ok = true;
    for (uint32_t k = 0; ok; ++k) {
      const bool more = ready(k);
      // (all warps decide together whether to go on: a wait may fail in one of them)
      if (named_barrier_any(1, SM_THREADS, !more && *abort != 0) || !more) break;
      const AtUnit& x = sh.queue[k % AB_QUEUE];  // (its members are read where they are needed, not kept in registers)
      int nrow = min(R - x.r0, N), nt = x.nt;
      const int ncache = x.ncache;
      if (nt == 0) {  // nothing to see
        for (int r = warp - 2; r < nrow; r += 4 * C::GROUPS) {
          const int row = x.r0 + r, h = row_head(dm.window, a.tdiv, row), t = row - h * dm.window;
          put_row(dm, a, x.s, x.l, x.g * dm.G + h, t, t < x.rows, make_float4(0.f, 0.f, 0.f, 0.f), -INFINITY, 0.f, lane);
        }
        __syncwarp();
        if (lane == 0) done(k);
        continue;
      }
      if (nt > ncache) {
        if (tsm < N) sh.rowmask[tsm] = x.r0 + tsm < R ? at_mask(dm, a, x, (x.r0 + tsm) % dm.window) : 0;
        named_barrier_sync(1, SM_THREADS);
      }
      const float* ksp = sc.ks + x.l * sc.strides[0] + x.g * sc.strides[1] + x.s * sc.strides[2];
      const float* vsp = sc.vs + x.l * sc.strides[0] + x.g * sc.strides[1] + x.s * sc.strides[2];
      // tile i is this group's; the block of its warp's tokens, if it holds any
      const int i_first = (int)((it0 ^ team) & 1), block0 = (x.tok0 + quarter * 32) / 64, blocks = (x.n + 63) / 64;
      const int nlive = x.tok1 - x.tok0;
      const auto block = [&](int i) { return block0 + i * (AB_TOK / 64); };
      float ref = -INFINITY, deep = -INFINITY;  // of row `mine`: the reference, and the least that it goes down to
      float2 z[GR / 2];                         // the lane's sums
#pragma unroll
      for (int r = 0; r < GR / 2; ++r) z[r] = make_float2(0.f, 0.f);
      const bool active = first < nrow;  // (a group without rows passes the tiles on)
      float qfac = 0.f, ks_next = 0.f, vs_next = 0.f, lv = AB_UNIT;  // lv: log2 of V's scale (far ones and 0 keep the one before)
      if (i_first < ncache && block(i_first) < blocks)
        ks_next = __ldg(ksp + block(i_first)), vs_next = __ldg(vsp + block(i_first));
#pragma unroll 1
      for (int i = i_first; i < nt; i += TURNS) {
        const uint32_t it = it0 + i, b = it & 1, sb = it % SBUF;
        const bool drafted = i >= ncache;
        const float ks = ks_next;
        const bool far = is_far(vs_next);
        if (vs_next > 0.f && !far) lv = log2_scale(vs_next);
        if (i + TURNS < ncache && block(i + TURNS) < blocks)
          ks_next = __ldg(ksp + block(i + TURNS)), vs_next = __ldg(vsp + block(i + TURNS));
        // One warp looks, the others are held by the barrier (the looks of all took a third of the issue slots). A wait
        // that failed in one warp is known to its group here, and to all at the item's end.
        if (quarter == 0) ok = ok && wait_for(smem_u32(&sh.sfull[sb]), (it / SBUF) & 1, a.status, abort);
        if (named_barrier_any(3 + gi, 128, !ok)) {
          ok = false;
          break;
        }
        tc_fence_after();
        // (not before: with this tile's S the place's filling before V of it, at most that of its K, has been used)
        if (far && !drafted) ok = drop_far<N>(sh, ring, 2 * it0 + place_v(i, nt), quarter, lane, a.status);
        const int nv = drafted ? x.nd : min(AB_TOK, nlive - i * AB_TOK);  // rows of the tile that hold tokens
        if (i < TURNS) qfac = sh.qfac[k % AB_QUEUE][first + mine];  // (there with the first product)
        const float c = drafted ? sc.scale2 : qfac * ks;            // of row `mine`
        const float w_lv = drafted ? 0.f : lv;  // (drafted weights are bf16, and V as it is)
        const uint32_t scol = tmem + N * sb + first + lanes, tops = smem_u32(&sh.top[b][first + mine]);
        const bool seen = tok < nv, part = drafted || nv < AB_TOK;
        const auto sees = [&](int r) { return seen && (!drafted || (sh.rowmask[first + r] >> (tok & 63) & 1) != 0); };
        if (!active && i >= TURNS)  // (not two arrivals for one tile: the products of S are ahead of those of V)
          ok = ok && wait_for(smem_u32(&sh.pvdone[b]), ((it - TURNS) >> 1) & 1, a.status, abort);
        if (active) {
          // the warp's maxima of what the rows see, to its lanes, which scale them and meet those of the other warps
          float s[GR];
          tmem_ld_cols(scol, s);
          if (part) {
#pragma unroll
            for (int e = 0; e < GR; ++e) s[e] = sees(e) ? s[e] : -INFINITY;
          }
#pragma unroll
          for (int c0 = 0; c0 < GR; c0 += CH) {
            if (c0 > 0 && first + c0 >= nrow) break;
            float v[CH];
#pragma unroll
            for (int e = 0; e < CH; ++e) v[e] = warp_max(s[c0 + e]);
            if (lane == 0) {
#pragma unroll
              for (int e = 0; e < CH; e += 4)
                asm volatile("st.shared.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(bases + (c0 + e) * 4), "f"(v[e]), "f"(v[e + 1]),
                             "f"(v[e + 2]), "f"(v[e + 3]) : "memory");
            }
          }
          __syncwarp();
          {
            const float y = lds_f32(bases + mine * 4);
            if (lane < GR) sts_f32(tops + quarter * 4, y == -INFINITY ? y : fmaf(y, c, drafted ? AB_UNIT : lv));
          }
          named_barrier_sync(3 + gi, 128);
          const float4 top4 = lds_f32x4(tops);
          const float top = fmaxf(fmaxf(top4.x, top4.y), fmaxf(top4.z, top4.w));
          const bool wide = top > fminf(fminf(top4.x, top4.y), fminf(top4.z, top4.w)) + AB_WIDE;
          float f = 1.f;
          if (top > ref + AB_HIGH || top < ref + (wide ? AB_WIDE_LOW : AB_LOW)) {
            const float to = fmaxf(top - (wide ? AB_WIDE_TOP : AB_TOP), deep);
            if (top > -INFINITY && to != ref) {
              f = ref == -INFINITY ? 0.f : ex2(ref - to);
              ref = to;
              deep = fmaxf(deep, to - AB_DEEP);
            }
          }
          if (lane < GR) {
            sts_f32(bases + lane * 4, ref == -INFINITY ? 0.f : w_lv - ref);
            sts_f32(coefs + lane * 4, c);
          }
          __syncwarp();
          // the tile before's weights are read (and its sums in the accumulators, should they be rescaled)
          if (i >= TURNS) {
            ok = wait_for(smem_u32(&sh.pvdone[b]), ((it - TURNS) >> 1) & 1, a.status, abort) && ok;
            tc_fence_after();
            if (__any_sync(0xffffffffu, f != 1.f)) {  // (the same in all warps of the group)
#pragma unroll
              for (int c0 = 0; c0 < GR; c0 += CH) {
                if (c0 > 0 && first + c0 >= nrow) break;
                float v[CH];
                tmem_ld_cols(ocol + c0, v);
#pragma unroll
                for (int e = 0; e < CH; e += 2) {
                  const float f0 = __shfl_sync(0xffffffffu, f, c0 + e), f1 = __shfl_sync(0xffffffffu, f, c0 + e + 1);
                  v[e] *= f0, v[e + 1] *= f1;
                  float2& zr = z[(c0 + e) / 2];
                  zr.x *= f0, zr.y *= f1;
                }
                tmem_st_cols(ocol + c0, v);
              }
              tmem_wait_st();
            }
          }
          // The weights, and the lane's sums of what they are of Z.
          const float iv1 = ex2(AB_UNIT - w_lv);
          const float2 iv = make_float2(iv1, iv1);
#pragma unroll
          for (int c0 = 0; c0 < GR; c0 += CH) {
            if (c0 > 0 && first + c0 >= nrow) break;
            float s1[CH];
            if constexpr (KEEP) {
#pragma unroll
              for (int e = 0; e < CH; ++e) s1[e] = s[c0 + e];
            } else {
              tmem_ld_cols(scol + c0, s1);
            }
            float2 v[CH / 2];
#pragma unroll
            for (int e = 0; e < CH / 2; e += 2) {
              const float4 bs = lds_f32x4(bases + (c0 + 2 * e) * 4), cs = lds_f32x4(coefs + (c0 + 2 * e) * 4);
              v[e] = fma2(make_float2(s1[2 * e], s1[2 * e + 1]), make_float2(cs.x, cs.y), make_float2(bs.x, bs.y));
              v[e + 1] = fma2(make_float2(s1[2 * e + 2], s1[2 * e + 3]), make_float2(cs.z, cs.w), make_float2(bs.z, bs.w));
            }
#pragma unroll
            for (int e = 0; e < CH / 2; ++e) v[e] = make_float2(ex2(v[e].x), ex2(v[e].y));
            if (part) {
#pragma unroll
              for (int e = 0; e < CH / 2; ++e)
                v[e].x = sees(c0 + 2 * e) ? v[e].x : 0.f, v[e].y = sees(c0 + 2 * e + 1) ? v[e].y : 0.f;
            }
#pragma unroll
            for (int e = 0; e < CH / 2; ++e) {
              z[c0 / 2 + e] = fma2(v[e], iv, z[c0 / 2 + e]);
            }
            const int r0 = first + c0;
            if (!drafted) {
              uint32_t hi[CH / 4], lo[CH / 4];
#pragma unroll
              for (int e = 0; e < CH / 4; ++e)
                split_f8(v[2 * e].x, v[2 * e].y, v[2 * e + 1].x, v[2 * e + 1].y, hi[e], lo[e]);
              sts_u32s(line + (swizzle ^ (c0 & ~15)) + (c0 & 15), hi);
              sts_u32s(line + (swizzle ^ (N | (c0 & ~15))) + (c0 & 15), lo);
            } else if (tok < 64) {
#pragma unroll
              for (int e = 0; e < CH; ++e)
                *(__nv_bfloat16*)(ps + team * WBUF + sw128_off(r0 + e, tok >> 3) + (tok & 7) * 2) =
                    __float2bfloat16(e & 1 ? v[e / 2].y : v[e / 2].x);
            }
          }
        }
        if (part) {
          const uint32_t n = 2 * it0 + place_v(i, nt);
          ok = ok && wait_for(smem_u32(&sh.full[n % RING]), (n / RING) & 1, a.status, abort);
          uint8_t* vt = ring + n % RING * AB_TILE;
          constexpr int TEAM = 128 * CG;  // threads that have the tile
          const int mate = cg * 128 + tok;
          if (!drafted) {  // rows past the live tokens: 0 times what they hold may be NaN
#pragma unroll 1
            for (int e = mate + nv * 8; e < AB_TOK * 8; e += TEAM) ((uint4*)vt)[e] = make_uint4(0, 0, 0, 0);
          } else {
#pragma unroll 1
            for (int e = mate; e < 64 * 16; e += TEAM) {
              const int t = e >> 4, c16 = e & 15;
              uint4* at = (uint4*)(vt + (c16 >> 3) * (AB_TILE / 2) + sw128_off(t, c16 & 7));
              if (t >= nv) {
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
                atomicOr(&sh.bad[t >> 5], 1u << (t & 31));
              }
            }
          }
        }
        fence_proxy_async_smem();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&sh.pready[b]));
      }
      // the item's last products are done, of both turns
      it0 += nt;
      for (uint32_t t = nt > 1 ? it0 - 2 : it0 - 1; t != it0; ++t)
        ok = ok && wait_for(smem_u32(&sh.pvdone[t & 1]), (t >> 1) & 1, a.status, abort);
      // the rows' sums over the warps
      float zs[GR];
#pragma unroll
      for (int r = 0; r < GR; ++r) zs[r] = r & 1 ? z[r / 2].y : z[r / 2].x;
      const float zsum = lane_sums<GR>(zs, lane);
      if (lane < GR) {
        sh.sum[team][quarter][first + lane] = zsum;
        if (quarter == 0) sh.ref[team][first + lane] = ref;
      }
      // all warps meet here whether or not a wait failed, and leave together if one did
      if (named_barrier_any(1, SM_THREADS, !ok)) break;
      tc_fence_after();
      const auto slot = [&]() { return (int64_t)at_slot<__nv_bfloat16>(a, x, x.split) * a.srows; };
      if (tsm < nrow) {
        const int r = tsm, row = x.r0 + r, h = row_head(dm.window, a.tdiv, row), t = row - h * dm.window;
        float m = fmaxf(sh.ref[0][r], sh.ref[1][r]), sum = 0.f, share[TURNS];
#pragma unroll
        for (int j = 0; j < TURNS; ++j) {
          share[j] = sh.ref[j][r] == m ? 1.f : ex2(sh.ref[j][r] - m);
          sum += ((sh.sum[j][0][r] + sh.sum[j][1][r]) + (sh.sum[j][2][r] + sh.sum[j][3][r])) * share[j];
        }
        const float unit = ex2(AB_UNIT) * (x.nsp > 1 ? 1.f : (sum == 0.f ? 0.f : 1.f / sum));
#pragma unroll
        for (int j = 0; j < TURNS; ++j) sh.inv[j][r] = share[j] * unit;
        if (m > -INFINITY) m -= AB_UNIT;
        sh.norm[r] = make_float2(m, x.nsp > 1 ? 1.f : (sum == 0.f ? 0.f : 1.f / sum));
        if (x.nsp > 1) ((float2*)a.mlpart)[slot() + r] = make_float2(m, sum);
        else if (t < x.rows && a.lse != nullptr)
          a.lse[x.s * a.ls[0] + x.l * a.ls[1] + (x.g * dm.G + h) * a.ls[2] + t] = row_lse(m, sum);
      }
      named_barrier_sync(1, SM_THREADS);
      if (sh.any_far != 0) add_far<N>(dm, a, sc, sh, k, (int)((it0 - x.nt) & 1));
      nrow = min(R - x.r0, N), nt = x.nt;
      const bool parts = x.nsp > 1;
      // a lane has one channel of some rows, four at a time (few instructions: a CTA comes here once or twice)
      const uint64_t bad = (uint64_t)sh.bad[1] << 32 | sh.bad[0];
      const uint32_t o0 = tmem + AB_O + lanes;
      __nv_bfloat16* o = (__nv_bfloat16*)a.o + x.s * a.os[0] + x.l * a.os[1] + (int64_t)x.g * dm.G * a.os[2] + tok;
      const __nv_bfloat16* vd = (const __nv_bfloat16*)a.vd + x.s * a.vds[0] + x.l * a.vds[1] + x.g * a.vds[2] + tok;
      float* po = parts ? a.opart + slot() * D + tok : nullptr;
      const bool both = nt > 1;
      const int one = (int)((it0 - nt) & 1), rows = x.rows, row0 = x.r0;  // the first tile's team
#pragma unroll 1
      for (int c0 = 4 * gi; c0 < nrow; c0 += 4 * C::GROUPS) {
        float v[4], w[4] = {0.f, 0.f, 0.f, 0.f};
        tmem_ld_cols(o0 + N * one + c0, v);
        if (both) tmem_ld_cols(o0 + N * (one ^ 1) + c0, w);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int r = c0 + e, row = row0 + r, h = row_head(dm.window, a.tdiv, row), t = row - h * dm.window;
          if (r >= nrow || t >= rows) continue;
          float y = v[e] * sh.inv[one][r];
          if (both) y = fmaf(w[e], sh.inv[one ^ 1][r], y);
          if (bad != 0) y += bad_values(vd, a.vds[3], bad & sh.rowmask[r]);
          if (parts) po[r * D] = y;
          else o[h * a.os[2] + t * a.os[3]] = __float2bfloat16(y);
        }
      }
      tc_fence_before();
      if (parts) {  // the CTA that finishes the unit's last split joins them all
        __threadfence();
        named_barrier_sync(1, SM_THREADS);
        if (tsm == 0) {
          // (a CTA has the first split of one unit of several at most: the one that its end divides)
          sh.last = atomicAdd(a.counts + x.first, 1) == x.nsp - 1;
          if (sh.last) a.counts[x.first] = 0;  // (zero between calls)
          __threadfence();
        }
        named_barrier_sync(1, SM_THREADS);
        if (sh.last) join_rows(dm, a, x, warp - 2, 4 * C::GROUPS, nrow);
      }
      named_barrier_sync(1, SM_THREADS);  // the masks, sums and bits are read, and the item
      if (bad != 0 && tsm == 0) sh.bad[0] = sh.bad[1] = 0;
      if (tsm == 0) sh.any_far = 0;
      if (lane == 0) mbar_arrive(smem_u32(&sh.ofree)), done(k);
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc(tmem, C::COLS);
  }
}

template <int N>
static cudaError_t launch_n(const CUtensorMap* maps, const Dims& dm, const AttendArgs& a, const ByteScales& sc, int sms,
                            cudaStream_t st) {
  auto kern = attend_bytes_kernel<N>;
  JACAP_TRY(cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)ab_smem<N>()));
  const int64_t items = (int64_t)dm.L * dm.Hkv * dm.S * a.nsplit * a.nrb;
  const int places = min(AbCfg<N>::PER_SM * sms, attend_bytes_ctas(N));
  return launch_pdl(true, kern, (int)(items < places ? items : places), AbCfg<N>::THREADS, ab_smem<N>(), st, maps[0],
                    maps[1], maps[2], maps[3], dm, a, sc);
}

int attend_bytes_block(int rows) { return rows <= 16 ? 16 : (rows <= 32 ? 32 : 64); }
// (so many have slots for their splits' sums: two CTAs of 16 rows run on an SM, one of more)
int attend_bytes_ctas(int block) { return block == 16 ? ATTEND_CTAS : ATTEND_CTAS / 2; }
static_assert(AbCfg<16>::PER_SM == 2 && AbCfg<32>::PER_SM == 1 && AbCfg<64>::PER_SM == 1, "attend_bytes_ctas");

cudaError_t launch_attend_bytes(const CUtensorMap* maps, const Dims& dm, const AttendArgs& a, const ByteScales& sc,
                                int sms, cudaStream_t st) {
  switch (a.block) {
    case 16: return launch_n<16>(maps, dm, a, sc, sms, st);
    case 32: return launch_n<32>(maps, dm, a, sc, sms, st);
    default: return launch_n<64>(maps, dm, a, sc, sms, st);
  }
}

}  // namespace jacap
