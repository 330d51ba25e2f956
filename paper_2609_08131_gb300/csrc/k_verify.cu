// k_verify.cu - which of a request's drafted tokens the target model accepts, from given random numbers.
// At a node of the tree, r_0 = p (the target's probabilities after it), Z_0 = 1, and for its drafted tokens x in turn
//   x is accepted if u Z_j q(x) < r_j(x), else r_{j+1} = max(r_j - Z_j q, 0), Z_{j+1} = sum r_{j+1}
// (without q: r_j loses x, and Z_j r_j(x), with no sum over the row; where p does not sum to 1 Z is not quite r's); where
// none is left, the next token is the least y whose partial sum of r_j passes u_T sum r_j.
// As a value that is 0 stays 0, r_j = max(p - c_j q, 0) with c_j = Z_0 + .. + Z_{j-1}: one step, however many rejections.
//
// The tests need p and q at the drafted tokens alone, which all are fetched at once; rows are read only where a
// rejection is followed by a further drafted token of the same node, and once at the end. So a chain
// reads one row of p and one of q, of its T + 1 and T. A cluster of 8 CTAs (128 warps) has a request: every warp sums a
// contiguous part of the row, the sums meet through distributed shared memory, and the CTA whose part the drawn
// point falls into walks that part again. Every CTA takes all decisions alike, from the same numbers.
//
// Which token is drawn depends on sums over the whole vocabulary, so that float32 sums (off by some 2^-24) would
// draw a neighbour now and then; the card adds 64-bit floats at 1/64 of float32's rate (the decisions alone, in 64
// bits by all threads, took 15 us). So all numbers are unevaluated pairs of float32 (some 2^-46
// relative; Dekker's and Knuth's exact sums and products).
//
// Bound by latency, not by the rows' bytes: a chain of 4 over 32000 tokens takes 8 us, 16 chains of 8 over 128256 12.6 us (16 MB,
// 2.4 us at a copy's rate), 32 trees of 16 over 151936 33 us (39 MB, 5.7 us): a launch of clusters, the fetch of the drafted
// tokens' numbers, and for each node with a rejection a sum over the row and its exchange between the CTAs.
#include "jacap_dev.cuh"
#include "jacap_internal.h"

namespace jacap {

constexpr int VF_CTAS = 8, VF_WARPS = 16, VF_THREADS = 32 * VF_WARPS, VF_PARTS = VF_CTAS * VF_WARPS;
constexpr int VF_DRAFTS = 64, VF_BATCH = 8;
constexpr int VF_LIST = 768;  // values that a warp keeps between two sums: 96 KB of two CTAs on an SM
constexpr size_t VF_SMEM = (size_t)VF_WARPS * VF_LIST * sizeof(float2);

struct __align__(8) Pair {  // (one 8-byte access)
  float hi, lo;
};
// a + b exactly, |a| >= |b| (or any order: two_sum).
__device__ __forceinline__ Pair quick_sum(float a, float b) {
  const float s = __fadd_rn(a, b);
  return {s, __fsub_rn(b, __fsub_rn(s, a))};
}
__device__ __forceinline__ Pair two_sum(float a, float b) {
  const float s = __fadd_rn(a, b), t = __fsub_rn(s, a);
  return {s, __fadd_rn(__fsub_rn(a, __fsub_rn(s, t)), __fsub_rn(b, t))};
}
__device__ __forceinline__ Pair operator+(Pair x, Pair y) {
  const Pair s = two_sum(x.hi, y.hi);
  return quick_sum(s.hi, __fadd_rn(s.lo, __fadd_rn(x.lo, y.lo)));
}
__device__ __forceinline__ Pair operator-(Pair x, Pair y) { return x + Pair{-y.hi, -y.lo}; }
__device__ __forceinline__ Pair operator*(Pair x, float y) {
  const float h = __fmul_rn(x.hi, y);
  return quick_sum(h, __fmaf_rn(x.lo, y, __fmaf_rn(x.hi, y, -h)));
}
__device__ __forceinline__ bool positive(Pair x) { return x.hi > 0.f || (x.hi == 0.f && x.lo > 0.f); }
__device__ __forceinline__ bool operator>(Pair x, Pair y) { return positive(x - y); }
// sum + x, where the sum's low part collects the roundings and is added to the high one at the end (whole).
__device__ __forceinline__ void collect(Pair& sum, Pair x) {
  const Pair s = two_sum(sum.hi, x.hi);
  sum = {s.hi, __fadd_rn(sum.lo, __fadd_rn(s.lo, x.lo))};
}
__device__ __forceinline__ Pair whole_of(Pair x) { return quick_sum(x.hi, x.lo); }
// max(p - q, 0): what a first rejection leaves (and all of p, with q = 0)
__device__ __forceinline__ Pair rest(float p, float q) {
  const Pair d = two_sum(p, -q);  // (of the sign of its high part)
  return {d.hi < 0.f ? 0.f : d.hi, d.hi < 0.f ? 0.f : d.lo};
}
// max(r - z q, 0)
__device__ __forceinline__ Pair rest(Pair r, Pair z, float q) {
  const Pair d = r - z * q;
  const bool some = !(d.hi < 0.f) && !(d.hi == 0.f && d.lo <= 0.f);  // (a NaN stays)
  return {some ? d.hi : 0.f, some ? d.lo : 0.f};
}
__device__ __forceinline__ Pair shfl_xor(Pair x, int off) {
  return {__shfl_xor_sync(0xffffffffu, x.hi, off), __shfl_xor_sync(0xffffffffu, x.lo, off)};
}
__device__ __forceinline__ Pair shfl(Pair x, int from) {
  return {__shfl_sync(0xffffffffu, x.hi, from), __shfl_sync(0xffffffffu, x.lo, from)};
}
// The sum over the lanes, in all of them; and over the lanes up to the own one.
__device__ __forceinline__ Pair lanes_sum(Pair x) {
#pragma unroll
  for (int off = 16; off >= 1; off >>= 1) x = x + shfl_xor(x, off);
  return x;
}
__device__ __forceinline__ Pair lanes_scan(Pair x, int lane) {
#pragma unroll
  for (int off = 1; off < 32; off <<= 1) {
    const Pair y = {__shfl_up_sync(0xffffffffu, x.hi, off), __shfl_up_sync(0xffffffffu, x.lo, off)};
    if (lane >= off) x = x + y;
  }
  return x;
}

__device__ __forceinline__ float prob(const float* p) { return __ldg(p); }
__device__ __forceinline__ float prob(const __nv_bfloat16* p) { return __uint_as_float((uint32_t)__ldg((const uint16_t*)p) << 16); }

__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release;\n\tbarrier.cluster.wait.acquire;" ::: "memory");
}
__device__ __forceinline__ Pair remote_pair(const Pair* p, uint32_t rank) {  // p's of the cluster's CTA `rank`
  uint32_t at;
  Pair x;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(smem_u32(p)), "r"(rank));
  asm volatile("ld.shared::cluster.v2.f32 {%0, %1}, [%2];" : "=f"(x.hi), "=f"(x.lo) : "r"(at) : "memory");
  return x;
}

// What is left of the target's probabilities at a node after its first `n` rejections.
template <typename T>
struct Left {
  const T *p, *q;        // the node's rows; q null: the rejected tokens are taken out
  Pair c;                // with q: c_n
  const int32_t* gone;   // [n] rejected tokens (without q)
  int n;
  // p and q at y, y + step, ..; 0 from `end` on, and of tokens taken out
  template <int B>
  __device__ __forceinline__ void load(int y, int step, int end, float (&pr)[B], float (&qr)[B]) const {
    const bool both = q != nullptr && n > 0;
#pragma unroll
    for (int i = 0; i < B; ++i) {
      const bool on = y + i * step < end;
      pr[i] = on ? prob(p + y + i * step) : 0.f;
      qr[i] = on && both ? prob(q + y + i * step) : 0.f;
    }
    if (q == nullptr) {
#pragma unroll 1
      for (int j = 0; j < n; ++j) {
        const int out = gone[j] - y;
#pragma unroll
        for (int i = 0; i < B; ++i) pr[i] = out == i * step ? 0.f : pr[i];
      }
    }
  }
  // what is left of p[], into r[]
  template <bool TREE, int B>
  __device__ __forceinline__ void values(const float (&pr)[B], const float (&qr)[B], Pair (&r)[B]) const {
    if (TREE && q != nullptr && n > 1) {
#pragma unroll
      for (int i = 0; i < B; ++i) r[i] = rest({pr[i], 0.f}, c, qr[i]);
    } else {
#pragma unroll
      for (int i = 0; i < B; ++i) r[i] = rest(pr[i], qr[i]);
    }
  }
};

// The sum of what is left over [y0, y1), in all lanes. With `list` the (p, q) of which something is left go there,
// `kept` of them (-1: more than its VF_LIST): after further rejections nothing is left elsewhere.
template <bool TREE, typename T>
__device__ __forceinline__ Pair sum_left(const Left<T>& left, int y0, int y1, float2* list, int& kept) {
  constexpr int B = VF_BATCH;
  const int lane = threadIdx.x & 31;
  Pair acc[2] = {{0.f, 0.f}, {0.f, 0.f}};
  float pr[B], qr[B];
  int y = y0 + lane, count = 0;
  left.load(y, 32, y1, pr, qr);
#pragma unroll 1
  for (; y - lane < y1; y += 32 * B) {
    Pair r[B];
    left.template values<TREE>(pr, qr, r);
    if (TREE && list != nullptr) {
#pragma unroll
      for (int i = 0; i < B; ++i) {
        const bool some = positive(r[i]);
        const uint32_t who = __ballot_sync(0xffffffffu, some);
        const int at = count + __popc(who & ((1u << lane) - 1));
        if (some && at < VF_LIST) list[at] = make_float2(pr[i], qr[i]);
        count += __popc(who);
      }
    }
    left.load(y + 32 * B, 32, y1, pr, qr);  // (on their way while these are added)
#pragma unroll
    for (int i = 0; i < B; ++i) collect(acc[i & 1], r[i]);
  }
  if (TREE && list != nullptr) {
    kept = count <= VF_LIST ? count : -1;
    __syncwarp();
  }
  return lanes_sum(whole_of(acc[0]) + whole_of(acc[1]));
}
__device__ __forceinline__ Pair sum_listed(const float2* list, int kept, Pair c) {  // after more than one rejection
  const int lane = threadIdx.x & 31;
  Pair acc = {0.f, 0.f};
#pragma unroll 4
  for (int i = lane; i < kept; i += 32) {
    const float2 a = list[i];
    collect(acc, rest({a.x, 0.f}, c, a.y));
  }
  return lanes_sum(whole_of(acc));
}

// TREE: a node may have several drafted tokens after it (a chain's walk needs one sum, and keeps nothing).
template <typename T, bool TREE>
__global__ void __cluster_dims__(VF_CTAS, 1, 1) __launch_bounds__(VF_THREADS, 2)
    verify_kernel(const __grid_constant__ jacap_verification a, uint32_t* status) {
  __shared__ int32_t parent[VF_DRAFTS], token[VF_DRAFTS], accepted[VF_DRAFTS], gone[VF_DRAFTS], yes0[VF_DRAFTS];
  __shared__ float u[VF_DRAFTS + 1], pt[VF_DRAFTS], qt[VF_DRAFTS];
  __shared__ Pair z[VF_DRAFTS + 1], sums[2][VF_WARPS], all[VF_PARTS], ends[VF_WARPS], known_sum, start;
  __shared__ Pair node_c;
  __shared__ int32_t node, rejected, count, more, drawn_part;
  extern __shared__ float2 lists[];
  pdl_wait();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const uint32_t rank = blockIdx.x % VF_CTAS;
  const int s = blockIdx.x / VF_CTAS, Td = a.tokens, V = a.vocab;
  const int want = a.draft_lens != nullptr ? a.draft_lens[s] : Td, n = want < 0 ? 0 : (want < Td ? want : Td);
  const T* p = (const T*)a.p + s * a.p_strides[0];
  const T* q = a.q != nullptr ? (const T*)a.q + s * a.q_strides[0] : nullptr;
  bool bad = n != want;
  if (tid < VF_DRAFTS) {
    int up = -2, x = -1, yes = 0;  // (-2: nobody's)
    if (tid < n) {
      const uint64_t mask = a.tree != nullptr ? a.tree[(int64_t)s * Td + tid] & ((1ull << tid) - 1) : 0;
      up = a.tree != nullptr ? 63 - __clzll((long long)mask) : tid - 1;  // (63 - 64 for no bit)
      x = a.tokens_in[(int64_t)s * Td + tid];
      const float ut = a.u[(int64_t)s * (Td + 1) + tid];
      u[tid] = ut;
      if (x >= 0 && x < V) {
        const float px = prob(p + (up + 1) * a.p_strides[1] + x);
        const float qx = q != nullptr ? prob(q + (up + 1) * a.q_strides[1] + x) : 1.f;
        pt[tid] = px, qt[tid] = qx;
        yes = Pair{px, 0.f} > Pair{qx, 0.f} * ut;  // as a node's first one
      } else {
        bad = true;
        up = -2, x = -1;
      }
    }
    parent[tid] = up, token[tid] = x, yes0[tid] = yes;
  } else if (tid == VF_DRAFTS) {
    u[VF_DRAFTS] = a.u[(int64_t)s * (Td + 1) + Td];
    z[0] = {1.f, 0.f};
  }
  if (bad && rank == 0) atomicOr(status, (uint32_t)ST_INVALID);
  __syncthreads();

  const int per = (V + VF_PARTS - 1) / VF_PARTS;  // of a warp
  const auto part_end = [&](int part) { return (int)min((int64_t)V, (int64_t)part * per); };
  const int mine = (int)rank * VF_WARPS + warp, y0 = part_end(mine), y1 = part_end(mine + 1);
  int passes = 0;
  float2* list = lists + warp * VF_LIST;
  int kept = -1, kept_at = -2;  // the list's values, and their node
  Left<T> left = {p, q, {0.f, 0.f}, gone, 0};
  const auto at_node = [&](int at, int rejections) {
    left.p = p + (at + 1) * a.p_strides[1];
    left.q = q != nullptr && rejections > 0 ? q + (at + 1) * a.q_strides[1] : q;
    left.n = rejections;
    left.c = rejections > 0 && q != nullptr ? node_c : Pair{0.f, 0.f};
    if (kept_at != at) kept = -1;
  };
  // sum of what is left, to known_sum; all[] has the parts' sums. All threads of the cluster.
  const auto total = [&](bool keep) {
    Pair w;
    if (TREE && left.n > 1 && kept >= 0) {
      w = sum_listed(list, kept, left.c);
    } else {
      w = sum_left<TREE>(left, y0, y1, keep ? list : nullptr, kept);
      if (keep) kept_at = node;
    }
    // (the sums of the pass before are read: each CTA writes these again two passes later)
    Pair* own = sums[passes++ & 1];
    if (lane == 0) own[warp] = w;
    cluster_sync();
    if (tid < VF_PARTS) all[tid] = remote_pair(own + tid % VF_WARPS, tid / VF_WARPS);
    __syncthreads();
    if (warp == 0) {
      Pair t = all[lane];
#pragma unroll
      for (int i = 32; i < VF_PARTS; i += 32) t = t + all[i + lane];
      t = lanes_sum(t);
      if (lane == 0) known_sum = t;
    }
    __syncthreads();
  };

  // The walk, by the first warp, until it needs a sum over the vocabulary (of what a second rejection is
  // measured by) or ends. A lane has the parents of drafted tokens lane and lane + 32.
  int at = -1, taken = 0, known = 1, turned = 0;  // known: how many of the node's Z are there; turned: rejections
  const int up0 = parent[lane], up1 = parent[lane + 32];
  const uint64_t ok0 = (uint64_t)__ballot_sync(0xffffffffu, yes0[lane + 32] != 0) << 32 |
                       __ballot_sync(0xffffffffu, yes0[lane] != 0);
  const auto children = [&](int of) {
    return (uint64_t)__ballot_sync(0xffffffffu, up1 == of) << 32 | __ballot_sync(0xffffffffu, up0 == of);
  };
  uint64_t pending = children(-1);
  Pair turned_c = {0.f, 0.f};  // c of the node's rejections
  const auto walk = [&]() {
    bool need = false;
    while (pending != 0) {
      const int t = __ffsll((long long)pending) - 1;
      bool yes = ok0 >> t & 1;
      Pair r = {pt[t], 0.f};
      if (turned > 0) {
        if (q != nullptr && turned == known) {
          need = true;
          break;
        }
        if (q != nullptr) {
          r = rest(r, turned_c, qt[t]);
        } else {
          for (int j = 0; j < turned; ++j)
            if (gone[j] == token[t]) r = {0.f, 0.f};
        }
        yes = r > z[turned] * qt[t] * u[t];
      }
      pending &= pending - 1;
      if (yes) {
        if (lane == 0) accepted[taken] = t;
        ++taken;
        at = t, turned = 0, known = 1, turned_c = {0.f, 0.f};
        pending = children(at);
      } else {
        if (q == nullptr && lane == 0) {
          gone[turned] = token[t];
          z[turned + 1] = z[turned] - r;
        }
        turned_c = turned_c + z[turned];
        ++turned;
        __syncwarp();
      }
    }
    if (lane == 0) node = at, rejected = turned, node_c = turned_c, count = taken, more = need ? 1 : 0;
  };
  if (warp == 0) walk();
  __syncthreads();
  for (bool again = false;;) {  // the sums that the walk needs, and the one to draw by
    const bool last = more == 0;
    at_node(node, again ? 0 : rejected);
    total(!last && q != nullptr);
    if (last) {
      if (again || known_sum.hi != 0.f || left.n == 0) break;
      again = true;     // nothing left, by rounding: the target's own
      __syncthreads();  // known_sum is read
      continue;
    }
    if (warp == 0) {
      if (lane == 0) z[known] = known_sum;
      ++known;
      __syncwarp();
      walk();
    }
    __syncthreads();
  }
  const Pair whole = known_sum, point = whole * u[VF_DRAFTS];
  const bool fine = whole.hi > 0.f && whole.hi <= 3.4e38f;
  if (warp == 0) {  // the first part whose end passes the point, or the last one of any weight
    constexpr int PER = VF_PARTS / 32;
    Pair own[PER], sum = {0.f, 0.f};
#pragma unroll
    for (int i = 0; i < PER; ++i) sum = sum + (own[i] = all[lane * PER + i]);
    Pair c = lanes_scan(sum, lane);
    c = {__shfl_up_sync(0xffffffffu, c.hi, 1), __shfl_up_sync(0xffffffffu, c.lo, 1)};
    if (lane == 0) c = {0.f, 0.f};
    int found = -1, last = -1;
    Pair found_at = c, last_at = c;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const Pair next = c + own[i];
      if (found < 0 && positive(own[i]) && next > point) found = lane * PER + i, found_at = c;
      if (positive(own[i])) last = lane * PER + i, last_at = c;
      c = next;
    }
    const uint32_t who = __ballot_sync(0xffffffffu, found >= 0), any = __ballot_sync(0xffffffffu, last >= 0);
    const int from = who != 0 ? __ffs((int)who) - 1 : (any != 0 ? 31 - __clz((int)any) : 0);
    const int part = __shfl_sync(0xffffffffu, who != 0 ? found : last, from);
    const Pair part_at = shfl(who != 0 ? found_at : last_at, from);
    if (lane == 0) drawn_part = part < 0 ? 0 : part, start = part_at;
  }
  __syncthreads();
  if (rank == 0) {
    if (tid < Td) a.path[(int64_t)s * Td + tid] = tid < count ? accepted[tid] : -1;
    if (tid == 0) {
      a.taken[s] = count;
      if (!fine) {
        a.next[s] = 0;
        atomicOr(status, (uint32_t)ST_NONFINITE);
      }
    }
  }
  if (fine && drawn_part / VF_WARPS == (int)rank) {  // (the whole CTA) the part, shared out among the warps
    const int b0 = part_end(drawn_part), b1 = part_end(drawn_part + 1), each = (b1 - b0 + VF_WARPS - 1) / VF_WARPS;
    const int w0 = min(b1, b0 + warp * each), w1 = min(b1, w0 + each);
    const Pair own = sum_left<TREE>(left, w0, w1, nullptr, kept);
    if (lane == 0) ends[warp] = own;
    __syncthreads();
    // the first warp whose end passes the point, or the last one of any weight
    const Pair e = lane < VF_WARPS ? ends[lane] : Pair{0.f, 0.f}, upto = start + lanes_scan(e, lane);
    const uint32_t past_it = __ballot_sync(0xffffffffu, positive(e) && upto > point);
    const uint32_t heavy_ones = __ballot_sync(0xffffffffu, positive(e));
    const bool passes_it = past_it != 0;
    const int pick = passes_it ? __ffs((int)past_it) - 1 : 31 - __clz((int)heavy_ones);
    const Pair mine_at = shfl(upto - e, warp);
    if (pick == warp) {
      int got = -1, heavy = w0;
      Pair c = mine_at;
      for (int y = w0; y < w1 && got < 0; y += 128) {
        Pair r[4];
        float pr[4], qr[4];
        left.load(y + 4 * lane, 1, w1, pr, qr);
        left.template values<TREE>(pr, qr, r);
        const Pair four = (r[0] + r[1]) + (r[2] + r[3]), upto = lanes_scan(four, lane);
        const uint32_t past = __ballot_sync(0xffffffffu, positive(four) && c + upto > point);
        const uint32_t some = __ballot_sync(0xffffffffu, positive(four));
        // the lane of the point, else the last one of any weight: its first value that passes, else its last of any
        const int who = past != 0 && passes_it ? __ffs((int)past) - 1 : (some != 0 ? 31 - __clz((int)some) : -1);
        if (who >= 0) {
          Pair b = c + (upto - four);
          int first = -1, end = 0;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            b = b + r[i];
            if (positive(r[i])) end = i;
            if (first < 0 && positive(r[i]) && b > point) first = i;
          }
          const int at_lane = __shfl_sync(0xffffffffu, first >= 0 ? first : end, who);
          heavy = y + 4 * who + at_lane;
          if (past != 0 && passes_it) got = heavy;
        }
        c = c + shfl(upto, 31);
      }
      if (lane == 0) a.next[s] = got >= 0 ? got : heavy;
    }
  }
  cluster_sync();  // nobody leaves while its sums may be read
}

template <typename T, bool TREE>
static cudaError_t launch_t(const jacap_verification& a, uint32_t* status, cudaStream_t st) {
  const size_t smem = TREE ? VF_SMEM : 0;
  JACAP_TRY(cudaFuncSetAttribute(verify_kernel<T, TREE>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem));
  return launch_pdl(true, verify_kernel<T, TREE>, dim3((unsigned)(a.num_seqs * VF_CTAS)), VF_THREADS, smem, st, a, status);
}
cudaError_t launch_verify(const jacap_verification& a, uint32_t* status, cudaStream_t st) {
  if (a.dtype == JACAP_BF16)
    return a.tree != nullptr ? launch_t<__nv_bfloat16, true>(a, status, st) : launch_t<__nv_bfloat16, false>(a, status, st);
  return a.tree != nullptr ? launch_t<float, true>(a, status, st) : launch_t<float, false>(a, status, st);
}

}  // namespace jacap
