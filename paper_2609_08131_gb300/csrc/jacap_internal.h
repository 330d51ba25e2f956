// jacap_internal.h - host-side launchers of the libjacap kernels.
// All launchers enqueue on `st` and return the launch error (cudaSuccess if
// the kernel was enqueued).
#pragma once

#include "jacap.h"
#include "jacap_dev.cuh"

namespace jacap {

// Bytes of the workspace of a layout without the run tables at its end (0 for
// an invalid layout).
size_t workspace_base(const jacap_layout* layout);

// Shared by the entry points (jacap_api.cu). check_layout needs no GPU; check_device
// gives the SM count of the current device, which must be a GB300.
jacap_status check_layout(const jacap_layout* L);
jacap_status check_device(int* sms);
void make_dims(const jacap_layout* L, const jacap_params* P, Dims& dm);
bool encode_kv_map(CUtensorMap* map, const jacap_layout* L, const void* base, int box_tokens = TILE);
bool encode_draft_map(CUtensorMap* map, const jacap_layout* L, const void* base, const int64_t* strides, int tokens);
bool encode_byte_map(CUtensorMap* map, const jacap_byte_cache* c, const void* base);
// The work plan's choices: work items of a pass over `L`, runs of the streaming
// kernels, CTAs of a persistent grid.
int64_t plan_items(const jacap_layout* L, const Dims& dm);
void plan_runs(Dims& dm, int64_t items, int sms);
int plan_grid(int64_t items, int sms);
// Units (layer, KV head, request) of a layout, 2^31 where there are more.
inline int64_t layout_units(const jacap_layout* L) {
  const int64_t top = (int64_t)1 << 31, planes = (int64_t)L->num_layers * L->num_kv_heads;
  const int64_t units = (planes < top ? planes : top) * L->num_seqs;
  return units < top ? units : top;
}
inline bool aligned16(const void* p) { return ((uintptr_t)p & 15u) == 0; }
inline jacap_status map_cuda(cudaError_t e) { return e == cudaSuccess ? JACAP_OK : JACAP_ERR_CUDA; }

// Tracing: built with -DJACAP_NVTX (JACAP_NVTX=1 in the environment of the
// build), the host side marks each kernel's launch with an NVTX range named
// "jacap/<step>" so a profiler timeline groups the GPU work by step of the
// pass; otherwise the ranges compile to nothing.
#ifdef JACAP_NVTX
#include <nvtx3/nvToolsExt.h>
inline void trace_push(const char* name) { nvtxRangePushA(name); }
inline void trace_pop() { nvtxRangePop(); }
#else
inline void trace_push(const char*) {}
inline void trace_pop() {}
#endif
struct TraceRange {
  explicit TraceRange(const char* name) { trace_push(name); }
  ~TraceRange() { trace_pop(); }
  TraceRange(const TraceRange&) = delete;
  TraceRange& operator=(const TraceRange&) = delete;
};

// Returns a failed CUDA call's error from the enclosing launcher.
#define JACAP_TRY(call)                     \
  do {                                      \
    const cudaError_t e_ = (call);          \
    if (e_ != cudaSuccess) return e_;       \
  } while (0)

// Launch `kernel`, with programmatic stream serialization when `pdl` (see
// pdl_wait()): the launch is prepared while the previous kernel of the stream
// runs and the kernel waits for it inside. Returns the launch error.
template <typename... KArgs, typename... Args>
cudaError_t launch_pdl(bool pdl, void (*kernel)(KArgs...), dim3 grid, dim3 block, size_t smem, cudaStream_t st,
                       Args&&... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = block;
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = pdl ? attr : nullptr;
  cfg.numAttrs = pdl ? 1 : 0;
  return cudaLaunchKernelEx(&cfg, kernel, static_cast<KArgs>(args)...);
}

// lengths: tokens of each request (the first ones of its range), or null: all.
cudaError_t launch_plan(const Dims& dm, const Ws& ws, const int32_t* cu, cudaStream_t st,
                        const int32_t* lengths = nullptr);
cudaError_t launch_window_stats(const Dims& dm, const Ws& ws, int dtype, const void* q, cudaStream_t st);
cudaError_t launch_kpass(const CUtensorMap& kmap, const Dims& dm, const Ws& ws, int dtype, const int32_t* cu,
                         int grid, cudaStream_t st);
cudaError_t launch_kpass_bf16(const CUtensorMap& kmap, const Dims& dm, const Ws& ws, const int32_t* cu, int grid,
                              cudaStream_t st);
// Full covariance (App. B.2): with a bf16 cache and a supported window shape
// (kfull_uses_tensor_cores) launch_kpass_full replaces the K pass (logits,
// full-covariance kappa and softmax statistics in one read of K); otherwise
// the K pass runs and launch_kfull (CUDA cores) overwrites its diagonal kappa.
bool kfull_uses_tensor_cores(const Dims& dm, int dtype);
cudaError_t launch_kpass_full(const CUtensorMap& kmap, const Dims& dm, const Ws& ws, int grid, cudaStream_t st);
// one thread waits (bounded by limit_ns) on an mbarrier nothing arrives on
cudaError_t launch_selftest_wait(const Ws& ws, unsigned long long limit_ns, cudaStream_t st);
cudaError_t launch_kfull(const CUtensorMap& kmap, const Dims& dm, const Ws& ws, int dtype, const void* k, int grid,
                         cudaStream_t st);
// The pool-softmax normaliser (M_h, 1 / Z_h) of every unit and query head,
// merged once from the K pass's chunk statistics into ws.ustats.
cudaError_t launch_unit_stats(const Dims& dm, const Ws& ws, cudaStream_t st);
cudaError_t launch_weights(const Dims& dm, const Ws& ws, const int32_t* cu, int grid, cudaStream_t st);
cudaError_t launch_gram(const CUtensorMap& vmap, const Dims& dm, const Ws& ws, int dtype, const void* v,
                        const int32_t* cu, int grid, cudaStream_t st);
// `partials`: about how many partial Grams a unit has.
cudaError_t launch_factor(const Dims& dm, const Ws& ws, const float* out_factor, int partials, int sms,
                          cudaStream_t st);
cudaError_t launch_score(const CUtensorMap& vmap, const Dims& dm, const Ws& ws, int dtype, const void* v,
                         const int32_t* cu, float* scores, int grid, cudaStream_t st);
// The fused schedule (k_fused.cu): CTAs of the factor, Gram and score roles.
struct FusedRoles {
  int nf, ng, ns;
};
// Gram, factor and scores of a bf16 cache in one cooperative launch of
// nf + ng + ns CTAs (at most one per SM); dm.keep_tiles set by the caller.
cudaError_t launch_fused(const CUtensorMap& vmap, const Dims& dm, const Ws& ws, float* scores, const FusedRoles& r,
                         cudaStream_t st);
// Selection only when k and kio are null. With k: the kept rows of k and v
// (dtype 1 = bf16, 0 = float32) are also copied into k_out and v_out, as
// launch_compact does (and the kept tokens' weights wt into wt_out, unless null).
// With kio: the holes of kio, vio (and pos, wt) are filled in place, as
// launch_compact_inplace does without preserve_order. With sinks >= 0 (and k) the
// scores are attention weights, and the first `sinks` and last `recent` tokens stay.
cudaError_t launch_select(const Dims& dm, const Ws& ws, const int32_t* cu, const float* scores, int budget,
                          int32_t* idx, int32_t* kept, int max_seqlen, cudaStream_t st, int dtype = 1,
                          const void* k = nullptr, const void* v = nullptr, void* k_out = nullptr,
                          void* v_out = nullptr, void* kio = nullptr, void* vio = nullptr, int32_t* pos = nullptr,
                          const WeightRef& wt = WeightRef{}, float* wt_out = nullptr, int sinks = -1,
                          int recent = -1);
// Blocks of launch_protect per unit.
int protect_parts(int max_seqlen, const int32_t* pos);
// Selection keys from attention weights: +inf for the first `sinks` and the last
// `recent` tokens of every unit.
cudaError_t launch_protect(const Dims& dm, const Ws& ws, const int32_t* cu, const WeightRef& weights,
                           const int32_t* pos, int sinks, int recent, float* keys, int max_seqlen, cudaStream_t st);
cudaError_t launch_compact(const Dims& dm, int dtype, const int32_t* cu, const void* k, const void* v,
                           const int32_t* idx, int budget, void* k_out, void* v_out, cudaStream_t st);
cudaError_t launch_stats_update(const Dims& dm, int dtype, const void* q, float* stats, int32_t* counts, int reset,
                                cudaStream_t st);
// One decode step (jacap_append): new rows, slots and running statistics (unless
// stats is null).
struct AppendArgs {
  const void *k_new, *v_new, *q_new;
  int64_t strides[6];
  int64_t tok_stride_k, tok_stride_v;  // between a request's new tokens (jacap_append_path)
  int64_t slot_rows;
  void *k, *v;
  int32_t* pos;
  float* stats;
  int32_t* counts;
};
// With `path` (host, [S][depth]): request s's new token path[s][step] to row
// lengths[s] + step, where step < taken[s].
cudaError_t launch_append(const Dims& dm, int dtype, const AppendArgs& a, const int32_t* lengths, const int32_t* ids,
                          cudaStream_t st, const int32_t* path = nullptr, int depth = 0,
                          const int32_t* taken = nullptr, int step = 0);
cudaError_t launch_stats_moments(const Dims& dm, const Ws& ws, const float* stats, const int32_t* counts,
                                 cudaStream_t st);
cudaError_t launch_compact_inplace(const Dims& dm, const Ws& ws, int dtype, const int32_t* cu, void* k, void* v,
                                   int32_t* pos, const int32_t* idx, int budget, int preserve_order,
                                   cudaStream_t st, const WeightRef& wt = WeightRef{});

// Rotary positions (k_rope.cu): token j of request s is row s, j of x and y.
struct RopeTensor {
  const void* x;
  void* y;
  int heads;
  int64_t xs[3], ys[3];  // request, token, head (elements)
};
struct RopeArgs {
  RopeTensor q, k;
  const int32_t* pos;
  int64_t ps[2];  // request, token
  const uint64_t* turns;
  int seqs, tokens, rot, interleaved, inverse;
  float amplitude;
};
// `vec`: every row of x and y starts on 16 bytes and no 16-byte piece splits a pair.
cudaError_t launch_rope(const RopeArgs& a, int dtype, bool vec, int sms, cudaStream_t st);

// Attention of a request's queries over its cached and drafted tokens (k_attend.cu);
// the layout's window is the number of queries.
struct AttendArgs {
  const void *q, *k, *v;
  const void *kd, *vd;        // drafted K and V, or null
  void* o;
  float* lse;                 // or null
  const int32_t* lengths;     // live tokens of each request, or null: all
  const int32_t* draft_lens;  // queries (and drafted tokens) of each request, or null: all
  const uint64_t* tree;       // [S][window] masks, or null: a chain
  int64_t os[4], kds[4], vds[4];  // strides of o and of the drafted K and V: request, layer, head, token
  int64_t ls[3];              // of lse: request, layer, head
  float scale2;               // scale log2 e, recentred for the tensor cores' truncation
  int chunk, nsplit, nrb, max_seqlen;  // tokens per split (float32), splits of a request at most, row blocks
  int block;                  // rows of a row block
  int least, edge;            // bf16: least tiles of a CTA's share, and between a split's border and a unit's start
                              // or end
  int slots;                  // bf16: of splits' sums
  int srows, prows;           // rows of a split's sums, and of a block of them (attend_part_rows)
  uint32_t tdiv;              // 2^32 / window, rounded up (window > 1)
  float *opart, *mlpart;      // the splits' sums [slots][blocks of srows][32][prows][4], and their
                              // [slots][srows][2] (maximum, sum); slot of a split: at_slot (k_attend.cu)
  int32_t* counts;            // [ATTEND_CTAS] splits done of the unit whose first split is the CTA's, where the last
                              // one joins them (zero between calls, and at one place in every layout's workspace)
  int32_t* nsps;              // bf16: [units][row blocks] this call's splits (<< 16) and the CTA of the first
  uint32_t* status;
};
// CTAs that share out a bf16 call's tiles, at most (two to each of 160 SMs; a GB300 has 152)
constexpr int ATTEND_CTAS = 320;
int attend_row_block(int dtype, int rows);  // rows of a CTA
int attend_part_rows(int rows);
// maps: K, V, drafted K, drafted V (bf16)
cudaError_t launch_attend(const CUtensorMap* maps, const Dims& dm, int dtype, const AttendArgs& a, const int32_t* cu,
                          int sms, cudaStream_t st);

// Rows into a cache held in 8 bits (k_bytes.cu); [0] of K, [1] of V.
struct ByteArgs {
  uint8_t* bytes[2];
  float* scales[2];
  int64_t strides[3], scale_strides[3];  // layer, head, slot
  const void* rows_in[2];
  int64_t row_strides[8];     // request, layer, head, token of K's rows, then of V's (elements)
  int S, L, Hkv;
  int rows;                   // store: rows of a request at most; append: of a slot
  int blocks;                 // store: blocks of 64 of them
  int tokens;                 // append: new tokens of a request
  const int32_t *lengths, *path, *taken;
  int32_t *lengths_out, *counts;  // counts: [S] CTAs of a request that have read its length (zero between calls)
  uint32_t* status;
};
cudaError_t launch_bytes_store(const ByteArgs& a, int dtype, cudaStream_t st);
cudaError_t launch_bytes_append(const ByteArgs& a, int dtype, cudaStream_t st);
// Which drafted tokens are accepted (k_verify.cu).
cudaError_t launch_verify(const jacap_verification& a, uint32_t* status, cudaStream_t st);

// Attention over a cache held in 8 bits (k_attend_bytes.cu): its blocks' scales, and its bytes. The AttendArgs' scale2 is 1 (partial
// maxima are log2 of weights), its lengths are given, and a request's tokens are a slot of max_seqlen.
struct ByteScales {
  const float *ks, *vs;
  int64_t strides[3];  // layer, head, slot
  const uint8_t *k, *v;
  int64_t row_strides[3];
  float scale2;        // scale log2 e
};
int attend_bytes_block(int rows);  // rows of a CTA
int attend_bytes_ctas(int block);  // CTAs at most
// maps: K, V, drafted K, drafted V
cudaError_t launch_attend_bytes(const CUtensorMap* maps, const Dims& dm, const AttendArgs& a, const ByteScales& sc,
                                int sms, cudaStream_t st);

// Attention weights that tokens received from a window of queries (k_weigh.cu).
struct WeighArgs {
  const void *q, *k;
  const int32_t* lengths;  // live tokens of each request, or null: all
  const int32_t* q_lens;   // queries of each request, or null: the window
  const int32_t* q_rows;   // [S][window] which query is the j-th, or null: j
  float* lse;              // [S][L][Hq][window]
  int given;               // 1: lse is an input
  const float* before;     // earlier weights, or null
  float* weights;          // [L*Hkv][Ntot]
  float scale2;            // scale log2 e, recentred for the tensor cores' truncation
  uint32_t tdiv;           // 2^32 / window, rounded up (window > 1)
  float2* norm;            // [L*Hkv][S][row blocks][128] a row's (maximum, sum) over all its request's tokens
  float2* stat;            // [L*Hkv][c_cap][2][row blocks][128] (maximum, sum) of a run (float32: a chunk)
};
constexpr int WEIGH_ROWS_MAX = 512;  // query rows per KV head
cudaError_t launch_weigh(const CUtensorMap& kmap, const Dims& dm, const Ws& ws, int dtype, const WeighArgs& a,
                         const int32_t* cu, int grid, cudaStream_t st);

}  // namespace jacap
