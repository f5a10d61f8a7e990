// Internal declarations shared by the translation units of libacx (not part of the C ABI).
#pragma once
#include <cuda_runtime.h>
#include <atomic>
#include <cstddef>
#include <cstdint>

#include "../../include/acx.h"
#include "acx_device.h"
#include "acx_sketch.cuh"

namespace acx {

// Everything a launcher needs, derived from a validated acx_desc.
struct Problem {
  int64_t m, d_in, d_out;
  int r;
  bool bf16;
  SketchParams sp;
};

// A validated acx_rows_desc.
struct Rows {
  int64_t rows, cols;
  bool bf16;
};

// A validated acx_ce_desc.
struct CeProblem {
  int64_t m, d, vocab;
  float logit_scale;
};

// Device-side status word values (written by kernels whose bounded waits expire).
constexpr int kDevOk = 0;
constexpr int kDevTimeout = 1;

// Counts every kernel launch the library makes (reported by acx_kernel_launches()).
inline std::atomic<unsigned long long>& kernel_launch_counter() {
  static std::atomic<unsigned long long> counter{0};
  return counter;
}
inline cudaError_t launched() {
  kernel_launch_counter().fetch_add(1, std::memory_order_relaxed);
  return cudaGetLastError();
}

// Launches with programmatic stream serialization: the kernel may start before the launch before it has finished, and waits
// for that itself (wait_for_launch_before, first thing or as soon as it needs to).  In clusters of `cluster` blocks along x.
//
// That wait covers the launch before and no other.  So every kernel of the library that is launched this way ends only after
// the launch before it has ended, whether or not it needs anything of it (what it waits for is then all that was launched
// before); and one that needs nothing of it lets the next launch start only then, too.
template <typename... K, typename... A>
cudaError_t launch_lined_up_in_clusters(unsigned cluster, void (*kernel)(K...), dim3 grid, dim3 block, size_t smem, cudaStream_t st, const A&... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = block;
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim = {cluster, 1, 1};
  cfg.attrs = attr;
  cfg.numAttrs = cluster > 1 ? 2 : 1;
  const cudaError_t e = cudaLaunchKernelEx(&cfg, kernel, args...);
  kernel_launch_counter().fetch_add(1, std::memory_order_relaxed);
  return e;
}
template <typename... K, typename... A>
cudaError_t launch_lined_up(void (*kernel)(K...), dim3 grid, dim3 block, size_t smem, cudaStream_t st, const A&... args) {
  return launch_lined_up_in_clusters(1, kernel, grid, block, smem, st, args...);
}
#ifdef __CUDACC__
__device__ __forceinline__ void wait_for_launch_before() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void let_next_launch_start() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
#endif

// Checks a caller's descriptor and derives the launch problem from it (defined with the C ABI).
acx_status validate(const acx_desc* d, Problem* out);
// Device address of the status word on the current device (nullptr on a CUDA error).
int* device_status_ptr();

// ---- SIMT path (fp32 I/O; any valid shape) -------------------------------------------------------
size_t simt_bwd_workspace_bytes(const Problem& p);
// Vt != nullptr in the calls below: the second factor V^T (r x d_in) is read from memory instead of generated.
cudaError_t simt_fwd(const Problem& p, const void* X, const void* W, void* Y, void* XS, cudaStream_t st, const void* Vt = nullptr);
cudaError_t simt_bwd(const Problem& p, const void* G, const void* W, const void* XS, void* dX, float* A,
                     void* ws, cudaStream_t st);
cudaError_t simt_reconstruct(const Problem& p, const float* A, float* dW, float beta, cudaStream_t st, const void* Vt = nullptr);
cudaError_t sketch_materialize(const Problem& p, void* S_out, cudaStream_t st);

// ---- tcgen05 path (bf16 I/O; any valid shape) ----------------------------------------------------
size_t sm100_bwd_workspace_bytes(const Problem& p);
// Vt != nullptr: the second factor V^T (r x d_in, bf16) is read from memory instead of generated from the seed.
// Vt == nullptr and ws != nullptr: S^T is written once into ws (sm100_fwd_workspace_bytes) by a small grid and the
// GEMM reads it from there; with neither, each CTA generates its slices of S in shared memory.
size_t sm100_fwd_workspace_bytes(const Problem& p);
cudaError_t sm100_fwd(const Problem& p, const void* X, const void* W, void* Y, void* XS, int* status, cudaStream_t st,
                      const void* Vt = nullptr, void* ws = nullptr, const void* bias = nullptr);
// db[c] = sum over the tokens of G[t][c] (bf16 in, fp32 out), two deterministic stages through ws.
size_t bias_grad_workspace_bytes(const Problem& p);
cudaError_t bias_grad(const Problem& p, const void* G, float* db, void* ws, cudaStream_t st);
// db[c] = sum over z < splits of part[z][c], in order.
cudaError_t sum_column_partials(const float* part, float* db, int64_t d_out, int splits, cudaStream_t st);
constexpr int kMaxFactorSplits = 128;  // upper bound of the token ranges of the gradient factor (sizes the partial column sums)
cudaError_t sm100_dx(const Problem& p, const void* G, const void* W, void* dX, int* status, cudaStream_t st);
size_t sm100_reconstruct_workspace_bytes(const Problem& p);
cudaError_t sm100_reconstruct(const Problem& p, const float* A, float* dW, float beta, void* ws, int* status, cudaStream_t st,
                              const void* Vt = nullptr);
cudaError_t sm100_reconstruct_adamw(const Problem& p, const float* A, float* W, float* m, float* v, void* W_lp, float lr, float beta1,
                                    float beta2, float eps, float weight_decay, int step, void* ws, int* status, cudaStream_t st);
cudaError_t sm100_lowrank_adamw(const Problem& p, const float* A, float* mA, float* vA, const void* Vt, float* W, float lr,
                                float beta1, float beta2, float eps, float weight_decay, int step, void* ws, int* status,
                                cudaStream_t st);
// Second factor of the randomized-SVD compressor: Vt = (U^T U)^-1 U^T X (r x d_in, bf16).
size_t sm100_rsvd_workspace_bytes(const Problem& p);
cudaError_t sm100_rsvd_factor(const Problem& p, const void* X, const void* U, void* Vt, void* ws, int* status, cudaStream_t st);
size_t sm100_factor_scratch_bytes(const Problem& p);  // split-K partials through global memory (no cluster)
// db_part != nullptr: the kernel also adds up G's columns over each token range into db_part[range][d_out] (room for
// kMaxFactorSplits ranges) and *db_splits receives the number of ranges.
cudaError_t sm100_factor(const Problem& p, const void* G, const void* XS, float* A, void* ws, int* status, cudaStream_t st,
                         bool allow_cluster, float* db_part = nullptr, int* db_splits = nullptr, bool after_dx = false);

// ---- row operators (bf16 or fp32) -----------------------------------------------------------------
cudaError_t q8_store(const Rows& d, const void* X, int64_t ldx, int8_t* codes, float* scales, cudaStream_t st);
cudaError_t q8_load(const Rows& d, const int8_t* codes, const float* scales, void* X, int64_t ldx, cudaStream_t st);
// Gq == nullptr: no checkpoints (then Gs, Uq, Us are not read either).
cudaError_t swiglu_fwd(const Rows& d, const void* G, int64_t ldg, const void* U, int64_t ldu, void* H, int8_t* Gq, float* Gs, int8_t* Uq,
                       float* Us, cudaStream_t st);
cudaError_t swiglu_bwd(const Rows& d, const void* dH, const int8_t* Gq, const float* Gs, const int8_t* Uq, const float* Us, void* dG,
                       int64_t lddg, void* dU, int64_t lddu, cudaStream_t st);
constexpr int64_t kMaxNormCols = 32768;
cudaError_t norm_join_fwd(const Rows& d, const void* h, const void* b, const void* w_post, const void* gate, const void* w_pre, void* h_out,
                          void* y, int8_t* Hq, float* Hs, int8_t* Bq, float* Bs, float* rstd_post, float* rstd_pre, float eps, float alpha,
                          cudaStream_t st);
size_t norm_join_bwd_workspace_bytes(const Rows& d);
cudaError_t norm_join_bwd(const Rows& d, const void* dy, const void* dh_next, const void* w_post, const void* gate, const void* w_pre,
                          const int8_t* Hq, const float* Hs, const int8_t* Bq, const float* Bs, const float* rstd_post,
                          const float* rstd_pre, void* dh, void* db, float* dw_post, float* dgate, float* dw_pre, float alpha, void* ws,
                          cudaStream_t st);

// ---- softmax cross entropy over a vocabulary (bf16 X and W) ---------------------------------------
size_t ce_fwd_workspace_bytes(const CeProblem& p);
cudaError_t ce_fwd(const CeProblem& p, const void* X, const void* W, const int64_t* targets, const float* weight, float* loss, float* lse,
                   float* total, void* ws, int* status, cudaStream_t st);
size_t ce_bwd_workspace_bytes(const CeProblem& p);
cudaError_t ce_bwd(const CeProblem& p, const void* X, const void* W, const int64_t* targets, const float* weight, const float* lse,
                   const float* loss, const float* denom, float scale, void* dX, void* dW, void* ws, int* status, cudaStream_t st);

// Test/debug: overrides the tile-shape cost models of the forward and dX (0 = off, 1..4 = a GEMM mode).
void sm100_force_gemm_mode(int mode);

}  // namespace acx
