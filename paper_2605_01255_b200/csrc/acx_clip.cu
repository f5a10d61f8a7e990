// The norm of many gradients and clipping:
//     norm = sqrt(sum over the tensors i of weight_i * sum of x^2),   f = min(1, max_norm / norm),   out = f x.
// A norm that is not finite leaves the gradients as they are (f = 1): the caller sees it in `total` and decides.
//
// Two launches.  The first takes each block's part of the sum, the second adds the parts up in every block, in the same order (so
// all of them have the same f, and two calls the same bits), and scales.  Bound by HBM: the gradients are read twice and
// written once; the second launch goes through the chunks from the last to the first and so finds what the first one read last
// still in L2.  With out = x and f = 1 nothing is left to do and it ends there.  Measured: factors of 16 layers of width 2048 and a bf16
// head, 717 MB, 369 us (the norm 101: 7.1 TB/s); factors of 24 layers of width 896, 78 MB, 46 us.
//
// Squares are summed in fp32 over eight elements and in 64 bits from there on; eight whose fp32 sum leaves the range in which it has
// all its digits are taken again in 64 bits.
#include <algorithm>

#include "acx_internal.h"
#include "acx_q8.cuh"

namespace acx {
namespace clip {
namespace {

constexpr int kThreads = 256, kVec = 8;
constexpr int kChunk = int(kGradChunk);                 // elements of a tensor that a block takes at a time
constexpr int kBlocksPerSm = 4;
constexpr int kMaxParts = 148 * kBlocksPerSm;           // blocks of the first launch at most

// The plan in device memory: one record per chunk.
struct Chunk {
  const void* src;
  void* dst;
  int32_t n;
  float weight;
  int32_t src_bf16, dst_bf16;
};
static_assert(sizeof(Chunk) == 32, "two loads");

// Tensors arrive as kernel parameters, so that nothing of the caller's memory is read after the call.
constexpr int kBatch = 64;
struct Tensor {
  const void* src;
  void* dst;
  int64_t n, first_chunk;
  float weight;
  int16_t src_bf16, dst_bf16;
};
struct Batch { Tensor t[kBatch]; };
__global__ void __launch_bounds__(kThreads) plan_kernel(const __grid_constant__ Batch b, Chunk* chunks) {
  wait_for_launch_before();
  let_next_launch_start();
  const Tensor& t = b.t[blockIdx.x];
  const int64_t n = (t.n + kChunk - 1) / kChunk;
  for (int64_t k = int64_t(blockIdx.y) * kThreads + threadIdx.x; k < n; k += int64_t(gridDim.y) * kThreads)
    chunks[t.first_chunk + k] = Chunk{static_cast<const uint8_t*>(t.src) + k * (kChunk * (t.src_bf16 ? 2 : 4)),
                                      static_cast<uint8_t*>(t.dst) + k * (kChunk * (t.dst_bf16 ? 2 : 4)),
                                      int32_t(t.n - k * kChunk < kChunk ? t.n - k * kChunk : kChunk), t.weight, t.src_bf16, t.dst_bf16};
}

// Chunk i, or nothing to do if it is none
__device__ __forceinline__ Chunk fetch_chunk(const Chunk* chunks, int64_t i, int64_t count) {
  union { int4 v[2]; Chunk c; } u;
  u.c.n = 0;
  if (i >= 0 && i < count) {
    u.v[0] = __ldcg(reinterpret_cast<const int4*>(chunks + i));
    u.v[1] = __ldcg(reinterpret_cast<const int4*>(chunks + i) + 1);
  }
  return u.c;
}

template <typename T>
__device__ __forceinline__ float element(const T* p) { return float(__ldcg(p)); }
template <>
__device__ __forceinline__ float element(const __nv_bfloat16* p) { return __bfloat162float(__ushort_as_bfloat16(__ldcg(reinterpret_cast<const unsigned short*>(p)))); }

// Sum of eight squares.  fp32 sums between these bounds have no square that overflowed, and none that lost digits counts in them.
__device__ __forceinline__ double squares(const float2 (&v)[4]) {
  float2 s = q8::mul2(v[0], v[0]);
#pragma unroll
  for (int k = 1; k < 4; ++k) s = q8::fma2(v[k], v[k], s);
  const float f = s.x + s.y;
  if (f >= 1e-24f && f <= 1e37f) return double(f);
  double d = 0.;
  if (f == 0.f && v[0].x == 0.f && v[0].y == 0.f && v[1].x == 0.f && v[1].y == 0.f && v[2].x == 0.f && v[2].y == 0.f && v[3].x == 0.f && v[3].y == 0.f)
    return d;
#pragma unroll
  for (int k = 0; k < 4; ++k) d += double(v[k].x) * double(v[k].x) + double(v[k].y) * double(v[k].y);
  return d;
}

// Vectors of eight that a thread asks for before it uses the first: 128 bytes of either type, half of that where it writes too (16 x 2048
// factors and a head: the norm 164 us with 64 bytes and 101 with 128, the scaling 259 with 128 and 245 with 64).
template <typename T>
constexpr int kUnroll = 16 / int(sizeof(T));

template <typename T>
__device__ __forceinline__ double chunk_squares(const T* x, int n) {
  constexpr int kUnroll = clip::kUnroll<T>;
  double sum = 0.;
  const int whole = n / kVec;
  const T* p = x + threadIdx.x * kVec;
  for (int left = whole - int(threadIdx.x); left > 0; left -= kThreads * kUnroll, p += kThreads * kUnroll * kVec) {
    q8::Raw<T> r[kUnroll];
#pragma unroll
    for (int k = 0; k < kUnroll; ++k) {
      r[k].zero();
      if (k * kThreads < left) r[k].load(p + k * kThreads * kVec);
    }
#pragma unroll
    for (int k = 0; k < kUnroll; ++k) {
      float2 v[4];
      r[k].get(v);
      sum += squares(v);
    }
  }
  const int i = whole * kVec + int(threadIdx.x);
  if (i < n) {
    const double v = element(x + i);
    sum += v * v;
  }
  return sum;
}

// All threads get the block's sum, added up in one order.
__device__ __forceinline__ double block_sum(double x, double* warps) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(0xFFFFFFFFu, x, o);
  __syncthreads();
  if ((threadIdx.x & 31) == 0) warps[threadIdx.x >> 5] = x;
  __syncthreads();
  double s = 0.;
#pragma unroll
  for (int w = 0; w < kThreads / 32; ++w) s += warps[w];
  return s;
}

__global__ void __launch_bounds__(kThreads, kBlocksPerSm) norm_kernel(const Chunk* __restrict__ chunks, int64_t count,
                                                        double* __restrict__ parts) {
  __shared__ double warps[kThreads / 32];
  wait_for_launch_before();
  let_next_launch_start();
  double sum = 0.;
  Chunk next = fetch_chunk(chunks, blockIdx.x, count);
  for (int64_t c = blockIdx.x; c < count; c += gridDim.x) {
    const Chunk t = next;
    next = fetch_chunk(chunks, c + gridDim.x, count);
    const double s = t.src_bf16 ? chunk_squares(static_cast<const __nv_bfloat16*>(t.src), t.n) : chunk_squares(static_cast<const float*>(t.src), t.n);
    sum += double(t.weight) * s;
  }
  sum = block_sum(sum, warps);
  if (threadIdx.x == 0) parts[blockIdx.x] = sum;
}

template <typename S, typename D>
__device__ __forceinline__ void chunk_scale(const S* x, D* y, int n, float f) {
  constexpr int kUnroll = clip::kUnroll<S> / 2;
  const int whole = n / kVec;
  const S* p = x + threadIdx.x * kVec;
  D* to = y + threadIdx.x * kVec;
  constexpr int kRound = kThreads * kUnroll;
  for (int left = whole - int(threadIdx.x); left > 0; left -= kRound, p += kRound * kVec, to += kRound * kVec) {
    q8::Raw<S> r[kUnroll];
#pragma unroll
    for (int k = 0; k < kUnroll; ++k) {
      r[k].zero();   // also what keeps the vectors of one chunk from living on to the next: the kernel spilled
      if (k * kThreads < left) r[k].load(p + k * kThreads * kVec);
    }
#pragma unroll
    for (int k = 0; k < kUnroll; ++k) {
      float2 v[4];
      r[k].get(v);
#pragma unroll
      for (int q = 0; q < 4; ++q) v[q] = q8::mul2(v[q], q8::both(f));
      if (k * kThreads < left) q8::store8(to + k * kThreads * kVec, v);
    }
  }
  const int i = whole * kVec + int(threadIdx.x);
  if (i < n) y[i] = D(element(x + i) * f);
}

__global__ void __launch_bounds__(kThreads, kBlocksPerSm) scale_kernel(const Chunk* __restrict__ chunks, int64_t count,
                                                         const double* __restrict__ parts, int part_count, float max_norm, float* __restrict__ total) {
  __shared__ double warps[kThreads / 32];
  wait_for_launch_before();
  let_next_launch_start();
  double sum = 0.;
  for (int i = threadIdx.x; i < part_count; i += kThreads) sum += __ldcg(parts + i);
  sum = block_sum(sum, warps);
  const double norm = sqrt(sum);
  const float f = norm > double(max_norm) && norm <= 1.7976931348623157e308 ? float(double(max_norm) / norm) : 1.f;
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    total[0] = float(norm);
    total[1] = f;
  }
  Chunk next = fetch_chunk(chunks, count - 1 - int64_t(blockIdx.x), count);
  for (int64_t c = count - 1 - int64_t(blockIdx.x); c >= 0; c -= gridDim.x) {
    const Chunk t = next;
    next = fetch_chunk(chunks, c - gridDim.x, count);
    if (f == 1.f && t.src == t.dst) continue;
    if (t.src_bf16) {
      const __nv_bfloat16* x = static_cast<const __nv_bfloat16*>(t.src);
      if (t.dst_bf16) chunk_scale(x, static_cast<__nv_bfloat16*>(t.dst), t.n, f);
      else chunk_scale(x, static_cast<float*>(t.dst), t.n, f);
    } else {
      const float* x = static_cast<const float*>(t.src);
      if (t.dst_bf16) chunk_scale(x, static_cast<__nv_bfloat16*>(t.dst), t.n, f);
      else chunk_scale(x, static_cast<float*>(t.dst), t.n, f);
    }
  }
}

unsigned blocks_for(int64_t chunks) { return unsigned(std::max<int64_t>(1, std::min<int64_t>(chunks, kMaxParts))); }

}  // namespace
}  // namespace clip

using namespace clip;

size_t grad_plan_bytes(const GradProblem& q) { return size_t(std::max<int64_t>(q.chunks, 1)) * sizeof(Chunk); }
size_t grad_clip_workspace_bytes(const GradProblem&) { return kMaxParts * sizeof(double); }

cudaError_t grad_plan(const GradProblem& q, const acx_grad* list, void* plan, cudaStream_t st) {
  Chunk* chunks = static_cast<Chunk*>(plan);
  int64_t chunk = 0;
  for (int64_t i0 = 0; i0 < q.tensors; i0 += kBatch) {
    Batch b{};
    const int count = int(std::min<int64_t>(kBatch, q.tensors - i0));
    int64_t most = 1;
    for (int i = 0; i < count; ++i) {
      const acx_grad& g = list[i0 + i];
      b.t[i] = Tensor{g.src, g.dst, g.n, chunk, g.weight, int16_t(g.src_dtype == ACX_BF16), int16_t(g.dst_dtype == ACX_BF16)};
      const int64_t n = (g.n + kChunk - 1) / kChunk;
      chunk += n;
      most = std::max(most, n);
    }
    const unsigned y = unsigned(std::min<int64_t>(64, (most + kThreads - 1) / kThreads));
    const cudaError_t e = launch_lined_up(plan_kernel, dim3(unsigned(count), y), dim3(kThreads), 0, st, b, chunks);
    if (e != cudaSuccess) return e;
  }
  return cudaSuccess;
}

cudaError_t grad_clip(const GradProblem& q, const void* plan, float max_norm, float* total, void* ws, cudaStream_t st) {
  const Chunk* chunks = static_cast<const Chunk*>(plan);
  double* parts = static_cast<double*>(ws);
  const unsigned blocks = blocks_for(q.chunks);
  const cudaError_t e = launch_lined_up(norm_kernel, dim3(blocks), dim3(kThreads), 0, st, chunks, q.chunks, parts);
  if (e != cudaSuccess) return e;
  return launch_lined_up(scale_kernel, dim3(blocks), dim3(kThreads), 0, st, chunks, q.chunks, static_cast<const double*>(parts), int(blocks),
                         max_norm, total);
}

}  // namespace acx
