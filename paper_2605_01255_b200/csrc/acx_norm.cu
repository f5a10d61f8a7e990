// Residual join between two blocks of a layer, with the norm behind the first and the norm in front of the second:
//     t = h + alpha * gate * (w_post * b * r_b),   y = w_pre * t * r_t,   r_x = 1 / sqrt(mean(x^2) + eps)
// (b: the block's output, h: the residual stream; without w_post the block's output joins as it is, without gate the gate
// is one, without b it is the norm alone).  The training form keeps h and b in 8 bits and r_b, r_t exactly; the backward
// recomputes t^ = h^ + alpha gate w_post b^ r_b from them:
//     that = t^ r_t,  bhat = b^ r_b,  k = alpha gate w_post,
//     dt = dh_next + r_t (dy w_pre - that m1),      m1 = mean(dy w_pre that)
//     dh = dt,   db = r_b (k dt - bhat m2),         m2 = mean(k dt bhat)
//     dw_pre = sum_t dy that,   dw_post = alpha gate c,   dgate = alpha w_post c,   c = sum_t dt bhat.
#include <algorithm>

#include "acx_internal.h"
#include "acx_q8.cuh"
#include "acx_tmap.h"

namespace acx {
namespace {

using namespace q8;

// Sums over a thread block, the same in every thread: warps by shuffles, then the warps' sums in order.  `red`: one row
// per call of a loop turn (a row is written again only after a barrier that follows its last reading).
template <int N>
__device__ __forceinline__ void block_sum(float (&s)[N], float* red) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1)
#pragma unroll
    for (int k = 0; k < N; ++k) s[k] += __shfl_xor_sync(0xFFFFFFFFu, s[k], o);
  const int warps = int(blockDim.x) >> 5;
  if (warps == 1) return;
  if ((threadIdx.x & 31) == 0)
#pragma unroll
    for (int k = 0; k < N; ++k) red[k * 32 + (threadIdx.x >> 5)] = s[k];
  __syncthreads();
#pragma unroll
  for (int k = 0; k < N; ++k) s[k] = 0.f;
  for (int w = 0; w < warps; ++w)
#pragma unroll
    for (int k = 0; k < N; ++k) s[k] += red[k * 32 + w];
}

struct FwdArgs {
  const void *h, *b, *w_post, *gate, *w_pre;
  void *h_out, *y;
  int8_t *Hq, *Bq;
  float *Hs, *Bs, *rstd_post, *rstd_pre;
  int64_t rows;
  int cols;
  float eps, alpha;
};

// One row per thread block; a thread holds NV vectors of 8 columns, threadIdx.x + i * blockDim.x.
template <typename T, int NV, bool JOIN, bool KEEP>
__global__ void __launch_bounds__(NV == 4 ? 1024 : 512, 1) norm_join_fwd_kernel(const FwdArgs a) {
  __shared__ float red[2][32];
  const int64_t row = blockIdx.x, at = row * a.cols;
  const int ng = (a.cols + kGroup - 1) / kGroup;
  const float inv_n = 1.f / float(a.cols);
  float t[NV][8], b[JOIN ? NV : 1][8];
  auto col_of = [&](int i) { return (int(threadIdx.x) + i * int(blockDim.x)) * kVec; };
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int c = col_of(i);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      t[i][e] = 0.f;
      if (JOIN) b[i][e] = 0.f;
    }
    if (c < a.cols) {
      load8(static_cast<const T*>(a.h) + at + c, t[i]);
      if (JOIN) load8(static_cast<const T*>(a.b) + at + c, b[i]);
    }
  }
  if (KEEP) {
    auto keep = [&](const float (&v)[8], int c, int8_t* codes, float* scales) {
      const GroupScale g = group_scale(group_amax_bits(v));
      if (c < a.cols) {
        *reinterpret_cast<uint2*>(codes + at + c) = encode8(v, g.inv);
        if (threadIdx.x % kLanes == 0) scales[row * ng + c / kGroup] = g.scale;
      }
    };
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      keep(t[i], col_of(i), a.Hq, a.Hs);
      if (JOIN) keep(b[i], col_of(i), a.Bq, a.Bs);
    }
  }
  if (JOIN) {
    float r_b = 1.f;
    if (a.w_post) {
      float s[1] = {0.f};
#pragma unroll
      for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int e = 0; e < 8; ++e) s[0] += b[i][e] * b[i][e];
      block_sum(s, red[0]);
      r_b = rsqrtf(s[0] * inv_n + a.eps);
      if (KEEP && threadIdx.x == 0) a.rstd_post[row] = r_b;
    }
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = col_of(i);
      if (c >= a.cols) continue;
      float k[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) k[e] = a.alpha * r_b;
      if (a.w_post) {
        float w[8];
        load8(static_cast<const T*>(a.w_post) + c, w);
#pragma unroll
        for (int e = 0; e < 8; ++e) k[e] *= w[e];
      }
      if (a.gate) {
        float w[8];
        load8(static_cast<const T*>(a.gate) + c, w);
#pragma unroll
        for (int e = 0; e < 8; ++e) k[e] *= w[e];
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) t[i][e] += k[e] * b[i][e];
      store8(static_cast<T*>(a.h_out) + at + c, t[i]);
    }
  }
  float s[1] = {0.f};
#pragma unroll
  for (int i = 0; i < NV; ++i)
#pragma unroll
    for (int e = 0; e < 8; ++e) s[0] += t[i][e] * t[i][e];
  block_sum(s, red[1]);
  const float r_t = rsqrtf(s[0] * inv_n + a.eps);
  if (KEEP && threadIdx.x == 0) a.rstd_pre[row] = r_t;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int c = col_of(i);
    if (c >= a.cols) continue;
    float w[8];
    load8(static_cast<const T*>(a.w_pre) + c, w);
#pragma unroll
    for (int e = 0; e < 8; ++e) w[e] *= t[i][e] * r_t;
    store8(static_cast<T*>(a.y) + at + c, w);
  }
}

struct BwdArgs {
  const void *dy, *dh_next, *w_post, *gate, *w_pre;
  const int8_t *Hq, *Bq;
  const float *Hs, *Bs, *rstd_post, *rstd_pre;
  void *dh, *db;
  float* part;   // [gridDim.x][JOIN ? 2 : 1][cols]: this block's column sums of dy that and of dt bhat
  int64_t rows;
  int cols;
  float alpha;
};

// Persistent: a block walks the rows blockIdx.x, + gridDim.x, ... and keeps the column sums of its columns in registers.
// Both means of a row come out of one reduction: with dt = a + f that, a = dh_next + r_t dy w_pre and f = -r_t m1,
//     sum(k dt bhat) = sum(k a bhat) + f sum(k that bhat),
// so a row costs one barrier instead of two.
template <typename T, int NV, bool JOIN>
__global__ void __launch_bounds__(NV == 4 ? 1024 : 512, 1) norm_join_bwd_kernel(const BwdArgs a) {
  __shared__ float red[2][3 * 32];
  const int ng = (a.cols + kGroup - 1) / kGroup;
  const float inv_n = 1.f / float(a.cols);
  float sum_pre[NV][8], sum_c[JOIN ? NV : 1][8];
#pragma unroll
  for (int i = 0; i < NV; ++i)
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      sum_pre[i][e] = 0.f;
      if (JOIN) sum_c[i][e] = 0.f;
    }
  auto col_of = [&](int i) { return (int(threadIdx.x) + i * int(blockDim.x)) * kVec; };
  int turn = 0;
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x, turn ^= 1) {
    const int64_t at = row * a.cols;
    const float r_t = __ldg(a.rstd_pre + row), r_b = (JOIN && a.w_post) ? __ldg(a.rstd_post + row) : 1.f;
    float that[NV][8], av[NV][8], bhat[JOIN ? NV : 1][8], k[JOIN ? NV : 1][8];
    float s[3] = {0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = col_of(i);
      if (c >= a.cols) continue;
      float dy[8], w[8];
      const uint2 hq = __ldg(reinterpret_cast<const uint2*>(a.Hq + at + c));
      const float hs = __ldg(a.Hs + row * ng + c / kGroup);
      load8(static_cast<const T*>(a.dy) + at + c, dy);
#pragma unroll
      for (int e = 0; e < 8; ++e) av[i][e] = 0.f;
      if (a.dh_next) load8(static_cast<const T*>(a.dh_next) + at + c, av[i]);
      decode8(hq, hs, that[i]);
      if (JOIN) {
        const uint2 bq = __ldg(reinterpret_cast<const uint2*>(a.Bq + at + c));
        const float bs = __ldg(a.Bs + row * ng + c / kGroup);
        decode8(bq, bs * r_b, bhat[i]);
#pragma unroll
        for (int e = 0; e < 8; ++e) k[i][e] = a.alpha;
        if (a.w_post) {
          load8(static_cast<const T*>(a.w_post) + c, w);
#pragma unroll
          for (int e = 0; e < 8; ++e) k[i][e] *= w[e];
        }
        if (a.gate) {
          load8(static_cast<const T*>(a.gate) + c, w);
#pragma unroll
          for (int e = 0; e < 8; ++e) k[i][e] *= w[e];
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) that[i][e] += k[i][e] * bhat[i][e];
      }
      load8(static_cast<const T*>(a.w_pre) + c, w);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        that[i][e] *= r_t;
        const float gy = dy[e] * w[e];
        s[0] += gy * that[i][e];
        sum_pre[i][e] += dy[e] * that[i][e];
        av[i][e] += r_t * gy;
        if (JOIN) {
          const float kb = k[i][e] * bhat[i][e];
          s[1] += av[i][e] * kb;
          s[2] += that[i][e] * kb;
        }
      }
    }
    block_sum(s, red[turn]);
    const float f = -r_t * s[0] * inv_n, m2 = JOIN ? (s[1] + f * s[2]) * inv_n : 0.f;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = col_of(i);
      if (c >= a.cols) continue;
#pragma unroll
      for (int e = 0; e < 8; ++e) av[i][e] += f * that[i][e];
      store8(static_cast<T*>(a.dh) + at + c, av[i]);
      if (JOIN) {
        float db[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          sum_c[i][e] += av[i][e] * bhat[i][e];
          db[e] = a.w_post ? r_b * (k[i][e] * av[i][e] - bhat[i][e] * m2) : k[i][e] * av[i][e];
        }
        store8(static_cast<T*>(a.db) + at + c, db);
      }
    }
  }
  float* part = a.part + int64_t(blockIdx.x) * (JOIN ? 2 : 1) * a.cols;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int c = col_of(i);
    if (c >= a.cols) continue;
    store8(part + c, sum_pre[i]);
    if (JOIN) store8(part + a.cols + c, sum_c[i]);
  }
}

// Adds the blocks' column sums in a fixed order: 32 columns by 32 strips of blocks per thread block, strips then added in
// order; turns c into the gradients of w_post and of the gate.
template <typename T>
__global__ void __launch_bounds__(1024) norm_join_columns_kernel(const float* __restrict__ part, int blocks, int cols, int planes, float alpha,
                                                                 const T* __restrict__ w_post, const T* __restrict__ gate,
                                                                 float* __restrict__ dw_pre, float* __restrict__ dw_post,
                                                                 float* __restrict__ dgate) {
  __shared__ float red[32][33];
  const int x = threadIdx.x & 31, y = threadIdx.x >> 5, plane = blockIdx.y;
  const int c = int(blockIdx.x) * 32 + x;
  float s = 0.f;
  if (c < cols)
    for (int k = y; k < blocks; k += 32) s += part[(int64_t(k) * planes + plane) * cols + c];
  red[y][x] = s;
  __syncthreads();
  if (y != 0 || c >= cols) return;
  s = 0.f;
#pragma unroll
  for (int k = 0; k < 32; ++k) s += red[k][x];
  if (plane == 0) {
    if (dw_pre) dw_pre[c] = s;
    return;
  }
  s *= alpha;
  if (dw_post) dw_post[c] = gate ? s * float(gate[c]) : s;
  if (dgate) dgate[c] = w_post ? s * float(w_post[c]) : s;
}

// Vectors per thread and threads per block for a row of `cols` columns (at most 32768): one vector up to 4096 columns, two
// up to 8192 (512 threads with 128 registers hold both), four beyond (1024 threads, 64 registers).
struct Shape { int nv, threads; };
Shape shape_of(int64_t cols) {
  const int vecs = int(cols / kVec);
  const int nv = vecs <= 512 ? 1 : (vecs <= 1024 ? 2 : 4);
  return Shape{nv, ((vecs + nv - 1) / nv + 31) / 32 * 32};
}

template <typename T, bool JOIN, bool KEEP>
void launch_fwd(const FwdArgs& a, cudaStream_t st) {
  const Shape s = shape_of(a.cols);
  const unsigned grid = unsigned(a.rows);
  if (s.nv == 1) norm_join_fwd_kernel<T, 1, JOIN, KEEP><<<grid, s.threads, 0, st>>>(a);
  else if (s.nv == 2) norm_join_fwd_kernel<T, 2, JOIN, KEEP><<<grid, s.threads, 0, st>>>(a);
  else norm_join_fwd_kernel<T, 4, JOIN, KEEP><<<grid, s.threads, 0, st>>>(a);
}
template <typename T>
void launch_fwd(const FwdArgs& a, cudaStream_t st) {
  if (a.b) {
    if (a.Hq) launch_fwd<T, true, true>(a, st);
    else launch_fwd<T, true, false>(a, st);
  } else {
    if (a.Hq) launch_fwd<T, false, true>(a, st);
    else launch_fwd<T, false, false>(a, st);
  }
}

// Blocks of the backward: as many as are resident (2048 threads per SM, fewer where registers bound it), so that every
// block walks several rows and the column sums that leave the SMs stay small next to the rows.
int bwd_blocks(int64_t rows, int64_t cols) {
  const Shape s = shape_of(cols);
  const int per_sm = std::max(1, (s.nv == 1 ? 1024 : 512) / s.threads);
  return int(std::min<int64_t>(rows, int64_t(sm_count()) * per_sm));
}

template <typename T>
void launch_bwd(const BwdArgs& a, cudaStream_t st) {
  const Shape s = shape_of(a.cols);
  const int grid = bwd_blocks(a.rows, a.cols);
  if (a.Bq) {
    if (s.nv == 1) norm_join_bwd_kernel<T, 1, true><<<grid, s.threads, 0, st>>>(a);
    else if (s.nv == 2) norm_join_bwd_kernel<T, 2, true><<<grid, s.threads, 0, st>>>(a);
    else norm_join_bwd_kernel<T, 4, true><<<grid, s.threads, 0, st>>>(a);
  } else {
    if (s.nv == 1) norm_join_bwd_kernel<T, 1, false><<<grid, s.threads, 0, st>>>(a);
    else if (s.nv == 2) norm_join_bwd_kernel<T, 2, false><<<grid, s.threads, 0, st>>>(a);
    else norm_join_bwd_kernel<T, 4, false><<<grid, s.threads, 0, st>>>(a);
  }
}

}  // namespace

cudaError_t norm_join_fwd(const Rows& d, const void* h, const void* b, const void* w_post, const void* gate, const void* w_pre, void* h_out,
                          void* y, int8_t* Hq, float* Hs, int8_t* Bq, float* Bs, float* rstd_post, float* rstd_pre, float eps, float alpha,
                          cudaStream_t st) {
  FwdArgs a{h, b, w_post, gate, w_pre, h_out, y, Hq, Bq, Hs, Bs, rstd_post, rstd_pre, d.rows, int(d.cols), eps, alpha};
  if (d.bf16) launch_fwd<__nv_bfloat16>(a, st);
  else launch_fwd<float>(a, st);
  return launched();
}

size_t norm_join_bwd_workspace_bytes(const Rows& d) { return size_t(bwd_blocks(d.rows, d.cols)) * 2 * size_t(d.cols) * 4; }

cudaError_t norm_join_bwd(const Rows& d, const void* dy, const void* dh_next, const void* w_post, const void* gate, const void* w_pre,
                          const int8_t* Hq, const float* Hs, const int8_t* Bq, const float* Bs, const float* rstd_post,
                          const float* rstd_pre, void* dh, void* db, float* dw_post, float* dgate, float* dw_pre, float alpha, void* ws,
                          cudaStream_t st) {
  BwdArgs a{dy, dh_next, w_post, gate, w_pre, Hq, Bq, Hs, Bs, rstd_post, rstd_pre, dh, db, static_cast<float*>(ws), d.rows, int(d.cols), alpha};
  if (d.bf16) launch_bwd<__nv_bfloat16>(a, st);
  else launch_bwd<float>(a, st);
  cudaError_t e = launched();
  if (e != cudaSuccess || (!dw_pre && !dw_post && !dgate)) return e;
  const int planes = Bq ? 2 : 1;
  const dim3 grid(unsigned((d.cols + 31) / 32), unsigned((dw_post || dgate) ? 2 : 1));
  const int blocks = bwd_blocks(d.rows, d.cols);
  if (d.bf16)
    norm_join_columns_kernel<__nv_bfloat16><<<grid, 1024, 0, st>>>(a.part, blocks, a.cols, planes, alpha,
                                                                   static_cast<const __nv_bfloat16*>(w_post),
                                                                   static_cast<const __nv_bfloat16*>(gate), dw_pre, dw_post, dgate);
  else
    norm_join_columns_kernel<float><<<grid, 1024, 0, st>>>(a.part, blocks, a.cols, planes, alpha, static_cast<const float*>(w_post),
                                                           static_cast<const float*>(gate), dw_pre, dw_post, dgate);
  return launched();
}

}  // namespace acx
