// Element-wise row operators: the 8-bit checkpoint of a matrix (store, load) and the gated activation
//     H = silu(G) * U,   silu(g) = g s(g),   s(g) = 1 / (1 + exp(-g)),
// whose backward reads G and U from their 8-bit checkpoints:
//     dU = dH G s,   dG = dH U s (1 + G (1 - s)).
//
// All of them are bound by HBM: each element is read once and written once, 16 bytes per thread and access, and 16
// consecutive lanes hold one group of 128 columns, so a group's scale costs four shuffles and no shared memory.
#include <algorithm>

#include "acx_internal.h"
#include "acx_q8.cuh"

namespace acx {
namespace {

using namespace q8;

constexpr int kThreads = 256;
constexpr int kGroupsPerPass = kThreads / kLanes;   // groups a thread block handles at a time

// Where a thread's 8 columns are.  Groups are numbered through all rows (ng per row); a block takes a contiguous run.
struct Place {
  int64_t row;
  int col;      // first of the 8 columns
  int64_t group;
  bool live;    // inside the matrix (a partly filled last group has idle lanes)
};
template <int PASSES>
struct Places {
  int64_t g0, row0, rows;
  uint32_t rem0, ng;
  int cols;
  __device__ Places(int64_t rows_, int cols_) : rows(rows_), cols(cols_) {
    ng = uint32_t(cols + kGroup - 1) / kGroup;
    g0 = int64_t(blockIdx.x) * (kGroupsPerPass * PASSES);
    row0 = g0 / ng;
    rem0 = uint32_t(g0 - row0 * ng);
  }
  __device__ Place at(int pass) const {
    const uint32_t k = uint32_t(pass) * kGroupsPerPass + (threadIdx.x / kLanes);
    const uint32_t off = rem0 + k, dr = off / ng;
    Place p;
    p.row = row0 + dr;
    p.group = g0 + k;
    p.col = int(off - dr * ng) * kGroup + int(threadIdx.x % kLanes) * kVec;
    p.live = p.row < rows && p.col < cols;
    return p;
  }
};

template <typename T, int PASSES>
__global__ void __launch_bounds__(kThreads) q8_store_kernel(const T* __restrict__ X, int64_t ldx, int8_t* __restrict__ codes,
                                                            float* __restrict__ scales, int64_t rows, int cols) {
  const Places<PASSES> places(rows, cols);
  float v[PASSES][8];
#pragma unroll
  for (int u = 0; u < PASSES; ++u) {   // every load is under way before the first is used
    const Place p = places.at(u);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[u][i] = 0.f;
    if (p.live) load8(X + p.row * ldx + p.col, v[u]);
  }
#pragma unroll
  for (int u = 0; u < PASSES; ++u) {
    const Place p = places.at(u);
    const GroupScale g = group_scale(group_amax_bits(v[u]));
    if (!p.live) continue;
    *reinterpret_cast<uint2*>(codes + p.row * int64_t(cols) + p.col) = encode8(v[u], g.inv);
    if (threadIdx.x % kLanes == 0) scales[p.group] = g.scale;
  }
}

template <typename T, int PASSES>
__global__ void __launch_bounds__(kThreads) q8_load_kernel(const int8_t* __restrict__ codes, const float* __restrict__ scales,
                                                           T* __restrict__ X, int64_t ldx, int64_t rows, int cols) {
  const Places<PASSES> places(rows, cols);
  uint2 c[PASSES];
  float s[PASSES];
#pragma unroll
  for (int u = 0; u < PASSES; ++u) {
    const Place p = places.at(u);
    if (!p.live) continue;
    c[u] = __ldg(reinterpret_cast<const uint2*>(codes + p.row * int64_t(cols) + p.col));
    s[u] = __ldg(scales + p.group);
  }
#pragma unroll
  for (int u = 0; u < PASSES; ++u) {
    const Place p = places.at(u);
    if (!p.live) continue;
    float v[8];
    decode8(c[u], s[u], v);
    store8(X + p.row * ldx + p.col, v);
  }
}

// s(g) from e = exp(-|g|) <= 1, which cannot overflow: 1 / (1 + e), or e / (1 + e) for negative g, so that a very negative
// gate keeps the tiny values it has (1 / (1 + exp(-g)) is 0 from g = -89 on).  bf16 outputs take the hardware's exponential
// and quotient (relative error about 2^-21, far below the output's rounding of 2^-9); fp32 outputs the library's.
__device__ __forceinline__ float sigmoid_of(float g, __nv_bfloat16) {
  const float e = __expf(-fabsf(g));
  return __fdividef(g < 0.f ? e : 1.f, 1.f + e);
}
__device__ __forceinline__ float sigmoid_of(float g, float) {
  const float e = expf(-fabsf(g));
  return __fdiv_rn(g < 0.f ? e : 1.f, 1.f + e);
}

template <typename T, int PASSES, bool KEEP>
__global__ void __launch_bounds__(kThreads) swiglu_fwd_kernel(const T* __restrict__ G, int64_t ldg, const T* __restrict__ U, int64_t ldu,
                                                              T* __restrict__ H, int8_t* __restrict__ Gq, float* __restrict__ Gs,
                                                              int8_t* __restrict__ Uq, float* __restrict__ Us, int64_t rows, int cols) {
  const Places<PASSES> places(rows, cols);
  float g[PASSES][8], u[PASSES][8];
#pragma unroll
  for (int k = 0; k < PASSES; ++k) {
    const Place p = places.at(k);
#pragma unroll
    for (int i = 0; i < 8; ++i) g[k][i] = u[k][i] = 0.f;
    if (p.live) {
      load8(G + p.row * ldg + p.col, g[k]);
      load8(U + p.row * ldu + p.col, u[k]);
    }
  }
#pragma unroll
  for (int k = 0; k < PASSES; ++k) {
    const Place p = places.at(k);
    GroupScale qg, qu;
    if (KEEP) {
      qg = group_scale(group_amax_bits(g[k]));
      qu = group_scale(group_amax_bits(u[k]));
    }
    if (!p.live) continue;
    if (KEEP) {
      *reinterpret_cast<uint2*>(Gq + p.row * int64_t(cols) + p.col) = encode8(g[k], qg.inv);
      *reinterpret_cast<uint2*>(Uq + p.row * int64_t(cols) + p.col) = encode8(u[k], qu.inv);
      if (threadIdx.x % kLanes == 0) {
        Gs[p.group] = qg.scale;
        Us[p.group] = qu.scale;
      }
    }
    float h[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) h[i] = g[k][i] * sigmoid_of(g[k][i], T()) * u[k][i];
    store8(H + p.row * int64_t(cols) + p.col, h);
  }
}

template <typename T, int PASSES>
__global__ void __launch_bounds__(kThreads) swiglu_bwd_kernel(const T* __restrict__ dH, const int8_t* __restrict__ Gq,
                                                              const float* __restrict__ Gs, const int8_t* __restrict__ Uq,
                                                              const float* __restrict__ Us, T* __restrict__ dG, int64_t lddg,
                                                              T* __restrict__ dU, int64_t lddu, int64_t rows, int cols) {
  const Places<PASSES> places(rows, cols);
  uint2 cg[PASSES], cu[PASSES];
  float sg[PASSES], su[PASSES], dh[PASSES][8];
#pragma unroll
  for (int k = 0; k < PASSES; ++k) {
    const Place p = places.at(k);
    if (!p.live) continue;
    const int64_t at = p.row * int64_t(cols) + p.col;
    cg[k] = __ldg(reinterpret_cast<const uint2*>(Gq + at));
    cu[k] = __ldg(reinterpret_cast<const uint2*>(Uq + at));
    sg[k] = __ldg(Gs + p.group);
    su[k] = __ldg(Us + p.group);
    load8(dH + at, dh[k]);
  }
#pragma unroll
  for (int k = 0; k < PASSES; ++k) {
    const Place p = places.at(k);
    if (!p.live) continue;
    float g[8], u[8];
    decode8(cg[k], sg[k], g);
    decode8(cu[k], su[k], u);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float s = sigmoid_of(g[i], T()), e = dh[k][i] * s;
      const float dg = e * u[i] * (1.f + g[i] * (1.f - s));
      u[i] = e * g[i];
      g[i] = dg;
    }
    store8(dG + p.row * lddg + p.col, g);
    store8(dU + p.row * lddu + p.col, u);
  }
}

template <int PASSES>
unsigned grid_for(int64_t rows, int64_t cols) {
  const int64_t groups = rows * ((cols + kGroup - 1) / kGroup), per_block = int64_t(kGroupsPerPass) * PASSES;
  return unsigned((groups + per_block - 1) / per_block);
}

}  // namespace

cudaError_t q8_store(const Rows& d, const void* X, int64_t ldx, int8_t* codes, float* scales, cudaStream_t st) {
  constexpr int P = 2;
  const unsigned grid = grid_for<P>(d.rows, d.cols);
  if (d.bf16)
    q8_store_kernel<__nv_bfloat16, P><<<grid, kThreads, 0, st>>>(static_cast<const __nv_bfloat16*>(X), ldx, codes, scales, d.rows, int(d.cols));
  else
    q8_store_kernel<float, P><<<grid, kThreads, 0, st>>>(static_cast<const float*>(X), ldx, codes, scales, d.rows, int(d.cols));
  return launched();
}

cudaError_t q8_load(const Rows& d, const int8_t* codes, const float* scales, void* X, int64_t ldx, cudaStream_t st) {
  constexpr int P = 2;
  const unsigned grid = grid_for<P>(d.rows, d.cols);
  if (d.bf16)
    q8_load_kernel<__nv_bfloat16, P><<<grid, kThreads, 0, st>>>(codes, scales, static_cast<__nv_bfloat16*>(X), ldx, d.rows, int(d.cols));
  else
    q8_load_kernel<float, P><<<grid, kThreads, 0, st>>>(codes, scales, static_cast<float*>(X), ldx, d.rows, int(d.cols));
  return launched();
}

namespace {
template <typename T, bool KEEP>
void launch_swiglu_fwd(const Rows& d, const void* G, int64_t ldg, const void* U, int64_t ldu, void* H, int8_t* Gq, float* Gs, int8_t* Uq,
                       float* Us, cudaStream_t st) {
  constexpr int P = 2;
  swiglu_fwd_kernel<T, P, KEEP><<<grid_for<P>(d.rows, d.cols), kThreads, 0, st>>>(
      static_cast<const T*>(G), ldg, static_cast<const T*>(U), ldu, static_cast<T*>(H), Gq, Gs, Uq, Us, d.rows, int(d.cols));
}
template <typename T>
void launch_swiglu_bwd(const Rows& d, const void* dH, const int8_t* Gq, const float* Gs, const int8_t* Uq, const float* Us, void* dG,
                       int64_t lddg, void* dU, int64_t lddu, cudaStream_t st) {
  constexpr int P = 2;
  swiglu_bwd_kernel<T, P><<<grid_for<P>(d.rows, d.cols), kThreads, 0, st>>>(static_cast<const T*>(dH), Gq, Gs, Uq, Us, static_cast<T*>(dG),
                                                                           lddg, static_cast<T*>(dU), lddu, d.rows, int(d.cols));
}
}  // namespace

cudaError_t swiglu_fwd(const Rows& d, const void* G, int64_t ldg, const void* U, int64_t ldu, void* H, int8_t* Gq, float* Gs, int8_t* Uq,
                       float* Us, cudaStream_t st) {
  if (d.bf16) {
    if (Gq) launch_swiglu_fwd<__nv_bfloat16, true>(d, G, ldg, U, ldu, H, Gq, Gs, Uq, Us, st);
    else launch_swiglu_fwd<__nv_bfloat16, false>(d, G, ldg, U, ldu, H, Gq, Gs, Uq, Us, st);
  } else {
    if (Gq) launch_swiglu_fwd<float, true>(d, G, ldg, U, ldu, H, Gq, Gs, Uq, Us, st);
    else launch_swiglu_fwd<float, false>(d, G, ldg, U, ldu, H, Gq, Gs, Uq, Us, st);
  }
  return launched();
}

cudaError_t swiglu_bwd(const Rows& d, const void* dH, const int8_t* Gq, const float* Gs, const int8_t* Uq, const float* Us, void* dG,
                       int64_t lddg, void* dU, int64_t lddu, cudaStream_t st) {
  if (d.bf16) launch_swiglu_bwd<__nv_bfloat16>(d, dH, Gq, Gs, Uq, Us, dG, lddg, dU, lddu, st);
  else launch_swiglu_bwd<float>(d, dH, Gq, Gs, Uq, Us, dG, lddg, dU, lddu, st);
  return launched();
}

}  // namespace acx
