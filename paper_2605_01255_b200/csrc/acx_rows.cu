// Element-wise row operators: the 8-bit checkpoint of a matrix (store, load) and the gated activation
//     H = silu(G) * U,   silu(g) = g s(g),   s(g) = 1 / (1 + exp(-g)),
// whose backward reads G and U from their 8-bit checkpoints:
//     dU = dH G s,   dG = dH U s (1 + G (1 - s)).
//
// All of them are bound by HBM: each element is read once and written once, 16 bytes per thread and access.  Eight lanes
// hold one group of 128 columns, two vectors of 8 columns each (64 columns apart, so that the eight lanes read 128
// contiguous bytes): what a group costs once (three shuffles, its scale, where it is) is spread over 16 elements per
// thread; with one vector per thread and sixteen lanes the forward of the gated activation was bound by instructions.
#include <algorithm>

#include "acx_internal.h"
#include "acx_q8.cuh"

namespace acx {
namespace {

using namespace q8;

constexpr int kThreads = 256;
constexpr int kLanes = 8;                           // threads that hold one group
constexpr int kHalf = kLanes * kVec;                // columns between a thread's two vectors
constexpr int kGroupsPerBlock = kThreads / kLanes;

// Where a thread's columns are.  Groups are numbered through all rows (ng per row); a block takes 32 in a row.
struct Place {
  int64_t row, group;
  int col;
  bool live[2];   // whether each vector is inside the matrix (a partly filled last group has idle lanes)
};
struct Div {      // quotients by ng of numbers below ng + 32
  uint32_t ng, inv16;   // inv16 = ceil(2^16 / ng)
};
__device__ __forceinline__ Place place_of(int64_t rows, int cols, Div d) {
  const int64_t g0 = int64_t(blockIdx.x) * kGroupsPerBlock, row0 = g0 / d.ng;
  const uint32_t k = threadIdx.x / kLanes, off = uint32_t(g0 - row0 * d.ng) + k;
  // off < ng + 32: at most one row further where ng >= 32; else off < 64 and the 16-bit reciprocal is exact
  const uint32_t dr = d.ng >= 32 ? (off >= d.ng ? 1u : 0u) : (off * d.inv16) >> 16;
  Place p;
  p.row = row0 + dr;
  p.group = g0 + k;
  p.col = int(off - dr * d.ng) * kGroup + int(threadIdx.x % kLanes) * kVec;
#pragma unroll
  for (int v = 0; v < 2; ++v) p.live[v] = p.row < rows && p.col + v * kHalf < cols;
  return p;
}
__device__ __forceinline__ bool first_lane() { return threadIdx.x % kLanes == 0; }

template <typename T>
__global__ void __launch_bounds__(kThreads) q8_store_kernel(const T* __restrict__ X, int64_t ldx, int8_t* __restrict__ codes,
                                                            float* __restrict__ scales, int64_t rows, int cols, Div d) {
  wait_for_launch_before();
  let_next_launch_start();
  const Place p = place_of(rows, cols, d);
  Raw<T> x[2];
#pragma unroll
  for (int v = 0; v < 2; ++v) {
    x[v].zero();
    if (p.live[v]) x[v].load(X + p.row * ldx + p.col + v * kHalf);
  }
  const GroupScale g = group_scale(max_over<kLanes>(max(x[0].amax_bits(), x[1].amax_bits())));
#pragma unroll
  for (int v = 0; v < 2; ++v) {
    float2 f[4];
    x[v].get(f);
    if (p.live[v]) *reinterpret_cast<uint2*>(codes + p.row * int64_t(cols) + p.col + v * kHalf) = encode8(f, g.inv);
  }
  if (first_lane() && p.live[0]) scales[p.group] = g.scale;
}

template <typename T>
__global__ void __launch_bounds__(kThreads) q8_load_kernel(const int8_t* __restrict__ codes, const float* __restrict__ scales,
                                                           T* __restrict__ X, int64_t ldx, int64_t rows, int cols, Div d) {
  wait_for_launch_before();
  let_next_launch_start();
  const Place p = place_of(rows, cols, d);
  uint2 c[2];
  if (!p.live[0]) return;
  const int64_t at = p.row * int64_t(cols) + p.col;
  c[0] = __ldcg(reinterpret_cast<const uint2*>(codes + at));
  if (p.live[1]) c[1] = __ldcg(reinterpret_cast<const uint2*>(codes + at + kHalf));
  const float s = __ldcg(scales + p.group);
#pragma unroll
  for (int v = 0; v < 2; ++v) {
    if (!p.live[v]) break;
    float2 f[4];
    decode8(c[v], s, f);
    store8(X + p.row * ldx + p.col + v * kHalf, f);
  }
}

// s(g) from e = exp(-|g|) <= 1, which cannot overflow: 1 / (1 + e), or e / (1 + e) for negative g, so that a very negative
// gate keeps the tiny values it has (1 / (1 + exp(-g)) is 0 from g = -89 on).  bf16 outputs take the hardware's exponential
// and quotient (relative error about (4 + 1.2 |g|) 2^-23: 2^-21 at small gates, 2^-16 at -88, below which nothing is left;
// the output's rounding is 2^-9); fp32 outputs the library's.
__device__ __forceinline__ float sigmoid_of(float g, __nv_bfloat16) {
  const float e = __expf(-fabsf(g));
  return __fdividef(g < 0.f ? e : 1.f, 1.f + e);
}
__device__ __forceinline__ float sigmoid_of(float g, float) {
  const float e = expf(-fabsf(g));
  return __fdiv_rn(g < 0.f ? e : 1.f, 1.f + e);
}

template <typename T>
__device__ __forceinline__ float2 sigmoid2(float2 g, T) { return make_float2(sigmoid_of(g.x, T()), sigmoid_of(g.y, T())); }

template <typename T, bool KEEP>
__global__ void __launch_bounds__(kThreads) swiglu_fwd_kernel(const T* __restrict__ G, int64_t ldg, const T* __restrict__ U, int64_t ldu,
                                                              T* __restrict__ H, int8_t* __restrict__ Gq, float* __restrict__ Gs,
                                                              int8_t* __restrict__ Uq, float* __restrict__ Us, int64_t rows, int cols,
                                                              Div d) {
  wait_for_launch_before();
  let_next_launch_start();
  const Place p = place_of(rows, cols, d);
  Raw<T> g[2], u[2];
#pragma unroll
  for (int v = 0; v < 2; ++v) {
    g[v].zero();
    u[v].zero();
    if (p.live[v]) {
      g[v].load(G + p.row * ldg + p.col + v * kHalf);
      u[v].load(U + p.row * ldu + p.col + v * kHalf);
    }
  }
  GroupScale qg, qu;
  if (KEEP) {
    uint32_t mg = max(g[0].amax_bits(), g[1].amax_bits()), mu = max(u[0].amax_bits(), u[1].amax_bits());
    max_pair_over<T, kLanes>(mg, mu);
    qg = group_scale(mg);
    qu = group_scale(mu);
  }
  const int64_t at = p.row * int64_t(cols) + p.col;
#pragma unroll
  for (int v = 0; v < 2; ++v) {
    if (!p.live[v]) break;
    float2 gf[4], uf[4];
    g[v].get(gf);
    u[v].get(uf);
    if (KEEP) {
      *reinterpret_cast<uint2*>(Gq + at + v * kHalf) = encode8(gf, qg.inv);
      *reinterpret_cast<uint2*>(Uq + at + v * kHalf) = encode8(uf, qu.inv);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) uf[i] = mul2(uf[i], mul2(gf[i], sigmoid2(gf[i], T())));
    store8(H + at + v * kHalf, uf);
  }
  if (KEEP && first_lane() && p.live[0]) {
    Gs[p.group] = qg.scale;
    Us[p.group] = qu.scale;
  }
}

template <typename T>
__global__ void __launch_bounds__(kThreads) swiglu_bwd_kernel(const T* __restrict__ dH, const int8_t* __restrict__ Gq,
                                                              const float* __restrict__ Gs, const int8_t* __restrict__ Uq,
                                                              const float* __restrict__ Us, T* __restrict__ dG, int64_t lddg,
                                                              T* __restrict__ dU, int64_t lddu, int64_t rows, int cols, Div d) {
  wait_for_launch_before();
  let_next_launch_start();
  const Place p = place_of(rows, cols, d);
  if (!p.live[0]) return;
  uint2 cg[2], cu[2];
  Raw<T> x[2];
  const int64_t at = p.row * int64_t(cols) + p.col;
#pragma unroll
  for (int v = 0; v < 2; ++v) {
    if (!p.live[v]) break;
    cg[v] = __ldcg(reinterpret_cast<const uint2*>(Gq + at + v * kHalf));
    cu[v] = __ldcg(reinterpret_cast<const uint2*>(Uq + at + v * kHalf));
    x[v].load(dH + at + v * kHalf);
  }
  const float sg = __ldcg(Gs + p.group), su = __ldcg(Us + p.group);
#pragma unroll
  for (int v = 0; v < 2; ++v) {
    if (!p.live[v]) break;
    float2 g[4], u[4], dh[4];
    decode8(cg[v], sg, g);
    decode8(cu[v], su, u);
    x[v].get(dh);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 s = sigmoid2(g[i], T()), e = mul2(dh[i], s);
      const float2 slope = fma2(g[i], fma2(s, both(-1.f), both(1.f)), both(1.f));   // 1 + g (1 - s)
      u[i] = mul2(mul2(e, u[i]), slope);
      g[i] = mul2(e, g[i]);
    }
    store8(dG + p.row * lddg + p.col + v * kHalf, u);
    store8(dU + p.row * lddu + p.col + v * kHalf, g);
  }
}

struct Launch {
  unsigned grid;
  Div div;
};
Launch launch_of(const Rows& d) {
  const int64_t ng = (d.cols + kGroup - 1) / kGroup;
  return Launch{unsigned((d.rows * ng + kGroupsPerBlock - 1) / kGroupsPerBlock), Div{uint32_t(ng), uint32_t((65536 + ng - 1) / ng)}};
}

template <typename T>
cudaError_t launch_store(const Rows& d, const void* X, int64_t ldx, int8_t* codes, float* scales, cudaStream_t st) {
  const Launch l = launch_of(d);
  return launch_lined_up(q8_store_kernel<T>, dim3(l.grid), dim3(kThreads), 0, st, static_cast<const T*>(X), ldx, codes, scales, d.rows, int(d.cols), l.div);
}
template <typename T>
cudaError_t launch_load(const Rows& d, const int8_t* codes, const float* scales, void* X, int64_t ldx, cudaStream_t st) {
  const Launch l = launch_of(d);
  return launch_lined_up(q8_load_kernel<T>, dim3(l.grid), dim3(kThreads), 0, st, codes, scales, static_cast<T*>(X), ldx, d.rows, int(d.cols), l.div);
}
template <typename T, bool KEEP>
cudaError_t launch_swiglu_fwd(const Rows& d, const void* G, int64_t ldg, const void* U, int64_t ldu, void* H, int8_t* Gq, float* Gs, int8_t* Uq,
                       float* Us, cudaStream_t st) {
  const Launch l = launch_of(d);
  return launch_lined_up(swiglu_fwd_kernel<T, KEEP>, dim3(l.grid), dim3(kThreads), 0, st, static_cast<const T*>(G), ldg, static_cast<const T*>(U), ldu, static_cast<T*>(H),
                                                         Gq, Gs, Uq, Us, d.rows, int(d.cols), l.div);
}
template <typename T>
cudaError_t launch_swiglu_bwd(const Rows& d, const void* dH, const int8_t* Gq, const float* Gs, const int8_t* Uq, const float* Us, void* dG,
                       int64_t lddg, void* dU, int64_t lddu, cudaStream_t st) {
  const Launch l = launch_of(d);
  return launch_lined_up(swiglu_bwd_kernel<T>, dim3(l.grid), dim3(kThreads), 0, st, static_cast<const T*>(dH), Gq, Gs, Uq, Us, static_cast<T*>(dG), lddg,
                                                   static_cast<T*>(dU), lddu, d.rows, int(d.cols), l.div);
}

}  // namespace

cudaError_t q8_store(const Rows& d, const void* X, int64_t ldx, int8_t* codes, float* scales, cudaStream_t st) {
  return d.bf16 ? launch_store<__nv_bfloat16>(d, X, ldx, codes, scales, st) : launch_store<float>(d, X, ldx, codes, scales, st);
}

cudaError_t q8_load(const Rows& d, const int8_t* codes, const float* scales, void* X, int64_t ldx, cudaStream_t st) {
  return d.bf16 ? launch_load<__nv_bfloat16>(d, codes, scales, X, ldx, st) : launch_load<float>(d, codes, scales, X, ldx, st);
}

cudaError_t swiglu_fwd(const Rows& d, const void* G, int64_t ldg, const void* U, int64_t ldu, void* H, int8_t* Gq, float* Gs, int8_t* Uq,
                       float* Us, cudaStream_t st) {
  if (d.bf16)
    return Gq ? launch_swiglu_fwd<__nv_bfloat16, true>(d, G, ldg, U, ldu, H, Gq, Gs, Uq, Us, st)
              : launch_swiglu_fwd<__nv_bfloat16, false>(d, G, ldg, U, ldu, H, Gq, Gs, Uq, Us, st);
  return Gq ? launch_swiglu_fwd<float, true>(d, G, ldg, U, ldu, H, Gq, Gs, Uq, Us, st)
            : launch_swiglu_fwd<float, false>(d, G, ldg, U, ldu, H, Gq, Gs, Uq, Us, st);
}

cudaError_t swiglu_bwd(const Rows& d, const void* dH, const int8_t* Gq, const float* Gs, const int8_t* Uq, const float* Us, void* dG,
                       int64_t lddg, void* dU, int64_t lddu, cudaStream_t st) {
  return d.bf16 ? launch_swiglu_bwd<__nv_bfloat16>(d, dH, Gq, Gs, Uq, Us, dG, lddg, dU, lddu, st)
                : launch_swiglu_bwd<float>(d, dH, Gq, Gs, Uq, Us, dG, lddg, dU, lddu, st);
}

}  // namespace acx
