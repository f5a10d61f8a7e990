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

// One row per thread block; a thread holds NV vectors of 8 columns, threadIdx.x + i * blockDim.x: 16 consecutive lanes
// hold a group of an 8-bit checkpoint.  Bound by HBM; what it needs for that is enough loads under way, so a row is
// spread over few threads with several vectors each (about 128 threads) and many rows are resident per SM; the weight
// vectors are asked for before the barrier that the row's sums wait at.
template <typename T, int NV, int MAXT, bool JOIN, bool KEEP>
__global__ void __launch_bounds__(MAXT) norm_join_fwd_kernel(const FwdArgs a) {
  __shared__ float red[2][32];
  const int64_t row = blockIdx.x, at = row * a.cols;
  const int ng = (a.cols + kGroup - 1) / kGroup;
  const float inv_n = 1.f / float(a.cols);
  Raw<T> h[NV], b[JOIN ? NV : 1];
  auto col_of = [&](int i) { return (int(threadIdx.x) + i * int(blockDim.x)) * kVec; };
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int c = col_of(i);
    h[i].zero();
    if (JOIN) b[i].zero();
    if (c < a.cols) {
      h[i].load(static_cast<const T*>(a.h) + at + c);
      if (JOIN) b[i].load(static_cast<const T*>(a.b) + at + c);
    }
  }
  Raw<T> w1[JOIN ? NV : 1], w2[JOIN ? NV : 1];
  if (JOIN) {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = col_of(i);
      if (c >= a.cols) continue;
      if (a.w_post) w1[i].load(static_cast<const T*>(a.w_post) + c);
      if (a.gate) w2[i].load(static_cast<const T*>(a.gate) + c);
    }
  }
  if (KEEP) {
    auto keep = [&](const Raw<T>& x, uint32_t amax, int c, int8_t* codes, float* scales) {
      const GroupScale g = group_scale(amax);
      if (c >= a.cols) return;
      float v[8];
      x.get(v);
      *reinterpret_cast<uint2*>(codes + at + c) = encode8(v, g.inv);
      if (threadIdx.x % 16 == 0) scales[row * ng + c / kGroup] = g.scale;
    };
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      uint32_t mh = h[i].amax_bits(), mb = JOIN ? b[JOIN ? i : 0].amax_bits() : 0u;
      if (JOIN) max_pair_over<T, 16>(mh, mb);
      else mh = max_over<16>(mh);
      keep(h[i], mh, col_of(i), a.Hq, a.Hs);
      if (JOIN) keep(b[JOIN ? i : 0], mb, col_of(i), a.Bq, a.Bs);
    }
  }
  float t[NV][8];
#pragma unroll
  for (int i = 0; i < NV; ++i) h[i].get(t[i]);
  if (JOIN) {
    float r_b = 1.f;
    if (a.w_post) {
      float s[1] = {0.f};
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        float v[8];
        b[JOIN ? i : 0].get(v);
#pragma unroll
        for (int e = 0; e < 8; ++e) s[0] += v[e] * v[e];
      }
      block_sum(s, red[0]);
      r_b = rsqrtf(s[0] * inv_n + a.eps);
      if (KEEP && threadIdx.x == 0) a.rstd_post[row] = r_b;
    }
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = col_of(i);
      if (c >= a.cols) continue;
      float k[8], v[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) k[e] = a.alpha * r_b;
      if (a.w_post) {
        w1[JOIN ? i : 0].get(v);
#pragma unroll
        for (int e = 0; e < 8; ++e) k[e] *= v[e];
      }
      if (a.gate) {
        w2[JOIN ? i : 0].get(v);
#pragma unroll
        for (int e = 0; e < 8; ++e) k[e] *= v[e];
      }
      b[JOIN ? i : 0].get(v);
#pragma unroll
      for (int e = 0; e < 8; ++e) t[i][e] += k[e] * v[e];
      store8(static_cast<T*>(a.h_out) + at + c, t[i]);
    }
  }
  Raw<T> w3[NV];
#pragma unroll
  for (int i = 0; i < NV; ++i)
    if (col_of(i) < a.cols) w3[i].load(static_cast<const T*>(a.w_pre) + col_of(i));
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
    w3[i].get(w);
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

__device__ __forceinline__ void copy_async(uint32_t dst, const void* src, int bytes) {   // 8 or 16 bytes, both aligned to them
  if (bytes == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
  else asm volatile("cp.async.ca.shared.global [%0], [%1], 8;" ::"r"(dst), "l"(src) : "memory");
}

// Persistent: a block walks the rows blockIdx.x, + gridDim.x, ... and keeps the column sums of its columns in registers.
// Both means of a row come out of one reduction: with dt = a + f that, a = dh_next + r_t dy w_pre and f = -r_t m1,
//     sum(k dt bhat) = sum(k a bhat) + f sum(k that bhat),
// so a row costs one barrier instead of two.  The registers that the sums and the weights take leave room for few
// threads, too few to keep HBM busy with their own loads: with DEPTH > 0 every thread copies its vectors of the next
// DEPTH rows into shared memory asynchronously (its own slots, so no barrier guards them).
template <typename T, int NV, int MAXT, int MINB, int DEPTH, bool JOIN>
__global__ void __launch_bounds__(MAXT, MINB) norm_join_bwd_kernel(const BwdArgs a) {
  extern __shared__ __align__(16) uint8_t ring[];
  __shared__ float red[2][3 * 32];
  constexpr int kParts = sizeof(T) == 2 ? 1 : 2;          // 16-byte parts of a vector of T
  constexpr int kSlot = 2 * 16 * kParts + (JOIN ? 16 : 8);   // dy, dh_next, codes of h and b
  const int ng = (a.cols + kGroup - 1) / kGroup, threads = int(blockDim.x);
  const float inv_n = 1.f / float(a.cols);
  auto col_of = [&](int i) { return (int(threadIdx.x) + i * threads) * kVec; };
  // Shared memory: stage, vector, then dy parts | dh_next parts | codes of h | codes of b, each for all threads
  const uint32_t ring0 = static_cast<uint32_t>(__cvta_generic_to_shared(ring));
  auto base_of = [&](int stage, int i) { return uint32_t((stage * NV + i) * threads * kSlot); };
  auto fetch = [&](int64_t row, int stage) {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = col_of(i);
      if (c >= a.cols) continue;
      const int64_t at = row * a.cols + c;
      const uint32_t s0 = ring0 + base_of(stage, i);
      const uint8_t* dy = reinterpret_cast<const uint8_t*>(static_cast<const T*>(a.dy) + at);
      const uint8_t* dn = reinterpret_cast<const uint8_t*>(static_cast<const T*>(a.dh_next) + at);
#pragma unroll
      for (int q = 0; q < kParts; ++q) {
        copy_async(s0 + (q * threads + threadIdx.x) * 16, dy + 16 * q, 16);
        if (a.dh_next) copy_async(s0 + ((kParts + q) * threads + threadIdx.x) * 16, dn + 16 * q, 16);
      }
      copy_async(s0 + 2 * kParts * threads * 16 + threadIdx.x * 8, a.Hq + at, 8);
      if (JOIN) copy_async(s0 + (2 * kParts * 16 + 8) * threads + threadIdx.x * 8, a.Bq + at, 8);
    }
  };
  auto vec_at = [&](uint32_t off, float (&v)[8]) {     // a vector of T in the ring
    if (sizeof(T) == 2) {
      Raw<__nv_bfloat16> r;
      r.u = *reinterpret_cast<const uint4*>(ring + off + threadIdx.x * 16);
      r.get(v);
    } else {
      Raw<float> r;
      r.a = *reinterpret_cast<const float4*>(ring + off + threadIdx.x * 16);
      r.b = *reinterpret_cast<const float4*>(ring + off + (threads + threadIdx.x) * 16);
      r.get(v);
    }
  };

  // what a column is multiplied with in every row
  float k[JOIN ? NV : 1][8], wp[NV][8], sum_pre[NV][8], sum_c[JOIN ? NV : 1][8];
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int c = col_of(i);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      sum_pre[i][e] = wp[i][e] = 0.f;
      if (JOIN) {
        sum_c[i][e] = 0.f;
        k[i][e] = a.alpha;
      }
    }
    if (c >= a.cols) continue;
    load8(static_cast<const T*>(a.w_pre) + c, wp[i]);
    float w[8];
    if (JOIN && a.w_post) {
      load8(static_cast<const T*>(a.w_post) + c, w);
#pragma unroll
      for (int e = 0; e < 8; ++e) k[i][e] *= w[e];
    }
    if (JOIN && a.gate) {
      load8(static_cast<const T*>(a.gate) + c, w);
#pragma unroll
      for (int e = 0; e < 8; ++e) k[i][e] *= w[e];
    }
  }
  const int64_t step = gridDim.x;
#pragma unroll
  for (int s = 0; s < DEPTH; ++s) {
    if (blockIdx.x + s * step < a.rows) fetch(blockIdx.x + s * step, s);
    asm volatile("cp.async.commit_group;" ::: "memory");
  }
  // a row's scales are asked for one row ahead
  float hs[NV], bs[JOIN ? NV : 1], r_t = 0.f, r_b = 1.f;
  auto scales = [&](int64_t row) {
    if (row >= a.rows) return;
    r_t = __ldg(a.rstd_pre + row);
    if (JOIN && a.w_post) r_b = __ldg(a.rstd_post + row);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = col_of(i);
      if (c >= a.cols) continue;
      hs[i] = __ldg(a.Hs + row * ng + c / kGroup);
      if (JOIN) bs[i] = __ldg(a.Bs + row * ng + c / kGroup);
    }
  };
  scales(blockIdx.x);
  int turn = 0, stage = 0;
  for (int64_t row = blockIdx.x; row < a.rows; row += step, turn ^= 1) {
    const int64_t at = row * a.cols;
    float that[NV][8], av[NV][8], bhat[JOIN ? NV : 1][8];
    float s[3] = {0.f, 0.f, 0.f};
    if (DEPTH > 0) asm volatile("cp.async.wait_group %0;" ::"n"(DEPTH > 0 ? DEPTH - 1 : 0) : "memory");
    const float rt = r_t, rb = r_b;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = col_of(i);
      if (c >= a.cols) continue;
      float dy[8];
      uint2 hq, bq;
#pragma unroll
      for (int e = 0; e < 8; ++e) av[i][e] = 0.f;
      if (DEPTH > 0) {
        const uint32_t s0 = base_of(stage, i);
        vec_at(s0, dy);
        if (a.dh_next) vec_at(s0 + kParts * threads * 16, av[i]);
        hq = *reinterpret_cast<const uint2*>(ring + s0 + 2 * kParts * threads * 16 + threadIdx.x * 8);
        if (JOIN) bq = *reinterpret_cast<const uint2*>(ring + s0 + (2 * kParts * 16 + 8) * threads + threadIdx.x * 8);
      } else {
        load8(static_cast<const T*>(a.dy) + at + c, dy);
        if (a.dh_next) load8(static_cast<const T*>(a.dh_next) + at + c, av[i]);
        hq = __ldg(reinterpret_cast<const uint2*>(a.Hq + at + c));
        if (JOIN) bq = __ldg(reinterpret_cast<const uint2*>(a.Bq + at + c));
      }
      decode8(hq, hs[i], that[i]);
      if (JOIN) {
        decode8(bq, bs[i] * rb, bhat[i]);
#pragma unroll
        for (int e = 0; e < 8; ++e) that[i][e] += k[i][e] * bhat[i][e];
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        that[i][e] *= rt;
        const float gy = dy[e] * wp[i][e];
        s[0] += gy * that[i][e];
        sum_pre[i][e] += dy[e] * that[i][e];
        av[i][e] += rt * gy;
        if (JOIN) {
          const float kb = k[i][e] * bhat[i][e];
          s[1] += av[i][e] * kb;
          s[2] += that[i][e] * kb;
        }
      }
    }
    scales(row + step);
    block_sum(s, red[turn]);
    if (DEPTH > 0) {   // this stage's values are in registers: its slots take the row DEPTH turns on
      if (row + DEPTH * step < a.rows) fetch(row + DEPTH * step, stage);
      asm volatile("cp.async.commit_group;" ::: "memory");
      if (++stage == DEPTH) stage = 0;
    }
    const float f = -rt * s[0] * inv_n, m2 = JOIN ? (s[1] + f * s[2]) * inv_n : 0.f;
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
          db[e] = a.w_post ? rb * (k[i][e] * av[i][e] - bhat[i][e] * m2) : k[i][e] * av[i][e];
        }
        store8(static_cast<T*>(a.db) + at + c, db);
      }
    }
  }
  if (DEPTH > 0) asm volatile("cp.async.wait_all;" ::: "memory");
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
    for (int k = y; k < blocks; k += 8 * 32) {   // eight loads under way, added in order
      float v[8];
#pragma unroll
      for (int u = 0; u < 8; ++u) v[u] = k + 32 * u < blocks ? __ldg(part + (int64_t(k + 32 * u) * planes + plane) * cols + c) : 0.f;
#pragma unroll
      for (int u = 0; u < 8; ++u) s += v[u];
    }
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

int round_warp(int threads) { return (threads + 31) / 32 * 32; }

template <typename T, int NV, int MAXT, bool JOIN, bool KEEP>
void launch_fwd(const FwdArgs& a, cudaStream_t st) {
  const int threads = round_warp((a.cols / kVec + NV - 1) / NV);
  norm_join_fwd_kernel<T, NV, MAXT, JOIN, KEEP><<<unsigned(a.rows), threads, 0, st>>>(a);
}
template <typename T, bool JOIN, bool KEEP>
void launch_fwd(const FwdArgs& a, cudaStream_t st) {
  const int vecs = a.cols / kVec;
  if (vecs <= 128) launch_fwd<T, 1, 128, JOIN, KEEP>(a, st);
  else if (vecs <= 256) launch_fwd<T, 2, 128, JOIN, KEEP>(a, st);
  else if (vecs <= 384) launch_fwd<T, 3, 128, JOIN, KEEP>(a, st);
  else if (vecs <= 1024) launch_fwd<T, 4, 256, JOIN, KEEP>(a, st);
  else launch_fwd<T, 4, 1024, JOIN, KEEP>(a, st);
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

// The backward's shape for a row of `cols` columns (at most 32768): one vector per thread up to 3072 columns, two up to
// 8192, four beyond; as many blocks as are resident at the registers that leaves (768, 512 or fewer threads per SM), so
// that every block walks several rows and the column sums that leave the SMs stay small next to the rows.
struct BwdShape { int nv, threads, per_sm; };
BwdShape bwd_shape(int64_t cols) {
  const int vecs = int(cols / kVec);
  const int nv = vecs <= 384 ? 1 : (vecs <= 1024 ? 2 : 4);
  const int threads = round_warp((vecs + nv - 1) / nv);
  return BwdShape{nv, threads, std::max(1, std::min(16, (nv == 1 ? 768 : 512) / threads))};
}
int bwd_blocks(int64_t rows, int64_t cols) { return int(std::min<int64_t>(rows, int64_t(sm_count()) * bwd_shape(cols).per_sm)); }

template <typename T, int NV, int MAXT, int MINB, int DEPTH, bool JOIN>
cudaError_t launch_bwd(const BwdArgs& a, int threads, cudaStream_t st) {
  auto kernel = norm_join_bwd_kernel<T, NV, MAXT, MINB, DEPTH, JOIN>;
  constexpr int kSlot = 2 * 8 * int(sizeof(T)) + (JOIN ? 16 : 8);
  static DeviceOnce once;
  if (DEPTH > 0 && once.needed()) {
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, DEPTH * NV * MAXT * kSlot);
    if (e != cudaSuccess) return e;
    once.done();
  }
  kernel<<<bwd_blocks(a.rows, a.cols), threads, DEPTH * NV * threads * kSlot, st>>>(a);
  return launched();
}
template <typename T, bool JOIN>
cudaError_t launch_bwd(const BwdArgs& a, cudaStream_t st) {
  const BwdShape s = bwd_shape(a.cols);
  constexpr int kDepth = sizeof(T) == 2 ? 4 : 2;
  if (s.nv == 1) return launch_bwd<T, 1, 384, 2, kDepth, JOIN>(a, s.threads, st);
  if (s.nv == 2 && s.threads <= 256) return launch_bwd<T, 2, 256, 2, kDepth, JOIN>(a, s.threads, st);
  if (s.nv == 2) return launch_bwd<T, 2, 512, 1, kDepth, JOIN>(a, s.threads, st);
  return launch_bwd<T, 4, 1024, 1, 0, JOIN>(a, s.threads, st);
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
  cudaError_t e;
  if (d.bf16) e = Bq ? launch_bwd<__nv_bfloat16, true>(a, st) : launch_bwd<__nv_bfloat16, false>(a, st);
  else e = Bq ? launch_bwd<float, true>(a, st) : launch_bwd<float, false>(a, st);
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
