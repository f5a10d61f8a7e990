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
#include <climits>

#include "acx_internal.h"
#include "acx_q8.cuh"
#include "acx_tmap.h"

namespace acx {
namespace {

using namespace q8;

// Three sums over a warp at once: the first two exchanges of the butterfly halve the values a lane carries, so that all
// three take six shuffles instead of fifteen.  Value k ends in the lanes with lane >> 3 = k.
__device__ __forceinline__ float warp_sum3(float s0, float s1, float s2) {
  const int lane = threadIdx.x & 31;
  const bool up = lane & 16, odd = lane & 8;
  float a = up ? s2 : s0, b = up ? 0.f : s1;
  a += __shfl_xor_sync(0xFFFFFFFFu, up ? s0 : s2, 16);
  b += __shfl_xor_sync(0xFFFFFFFFu, up ? s1 : 0.f, 16);
  float v = odd ? b : a;
  v += __shfl_xor_sync(0xFFFFFFFFu, odd ? a : b, 8);
#pragma unroll
  for (int o = 4; o > 0; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
  return v;
}
// Sums over the thread block, the same in every thread.  `red` may be written again after a later barrier only.
__device__ __forceinline__ float3 block_sum3(float s0, float s1, float s2, float4* red) {
  const int lane = threadIdx.x & 31, warps = int(blockDim.x) >> 5;
  float v = warp_sum3(s0, s1, s2);
  if (warps > 1) {
    if ((lane & 7) == 0) reinterpret_cast<float*>(red)[4 * (threadIdx.x >> 5) + (lane >> 3)] = v;
    __syncthreads();
    const float4 q = lane < warps ? red[lane] : make_float4(0.f, 0.f, 0.f, 0.f);
    v = warp_sum3(q.x, q.y, q.z);
  }
  return make_float3(__shfl_sync(0xFFFFFFFFu, v, 0), __shfl_sync(0xFFFFFFFFu, v, 8), __shfl_sync(0xFFFFFFFFu, v, 16));
}
__device__ __forceinline__ float block_sum(float s, float* red) {
  const int lane = threadIdx.x & 31, warps = int(blockDim.x) >> 5;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, o);
  if (warps > 1) {
    if (lane == 0) red[threadIdx.x >> 5] = s;
    __syncthreads();
    s = lane < warps ? red[lane] : 0.f;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, o);
  }
  return s;
}

__device__ __forceinline__ void copy_async(uint32_t dst, const void* src, int bytes) {   // 8 or 16 bytes, both aligned to them
  if (bytes == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
  else asm volatile("cp.async.ca.shared.global [%0], [%1], 8;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// Slots in shared memory for the vectors of a block's threads on their way.  `src` is where the thread's own vector is, `left`
// how many columns of the row there are from it on.
//
// bf16: MAXT slots of 16 bytes; a thread only ever touches its own.
// fp32: a vector is two pieces of 16 bytes.  The lanes of a warp copy its pieces in the order they have in memory, which is
// also theirs in the slots (each lane its own two: 32 passes of the load unit per copy instruction instead of 16: forward and
// backward of 8192 x 2048 took 66 and 72 us, 57 and 58 this way).
// So a warp's lanes have to meet between the end of the copies and the reads, and before the next copies.  Four lanes of
// eight read the second halves first: eight consecutive lanes then cover all banks.
template <typename T, int MAXT>
struct Slots;
template <int MAXT>
struct Slots<__nv_bfloat16, MAXT> {
  static constexpr int kBytes = MAXT * 16;
  static __device__ __forceinline__ void meet() {}
  static __device__ __forceinline__ void fetch(uint32_t smem, const __nv_bfloat16* src, int left) {
    if (left > 0) copy_async(smem + threadIdx.x * 16, src, 16);
  }
  static __device__ __forceinline__ Raw<__nv_bfloat16> take(const uint8_t* smem) {
    Raw<__nv_bfloat16> r;
    r.u = *reinterpret_cast<const uint4*>(smem + threadIdx.x * 16);
    return r;
  }
};
template <int MAXT>
struct Slots<float, MAXT> {
  static constexpr int kBytes = MAXT * 32;
  static __device__ __forceinline__ void meet() { __syncwarp(); }
  static __device__ __forceinline__ void fetch(uint32_t smem, const float* src, int left) {
    const int lane = int(threadIdx.x & 31);
#pragma unroll
    for (int q = 0; q < 2; ++q) {
      const int ahead = 128 * q - 4 * lane;   // this lane's piece, in columns from its own vector
      if (ahead < left) copy_async(smem + (threadIdx.x & ~31u) * 32 + q * 512 + lane * 16, src + ahead, 16);
    }
  }
  static __device__ __forceinline__ Raw<float> take(const uint8_t* smem) {
    const bool swap = threadIdx.x & 4;
    const uint8_t* o = smem + threadIdx.x * 32;
    const float4 x = *reinterpret_cast<const float4*>(o + (swap ? 16 : 0)), y = *reinterpret_cast<const float4*>(o + (swap ? 0 : 16));
    Raw<float> r;
    r.a = swap ? y : x;
    r.b = swap ? x : y;
    return r;
  }
};

// The weight vectors a column is multiplied with in every row: k = alpha gate w_post, w = w_pre.
template <typename T>
__device__ __forceinline__ void column_weights(const void* w_post, const void* gate, float alpha, int c, float2 (&k)[4]) {
  float2 v[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) k[e] = both(alpha);
  if (w_post) {
    load8(static_cast<const T*>(w_post) + c, v);
#pragma unroll
    for (int e = 0; e < 4; ++e) k[e] = mul2(k[e], v[e]);
  }
  if (gate) {
    load8(static_cast<const T*>(gate) + c, v);
#pragma unroll
    for (int e = 0; e < 4; ++e) k[e] = mul2(k[e], v[e]);
  }
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

// Persistent: a block walks the rows blockIdx.x, + gridDim.x, ...; a thread holds NV vectors of 8 columns, threadIdx.x +
// i * blockDim.x (16 consecutive lanes hold a group of an 8-bit checkpoint), and keeps their weights in registers as
// binary32.  (One block per row, the weights read and unpacked again for each, was bound by instructions: 431 per vector
// and 131 us at 16384 x 3072.)  With DEPTH > 0 a thread copies its vectors of the next DEPTH rows into shared memory
// asynchronously, into its own slots, so no barrier guards them.  FULL: every vector of every thread is inside the row.
template <typename T, int NV, int MAXT, int MINB, int DEPTH, bool JOIN, bool KEEP, bool FULL>
__global__ void __launch_bounds__(MAXT, MINB) norm_join_fwd_kernel(const FwdArgs a) {
  extern __shared__ __align__(16) uint8_t ring[];
  __shared__ float red[2][2][32];
  wait_for_launch_before();
  let_next_launch_start();
  using S = Slots<T, MAXT>;
  constexpr int kVecSlot = S::kBytes * (JOIN ? 2 : 1);
  const int ng = (a.cols + kGroup - 1) / kGroup, lane16 = threadIdx.x & 15;
  const float inv_n = 1.f / float(a.cols);
  const uint32_t ring0 = static_cast<uint32_t>(__cvta_generic_to_shared(ring));
  auto col_of = [&](int i) { return (int(threadIdx.x) + i * int(blockDim.x)) * kVec; };
  auto live = [&](int i) { return FULL || col_of(i) < a.cols; };
  auto fetch = [&](int64_t row, int stage) {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int64_t at = row * a.cols + col_of(i);
      const int left = FULL ? INT_MAX : a.cols - col_of(i);
      const uint32_t o = ring0 + (stage * NV + i) * kVecSlot;
      S::fetch(o, static_cast<const T*>(a.h) + at, left);
      if (JOIN) S::fetch(o + S::kBytes, static_cast<const T*>(a.b) + at, left);
    }
  };
  const int64_t step = gridDim.x;
#pragma unroll
  for (int s = 0; s < DEPTH; ++s) {
    if (blockIdx.x + s * step < a.rows) fetch(blockIdx.x + s * step, s);
    copies_commit();
  }
  float2 k[JOIN ? NV : 1][4], wp[NV][4];
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    if (!live(i)) continue;
    if (JOIN) column_weights<T>(a.w_post, a.gate, a.alpha, col_of(i), k[JOIN ? i : 0]);
    load8(static_cast<const T*>(a.w_pre) + col_of(i), wp[i]);
  }
  int turn = 0, stage = 0;
  for (int64_t row = blockIdx.x; row < a.rows; row += step, turn ^= 1) {
    const int64_t at = row * a.cols;
    Raw<T> h[NV], b[JOIN ? NV : 1];
    copies_wait<(DEPTH > 0 ? DEPTH - 1 : 0)>();
    S::meet();
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      h[i].zero();
      if (JOIN) b[JOIN ? i : 0].zero();
      if (!live(i)) continue;
      if (DEPTH > 0) {
        const uint8_t* o = ring + (stage * NV + i) * kVecSlot;
        h[i] = S::take(o);
        if (JOIN) b[JOIN ? i : 0] = S::take(o + S::kBytes);
      } else {
        h[i].load(static_cast<const T*>(a.h) + at + col_of(i));
        if (JOIN) b[JOIN ? i : 0].load(static_cast<const T*>(a.b) + at + col_of(i));
      }
    }
    float2 t[NV][4], bf[JOIN ? NV : 1][4];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      h[i].get(t[i]);
      if (JOIN) b[JOIN ? i : 0].get(bf[JOIN ? i : 0]);
    }
    if (KEEP) {
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        // the even lanes of a group take h's scale, the odd ones b's: the reciprocal is the dear part of it
        uint32_t mh = h[i].amax_bits(), mb = 0u;
        if (JOIN) {
          mb = b[JOIN ? i : 0].amax_bits();
          max_pair_over<T, 16>(mh, mb);
        } else {
          mh = max_over<16>(mh);
        }
        const GroupScale g = group_scale(JOIN && (lane16 & 1) ? mb : mh);
        const float inv_h = JOIN ? __shfl_sync(0xFFFFFFFFu, g.inv, threadIdx.x & 30) : g.inv;
        const float inv_b = JOIN ? __shfl_sync(0xFFFFFFFFu, g.inv, threadIdx.x | 1) : 0.f;
        const int c = col_of(i);
        if (lane16 < (JOIN ? 2 : 1) && (FULL || c - lane16 * kVec < a.cols))   // the group exists, whether or not this lane's vector does
          (JOIN && lane16 == 1 ? a.Bs : a.Hs)[row * ng + c / kGroup] = g.scale;
        if (!live(i)) continue;
        *reinterpret_cast<uint2*>(a.Hq + at + c) = encode8(t[i], inv_h);
        if (JOIN) *reinterpret_cast<uint2*>(a.Bq + at + c) = encode8(bf[JOIN ? i : 0], inv_b);
      }
    }
    if (JOIN) {
      float r_b = 1.f;
      if (a.w_post) {
        float2 s = both(0.f);
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e) s = fma2(bf[JOIN ? i : 0][e], bf[JOIN ? i : 0][e], s);
        r_b = rsqrtf(block_sum(s.x + s.y, red[turn][0]) * inv_n + a.eps);
        if (KEEP && threadIdx.x == 0) a.rstd_post[row] = r_b;
      }
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        if (!live(i)) continue;
#pragma unroll
        for (int e = 0; e < 4; ++e) t[i][e] = fma2(mul2(k[JOIN ? i : 0][e], both(r_b)), bf[JOIN ? i : 0][e], t[i][e]);
        store8(static_cast<T*>(a.h_out) + at + col_of(i), t[i]);
      }
    }
    float2 s = both(0.f);
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) s = fma2(t[i][e], t[i][e], s);
    const float r_t = rsqrtf(block_sum(s.x + s.y, red[turn][1]) * inv_n + a.eps);
    if (DEPTH > 0) {   // this stage's values are in registers: its slots take the row DEPTH turns on
      S::meet();
      if (row + DEPTH * step < a.rows) fetch(row + DEPTH * step, stage);
      copies_commit();
      if (++stage == DEPTH) stage = 0;
    }
    if (KEEP && threadIdx.x == 0) a.rstd_pre[row] = r_t;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      if (!live(i)) continue;
      float2 y[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) y[e] = mul2(wp[i][e], mul2(t[i][e], both(r_t)));
      store8(static_cast<T*>(a.y) + at + col_of(i), y);
    }
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

// Persistent like the forward; the column sums of a block's rows stay in registers.  Both means of a row come out of one
// reduction: with dt = a + f that, a = dh_next + r_t dy w_pre and f = -r_t m1,
//     sum(k dt bhat) = sum(k a bhat) + f sum(k that bhat),
// so a row costs one barrier instead of two.  The registers that the sums and the weights take leave room for few threads,
// too few to keep HBM busy with their own loads: hence the copies ahead (DEPTH rows; without them 193 us at 16384 x 3072).
template <typename T, int NV, int MAXT, int MINB, int DEPTH, bool JOIN, bool FULL>
__global__ void __launch_bounds__(MAXT, MINB) norm_join_bwd_kernel(const BwdArgs a) {
  extern __shared__ __align__(16) uint8_t ring[];
  __shared__ float4 red[2][32];
  wait_for_launch_before();
  let_next_launch_start();
  using S = Slots<T, MAXT>;
  constexpr int kCodes = MAXT * 8, kVecSlot = 2 * S::kBytes + (JOIN ? 2 : 1) * kCodes;   // dy, dh_next, codes of h and b
  const int ng = (a.cols + kGroup - 1) / kGroup;
  const float inv_n = 1.f / float(a.cols);
  const uint32_t ring0 = static_cast<uint32_t>(__cvta_generic_to_shared(ring));
  auto col_of = [&](int i) { return (int(threadIdx.x) + i * int(blockDim.x)) * kVec; };
  auto live = [&](int i) { return FULL || col_of(i) < a.cols; };
  auto fetch = [&](int64_t row, int stage) {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int64_t at = row * a.cols + col_of(i);
      const int left = FULL ? INT_MAX : a.cols - col_of(i);
      const uint32_t o = ring0 + (stage * NV + i) * kVecSlot;
      S::fetch(o, static_cast<const T*>(a.dy) + at, left);
      if (a.dh_next) S::fetch(o + S::kBytes, static_cast<const T*>(a.dh_next) + at, left);
      if (!live(i)) continue;
      copy_async(o + 2 * S::kBytes + threadIdx.x * 8, a.Hq + at, 8);
      if (JOIN) copy_async(o + 2 * S::kBytes + kCodes + threadIdx.x * 8, a.Bq + at, 8);
    }
  };
  const int64_t step = gridDim.x;
#pragma unroll
  for (int s = 0; s < DEPTH; ++s) {
    if (blockIdx.x + s * step < a.rows) fetch(blockIdx.x + s * step, s);
    copies_commit();
  }
  float2 k[JOIN ? NV : 1][4], wp[NV][4], sum_pre[NV][4], sum_c[JOIN ? NV : 1][4];
#pragma unroll
  for (int i = 0; i < NV; ++i) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      sum_pre[i][e] = both(0.f);
      if (JOIN) sum_c[JOIN ? i : 0][e] = both(0.f);
    }
    if (!live(i)) continue;
    if (JOIN) column_weights<T>(a.w_post, a.gate, a.alpha, col_of(i), k[JOIN ? i : 0]);
    load8(static_cast<const T*>(a.w_pre) + col_of(i), wp[i]);
  }
  // a row's scales are asked for one row ahead, when half of the row before is done (asked for at its start, they cost
  // registers and 10 %)
  struct RowScales {
    float hs[NV], bs[JOIN ? NV : 1], r_t, r_b;
  } next = {};
  next.r_b = 1.f;
  auto scales = [&](int64_t row) {
    if (row >= a.rows) return;
    next.r_t = __ldcg(a.rstd_pre + row);
    if (JOIN && a.w_post) next.r_b = __ldcg(a.rstd_post + row);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      if (!live(i)) continue;
      const int64_t g = row * ng + col_of(i) / kGroup;
      next.hs[i] = __ldcg(a.Hs + g);
      if (JOIN) next.bs[JOIN ? i : 0] = __ldcg(a.Bs + g);
    }
  };
  scales(blockIdx.x);
  int turn = 0, stage = 0;
  for (int64_t row = blockIdx.x; row < a.rows; row += step, turn ^= 1) {
    const int64_t at = row * a.cols;
    float2 that[NV][4], av[NV][4], bhat[JOIN ? NV : 1][4];
    float2 s0 = both(0.f), s1 = both(0.f), s2 = both(0.f);
    copies_wait<(DEPTH > 0 ? DEPTH - 1 : 0)>();
    S::meet();
    const RowScales now = next;
    const float rt = now.r_t, rb = now.r_b;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      if (!live(i)) continue;
      const int j = JOIN ? i : 0;
      float2 dy[4];
      uint2 hq, bq;
#pragma unroll
      for (int e = 0; e < 4; ++e) av[i][e] = both(0.f);
      if (DEPTH > 0) {
        const uint8_t* o = ring + (stage * NV + i) * kVecSlot;
        S::take(o).get(dy);
        if (a.dh_next) S::take(o + S::kBytes).get(av[i]);
        hq = *reinterpret_cast<const uint2*>(o + 2 * S::kBytes + threadIdx.x * 8);
        if (JOIN) bq = *reinterpret_cast<const uint2*>(o + 2 * S::kBytes + kCodes + threadIdx.x * 8);
      } else {
        const int64_t ac = at + col_of(i);
        load8(static_cast<const T*>(a.dy) + ac, dy);
        if (a.dh_next) load8(static_cast<const T*>(a.dh_next) + ac, av[i]);
        hq = __ldcg(reinterpret_cast<const uint2*>(a.Hq + ac));
        if (JOIN) bq = __ldcg(reinterpret_cast<const uint2*>(a.Bq + ac));
      }
      decode8(hq, now.hs[i], that[i]);
      if (JOIN) decode8(bq, now.bs[j] * rb, bhat[j]);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        float2 kb;
        if (JOIN) {
          kb = mul2(k[j][e], bhat[j][e]);
          that[i][e] = add2(that[i][e], kb);
        }
        that[i][e] = mul2(that[i][e], both(rt));
        const float2 gy = mul2(dy[e], wp[i][e]);
        s0 = fma2(gy, that[i][e], s0);
        sum_pre[i][e] = fma2(dy[e], that[i][e], sum_pre[i][e]);
        av[i][e] = fma2(both(rt), gy, av[i][e]);
        if (JOIN) {
          s1 = fma2(av[i][e], kb, s1);
          s2 = fma2(that[i][e], kb, s2);
        }
      }
    }
    scales(row + step);
    const float3 sums = block_sum3(s0.x + s0.y, s1.x + s1.y, s2.x + s2.y, red[turn]);
    if (DEPTH > 0) {   // this stage's values are in registers: its slots take the row DEPTH turns on
      S::meet();
      if (row + DEPTH * step < a.rows) fetch(row + DEPTH * step, stage);
      copies_commit();
      if (++stage == DEPTH) stage = 0;
    }
    const float f = -rt * sums.x * inv_n, m2 = JOIN ? (sums.y + f * sums.z) * inv_n : 0.f;
    // db = r_b (k dt - bhat m2); without w_post r_b is 1 and nothing is taken off
    const float r1 = a.w_post ? rb : 1.f, r2 = a.w_post ? -rb * m2 : 0.f;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      if (!live(i)) continue;
      const int j = JOIN ? i : 0;
      const int64_t ac = at + col_of(i);
#pragma unroll
      for (int e = 0; e < 4; ++e) av[i][e] = fma2(both(f), that[i][e], av[i][e]);
      store8(static_cast<T*>(a.dh) + ac, av[i]);
      if (JOIN) {
        float2 db[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          sum_c[j][e] = fma2(av[i][e], bhat[j][e], sum_c[j][e]);
          db[e] = mul2(mul2(k[j][e], av[i][e]), both(r1));
          if (a.w_post) db[e] = fma2(bhat[j][e], both(r2), db[e]);
        }
        store8(static_cast<T*>(a.db) + ac, db);
      }
    }
  }
  float* part = a.part + int64_t(blockIdx.x) * (JOIN ? 2 : 1) * a.cols;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    if (!live(i)) continue;
    store8(part + col_of(i), sum_pre[i]);
    if (JOIN) store8(part + a.cols + col_of(i), sum_c[JOIN ? i : 0]);
  }
}

// Adds the blocks' column sums in a fixed order: 32 columns by 32 strips of blocks per thread block, strips then added in
// order; turns c into the gradients of w_post and of the gate.
template <typename T>
__global__ void __launch_bounds__(1024) norm_join_columns_kernel(const float* part, int blocks, int cols, int planes, float alpha,
                                                                 const T* __restrict__ w_post, const T* __restrict__ gate,
                                                                 float* __restrict__ dw_pre, float* __restrict__ dw_post,
                                                                 float* __restrict__ dgate) {
  __shared__ float red[32][33];
  const int x = threadIdx.x & 31, y = threadIdx.x >> 5, plane = blockIdx.y;
  const int c = int(blockIdx.x) * 32 + x;
  float s = 0.f;
  wait_for_launch_before();
  let_next_launch_start();
  if (c < cols)
    for (int k = y; k < blocks; k += 16 * 32) {   // sixteen loads under way, added in order
      float v[16];
#pragma unroll
      for (int u = 0; u < 16; ++u) v[u] = k + 32 * u < blocks ? __ldcg(part + (int64_t(k + 32 * u) * planes + plane) * cols + c) : 0.f;
#pragma unroll
      for (int u = 0; u < 16; ++u) s += v[u];
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

// Vectors per thread, threads per block and blocks per SM for a row of `cols` columns (at most 32768).  `one`, `two`: up to
// how many threads one and two vectors are taken; `per_sm`: threads per SM at the registers the kernel is bounded to.
struct Shape { int nv, threads, blocks; };
Shape shape_of(int64_t rows, int64_t cols, int one, int two, int per_sm_1, int per_sm_2) {
  const int vecs = int(cols / kVec);
  const int nv = vecs <= one ? 1 : (vecs <= 2 * two ? 2 : 4), threads = round_warp((vecs + nv - 1) / nv);
  const int per_sm = std::max(1, std::min(16, (nv == 1 ? per_sm_1 : (nv == 2 ? per_sm_2 : 1024)) / threads));
  return Shape{nv, threads, int(std::min<int64_t>(rows, int64_t(sm_count()) * per_sm))};
}
Shape fwd_shape(int64_t rows, int64_t cols) { return shape_of(rows, cols, 384, 512, 1152, 512); }
Shape bwd_shape(int64_t rows, int64_t cols) { return shape_of(rows, cols, 384, 512, 768, 512); }
bool is_full(const Shape& s, int64_t cols) { return cols == int64_t(s.nv) * s.threads * kVec; }

template <typename K, typename A>
cudaError_t launch_rows(K kernel, DeviceOnce& once, const A& a, const Shape& s, int smem, cudaStream_t st) {
  if (smem > 0 && once.needed()) {
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
    if (e != cudaSuccess) return e;
    once.done();
  }
  return launch_lined_up(kernel, dim3(unsigned(s.blocks)), dim3(unsigned(s.threads)), size_t(smem), st, a);
}
template <typename T>
constexpr int depth_of() { return sizeof(T) == 2 ? 4 : 2; }   // rows ahead in the forward: the same bytes for both types

template <typename T, int NV, int MAXT, int MINB, int DEPTH, bool JOIN, bool KEEP, bool FULL>
cudaError_t launch_fwd(const FwdArgs& a, const Shape& s, cudaStream_t st) {
  static DeviceOnce once;
  return launch_rows(norm_join_fwd_kernel<T, NV, MAXT, MINB, DEPTH, JOIN, KEEP, FULL>, once, a, s,
                     DEPTH * NV * MAXT * 8 * int(sizeof(T)) * (JOIN ? 2 : 1), st);
}
template <typename T, bool JOIN, bool KEEP>
cudaError_t launch_fwd(const FwdArgs& a, cudaStream_t st) {
  const Shape s = fwd_shape(a.rows, a.cols);
  constexpr int D = depth_of<T>();
  if (s.nv == 1 && s.threads <= 128) return launch_fwd<T, 1, 128, 9, D, JOIN, KEEP, false>(a, s, st);
  if (s.nv == 1) return is_full(s, a.cols) ? launch_fwd<T, 1, 384, 3, D, JOIN, KEEP, true>(a, s, st) : launch_fwd<T, 1, 384, 3, D, JOIN, KEEP, false>(a, s, st);
  if (s.nv == 2 && s.threads <= 256) return launch_fwd<T, 2, 256, 2, D, JOIN, KEEP, false>(a, s, st);
  if (s.nv == 2) return launch_fwd<T, 2, 512, 1, D, JOIN, KEEP, false>(a, s, st);
  return launch_fwd<T, 4, 1024, 1, 0, JOIN, KEEP, false>(a, s, st);
}
template <typename T>
cudaError_t launch_fwd(const FwdArgs& a, cudaStream_t st) {
  if (a.b) return a.Hq ? launch_fwd<T, true, true>(a, st) : launch_fwd<T, true, false>(a, st);
  return a.Hq ? launch_fwd<T, false, true>(a, st) : launch_fwd<T, false, false>(a, st);
}

template <typename T, int NV, int MAXT, int MINB, int DEPTH, bool JOIN, bool FULL>
cudaError_t launch_bwd(const BwdArgs& a, const Shape& s, cudaStream_t st) {
  static DeviceOnce once;
  return launch_rows(norm_join_bwd_kernel<T, NV, MAXT, MINB, DEPTH, JOIN, FULL>, once, a, s,
                     DEPTH * NV * MAXT * (2 * 8 * int(sizeof(T)) + (JOIN ? 16 : 8)), st);
}
template <typename T, bool JOIN>
cudaError_t launch_bwd(const BwdArgs& a, cudaStream_t st) {
  const Shape s = bwd_shape(a.rows, a.cols);
  constexpr int D = 2;   // rows ahead; 3, 4 and 6 are 1 to 3 % slower (bf16, 16384 x 3072)
  if (s.nv == 1 && s.threads <= 128) return launch_bwd<T, 1, 128, 6, D, JOIN, false>(a, s, st);
  if (s.nv == 1) return is_full(s, a.cols) ? launch_bwd<T, 1, 384, 2, D, JOIN, true>(a, s, st) : launch_bwd<T, 1, 384, 2, D, JOIN, false>(a, s, st);
  if (s.nv == 2 && s.threads <= 256) return launch_bwd<T, 2, 256, 2, D, JOIN, false>(a, s, st);
  if (s.nv == 2) return launch_bwd<T, 2, 512, 1, D, JOIN, false>(a, s, st);
  return launch_bwd<T, 4, 1024, 1, 0, JOIN, false>(a, s, st);
}

}  // namespace

cudaError_t norm_join_fwd(const Rows& d, const void* h, const void* b, const void* w_post, const void* gate, const void* w_pre, void* h_out,
                          void* y, int8_t* Hq, float* Hs, int8_t* Bq, float* Bs, float* rstd_post, float* rstd_pre, float eps, float alpha,
                          cudaStream_t st) {
  FwdArgs a{h, b, w_post, gate, w_pre, h_out, y, Hq, Bq, Hs, Bs, rstd_post, rstd_pre, d.rows, int(d.cols), eps, alpha};
  return d.bf16 ? launch_fwd<__nv_bfloat16>(a, st) : launch_fwd<float>(a, st);
}

size_t norm_join_bwd_workspace_bytes(const Rows& d) { return size_t(bwd_shape(d.rows, d.cols).blocks) * 2 * size_t(d.cols) * 4; }

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
  const int blocks = bwd_shape(d.rows, d.cols).blocks;
  const float* part = a.part;
  if (d.bf16)
    return launch_lined_up(norm_join_columns_kernel<__nv_bfloat16>, grid, dim3(1024), 0, st, part, blocks, a.cols, planes, alpha,
                           static_cast<const __nv_bfloat16*>(w_post), static_cast<const __nv_bfloat16*>(gate), dw_pre, dw_post, dgate);
  return launch_lined_up(norm_join_columns_kernel<float>, grid, dim3(1024), 0, st, part, blocks, a.cols, planes, alpha,
                         static_cast<const float*>(w_post), static_cast<const float*>(gate), dw_pre, dw_post, dgate);
}

}  // namespace acx
