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
#include <atomic>
#include <climits>

#include "acx_internal.h"
#include "acx_q8.cuh"
#include "acx_tmap.h"
#include "acx_umma.cuh"

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

// Wide rows: a row is shared by the blocks of a cluster, each with its own columns.  A block sends its sums to all of them and
// adds what it gets in the order of the ranks.  Stores that count on the receiver's barrier order nothing else: a cluster
// barrier would first wait for all that the block has written to global memory (2000 x 16384 forward: 129 us
// with one, 87 this way).
// SUMS per row, each with slots for two rows in turn, since a peer may be one row ahead.
template <int SUMS>
struct Peers {
  float4 slot[2][SUMS][8];
  uint64_t bar[2][SUMS];
  int gave_up;

  __device__ __forceinline__ void start() {
    if (threadIdx.x == 0) {
      for (int k = 0; k < 2 * SUMS; ++k) ptx::mbar_init(ptx::smem_u32(&bar[0][0] + k), 1);
      gave_up = 0;
      ptx::fence_barrier_init();
    }
    ptx::cluster_sync_all();
  }
  // Ends when no block of the cluster sends any more.
  __device__ __forceinline__ void end() { ptx::cluster_sync_all(); }
  __device__ __forceinline__ float3 sum(float3 s, int turn, int which, uint32_t parity, uint32_t ranks, int* status) {
    const uint32_t mine = ptx::smem_u32(&bar[turn][which]);
    if (threadIdx.x == 0) ptx::mbar_arrive_expect_tx(mine, ranks * 16);
    if (threadIdx.x < ranks)
      asm volatile("st.async.weak.shared::cluster.mbarrier::complete_tx::bytes.v4.f32 [%0], {%1, %2, %3, %4}, [%5];" ::"r"(
                       ptx::map_to_rank(ptx::smem_u32(&slot[turn][which][ptx::cluster_ctarank()]), threadIdx.x)),
                   "f"(s.x), "f"(s.y), "f"(s.z), "f"(0.f), "r"(ptx::map_to_rank(mine, threadIdx.x))
                   : "memory");
    if (!ptx::mbar_wait_cluster(mine, parity, &gave_up)) {
      *static_cast<volatile int*>(&gave_up) = 1;
      atomicExch(status, kDevTimeout);
    }
    float3 r = make_float3(0.f, 0.f, 0.f);
    for (uint32_t k = 0; k < ranks; ++k) {
      const float4 q = slot[turn][which][k];
      r.x += q.x;
      r.y += q.y;
      r.z += q.z;
    }
    return r;
  }
};
template <>
struct Peers<0> {};

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
  unsigned rows;   // below 2^31: numbers of rows, also some steps past the last, fit 32 bits
  int cols;
  float eps, alpha;
  int cluster;   // blocks that share a row (1 unless WIDE)
  int* status;
};

// Persistent: a block walks the rows blockIdx.x, + gridDim.x, ...; a thread holds NV vectors of 8 columns, threadIdx.x +
// i * blockDim.x (16 consecutive lanes hold a group of an 8-bit checkpoint), and keeps their weights in registers as
// binary32.  (One block per row, the weights read and unpacked again for each, was bound by instructions: 431 per vector
// and 131 us at 16384 x 3072.)  The vectors of the next DEPTH rows are on their way into
// shared memory meanwhile (see Slots).  FULL: every vector of every thread is inside the row.  WIDE: see Peers.
// 16384 x 3072 bf16: 87 us, 89 % of the copy rate.
template <typename T, int NV, int MAXT, int MINB, int DEPTH, bool JOIN, bool KEEP, bool FULL, bool WIDE>
__global__ void __launch_bounds__(MAXT, MINB) norm_join_fwd_kernel(const FwdArgs a) {
  extern __shared__ __align__(16) uint8_t ring[];
  __shared__ float red[2][2][32];
  __shared__ Peers<WIDE ? 2 : 0> peers;
  wait_for_launch_before();
  let_next_launch_start();
  using S = Slots<T, MAXT>;
  constexpr int kVecSlot = S::kBytes * (JOIN ? 2 : 1);
  const int ng = (a.cols + kGroup - 1) / kGroup, lane16 = threadIdx.x & 15;
  const float inv_n = 1.f / float(a.cols);
  const uint32_t ring0 = static_cast<uint32_t>(__cvta_generic_to_shared(ring));
  const int rank = WIDE ? int(blockIdx.x) % a.cluster : 0, first = rank * NV * int(blockDim.x);   // of this block's vectors
  const unsigned row0 = WIDE ? blockIdx.x / unsigned(a.cluster) : blockIdx.x;
  auto col_of = [&](int i) { return (first + int(threadIdx.x) + i * int(blockDim.x)) * kVec; };
  auto live = [&](int i) { return FULL || col_of(i) < a.cols; };
  auto fetch = [&](unsigned row, int stage) {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int64_t at = int64_t(row) * a.cols + col_of(i);
      const int left = FULL ? INT_MAX : a.cols - col_of(i);
      const uint32_t o = ring0 + (stage * NV + i) * kVecSlot;
      S::fetch(o, static_cast<const T*>(a.h) + at, left);
      if (JOIN) S::fetch(o + S::kBytes, static_cast<const T*>(a.b) + at, left);
    }
  };
  const unsigned step = WIDE ? gridDim.x / unsigned(a.cluster) : gridDim.x;
#pragma unroll
  for (int s = 0; s < DEPTH; ++s) {
    if (row0 + s * step < a.rows) fetch(row0 + s * step, s);
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
  uint32_t parity = 0;   // of the barriers of this turn
  if constexpr (WIDE) peers.start();
  for (unsigned row = row0; row < a.rows; row += step, parity ^= turn, turn ^= 1) {
    const int64_t at = int64_t(row) * a.cols;
    Raw<T> h[NV], b[JOIN ? NV : 1];
    copies_wait<DEPTH - 1>();
    S::meet();
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      h[i].zero();
      if (JOIN) b[JOIN ? i : 0].zero();
      if (!live(i)) continue;
      const uint8_t* o = ring + (stage * NV + i) * kVecSlot;
      h[i] = S::take(o);
      if (JOIN) b[JOIN ? i : 0] = S::take(o + S::kBytes);
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
          (JOIN && lane16 == 1 ? a.Bs : a.Hs)[int64_t(row) * ng + c / kGroup] = g.scale;
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
        float sum = block_sum(s.x + s.y, red[turn][0]);
        if constexpr (WIDE) sum = peers.sum(make_float3(sum, 0.f, 0.f), turn, 0, parity, a.cluster, a.status).x;
        r_b = rsqrtf(sum * inv_n + a.eps);
        if (KEEP && threadIdx.x == 0 && rank == 0) a.rstd_post[row] = r_b;
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
    float sum = block_sum(s.x + s.y, red[turn][1]);
    if constexpr (WIDE) sum = peers.sum(make_float3(sum, 0.f, 0.f), turn, 1, parity, a.cluster, a.status).x;
    const float r_t = rsqrtf(sum * inv_n + a.eps);
    // this stage's values are in registers: its slots take the row DEPTH turns on
    S::meet();
    if (row + DEPTH * step < a.rows) fetch(row + DEPTH * step, stage);
    copies_commit();
    if (++stage == DEPTH) stage = 0;
    if (KEEP && threadIdx.x == 0 && rank == 0) a.rstd_pre[row] = r_t;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      if (!live(i)) continue;
      float2 y[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) y[e] = mul2(wp[i][e], mul2(t[i][e], both(r_t)));
      store8(static_cast<T*>(a.y) + at + col_of(i), y);
    }
  }
  if constexpr (WIDE) peers.end();
}

struct BwdArgs {
  const void *dy, *dh_next, *w_post, *gate, *w_pre;
  const int8_t *Hq, *Bq;
  const float *Hs, *Bs, *rstd_post, *rstd_pre;
  void *dh, *db;
  float* part;   // [gridDim.x][JOIN ? 2 : 1][cols]: this block's column sums of dy that and of dt bhat
  unsigned rows;   // below 2^31: numbers of rows, also some steps past the last, fit 32 bits
  int cols;
  float alpha;
  int cluster;   // blocks that share a row (1 unless WIDE)
  int* status;
};

// Persistent like the forward; the column sums of a block's rows stay in registers.  Both means of a row come out of one
// reduction: with dt = a + f that, a = dh_next + r_t dy w_pre and f = -r_t m1,
//     sum(k dt bhat) = sum(k a bhat) + f sum(k that bhat),
// so a row costs one barrier instead of two.  The registers that the sums and the weights take leave room for few threads,
// too few to keep HBM busy with their own loads: hence the copies ahead (DEPTH rows; 16384 x 3072 bf16: 97 us, 193 without).
template <typename T, int NV, int MAXT, int MINB, int DEPTH, bool JOIN, bool FULL, bool WIDE>
__global__ void __launch_bounds__(MAXT, MINB) norm_join_bwd_kernel(const BwdArgs a) {
  extern __shared__ __align__(16) uint8_t ring[];
  __shared__ float4 red[2][32];
  __shared__ Peers<WIDE ? 1 : 0> peers;
  wait_for_launch_before();
  let_next_launch_start();
  using S = Slots<T, MAXT>;
  constexpr int kCodes = MAXT * 8, kVecSlot = 2 * S::kBytes + (JOIN ? 2 : 1) * kCodes;   // dy, dh_next, codes of h and b
  const int ng = (a.cols + kGroup - 1) / kGroup;
  const float inv_n = 1.f / float(a.cols);
  const uint32_t ring0 = static_cast<uint32_t>(__cvta_generic_to_shared(ring));
  const int rank = WIDE ? int(blockIdx.x) % a.cluster : 0, first = rank * NV * int(blockDim.x);   // of this block's vectors
  const unsigned row0 = WIDE ? blockIdx.x / unsigned(a.cluster) : blockIdx.x;
  auto col_of = [&](int i) { return (first + int(threadIdx.x) + i * int(blockDim.x)) * kVec; };
  auto live = [&](int i) { return FULL || col_of(i) < a.cols; };
  auto fetch = [&](unsigned row, int stage) {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int64_t at = int64_t(row) * a.cols + col_of(i);
      const int left = FULL ? INT_MAX : a.cols - col_of(i);
      const uint32_t o = ring0 + (stage * NV + i) * kVecSlot;
      S::fetch(o, static_cast<const T*>(a.dy) + at, left);
      if (a.dh_next) S::fetch(o + S::kBytes, static_cast<const T*>(a.dh_next) + at, left);
      if (!live(i)) continue;
      copy_async(o + 2 * S::kBytes + threadIdx.x * 8, a.Hq + at, 8);
      if (JOIN) copy_async(o + 2 * S::kBytes + kCodes + threadIdx.x * 8, a.Bq + at, 8);
    }
  };
  const unsigned step = WIDE ? gridDim.x / unsigned(a.cluster) : gridDim.x;
#pragma unroll
  for (int s = 0; s < DEPTH; ++s) {
    if (row0 + s * step < a.rows) fetch(row0 + s * step, s);
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
  auto scales = [&](unsigned row) {
    if (row >= a.rows) return;
    next.r_t = __ldcg(a.rstd_pre + row);
    if (JOIN && a.w_post) next.r_b = __ldcg(a.rstd_post + row);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      if (!live(i)) continue;
      const int64_t g = int64_t(row) * ng + col_of(i) / kGroup;
      next.hs[i] = __ldcg(a.Hs + g);
      if (JOIN) next.bs[JOIN ? i : 0] = __ldcg(a.Bs + g);
    }
  };
  scales(row0);
  int turn = 0, stage = 0;
  uint32_t parity = 0;   // of the barriers of this turn
  if constexpr (WIDE) peers.start();
  for (unsigned row = row0; row < a.rows; row += step, parity ^= turn, turn ^= 1) {
    const int64_t at = int64_t(row) * a.cols;
    float2 that[NV][4], av[NV][4], bhat[JOIN ? NV : 1][4];
    float2 s0 = both(0.f), s1 = both(0.f), s2 = both(0.f);
    copies_wait<DEPTH - 1>();
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
      const uint8_t* o = ring + (stage * NV + i) * kVecSlot;
      S::take(o).get(dy);
      if (a.dh_next) S::take(o + S::kBytes).get(av[i]);
      hq = *reinterpret_cast<const uint2*>(o + 2 * S::kBytes + threadIdx.x * 8);
      if (JOIN) bq = *reinterpret_cast<const uint2*>(o + 2 * S::kBytes + kCodes + threadIdx.x * 8);
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
    float3 sums = block_sum3(s0.x + s0.y, s1.x + s1.y, s2.x + s2.y, red[turn]);
    if constexpr (WIDE) sums = peers.sum(sums, turn, 0, parity, a.cluster, a.status);
    // this stage's values are in registers: its slots take the row DEPTH turns on
    S::meet();
    if (row + DEPTH * step < a.rows) fetch(row + DEPTH * step, stage);
    copies_commit();
    if (++stage == DEPTH) stage = 0;
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
  if constexpr (WIDE) peers.end();
  float* part = a.part + int64_t(row0) * (JOIN ? 2 : 1) * a.cols;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    if (!live(i)) continue;
    store8(part + col_of(i), sum_pre[i]);
    if (JOIN) store8(part + a.cols + col_of(i), sum_c[JOIN ? i : 0]);
  }
}

// Adds the blocks' column sums in a fixed order: 32 columns by STRIPS strips of blocks per thread block, strips then added in
// order; turns c into the gradients of w_post and of the gate.
template <typename T, int STRIPS>
__global__ void __launch_bounds__(32 * STRIPS) norm_join_columns_kernel(const float* part, int blocks, int cols, int planes, float alpha,
                                                                 const T* __restrict__ w_post, const T* __restrict__ gate,
                                                                 float* __restrict__ dw_pre, float* __restrict__ dw_post,
                                                                 float* __restrict__ dgate) {
  __shared__ float red[STRIPS][33];
  const int x = threadIdx.x & 31, y = threadIdx.x >> 5, plane = blockIdx.y;
  const int c = int(blockIdx.x) * 32 + x;
  float s = 0.f;
  wait_for_launch_before();
  let_next_launch_start();
  if (c < cols)
    for (int k = y; k < blocks; k += 16 * STRIPS) {   // sixteen loads under way, added in order
      float v[16];
#pragma unroll
      for (int u = 0; u < 16; ++u) v[u] = k + STRIPS * u < blocks ? __ldcg(part + (int64_t(k + STRIPS * u) * planes + plane) * cols + c) : 0.f;
#pragma unroll
      for (int u = 0; u < 16; ++u) s += v[u];
    }
  red[y][x] = s;
  __syncthreads();
  if (y != 0 || c >= cols) return;
  s = 0.f;
#pragma unroll
  for (int k = 0; k < STRIPS; ++k) s += red[k][x];
  if (plane == 0) {
    if (dw_pre) dw_pre[c] = s;
    return;
  }
  s *= alpha;
  if (dw_post) dw_post[c] = gate ? s * float(gate[c]) : s;
  if (dgate) dgate[c] = w_post ? s * float(w_post[c]) : s;
}

int round_warp(int threads) { return (threads + 31) / 32 * 32; }

// Vectors per thread, threads per block, blocks that share a row, and rows under way.
struct Shape { int nv, threads, cluster, blocks; };
constexpr int kOneVec = 384;     // threads of a block with one vector each, at most
constexpr int kTwoVecs = 512;    // with two: alone on its SM above 256
// `per_sm`: threads per SM at the registers that the kernels with one and with two vectors are bounded to.
struct PerSm { int one, two; };
Shape shape_of(int64_t rows, int vecs, int nv, int cluster, PerSm p) {
  const int threads = round_warp((vecs + nv * cluster - 1) / (nv * cluster));
  const int per_sm = std::max(1, std::min(16, (nv == 1 ? p.one : p.two) / threads));
  return Shape{nv, threads, cluster, int(std::min<int64_t>(rows, int64_t(sm_count()) * per_sm / cluster))};
}
// Forward: rows of more than 8192 columns are shared by three to eight blocks of 256 threads with two vectors each.  (One block,
// four vectors of 1024 threads: its values spilled, 2000 x 16384 took 142 us, shared by four 87.  Narrower rows are faster
// alone: 8192 x 8192 110 us, shared by four 182.)
Shape fwd_shape(int64_t rows, int64_t cols) {
  const int vecs = int(cols / kVec);
  return shape_of(rows, vecs, vecs <= kOneVec ? 1 : 2, vecs <= 2 * kTwoVecs ? 1 : (vecs + 511) / 512, PerSm{1152, 512});
}
// Backward: the sums take more registers, so rows are shared as soon as one vector per thread does for two blocks (8192 x 6144:
// 152 us, 164 in one block with two vectors) and, from 8192 columns on, for four or eight (4096 x 12288: 164 us, 250 with two
// vectors in three blocks, 512 with four in one; 2000 x 16384: 117, 376 in one).  Between the two one block of two vectors
// per thread is faster (8192 x 8192: 181 us, 221 shared by four).
Shape bwd_shape(int64_t rows, int64_t cols) {
  const int vecs = int(cols / kVec);
  int cluster = 1;
  if ((vecs > kTwoVecs && vecs <= 2 * kOneVec) || vecs > 2 * kTwoVecs)
    while (cluster < 8 && cluster * kOneVec < vecs) cluster *= 2;
  return shape_of(rows, vecs, vecs <= cluster * kOneVec ? 1 : 2, cluster, PerSm{768, 512});
}
bool is_full(const Shape& s, int64_t cols) { return cols == int64_t(s.nv) * s.threads * kVec; }

// How many clusters of a size and of blocks of so many warps run at once on a device, asked once for each: the last clusters of
// a persistent grid that does not fit would start when the others end and double the time.
constexpr int kMaxWarps = kOneVec / 32;
using ClusterLimit = DeviceNumbers<9 * (kMaxWarps + 1)>;

// s.blocks: at most as many rows under way as run at once.
template <typename K, typename A>
cudaError_t launch_rows(K kernel, DeviceOnce& once, ClusterLimit& limit, const A& a, Shape& s, int smem, cudaStream_t st) {
  if (once.needed()) {
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
    if (e != cudaSuccess) return e;
    once.done();
  }
  if (s.cluster > 1) {
    std::atomic<int>* known = limit.here();
    if (known) known += s.cluster * (kMaxWarps + 1) + s.threads / 32;
    int n = known ? known->load(std::memory_order_relaxed) : 0;
    if (n == 0) {
      cudaLaunchConfig_t cfg = {};
      cudaLaunchAttribute attr[1];
      cfg.gridDim = dim3(unsigned(s.cluster));
      cfg.blockDim = dim3(unsigned(s.threads));
      cfg.dynamicSmemBytes = size_t(smem);
      attr[0].id = cudaLaunchAttributeClusterDimension;
      attr[0].val.clusterDim = {unsigned(s.cluster), 1, 1};
      cfg.attrs = attr;
      cfg.numAttrs = 1;
      const cudaError_t e = cudaOccupancyMaxActiveClusters(&n, kernel, &cfg);
      if (e != cudaSuccess) return e;
      n = std::max(n, 1);
      if (known) known->store(n, std::memory_order_relaxed);
    }
    s.blocks = std::min(s.blocks, n);
  }
  return launch_lined_up_in_clusters(unsigned(s.cluster), kernel, dim3(unsigned(s.blocks * s.cluster)), dim3(unsigned(s.threads)), size_t(smem), st, a);
}
template <typename T>
constexpr int depth_of() { return sizeof(T) == 2 ? 4 : 2; }   // rows ahead in the forward: the same bytes for both types

template <typename T, int NV, int MAXT, int MINB, int DEPTH, bool JOIN, bool KEEP, bool FULL, bool WIDE = false>
cudaError_t launch_fwd(const FwdArgs& a, Shape s, cudaStream_t st) {
  static DeviceOnce once;
  static ClusterLimit limit;
  return launch_rows(norm_join_fwd_kernel<T, NV, MAXT, MINB, DEPTH, JOIN, KEEP, FULL, WIDE>, once, limit, a, s,
                     DEPTH * NV * MAXT * 8 * int(sizeof(T)) * (JOIN ? 2 : 1), st);
}
template <typename T, bool JOIN, bool KEEP>
cudaError_t launch_fwd(const FwdArgs& a, cudaStream_t st) {
  const Shape s = fwd_shape(a.rows, a.cols);
  constexpr int D = depth_of<T>();
  if (s.cluster > 1) return launch_fwd<T, 2, 256, 2, D, JOIN, KEEP, false, true>(a, s, st);
  if (s.nv == 1 && s.threads <= 128) return launch_fwd<T, 1, 128, 9, D, JOIN, KEEP, false>(a, s, st);
  if (s.nv == 1) return is_full(s, a.cols) ? launch_fwd<T, 1, 384, 3, D, JOIN, KEEP, true>(a, s, st) : launch_fwd<T, 1, 384, 3, D, JOIN, KEEP, false>(a, s, st);
  if (s.nv == 2 && s.threads <= 256) return launch_fwd<T, 2, 256, 2, D, JOIN, KEEP, false>(a, s, st);
  return launch_fwd<T, 2, 512, 1, D, JOIN, KEEP, false>(a, s, st);
}
template <typename T>
cudaError_t launch_fwd(const FwdArgs& a, cudaStream_t st) {
  if (a.b) return a.Hq ? launch_fwd<T, true, true>(a, st) : launch_fwd<T, true, false>(a, st);
  return a.Hq ? launch_fwd<T, false, true>(a, st) : launch_fwd<T, false, false>(a, st);
}

template <typename T, int NV, int MAXT, int MINB, int DEPTH, bool JOIN, bool FULL, bool WIDE = false>
cudaError_t launch_bwd(const BwdArgs& a, Shape& s, cudaStream_t st) {
  static DeviceOnce once;
  static ClusterLimit limit;
  return launch_rows(norm_join_bwd_kernel<T, NV, MAXT, MINB, DEPTH, JOIN, FULL, WIDE>, once, limit, a, s,
                     DEPTH * NV * MAXT * (2 * 8 * int(sizeof(T)) + (JOIN ? 16 : 8)), st);
}
template <typename T, bool JOIN>
cudaError_t launch_bwd(const BwdArgs& a, Shape& s, cudaStream_t st) {
  constexpr int D = 2;   // rows ahead; 3, 4 and 6 are 1 to 3 % slower (bf16, 16384 x 3072)
  if (s.cluster > 1 && s.nv == 1) return launch_bwd<T, 1, kOneVec, 2, D, JOIN, false, true>(a, s, st);
  if (s.cluster > 1) return launch_bwd<T, 2, 256, 2, D, JOIN, false, true>(a, s, st);
  if (s.nv == 1 && s.threads <= 128) return launch_bwd<T, 1, 128, 6, D, JOIN, false>(a, s, st);
  if (s.nv == 1) return is_full(s, a.cols) ? launch_bwd<T, 1, 384, 2, D, JOIN, true>(a, s, st) : launch_bwd<T, 1, 384, 2, D, JOIN, false>(a, s, st);
  if (s.nv == 2 && s.threads <= 256) return launch_bwd<T, 2, 256, 2, D, JOIN, false>(a, s, st);
  return launch_bwd<T, 2, 512, 1, D, JOIN, false>(a, s, st);
}

}  // namespace

cudaError_t norm_join_fwd(const Rows& d, const void* h, const void* b, const void* w_post, const void* gate, const void* w_pre, void* h_out,
                          void* y, int8_t* Hq, float* Hs, int8_t* Bq, float* Bs, float* rstd_post, float* rstd_pre, float eps, float alpha,
                          cudaStream_t st) {
  FwdArgs a{h, b, w_post, gate, w_pre, h_out, y, Hq, Bq, Hs, Bs, rstd_post, rstd_pre, unsigned(d.rows), int(d.cols), eps, alpha, fwd_shape(d.rows, d.cols).cluster, nullptr};
  if (a.cluster > 1 && !(a.status = device_status_ptr())) return cudaErrorMemoryAllocation;
  return d.bf16 ? launch_fwd<__nv_bfloat16>(a, st) : launch_fwd<float>(a, st);
}

size_t norm_join_bwd_workspace_bytes(const Rows& d) { return size_t(bwd_shape(d.rows, d.cols).blocks) * 2 * size_t(d.cols) * 4; }

cudaError_t norm_join_bwd(const Rows& d, const void* dy, const void* dh_next, const void* w_post, const void* gate, const void* w_pre,
                          const int8_t* Hq, const float* Hs, const int8_t* Bq, const float* Bs, const float* rstd_post,
                          const float* rstd_pre, void* dh, void* db, float* dw_post, float* dgate, float* dw_pre, float alpha, void* ws,
                          cudaStream_t st) {
  Shape s = bwd_shape(d.rows, d.cols);
  BwdArgs a{dy, dh_next, w_post, gate, w_pre, Hq, Bq, Hs, Bs, rstd_post, rstd_pre, dh, db, static_cast<float*>(ws), unsigned(d.rows), int(d.cols), alpha, s.cluster, nullptr};
  if (s.cluster > 1 && !(a.status = device_status_ptr())) return cudaErrorMemoryAllocation;
  cudaError_t e;
  if (d.bf16) e = Bq ? launch_bwd<__nv_bfloat16, true>(a, s, st) : launch_bwd<__nv_bfloat16, false>(a, s, st);
  else e = Bq ? launch_bwd<float, true>(a, s, st) : launch_bwd<float, false>(a, s, st);
  if (e != cudaSuccess || (!dw_pre && !dw_post && !dgate)) return e;
  const int planes = Bq ? 2 : 1;
  const dim3 grid(unsigned((d.cols + 31) / 32), unsigned((dw_post || dgate) ? 2 : 1));
  const int blocks = s.blocks;
  const float* part = a.part;
  // wide rows: few sums for each of many columns, and more thread blocks of 32 strips than run at once
  const bool many = int64_t(grid.x) * grid.y > 2 * sm_count();
  if (d.bf16)
    return launch_lined_up(many ? norm_join_columns_kernel<__nv_bfloat16, 8> : norm_join_columns_kernel<__nv_bfloat16, 32>, grid,
                           dim3(many ? 256 : 1024), 0, st, part, blocks, a.cols, planes, alpha, static_cast<const __nv_bfloat16*>(w_post),
                           static_cast<const __nv_bfloat16*>(gate), dw_pre, dw_post, dgate);
  return launch_lined_up(many ? norm_join_columns_kernel<float, 8> : norm_join_columns_kernel<float, 32>, grid, dim3(many ? 256 : 1024), 0,
                         st, part, blocks, a.cols, planes, alpha, static_cast<const float*>(w_post), static_cast<const float*>(gate), dw_pre,
                         dw_post, dgate);
}

}  // namespace acx
