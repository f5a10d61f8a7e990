// Attention: the backward kernels.
//
// With dO and the forward's lse, and delta_i = sum over the columns of dO_i O_i,
//     P = 2^(x - lse),   dP = dO V^T,   dS = P (dP - delta) dx/ds,
//     dQ = scale dS K,   dK = scale dS^T Q,   dV = P^T dO.
// Two kernels, each with sums that no other work item adds to, so that no atomics are needed and results are reproducible bit for
// bit: one per tile of queries (three products: S, dP, dQ), one per tile of keys and key head (four: S^T, dP^T, dV, dK), which
// goes through the query heads of the group and the queries that see the tile.  The price is that S and dP are computed twice: seven
// products instead of five.
//
// Queries (dQ): S is double buffered, dP and dQ are not: 4 x 128 columns of tensor memory.  Lane = query; eight warps take 64
// keys each of their 32 rows.  dS is written over dP as bf16 and multiplied with K from there.
// Keys (dK, dV): S^T, dP^T, dV, dK fill the tensor memory.  Lane = key, columns = queries.  While the exponentials of a tile are
// taken the tensor core runs dK of the tile before and dP^T, while dS is formed dV and the next S^T.
//
// A query that sees one key only has p = 1 and no gradient through its scores: exactly zero, not the difference of two roundings.
//
// Where a batch has few key tiles for the SMs a group's query heads are dealt to several work items, whose fp32 sums a last kernel adds
// in a fixed order.
#include <algorithm>

#include "acx_attn.cuh"
#include "acx_tmap.h"

namespace acx {
namespace attn {
namespace {

constexpr int kThreads = 384;
constexpr int kRowWarps = 8;
constexpr int kPanel = 64;        // columns of a tile that one warp takes

// ------------------------------------------------------------------------------------------------------------------ delta
// delta[head][token] = sum of dO O over the head's columns.  Sixteen lanes per row.
constexpr int kDeltaTokens = 64, kDeltaThreads = 256;
__global__ void __launch_bounds__(kDeltaThreads) attn_delta_kernel(const __nv_bfloat16* __restrict__ O, int64_t ldo,
                                                                   const __nv_bfloat16* __restrict__ dO, int64_t lddo, int tokens, int d,
                                                                   float* __restrict__ delta) {
  __shared__ float out[kDeltaTokens];
  wait_for_launch_before();
  let_next_launch_start();
  const int head = blockIdx.y, t0 = blockIdx.x * kDeltaTokens, sub = threadIdx.x & 15;
#pragma unroll
  for (int i = 0; i < kDeltaTokens / 16; ++i) {
    const int r = i * 16 + int(threadIdx.x >> 4);
    float sum = 0.f;
    if (t0 + r < tokens && 8 * sub < d) {
      float2 a[4], b[4];
      q8::load8(O + int64_t(t0 + r) * ldo + int64_t(head) * d + 8 * sub, a);
      q8::load8(dO + int64_t(t0 + r) * lddo + int64_t(head) * d + 8 * sub, b);
#pragma unroll
      for (int k = 0; k < 4; ++k) sum = fmaf(a[k].x, b[k].x, fmaf(a[k].y, b[k].y, sum));
    }
#pragma unroll
    for (int o = 8; o > 0; o >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, o);
    if (sub == 0) out[r] = sum;
  }
  __syncthreads();
  if (threadIdx.x < kDeltaTokens && t0 + int(threadIdx.x) < tokens) delta[int64_t(head) * tokens + t0 + threadIdx.x] = out[threadIdx.x];
}

struct Ring {   // stages of a tile each
  int count, stage = 0;
  uint32_t phase = 0;
  struct Slot { int stage; uint32_t phase; };
  __device__ explicit Ring(int n) : count(n) {}
  __device__ Slot next() {
    const Slot s{stage, phase};
    if (++stage == count) { stage = 0; phase ^= 1u; }
    return s;
  }
};

__device__ __forceinline__ Item fetch_item(const Params& p, int k) {
  const int4 v = __ldcg(reinterpret_cast<const int4*>(p.items) + k);
  return Item{v.x, v.y, v.z, v.w};
}

// ---------------------------------------------------------------------------------------------------------------- queries
template <int HD>
struct QuerySmem {
  static constexpr int kK = HD == 128 ? 3 : 4, kV = HD == 128 ? 2 : 4;   // stages
  static constexpr int kTiles = 2 + kK + kV, kBars = kTiles * Tile<HD>::kBytes, kBytes = kBars + 512 + 1024;
  static_assert(kBytes <= 232448, "shared memory of one CTA");
};

template <int HD, bool CAP, bool BIAS>
__global__ void __launch_bounds__(kThreads, 1)
    attn_dq_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v,
                   const __grid_constant__ CUtensorMap map_do, const Params p) {
  using T = Tile<HD>;
  using M = QuerySmem<HD>;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t base = (ptx::smem_u32(smem_raw) + 1023u) & ~1023u;
  uint8_t* gen = smem_raw + (base - ptx::smem_u32(smem_raw));
  const uint32_t q_tile = base, do_tile = base + T::kBytes, k_tiles = base + 2 * T::kBytes, v_tiles = k_tiles + M::kK * T::kBytes;
  const uint32_t bars = base + M::kBars;
  auto k_full = [&](int s) { return bars + 8u * s; };
  auto k_empty = [&](int s) { return bars + 32 + 8u * s; };
  auto v_full = [&](int s) { return bars + 64 + 8u * s; };
  auto v_empty = [&](int s) { return bars + 96 + 8u * s; };
  const uint32_t q_full = bars + 128, q_empty = bars + 136, dp_full = bars + 160, ds_full = bars + 168, out_full = bars + 176, out_free = bars + 184,
                 done = bars + 192;
  auto s_full = [&](int b) { return bars + 144 + 8u * b; };
  volatile uint32_t* tmem_slot = reinterpret_cast<volatile uint32_t*>(gen + M::kBars + 200);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(gen + M::kBars + 204);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

  if (threadIdx.x == 0) {
    for (int s = 0; s < 4; ++s) {
      ptx::mbar_init(k_full(s), 1);
      ptx::mbar_init(k_empty(s), 1);
      ptx::mbar_init(v_full(s), 1);
      ptx::mbar_init(v_empty(s), 1);
    }
    ptx::mbar_init(q_full, 1);
    ptx::mbar_init(q_empty, 1);
    ptx::mbar_init(s_full(0), 1);
    ptx::mbar_init(s_full(1), 1);
    ptx::mbar_init(dp_full, 1);
    ptx::mbar_init(ds_full, kRowWarps);
    ptx::mbar_init(out_full, 1);
    ptx::mbar_init(out_free, kRowWarps);
    ptx::mbar_init(done, 1);
    *abort_flag = 0;
    ptx::fence_barrier_init();   // no prefetch of the tensor maps: a block without work would leave with it in flight
  }
  if (warp == 1) {
    ptx::tmem_alloc(bars + 200, 512);
    ptx::tmem_relinquish_alloc_permit();
  }
  ptx::tcgen05_fence_before_sync();
  __syncthreads();
  ptx::tcgen05_fence_after_sync();
  const uint32_t tmem = *tmem_slot;
  auto tmem_s = [&](int b) { return tmem + 128u * b; };
  const uint32_t tmem_dp = tmem + 256, tmem_dq = tmem + 384;
  wait_for_launch_before();
  let_next_launch_start();
  const int units = __ldcg(&p.plan->tiles) * p.heads;
  auto give_up = [&]() {
    *abort_flag = 1;
    atomicExch(p.status, kDevTimeout);
  };
  auto key_tiles = [&](const Item& t) {
    return ((p.causal ? max(min(t.row0 + kRows, t.end), t.prefix) : t.end) - t.start + kRows - 1) / kRows;
  };

  if (warp == 0) {
    // ---------------------------------------------------------------------------------------------------- copies
    if (lane == 0) {
      Ring rk(M::kK), rv(M::kV);
      int it = 0;
      bool ok = true;
      auto push = [&](Ring& r, uint32_t full, uint32_t empty, uint32_t tiles, const CUtensorMap* map, int head, int row) {
        const Ring::Slot s = r.next();
        if (!ptx::mbar_wait(empty + 8u * s.stage, s.phase ^ 1u, abort_flag)) { give_up(); ok = false; return; }
        ptx::mbar_arrive_expect_tx(full + 8u * s.stage, T::kBytes);
        T::load(tiles + s.stage * T::kBytes, map, full + 8u * s.stage, head, row);
      };
      for (int u = blockIdx.x; ok && u < units; u += gridDim.x, ++it) {
        const Item t = fetch_item(p, u / p.heads);
        const int h = u % p.heads, g = h / p.group, n = key_tiles(t);
        if (!ptx::mbar_wait(q_empty, (it & 1) ^ 1u, abort_flag)) { give_up(); ok = false; break; }
        ptx::mbar_arrive_expect_tx(q_full, 2 * T::kBytes);
        T::load(q_tile, &map_q, q_full, h, t.row0);
        T::load(do_tile, &map_do, q_full, h, t.row0);
        for (int j = 0; ok && j < n; ++j) {
          push(rk, k_full(0), k_empty(0), k_tiles, &map_k, g, t.start + j * kRows);
          if (ok) push(rv, v_full(0), v_empty(0), v_tiles, &map_v, g, t.start + j * kRows);
        }
      }
      if (!ok) {   // copies in flight land before the CTA leaves: one limit, well above a copy's time
        const uint64_t t0 = ptx::globaltimer_ns();
        while (ptx::globaltimer_ns() - t0 < 10000000ull) {}
      }
    }
    __syncwarp();
  } else if (warp == 1) {
    // ---------------------------------------------------------------------------------------------------- products
    if (lane == 0) {
      Ring rk(M::kK), rv(M::kV);
      int it = 0, turns = 0;
      bool ok = true;
      const int d16 = (p.d + 15) / 16;
      auto wait = [&](uint32_t bar, uint32_t parity) {
        if (ok && !ptx::mbar_wait(bar, parity, abort_flag)) { give_up(); ok = false; }
        return ok;
      };
      for (int u = blockIdx.x; ok && u < units; u += gridDim.x, ++it) {
        const Item t = fetch_item(p, u / p.heads);
        const int n = key_tiles(t);
        // K of tile j is here: rows behind the document's end become zeros (dS K sums over them)
        auto ready = [&](Ring::Slot k, int j) {
          if (!wait(k_full(k.stage), k.phase)) return false;
          const int left = t.end - (t.start + j * kRows);
          if (left < kRows && left % 16) T::zero_rows(gen + (k_tiles - base) + k.stage * T::kBytes, left, (left + 15) & ~15);
          ptx::tcgen05_fence_after_sync();
          return true;
        };
        auto scores = [&](Ring::Slot k, int turn) {
          scores_mma<HD>(tmem_s(turn & 1), q_tile, k_tiles + k.stage * T::kBytes, d16);
          ptx::umma_commit(s_full(turn & 1));
        };
        auto dprobs = [&](Ring::Slot v) {
          scores_mma<HD>(tmem_dp, do_tile, v_tiles + v.stage * T::kBytes, d16);
          ptx::umma_commit(dp_full);
          ptx::umma_commit(v_empty(v.stage));
        };
        wait(q_full, it & 1);
        Ring::Slot k = rk.next(), k_next = k, v = rv.next();
        if (!ready(k, 0)) break;
        scores(k, turns);
        if (!wait(v_full(v.stage), v.phase)) break;
        ptx::tcgen05_fence_after_sync();
        dprobs(v);
        for (int j = 0; ok && j < n; ++j, ++turns) {
          if (j + 1 < n) {
            k_next = rk.next();
            if (!ready(k_next, j + 1)) break;
            scores(k_next, turns + 1);   // its buffer was read before the dS of the tile before
          }
          if (j == 0 && !wait(out_free, (it & 1) ^ 1u)) break;
          if (!wait(ds_full, turns & 1)) break;
          ptx::tcgen05_fence_after_sync();
          const int steps = min(kRows, t.end - (t.start + j * kRows) + 15) / 16;
          rows_mma<HD>(tmem_dq, tmem_dp, tmem_dp + kPanel, k_tiles + k.stage * T::kBytes, steps, d16, j > 0);
          ptx::umma_commit(k_empty(k.stage));
          if (j == n - 1) {
            ptx::umma_commit(out_full);
            ptx::umma_commit(q_empty);
          }
          if (j + 1 < n) {
            v = rv.next();
            if (!wait(v_full(v.stage), v.phase)) break;
            ptx::tcgen05_fence_after_sync();
            dprobs(v);
          }
          k = k_next;
        }
      }
      if (it > 0 || !ok) {
        ptx::umma_commit(done);
        const uint64_t t0 = ptx::globaltimer_ns();
        while (!ptx::mbar_try_wait(done, 0) && ptx::globaltimer_ns() - t0 < ptx::kWaitLimitNs) {}
      }
    }
    __syncwarp();
  } else if (warp >= 4) {
    // ---------------------------------------------------------------------------------------------------- rows
    const int panel = (warp - 4) >> 2, quarter = warp & 3;
    const uint32_t lanes = uint32_t(32 * quarter) << 16, col0 = kPanel * panel;
    int turns = 0, it = 0;
    bool ok = true;
    for (int u = blockIdx.x; ok && u < units; u += gridDim.x, ++it) {
      const Item t = fetch_item(p, u / p.heads);
      const int n = key_tiles(t), head = u % p.heads;
      const int row = t.row0 + 32 * quarter + lane;
      const int sees = p.causal ? min(max(row + 1, t.prefix), t.end) : t.end;
      const int all_see = p.causal ? min(max(t.row0 + 1, t.prefix), t.end) : t.end;
      const float slope2 = BIAS ? __ldg(p.slopes + head) * kLog2e : 0.f;
      const bool live = row < t.end;
      const int64_t at = int64_t(head) * p.tokens + row;
      const float lse2 = live ? __ldcg(p.lse + at) * kLog2e : 0.f, delta = live ? __ldcg(p.delta + at) : 0.f;
      const float one = sees - t.start > 1 ? 1.f : 0.f;
      for (int j = 0; j < n; ++j, ++turns) {
        if (!warp_wait(s_full(turns & 1), (turns >> 1) & 1, abort_flag)) { give_up(); ok = false; break; }
        ptx::tcgen05_fence_after_sync();
        uint32_t s[2][32];
#pragma unroll
        for (int c = 0; c < 2; ++c) ptx::tmem_ld_x32(tmem_s(turns & 1) + lanes + col0 + 32 * c, s[c]);
        tmem_loaded(s[0], s[1]);
        const int k0 = t.start + j * kRows + int(col0);
        const bool masked = k0 + kPanel > all_see;
        const int limit = sees - k0;
#pragma unroll
        for (int c = 0; c < 2; ++c)
#pragma unroll
          for (int i = 0; i < 32; ++i) {
            float slope = 1.f;
            float x;
            if (!CAP && !BIAS) x = fmaf(__uint_as_float(s[c][i]), p.c, -lse2);
            else x = exponent<CAP, BIAS>(p, __uint_as_float(s[c][i]), float(row - k0) - float(32 * c + i), slope2, &slope) - lse2;
            float w = exp2_fast(x);
            if (CAP) w *= slope;
            s[c][i] = __float_as_uint(w);
          }
        if (masked) {
#pragma unroll
          for (int c = 0; c < 2; ++c)
#pragma unroll
            for (int i = 0; i < 32; ++i) s[c][i] = 32 * c + i < limit ? __float_as_uint(__uint_as_float(s[c][i]) * one) : 0u;
        }
        if (!warp_wait(dp_full, turns & 1, abort_flag)) { give_up(); ok = false; break; }
        ptx::tcgen05_fence_after_sync();
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          uint32_t g[32], w[16];
          ptx::tmem_ld_x32(tmem_dp + lanes + col0 + 32 * c, g);
          tmem_loaded(g);
          // a masked key's dP may be anything (rows of another document): selected away, not multiplied
          if (masked) {
#pragma unroll
            for (int i = 0; i < 32; ++i) g[i] = 32 * c + i < limit ? g[i] : __float_as_uint(delta);
          }
#pragma unroll
          for (int i = 0; i < 16; ++i)
            w[i] = pack2(__uint_as_float(s[c][2 * i]) * (__uint_as_float(g[2 * i]) - delta),
                         __uint_as_float(s[c][2 * i + 1]) * (__uint_as_float(g[2 * i + 1]) - delta));
          ptx::tmem_st_x16(tmem_dp + lanes + col0 + 16 * c, w);
        }
        ptx::tmem_st_wait();
        ptx::tcgen05_fence_before_sync();
        __syncwarp();
        if (lane == 0) ptx::mbar_arrive(ds_full);
        __syncwarp();
      }
      if (!ok) break;
      if (!warp_wait(out_full, it & 1, abort_flag)) { give_up(); break; }
      ptx::tcgen05_fence_after_sync();
      // the panel's half of the head's columns
      __nv_bfloat16* out = p.dQ + int64_t(row) * p.lddq + int64_t(head) * p.d;
      uint32_t o[HD / 64][32];
#pragma unroll
      for (int c = 0; c < HD / 64; ++c) ptx::tmem_ld_x32(tmem_dq + lanes + HD / 2 * panel + 32 * c, o[c]);
      ptx::tmem_ld_wait();
#pragma unroll
      for (int c = 0; c < HD / 64; ++c) hand_over(o[c]);
      ptx::tcgen05_fence_before_sync();
      __syncwarp();
      if (lane == 0) ptx::mbar_arrive(out_free);
      __syncwarp();
#pragma unroll
      for (int c = 0; c < HD / 64; ++c) {
        const int at_col = HD / 2 * panel + 32 * c;
        if (live && at_col < p.d) store_bf16(out + at_col, o[c], p.scale, p.d - at_col);
      }
    }
  }
  zero_rows_outside(p, p.dQ, p.lddq, p.heads, nullptr, 0.f);
  __syncwarp();
  ptx::tcgen05_fence_before_sync();
  __syncthreads();
  if (warp == 1) {
    __syncwarp();
    ptx::tcgen05_fence_after_sync();
    ptx::tmem_dealloc(tmem, 512);
  }
}

// ------------------------------------------------------------------------------------------------------------------- keys
template <int HD>
struct KeySmem {
  static constexpr int kStages = 2;   // of Q and of dO each
  static constexpr int kTiles = 2 + 2 * kStages, kVec = kTiles * Tile<HD>::kBytes;
  static constexpr int kVecStages = 4, kVecBytes = 2 * kRows * 4;     // lse and delta of a tile of queries
  static constexpr int kBars = kVec + kVecStages * kVecBytes, kBytes = kBars + 512 + 1024;
  static_assert(kBytes <= 232448, "shared memory of one CTA");
};

template <int HD, bool CAP, bool BIAS>
__global__ void __launch_bounds__(kThreads, 1)
    attn_dkv_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v,
                    const __grid_constant__ CUtensorMap map_do, const Params p) {
  using T = Tile<HD>;
  using M = KeySmem<HD>;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t base = (ptx::smem_u32(smem_raw) + 1023u) & ~1023u;
  uint8_t* gen = smem_raw + (base - ptx::smem_u32(smem_raw));
  const uint32_t k_tile = base, v_tile = base + T::kBytes, q_tiles = base + 2 * T::kBytes, do_tiles = q_tiles + M::kStages * T::kBytes;
  const uint32_t bars = base + M::kBars;
  auto q_full = [&](int s) { return bars + 8u * s; };
  auto q_empty = [&](int s) { return bars + 16 + 8u * s; };
  auto do_full = [&](int s) { return bars + 32 + 8u * s; };
  auto do_empty = [&](int s) { return bars + 48 + 8u * s; };
  auto vec_full = [&](int s) { return bars + 64 + 8u * s; };
  auto vec_empty = [&](int s) { return bars + 96 + 8u * s; };
  const uint32_t kv_full = bars + 128, kv_empty = bars + 136, s_full = bars + 144, p_full = bars + 152, dp_full = bars + 160, ds_full = bars + 168,
                 out_full = bars + 176, out_free = bars + 184, done = bars + 192;
  volatile uint32_t* tmem_slot = reinterpret_cast<volatile uint32_t*>(gen + M::kBars + 200);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(gen + M::kBars + 204);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

  if (threadIdx.x == 0) {
    for (int s = 0; s < M::kStages; ++s) {
      ptx::mbar_init(q_full(s), 1);
      ptx::mbar_init(q_empty(s), 1);
      ptx::mbar_init(do_full(s), 1);
      ptx::mbar_init(do_empty(s), 1);
    }
    for (int s = 0; s < M::kVecStages; ++s) {
      ptx::mbar_init(vec_full(s), 1);
      ptx::mbar_init(vec_empty(s), kRowWarps);
    }
    ptx::mbar_init(kv_full, 1);
    ptx::mbar_init(kv_empty, 1);
    ptx::mbar_init(s_full, 1);
    ptx::mbar_init(p_full, kRowWarps);
    ptx::mbar_init(dp_full, 1);
    ptx::mbar_init(ds_full, kRowWarps);
    ptx::mbar_init(out_full, 1);
    ptx::mbar_init(out_free, kRowWarps);
    ptx::mbar_init(done, 1);
    *abort_flag = 0;
    ptx::fence_barrier_init();   // no prefetch of the tensor maps: a block without work would leave with it in flight
  }
  if (warp == 1) {
    ptx::tmem_alloc(bars + 200, 512);
    ptx::tmem_relinquish_alloc_permit();
  }
  ptx::tcgen05_fence_before_sync();
  __syncthreads();
  ptx::tcgen05_fence_after_sync();
  const uint32_t tmem = *tmem_slot;
  const uint32_t tmem_s = tmem, tmem_dp = tmem + 128, tmem_dv = tmem + 256, tmem_dk = tmem + 384;
  wait_for_launch_before();
  let_next_launch_start();
  const int per_tile = p.kv_heads * p.parts;
  const int units = __ldcg(&p.plan->tiles) * per_tile;
  auto give_up = [&]() {
    *abort_flag = 1;
    atomicExch(p.status, kDevTimeout);
  };
  struct Unit {
    Item t;
    int kv_head, part, first_head, heads, q0, tiles;   // query heads, first query, tiles of queries
  };
  auto decode = [&](int u) {
    Unit w;
    w.t = fetch_item(p, u / per_tile);
    const int r = u % per_tile;
    w.kv_head = r / p.parts;
    w.part = r % p.parts;
    w.first_head = w.kv_head * p.group + w.part * p.heads_per_part;
    w.heads = min(p.heads_per_part, p.group - w.part * p.heads_per_part);
    w.q0 = p.causal && w.t.row0 >= w.t.prefix ? w.t.row0 : w.t.start;
    w.tiles = (w.t.end - w.q0 + kRows - 1) / kRows;
    return w;
  };

  if (warp == 0) {
    // ---------------------------------------------------------------------------------------------------- copies
    if (lane == 0) {
      Ring rq(M::kStages), rd(M::kStages);
      int it = 0;
      bool ok = true;
      auto push = [&](Ring& r, uint32_t full, uint32_t empty, uint32_t tiles, const CUtensorMap* map, int head, int row) {
        const Ring::Slot s = r.next();
        if (!ptx::mbar_wait(empty + 8u * s.stage, s.phase ^ 1u, abort_flag)) { give_up(); ok = false; return; }
        ptx::mbar_arrive_expect_tx(full + 8u * s.stage, T::kBytes);
        T::load(tiles + s.stage * T::kBytes, map, full + 8u * s.stage, head, row);
      };
      for (int u = blockIdx.x; ok && u < units; u += gridDim.x, ++it) {
        const Unit w = decode(u);
        if (!ptx::mbar_wait(kv_empty, (it & 1) ^ 1u, abort_flag)) { give_up(); ok = false; break; }
        ptx::mbar_arrive_expect_tx(kv_full, 2 * T::kBytes);
        T::load(k_tile, &map_k, kv_full, w.kv_head, w.t.row0);
        T::load(v_tile, &map_v, kv_full, w.kv_head, w.t.row0);
        for (int h = w.first_head; ok && h < w.first_head + w.heads; ++h)
          for (int i = 0; ok && i < w.tiles; ++i) {
            push(rq, q_full(0), q_empty(0), q_tiles, &map_q, h, w.q0 + i * kRows);
            if (ok) push(rd, do_full(0), do_empty(0), do_tiles, &map_do, h, w.q0 + i * kRows);
          }
      }
      if (!ok) {
        const uint64_t t0 = ptx::globaltimer_ns();
        while (ptx::globaltimer_ns() - t0 < 10000000ull) {}
      }
    }
    __syncwarp();
  } else if (warp == 1) {
    // ---------------------------------------------------------------------------------------------------- products
    if (lane == 0) {
      Ring rq(M::kStages), rd(M::kStages);
      int it = 0, turns = 0;
      bool ok = true;
      const int d16 = (p.d + 15) / 16;
      auto wait = [&](uint32_t bar, uint32_t parity) {
        if (ok && !ptx::mbar_wait(bar, parity, abort_flag)) { give_up(); ok = false; }
        return ok;
      };
      for (int u = blockIdx.x; ok && u < units; u += gridDim.x, ++it) {
        const Unit w = decode(u);
        const int n = w.heads * w.tiles;
        auto rows_of = [&](int i) { return w.t.end - (w.q0 + (i % w.tiles) * kRows); };   // queries from this tile's start to the end
        // a tile of Q or dO is here: rows behind the document's end become zeros
        auto ready = [&](uint32_t full, Ring::Slot s, uint32_t tiles, int i) {
          if (!wait(full + 8u * s.stage, s.phase)) return false;
          const int left = rows_of(i);
          if (left < kRows && left % 16) T::zero_rows(gen + (tiles - base) + s.stage * T::kBytes, left, (left + 15) & ~15);
          ptx::tcgen05_fence_after_sync();
          return true;
        };
        auto scores = [&](Ring::Slot q) {
          scores_mma<HD>(tmem_s, k_tile, q_tiles + q.stage * T::kBytes, d16);
          ptx::umma_commit(s_full);
        };
        auto dprobs = [&](Ring::Slot d, bool last) {
          scores_mma<HD>(tmem_dp, v_tile, do_tiles + d.stage * T::kBytes, d16);
          ptx::umma_commit(dp_full);
          if (last) ptx::umma_commit(kv_empty);
        };
        wait(kv_full, it & 1);
        Ring::Slot q = rq.next(), d = rd.next(), q_next = q, d_next = d;
        if (!ready(q_full(0), q, q_tiles, 0)) break;
        scores(q);
        if (!ready(do_full(0), d, do_tiles, 0)) break;
        dprobs(d, n == 1);
        for (int i = 0; ok && i < n; ++i, ++turns) {
          const int steps = min(kRows, rows_of(i) + 15) / 16;
          if (i == 0 && !wait(out_free, (it & 1) ^ 1u)) break;
          if (!wait(p_full, turns & 1)) break;
          ptx::tcgen05_fence_after_sync();
          rows_mma<HD>(tmem_dv, tmem_s, tmem_s + kPanel, do_tiles + d.stage * T::kBytes, steps, d16, i > 0);
          ptx::umma_commit(do_empty(d.stage));
          if (i + 1 < n) {
            q_next = rq.next();
            if (!ready(q_full(0), q_next, q_tiles, i + 1)) break;
            scores(q_next);
          }
          if (!wait(ds_full, turns & 1)) break;
          ptx::tcgen05_fence_after_sync();
          rows_mma<HD>(tmem_dk, tmem_dp, tmem_dp + kPanel, q_tiles + q.stage * T::kBytes, steps, d16, i > 0);
          ptx::umma_commit(q_empty(q.stage));
          if (i == n - 1) ptx::umma_commit(out_full);
          if (i + 1 < n) {
            d_next = rd.next();
            if (!ready(do_full(0), d_next, do_tiles, i + 1)) break;
            dprobs(d_next, i + 2 == n);
          }
          q = q_next;
          d = d_next;
        }
      }
      if (it > 0 || !ok) {
        ptx::umma_commit(done);
        const uint64_t t0 = ptx::globaltimer_ns();
        while (!ptx::mbar_try_wait(done, 0) && ptx::globaltimer_ns() - t0 < ptx::kWaitLimitNs) {}
      }
    }
    __syncwarp();
  } else if (warp == 2) {
    // ---------------------------------------------------------------------------------------------------- lse and delta
    Ring rv(M::kVecStages);
    bool ok = true;
    for (int u = blockIdx.x; ok && u < units; u += gridDim.x) {
      const Unit w = decode(u);
      for (int h = w.first_head; ok && h < w.first_head + w.heads; ++h)
        for (int i = 0; ok && i < w.tiles; ++i) {
          const Ring::Slot s = rv.next();
          float a[4], b[4];
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const int row = w.q0 + i * kRows + 32 * k + lane;
            const int64_t at = int64_t(h) * p.tokens + row;
            a[k] = row < w.t.end ? __ldcg(p.lse + at) * kLog2e : 0.f;   // behind the document's end: masked
            b[k] = row < w.t.end ? __ldcg(p.delta + at) : 0.f;
          }
          if (!warp_wait(vec_empty(s.stage), s.phase ^ 1u, abort_flag)) { give_up(); ok = false; break; }
          float* v = reinterpret_cast<float*>(gen + M::kVec + s.stage * M::kVecBytes);
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            v[32 * k + lane] = a[k];
            v[kRows + 32 * k + lane] = b[k];
          }
          __syncwarp();
          if (lane == 0) ptx::mbar_arrive(vec_full(s.stage));
          __syncwarp();
        }
    }
  } else if (warp >= 4) {
    // ---------------------------------------------------------------------------------------------------- rows
    const int panel = (warp - 4) >> 2, quarter = warp & 3;
    const uint32_t lanes = uint32_t(32 * quarter) << 16, col0 = kPanel * panel;
    int turns = 0, it = 0;
    Ring rv(M::kVecStages);
    bool ok = true;
    for (int u = blockIdx.x; ok && u < units; u += gridDim.x, ++it) {
      const Unit w = decode(u);
      const int key = w.t.row0 + 32 * quarter + lane;
      // this key is seen by the queries from here on, and by none before; from `all_from` on every key of the tile is
      const int from = p.causal && key >= w.t.prefix ? key : w.t.start;
      const int all_from = p.causal && min(w.t.row0 + kRows, w.t.end) > w.t.prefix ? min(w.t.row0 + kRows, w.t.end) - 1 : w.t.start;
      // the document's first query sees one key only
      const bool lonely = w.t.end - w.t.start == 1 || (p.causal && w.t.prefix <= w.t.start + 1);
      for (int h = w.first_head; ok && h < w.first_head + w.heads; ++h) {
        const float slope2 = BIAS ? __ldg(p.slopes + h) * kLog2e : 0.f;
        for (int i = 0; i < w.tiles; ++i, ++turns) {
          const Ring::Slot vs = rv.next();
          const float* vec = reinterpret_cast<const float*>(gen + M::kVec + vs.stage * M::kVecBytes) + col0;
          const int c0 = w.q0 + i * kRows + int(col0);     // the query of column 0
          if (!warp_wait(vec_full(vs.stage), vs.phase, abort_flag) || !warp_wait(s_full, turns & 1, abort_flag)) {
            give_up();
            ok = false;
            break;
          }
          ptx::tcgen05_fence_after_sync();
          uint32_t s[2][32];
#pragma unroll
          for (int c = 0; c < 2; ++c) ptx::tmem_ld_x32(tmem_s + lanes + col0 + 32 * c, s[c]);
          tmem_loaded(s[0], s[1]);
          const bool masked = c0 < all_from || c0 + kPanel > w.t.end;
          const int first = from - c0, last = w.t.end - c0;
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            uint32_t pk[16];
#pragma unroll
            for (int i4 = 0; i4 < 8; ++i4) {
              const float4 l4 = *reinterpret_cast<const float4*>(vec + 32 * c + 4 * i4);
              const float l[4] = {l4.x, l4.y, l4.z, l4.w};
              float e[4];
#pragma unroll
              for (int k = 0; k < 4; ++k) {
                const int col = 4 * i4 + k;
                float slope = 1.f, x;
                if (!CAP && !BIAS) x = fmaf(__uint_as_float(s[c][col]), p.c, -l[k]);
                else x = exponent<CAP, BIAS>(p, __uint_as_float(s[c][col]), float(c0 - key) + float(32 * c + col), slope2, &slope) - l[k];
                e[k] = exp2_fast(x);
                if (masked) e[k] = 32 * c + col < first || 32 * c + col >= last ? 0.f : e[k];
                s[c][col] = __float_as_uint(CAP ? e[k] * slope : e[k]);
              }
              pk[2 * i4] = pack2(e[0], e[1]);
              pk[2 * i4 + 1] = pack2(e[2], e[3]);
            }
            ptx::tmem_st_x16(tmem_s + lanes + col0 + 16 * c, pk);
          }
          ptx::tmem_st_wait();
          ptx::tcgen05_fence_before_sync();
          __syncwarp();
          if (lane == 0) ptx::mbar_arrive(p_full);
          __syncwarp();
          if (lonely && c0 == w.t.start) s[0][0] = 0u;
          if (!warp_wait(dp_full, turns & 1, abort_flag)) { give_up(); ok = false; break; }
          ptx::tcgen05_fence_after_sync();
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            uint32_t g[32], pk[16];
            ptx::tmem_ld_x32(tmem_dp + lanes + col0 + 32 * c, g);
            tmem_loaded(g);
            if (masked) {   // queries of another document: their dP may be anything
#pragma unroll
              for (int i = 0; i < 32; ++i) g[i] = 32 * c + i < last ? g[i] : 0u;
            }
#pragma unroll
            for (int i4 = 0; i4 < 8; ++i4) {
              const float4 d4 = *reinterpret_cast<const float4*>(vec + kRows + 32 * c + 4 * i4);
              const float dl[4] = {d4.x, d4.y, d4.z, d4.w};
              float e[4];
#pragma unroll
              for (int k = 0; k < 4; ++k) e[k] = __uint_as_float(s[c][4 * i4 + k]) * (__uint_as_float(g[4 * i4 + k]) - dl[k]);
              pk[2 * i4] = pack2(e[0], e[1]);
              pk[2 * i4 + 1] = pack2(e[2], e[3]);
            }
            ptx::tmem_st_x16(tmem_dp + lanes + col0 + 16 * c, pk);
          }
          ptx::tmem_st_wait();
          ptx::tcgen05_fence_before_sync();
          __syncwarp();
          if (lane == 0) {
            ptx::mbar_arrive(ds_full);
            ptx::mbar_arrive(vec_empty(vs.stage));
          }
          __syncwarp();
        }
      }
      if (!ok) break;
      if (!warp_wait(out_full, it & 1, abort_flag)) { give_up(); break; }
      ptx::tcgen05_fence_after_sync();
      const bool live = key < w.t.end;
      // panel 0 stores dV, panel 1 dK
      const uint32_t from_col = (panel ? tmem_dk : tmem_dv) + lanes;
      const float f = panel ? p.scale : 1.f;
      float* part = panel ? p.dk_part : p.dv_part;
      if (part) part += ((int64_t(w.part) * p.tokens + key) * p.kv_heads + w.kv_head) * p.d;
      __nv_bfloat16* out = panel ? p.dK + int64_t(key) * p.lddk : p.dV + int64_t(key) * p.lddv;
      out += int64_t(w.kv_head) * p.d;
#pragma unroll
      for (int c = 0; c < HD / 32; ++c) {
        uint32_t o[32];
        ptx::tmem_ld_x32(from_col + 32 * c, o);
        tmem_loaded(o);
        if (c == HD / 32 - 1) {
          ptx::tcgen05_fence_before_sync();
          __syncwarp();
          if (lane == 0) ptx::mbar_arrive(out_free);
          __syncwarp();
        }
        if (live && 32 * c < p.d) {
          if (part) store_f32(part + 32 * c, o, f, p.d - 32 * c);
          else store_bf16(out + 32 * c, o, f, p.d - 32 * c);
        }
        __syncwarp();
      }
    }
  }
  zero_rows_outside(p, p.dK, p.lddk, p.kv_heads, nullptr, 0.f);
  zero_rows_outside(p, p.dV, p.lddv, p.kv_heads, nullptr, 0.f);
  __syncwarp();
  ptx::tcgen05_fence_before_sync();
  __syncthreads();
  if (warp == 1) {
    __syncwarp();
    ptx::tcgen05_fence_after_sync();
    ptx::tmem_dealloc(tmem, 512);
  }
}

// dK and dV from the parts' fp32 sums, in order; eight columns per thread, rows outside the documents left alone.
__global__ void __launch_bounds__(256) attn_join_kernel(const Params p) {
  wait_for_launch_before();
  let_next_launch_start();
  const int head_end = __ldcg(&p.plan->head_end), tail = __ldcg(&p.plan->tail_begin);
  const int per_row = p.kv_heads * (p.d / 8);
  const int64_t n = int64_t(p.tokens) * per_row, k = int64_t(blockIdx.x) * blockDim.x + threadIdx.x;
  if (k >= n) return;
  const int64_t row = k / per_row, col = (k - row * per_row) * 8;
  if (row < head_end || row >= tail) return;
  const bool v = blockIdx.y != 0;
  const float* part = (v ? p.dv_part : p.dk_part) + row * (int64_t(p.kv_heads) * p.d) + col;
  float2 sum[4] = {};
  for (int i = 0; i < p.parts; ++i) {
    float2 x[4];
    q8::load8(part + int64_t(i) * p.tokens * p.kv_heads * p.d, x);
#pragma unroll
    for (int j = 0; j < 4; ++j) sum[j] = q8::add2(sum[j], x[j]);
  }
  q8::store8(v ? p.dV + row * p.lddv + col : p.dK + row * p.lddk + col, sum);
}

struct Maps { CUtensorMap q, k, v, g; };

template <typename K>
cudaError_t launch(DeviceOnce& once, K kernel, int smem, const Maps& m, const Params& p, unsigned grid, cudaStream_t st) {
  if (once.needed()) {
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
    if (e != cudaSuccess) return e;
    once.done();
  }
  return launch_lined_up(kernel, dim3(grid), dim3(kThreads), smem, st, m.q, m.k, m.v, m.g, p);
}
template <int HD, bool CAP, bool BIAS>
cudaError_t launch_both(const Maps& m, const Params& pq, unsigned grid_q, const Params& pk, unsigned grid_k, cudaStream_t st) {
  static DeviceOnce once_q, once_k;
  const cudaError_t e = launch(once_q, attn_dq_kernel<HD, CAP, BIAS>, QuerySmem<HD>::kBytes, m, pq, grid_q, st);
  return e != cudaSuccess ? e : launch(once_k, attn_dkv_kernel<HD, CAP, BIAS>, KeySmem<HD>::kBytes, m, pk, grid_k, st);
}
template <int HD>
cudaError_t launch_both(bool cap, bool bias, const Maps& m, const Params& pq, unsigned grid_q, const Params& pk, unsigned grid_k, cudaStream_t st) {
  if (cap) return bias ? launch_both<HD, true, true>(m, pq, grid_q, pk, grid_k, st) : launch_both<HD, true, false>(m, pq, grid_q, pk, grid_k, st);
  return bias ? launch_both<HD, false, true>(m, pq, grid_q, pk, grid_k, st) : launch_both<HD, false, false>(m, pq, grid_q, pk, grid_k, st);
}

// Work items of the keys' kernel: a group's query heads are dealt to as many parts as make three items for each SM, as far as there
// are heads.
struct KeyParts { int parts, heads_per_part; };
KeyParts key_parts(const AttnProblem& q) {
  const int group = q.heads / q.kv_heads;
  const int64_t tiles = (q.tokens + kRows - 1) / kRows;
  const int64_t want = 3 * 148;
  KeyParts k;
  k.heads_per_part = int(std::max<int64_t>(1, std::min<int64_t>(group, tiles * q.heads / want)));
  k.parts = (group + k.heads_per_part - 1) / k.heads_per_part;
  return k;
}
size_t aligned(size_t n) { return (n + 255) & ~size_t(255); }

}  // namespace
}  // namespace attn

using namespace attn;

size_t attn_bwd_workspace_bytes(const AttnProblem& q) {
  const KeyParts k = key_parts(q);
  const size_t part = aligned(size_t(q.tokens) * q.kv_heads * q.d * 4 * k.parts);
  return aligned(size_t(q.tokens) * q.heads * 4) + (k.parts > 1 ? 2 * part : 0);
}

cudaError_t attn_bwd(const AttnProblem& q, const AttnMatrix& Q, const AttnMatrix& K, const AttnMatrix& V, const float* slopes, const void* plan,
                     const AttnMatrix& O, const AttnMatrix& dO, const float* lse, const AttnMatrix& dQ, const AttnMatrix& dK, const AttnMatrix& dV,
                     void* ws, int* status, cudaStream_t st) {
  float* delta = static_cast<float*>(ws);
  cudaError_t e = launch_lined_up(attn_delta_kernel, dim3(unsigned((q.tokens + kDeltaTokens - 1) / kDeltaTokens), unsigned(q.heads)),
                                  dim3(kDeltaThreads), 0, st, static_cast<const __nv_bfloat16*>(O.p), O.ld, static_cast<const __nv_bfloat16*>(dO.p),
                                  dO.ld, int(q.tokens), q.d, delta);
  if (e != cudaSuccess) return e;
  Maps m;
  if (!make_tmap_heads(&m.q, Q.p, q.tokens, q.heads, q.d, Q.ld, kRows) || !make_tmap_heads(&m.k, K.p, q.tokens, q.kv_heads, q.d, K.ld, kRows) ||
      !make_tmap_heads(&m.v, V.p, q.tokens, q.kv_heads, q.d, V.ld, kRows) || !make_tmap_heads(&m.g, dO.p, q.tokens, q.heads, q.d, dO.ld, kRows))
    return cudaErrorInvalidValue;
  const PlanLayout at = plan_layout(q.tokens, q.docs);
  const KeyParts kp = key_parts(q);
  Params p = common_params(q, plan, slopes, const_cast<float*>(lse), status);
  p.delta = delta;
  p.dQ = static_cast<__nv_bfloat16*>(dQ.p);
  p.dK = static_cast<__nv_bfloat16*>(dK.p);
  p.dV = static_cast<__nv_bfloat16*>(dV.p);
  p.lddq = dQ.ld;
  p.lddk = dK.ld;
  p.lddv = dV.ld;
  p.parts = kp.parts;
  p.heads_per_part = kp.heads_per_part;
  if (kp.parts > 1) {
    uint8_t* w8 = static_cast<uint8_t*>(ws) + aligned(size_t(q.tokens) * q.heads * 4);
    p.dk_part = reinterpret_cast<float*>(w8);
    p.dv_part = reinterpret_cast<float*>(w8 + aligned(size_t(q.tokens) * q.kv_heads * q.d * 4 * kp.parts));
  }
  Params pk = p;
  const uint8_t* plan8 = static_cast<const uint8_t*>(plan);
  p.items = reinterpret_cast<const Item*>(plan8 + at.queries);
  pk.items = reinterpret_cast<const Item*>(plan8 + at.keys);
  const unsigned grid_q = unsigned(std::min<int64_t>(at.tile_cap * q.heads, sm_count()));
  const unsigned grid_k = unsigned(std::min<int64_t>(at.tile_cap * q.kv_heads * kp.parts, sm_count()));
  const bool cap = q.softcap > 0.f, bias = slopes != nullptr;
  e = q.d <= 64 ? launch_both<64>(cap, bias, m, p, grid_q, pk, grid_k, st) : launch_both<128>(cap, bias, m, p, grid_q, pk, grid_k, st);
  if (e != cudaSuccess || kp.parts == 1) return e;
  const int64_t n = q.tokens * q.kv_heads * (q.d / 8);
  return launch_lined_up(attn_join_kernel, dim3(unsigned((n + 255) / 256), 2), dim3(256), 0, st, pk);
}

}  // namespace acx
