// Attention: the backward kernels.
//
// With dO and the forward's lse, and delta_i = sum over the keys of p_ij dP_ij (which is dO_i O_i),
//     P = 2^(x - lse),   dP = dO V^T,   dS = P (dP - delta) dx/ds,
//     dQ = scale dS K,   dK = scale dS^T Q,   dV = P^T dO.
// Two launches of one kernel, each with sums that no other work item adds to, so that no atomics are needed and results are
// reproducible bit for bit.  Rows of the tile: queries (dQ) or keys (dK, dV).  Either has two tiles that stay (Q, dO or K, V) and goes
// through pairs of others (K, V of the keys that the queries see; Q, dO of the queries that see the keys, head by head of the group):
//     S = R0 T0^T,   dP = R1 T1^T,   first += P T,   second += dS T0.
// For keys `first` is dV (T = dO) and `second` dK.  For queries `second` is dQ, and `first` = P K corrects it: O rounded to bf16
// gives delta to within that rounding only, and an error e of delta is one of -e P K in dQ, which was as large as the rounding of dS and dQ
// together (errors of dQ 0.0029 relative to its size without it).  So dS is taken with the delta that O gives, r_i = sum of
// p (dP - delta) summed in fp32 beside it, delta + r is what the launch for the keys uses, and dQ = scale (second - r' first) with
// the sum r' of the dS as they were rounded: exact ones sum to zero, so r' is e and what the roundings leave of the keys' mean (errors
// of dQ 0.00245 with r, 0.0022 to 0.0023 with r', where the keys have a mean; the rounding of dS and of dQ themselves make 0.0023).
// The price of two launches is that S and dP are computed twice: eight products instead of five.  Measured: 8192 tokens x 24 heads (8
// of keys) x 128, causal, 609 us for the queries and 709 for the keys, 1.25 PFLOP/s over the eight, 75 % of the rate of a large product (tensor
// pipe 70 and 56 % busy); 2650 and 3180 cycles per tile of 128 x 128 where the products alone need 2048, the rest is rows' work in between.
//
// S, dP, first and second fill the tensor memory (4 x 128 columns); dS goes over dP as bf16 and is multiplied from there, P goes to shared
// memory, so that the next S can be taken as soon as this one has been read: the rows' warps never wait for it (with P over S they
// waited 1600 of 3900 cycles a tile).  Sixteen warps share a tile, 32 rows x 32 columns each.
//
// A query that sees one key only has p = 1 and no gradient through its scores: exactly zero, not the difference of two roundings.
//
// Of a document of a few tokens (kFewTokens) dS goes into dK as two bf16 parts, the rounded one and what is left: nothing averages out between so few
// queries.  It is the document that decides, not the batch: the same one has the same errors (and, where a group's heads are not dealt to
// parts, the same bits) whatever stands beside it.  Errors of dK 0.0023 to 0.0025 -> 0.0017, its own rounding; the backward of 256 tokens
// x 14 heads x 64 20.2 -> 20.5 us, 512 x 8 x 64 23.7 -> 24.7, but 2048 x 6 x 128 80 -> 85 and 8192 x 24 x 128 1323 -> 1434.
//
// Where a batch has few key tiles for the SMs a group's query heads are dealt to several work items, whose fp32 sums a last kernel adds
// in a fixed order.
#include <cuda_fp16.h>

#include <algorithm>

#include "acx_attn.cuh"
#include "acx_tmap.h"

namespace acx {
namespace attn {
namespace {

constexpr int kRowWarp0 = 4, kRowWarps = 16, kThreads = 32 * (kRowWarp0 + kRowWarps);
constexpr int kPanel = 32;        // columns of a tile that one warp takes
constexpr int kPanels = kRows / kPanel;
constexpr int kFewTokens = 512;
// A probability 2^(x - lse) is at most 1, but x and lse are known to some 2^-22 of their size only: above this size (where that is
// 2^-10) a probability is bounded.  Unbounded, one of scores of 1e8 was up to 2^9, one of 1e10 an infinity, which times a dO of zero
// made every key's gradient NaN.  By row, not by warp: a row's bits do not depend on its neighbours.
constexpr float kLargeLse = 4096.f;
__device__ __forceinline__ float bounded_exponent(float x, float lse2, float top) { return fabsf(lse2) > kLargeLse ? min_nan(x, top) : x; }
// With a cap the probabilities are 2^-14 of what they are and its slopes 2^14, as fp16: those from 2^-28 on have all digits of that (a score
// of 10.4 caps), and their product is dS.  The exponents get -14 with lse; dV and the sums of p (dP - delta) are put right at their end.
constexpr float kCapShift = 14.f;
static_assert(kSlopeUnit == 16384.f, "2^kCapShift");

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

__device__ __forceinline__ void load_columns(uint32_t at, uint32_t (&v)[32]) { ptx::tmem_ld_x32(at, v); }
__device__ __forceinline__ void load_columns(uint32_t at, uint32_t (&v)[16]) { ptx::tmem_ld_x16(at, v); }

// KEYS: rows are keys
template <int HD, bool KEYS>
struct Smem {
  // Stages.  T0 is read by S, a tile ahead, and by `second` at the end (and by `first` for queries); T1 by dP alone for queries, and by
  // `first` for keys.  At d = 128 six tiles fit beside P.
  static constexpr int kT0 = KEYS && HD == 128 ? 2 : 3, kT1 = !KEYS && HD == 128 ? 1 : 2;
  static constexpr int kP = (2 + kT0 + kT1) * Tile<HD>::kBytes, kPBytes = kRows * kRows * 2;
  static constexpr int kVec = kP + kPBytes;
  static constexpr int kVecStages = KEYS ? 2 : 0, kVecBytes = 2 * kRows * 4;   // KEYS: lse and delta of a tile of queries
  static constexpr int kPartBytes = kPanels / 2 * kRows * 8;
  static constexpr int kExchange = kVec + kVecStages * kVecBytes;              // else: partial sums of the rows
  static constexpr int kBars = kExchange + (KEYS ? 0 : kPartBytes), kBytes = kBars + 256;
  static_assert(kBytes <= 232448, "shared memory of one CTA");
};

// Whether dS goes into dK in two parts.
__device__ __forceinline__ bool two_parts(const Item& t) { return t.end - t.start <= kFewTokens; }

// What one work item goes through.
struct Unit {
  Item t;
  int head, heads;       // query heads: the first, how many
  int kv_head, part;
  int other0, tiles;     // first token and number of the tiles on the other side
};

template <int HD, bool KEYS, bool CAP, bool BIAS>
__global__ void __launch_bounds__(kThreads, 1)
    attn_bwd_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v,
                    const __grid_constant__ CUtensorMap map_do, const Params p) {
  using T = Tile<HD>;
  using M = Smem<HD, KEYS>;
  extern __shared__ __align__(1024) uint8_t gen[];   // tiles start on their swizzle's boundary
  const uint32_t base = ptx::smem_u32(gen);
  const uint32_t r0_tile = base, r1_tile = base + T::kBytes, t0_tiles = base + 2 * T::kBytes, t1_tiles = t0_tiles + M::kT0 * T::kBytes,
                 p_tile = base + M::kP;
  const uint32_t bars = base + M::kBars;
  auto t0_full = [&](int s) { return bars + 8u * s; };
  auto t0_empty = [&](int s) { return bars + 24 + 8u * s; };
  auto t1_full = [&](int s) { return bars + 48 + 8u * s; };
  auto t1_empty = [&](int s) { return bars + 64 + 8u * s; };
  auto vec_full = [&](int s) { return bars + 80 + 8u * s; };
  auto vec_empty = [&](int s) { return bars + 96 + 8u * s; };
  const uint32_t r_full = bars + 112, r_empty = bars + 120, s_full = bars + 128, s_free = bars + 136, p_full = bars + 144, p_free = bars + 152,
                 dp_full = bars + 160, ds_full = bars + 168, out_full = bars + 176, out_free = bars + 184, parts_full = bars + 192,
                 parts_free = bars + 200, done = bars + 208;
  volatile uint32_t* tmem_slot = reinterpret_cast<volatile uint32_t*>(gen + M::kBars + 216);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(gen + M::kBars + 220);
  volatile int* no_abort = abort_flag + 1;   // for the one wait that has to run its time even so
  const int warp = __shfl_sync(0xFFFFFFFFu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;   // the warp's number, known to be the same in all lanes

  if (base & 1023u) {   // not a place for tiles: nothing is done, and said so
    if (threadIdx.x == 0) atomicExch(p.status, kDevTimeout);
    return;
  }

  if (threadIdx.x == 0) {
    for (int s = 0; s < M::kT0; ++s) {
      ptx::mbar_init(t0_full(s), 1);
      ptx::mbar_init(t0_empty(s), 1);
    }
    for (int s = 0; s < M::kT1; ++s) {
      ptx::mbar_init(t1_full(s), 1);
      ptx::mbar_init(t1_empty(s), 1);
    }
    for (int s = 0; s < M::kVecStages; ++s) {
      ptx::mbar_init(vec_full(s), 1);
      ptx::mbar_init(vec_empty(s), kRowWarps);
    }
    ptx::mbar_init(r_full, 1);
    ptx::mbar_init(r_empty, 1);
    ptx::mbar_init(s_full, 1);
    ptx::mbar_init(s_free, kRowWarps);
    ptx::mbar_init(p_full, kRowWarps);
    ptx::mbar_init(p_free, 1);
    ptx::mbar_init(dp_full, 1);
    ptx::mbar_init(ds_full, kRowWarps);
    ptx::mbar_init(out_full, 1);
    ptx::mbar_init(out_free, kRowWarps);
    ptx::mbar_init(done, 1);
    *no_abort = 0;
    ptx::mbar_init(parts_full, kRowWarps);
    ptx::mbar_init(parts_free, kRowWarps);
    *abort_flag = 0;
    ptx::fence_barrier_init();
  }
  // A warp comes to the barrier as a whole: halves of it would count as two, and let the others read the address before it is there
  __syncwarp();
  if (warp == 1) {
    ptx::tmem_alloc(bars + 216, 512);
    ptx::tmem_relinquish_alloc_permit();
    __syncwarp();
  }
  ptx::tcgen05_fence_before_sync();
  __syncthreads();
  ptx::tcgen05_fence_after_sync();
  const uint32_t tmem = *tmem_slot;
  const uint32_t tmem_s = tmem, tmem_dp = tmem + 128, tmem_first = tmem + 256, tmem_second = tmem + 384;
  wait_for_launch_before();
  let_next_launch_start();
  const int per_tile = KEYS ? p.kv_heads * p.parts : p.heads;
  const bool fits = plan_fits(p);
  const int units = fits ? __ldcg(&p.plan->tiles) * per_tile : 0;
  auto give_up = [&]() {
    *abort_flag = 1;
    atomicExch(p.status, kDevTimeout);
  };
  auto decode = [&](int u, const Item& t) {
    Unit w;
    w.t = t;
    const int r = u % per_tile;
    if (KEYS) {
      w.kv_head = r / p.parts;
      w.part = r % p.parts;
      w.head = w.kv_head * p.group + w.part * p.heads_per_part;
      w.heads = min(p.heads_per_part, p.group - w.part * p.heads_per_part);
      w.other0 = p.causal && w.t.row0 >= w.t.prefix ? w.t.row0 : w.t.start;
      w.tiles = (w.t.end - w.other0 + kRows - 1) / kRows;
    } else {
      w.head = r;
      w.heads = 1;
      w.kv_head = r / p.group;
      w.part = 0;
      w.other0 = w.t.start;
      w.tiles = ((p.causal ? max(min(w.t.row0 + kRows, w.t.end), w.t.prefix) : w.t.end) - w.t.start + kRows - 1) / kRows;
    }
    return w;
  };

  if (warp == 0) {
    // ---------------------------------------------------------------------------------------------------- copies
    if (lane == 0) {
      Ring r0(M::kT0), r1(M::kT1);
      int it = 0;
      bool ok = true;
      auto push = [&](Ring& r, uint32_t full, uint32_t empty, uint32_t tiles, const CUtensorMap* map, int head, int row) {
        const Ring::Slot s = r.next();
        if (!ptx::mbar_wait(empty + 8u * s.stage, s.phase ^ 1u, abort_flag)) { give_up(); ok = false; return; }
        ptx::mbar_arrive_expect_tx(full + 8u * s.stage, T::kBytes);
        T::load(tiles + s.stage * T::kBytes, map, full + 8u * s.stage, head, row);
      };
      for (int u; ok && (u = unit_of(it)) < units; ++it) {
        const Unit w = decode(u, fetch_item(p.items, u / per_tile));
        if (!ptx::mbar_wait(r_empty, (it & 1) ^ 1u, abort_flag)) { give_up(); ok = false; break; }
        ptx::mbar_arrive_expect_tx(r_full, 2 * T::kBytes);
        T::load(r0_tile, KEYS ? &map_k : &map_q, r_full, KEYS ? w.kv_head : w.head, w.t.row0);
        T::load(r1_tile, KEYS ? &map_v : &map_do, r_full, KEYS ? w.kv_head : w.head, w.t.row0);
        for (int h = w.head; ok && h < w.head + w.heads; ++h)
          for (int i = 0; ok && i < w.tiles; ++i) {
            const int other = KEYS ? h : w.kv_head, row = w.other0 + i * kRows;
            push(r0, t0_full(0), t0_empty(0), t0_tiles, KEYS ? &map_q : &map_k, other, row);
            if (ok) push(r1, t1_full(0), t1_empty(0), t1_tiles, KEYS ? &map_do : &map_v, other, row);
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
    Ring r0(M::kT0), r1(M::kT1);
    int it = 0, turns = 0;
    bool ok = true;
    const int d16 = (p.d + 15) / 16;
    auto wait = [&](uint32_t bar, uint32_t parity) {
      if (ok && !warp_wait(bar, parity, abort_flag)) { give_up(); ok = false; }
      return ok;
    };
    for (int u; ok && (u = unit_of(it)) < units; ++it) {
      const Unit w = decode(u, fetch_item_warp(p.items, u / per_tile));
      const int n = w.heads * w.tiles;
      auto left_of = [&](int i) { return w.t.end - (w.other0 + (i % w.tiles) * kRows); };   // tokens from this tile's start to the end
      // a tile is here; if products sum over its rows, those behind the document's end become zeros up to a whole step
      auto ready = [&](uint32_t full, Ring::Slot s, uint32_t tiles, int i, bool summed) {
        if (!wait(full + 8u * s.stage, s.phase)) return false;
        const int left = left_of(i);
        if (summed && left < kRows && left % 16)
          T::zero_rows(gen + (tiles - base) + s.stage * T::kBytes, left, (left + 15) & ~15);
        ptx::tcgen05_fence_after_sync();
        return true;
      };
      auto scores = [&](Ring::Slot a) {
        scores_mma<HD>(tmem_s, r0_tile, t0_tiles + a.stage * T::kBytes, d16);
        ptx::umma_commit_elected(s_full);
      };
      auto dprobs = [&](Ring::Slot b, bool last) {
        scores_mma<HD>(tmem_dp, r1_tile, t1_tiles + b.stage * T::kBytes, d16);
        ptx::umma_commit_elected(dp_full);
        if (!KEYS) ptx::umma_commit_elected(t1_empty(b.stage));
        if (last) ptx::umma_commit_elected(r_empty);
      };
      wait(r_full, it & 1);
      Ring::Slot a = r0.next(), b = r1.next(), a_next = a, b_next = b;
      if (!ready(t0_full(0), a, t0_tiles, 0, true)) break;
      scores(a);
      if (!ready(t1_full(0), b, t1_tiles, 0, KEYS)) break;
      dprobs(b, n == 1);
      for (int i = 0; ok && i < n; ++i, ++turns) {
        const int steps = min(kRows, left_of(i) + 15) / 16;
        if (i + 1 < n) {   // the next scores as soon as these have been read
          a_next = r0.next();
          if (!ready(t0_full(0), a_next, t0_tiles, i + 1, true)) break;
          if (!wait(s_free, turns & 1)) break;
          ptx::tcgen05_fence_after_sync();
          scores(a_next);
        }
        if (i == 0 && !wait(out_free, (it & 1) ^ 1u)) break;
        if (!wait(p_full, turns & 1)) break;
        ptx::tcgen05_fence_after_sync();
        smem_rows_mma<HD>(tmem_first, p_tile, KEYS ? t1_tiles + b.stage * T::kBytes : t0_tiles + a.stage * T::kBytes, steps, d16, i > 0);
        ptx::umma_commit_elected(p_free);
        if (KEYS) ptx::umma_commit_elected(t1_empty(b.stage));
        if (!wait(ds_full, turns & 1)) break;
        ptx::tcgen05_fence_after_sync();
        rows_mma<HD, 16>(tmem_second, tmem_dp, t0_tiles + a.stage * T::kBytes, steps, d16, i > 0);
        if (KEYS && two_parts(w.t)) rows_mma<HD, 16>(tmem_second, tmem_dp + 16, t0_tiles + a.stage * T::kBytes, steps, d16, true);
        ptx::umma_commit_elected(t0_empty(a.stage));
        if (i == n - 1) ptx::umma_commit_elected(out_full);
        if (i + 1 < n) {
          b_next = r1.next();
          if (!ready(t1_full(0), b_next, t1_tiles, i + 1, KEYS)) break;
          dprobs(b_next, i + 2 == n);
        } else if (!wait(s_free, turns & 1)) {   // (no scores follow in this item: the phase is taken all the same)
          break;
        }
        a = a_next;
        b = b_next;
      }
    }
    if (it > 0 || !ok) {   // everything that was issued has to be done before the tensor memory is given back
      ptx::umma_commit_elected(done);
      warp_wait(done, 0, no_abort);
    }
    __syncwarp();
  } else if (warp == 2) {
    // ---------------------------------------------------------------------------------------------------- lse and delta of queries
    if (KEYS) {
      Ring rv(M::kVecStages);
      bool ok = true;
      int it = 0;
      for (int u; ok && (u = unit_of(it)) < units; ++it) {
        const Unit w = decode(u, fetch_item_warp(p.items, u / per_tile));
        for (int h = w.head; ok && h < w.head + w.heads; ++h)
          for (int i = 0; ok && i < w.tiles; ++i) {
            const Ring::Slot s = rv.next();
            float a[4], b[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              const int row = w.other0 + i * kRows + 32 * k + lane;
              const int64_t at = int64_t(h) * p.tokens + row;
              a[k] = row < w.t.end ? fmaf(__ldcg(p.lse + at), kLog2e, CAP ? kCapShift : 0.f) : 0.f;   // behind the document's end: masked
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
    }
  } else if (warp >= kRowWarp0) {
    // ---------------------------------------------------------------------------------------------------- rows
    const int panel = (warp - kRowWarp0) >> 2, quarter = warp & 3, r = 32 * quarter + lane;
    const uint32_t lanes = uint32_t(32 * quarter) << 16, col0 = kPanel * panel;
    const uint32_t s_at = tmem_s + lanes + col0, dp_at = tmem_dp + lanes + col0;
    uint8_t* const p_row = gen + M::kP + (panel >> 1) * (kRows * 128) + r * 128;
    int turns = 0, it = 0;
    Ring rv(KEYS ? M::kVecStages : 1);
    bool ok = true;
    for (int u; ok && (u = unit_of(it)) < units; ++it) {
      const Unit w = decode(u, fetch_item_warp(p.items, u / per_tile));
      const int row = w.t.row0 + r;              // the token of this lane
      const bool live = row < w.t.end;
      // the columns that this row's mask leaves in a tile are [first, last) once the tile's first token is taken off; every row of
      // the tile keeps those in [all_first, all_last)
      int first, last, all_first, all_last;
      if (KEYS) {
        first = p.causal && row >= w.t.prefix ? row : w.t.start;
        all_first = p.causal && min(w.t.row0 + kRows, w.t.end) > w.t.prefix ? min(w.t.row0 + kRows, w.t.end) - 1 : w.t.start;
        last = all_last = w.t.end;
      } else {
        first = all_first = w.t.start;
        last = p.causal ? min(max(row + 1, w.t.prefix), w.t.end) : w.t.end;
        all_last = p.causal ? min(max(w.t.row0 + 1, w.t.prefix), w.t.end) : w.t.end;
      }
      // KEYS: the document's first query sees one key only; else: this row does
      const bool lonely = KEYS ? w.t.end - w.t.start == 1 || (p.causal && w.t.prefix <= w.t.start + 1) : last - w.t.start == 1;
      float lse2 = 0.f, delta = 0.f;
      float2 rest2 = make_float2(0.f, 0.f), kept2 = rest2;   // sums of p (dP - delta), and of what dS's rounding makes of them
      if (!KEYS) {
        const int64_t at = int64_t(w.head) * p.tokens + row;
        lse2 = live ? fmaf(__ldcg(p.lse + at), kLog2e, CAP ? kCapShift : 0.f) : 0.f;
        delta = live ? __ldcg(p.delta + at) : 0.f;
      }
      const bool large_row = !KEYS && __any_sync(0xFFFFFFFFu, fabsf(lse2) > kLargeLse);
      for (int h = w.head; ok && h < w.head + w.heads; ++h) {
        const float slope2 = BIAS ? __ldg(p.slopes + h) * kLog2e : 0.f;
        for (int i = 0; i < w.tiles; ++i, ++turns) {
          const Ring::Slot vs = rv.next();
          const float* vec = reinterpret_cast<const float*>(gen + M::kVec + vs.stage * M::kVecBytes) + col0;
          const int c0 = w.other0 + i * kRows + int(col0);     // the token of column 0
          if ((KEYS && !warp_wait(vec_full(vs.stage), vs.phase, abort_flag)) || !warp_wait(s_full, turns & 1, abort_flag)) {
            give_up();
            ok = false;
            break;
          }
          ptx::tcgen05_fence_after_sync();
          uint32_t s[32];
          ptx::tmem_ld_x32(s_at, s);
          tmem_loaded(s);
          ptx::tcgen05_fence_before_sync();
          __syncwarp();
          if (lane == 0) ptx::mbar_arrive(s_free);
          __syncwarp();
          const bool masked = c0 < all_first || c0 + kPanel > all_last;
          const int lo = first - c0, hi = last - c0;
          // dx/ds of the cap, as fp16: off by 2^-11 at most, beside the 2^-8 of dS
          __half2 slopes[CAP ? 16 : 1];
          uint32_t pk[16];
          auto probabilities = [&](auto with_mask, auto is_small, auto is_large) {
            constexpr bool kMask = decltype(with_mask)::value, kSmall = decltype(is_small)::value, kLarge = decltype(is_large)::value;
#pragma unroll
            for (int i4 = 0; i4 < 8; ++i4) {
              float l[4] = {lse2, lse2, lse2, lse2};
              if (KEYS) {
                const float4 v = *reinterpret_cast<const float4*>(vec + 4 * i4);
                l[0] = v.x; l[1] = v.y; l[2] = v.z; l[3] = v.w;
              }
              float e[4], slope[4];
              auto score = [&](int k) { return make_float2(__uint_as_float(s[4 * i4 + k]), __uint_as_float(s[4 * i4 + k + 1])); };
              const float2 x01 = q8::fma2(score(0), q8::both(p.c), make_float2(-l[0], -l[1])),
                           x23 = q8::fma2(score(2), q8::both(p.c), make_float2(-l[2], -l[3]));
              float2 x[2] = {x01, x23};
              if (CAP || BIAS) {
                auto at = [&](int k) {
                  const int col = 4 * i4 + k;
                  return exponent<CAP, BIAS, kSmall>(p, __uint_as_float(s[col]), float(c0 - row) + float(col), slope2, &slope[k]) - l[k];
                };
                x[0] = make_float2(at(0), at(1));
                x[1] = make_float2(at(2), at(3));
              }
              if (kLarge) {
                constexpr float kTop = CAP ? -kCapShift : 0.f;
                x[0] = make_float2(bounded_exponent(x[0].x, l[0], kTop), bounded_exponent(x[0].y, l[1], kTop));
                x[1] = make_float2(bounded_exponent(x[1].x, l[2], kTop), bounded_exponent(x[1].y, l[3], kTop));
              }
#pragma unroll
              for (int k = 0; k < 2; ++k) {
                e[2 * k] = exp2_fast(x[k].x);
                e[2 * k + 1] = exp2_fast(x[k].y);
              }
#pragma unroll
              for (int k = 0; k < 4; ++k) {
                const int col = 4 * i4 + k;
                if (kMask) e[k] = col >= lo && col < hi ? e[k] : 0.f;
                if (CAP && kMask) slope[k] = col >= lo && col < hi ? slope[k] : 0.f;   // that of another document's tokens may be no number
                s[col] = __float_as_uint(e[k]);
                if (CAP && !KEYS) e[k] *= slope[k];   // what an error of delta is multiplied with
              }
              if (CAP) {
                slopes[CAP ? 2 * i4 : 0] = __floats2half2_rn(slope[0], slope[1]);
                slopes[CAP ? 2 * i4 + 1 : 0] = __floats2half2_rn(slope[2], slope[3]);
              }
              pk[2 * i4] = pack2(e[0], e[1]);
              pk[2 * i4 + 1] = pack2(e[2], e[3]);
            }
            if (kMask && KEYS && lonely && c0 == w.t.start) s[0] = 0u;
            if (kMask && !KEYS && lonely) {
#pragma unroll
              for (int k = 0; k < 32; ++k) s[k] = 0u;
            }
          };
          constexpr std::true_type yes{};
          constexpr std::false_type no{};
          // (the mask's bounds hold for tiles without one too: one form for all that is large)
          if (KEYS ? __any_sync(0xFFFFFFFFu, fabsf(vec[lane]) > kLargeLse) : large_row) probabilities(yes, no, yes);
          else if (masked) probabilities(yes, no, no);
          else if (CAP && small_scores(p, s, live)) probabilities(no, yes, no);
          else probabilities(no, no, no);
          // P to shared memory: this row's 64 bytes of the panel's 64-column chunk
          if (!warp_wait(p_free, (turns & 1) ^ 1u, abort_flag)) { give_up(); ok = false; break; }
#pragma unroll
          for (int q = 0; q < 4; ++q)
            *reinterpret_cast<uint4*>(p_row + ((((panel & 1) * 4 + q) ^ (r & 7)) << 4)) = make_uint4(pk[4 * q], pk[4 * q + 1], pk[4 * q + 2], pk[4 * q + 3]);
          ptx::fence_proxy_async_smem();
          __syncwarp();
          if (lane == 0) ptx::mbar_arrive(p_full);
          __syncwarp();
          if (!warp_wait(dp_full, turns & 1, abort_flag)) { give_up(); ok = false; break; }
          ptx::tcgen05_fence_after_sync();
          uint32_t g[32];
          ptx::tmem_ld_x32(dp_at, g);
          tmem_loaded(g);
          if (masked) {   // tokens of another document: their dP may be anything
#pragma unroll
            for (int k = 0; k < 32; ++k) g[k] = k >= lo && k < hi ? g[k] : __float_as_uint(delta);
          }
#pragma unroll
          for (int i4 = 0; i4 < 8; ++i4) {
            float2 d0 = q8::both(-delta), d1 = d0;
            if (KEYS) {
              const float4 v = *reinterpret_cast<const float4*>(vec + kRows + 4 * i4);
              d0 = make_float2(-v.x, -v.y);
              d1 = make_float2(-v.z, -v.w);
            }
            auto pair = [&](int k) { return make_float2(__uint_as_float(g[k]), __uint_as_float(g[k + 1])); };
            auto prob = [&](int k) { return make_float2(__uint_as_float(s[k]), __uint_as_float(s[k + 1])); };
            float2 e0 = q8::mul2(prob(4 * i4), q8::add2(pair(4 * i4), d0)), e1 = q8::mul2(prob(4 * i4 + 2), q8::add2(pair(4 * i4 + 2), d1));
            if (!KEYS) rest2 = q8::add2(rest2, q8::add2(e0, e1));
            if (CAP) {
              e0 = q8::mul2(e0, __half22float2(slopes[CAP ? 2 * i4 : 0]));
              e1 = q8::mul2(e1, __half22float2(slopes[CAP ? 2 * i4 + 1 : 0]));
            }
            pk[2 * i4] = pack2(e0.x, e0.y);
            pk[2 * i4 + 1] = pack2(e1.x, e1.y);
            if (KEYS) {
              s[4 * i4] = __float_as_uint(e0.x);
              s[4 * i4 + 1] = __float_as_uint(e0.y);
              s[4 * i4 + 2] = __float_as_uint(e1.x);
              s[4 * i4 + 3] = __float_as_uint(e1.y);
            }
            if (!KEYS) {
              const float2 r0 = unpack2(pk[2 * i4]), r1 = unpack2(pk[2 * i4 + 1]);
              // with a cap, whose slopes are in e by now, the roundings alone
              if (CAP) kept2 = q8::add2(kept2, q8::add2(q8::add2(r0, neg2(e0)), q8::add2(r1, neg2(e1))));
              else kept2 = q8::add2(kept2, q8::add2(r0, r1));
            }
          }
          ptx::tmem_st_x16(dp_at, pk);
          if (KEYS && two_parts(w.t)) {   // what the rounding left
#pragma unroll
            for (int i = 0; i < 16; ++i) {
              const float2 l = q8::add2(make_float2(__uint_as_float(s[2 * i]), __uint_as_float(s[2 * i + 1])), neg2(unpack2(pk[i])));
              pk[i] = pack2(l.x, l.y);
            }
            ptx::tmem_st_x16(dp_at + 16, pk);
          }
          ptx::tmem_st_wait();
          ptx::tcgen05_fence_before_sync();
          __syncwarp();
          if (lane == 0) {
            ptx::mbar_arrive(ds_full);
            if (KEYS) ptx::mbar_arrive(vec_empty(vs.stage));
          }
          __syncwarp();
        }
      }
      if (!ok) break;
      if (!KEYS) {
        // r of the row: the panels' parts, [0] + [2] and [1] + [3] first (room for two)
        float2 rest = make_float2(rest2.x + rest2.y, kept2.x + kept2.y);
        if (CAP) {
          rest.x *= kSlopeUnit;
          rest.y += rest.x;
        }
        float2* part = reinterpret_cast<float2*>(gen + M::kExchange);
        if (!warp_wait(parts_free, (it & 1) ^ 1u, abort_flag)) { give_up(); break; }   // those of the item before have been read
        if (panel < 2) part[panel * kRows + r] = rest;
        __syncwarp();
        if (lane == 0) ptx::mbar_arrive(parts_full);
        __syncwarp();
        if (!warp_wait(parts_full, 0u, abort_flag)) { give_up(); break; }
        if (panel >= 2) part[(panel - 2) * kRows + r] = q8::add2(part[(panel - 2) * kRows + r], rest);
        __syncwarp();
        if (lane == 0) ptx::mbar_arrive(parts_full);
        __syncwarp();
        if (!warp_wait(parts_full, 1u, abort_flag)) { give_up(); break; }
        rest = q8::add2(part[r], part[kRows + r]);
        __syncwarp();
        if (lane == 0) ptx::mbar_arrive(parts_free);
        __syncwarp();
        if (panel == 0 && live) p.delta[int64_t(w.head) * p.tokens + row] = delta + rest.x;
        __syncwarp();
        rest2.x = rest.y;
      }
      if (!warp_wait(out_full, it & 1, abort_flag)) { give_up(); break; }
      ptx::tcgen05_fence_after_sync();
      if (KEYS) {
        // panels 0 and 1 store dV's halves, 2 and 3 dK's
        const bool dk = panel >= 2;
        const int half = (panel & 1) * (HD / 2);
        const float f = dk ? p.scale : CAP ? kSlopeUnit : 1.f;
        float* part = dk ? p.dk_part : p.dv_part;
        if (part) part += ((int64_t(w.part) * p.tokens + row) * p.kv_heads + w.kv_head) * p.d;
        __nv_bfloat16* out = (dk ? p.dK + int64_t(row) * p.lddk : p.dV + int64_t(row) * p.lddv) + int64_t(w.kv_head) * p.d;
#pragma unroll
        for (int c = 0; c < HD / 64; ++c) {
          const int col = half + 32 * c;
          uint32_t o[32];
          ptx::tmem_ld_x32((dk ? tmem_second : tmem_first) + lanes + col, o);
          tmem_loaded(o);
          if (c == HD / 64 - 1) {
            ptx::tcgen05_fence_before_sync();
            __syncwarp();
            if (lane == 0) ptx::mbar_arrive(out_free);
            __syncwarp();
          }
          if (live && col < p.d) {
            if (part) store_f32(part + col, o, f, p.d - col);
            else store_bf16(out + col, o, f, p.d - col);
          }
          __syncwarp();
        }
      } else {
        // a panel stores a quarter of dQ's columns
        const int quarter_cols = HD / 4, col = panel * quarter_cols;
        uint32_t a[quarter_cols], b[quarter_cols];
        load_columns(tmem_second + lanes + col, a);
        load_columns(tmem_first + lanes + col, b);
        ptx::tmem_ld_wait();
        hand_over(a);
        hand_over(b);
        ptx::tcgen05_fence_before_sync();
        __syncwarp();
        if (lane == 0) ptx::mbar_arrive(out_free);
        __syncwarp();
#pragma unroll
        for (int k = 0; k < quarter_cols; ++k) a[k] = __float_as_uint(fmaf(-rest2.x, __uint_as_float(b[k]), __uint_as_float(a[k])));
        if (live && col < p.d) store_bf16(p.dQ + int64_t(row) * p.lddq + int64_t(w.head) * p.d + col, a, p.scale, p.d - col);
        __syncwarp();
      }
    }
  }
  __syncwarp();
  if (!fits) {
    // nothing
  } else if (KEYS) {
    zero_rows_outside(p, p.dK, p.lddk, p.kv_heads, nullptr, 0.f);
    zero_rows_outside(p, p.dV, p.lddv, p.kv_heads, nullptr, 0.f);
  } else {
    zero_rows_outside(p, p.dQ, p.lddq, p.heads, nullptr, 0.f);
  }
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
  if (!plan_fits(p)) return;
  const int head_end = __ldcg(&p.plan->head_end), tail = __ldcg(&p.plan->tail_begin);
  const int per_row = p.kv_heads * (p.d / 8);
  const int64_t n = int64_t(p.tokens) * per_row, k = int64_t(blockIdx.x) * blockDim.x + threadIdx.x;
  if (k >= n) return;
  const int64_t row = k / per_row, col = (k - row * per_row) * 8;
  if (row < head_end || row >= tail) return;
  const bool v = blockIdx.y != 0;
  const float* part = (v ? p.dv_part : p.dk_part) + row * (int64_t(p.kv_heads) * p.d) + col;
  float2 sum[4] = {};
#pragma unroll 4
  for (int i = 0; i < p.parts; ++i) {   // several on their way at a time
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
  const cudaError_t e = launch(once_q, attn_bwd_kernel<HD, false, CAP, BIAS>, Smem<HD, false>::kBytes, m, pq, grid_q, st);
  return e != cudaSuccess ? e : launch(once_k, attn_bwd_kernel<HD, true, CAP, BIAS>, Smem<HD, true>::kBytes, m, pk, grid_k, st);
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
