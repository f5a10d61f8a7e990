// Attention: the plan and the forward kernel.
//
// Forward, one work item: 256 queries of one head (two halves of 128) against the keys they see, tile by tile from the last one
// to the first (so that the masked tiles, and with a distance bias the largest scores, come first).  S = Q K^T of a half lies
// in 128 columns of tensor memory, one query per lane; a warpgroup reads its rows whole into registers, takes their maxima, and
// writes P = 2^(x - m) to shared memory as bf16, from where the tensor core multiplies it with V.  The next S is taken as soon as this
// one is in registers, so the warpgroups never wait for scores: with P written over S they did, for as long as they
// worked.
//
// The sums O are rescaled only where a row's maximum has grown by more than 2^8 since its reference m was taken (P then is at
// most 2^8, bf16 and fp32 hold that without loss of digits), which after the first tiles hardly ever happens; the row sums are
// taken from the unrounded fp32 exponentials.
//
// What bounds it: per tile of 128 x 128 and d = 128 the tensor core needs 2 x 512 cycles and the 16384 exponentials 1024 cycles of
// the special function units: both at once.  Measured: 8192 tokens x 24 heads (8 of keys) x 128, causal, 352 us, 1.17 PFLOP/s, 71 % of
// the rate of a large product, tensor pipe 60 % busy and exponentials 61 %; 16384 x 32 x 8 x 64 with distances 1603 us, 0.69 PFLOP/s: half
// the products per score.  No unit is full: one document of 4096 x 32 x 8, d = 64 with distances has exponentials 58 %, issue slots 49 %, tensor
// pipe 29 % (without 65, 38, 33; d = 128 58, 35, 58).  A scheduler has two rows' warps, which go through reading scores, maximum, exponentials
// and storing one after the other; of the cycles between two instructions of a warp the largest parts are fixed latencies and scores
// on their way from tensor memory.
//
// Roles (384 threads, one CTA per SM, persistent): warp 0 copies, warp 1 products and tensor memory, warps 4..7 and 8..11
// the rows of the two halves, with 208 registers a thread (the first warpgroup's threads keep 88: 128 x 88 + 256 x 208 is what
// the launch has).
#include <algorithm>

#include "acx_attn.cuh"
#include "acx_tmap.h"

namespace acx {
namespace attn {
namespace {

// ------------------------------------------------------------------------------------------------------------------- plan
constexpr int kPlanThreads = 1024, kBins = 1024;

__device__ __forceinline__ int block_scan(int v, int* warp_sums, int* total) {   // exclusive, over the block
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int x = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int y = __shfl_up_sync(0xFFFFFFFFu, x, o);
    if (lane >= o) x += y;
  }
  __syncthreads();
  if (lane == 31) warp_sums[warp] = x;
  __syncthreads();
  if (warp == 0) {
    int s = warp_sums[lane];
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int y = __shfl_up_sync(0xFFFFFFFFu, s, o);
      if (lane >= o) s += y;
    }
    warp_sums[lane] = s;
  }
  __syncthreads();
  *total = warp_sums[31];
  return x - v + (warp ? warp_sums[warp - 1] : 0);
}

// Three blocks, one for each list; all of them take the documents' running counts, the first writes the header.  Offsets that
// decrease or lie outside [0, tokens] are brought into it, lists never grow beyond their room: whatever the offsets hold, items name only
// tokens that exist.  Up to kHeld items stay in registers between the count of the bins and their places (7.5 us for one block and
// all three lists, one after the other).
constexpr int kHeld = 4;
__global__ void __launch_bounds__(kPlanThreads) plan_kernel(const int* __restrict__ offsets, const int* __restrict__ prefix, int docs, int tokens,
                                                            int causal, uint8_t* __restrict__ plan) {
  __shared__ int warp_sums[32];
  __shared__ int bins[kBins];
  __shared__ int cum_held[kPlanThreads + 1];
  bins[threadIdx.x] = 0;
  wait_for_launch_before();
  let_next_launch_start();
  const int list = blockIdx.x, rows = list == 0 ? 256 : 128;
  const PlanLayout at = plan_layout(tokens, docs);
  const int cap = int(list == 0 ? at.wide_cap : at.tile_cap);
  // running counts of the documents' tiles: in shared memory as far as they fit, else in the plan
  int* const cum = docs <= kPlanThreads ? cum_held : reinterpret_cast<int*>(plan + at.cum) + int64_t(list) * (docs + 1);
  auto clamped = [&](int i) { return min(max(__ldcg(offsets + i), 0), tokens); };
  int count = 0;
  for (int base = 0; base < docs; base += kPlanThreads) {
    const int i = base + int(threadIdx.x);
    const int n = i < docs ? max(clamped(i + 1) - clamped(i), 0) : 0;
    int total, before = 0;
    if (docs > 1) {
      before = block_scan((n + rows - 1) / rows, warp_sums, &total) + count;
    } else {
      total = __shfl_sync(0xFFFFFFFFu, (n + rows - 1) / rows, 0);   // of the first warp; the others read it below
      if (threadIdx.x == 0) warp_sums[0] = total;
      __syncthreads();
      total = warp_sums[0];
    }
    if (i < docs) cum[i] = min(before, cap);
    count = min(count + total, cap);
  }
  if (threadIdx.x == 0) {
    cum[docs] = count;
    PlanHeader* header = reinterpret_cast<PlanHeader*>(plan);
    if (list == 0) {
      header->wide = count;
      header->tokens = tokens;
      header->docs = docs;
      header->causal = causal;
      header->unused = 0;
      const int first = docs > 0 ? clamped(0) : tokens;
      header->head_end = first;
      header->tail_begin = docs > 0 ? max(clamped(docs), first) : tokens;
    } else if (list == 1) {
      header->tiles = count;
    }
  }
  __syncthreads();
  const int most = (tokens + 127) / 128 + 1;
  Item* out = reinterpret_cast<Item*>(plan + (list == 0 ? at.wide : list == 1 ? at.queries : at.keys));
  auto item = [&](int k, int* bin) {
    int lo = 0, hi = docs;   // the last document whose first tile is at or before k
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (cum[mid] <= k) lo = mid; else hi = mid;
    }
    Item t;
    t.start = clamped(lo);
    t.end = max(clamped(lo + 1), t.start);
    t.prefix = causal && prefix ? t.start + min(max(__ldcg(prefix + lo), 0), t.end - t.start) : t.start;
    t.row0 = t.start + (k - cum[lo]) * rows;
    int work;   // tiles on the other side
    if (list < 2) work = (causal ? max(min(t.row0 + rows, t.end), t.prefix) : t.end) - t.start;
    else work = t.end - (causal && t.row0 >= t.prefix ? t.row0 : t.start);
    *bin = kBins - 1 - int(int64_t(min((work + 127) / 128, most)) * (kBins - 1) / most);
    return t;
  };
  Item held[kHeld];
  int bin[kHeld];
#pragma unroll
  for (int h = 0; h < kHeld; ++h) {
    const int k = h * kPlanThreads + int(threadIdx.x);
    if (k < count) {
      held[h] = item(k, &bin[h]);
      atomicAdd(&bins[bin[h]], 1);
    }
  }
  for (int k = kHeld * kPlanThreads + int(threadIdx.x); k < count; k += kPlanThreads) {
    int b;
    item(k, &b);
    atomicAdd(&bins[b], 1);
  }
  __syncthreads();
  int total;
  const int first = block_scan(bins[threadIdx.x], warp_sums, &total);
  bins[threadIdx.x] = first;
  __syncthreads();
  // the order within a bin does not matter: an item's results are its own
#pragma unroll
  for (int h = 0; h < kHeld; ++h)
    if (h * kPlanThreads + int(threadIdx.x) < count) out[atomicAdd(&bins[bin[h]], 1)] = held[h];
  for (int k = kHeld * kPlanThreads + int(threadIdx.x); k < count; k += kPlanThreads) {
    int b;
    const Item t = item(k, &b);
    out[atomicAdd(&bins[b], 1)] = t;
  }
}
static_assert(kBins == kPlanThreads, "one bin per thread");

// ---------------------------------------------------------------------------------------------------------------- forward
constexpr int kFwdThreads = 384;
// Work items have 256 queries, whose halves take turns with the products; where that leaves SMs without an item they have 128, and one
// half of the rows' warps has nothing to do.  Items are counted from the batch's tokens; uneven documents make more of them, which the host does
// not know (2048 tokens x 16 heads x 64, 128 items of 256: 30.2 us, 24.1 in items of 128; 3001 x 6 x
// 72 with a cap 52.9 and 48.6; but 4096 x 14 x 64, 224 items: 54 and 70).
template <int HD>
struct FwdSmem {
  static constexpr int kStages = HD == 128 ? 3 : 6;
  static constexpr int kP = 2 * Tile<HD>::kBytes, kPBytes = kRows * kRows * 2;      // behind the two halves of Q
  static constexpr int kTiles = kP + 2 * kPBytes, kBars = kTiles + kStages * Tile<HD>::kBytes;
  static constexpr int kBytes = kBars + 256;
  static_assert(kBytes <= 232448, "shared memory of one CTA");
};

template <int HD, bool CAP, bool BIAS, int HALVES>
__global__ void __launch_bounds__(kFwdThreads, 1)
    attn_fwd_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k,
                    const __grid_constant__ CUtensorMap map_v, const Params p) {
  using T = Tile<HD>;
  constexpr int kStages = FwdSmem<HD>::kStages;
  extern __shared__ __align__(1024) uint8_t gen[];   // tiles start on their swizzle's boundary
  const uint32_t base = ptx::smem_u32(gen);
  const uint32_t bars = base + FwdSmem<HD>::kBars;
  auto full = [&](int s) { return bars + 8u * s; };
  auto empty = [&](int s) { return bars + 8u * (kStages + s); };
  const uint32_t misc = bars + 16u * kStages;
  const uint32_t q_full = misc, q_empty = misc + 8, done = misc + 16;
  auto s_full = [&](int h) { return misc + 24 + 8u * h; };
  auto s_free = [&](int h) { return misc + 40 + 8u * h; };
  auto p_full = [&](int h) { return misc + 56 + 8u * h; };
  auto p_free = [&](int h) { return misc + 72 + 8u * h; };
  auto o_full = [&](int h) { return misc + 88 + 8u * h; };
  auto o_free = [&](int h) { return misc + 104 + 8u * h; };
  constexpr int kSlot = FwdSmem<HD>::kBars + 16 * kStages + 120;
  volatile uint32_t* tmem_slot = reinterpret_cast<volatile uint32_t*>(gen + kSlot);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(gen + kSlot + 4);
  volatile int* no_abort = abort_flag + 1;   // for the one wait that has to run its time even so
  const int warp = __shfl_sync(0xFFFFFFFFu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;   // the warp's number, known to be the same in all lanes

  if (threadIdx.x == 0) {
    for (int s = 0; s < kStages; ++s) {
      ptx::mbar_init(full(s), 1);
      ptx::mbar_init(empty(s), 1);
    }
    ptx::mbar_init(q_full, 1);
    ptx::mbar_init(q_empty, 1);
    ptx::mbar_init(done, 1);
    *no_abort = 0;
    for (int h = 0; h < 2; ++h) {
      ptx::mbar_init(s_full(h), 1);
      ptx::mbar_init(s_free(h), 4);
      ptx::mbar_init(p_full(h), 4);
      ptx::mbar_init(p_free(h), 1);
      ptx::mbar_init(o_full(h), 1);
      ptx::mbar_init(o_free(h), 4);
    }
    *abort_flag = 0;
    ptx::fence_barrier_init();   // no prefetch of the tensor maps: a block without work would leave with it in flight
  }
  // A warp comes to the barrier as a whole: halves of it would count as two, and let the others read the address before it is there
  __syncwarp();
  if (warp == 1) {
    ptx::tmem_alloc(base + kSlot, 512);
    ptx::tmem_relinquish_alloc_permit();
    __syncwarp();
  }
  ptx::tcgen05_fence_before_sync();
  __syncthreads();
  ptx::tcgen05_fence_after_sync();
  const uint32_t tmem = *tmem_slot;
  auto tmem_s = [&](int h) { return tmem + 128u * h; };
  auto tmem_o = [&](int h) { return tmem + 256u + HD * h; };
  wait_for_launch_before();
  let_next_launch_start();
  const bool fits = plan_fits(p);
  const int units = fits ? __ldcg(HALVES == 2 ? &p.plan->wide : &p.plan->tiles) * p.heads : 0;
  auto give_up = [&]() {
    *abort_flag = 1;
    atomicExch(p.status, kDevTimeout);
  };
  // key tiles that a half of the queries sees
  auto key_tiles = [&](const Item& t, int half) {
    const int r = t.row0 + kRows * half;
    if (r >= t.end) return 0;
    return ((p.causal ? max(min(r + kRows, t.end), t.prefix) : t.end) - t.start + kRows - 1) / kRows;
  };

  if (warp < 4) asm volatile("setmaxnreg.dec.sync.aligned.u32 88;");
  if (warp == 0) {
    // ---------------------------------------------------------------------------------------------------- copies
    if (lane == 0) {
      int stage = 0, it = 0;
      uint32_t phase = 0;
      bool ok = true;
      auto push = [&](const CUtensorMap* map, int head, int row) {
        if (!ptx::mbar_wait(empty(stage), phase ^ 1u, abort_flag)) { give_up(); ok = false; return; }
        ptx::mbar_arrive_expect_tx(full(stage), T::kBytes);
        T::load(base + FwdSmem<HD>::kTiles + stage * T::kBytes, map, full(stage), head, row);
        if (++stage == kStages) { stage = 0; phase ^= 1u; }
      };
      for (int u; ok && (u = unit_of(it)) < units; ++it) {
        const Item t = fetch_item(p.items, u / p.heads);
        const int h = u % p.heads, g = h / p.group;
        const int n1 = HALVES == 2 ? key_tiles(t, 1) : 0, n = max(key_tiles(t, 0), n1);
        if (!ptx::mbar_wait(q_empty, (it & 1) ^ 1u, abort_flag)) { give_up(); ok = false; break; }
        ptx::mbar_arrive_expect_tx(q_full, (n1 ? 2 : 1) * T::kBytes);
        T::load(base, &map_q, q_full, h, t.row0);
        if (n1) T::load(base + T::kBytes, &map_q, q_full, h, t.row0 + kRows);
        // in the order of their use: a tile's keys one turn ahead of its values
        push(&map_k, g, t.start + (n - 1) * kRows);
        for (int j = n - 1; ok && j >= 0; --j) {
          if (j > 0) push(&map_k, g, t.start + (j - 1) * kRows);
          if (ok) push(&map_v, g, t.start + j * kRows);
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
    int stage = 0, it = 0, reads[2] = {0, 0}, turns[2] = {0, 0}, outs[2] = {0, 0};
    uint32_t phase = 0;
    bool ok = true;
    const int d16 = (p.d + 15) / 16;
    auto wait = [&](uint32_t bar, uint32_t parity) {
      if (ok && !warp_wait(bar, parity, abort_flag)) { give_up(); ok = false; }
      return ok;
    };
    struct Slot { int stage; uint32_t phase; };
    auto next = [&]() {
      const Slot s{stage, phase};
      if (++stage == kStages) { stage = 0; phase ^= 1u; }
      return s;
    };
    auto addr = [&](Slot s) { return base + FwdSmem<HD>::kTiles + s.stage * T::kBytes; };
    for (int u; ok && (u = unit_of(it)) < units; ++it) {
      const Item t = fetch_item_warp(p.items, u / p.heads);
      const int nt[2] = {key_tiles(t, 0), HALVES == 2 ? key_tiles(t, 1) : 0}, n = max(nt[0], nt[1]);
      // scores of key tile j for the halves that see it, each once its scores before have been read
      auto scores = [&](int j) {
        const Slot k = next();
        if (!wait(full(k.stage), k.phase)) return;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          if (j >= nt[h]) continue;
          if (!wait(s_free(h), (reads[h] & 1) ^ 1u)) return;
          ++reads[h];
          ptx::tcgen05_fence_after_sync();
          scores_mma<HD>(tmem_s(h), base + h * T::kBytes, addr(k), d16);
          ptx::umma_commit_elected(s_full(h));
        }
        ptx::umma_commit_elected(empty(k.stage));
        if (j == 0) ptx::umma_commit_elected(q_empty);
      };
      if (!wait(q_full, it & 1)) break;
      scores(n - 1);
      for (int j = n - 1; ok && j >= 0; --j) {
        if (j > 0) scores(j - 1);
        const Slot v = next();
        if (!wait(full(v.stage), v.phase)) break;
        const int left = t.end - (t.start + j * kRows);   // keys of this tile inside the document
        const int steps = min(kRows, left + 15) / 16;
        if (left < 16 * steps) T::zero_rows(gen + (addr(v) - base), left, 16 * steps);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          if (j >= nt[h]) continue;
          if (j == nt[h] - 1 && !wait(o_free(h), (outs[h] & 1) ^ 1u)) break;
          if (!wait(p_full(h), turns[h] & 1)) break;
          ++turns[h];
          ptx::tcgen05_fence_after_sync();
          smem_rows_mma<HD>(tmem_o(h), base + FwdSmem<HD>::kP + h * FwdSmem<HD>::kPBytes, addr(v), steps, d16, j < nt[h] - 1);
          ptx::umma_commit_elected(p_free(h));
          if (j == 0) {
            ptx::umma_commit_elected(o_full(h));
            ++outs[h];
          }
        }
        ptx::umma_commit_elected(empty(v.stage));
      }
    }
    // everything that was issued has to be done before the tensor memory is given back
    if (it > 0 || !ok) {
      ptx::umma_commit_elected(done);
      warp_wait(done, 0, no_abort);
    }
    __syncwarp();
  } else if (warp >= 4) {
    // ---------------------------------------------------------------------------------------------------- rows
    asm volatile("setmaxnreg.inc.sync.aligned.u32 208;");
    const int half = (warp - 4) >> 2, quarter = warp & 3, r = 32 * quarter + lane;
    const uint32_t lanes = uint32_t(32 * quarter) << 16;
    const uint32_t s_at = tmem_s(half) + lanes, o_at = tmem_o(half) + lanes;
    uint8_t* const p_row = gen + FwdSmem<HD>::kP + half * FwdSmem<HD>::kPBytes + r * 128;
    int turns = 0, outs = 0, it = 0;
    bool ok = half < HALVES;
    for (int u; ok && (u = unit_of(it)) < units; ++it) {
      const Item t = fetch_item_warp(p.items, u / p.heads);
      const int n = key_tiles(t, half), head = u % p.heads;
      if (n == 0) continue;
      const int r0 = t.row0 + kRows * half, row = r0 + r;
      const int sees = p.causal ? min(max(row + 1, t.prefix), t.end) : t.end;       // this row: keys [start, sees)
      const int all_see = p.causal ? min(max(r0 + 1, t.prefix), t.end) : t.end;     // every row of the half
      const float slope2 = BIAS ? __ldg(p.slopes + head) * kLog2e : 0.f;
      float m = 0.f, l = 0.f;
      for (int j = n - 1; j >= 0; --j, ++turns) {
        if (!warp_wait(s_full(half), turns & 1, abort_flag)) { give_up(); ok = false; break; }
        ptx::tcgen05_fence_after_sync();
        uint32_t s[4][32];
#pragma unroll
        for (int c = 0; c < 4; ++c) ptx::tmem_ld_x32(s_at + 32 * c, s[c]);
        tmem_loaded(s[0], s[1], s[2], s[3]);
        ptx::tcgen05_fence_before_sync();
        __syncwarp();
        if (lane == 0) ptx::mbar_arrive(s_free(half));
        __syncwarp();
        const int k0 = t.start + j * kRows;
        constexpr bool kRaw = !CAP && !BIAS;   // raw scores: the scale is left to the exponent's fma
        float scale = kRaw ? p.c : 1.f;
        if (CAP) {
          auto capped = [&](auto is_small) {
#pragma unroll
            for (int c = 0; c < 4; ++c)
#pragma unroll
              for (int i = 0; i < 32; ++i)
                s[c][i] = __float_as_uint(exponent<CAP, BIAS, decltype(is_small)::value>(p, __uint_as_float(s[c][i]),
                                                                                          float(row - k0) - float(32 * c + i), slope2));
          };
          const bool live = row < t.end;
          if (small_scores(p, s[0], live) && small_scores(p, s[1], live) && small_scores(p, s[2], live) && small_scores(p, s[3], live)) capped(std::true_type{});
          else capped(std::false_type{});
        } else if (BIAS) {
          const float2 c2 = q8::both(p.c);
          const float d = float(row - k0);
          if (k0 + kRows <= r0) {
            // every key is before every query, the distance needs no magnitude: x = c s + slope column - slope (row - k0)
            const float2 slopes = q8::both(slope2), from = q8::both(-slope2 * d);
#pragma unroll
            for (int c = 0; c < 4; ++c)
#pragma unroll
              for (int i = 0; i < 32; i += 2) {
                const float2 x = q8::fma2(make_float2(__uint_as_float(s[c][i]), __uint_as_float(s[c][i + 1])), c2,
                                          q8::fma2(slopes, make_float2(float(32 * c + i), float(32 * c + i + 1)), from));
                s[c][i] = __float_as_uint(x.x);
                s[c][i + 1] = __float_as_uint(x.y);
              }
          } else {
#pragma unroll
            for (int c = 0; c < 4; ++c)
#pragma unroll
              for (int i = 0; i < 32; ++i)
                s[c][i] = __float_as_uint(fmaf(__uint_as_float(s[c][i]), p.c, -slope2 * fabsf(d - float(32 * c + i))));
          }
        }
        if (k0 + kRows > all_see) {
          const int limit = sees - k0;
#pragma unroll
          for (int c = 0; c < 4; ++c)
#pragma unroll
            for (int i = 0; i < 32; ++i)
              if (32 * c + i >= limit) s[c][i] = 0xFF800000u;   // minus infinity
        }
        float top[4];
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          top[c] = max_nan(__uint_as_float(s[c][0]), __uint_as_float(s[c][1]));
#pragma unroll
          for (int i = 2; i < 32; i += 2) top[c] = max_nan(top[c], __uint_as_float(s[c][i]), __uint_as_float(s[c][i + 1]));
        }
        const float mx = max_nan(max_nan(top[0], top[1], top[2]), top[3]) * scale;
        // The fma takes a rounded maximum from an exact product: off by 2^-24 |mx|, which is 2^-12 at 2^12 and anything for scores of
        // a mask's size.  Rows beyond round the products too.
        if (kRaw) {
          const bool large = fabsf(mx) > 4096.f;
          if (__any_sync(0xFFFFFFFFu, large)) {
            const float2 f = q8::both(large ? p.c : 1.f);
#pragma unroll
            for (int c = 0; c < 4; ++c)
#pragma unroll
              for (int i = 0; i < 32; i += 2) {
                const float2 x = q8::mul2(make_float2(__uint_as_float(s[c][i]), __uint_as_float(s[c][i + 1])), f);
                s[c][i] = __float_as_uint(x.x);
                s[c][i + 1] = __float_as_uint(x.y);
              }
            if (large) scale = 1.f;
          }
        }
        // the products with the P before are done: P's place is free, and the sums may be rescaled
        if (!warp_wait(p_free(half), (turns & 1) ^ 1u, abort_flag)) { give_up(); ok = false; break; }
        // (a score that is not a number: the row's sums become that.  A row's reference is its own affair, the warp only goes along:
        // rows behind the document's end, of another document, change nothing of the others' roundings.)
        const bool above = row < t.end && !(mx <= m + 8.f);
        if (j == n - 1) {
          m = max_nan(mx, -3.402823466e38f);   // (a tile whose scores are all minus infinity: weights of zero, and tiles to come may have others)
        } else if (__any_sync(0xFFFFFFFFu, above)) {
          ptx::tcgen05_fence_after_sync();
          const float m_new = above ? max_nan(m, mx) : m, f = above ? exp2_fast(m - m_new) : 1.f;
          m = m_new;
          l *= f;
#pragma unroll 1
          for (int c = 0; c < HD / 16; ++c) {
            uint32_t o[16];
            ptx::tmem_ld_x16(o_at + 16 * c, o);
            tmem_loaded(o);
#pragma unroll
            for (int i = 0; i < 16; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * f);
            ptx::tmem_st_x16(o_at + 16 * c, o);
          }
          ptx::tmem_st_wait();
          ptx::tcgen05_fence_before_sync();
        }
        float2 sum[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
        const float2 scale2 = q8::both(scale), m2 = q8::both(-m);
#pragma unroll
        for (int c = 0; c < 4; ++c) {
#pragma unroll
          for (int q = 0; q < 4; ++q) {   // eight columns: 16 bytes
            uint32_t w[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const int k = 8 * q + 2 * i;
              const float2 x = q8::fma2(make_float2(__uint_as_float(s[c][k]), __uint_as_float(s[c][k + 1])), scale2, m2);
              const float2 e = make_float2(exp2_fast(x.x), exp2_fast(x.y));
              sum[i & 1] = q8::add2(sum[i & 1], e);
              w[i] = pack2(e.x, e.y);
            }
            *reinterpret_cast<uint4*>(p_row + (c >> 1) * (kRows * 128) + ((((c & 1) * 4 + q) ^ (r & 7)) << 4)) = make_uint4(w[0], w[1], w[2], w[3]);
          }
        }
        l += (sum[0].x + sum[0].y) + (sum[1].x + sum[1].y);
        ptx::fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) ptx::mbar_arrive(p_full(half));
        __syncwarp();
      }
      if (!ok) break;
      if (!warp_wait(o_full(half), outs & 1, abort_flag)) { give_up(); break; }
      ++outs;
      ptx::tcgen05_fence_after_sync();
      const float f = 1.f / l;
      __nv_bfloat16* at = p.O + int64_t(row) * p.ldo + int64_t(head) * p.d;
#pragma unroll 1
      for (int c = 0; c < HD / 32; ++c) {
        if (32 * c >= p.d) break;
        uint32_t o[32];
        ptx::tmem_ld_x32(o_at + 32 * c, o);
        tmem_loaded(o);
        if (32 * (c + 1) >= p.d) {   // all read
          ptx::tcgen05_fence_before_sync();
          __syncwarp();
          if (lane == 0) ptx::mbar_arrive(o_free(half));
          __syncwarp();
        }
        if (row < t.end) store_bf16(at + 32 * c, o, f, p.d - 32 * c);
        __syncwarp();
      }
      if (p.lse && row < t.end) p.lse[int64_t(head) * p.tokens + row] = (m + log2f(l)) * kLn2;
      __syncwarp();
    }
  }
  __syncwarp();
  if (fits) zero_rows_outside(p, p.O, p.ldo, p.heads, p.lse, __int_as_float(0xFF800000));
  __syncwarp();
  ptx::tcgen05_fence_before_sync();
  __syncthreads();
  if (warp == 1) {
    __syncwarp();
    ptx::tcgen05_fence_after_sync();
    ptx::tmem_dealloc(tmem, 512);
  }
}

template <int HD, bool CAP, bool BIAS, int HALVES>
cudaError_t launch_fwd(const CUtensorMap& q, const CUtensorMap& k, const CUtensorMap& v, const Params& p, unsigned grid, cudaStream_t st) {
  static DeviceOnce once;
  const auto kernel = attn_fwd_kernel<HD, CAP, BIAS, HALVES>;
  if (once.needed()) {
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, FwdSmem<HD>::kBytes);
    if (e != cudaSuccess) return e;
    once.done();
  }
  return launch_lined_up(kernel, dim3(grid), dim3(kFwdThreads), FwdSmem<HD>::kBytes, st, q, k, v, p);
}
template <int HD, int HALVES>
cudaError_t launch_fwd(bool cap, bool bias, const CUtensorMap& q, const CUtensorMap& k, const CUtensorMap& v, const Params& p, unsigned grid,
                       cudaStream_t st) {
  if (cap) return bias ? launch_fwd<HD, true, true, HALVES>(q, k, v, p, grid, st) : launch_fwd<HD, true, false, HALVES>(q, k, v, p, grid, st);
  return bias ? launch_fwd<HD, false, true, HALVES>(q, k, v, p, grid, st) : launch_fwd<HD, false, false, HALVES>(q, k, v, p, grid, st);
}
template <int HD>
cudaError_t launch_fwd(int halves, bool cap, bool bias, const CUtensorMap& q, const CUtensorMap& k, const CUtensorMap& v, const Params& p,
                       unsigned grid, cudaStream_t st) {
  return halves == 2 ? launch_fwd<HD, 2>(cap, bias, q, k, v, p, grid, st) : launch_fwd<HD, 1>(cap, bias, q, k, v, p, grid, st);
}

}  // namespace

Params common_params(const AttnProblem& q, const void* plan, const float* slopes, float* lse, int* status) {
  Params p{};
  p.tokens = int(q.tokens);
  p.docs = int(q.docs);
  p.heads = q.heads;
  p.kv_heads = q.kv_heads;
  p.group = q.heads / q.kv_heads;
  p.d = q.d;
  p.causal = q.causal;
  p.plan = static_cast<const PlanHeader*>(plan);
  p.slopes = slopes;
  p.scale = q.scale;
  p.c = q.scale * kLog2e;
  p.cap_in = q.softcap > 0.f ? q.scale / q.softcap * kTanhUnit : 0.f;
  p.cap_out = q.softcap * kLog2e / kTanhUnit;
  p.lse = lse;
  p.status = status;
  return p;
}

}  // namespace attn

using namespace attn;

size_t attn_plan_bytes(const AttnProblem& q) { return plan_layout(q.tokens, q.docs).bytes; }

cudaError_t attn_plan(const AttnProblem& q, const int* offsets, const int* prefix, void* plan, cudaStream_t st) {
  return launch_lined_up(plan_kernel, dim3(3), dim3(kPlanThreads), 0, st, offsets, prefix, int(q.docs), int(q.tokens), q.causal,
                         static_cast<uint8_t*>(plan));
}

cudaError_t attn_fwd(const AttnProblem& q, const AttnMatrix& Q, const AttnMatrix& K, const AttnMatrix& V, const float* slopes, const void* plan,
                     const AttnMatrix& O, float* lse, int* status, cudaStream_t st) {
  Params p = common_params(q, plan, slopes, lse, status);
  const PlanLayout at = plan_layout(q.tokens, q.docs);
  const int halves = q.tokens / (2 * kRows) * q.heads > sm_count() ? 2 : 1;
  p.items = reinterpret_cast<const Item*>(static_cast<const uint8_t*>(plan) + (halves == 2 ? at.wide : at.queries));
  p.O = static_cast<__nv_bfloat16*>(O.p);
  p.ldo = O.ld;
  CUtensorMap mq, mk, mv;
  if (!make_tmap_heads(&mq, Q.p, q.tokens, q.heads, q.d, Q.ld, kRows) || !make_tmap_heads(&mk, K.p, q.tokens, q.kv_heads, q.d, K.ld, kRows) ||
      !make_tmap_heads(&mv, V.p, q.tokens, q.kv_heads, q.d, V.ld, kRows))
    return cudaErrorInvalidValue;
  const unsigned grid = unsigned(std::min<int64_t>((halves == 2 ? at.wide_cap : at.tile_cap) * q.heads, sm_count()));
  const bool cap = q.softcap > 0.f, bias = slopes != nullptr;
  return q.d <= 64 ? launch_fwd<64>(halves, cap, bias, mq, mk, mv, p, grid, st) : launch_fwd<128>(halves, cap, bias, mq, mk, mv, p, grid, st);
}

}  // namespace acx
