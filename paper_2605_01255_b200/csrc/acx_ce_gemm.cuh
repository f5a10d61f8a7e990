// The tcgen05 kernels of the vocabulary cross entropy: persistent, warp-specialised, on pairs of CTAs (a cluster of two
// drives tcgen05.mma.cta_group::2 on a tile of 256 x 256).  Three kinds share the mainloop and differ in their epilogue:
//
//   LSE      logits tile = X W^T; every row of the tile leaves its maximum and its sum of exponentials over 64 columns,
//            its target's left out: 32 bytes instead of 1 KiB of fp32 logits;
//   DLOGITS  the same tile again, now D = w (exp(logit - lse) - onehot), rounded to bf16, for one piece of the vocabulary;
//   GRADS    both products of a finished piece in one launch: dX += D W_piece (split over the piece when there are few
//            tiles; fp32 sums in global memory, added by the bulk-copy engine) and dW_piece = D^T X (bf16, complete).
//
// What bounds them: the tensor cores, from a few hundred tokens on; with fewer the bytes of W.  Per SM a 256 x 256 pair
// tile takes K / 16 instructions of 128 cycles.  Its epilogue (128 x 256 elements per CTA: 2048 cycles of exponentials at
// least) is hidden behind the next tile's mainloop by the second accumulator where d is large enough for that; sixteen
// warps share it: with eight the latencies of its dependent steps bound tiles of small d (LSE of 4096 x 128 x 65536: 172 us,
// 117 with sixteen and the accumulator handed back as soon as it is read).
//
// FEW: at most 64 tokens.  A tile of 256 tokens would be mostly empty rows, and the tensor core takes as long for those: with
// 64 tokens and 2048 columns the logits of 128256 words were bound by it (119 us under sustained load, at 1.3 GHz under the
// power limit) instead of by the 525 MB of W.  So the operands change places: W's rows (of the logits; W's columns for dX)
// are the 256 rows of the tile and the tokens its 32 or 64 columns, a quarter of the instructions' time, and the smaller
// stages leave room for nine.  A lane then has a word, and keeps its own maximum and sum per token over all its tiles.
//
// Roles per CTA (576 threads, one CTA per SM): warp 0 TMA producer, warp 1 UMMA issuer (of the leader) and owner of the
// tensor memory, warps 2..17 epilogue: four per TMEM lane quarter, 64 columns each.  Six 32 KiB stages; all waits bounded.
// Loads are plain bulk tensor copies (no cluster multicast).
#pragma once
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <type_traits>

#include "acx_internal.h"
#include "acx_q8.cuh"
#include "acx_umma.cuh"

namespace acx {
namespace ce {

constexpr int kBM = 128;                   // rows of the tile per CTA (a pair: 256)
constexpr int kTile = 256;                 // rows and columns of a pair's tile
constexpr int kBK = 64;                    // bf16 per stage along K: one 128-byte swizzle row
constexpr int kUmmaK = 16;
constexpr int kFewTokens = 64;
constexpr int kPutBackTokens = 512;        // see ce_put_back_kernel
constexpr int kABytes = kBM * kBK * 2, kBBytes = kBM * kBK * 2;
constexpr int kFewBBytes = kFewTokens / 2 * kBK * 2;   // FEW: half of the tokens per CTA
constexpr int kStagesBytes = 6 * (kABytes + kBBytes);
// Stages: six of 32 KiB; nine of 20 KiB where the tokens are the narrow operand of every unit (dW needs the whole 32 KiB)
template <int KIND, bool FEW>
struct Stages {
  static constexpr bool kNarrow = FEW && KIND != 2;
  static constexpr int kCount = kNarrow ? 9 : 6, kBytes = kABytes + (kNarrow ? kFewBBytes : kBBytes);
  static_assert(kCount * kBytes <= kStagesBytes, "stages");
};
constexpr int kChunkBytes = 64 * kBK * 2;  // MN-major operand: 64 k-rows of 128 bytes
constexpr int kAccCols = 256, kTmemCols = 512;
constexpr int kEpiWarp0 = 2, kEpiWarps = 16, kGroupCols = 64, kThreads = 32 * (kEpiWarp0 + kEpiWarps);
constexpr int kBoxBytes = 16 * 128;        // store staging, one box per epilogue warp: 16 rows of 128 bytes, 128-byte swizzle
constexpr int kBarBytes = 1024;
constexpr int kOutOffset = kStagesBytes + kBarBytes;
constexpr int kSmemBytes = kOutOffset + kEpiWarps * kBoxBytes + 1024;
static_assert(kSmemBytes <= 232448, "shared memory of one CTA");

enum Kind { LSE = 0, DLOGITS = 1, GRADS = 2 };
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
// The maximum of logits of which none is more than minus infinity, with a sum of zero: a finite number, so that no difference
// of two maxima is one of infinities (which would turn a sum that holds nothing into a NaN).
constexpr float kLowest = -0x1.fffffep127f;

struct Params {
  int tokens, d, vocab;
  int units;                    // work units of this launch: CTA pair c takes c, c + pairs, ...
  // LSE, DLOGITS: tiles (token tile, vocabulary tile); the token tiles go in groups of `group` that pass over all the
  // vocabulary tiles together, so that a group's rows of X stay in L2 while W streams by once per group.
  int m_tiles, n_tiles, group;
  int v0;                       // first vocabulary column of the piece (DLOGITS, GRADS)
  // GRADS: x_units of dX = splits x m_tiles x d_tiles (the long ones first), then dW: piece_tiles x d_tiles
  int d_tiles, d_width;         // columns of d per tile: a multiple of 32
  int x_units, kb_per_split, piece_kb, token_kb;
  int acc_rows;                 // rows of one split's fp32 sums (tokens rounded up to whole tiles)
  int first_piece;              // the sums are stored, not added
  int few_n;                    // FEW: tokens rounded up to 32
  __nv_bfloat16* D;             // FEW, DLOGITS: the piece's D, [tokens][ld_d]
  int64_t ld_d;
  float* acc;                   // FEW, GRADS: the fp32 sums of dX, [split][acc_rows][d]
  int wait_first;               // this launch needs what the launch before it writes (else only what the one before that does)
  float c;                      // logit_scale * log2(e): exponents are taken in base 2
  const int64_t* targets;
  const float* lse;             // natural logarithm
  const float* loss;            // DLOGITS: may be null; minus the logarithm of the target's probability
  const float* weight;          // may be null: one
  float2* part;                 // LSE: [.][tokens] (maximum, sum) in base 2 of all words but the target: of 64 columns each;
                                // FEW: of what 32 lanes met
  uint32_t* ticket;             // LSE: set to zero for the kernel behind it
  float* corr;                  // DLOGITS: [tokens] what rounding took from the target's element of D
  const int* row_key;           // GRADS: [tokens], may be null: the row of dW that `row_add` belongs to, -1: none
  const float* row_add;         // GRADS: [tokens][d], added to that row before it is rounded (see ce_put_back_kernel)
  const float* denom;           // GRADS: may be null; gradients are multiplied by scale / denom
  float scale;
  int* status;
};

struct Unit {
  bool x;          // GRADS: a tile of dX (else of dW)
  int m0, n0;      // first row and column of the pair's tile
  int bn;          // columns (a multiple of 32, at most 256)
  int kb0, kb1;    // k-blocks
  int split;
};

template <int KIND, bool FEW>
__device__ __forceinline__ Unit decode(const Params& p, int u) {
  Unit t;
  t.split = 0;
  t.x = false;
  t.bn = kTile;
  if (FEW && (KIND != GRADS || u < p.x_units)) {   // rows: words of the piece, or columns of d
    t.x = KIND == GRADS;
    t.n0 = 0;
    t.bn = p.few_n;
    if (KIND != GRADS) {
      t.m0 = u * kTile;
      t.kb0 = 0;
      t.kb1 = (p.d + kBK - 1) / kBK;
    } else {
      const int tiles = (p.d + kTile - 1) / kTile;
      t.m0 = (u % tiles) * kTile;
      t.split = u / tiles;
      t.kb0 = t.split * p.kb_per_split;
      t.kb1 = min(p.piece_kb, t.kb0 + p.kb_per_split);
    }
    return t;
  }
  if (KIND != GRADS) {
    const int per_group = p.group * p.n_tiles, g = u / per_group, r = u - g * per_group;
    const int gm = min(p.group, p.m_tiles - g * p.group);
    t.m0 = (g * p.group + r % gm) * kTile;
    t.n0 = (r / gm) * kTile;
    t.kb0 = 0;
    t.kb1 = (p.d + kBK - 1) / kBK;
    return t;
  }
  int nt;
  if (u < p.x_units) {
    t.x = true;
    nt = u % p.d_tiles;
    const int r = u / p.d_tiles;
    t.m0 = (r % p.m_tiles) * kTile;
    t.split = r / p.m_tiles;
    t.kb0 = t.split * p.kb_per_split;
    t.kb1 = min(p.piece_kb, t.kb0 + p.kb_per_split);
  } else {
    const int v = u - p.x_units;
    nt = v % p.d_tiles;
    t.m0 = (v / p.d_tiles) * kTile;
    t.kb0 = 0;
    t.kb1 = p.token_kb;
  }
  t.n0 = nt * p.d_width;
  t.bn = min(p.d_width, (p.d - t.n0 + 31) & ~31);
  return t;
}

__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ void tma_reduce_add_2d(const CUtensorMap* map, uint32_t src, int x, int y) {
  asm volatile("cp.reduce.async.bulk.tensor.2d.global.shared::cta.add.tile.bulk_group [%0, {%2, %3}], [%1];"
               ::"l"(reinterpret_cast<uint64_t>(map)), "r"(src), "r"(x), "r"(y)
               : "memory");
}

// LSE, DLOGITS: tmap_a = X (64 x 128 boxes), tmap_b = W (64 x 128 boxes), tmap_out = D (DLOGITS).
// FEW: the maps of X and of D as rows of tokens have boxes of 64 x few_n / 2.
// DLOGITS, the target's element: w (p - 1) = w expm1(log p), with log p = -loss where the losses are given.  Without them log p is the
// difference of the logit and the rounded log-sum-exp, good to about 2^-23 of those: nothing of 1 - p is left of it where
// that is smaller.
// GRADS: tmap_a = D as rows of tokens (64 x 128 boxes), tmap_a2 = D read MN-major (64 x 64 boxes), tmap_b = W, tmap_b2 = X
// (both 64 x 64 boxes, MN-major), tmap_out = the fp32 sums of dX (32 x 16 boxes), tmap_out2 = dW (64 x 16 boxes), tmap_out3 =
// dW (32 x 32 boxes, 64-byte swizzle).
template <int KIND, bool FEW>
__global__ void __launch_bounds__(kThreads, 1)
    ce_kernel(const __grid_constant__ CUtensorMap tmap_a, const __grid_constant__ CUtensorMap tmap_b,
              const __grid_constant__ CUtensorMap tmap_a2, const __grid_constant__ CUtensorMap tmap_b2,
              const __grid_constant__ CUtensorMap tmap_out, const __grid_constant__ CUtensorMap tmap_out2,
              const __grid_constant__ CUtensorMap tmap_out3, const Params p) {
  constexpr int kStages = Stages<KIND, FEW>::kCount, kStageBytes = Stages<KIND, FEW>::kBytes;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t smem_base = (ptx::smem_u32(smem_raw) + 1023u) & ~1023u;
  uint8_t* smem_gen = smem_raw + (smem_base - ptx::smem_u32(smem_raw));
  const uint32_t bar_base = smem_base + kStagesBytes;
  auto full_bar = [&](int s) { return bar_base + 8u * s; };
  auto empty_bar = [&](int s) { return bar_base + 8u * (kStages + s); };
  auto tfull_bar = [&](int a) { return bar_base + 8u * (2 * kStages + a); };
  auto tempty_bar = [&](int a) { return bar_base + 8u * (2 * kStages + 2 + a); };
  constexpr int kSlot = 8 * (2 * kStages + 4);
  volatile uint32_t* tmem_slot_gen = reinterpret_cast<volatile uint32_t*>(smem_gen + kStagesBytes + kSlot);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(smem_gen + kStagesBytes + kSlot + 4);

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = ptx::cluster_ctarank();
  const int pair = int(blockIdx.x) >> 1, pairs = int(gridDim.x) >> 1;
  auto on_leader = [&](uint32_t bar) { return ptx::map_to_rank(bar, 0u); };

  if (threadIdx.x == 0) {
    for (int s = 0; s < kStages; ++s) {
      ptx::mbar_init(full_bar(s), 1);
      ptx::mbar_init(empty_bar(s), 1);
    }
    for (int a = 0; a < 2; ++a) {
      ptx::mbar_init(tfull_bar(a), 1);
      ptx::mbar_init(tempty_bar(a), 2 * kEpiWarps);   // the epilogue warps of both CTAs
    }
    *abort_flag = 0;
    ptx::fence_barrier_init();
    ptx::prefetch_tensormap(&tmap_a);
    ptx::prefetch_tensormap(&tmap_b);
    if (KIND == GRADS) {
      ptx::prefetch_tensormap(&tmap_a2);
      ptx::prefetch_tensormap(&tmap_b2);
      ptx::prefetch_tensormap(&tmap_out2);
      ptx::prefetch_tensormap(&tmap_out3);
    }
    if (KIND != LSE) ptx::prefetch_tensormap(&tmap_out);
  }
  if (warp == 1) {
    ptx::tmem_alloc_pair(bar_base + kSlot, kTmemCols);
    ptx::tmem_relinquish_alloc_permit_pair();
  }
  ptx::tcgen05_fence_before_sync();
  ptx::cluster_sync_all();   // the peer's barriers are initialised before anything is signalled there
  ptx::tcgen05_fence_after_sync();
  const uint32_t tmem_base = *tmem_slot_gen;
  // Every launch may start while the one before it is still running.  One that needs its results waits for its end here, with
  // everything set up; one that does not waits at its own end (see below).  Either way a launch lets the next one start
  // only once the launch before itself has ended: whatever runs beside a launch is its direct neighbour.
  if (p.wait_first) {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  }
  if (KIND == LSE && blockIdx.x == 0 && threadIdx.x == 0) *p.ticket = 0u;
  auto give_up = [&]() {
    *abort_flag = 1;
    atomicExch(p.status, kDevTimeout);
  };

  if (warp == 0) {
    // ------------------------------------------------------------------ TMA producer
    if (lane == 0) {
      int stage = 0;
      uint32_t phase = 0, armed = 0;
      bool ok = true;
      for (int u = pair; ok && u < p.units; u += pairs) {
        const Unit t = decode<KIND, FEW>(p, u);
        const int a_row0 = t.m0 + int(rank) * kBM;
        const int hw = t.bn >> 1, b_row0 = t.n0 + int(rank) * hw;       // this CTA's half of the B rows
        // one loop per operand layout, so that everything that does not change along K is fixed in it
        auto stages = [&](auto load) {
          for (int kb = t.kb0; kb < t.kb1; ++kb) {
            if (!ptx::mbar_wait(empty_bar(stage), phase ^ 1u, abort_flag)) { give_up(); ok = false; break; }
            const uint32_t a_dst = smem_base + stage * kStageBytes;
            armed |= 1u << stage;
            load(a_dst, a_dst + kABytes, on_leader(full_bar(stage)), kb * kBK);   // both CTAs' bytes are counted on the leader's barrier
            if (++stage == kStages) { stage = 0; phase ^= 1u; }
          }
        };
        auto arm = [&](uint32_t bytes) {
          if (rank == 0) ptx::mbar_arrive_expect_tx(full_bar(stage), 2 * bytes);
        };
        if (FEW && KIND != GRADS) {
          const int w_row0 = p.v0 + a_row0;
          stages([&](uint32_t a_dst, uint32_t b_dst, uint32_t bar, int k0) {
            arm(kABytes + hw * kBK * 2);
            ptx::tma_load_2d_pair(a_dst, &tmap_b, bar, k0, w_row0);
            ptx::tma_load_2d_pair(b_dst, &tmap_a, bar, k0, b_row0);
          });
        } else if (FEW && t.x) {
          stages([&](uint32_t a_dst, uint32_t b_dst, uint32_t bar, int k0) {
            arm(kABytes + hw * kBK * 2);
            ptx::tma_load_2d_pair(a_dst, &tmap_b, bar, a_row0, p.v0 + k0);
            ptx::tma_load_2d_pair(a_dst + kChunkBytes, &tmap_b, bar, a_row0 + 64, p.v0 + k0);
            ptx::tma_load_2d_pair(b_dst, &tmap_a, bar, k0, b_row0);
          });
        } else if (KIND != GRADS) {
          const int w_row0 = p.v0 + b_row0;
          stages([&](uint32_t a_dst, uint32_t b_dst, uint32_t bar, int k0) {
            arm(kABytes + kBBytes);
            ptx::tma_load_2d_pair(a_dst, &tmap_a, bar, k0, a_row0);
            ptx::tma_load_2d_pair(b_dst, &tmap_b, bar, k0, w_row0);
          });
        } else {
          const bool two = hw > 64;     // 64-column chunks of this CTA's half
          const uint32_t bytes = kABytes + (two ? 2 : 1) * kChunkBytes;
          if (t.x) {
            stages([&](uint32_t a_dst, uint32_t b_dst, uint32_t bar, int k0) {
              arm(bytes);
              ptx::tma_load_2d_pair(a_dst, &tmap_a, bar, k0, a_row0);
              ptx::tma_load_2d_pair(b_dst, &tmap_b, bar, b_row0, p.v0 + k0);
              if (two) ptx::tma_load_2d_pair(b_dst + kChunkBytes, &tmap_b, bar, b_row0 + 64, p.v0 + k0);
            });
          } else {
            stages([&](uint32_t a_dst, uint32_t b_dst, uint32_t bar, int k0) {
              arm(bytes);
              ptx::tma_load_2d_pair(a_dst, &tmap_a2, bar, a_row0, k0);
              ptx::tma_load_2d_pair(a_dst + kChunkBytes, &tmap_a2, bar, a_row0 + 64, k0);
              ptx::tma_load_2d_pair(b_dst, &tmap_b2, bar, b_row0, k0);
              if (two) ptx::tma_load_2d_pair(b_dst + kChunkBytes, &tmap_b2, bar, b_row0 + 64, k0);
            });
          }
        }
      }
      if (!ok) {
        // wait (bounded, one limit for all stages) for the copies still in flight before the CTA leaves
        const uint64_t t0 = ptx::globaltimer_ns();
        for (int s = 0; s < kStages; ++s) {
          if (!(armed & (1u << s))) continue;
          const uint32_t ph = (s < stage) ? phase : (phase ^ 1u);
          while (!ptx::mbar_try_wait(full_bar(s), ph) && ptx::globaltimer_ns() - t0 < ptx::kWaitLimitNs) {}
        }
      } else {
        // stay until the leader's tensor core has released every stage this CTA filled: its arrivals must not reach the
        // memory of a CTA that left
        for (int s = 0; s < kStages && ok; ++s) {
          if (!(armed & (1u << s))) continue;
          const uint32_t ph = (s < stage) ? phase : (phase ^ 1u);
          if (!ptx::mbar_wait(empty_bar(s), ph, abort_flag)) { give_up(); ok = false; }
        }
      }
      if (!p.wait_first) {   // the launch before this one has long ended as a rule
        asm volatile("griddepcontrol.wait;" ::: "memory");
        asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
      }
    }
  } else if (warp == 1) {
    // ------------------------------------------------------------------ UMMA issuer (the leader's)
    if (lane == 0 && rank == 0) {
      int stage = 0, it = 0;
      uint32_t phase = 0;
      bool ok = true;
      for (int u = pair; ok && u < p.units; u += pairs, ++it) {
        const Unit t = decode<KIND, FEW>(p, u);
        const int acc = it & 1;
        const uint32_t d_tmem = tmem_base + acc * kAccCols;
        if (!ptx::mbar_wait_cluster(tempty_bar(acc), ((it >> 1) & 1) ^ 1u, abort_flag)) { give_up(); ok = false; break; }
        ptx::tcgen05_fence_after_sync();
        auto products = [&](auto a_is_mn, auto b_is_mn) {
          constexpr bool a_mn = decltype(a_is_mn)::value, b_mn = decltype(b_is_mn)::value;
          constexpr uint32_t a_lbo = a_mn ? kChunkBytes : 16, a_step = (a_mn ? kUmmaK * 128 : kUmmaK * 2) >> 4;
          constexpr uint32_t b_lbo = b_mn ? kChunkBytes : 16, b_step = (b_mn ? kUmmaK * 128 : kUmmaK * 2) >> 4;
          const uint32_t idesc = ptx::make_idesc_bf16(kTile, t.bn, a_mn, b_mn);
          for (int kb = t.kb0; kb < t.kb1; ++kb) {
            if (!ptx::mbar_wait_cluster(full_bar(stage), phase, abort_flag)) { give_up(); ok = false; break; }
            ptx::tcgen05_fence_after_sync();
            const uint32_t a_addr = smem_base + stage * kStageBytes, b_addr = a_addr + kABytes;
            const uint64_t da = ptx::make_smem_desc(a_addr, a_lbo, 1024), db = ptx::make_smem_desc(b_addr, b_lbo, 1024);
#pragma unroll
            for (int k = 0; k < kBK / kUmmaK; ++k)
              ptx::umma_bf16_pair(d_tmem, da + uint64_t(k * a_step), db + uint64_t(k * b_step), idesc, kb > t.kb0 || k > 0);
            ptx::umma_commit_pair(empty_bar(stage), 3);
            if (++stage == kStages) { stage = 0; phase ^= 1u; }
          }
        };
        using Yes = std::true_type;
        using No = std::false_type;
        if (KIND != GRADS) products(No{}, No{});
        else if (!t.x) products(Yes{}, Yes{});
        else if (FEW) products(Yes{}, No{});
        else products(No{}, Yes{});
        if (ok) ptx::umma_commit_pair(tfull_bar(acc), 3);
      }
    }
  } else {
    // ------------------------------------------------------------------ epilogue
    const int quarter = warp & 3;                       // TMEM lanes [32 * quarter, + 32) are the ones this warp may read
    const int group = (warp - kEpiWarp0) >> 2;          // columns [64 * group, + 64) of the tile
    uint8_t* out_gen = smem_gen + kOutOffset + (warp - kEpiWarp0) * kBoxBytes;
    const uint32_t out_addr = smem_base + kOutOffset + (warp - kEpiWarp0) * kBoxBytes;
    float f = 0.f;
    if (KIND == GRADS) {
      const float dn = p.denom ? __ldcg(p.denom) : 1.f;
      f = dn > 0.f ? p.scale / dn : 0.f;
    }
    // 32 rows of 32 words (64 bf16 or 32 fp32 columns), a row per lane, to (x, y) of a map whose boxes are 16 rows of 128 bytes
    // (16-byte unit j of row l at j ^ (l & 7)).  Rows of 128 bytes leave a CTA in half the time that twice as many of 64 take.
    auto store_rows = [&](const uint32_t (&words)[32], const CUtensorMap* map, int x, int y, bool add) {
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        if (lane == 0) ptx::tma_store_wait_read<0>();   // the store that last used the box has read it
        __syncwarp();
        if ((lane >> 4) == r) {
#pragma unroll
          for (int j = 0; j < 8; ++j)
            *reinterpret_cast<uint4*>(out_gen + (lane & 15) * 128 + ((j ^ (lane & 7)) << 4)) =
                make_uint4(words[4 * j], words[4 * j + 1], words[4 * j + 2], words[4 * j + 3]);
        }
        ptx::fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) {
          if (add) tma_reduce_add_2d(map, out_addr, x, y + 16 * r);
          else ptx::tma_store_2d(map, out_addr, x, y + 16 * r);
          ptx::tma_store_commit();
        }
      }
    };
    // 32 rows of 16 words (32 bf16 columns), boxes of 32 rows of 64 bytes (unit j of row l at j ^ ((l >> 1) & 3))
    auto store_narrow = [&](const uint32_t (&words)[32], const CUtensorMap* map, int x, int y) {
      if (lane == 0) ptx::tma_store_wait_read<0>();
      __syncwarp();
#pragma unroll
      for (int j = 0; j < 4; ++j)
        *reinterpret_cast<uint4*>(out_gen + lane * 64 + ((j ^ ((lane >> 1) & 3)) << 4)) =
            make_uint4(words[4 * j], words[4 * j + 1], words[4 * j + 2], words[4 * j + 3]);
      ptx::fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) {
        ptx::tma_store_2d(map, out_addr, x, y);
        ptx::tma_store_commit();
      }
    };
    auto pack2 = [](uint32_t lo, uint32_t hi) {
      const __nv_bfloat162 h = __floats2bfloat162_rn(__uint_as_float(lo), __uint_as_float(hi));
      return *reinterpret_cast<const uint32_t*>(&h);
    };
    // The token whose row_add belongs to row `first_row` + lane of dW, or -1.  At most one does.  The keys of up to 64 tokens
    // stay in registers (read for every tile: backward of 64 x 2048 x 128256 311 -> 324 us); more are read again for every tile,
    // while its products are on their way (eight in registers: 256 x 2048 x 65536 266 us, 229 without; sixteen spill).
    constexpr int kKeys = FEW ? kFewTokens / 32 : 8;
    int key[KIND == GRADS ? kKeys : 1];
    auto read_keys = [&](int t0) {
#pragma unroll
      for (int i = 0; i < kKeys; ++i) key[KIND == GRADS ? i : 0] = t0 + 32 * i + lane < p.tokens ? __ldcg(p.row_key + t0 + 32 * i + lane) : -1;
    };
    if (FEW && KIND == GRADS && p.row_key) read_keys(0);
    auto find_row_add = [&](int first_row) {
      int mine = -1;
      for (int t0 = 0; t0 < p.tokens; t0 += 32 * kKeys) {
        if (!FEW) read_keys(t0);
#pragma unroll
        for (int i = 0; i < kKeys; ++i) {
          const int r = key[KIND == GRADS ? i : 0] - first_row;
          for (uint32_t hits = __ballot_sync(0xFFFFFFFFu, r >= 0 && r < 32); hits; hits &= hits - 1) {
            const int src = __ffs(hits) - 1;
            if (__shfl_sync(0xFFFFFFFFu, r, src) == lane) mine = t0 + 32 * i + src;
          }
        }
      }
      return mine;
    };
    // FEW: this warp has the 16 tokens from few0 on (there may be none); a lane's own token's target, and in the staging what
    // the tokens need (DLOGITS)
    constexpr int kFew = 16;
    const int few0 = kFew * group;
    int few_y = -1;
    uint32_t few_trained = 0u;               // which of the tokens are trained on
    float few_m[FEW && KIND == LSE ? kFew : 1], few_s[FEW && KIND == LSE ? kFew : 1];
    float* const few_lse2 = reinterpret_cast<float*>(out_gen);
    float* const few_w = few_lse2 + 32;
    float* const few_loss = few_lse2 + 64;
    if (FEW) {
      const int tt = few0 + lane;
      if (KIND != GRADS && lane < kFew && tt < p.tokens) {
        const int64_t y = __ldcg(p.targets + tt);
        few_y = y >= 0 && y < p.vocab ? int(y) : -1;
      }
      few_trained = __ballot_sync(0xFFFFFFFFu, few_y >= 0);
      if (KIND == DLOGITS) {
        few_lse2[lane] = few_y >= 0 ? __ldcg(p.lse + tt) * kLog2e : 0.f;
        few_w[lane] = few_y >= 0 ? (p.weight ? __ldcg(p.weight + tt) : 1.f) : 0.f;
        few_loss[lane] = few_y >= 0 && p.loss ? __ldcg(p.loss + tt) : 0.f;
        __syncwarp();
      }
      if (KIND == LSE) {
#pragma unroll
        for (int j = 0; j < kFew; ++j) {
          few_m[FEW && KIND == LSE ? j : 0] = kLowest;
          few_s[FEW && KIND == LSE ? j : 0] = 0.f;
        }
      }
    }
    // What a lane's row needs besides the accumulator, asked for one tile ahead (from L2 it takes longer than a small tile)
    struct RowNeeds {
      int2 y;          // the target, as it is in memory
      float lse, weight, loss;
    };
    // e: the target's element of D, from log p = -loss or (without losses) from the logit's exponent x less the log-sum-exp in base 2
    auto target_element = [&](float w, float loss, float x) {
      const float e = w * expm1f(p.loss ? -loss : x * kLn2);
      return !p.loss && p.vocab == 1 && e == e ? 0.f : e;   // one word is certain: the difference would be its rounding only
    };
    auto needs_of = [&](int m0) {
      RowNeeds n{make_int2(-1, -1), 0.f, 1.f, 0.f};
      const int r = m0 + int(rank) * kBM + quarter * 32 + lane;
      if (!FEW && KIND != GRADS && r < p.tokens) {
        n.y = __ldcg(reinterpret_cast<const int2*>(p.targets) + r);
        if (KIND == DLOGITS) {
          n.lse = __ldcg(p.lse + r);
          if (p.weight) n.weight = __ldcg(p.weight + r);
          if (p.loss) n.loss = __ldcg(p.loss + r);
        }
      }
      return n;
    };
    int it = 0;
    Unit ahead = decode<KIND, FEW>(p, min(pair, p.units - 1));
    RowNeeds needs = needs_of(ahead.m0);
    for (int u = pair; u < p.units; u += pairs, ++it) {
      const Unit t = ahead;
      ahead = decode<KIND, FEW>(p, min(u + pairs, p.units - 1));
      const int acc = it & 1;
      const int row0 = t.m0 + int(rank) * kBM + quarter * 32, row = row0 + lane;
      const int col0 = t.n0 + group * kGroupCols;               // of the output; LSE, DLOGITS: of the piece
      // a target outside [0, vocab): not trained on
      const int y = needs.y.y == 0 && uint32_t(needs.y.x) < uint32_t(p.vocab) ? needs.y.x : -1;
      const float lse2 = needs.lse * kLog2e, weight = y >= 0 ? needs.weight : 0.f, loss = needs.loss;
      needs = needs_of(ahead.m0);
      const int add_token = (KIND == GRADS && !t.x && p.row_key) ? find_row_add(p.v0 + row0) : -1;
      const bool full_ok = ptx::mbar_wait_cluster(tfull_bar(acc), (it >> 1) & 1, abort_flag);
      if (!__all_sync(0xFFFFFFFFu, full_ok)) { give_up(); break; }
      ptx::tcgen05_fence_after_sync();
      const uint32_t taddr = tmem_base + (uint32_t(quarter * 32) << 16) + acc * kAccCols + group * kGroupCols;
      auto release_accumulator = [&]() {
        ptx::tcgen05_fence_before_sync();
        __syncwarp();
        if (lane == 0) ptx::mbar_arrive_remote(on_leader(tempty_bar(acc)));
      };
      if (FEW && (KIND != GRADS || t.x)) {
        uint32_t v[kFew];
        const uint32_t few_addr = tmem_base + (uint32_t(quarter * 32) << 16) + acc * kAccCols + few0;
        if (few0 < t.bn) {
          __syncwarp();
          ptx::tmem_ld_x16(few_addr, v);
          ptx::tmem_ld_wait();
          const bool word = KIND != GRADS && p.v0 + row < p.vocab;   // this lane's row is a word of the vocabulary
          // the targets among this warp's words: of tokens `hits`, each a word `r` of it
          const int r = few_y < 0 ? -1 : few_y - (p.v0 + row0);
          const uint32_t hits = KIND != GRADS ? __ballot_sync(0xFFFFFFFFu, r >= 0 && r < 32) : 0u;
          if (KIND == LSE) {
            uint32_t mine = 0u;                // tokens whose target is this lane's word
            for (uint32_t h = hits; h; h &= h - 1) {
              const int j = __ffs(h) - 1;
              if (__shfl_sync(0xFFFFFFFFu, r, j) == lane) mine |= 1u << j;
            }
            if (word) {
#pragma unroll
              for (int j = 0; j < kFew; ++j) {
                const int k = FEW && KIND == LSE ? j : 0;
                const float x = (mine >> j) & 1u ? -INFINITY : __uint_as_float(v[j]) * p.c, top = fmaxf(few_m[k], x);
                few_s[k] = few_s[k] * exp2_fast(few_m[k] - top) + exp2_fast(x - top);
                few_m[k] = top;
              }
            }
          } else if (KIND == DLOGITS) {
#pragma unroll
            for (int j = 0; j < kFew; ++j) {
              const float e = few_w[j] * exp2_fast(fmaf(__uint_as_float(v[j]), p.c, -few_lse2[j]));
              if (few0 + j < p.tokens) p.D[int64_t(few0 + j) * p.ld_d + row] = __float2bfloat16_rn(word && (few_trained >> j & 1u) ? e : 0.f);
            }
          } else if (row < p.d) {
            float* o = p.acc + (int64_t(t.split) * p.acc_rows + few0) * p.d + row;
#pragma unroll
            for (int j = 0; j < kFew; ++j)
              if (few0 + j < p.tokens) {     // one addition per element and launch: the order is that of the pieces
                if (p.first_piece) o[int64_t(j) * p.d] = __uint_as_float(v[j]);
                else atomicAdd(o + int64_t(j) * p.d, __uint_as_float(v[j]));
              }
          }
          if (KIND == DLOGITS) {
            for (uint32_t h = hits; h; h &= h - 1) {
              const int j = __ffs(h) - 1, owner = __shfl_sync(0xFFFFFFFFu, r, j), tt = few0 + j;
              const float x = __uint_as_float(ptx::tmem_ld_x1(few_addr + j));
              if (lane == owner) {
                const float e = target_element(few_w[j], few_loss[j], fmaf(x, p.c, -few_lse2[j]));
                const __nv_bfloat16 b = __float2bfloat16_rn(e);
                p.D[int64_t(tt) * p.ld_d + row] = b;
                p.corr[tt] = e - __bfloat162float(b);
              }
              __syncwarp();
            }
          }
        }
        release_accumulator();
        continue;
      }
      // Columns [32 c, + 32) of the row out of tensor memory; `last`: the accumulator is free for the tile after next.
      auto drain = [&](int c, uint32_t (&v)[32], bool last) {
        __syncwarp();
        ptx::tmem_ld_x32(taddr + 32 * c, v);
        ptx::tmem_ld_wait();
        if (last) release_accumulator();
      };
      if (KIND != GRADS) {
        const int valid = min(kGroupCols, p.vocab - (p.v0 + col0));   // columns of this warp that exist (may be negative)
        const int tc = y >= 0 ? y - (p.v0 + col0) : -1;               // the target's column here, if in [0, 64)
        const bool target_here = __any_sync(0xFFFFFFFFu, tc >= 0 && tc < kGroupCols);
        if (row0 >= p.tokens || (KIND == LSE && valid <= 0)) {
          release_accumulator();
          continue;
        }
        if (KIND == LSE) {
          uint32_t w[2][32];
          __syncwarp();
          ptx::tmem_ld_x32(taddr, w[0]);
          if (valid > 32) ptx::tmem_ld_x32(taddr + 32, w[1]);
          ptx::tmem_ld_wait();
          release_accumulator();
          // exponents are w c - max(w c); where c is negative, or columns do not exist or are a target, the products are made first
          float c1 = p.c;
          if (c1 < 0.f || valid < kGroupCols || target_here) {
#pragma unroll
            for (int c = 0; c < 2; ++c)
#pragma unroll
              for (int i = 0; i < 32; ++i)
                w[c][i] = __float_as_uint(32 * c + i < valid && 32 * c + i != tc ? __uint_as_float(w[c][i]) * c1 : -INFINITY);
            c1 = 1.f;
          }
          float top[4];
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            top[c] = __uint_as_float(w[c >> 1][16 * (c & 1)]);
#pragma unroll
            for (int i = 1; i < 16; ++i) top[c] = fmaxf(top[c], __uint_as_float(w[c >> 1][16 * (c & 1) + i]));
          }
          const float m = fmaxf(fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3])) * c1, kLowest);
          float2 sum[4];
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            sum[c] = q8::both(0.f);
#pragma unroll
            for (int i = 16 * (c & 1); i < 16 * (c & 1) + 16; i += 2) {
              const float2 x = q8::fma2(make_float2(__uint_as_float(w[c >> 1][i]), __uint_as_float(w[c >> 1][i + 1])), q8::both(c1), q8::both(-m));
              sum[c] = q8::add2(sum[c], make_float2(exp2_fast(x.x), exp2_fast(x.y)));
            }
          }
          sum[0] = q8::add2(q8::add2(sum[0], sum[1]), q8::add2(sum[2], sum[3]));
          if (row < p.tokens) p.part[int64_t(col0 / kGroupCols) * p.tokens + row] = make_float2(m, sum[0].x + sum[0].y);
        } else {
          uint32_t pk[32];
#pragma unroll
          for (int c = 0; c < 2; ++c) {            // (32 columns at a time: 96 registers do not hold 64 and the packed ones)
            uint32_t v[32];
            drain(c, v, c == 1);
            uint32_t target_bits = 0u;             // the target's element, taken on its own
            if (target_here) {
              float l = 0.f;
#pragma unroll
              for (int i = 0; i < 32; ++i) l = tc == 32 * c + i ? __uint_as_float(v[i]) : l;
              if (tc >= 32 * c && tc < 32 * c + 32) {
                const float e = target_element(weight, loss, fmaf(l, p.c, -lse2));
                target_bits = pack2(__float_as_uint(e), 0u);
                p.corr[row] = e - __uint_as_float(target_bits << 16);
              }
            }
#pragma unroll
            for (int i = 0; i < 16; ++i) {
              const float2 x = q8::fma2(make_float2(__uint_as_float(v[2 * i]), __uint_as_float(v[2 * i + 1])), q8::both(p.c), q8::both(-lse2));
              const float2 e = q8::mul2(make_float2(exp2_fast(x.x), exp2_fast(x.y)), q8::both(weight));
              pk[16 * c + i] = pack2(__float_as_uint(e.x), __float_as_uint(e.y));
            }
            if (target_here) {
#pragma unroll
              for (int i = 0; i < 16; ++i) {
                uint32_t& q = pk[16 * c + i];
                if (tc == 32 * c + 2 * i) q = (q & 0xFFFF0000u) | target_bits;
                if (tc == 32 * c + 2 * i + 1) q = (q & 0xFFFFu) | (target_bits << 16);
              }
            }
          }
          // columns past the vocabulary and rows that are not trained on are zero whatever the logit is
          if (valid < kGroupCols) {
#pragma unroll
            for (int i = 0; i < 32; ++i) pk[i] = 2 * i + 1 < valid ? pk[i] : (2 * i < valid ? pk[i] & 0xFFFFu : 0u);
          }
          if (y < 0) {
#pragma unroll
            for (int i = 0; i < 32; ++i) pk[i] = 0u;
          }
          store_rows(pk, &tmap_out, col0, row0, false);
        }
        continue;
      }
      const int cols = min(min(kGroupCols, t.bn - group * kGroupCols), p.d - col0);   // columns that exist (may be negative)
      const bool rows_exist = t.x ? row0 < p.tokens : p.v0 + row0 < p.vocab;
      if (cols <= 0 || !rows_exist) {
        release_accumulator();
        continue;
      }
      uint32_t pk[32];
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        if (32 * c >= cols) break;
        uint32_t v[32];
        drain(c, v, c == 1 || cols <= 32);
        if (t.x) {
          store_rows(v, &tmap_out, col0 + 32 * c, t.split * p.acc_rows + row0, !p.first_piece);
          continue;
        }
        if (add_token >= 0) {
          const float4* x = reinterpret_cast<const float4*>(p.row_add + int64_t(add_token) * p.d + col0 + 32 * c);
#pragma unroll
          for (int j = 0; j < 8; ++j)
            if (32 * c + 4 * j < cols) {
              const float4 q = __ldcg(x + j);
              v[4 * j] = __float_as_uint(__uint_as_float(v[4 * j]) + q.x);
              v[4 * j + 1] = __float_as_uint(__uint_as_float(v[4 * j + 1]) + q.y);
              v[4 * j + 2] = __float_as_uint(__uint_as_float(v[4 * j + 2]) + q.z);
              v[4 * j + 3] = __float_as_uint(__uint_as_float(v[4 * j + 3]) + q.w);
            }
        }
        __syncwarp();
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const float2 e = q8::mul2(make_float2(__uint_as_float(v[2 * i]), __uint_as_float(v[2 * i + 1])), q8::both(f));
          pk[16 * c + i] = pack2(__float_as_uint(e.x), __float_as_uint(e.y));
        }
      }
      if (t.x) continue;
      // columns that end after 32 inside d belong to two tiles: the store must not reach into the next one
      if (cols > 32) store_rows(pk, &tmap_out2, col0, p.v0 + row0, false);
      else store_narrow(pk, &tmap_out3, col0, p.v0 + row0);
    }
    if (FEW && KIND == LSE && few0 < p.few_n) {
      // the 32 lanes' pairs of every token into one: the token's own lane keeps it
      float m = 0.f, s = 0.f;
#pragma unroll
      for (int j = 0; j < kFew; ++j) {
        const int k = FEW && KIND == LSE ? j : 0;
        float top = few_m[k];
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, o));
        float sum = few_s[k] * exp2_fast(few_m[k] - top);
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, o);
        if (lane == j) {
          m = top;
          s = sum;
        }
      }
      if (lane < kFew && few0 + lane < p.tokens) p.part[int64_t((2 * pair + int(rank)) * 4 + quarter) * p.tokens + few0 + lane] = make_float2(m, s);
    }
    if (KIND != LSE && lane == 0) ptx::tma_store_wait_read<0>();   // shared memory must outlive the stores' reads
  }

  ptx::tcgen05_fence_before_sync();
  ptx::cluster_sync_all();   // neither CTA frees tensor memory or leaves while the other may still signal or read it
  if (warp == 1) {
    __syncwarp();
    ptx::tcgen05_fence_after_sync();
    ptx::tmem_dealloc_pair(tmem_base, kTmemCols);
  }
}

}  // namespace ce
}  // namespace acx
