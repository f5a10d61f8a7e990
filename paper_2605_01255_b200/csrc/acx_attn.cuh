// Softmax attention over packed documents: what its kernels share.
//
// For query i and key j of one document, with 2-based exponents throughout,
//     x_ij = log2(e) (cap(scale q_i k_j) - slope |i - j|),   cap(s) = c tanh(s / c) or s,
//     p_ij = 2^(x_ij - lse_i),   o_i = sum_j p_ij v_j        over the keys that i sees.
// Which those are is an interval for every query: from its document's start to its end (not causal), or to the larger of its own
// position and the prefix's end.  Tiles never reach over a document's border: the tiles of queries and of keys start
// at the document's own start (a bulk tensor copy may start at any token), so a tile is masked at most along the diagonal, at the
// prefix's end and behind the document's last token, and nothing of a neighbouring document or of padding is multiplied: rows
// behind the last token are overwritten with zeros in shared memory before a product sums over them.
//
// The plan, one kernel per batch, lists the tiles of every document with the longest first; work item u of a launch is tile
// u / heads for head u % heads, so that the heads that share a key head run beside one another.
#pragma once
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <type_traits>

#include "acx_internal.h"
#include "acx_q8.cuh"
#include "acx_umma.cuh"

namespace acx {
namespace attn {

constexpr int kRows = 128;          // rows of one tile: lanes of tensor memory
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

struct Item {
  int row0;        // first token of the tile
  int start, end;  // the document's tokens
  int prefix;      // end of the part that all of the document's tokens see (start: none)
};
// The plan in device memory: this, then the lists.
struct PlanHeader {
  int wide;          // items of 256 queries (forward)
  int tiles;         // items of 128 tokens (backward, both lists)
  int head_end;      // tokens [0, head_end) and [tail_begin, tokens) belong to no document
  int tail_begin;
  int tokens, docs, causal, unused;   // what it was made for
};
static_assert(sizeof(PlanHeader) == 32, "two loads");
constexpr size_t kPlanListOffset = 256;
struct PlanLayout {
  int64_t wide_cap, tile_cap;
  size_t wide, queries, keys, cum, bytes;   // byte offsets of the lists; cum: the documents' running tile counts, for each list its own
};
__host__ __device__ inline PlanLayout plan_layout(int64_t tokens, int64_t docs) {
  const int64_t d = docs < tokens ? docs : tokens;   // documents that hold a token
  PlanLayout p;
  p.wide_cap = tokens / 256 + d + 1;
  p.tile_cap = tokens / 128 + d + 1;
  p.wide = kPlanListOffset;
  p.queries = p.wide + size_t(p.wide_cap) * sizeof(Item);
  p.keys = p.queries + size_t(p.tile_cap) * sizeof(Item);
  p.cum = p.keys + size_t(p.tile_cap) * sizeof(Item);
  p.bytes = p.cum + size_t(docs + 1) * 12;
  return p;
}

struct Params {
  int tokens, docs, heads, kv_heads, group;
  int d;                     // columns of a head
  int causal;
  const PlanHeader* plan;
  const Item* items;         // the list that this launch works through
  const float* slopes;       // [heads], BIAS only
  float scale;
  float c;                   // scale log2(e): x = c s without a cap
  float cap_in;              // 2^7 scale / cap: the tanh's argument per unit of s
  float cap_out;             // 2^-7 cap log2(e)
  float* lse;                // [heads][tokens], natural logarithm
  int* status;
  __nv_bfloat16* O;
  int64_t ldo;
  // backward
  float* delta;              // [heads][tokens], made exact by the launch for the queries
  __nv_bfloat16 *dQ, *dK, *dV;
  int64_t lddq, lddk, lddv;
  float *dk_part, *dv_part;  // [part][tokens][kv_heads][d], or null: one part, written to dK and dV
  int parts, heads_per_part;
};

__device__ __forceinline__ float2 unpack2(uint32_t v) { return make_float2(__uint_as_float(v << 16), __uint_as_float(v & 0xFFFF0000u)); }
__device__ __forceinline__ float2 neg2(float2 v) { return make_float2(-v.x, -v.y); }
__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// Maxima that keep a NaN.
__device__ __forceinline__ float max_nan(float a, float b) {
  float y;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(a), "f"(b));
  return y;
}
__device__ __forceinline__ float max_nan(float a, float b, float c) {
  float y;
  asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(y) : "f"(a), "f"(b), "f"(c));
  return y;
}
__device__ __forceinline__ float min_nan(float a, float b) {
  float y;
  asm("min.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(a), "f"(b));
  return y;
}
__device__ __forceinline__ float rcp_fast(float x) {
  float y;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// 2^7 tanh(2^-7 u), and tanh' in units of 2^-14: with t for the former the latter is 2^14 - t^2.  With r = 1 / (1 + e^2|v|), v = 2^-7 u, they are
// 1 - 2 r and 4 r (1 - r): the latter keeps its digits where the tanh saturates (1 - tanh^2 loses them: 6 % at v = 8).  The former keeps
// about 2^-23 absolutely, which is too little near zero once a large cap multiplies it; up to 0.75 an odd polynomial, fitted to
// tanh(v) / v (relative error 1.2e-8 before rounding), takes over.  SMALL: all arguments are below that.
constexpr float kTanhUnit = 128.f, kSlopeUnit = kTanhUnit * kTanhUnit;
template <bool SMALL>
__device__ __forceinline__ float tanh_of(float u, float* slope) {
  constexpr float c1 = 1.f / kSlopeUnit, c2 = c1 * c1, c3 = c2 * c1, c4 = c3 * c1, c5 = c4 * c1, c6 = c5 * c1;
  const float q = u * u;
  float t = fmaf(q, fmaf(q, fmaf(q, fmaf(q, fmaf(q, 1.7277066e-3f * c6, -7.6394570e-3f * c5), 2.1438753e-2f * c4), -5.3887937e-2f * c3), 0.13332610f * c2),
                 -0.33333308f * c1);
  t = fmaf(u * q, t, u);
  if (SMALL) {
    if (slope) *slope = fmaf(-t, t, kSlopeUnit);
    return t;
  }
  const float r = rcp_fast(1.f + exp2_fast(fabsf(u) * (2.f * kLog2e / kTanhUnit)));
  if (slope) {
    const float f = 4.f * kSlopeUnit * r;
    *slope = fmaf(-f, r, f);
  }
  return fabsf(u) < 0.75f * kTanhUnit ? t : copysignf(fmaf(-2.f * kTanhUnit, r, kTanhUnit), u);
}

// x of a raw score s; `far` = query position - key position.  For CAP, *slope = d x / d s in units of 2^-14 c.
template <bool CAP, bool BIAS, bool SMALL>
__device__ __forceinline__ float exponent(const Params& p, float s, float far, float slope2, float* slope = nullptr) {
  float x;
  if (CAP) {
    x = tanh_of<SMALL>(s * p.cap_in, slope) * p.cap_out;
  } else {
    x = s * p.c;
  }
  if (BIAS) x = fmaf(-slope2, fabsf(far), x);
  return x;
}
// Whether the tanh's polynomial alone does for the scores of a warp's rows inside the document (the slopes that the two forms give may
// differ in their last bit, and other documents decide nothing here).
template <int N>
__device__ __forceinline__ bool small_scores(const Params& p, const uint32_t (&s)[N], bool live) {
  float top = 0.f;
#pragma unroll
  for (int i = 0; i < N; ++i) top = fmaxf(top, fabsf(__uint_as_float(s[i])));
  return __all_sync(0xFFFFFFFFu, !live || top * p.cap_in < 0.75f * kTanhUnit);
}

// A wait of a whole warp, which it leaves together: what follows (tensor memory loads and stores) has to be executed by converged
// warps, and lanes that find a barrier complete at different polls are not.
__device__ __forceinline__ bool warp_wait(uint32_t bar, uint32_t parity, volatile int* abort_flag) {
  return __all_sync(0xFFFFFFFFu, ptx::mbar_wait(bar, parity, abort_flag));
}

// Waits for the tensor memory loads issued so far and hands their registers over behind the wait: as far as the compiler can see
// an inline load has delivered at once, and what uses its registers need not stay behind a wait that does not name them.
__device__ __forceinline__ void hand_over(uint32_t (&v)[32]) {
  asm volatile("" : "+r"(v[0]), "+r"(v[1]), "+r"(v[2]), "+r"(v[3]), "+r"(v[4]), "+r"(v[5]), "+r"(v[6]), "+r"(v[7]), "+r"(v[8]), "+r"(v[9]),
               "+r"(v[10]), "+r"(v[11]), "+r"(v[12]), "+r"(v[13]), "+r"(v[14]), "+r"(v[15]), "+r"(v[16]), "+r"(v[17]), "+r"(v[18]), "+r"(v[19]),
               "+r"(v[20]), "+r"(v[21]), "+r"(v[22]), "+r"(v[23]), "+r"(v[24]), "+r"(v[25]), "+r"(v[26]), "+r"(v[27]), "+r"(v[28]), "+r"(v[29]),
               "+r"(v[30]), "+r"(v[31])::"memory");
}
__device__ __forceinline__ void hand_over(uint32_t (&v)[16]) {
  asm volatile("" : "+r"(v[0]), "+r"(v[1]), "+r"(v[2]), "+r"(v[3]), "+r"(v[4]), "+r"(v[5]), "+r"(v[6]), "+r"(v[7]), "+r"(v[8]), "+r"(v[9]),
               "+r"(v[10]), "+r"(v[11]), "+r"(v[12]), "+r"(v[13]), "+r"(v[14]), "+r"(v[15])::"memory");
}
template <typename... V>
__device__ __forceinline__ void tmem_loaded(V&... v) {
  ptx::tmem_ld_wait();
  (hand_over(v), ...);
}

// The unit of work that this block takes in round `it`: the longest come first, and rounds go through the blocks there and back
// again, so that no block gets the longer ones of every round (the keys' launch of 8192 x 24 x 8 x 128: a block's tiles at most 432 of 337
// on average without, 354 with it).
__device__ __forceinline__ int unit_of(int it) {
  const int g = int(gridDim.x), b = int(blockIdx.x);
  return it * g + ((it & 1) ? g - 1 - b : b);
}

__device__ __forceinline__ Item fetch_item(const Item* items, int k) {
  const int4 v = __ldcg(reinterpret_cast<const int4*>(items) + k);
  return Item{v.x, v.y, v.z, v.w};
}
// The same by a whole warp, as values that are known to be the same in all lanes.
__device__ __forceinline__ Item fetch_item_warp(const Item* items, int k) {
  const Item t = fetch_item(items, k);
  return Item{__shfl_sync(0xFFFFFFFFu, t.row0, 0), __shfl_sync(0xFFFFFFFFu, t.start, 0), __shfl_sync(0xFFFFFFFFu, t.end, 0),
              __shfl_sync(0xFFFFFFFFu, t.prefix, 0)};
}

__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
  const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}

// COLS columns (16 or 32) of a row from registers, times f, as bf16; `left` columns (a multiple of 8) are inside the head.  Stores
// of 32 bytes where the row's address allows them.
template <int COLS>
__device__ __forceinline__ void store_bf16(__nv_bfloat16* at, const uint32_t (&v)[COLS], float f, int left) {
  uint32_t w[COLS / 2];
#pragma unroll
  for (int i = 0; i < COLS / 2; ++i) w[i] = pack2(__uint_as_float(v[2 * i]) * f, __uint_as_float(v[2 * i + 1]) * f);
  if (left >= COLS && (reinterpret_cast<uintptr_t>(at) & 31) == 0) {
#pragma unroll
    for (int i = 0; i < COLS / 16; ++i)
      asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(at + 16 * i), "r"(w[8 * i]), "r"(w[8 * i + 1]), "r"(w[8 * i + 2]),
                   "r"(w[8 * i + 3]), "r"(w[8 * i + 4]), "r"(w[8 * i + 5]), "r"(w[8 * i + 6]), "r"(w[8 * i + 7])
                   : "memory");
    return;
  }
#pragma unroll
  for (int i = 0; i < COLS / 8; ++i)
    if (8 * i < left) *reinterpret_cast<uint4*>(at + 8 * i) = make_uint4(w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]);
}
__device__ __forceinline__ void store_f32(float* at, const uint32_t (&v)[32], float f, int left) {
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (8 * i < left) {
      float2 q[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) q[k] = make_float2(__uint_as_float(v[8 * i + 2 * k]) * f, __uint_as_float(v[8 * i + 2 * k + 1]) * f);
      q8::store8(at + 8 * i, q);
    }
}

// Whether the plan is one for this descriptor: any other (never written, of another batch's sizes) would name tokens that are not
// there.  If not, nothing is done, and the device's status word says so.
__device__ __forceinline__ bool plan_fits(const Params& p) {
  const int4 made = __ldcg(reinterpret_cast<const int4*>(p.plan) + 1);
  const bool fits = made.x == p.tokens && made.y == p.docs && made.z == p.causal;
  // (a wait that ran out, here or in another kernel, weighs more: its word stays)
  if (!fits && blockIdx.x == 0 && threadIdx.x == 0) atomicCAS(p.status, kDevOk, kDevBadInput);
  return fits;
}

// Rows that belong to no document: zeros (all threads of the grid; row r of `heads` heads of d columns, stride ld).
__device__ __forceinline__ void zero_rows_outside(const Params& p, __nv_bfloat16* out, int64_t ld, int heads, float* row_value, float value) {
  const int head_end = p.plan->head_end, tail = p.plan->tail_begin;
  const int64_t outside = int64_t(head_end) + (p.tokens - tail);
  const int per_row = heads * (p.d / 8);
  for (int64_t k = int64_t(blockIdx.x) * blockDim.x + threadIdx.x; k < outside * per_row; k += int64_t(gridDim.x) * blockDim.x) {
    const int64_t r = k / per_row;
    const int64_t row = r < head_end ? r : tail + (r - head_end);
    *reinterpret_cast<uint4*>(out + row * ld + (k - r * per_row) * 8) = make_uint4(0u, 0u, 0u, 0u);
  }
  if (!row_value) return;
  for (int64_t k = int64_t(blockIdx.x) * blockDim.x + threadIdx.x; k < outside * heads; k += int64_t(gridDim.x) * blockDim.x) {
    const int64_t h = k / outside, r = k - h * outside;
    row_value[h * p.tokens + (r < head_end ? r : tail + (r - head_end))] = value;
  }
}

// A tile of 128 rows in shared memory: chunks of 64 columns, rows of 128 bytes with the 128-byte swizzle.
template <int HD>
struct Tile {
  static constexpr int kChunks = HD / 64, kChunkBytes = kRows * 128, kBytes = kChunks * kChunkBytes;
  // One thread: the rows from `row` on of one head.
  static __device__ __forceinline__ void load(uint32_t dst, const CUtensorMap* map, uint32_t bar, int head, int row) {
#pragma unroll
    for (int c = 0; c < kChunks; ++c) ptx::tma_load_3d(dst + c * kChunkBytes, map, bar, 64 * c, head, row);
  }
  // A whole warp: zeros into rows [first, last), visible to the tensor core.
  static __device__ __forceinline__ void zero_rows(uint8_t* tile, int first, int last) {
    const int n = (last - first) * 8;   // 16-byte units; the swizzle stays within a row
    for (int c = 0; c < kChunks; ++c)
      for (int i = threadIdx.x & 31; i < n; i += 32)
        *reinterpret_cast<uint4*>(tile + c * kChunkBytes + first * 128 + i * 16) = make_uint4(0u, 0u, 0u, 0u);
    ptx::fence_proxy_async_smem();
    __syncwarp();
  }
};

// Products of 128-row tiles; a whole warp.  Unrolled without regard to where the operands live, the descriptors of all steps of all
// products of a kernel are live at once, more than there are uniform registers, and products were seen to run with another
// step's operand: each block of four steps takes its own from one base instead.
//
// D (128 x 128) = A B^T over the head's columns, both tiles K-major.
template <int HD>
__device__ __forceinline__ void scores_mma(uint32_t tmem_d, uint32_t a, uint32_t b, int d16) {
  const uint32_t idesc = ptx::make_idesc_bf16(kRows, kRows, false, false);
  const uint64_t da = ptx::make_smem_desc(a, 16, 1024), db = ptx::make_smem_desc(b, 16, 1024);
  const uint32_t hi = uint32_t(da >> 32);
#pragma unroll
  for (int c = 0; c < HD / 64; ++c) {
    const uint32_t al = uint32_t(da) + c * (Tile<HD>::kChunkBytes >> 4), bl = uint32_t(db) + c * (Tile<HD>::kChunkBytes >> 4);
    const int steps = d16 - 4 * c;
    if (steps >= 4) {
      ptx::umma_steps<4, 2>(tmem_d, al, bl, hi, idesc, c > 0);
    } else {
#pragma unroll 1
      for (int k = 0; k < steps; ++k) ptx::umma_steps<1, 0>(tmem_d, al + 2 * k, bl + 2 * k, hi, idesc, c > 0 || k > 0);
    }
  }
}
// D (128 x 16 d16) (+)= A B with A (128 x 16 steps, bf16) in tensor memory and B the first 16 * steps rows of a tile.  Every 32
// columns of A start 16 + GAP columns of tensor memory apart, 16 in use.
template <int HD, int GAP>
__device__ __forceinline__ void rows_mma(uint32_t tmem_d, uint32_t tmem_a, uint32_t b, int steps, int d16, bool add) {
  const uint32_t idesc = ptx::make_idesc_bf16(kRows, 16 * d16, false, true);
  const uint64_t db = ptx::make_smem_desc(b, Tile<HD>::kChunkBytes, 1024);
  const uint32_t lo = uint32_t(db), hi = uint32_t(db >> 32);
#pragma unroll
  for (int c = 0; c < 2; ++c) {
    const uint32_t at = tmem_a + c * (32 + 2 * GAP), bl = lo + c * 512;
    if (steps >= 4 * c + 4) {
      ptx::umma_steps_tmem_a<4, 8 + GAP>(tmem_d, at, bl, hi, idesc, add || c > 0);
    } else {
#pragma unroll 1
      for (int k = 0; k < steps - 4 * c; ++k)
        ptx::umma_steps_tmem_a<1, 0>(tmem_d, at + 8 * k + (k >= 2 ? GAP : 0), bl + 128 * k, hi, idesc, add || c > 0 || k > 0);
    }
  }
}

// The same with A in shared memory: two K-major chunks of 64 columns.
template <int HD>
__device__ __forceinline__ void smem_rows_mma(uint32_t tmem_d, uint32_t a, uint32_t b, int steps, int d16, bool add) {
  const uint32_t idesc = ptx::make_idesc_bf16(kRows, 16 * d16, false, true);
  const uint64_t da = ptx::make_smem_desc(a, 16, 1024), db = ptx::make_smem_desc(b, Tile<HD>::kChunkBytes, 1024);
#pragma unroll
  for (int c = 0; c < 2; ++c) {
    const uint32_t al = uint32_t(da) + c * (kRows * 128 >> 4), bl = uint32_t(db) + c * 512;
    if (steps >= 4 * c + 4) {
      ptx::umma_steps<4, 128>(tmem_d, al, bl, uint32_t(da >> 32), idesc, add || c > 0);
    } else {
#pragma unroll 1
      for (int k = 0; k < steps - 4 * c; ++k) ptx::umma_steps<1, 0>(tmem_d, al + 2 * k, bl + 128 * k, uint32_t(da >> 32), idesc, add || c > 0 || k > 0);
    }
  }
}

Params common_params(const AttnProblem& q, const void* plan, const float* slopes, float* lse, int* status);

}  // namespace attn
}  // namespace acx
