// Embedding table: rows looked up and scaled, Y_t = scale E[id_t], and the table's gradient
//     dE_v = beta dE_v + scale * sum of dY_t over the tokens with id_t = v.
// An id outside the vocabulary stands for no word: a row of zeros, no gradient.
//
// Both are bound by HBM.  The gradient's bytes are dY read once and the table written once (with beta = 1 the rows of the words that
// occur only).  Its sums are taken over the tokens sorted by word: a stable radix sort with up to nine bits per pass (a kernel of
// histograms and one that scatters), then runs of 32 sorted tokens per block.  A word whose tokens lie in one run is finished
// there; what runs over a border leaves an fp32 row, and those rows, still sorted, are summed the same way level by level.  Every
// sum has a fixed order: reproducible bits, and a word that fills an eighth of the batch costs no more than others.  Rows of words that
// do not occur are written by blocks of their own in the launch of the first level, beside its latency-bound gathers.
#include <algorithm>

#include "acx_internal.h"
#include "acx_q8.cuh"

namespace acx {
namespace embed {
namespace {

using q8::load8;
using q8::store8;

constexpr int kThreads = 256;

// ----------------------------------------------------------------------------------------------------------------- lookup
constexpr int kLookRows = 4;   // rows per thread, all asked for before the first is stored
// `lanes` threads (a power of two) share a row.
template <typename T>
__global__ void __launch_bounds__(kThreads) lookup_kernel(const int64_t* __restrict__ ids, const T* __restrict__ E, T* __restrict__ Y, int64_t tokens,
                                                          int d, int64_t vocab, float scale, int lanes) {
  wait_for_launch_before();
  let_next_launch_start();
  const int slots = kThreads / lanes, slot = threadIdx.x / lanes, lane = threadIdx.x & (lanes - 1);
  const int64_t row0 = int64_t(blockIdx.x) * (slots * kLookRows) + slot;
  int64_t id[kLookRows];
#pragma unroll
  for (int i = 0; i < kLookRows; ++i) id[i] = row0 + i * slots < tokens ? __ldcg(reinterpret_cast<const long long*>(ids) + row0 + i * slots) : -1;
  for (int c = lane * 8; c < d; c += lanes * 8) {
    q8::Raw<T> x[kLookRows];
#pragma unroll
    for (int i = 0; i < kLookRows; ++i) {
      x[i].zero();
      if (id[i] >= 0 && id[i] < vocab) x[i].load(E + id[i] * d + c);
    }
#pragma unroll
    for (int i = 0; i < kLookRows; ++i) {
      if (row0 + i * slots >= tokens) break;
      float2 v[4];
      x[i].get(v);
#pragma unroll
      for (int k = 0; k < 4; ++k) v[k] = q8::mul2(v[k], q8::both(scale));
      store8(Y + (row0 + i * slots) * d + c, v);
    }
  }
}

// ------------------------------------------------------------------------------------------------------------------- sort
constexpr int kSortThreads = 1024, kSortWarps = kSortThreads / 32, kRounds = 8;
constexpr int kSortItems = kSortThreads * kRounds;   // per block; a warp has 32 * kRounds of them in a row
constexpr int kMaxDigit = 9, kMaxBins = 1 << kMaxDigit;

struct SortPass {
  const int64_t* ids;        // first pass: keys from the ids, values 0, 1, 2, ...
  const uint2* in;           // later passes: (key, token)
  uint2* out;
  uint32_t* table;           // [block][bins]
  int64_t n;
  uint32_t vocab;            // the key of every id outside the vocabulary
  int shift, bins, blocks;
  uint32_t* present;         // last pass: one bit per word that occurs
};
__device__ __forceinline__ uint2 sort_item(const SortPass& s, int64_t i) {
  if (!s.ids) return __ldcg(s.in + i);
  const int64_t id = __ldcg(reinterpret_cast<const long long*>(s.ids) + i);
  return make_uint2(id >= 0 && id < int64_t(s.vocab) ? uint32_t(id) : s.vocab, uint32_t(i));
}
__device__ __forceinline__ int64_t sort_at(int round) {
  return int64_t(blockIdx.x) * kSortItems + (threadIdx.x >> 5) * (32 * kRounds) + 32 * round + (threadIdx.x & 31);
}

__global__ void __launch_bounds__(kSortThreads) histogram_kernel(const SortPass s, uint32_t* clear, int clear_words) {
  __shared__ uint32_t count[kMaxBins];
  for (int b = threadIdx.x; b < s.bins; b += kSortThreads) count[b] = 0;
  wait_for_launch_before();
  let_next_launch_start();
  for (int i = blockIdx.x * kSortThreads + threadIdx.x; i < clear_words; i += gridDim.x * kSortThreads) clear[i] = 0u;
  __syncthreads();
#pragma unroll
  for (int r = 0; r < kRounds; ++r) {
    const int64_t i = sort_at(r);
    const uint32_t digit = i < s.n ? (sort_item(s, i).x >> s.shift) & (s.bins - 1) : kMaxBins;
    const uint32_t same = __match_any_sync(0xFFFFFFFFu, digit);
    if (digit < kMaxBins && __ffs(same) - 1 == int(threadIdx.x & 31)) atomicAdd(&count[digit], __popc(same));
  }
  __syncthreads();
  for (int b = threadIdx.x; b < s.bins; b += kSortThreads) s.table[int64_t(blockIdx.x) * s.bins + b] = count[b];
}

// Where every digit of this block's warps goes: the items of smaller digits, those of the blocks before, of the warps before.
__global__ void __launch_bounds__(kSortThreads) scatter_kernel(const SortPass s) {
  extern __shared__ uint32_t place[];   // [warp][bins]
  __shared__ uint32_t warp_sums[kSortWarps];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  for (int b = threadIdx.x; b < kSortWarps * s.bins; b += kSortThreads) place[b] = 0u;
  wait_for_launch_before();
  let_next_launch_start();
  __syncthreads();
  uint2 item[kRounds];
  uint32_t same[kRounds];
#pragma unroll
  for (int r = 0; r < kRounds; ++r) {
    const int64_t i = sort_at(r);
    item[r] = i < s.n ? sort_item(s, i) : make_uint2(0u, 0xFFFFFFFFu);   // no token has that number
  }
  auto digit_of = [&](uint2 x) { return x.y == 0xFFFFFFFFu ? uint32_t(kMaxBins) : (x.x >> s.shift) & (s.bins - 1); };
#pragma unroll
  for (int r = 0; r < kRounds; ++r) {
    const uint32_t digit = digit_of(item[r]);
    same[r] = __match_any_sync(0xFFFFFFFFu, digit);
    if (digit < kMaxBins && __ffs(same[r]) - 1 == lane) place[warp * s.bins + digit] += __popc(same[r]);
    __syncwarp();
  }
  __syncthreads();
  // thread b (bins <= kSortThreads): all items of digit b, and those of the blocks before this one
  const int b = threadIdx.x;
  uint32_t all = 0, before = 0;
  if (b < s.bins) {
#pragma unroll 8
    for (int k = 0; k < s.blocks; ++k) {
      const uint32_t c = __ldcg(s.table + int64_t(k) * s.bins + b);
      all += c;
      if (k < int(blockIdx.x)) before += c;
    }
  }
  uint32_t x = all;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const uint32_t y = __shfl_up_sync(0xFFFFFFFFu, x, o);
    if (lane >= o) x += y;
  }
  if (lane == 31) warp_sums[warp] = x;
  __syncthreads();
  if (warp == 0) {
    uint32_t w = warp_sums[lane];
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const uint32_t y = __shfl_up_sync(0xFFFFFFFFu, w, o);
      if (lane >= o) w += y;
    }
    warp_sums[lane] = w;
  }
  __syncthreads();
  if (b < s.bins) {
    uint32_t at = x - all + (warp ? warp_sums[warp - 1] : 0u) + before;
    for (int w = 0; w < kSortWarps; ++w) {
      const uint32_t c = place[w * s.bins + b];
      place[w * s.bins + b] = at;
      at += c;
    }
  }
  __syncthreads();
#pragma unroll
  for (int r = 0; r < kRounds; ++r) {
    const uint32_t digit = digit_of(item[r]);
    const bool live = digit < kMaxBins, leader = __ffs(same[r]) - 1 == lane;
    const uint32_t at = live ? place[warp * s.bins + digit] : 0u;
    __syncwarp();
    if (live) {
      s.out[at + __popc(same[r] & ((1u << lane) - 1u))] = item[r];
      if (leader) place[warp * s.bins + digit] = at + __popc(same[r]);
    }
    __syncwarp();
    if (s.present && live && item[r].x < s.vocab) atomicOr(s.present + (item[r].x >> 5), 1u << (item[r].x & 31u));
  }
}

// ------------------------------------------------------------------------------------------------------------------- sums
constexpr int kRun = 32;            // sorted tokens, or rows of the level below, per block
constexpr int kSumThreads = 128;
constexpr int kFillRows = 16;       // rows of the table per block that looks after absent words

// What a level sums: rows of `src` named by `order`, sorted by word.  It leaves two rows per block: what its first word has there, if that
// word began before, and what its last word has there, if that goes on behind (a word that does both is in the first).
struct Level {
  const uint2* order;        // first level: (word, token); later ones: null
  const uint32_t* words;     // later levels: the word of each row below, or kNone
  int64_t n;                 // rows
  float* part;               // [block][2][d]
  uint32_t* part_word;       // [block][2]
  uint32_t vocab;
};
constexpr uint32_t kNone = 0xFFFFFFFFu;

template <typename S, typename G>
__global__ void __launch_bounds__(kSumThreads) sum_kernel(const Level l, const S* __restrict__ src, G* __restrict__ dE, int d, float scale, float beta,
                                                          int run_blocks, const uint32_t* __restrict__ present, int64_t vocab_rows) {
  __shared__ uint32_t word[kRun + 2];   // with a neighbour on either side
  __shared__ uint32_t token[kRun];
  wait_for_launch_before();
  let_next_launch_start();
  const int col = (blockIdx.y * kSumThreads + threadIdx.x) * 8;
  if (int(blockIdx.x) >= run_blocks) {
    // words that do not occur
    const int64_t row0 = int64_t(int(blockIdx.x) - run_blocks) * kFillRows;
    const uint32_t bits = __ldcg(present + (row0 >> 5)) >> (row0 & 31);
    if (col >= d) return;
#pragma unroll 4
    for (int r = 0; r < kFillRows; ++r) {
      if (row0 + r >= vocab_rows || ((bits >> r) & 1u)) continue;
      G* at = dE + (row0 + r) * d + col;
      float2 v[4] = {};
      if (beta != 0.f) {
        load8(at, v);
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] = q8::mul2(v[k], q8::both(beta));
      }
      store8(at, v);
    }
    return;
  }
  const int64_t i0 = int64_t(blockIdx.x) * kRun;
  const int count = int(min(int64_t(kRun), l.n - i0));
  const bool top = l.part == nullptr;     // the last level: one block, nothing on either side
  for (int k = threadIdx.x; k < kRun + 2; k += kSumThreads) {
    const int64_t i = i0 + k - 1;
    uint32_t w = kNone;
    if (i >= 0 && i < l.n) {
      if (l.order) {
        const uint2 o = __ldcg(l.order + i);
        w = o.x < l.vocab ? o.x : kNone;
        if (k >= 1 && k <= kRun) token[k - 1] = o.y;
      } else {
        w = __ldcg(l.words + i);
        if (k >= 1 && k <= kRun) token[k - 1] = uint32_t(i);
      }
    }
    word[k] = w;
  }
  __syncthreads();
  // Rows below without a word are holes; a run's neighbours are the words next to it that are none.  In the first level there are
  // holes at the end only; in later ones a hole beside the border may hide the neighbour, so the search goes on from there.
  uint32_t prev = word[0], next = word[count + 1];
  if (!l.order) {
    for (int64_t i = i0 - 2; prev == kNone && i >= 0 && i >= i0 - 4; --i) prev = __ldcg(l.words + i);
    for (int64_t i = i0 + count + 1; next == kNone && i < l.n && i <= i0 + count + 3; ++i) next = __ldcg(l.words + i);
  }
  uint32_t first = kNone, last = kNone;
  for (int k = 0; k < count; ++k) {
    const uint32_t w = word[k + 1];
    if (w != kNone) {
      if (first == kNone) first = w;
      last = w;
    }
  }
  const bool from_before = first != kNone && first == prev, goes_on = last != kNone && last == next;
  if (!top && blockIdx.y == 0 && threadIdx.x < 2)
    l.part_word[2 * int64_t(blockIdx.x) + threadIdx.x] =
        threadIdx.x == 0 ? (from_before ? first : kNone) : (goes_on && !(from_before && last == first) ? last : kNone);
  if (col >= d) return;
  float2 sum[4] = {};
  uint32_t current = kNone;
  auto flush = [&]() {
    if (current == kNone) return;
    float2 v[4];
    const bool head = from_before && current == first, tail = goes_on && current == last;
    if (!top && (head || tail)) {
      store8(l.part + (2 * int64_t(blockIdx.x) + (head ? 0 : 1)) * d + col, sum);
    } else {
      G* at = dE + int64_t(current) * d + col;
#pragma unroll
      for (int k = 0; k < 4; ++k) v[k] = make_float2(0.f, 0.f);
      if (beta != 0.f) {
        load8(at, v);
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] = q8::mul2(v[k], q8::both(beta));
      }
#pragma unroll
      for (int k = 0; k < 4; ++k) v[k] = q8::fma2(sum[k], q8::both(scale), v[k]);
      store8(at, v);
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) sum[k] = make_float2(0.f, 0.f);
  };
  constexpr int kAhead = 8;
  for (int k0 = 0; k0 < count; k0 += kAhead) {
    q8::Raw<S> x[kAhead];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      x[k].zero();
      if (k0 + k < count && word[k0 + k + 1] != kNone) x[k].load(src + int64_t(token[k0 + k]) * d + col);
    }
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      if (k0 + k >= count) break;
      const uint32_t w = word[k0 + k + 1];
      if (w == kNone) continue;
      if (w != current) {
        flush();
        current = w;
      }
      float2 v[4];
      x[k].get(v);
#pragma unroll
      for (int q = 0; q < 4; ++q) sum[q] = q8::add2(sum[q], v[q]);
    }
  }
  flush();
}

// A whole table times beta: a batch without tokens.
template <typename G>
__global__ void __launch_bounds__(kThreads) scale_kernel(G* __restrict__ dE, int64_t n, float beta) {
  wait_for_launch_before();
  let_next_launch_start();
  const int64_t at = (int64_t(blockIdx.x) * kThreads + threadIdx.x) * 8;
  if (at >= n) return;
  float2 v[4];
  load8(dE + at, v);
#pragma unroll
  for (int k = 0; k < 4; ++k) v[k] = q8::mul2(v[k], q8::both(beta));
  store8(dE + at, v);
}

size_t aligned(size_t n) { return (n + 255) & ~size_t(255); }
int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

struct Plan {
  int passes, digit, blocks;
  size_t items[2], table, present, part[2], part_word[2], bytes;
};
Plan plan_of(const EmbedProblem& q) {
  Plan p;
  int bits = 1;
  while ((int64_t(1) << bits) <= q.vocab) ++bits;   // keys 0 .. vocab
  p.passes = (bits + kMaxDigit - 1) / kMaxDigit;
  p.digit = (bits + p.passes - 1) / p.passes;
  p.blocks = int(ceil_div(q.tokens, kSortItems));
  size_t at = 0;
  auto take = [&](size_t n) { const size_t here = at; at += aligned(n); return here; };
  for (size_t& i : p.items) i = take(size_t(q.tokens) * 8);
  p.table = take(size_t(p.blocks) * (size_t(1) << p.digit) * 4);
  p.present = take(size_t(q.vocab / 32 + 2) * 4);
  int64_t n = ceil_div(q.tokens, kRun);   // blocks of the level that leaves these rows
  for (int k = 0; k < 2; ++k) {
    p.part[k] = take(size_t(n) * 2 * size_t(q.d) * 4);
    p.part_word[k] = take(size_t(n) * 2 * 4);
    n = ceil_div(2 * n, kRun);
  }
  p.bytes = at;
  return p;
}

template <typename S, typename G>
cudaError_t sums(const EmbedProblem& q, const Plan& p, const uint2* order, const S* dY, G* dE, float beta, uint8_t* ws, cudaStream_t st) {
  const unsigned cols = unsigned(ceil_div(q.d, kSumThreads * 8));
  const uint32_t* present = reinterpret_cast<const uint32_t*>(ws + p.present);
  const int64_t fill = beta == 1.f ? 0 : ceil_div(q.vocab, kFillRows);
  int64_t blocks = ceil_div(q.tokens, kRun);
  Level l{order, nullptr, q.tokens, nullptr, nullptr, uint32_t(q.vocab)};
  auto leave = [&](int level) {
    l.part = blocks > 1 ? reinterpret_cast<float*>(ws + p.part[level & 1]) : nullptr;
    l.part_word = reinterpret_cast<uint32_t*>(ws + p.part_word[level & 1]);
  };
  leave(0);
  cudaError_t e = launch_lined_up(sum_kernel<S, G>, dim3(unsigned(blocks + fill), cols), dim3(kSumThreads), 0, st, l, dY, dE, int(q.d), q.scale, beta,
                                  int(blocks), present, q.vocab);
  for (int level = 1; e == cudaSuccess && blocks > 1; ++level) {
    const float* src = l.part;
    l = Level{nullptr, l.part_word, 2 * blocks, nullptr, nullptr, uint32_t(q.vocab)};
    blocks = ceil_div(l.n, kRun);
    leave(level);
    e = launch_lined_up(sum_kernel<float, G>, dim3(unsigned(blocks), cols), dim3(kSumThreads), 0, st, l, src, dE, int(q.d), q.scale, beta, int(blocks),
                        present, q.vocab);
  }
  return e;
}

}  // namespace
}  // namespace embed

using namespace embed;

cudaError_t embed_fwd(const EmbedProblem& q, const int64_t* ids, const void* E, void* Y, cudaStream_t st) {
  int lanes = 1;
  while (lanes < kThreads && lanes * 8 < q.d) lanes *= 2;
  const int64_t rows = kThreads / lanes * kLookRows;
  const dim3 grid(unsigned(ceil_div(q.tokens, rows)));
  if (q.bf16)
    return launch_lined_up(lookup_kernel<__nv_bfloat16>, grid, dim3(kThreads), 0, st, ids, static_cast<const __nv_bfloat16*>(E),
                           static_cast<__nv_bfloat16*>(Y), q.tokens, int(q.d), q.vocab, q.scale, lanes);
  return launch_lined_up(lookup_kernel<float>, grid, dim3(kThreads), 0, st, ids, static_cast<const float*>(E), static_cast<float*>(Y), q.tokens,
                         int(q.d), q.vocab, q.scale, lanes);
}

size_t embed_bwd_workspace_bytes(const EmbedProblem& q) { return plan_of(q).bytes; }

cudaError_t embed_bwd(const EmbedProblem& q, const int64_t* ids, const void* dY, void* dE, float beta, void* ws, cudaStream_t st) {
  if (q.tokens == 0) {   // beta dE
    const size_t n = size_t(q.vocab) * size_t(q.d);
    if (beta == 1.f) return cudaSuccess;
    if (beta == 0.f) return cudaMemsetAsync(dE, 0, n * (q.grad_bf16 ? 2 : 4), st);
    const dim3 grid(unsigned((n / 8 + kThreads - 1) / kThreads));
    if (q.grad_bf16) return launch_lined_up(scale_kernel<__nv_bfloat16>, grid, dim3(kThreads), 0, st, static_cast<__nv_bfloat16*>(dE), int64_t(n), beta);
    return launch_lined_up(scale_kernel<float>, grid, dim3(kThreads), 0, st, static_cast<float*>(dE), int64_t(n), beta);
  }
  const Plan p = plan_of(q);
  uint8_t* w8 = static_cast<uint8_t*>(ws);
  uint2* items[2] = {reinterpret_cast<uint2*>(w8 + p.items[0]), reinterpret_cast<uint2*>(w8 + p.items[1])};
  uint32_t* present = reinterpret_cast<uint32_t*>(w8 + p.present);
  SortPass s{};
  s.table = reinterpret_cast<uint32_t*>(w8 + p.table);
  s.n = q.tokens;
  s.vocab = uint32_t(q.vocab);
  s.bins = 1 << p.digit;
  s.blocks = p.blocks;
  const int smem = kSortWarps * s.bins * 4;
  static DeviceOnce once;
  if (once.needed()) {
    const cudaError_t e = cudaFuncSetAttribute(scatter_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSortWarps * kMaxBins * 4);
    if (e != cudaSuccess) return e;
    once.done();
  }
  for (int k = 0; k < p.passes; ++k) {
    s.ids = k == 0 ? ids : nullptr;
    s.in = items[(k & 1) ^ 1];
    s.out = items[k & 1];
    s.shift = k * p.digit;
    s.present = k + 1 == p.passes ? present : nullptr;
    cudaError_t e = launch_lined_up(histogram_kernel, dim3(unsigned(p.blocks)), dim3(kSortThreads), 0, st, s, present,
                                    k == 0 ? int(q.vocab / 32 + 2) : 0);
    if (e == cudaSuccess) e = launch_lined_up(scatter_kernel, dim3(unsigned(p.blocks)), dim3(kSortThreads), size_t(smem), st, s);
    if (e != cudaSuccess) return e;
  }
  const uint2* order = items[(p.passes - 1) & 1];
  if (q.bf16) {
    const __nv_bfloat16* g = static_cast<const __nv_bfloat16*>(dY);
    return q.grad_bf16 ? sums(q, p, order, g, static_cast<__nv_bfloat16*>(dE), beta, w8, st) : sums(q, p, order, g, static_cast<float*>(dE), beta, w8, st);
  }
  const float* g = static_cast<const float*>(dY);
  return q.grad_bf16 ? sums(q, p, order, g, static_cast<__nv_bfloat16*>(dE), beta, w8, st) : sums(q, p, order, g, static_cast<float*>(dE), beta, w8, st);
}

}  // namespace acx
