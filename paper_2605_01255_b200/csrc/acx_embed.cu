// Embedding table: rows looked up and scaled, Y_t = scale E[id_t], and the table's gradient
//     dE_v = beta dE_v + scale * sum of dY_t over the tokens with id_t = v.
// An id outside the vocabulary stands for no word: a row of zeros, no gradient.
//
// Both are bound by HBM: together 198 us for 16384 tokens x 2048 in bf16, 128256 words and an fp32 gradient, 6.3 TB/s (96 % of a copy's
// rate); small tables are bound by the latency of the sort and the sums (5003 x 1000 fp32, 32003 words 56 us, 3.4 TB/s).  The
// gradient's bytes are dY read once and the table written once (with beta = 1 the rows of the words that occur only).
//
// Its sums are taken over the tokens sorted by word: a stable radix sort with up to nine bits per pass (histograms of the first
// digits by a launch of their own, of the others by the pass before; few tokens in one block), then runs of 32 sorted tokens per
// block.  A word whose tokens lie in one run is finished there; what runs over a border leaves an fp32 row, and those rows, still
// sorted, are summed the same way, 64 at a time, by the block that finishes the last of the runs they come from, level by level in
// the same launch.  Every sum has a fixed order, whichever block takes it: reproducible bits, and a word that fills an eighth of the
// batch costs no more than others.  Rows of words that do not occur are written by blocks of their own beside the latency-bound gathers.
#include <algorithm>

#include "acx_internal.h"
#include "acx_q8.cuh"

namespace acx {
namespace embed {
namespace {

using q8::load8;
using q8::store8;

constexpr int kThreads = 256;
constexpr uint32_t kNone = 0xFFFFFFFFu;

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
constexpr int kSortThreads = 1024, kSortWarps = kSortThreads / 32;
constexpr int kMaxDigit = 9, kMaxBins = 1 << kMaxDigit;
// Items per thread, ROUNDS: one as long as that gives every SM a block at most (a pass is all latency then: two blocks of eight rounds
// took 12 us for 16384 tokens), else eight, so that the table of every block's counts, which each block reads whole, stays small.
constexpr int kFewBlocks = 148, kManyRounds = 8;

struct SortPass {
  const int64_t* ids;        // first pass: keys from the ids, values 0, 1, 2, ...
  const uint2* in;           // later passes: (key, token)
  uint2* out;
  uint32_t* table;           // [block][bins]
  uint32_t* next_table;      // the next pass's, zeros; null in the last pass
  int64_t n;
  uint32_t vocab;            // the key of every id outside the vocabulary
  int shift, digit, blocks;
  uint32_t* present;         // last pass: one bit per word that occurs; null where nobody asks
};
__device__ __forceinline__ uint2 sort_item(const SortPass& s, int64_t i) {
  if (!s.ids) return __ldcg(s.in + i);
  const int64_t id = __ldcg(reinterpret_cast<const long long*>(s.ids) + i);
  return make_uint2(id >= 0 && id < int64_t(s.vocab) ? uint32_t(id) : s.vocab, uint32_t(i));
}
// The lanes of `among` whose v has this lane's lowest bits: a vote per bit (the instruction that matches whole words takes a turn for
// every word that differs: 22.1 us for the sort of 5003 tokens by itself, 20.7 with votes).
__device__ __forceinline__ uint32_t lanes_with(uint32_t v, int bits, uint32_t among) {
#pragma unroll
  for (int b = 0; b < kMaxDigit; ++b) {
    if (b >= bits) break;
    const bool mine = (v >> b) & 1u;
    const uint32_t set = __ballot_sync(0xFFFFFFFFu, mine);
    among &= mine ? set : ~set;
  }
  return among;
}
// A warp has 32 * ROUNDS items in a row.
template <int ROUNDS>
__device__ __forceinline__ int64_t sort_at(int round) {
  return int64_t(blockIdx.x) * (kSortThreads * ROUNDS) + (threadIdx.x >> 5) * (32 * ROUNDS) + 32 * round + (threadIdx.x & 31);
}

template <int ROUNDS>
__global__ void __launch_bounds__(kSortThreads) histogram_kernel(const SortPass s, uint32_t* clear, int64_t clear_words) {
  __shared__ uint32_t count[kMaxBins];
  const int bins = 1 << s.digit;
  for (int b = threadIdx.x; b < bins; b += kSortThreads) count[b] = 0;
  wait_for_launch_before();
  let_next_launch_start();
  for (int64_t i = int64_t(blockIdx.x) * kSortThreads + threadIdx.x; i < clear_words; i += int64_t(gridDim.x) * kSortThreads) clear[i] = 0u;
  if (int(blockIdx.x) >= s.blocks) return;
  __syncthreads();
#pragma unroll
  for (int r = 0; r < ROUNDS; ++r) {
    const int64_t i = sort_at<ROUNDS>(r);
    const bool live = i < s.n;
    const uint32_t digit = live ? (sort_item(s, i).x >> s.shift) & (bins - 1) : 0u;
    const uint32_t same = lanes_with(digit, s.digit, __ballot_sync(0xFFFFFFFFu, live));
    if (live && __ffs(same) - 1 == int(threadIdx.x & 31)) atomicAdd(&count[digit], __popc(same));
  }
  __syncthreads();
  for (int b = threadIdx.x; b < bins; b += kSortThreads) s.table[int64_t(blockIdx.x) * bins + b] = count[b];
}

// Adds up `all` over the threads before this one (of all threads of the block; warp_sums: a word per warp).
__device__ __forceinline__ uint32_t sum_before(uint32_t all, uint32_t* warp_sums) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
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
  return x - all + (warp ? warp_sums[warp - 1] : 0u);
}
// The warps' counts of digit b become their places, from `at` on.
__device__ __forceinline__ void places_of(uint32_t* place, int bins, int b, uint32_t at) {
#pragma unroll
  for (int w0 = 0; w0 < kSortWarps; w0 += 8) {
    uint32_t c[8];
#pragma unroll
    for (int w = 0; w < 8; ++w) c[w] = place[(w0 + w) * bins + b];
#pragma unroll
    for (int w = 0; w < 8; ++w) {
      place[(w0 + w) * bins + b] = at;
      at += c[w];
    }
  }
}

// The whole sort of a few tokens in one block, which keeps the items between the passes; the other blocks, if there are any, write zeros
// to the table meanwhile (every row: those of words that occur are written again by the sums, which then have the memory to themselves:
// the gradient of 5003 x 1000 fp32 with 32003 words 58.8 -> 57.3 us, and 43.6 with what else became faster then).
constexpr int kOneBlockRounds = 8, kOneBlockTokens = kSortThreads * kOneBlockRounds;
__global__ void __launch_bounds__(kSortThreads) small_sort_kernel(const SortPass s, int passes, uint32_t* clear, int64_t clear_words,
                                                                   uint4* zeros, int64_t zero_count) {
  extern __shared__ uint32_t place[];   // [warp][bins], then the items
  __shared__ uint32_t warp_sums[kSortWarps];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, bins = 1 << s.digit, n = int(s.n), rounds = (n + kSortThreads - 1) / kSortThreads;
  uint2* const held = reinterpret_cast<uint2*>(place + kSortWarps * bins);
  wait_for_launch_before();
  let_next_launch_start();
  if (blockIdx.x > 0) {
    for (int64_t i = int64_t(blockIdx.x - 1) * kSortThreads + threadIdx.x; i < zero_count; i += int64_t(gridDim.x - 1) * kSortThreads)
      zeros[i] = make_uint4(0u, 0u, 0u, 0u);
    return;
  }
  uint2 item[kOneBlockRounds];
  uint32_t same[kOneBlockRounds];
  auto at_of = [&](int r) { return warp * (32 * rounds) + 32 * r + lane; };
#pragma unroll
  for (int r = 0; r < kOneBlockRounds; ++r)
    item[r] = r < rounds && at_of(r) < n ? sort_item(s, at_of(r)) : make_uint2(0u, kNone);   // no token has that number
  for (int64_t i = threadIdx.x; i < clear_words; i += kSortThreads) clear[i] = 0u;
  for (int pass = 0; pass < passes; ++pass) {
    const int shift = pass * s.digit;
    const bool end = pass + 1 == passes;
    auto digit_of = [&](uint2 x) { return (x.x >> shift) & (bins - 1); };
    for (int b = threadIdx.x; b < kSortWarps * bins; b += kSortThreads) place[b] = 0u;
    __syncthreads();
#pragma unroll
    for (int r = 0; r < kOneBlockRounds; ++r) {
      if (r >= rounds) break;
      const uint32_t digit = digit_of(item[r]);
      const bool live = item[r].y != kNone;
      same[r] = lanes_with(digit, s.digit, __ballot_sync(0xFFFFFFFFu, live));
      if (live && __ffs(same[r]) - 1 == lane) place[warp * bins + digit] += __popc(same[r]);
      __syncwarp();
    }
    __syncthreads();
    const int b = threadIdx.x;
    uint32_t all = 0;
    if (b < bins) {
#pragma unroll 8
      for (int w = 0; w < kSortWarps; ++w) all += place[w * bins + b];
    }
    const uint32_t at0 = sum_before(all, warp_sums);
    if (b < bins) places_of(place, bins, b, at0);
    __syncthreads();
#pragma unroll
    for (int r = 0; r < kOneBlockRounds; ++r) {
      if (r >= rounds) break;
      const uint32_t digit = digit_of(item[r]);
      const bool live = item[r].y != kNone, leader = __ffs(same[r]) - 1 == lane;
      const uint32_t first = live ? place[warp * bins + digit] : 0u;
      __syncwarp();
      if (live) {
        const uint32_t at = first + __popc(same[r] & ((1u << lane) - 1u));
        (end ? s.out : held)[at] = item[r];
        if (leader) place[warp * bins + digit] = first + __popc(same[r]);
        if (end && s.present && item[r].x < s.vocab) atomicOr(s.present + (item[r].x >> 5), 1u << (item[r].x & 31u));
      }
      __syncwarp();
    }
    if (end) return;
    __syncthreads();
#pragma unroll
    for (int r = 0; r < kOneBlockRounds; ++r)
      if (r < rounds && at_of(r) < n) item[r] = held[at_of(r)];
  }
}

// Where every digit of this block's warps goes: the items of smaller digits, those of the blocks before, of the warps before.
template <int ROUNDS>
__global__ void __launch_bounds__(kSortThreads) scatter_kernel(const SortPass s) {
  extern __shared__ uint32_t place[];   // [warp][bins]
  __shared__ uint32_t warp_sums[kSortWarps];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, bins = 1 << s.digit;
  for (int b = threadIdx.x; b < kSortWarps * bins; b += kSortThreads) place[b] = 0u;
  wait_for_launch_before();
  let_next_launch_start();
  __syncthreads();
  uint2 item[ROUNDS];
  uint32_t same[ROUNDS];
#pragma unroll
  for (int r = 0; r < ROUNDS; ++r) {
    const int64_t i = sort_at<ROUNDS>(r);
    item[r] = i < s.n ? sort_item(s, i) : make_uint2(0u, kNone);   // no token has that number
  }
  // thread b (bins <= kSortThreads): all items of digit b, and those of the blocks before this one
  const int b = threadIdx.x;
  uint32_t all = 0, before = 0;
  if (b < bins) {
#pragma unroll 16
    for (int k = 0; k < s.blocks; ++k) {
      const uint32_t c = __ldcg(s.table + int64_t(k) * bins + b);
      all += c;
      if (k < int(blockIdx.x)) before += c;
    }
  }
  auto digit_of = [&](uint2 x) { return (x.x >> s.shift) & (bins - 1); };
#pragma unroll
  for (int r = 0; r < ROUNDS; ++r) {
    const uint32_t digit = digit_of(item[r]);
    const bool live = item[r].y != kNone;
    same[r] = lanes_with(digit, s.digit, __ballot_sync(0xFFFFFFFFu, live));
    if (live && __ffs(same[r]) - 1 == lane) place[warp * bins + digit] += __popc(same[r]);
    __syncwarp();
  }
  const uint32_t smaller = sum_before(all, warp_sums);
  if (b < bins) places_of(place, bins, b, smaller + before);
  __syncthreads();
#pragma unroll
  for (int r = 0; r < ROUNDS; ++r) {
    const uint32_t digit = digit_of(item[r]);
    const bool live = item[r].y != kNone, leader = __ffs(same[r]) - 1 == lane;
    const uint32_t first = live ? place[warp * bins + digit] : 0u;
    __syncwarp();
    const uint32_t at = first + __popc(same[r] & ((1u << lane) - 1u));
    if (live) {
      s.out[at] = item[r];
      if (leader) place[warp * bins + digit] = first + __popc(same[r]);
    }
    __syncwarp();
    if (s.next_table) {   // counts, whose order does not matter; lanes of one digit go to neighbouring places, of two blocks at most
      const uint32_t block = at / (kSortThreads * ROUNDS), digit2 = (item[r].x >> (s.shift + s.digit)) & (bins - 1);
      const uint32_t odd = __ballot_sync(0xFFFFFFFFu, block & 1u);
      const uint32_t peers = lanes_with(digit2, s.digit, same[r] & (block & 1u ? odd : ~odd));
      if (live && __ffs(peers) - 1 == lane) atomicAdd(s.next_table + block * bins + digit2, __popc(peers));
    }
    if (s.present && live && item[r].x < s.vocab) atomicOr(s.present + (item[r].x >> 5), 1u << (item[r].x & 31u));
  }
}

// ------------------------------------------------------------------------------------------------------------------- sums
constexpr int kRun = 32;            // sorted tokens per block
constexpr int kJoin = 32;           // blocks of a level whose rows are summed together in the next
constexpr int kSumThreads = 128;
constexpr int kFillRows = 16;       // rows of the table per block that looks after absent words
constexpr int kMaxLevels = 8;       // 32^8 tokens and more

// Block i of a level leaves up to two rows of sums: of its first word, if that began before the block, and of its last, if that
// goes on behind.  A word that does both is in the first row.  With them the words: word[2 i] or kNone, word[2 i + 1] or kNone,
// or kGoesOn there if the first row's word goes on behind.
constexpr uint32_t kGoesOn = 0xFFFFFFFEu;
struct Levels {
  int columns;               // blocks of columns
  int count;                 // levels; the last has one block, which leaves nothing
  int blocks[kMaxLevels];
  float* part[kMaxLevels];          // [block][2][d]
  uint32_t* word[kMaxLevels];       // [column block][block][2]
  uint32_t* arrived[kMaxLevels];    // [column block][block / kJoin], zeros at the start
};

// Columns per thread: 16 bytes of dY.  (Eight in fp32 too took 57 us for 5003 x 1000 with 32003 words: twice the blocks share what is
// latency, 43.  Four in bf16, copies of eight bytes: 16384 x 2048 with 128256 words 184 us, 176 with eight.)
template <typename S>
constexpr int kCols = 16 / int(sizeof(S));
__device__ __forceinline__ float4 load4(const float* p) { return __ldcg(reinterpret_cast<const float4*>(p)); }
__device__ __forceinline__ float4 load4(const __nv_bfloat16* p) {
  const uint2 u = __ldcg(reinterpret_cast<const uint2*>(p));
  return make_float4(__uint_as_float(u.x << 16), __uint_as_float(u.x & 0xFFFF0000u), __uint_as_float(u.y << 16), __uint_as_float(u.y & 0xFFFF0000u));
}
__device__ __forceinline__ void store4(float* p, float4 v) { *reinterpret_cast<float4*>(p) = v; }
__device__ __forceinline__ void store4(__nv_bfloat16* p, float4 v) {
  const __nv_bfloat162 a = __floats2bfloat162_rn(v.x, v.y), b = __floats2bfloat162_rn(v.z, v.w);
  *reinterpret_cast<uint2*>(p) = make_uint2(*reinterpret_cast<const uint32_t*>(&a), *reinterpret_cast<const uint32_t*>(&b));
}
template <typename T>
__device__ __forceinline__ void store_cols(T* p, const float4 (&v)[1]) { store4(p, v[0]); }
template <typename T>
__device__ __forceinline__ void store_cols(T* p, const float4 (&v)[2]) {
  const float2 e[4] = {make_float2(v[0].x, v[0].y), make_float2(v[0].z, v[0].w), make_float2(v[1].x, v[1].y), make_float2(v[1].z, v[1].w)};
  store8(p, e);
}

template <typename G, int FOURS>
struct Sink {
  G* dE;
  float* part;               // this block's two rows, null: the last level
  int d, col;
  float scale, beta;
  uint32_t first, last;      // words whose sums go there (kNone: none)
  float4 sum[FOURS];
  uint32_t current;

  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int q = 0; q < FOURS; ++q) sum[q] = make_float4(0.f, 0.f, 0.f, 0.f);
  }
  __device__ __forceinline__ void add(const float4 (&v)[FOURS]) {
#pragma unroll
    for (int q = 0; q < FOURS; ++q) sum[q] = make_float4(sum[q].x + v[q].x, sum[q].y + v[q].y, sum[q].z + v[q].z, sum[q].w + v[q].w);
  }
  __device__ __forceinline__ void flush() {
    if (current == kNone) return;
    if (current == first || current == last) {
      store_cols(part + (current == first ? 0 : d) + col, sum);
    } else {
      G* at = dE + int64_t(current) * d + col;
      float4 v[FOURS];
#pragma unroll
      for (int q = 0; q < FOURS; ++q) {
        v[q] = beta != 0.f ? load4(at + 4 * q) : make_float4(0.f, 0.f, 0.f, 0.f);
        v[q] = make_float4(fmaf(sum[q].x, scale, v[q].x * beta), fmaf(sum[q].y, scale, v[q].y * beta), fmaf(sum[q].z, scale, v[q].z * beta),
                           fmaf(sum[q].w, scale, v[q].w * beta));
      }
      store_cols(at, v);
    }
    clear();
  }
};

// A thread's columns of a row in pieces of 16 bytes, on their way through its own places of shared memory
template <int FOURS>
__device__ __forceinline__ void unpack(const uint4 (&u)[1], const __nv_bfloat16*, float4 (&v)[FOURS]) {
  v[0] = make_float4(__uint_as_float(u[0].x << 16), __uint_as_float(u[0].x & 0xFFFF0000u), __uint_as_float(u[0].y << 16), __uint_as_float(u[0].y & 0xFFFF0000u));
  v[1] = make_float4(__uint_as_float(u[0].z << 16), __uint_as_float(u[0].z & 0xFFFF0000u), __uint_as_float(u[0].w << 16), __uint_as_float(u[0].w & 0xFFFF0000u));
}
template <int FOURS>
__device__ __forceinline__ void unpack(const uint4 (&u)[FOURS], const float*, float4 (&v)[FOURS]) {
#pragma unroll
  for (int q = 0; q < FOURS; ++q) v[q] = make_float4(__uint_as_float(u[q].x), __uint_as_float(u[q].y), __uint_as_float(u[q].z), __uint_as_float(u[q].w));
}

// Rows src[row[k]], k < count, with words that are sorted.  A thread copies its columns of many rows into its own places of shared
// memory before it adds the first: one trip to memory for a run, and a loop that is short (with eight rows at a time in registers,
// unrolled, the kernel spilled and the code of the sums' ends was 18 times there: 69 us for 5003 x 1000 fp32).
constexpr int kStage = 32 * kSumThreads * 16;
template <typename S, typename G, int FOURS>
__device__ __forceinline__ void sum_rows(Sink<G, FOURS>& sink, const S* src, const uint32_t* word, const uint32_t* row, int count, uint8_t* stage) {
  constexpr int kPieces = FOURS * 4 * int(sizeof(S)) / 16, kAhead = kStage / (kSumThreads * 16 * kPieces);
  uint4* const mine = reinterpret_cast<uint4*>(stage) + threadIdx.x;
  const uint32_t at = uint32_t(__cvta_generic_to_shared(mine));
  auto staged = [&](int k, float4 (&v)[FOURS]) {
    uint4 u[kPieces];
#pragma unroll
    for (int h = 0; h < kPieces; ++h) u[h] = mine[(k * kPieces + h) * kSumThreads];
    unpack(u, src, v);
  };
  sink.current = kNone;
  sink.clear();
  for (int k0 = 0; k0 < count; k0 += kAhead) {
    const int rows = min(kAhead, count - k0);
#pragma unroll 4
    for (int k = 0; k < rows; ++k) {
      const uint8_t* from = reinterpret_cast<const uint8_t*>(src + int64_t(row[k0 + k]) * sink.d + sink.col);
#pragma unroll
      for (int h = 0; h < kPieces; ++h)
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(at + (k * kPieces + h) * (kSumThreads * 16)), "l"(from + 16 * h) : "memory");
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
    uint32_t w = word[k0];
    float4 v[FOURS];
    staged(0, v);
    for (int k = 0; k < rows; ++k) {
      if (w != sink.current) {
        sink.flush();
        sink.current = w;
      }
      sink.add(v);
      const int next = min(k + 1, rows - 1);
      w = word[k0 + next];
      staged(next, v);
    }
  }
  sink.flush();
}

template <typename S, typename G>
__global__ void __launch_bounds__(kSumThreads) sum_kernel(const Levels levels, const uint2* __restrict__ order, int64_t tokens, uint32_t vocab,
                                                          const S* __restrict__ src, G* __restrict__ dE, int d, float scale, float beta,
                                                          const uint32_t* __restrict__ present) {
  extern __shared__ __align__(16) uint8_t stage[];
  __shared__ uint32_t word[2 * kJoin];
  __shared__ uint32_t row[2 * kJoin];
  __shared__ uint32_t beside[2];
  __shared__ uint64_t there[2];   // bits: rows of a level that are there, and slots that say kGoesOn
  __shared__ bool finished;
  static_assert(kRun <= 2 * kJoin && kJoin == 32 && 2 * kJoin + 2 <= kSumThreads, "one thread per row, two warps");
  wait_for_launch_before();
  let_next_launch_start();
  const int run_blocks = levels.blocks[0], columns = levels.columns;   // (run, block of columns), run by run, then those of absent words
  if (int64_t(blockIdx.x) >= int64_t(run_blocks) * columns) {
    const int64_t row0 = (int64_t(blockIdx.x) - int64_t(run_blocks) * columns) * kFillRows;
    const uint32_t bits = __ldcg(present + (row0 >> 5)) >> (row0 & 31);
    for (int col = threadIdx.x * 8; col < d; col += kSumThreads * 8) {
#pragma unroll 4
      for (int r = 0; r < kFillRows; ++r) {
        if (row0 + r >= int64_t(vocab) || ((bits >> r) & 1u)) continue;
        G* at = dE + (row0 + r) * d + col;
        float2 v[4] = {};
        if (beta != 0.f) {
          load8(at, v);
#pragma unroll
          for (int k = 0; k < 4; ++k) v[k] = q8::mul2(v[k], q8::both(beta));
        }
        store8(at, v);
      }
    }
    return;
  }
  int block = int(blockIdx.x) / columns;
  const int column = int(blockIdx.x) % columns;
  Sink<G, kCols<S> / 4> sink;
  sink.col = (column * kSumThreads + int(threadIdx.x)) * kCols<S>;
  sink.d = d;
  sink.dE = dE;
  sink.scale = scale;
  sink.beta = beta;
  const int64_t i0 = int64_t(block) * kRun;
  int count = int(min(int64_t(kRun), tokens - i0));
  // the words of the run, and by two threads more those on either side
  const int t = threadIdx.x;
  const int64_t i = i0 + (t < count ? t : t == 2 * kJoin ? -1 : count);
  uint32_t w = kNone;
  if ((t < count || t == 2 * kJoin || t == 2 * kJoin + 1) && i >= 0 && i < tokens) {
    const uint2 o = __ldcg(order + i);
    w = o.x < vocab ? o.x : kNone;
    if (t < count) row[t] = o.y;
  }
  if (t < count) word[t] = w;
  if (t == 2 * kJoin || t == 2 * kJoin + 1) beside[t - 2 * kJoin] = w;
  const int live = __syncthreads_count(t < count && w != kNone);   // ids outside the vocabulary are last
  bool from_before = live > 0 && word[0] == beside[0], goes_on = live > 0 && live == count && word[live - 1] == beside[1];
  uint32_t first = live > 0 ? word[0] : kNone, last = live > 0 ? word[live - 1] : kNone;
  count = live;
  for (int level = 0;; ++level) {
    const bool top = level + 1 == levels.count;
    const int64_t pair = 2 * int64_t(block);
    uint32_t* const left = levels.word[level] + 2 * int64_t(column) * levels.blocks[level];
    sink.part = top ? nullptr : levels.part[level] + pair * d;
    sink.first = !top && from_before ? first : kNone;
    sink.last = !top && goes_on ? last : kNone;
    if (sink.col < d) {
      if (level == 0) sum_rows(sink, src, word, row, count, stage);
      else sum_rows(sink, static_cast<const float*>(levels.part[level - 1]), word, row, count, stage);
    }
    if (top) return;
    if (threadIdx.x == 0) {
      left[pair] = sink.first;
      left[pair + 1] = sink.last == kNone ? kNone : sink.last == sink.first ? kGoesOn : sink.last;
    }
    // the block that is the last of its group to come here sums the group's rows
    __threadfence();
    __syncthreads();
    const int group = block / kJoin, members = min(kJoin, levels.blocks[level] - group * kJoin);
    if (threadIdx.x == 0)
      finished = atomicAdd(levels.arrived[level] + int64_t(column) * levels.blocks[level + 1] + group, 1u) == uint32_t(members - 1);
    __syncthreads();
    if (!finished) return;
    __threadfence();
    block = group;
    uint32_t mark = kNone;
    if (t < 2 * members) mark = __ldcg(left + int64_t(group) * (2 * kJoin) + t);
    if (t < 2 * kJoin) {
      const uint32_t a = __ballot_sync(0xFFFFFFFFu, mark < kGoesOn), b = __ballot_sync(0xFFFFFFFFu, mark == kGoesOn);
      if ((t & 31) == 0) {
        reinterpret_cast<uint32_t*>(&there[0])[t >> 5] = a;
        reinterpret_cast<uint32_t*>(&there[1])[t >> 5] = b;
      }
    }
    __syncthreads();
    const uint64_t rows = there[0];
    if (mark < kGoesOn) {
      const int at = __popcll(rows & ((uint64_t(1) << t) - 1u));
      word[at] = mark;
      row[at] = uint32_t(group * (2 * kJoin) + t);
    }
    __syncthreads();
    // The first row that is there: one of a word from before is the group's first block's, as the block before its own would have
    // left a row too.  The last one likewise.
    count = __popcll(rows);
    first = last = kNone;
    from_before = goes_on = false;
    if (count > 0) {
      const int l = 63 - __clzll(rows);
      first = word[0];
      last = word[count - 1];
      from_before = ((__ffsll(rows) - 1) & 1) == 0;
      goes_on = (l & 1) == 1 || ((there[1] >> (l + 1)) & 1u);
    }
  }
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
  int passes, digit, rounds, blocks, columns, levels;
  int64_t level_blocks[kMaxLevels];
  size_t items[2], table, part[kMaxLevels], word[kMaxLevels];
  size_t clear, present, next_table, arrived[kMaxLevels], clear_end;   // zeros for the first launch to write
  size_t bytes;
};
Plan plan_of(const EmbedProblem& q) {
  Plan p{};
  int bits = 1;
  while ((int64_t(1) << bits) <= q.vocab) ++bits;   // keys 0 .. vocab
  p.passes = (bits + kMaxDigit - 1) / kMaxDigit;
  p.digit = (bits + p.passes - 1) / p.passes;
  p.rounds = q.tokens <= int64_t(kFewBlocks) * kSortThreads ? 1 : kManyRounds;
  p.blocks = int(ceil_div(q.tokens, kSortThreads * p.rounds));
  p.columns = int(ceil_div(q.d, kSumThreads * (q.bf16 ? kCols<__nv_bfloat16> : kCols<float>)));
  p.levels = 1;
  p.level_blocks[0] = ceil_div(q.tokens, kRun);
  while (p.level_blocks[p.levels - 1] > 1) {
    p.level_blocks[p.levels] = ceil_div(p.level_blocks[p.levels - 1], kJoin);
    ++p.levels;
  }
  size_t at = 0;
  auto take = [&](size_t n) { const size_t here = at; at += aligned(n); return here; };
  for (size_t& i : p.items) i = take(size_t(q.tokens) * 8);
  p.table = take(size_t(p.blocks) << (p.digit + 2));
  for (int k = 0; k + 1 < p.levels; ++k) {
    p.part[k] = take(size_t(p.level_blocks[k]) * 2 * size_t(q.d) * 4);
    p.word[k] = take(size_t(p.level_blocks[k]) * 2 * size_t(p.columns) * 4);
  }
  p.clear = at;
  p.present = take(size_t(q.vocab / 32 + 2) * 4);
  p.next_table = take((size_t(p.blocks) << (p.digit + 2)) * size_t(p.passes - 1));
  for (int k = 0; k + 1 < p.levels; ++k) p.arrived[k] = take(size_t(p.level_blocks[k + 1]) * size_t(p.columns) * 4);
  p.clear_end = at;
  p.bytes = at;
  return p;
}

template <typename S, typename G>
cudaError_t sums(const EmbedProblem& q, const Plan& p, const uint2* order, const void* dY, void* dE, float beta, bool absent, uint8_t* ws, cudaStream_t st) {
  static DeviceOnce once;
  if (once.needed()) {
    const cudaError_t e = cudaFuncSetAttribute(sum_kernel<S, G>, cudaFuncAttributeMaxDynamicSharedMemorySize, kStage);
    if (e != cudaSuccess) return e;
    once.done();
  }
  Levels l{};
  l.count = p.levels;
  l.columns = p.columns;
  for (int k = 0; k < p.levels; ++k) {
    l.blocks[k] = int(p.level_blocks[k]);
    if (k + 1 == p.levels) break;
    l.part[k] = reinterpret_cast<float*>(ws + p.part[k]);
    l.word[k] = reinterpret_cast<uint32_t*>(ws + p.word[k]);
    l.arrived[k] = reinterpret_cast<uint32_t*>(ws + p.arrived[k]);
  }
  const int64_t fill = absent ? ceil_div(q.vocab, kFillRows) : 0;
  return launch_lined_up(sum_kernel<S, G>, dim3(unsigned(p.level_blocks[0] * p.columns + fill)), dim3(kSumThreads), kStage, st, l, order, q.tokens,
                         uint32_t(q.vocab), static_cast<const S*>(dY), static_cast<G*>(dE), int(q.d), q.scale, beta,
                         reinterpret_cast<const uint32_t*>(ws + p.present));
}

// zeros: the table, or null if its rows are not to be written here.  absent: whether the sums have to know absent words.
cudaError_t small_sort(const EmbedProblem& q, const Plan& p, const int64_t* ids, uint8_t* ws, void* zeros, bool absent, const uint2** order,
                       cudaStream_t st) {
  constexpr int kMost = kSortWarps * kMaxBins * 4 + kOneBlockTokens * 8;
  static DeviceOnce once;
  if (once.needed()) {
    const cudaError_t e = cudaFuncSetAttribute(small_sort_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kMost);
    if (e != cudaSuccess) return e;
    once.done();
  }
  SortPass s{};
  s.ids = ids;
  s.out = reinterpret_cast<uint2*>(ws + p.items[0]);
  s.n = q.tokens;
  s.vocab = uint32_t(q.vocab);
  s.digit = p.digit;
  s.present = absent ? reinterpret_cast<uint32_t*>(ws + p.present) : nullptr;
  *order = s.out;
  const int64_t zero_count = zeros ? q.vocab * q.d * (q.grad_bf16 ? 2 : 4) / 16 : 0;
  const unsigned grid = unsigned(1 + std::min<int64_t>(ceil_div(zero_count, 8 * kSortThreads), 2 * kFewBlocks - 1));
  return launch_lined_up(small_sort_kernel, dim3(grid), dim3(kSortThreads), (size_t(kSortWarps) << (p.digit + 2)) + size_t(q.tokens) * 8, st, s, p.passes,
                         reinterpret_cast<uint32_t*>(ws + p.clear), int64_t(p.clear_end - p.clear) / 4, static_cast<uint4*>(zeros), zero_count);
}

template <int ROUNDS>
cudaError_t sort(const EmbedProblem& q, const Plan& p, const int64_t* ids, uint8_t* ws, bool absent, const uint2** order, cudaStream_t st) {
  static DeviceOnce once;
  if (once.needed()) {
    const cudaError_t e = cudaFuncSetAttribute(scatter_kernel<ROUNDS>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSortWarps * kMaxBins * 4);
    if (e != cudaSuccess) return e;
    once.done();
  }
  uint2* items[2] = {reinterpret_cast<uint2*>(ws + p.items[0]), reinterpret_cast<uint2*>(ws + p.items[1])};
  SortPass s{};
  s.ids = ids;
  s.out = items[0];
  s.table = reinterpret_cast<uint32_t*>(ws + p.table);
  s.n = q.tokens;
  s.vocab = uint32_t(q.vocab);
  s.digit = p.digit;
  s.blocks = p.blocks;
  const int64_t clear_words = int64_t(p.clear_end - p.clear) / 4;
  const unsigned grid = unsigned(std::max<int64_t>(p.blocks, std::min<int64_t>(kFewBlocks, clear_words / (4 * kSortThreads))));
  cudaError_t e = launch_lined_up(histogram_kernel<ROUNDS>, dim3(grid), dim3(kSortThreads), 0, st, s, reinterpret_cast<uint32_t*>(ws + p.clear), clear_words);
  for (int k = 0; k < p.passes && e == cudaSuccess; ++k) {
    uint32_t* const next = reinterpret_cast<uint32_t*>(ws + p.next_table) + (size_t(p.blocks) << p.digit) * size_t(k);
    s.next_table = k + 1 < p.passes ? next : nullptr;
    s.present = absent && k + 1 == p.passes ? reinterpret_cast<uint32_t*>(ws + p.present) : nullptr;
    e = launch_lined_up(scatter_kernel<ROUNDS>, dim3(unsigned(p.blocks)), dim3(kSortThreads), size_t(kSortWarps) << (p.digit + 2), st, s);
    *order = s.out;
    s.ids = nullptr;
    s.in = s.out;
    s.out = items[(k & 1) ^ 1];
    s.table = next;
    s.shift += p.digit;
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
  const uint2* order = nullptr;
  const bool filled = q.tokens <= kOneBlockTokens && beta == 0.f, absent = beta != 1.f && !filled;
  const cudaError_t e = q.tokens <= kOneBlockTokens ? small_sort(q, p, ids, w8, filled ? dE : nullptr, absent, &order, st) : p.rounds == 1 ? sort<1>(q, p, ids, w8, absent, &order, st) : sort<kManyRounds>(q, p, ids, w8, absent, &order, st);
  if (e != cudaSuccess) return e;
  if (q.bf16)
    return q.grad_bf16 ? sums<__nv_bfloat16, __nv_bfloat16>(q, p, order, dY, dE, beta, absent, w8, st) : sums<__nv_bfloat16, float>(q, p, order, dY, dE, beta, absent, w8, st);
  return q.grad_bf16 ? sums<float, __nv_bfloat16>(q, p, order, dY, dE, beta, absent, w8, st) : sums<float, float>(q, p, order, dY, dE, beta, absent, w8, st);
}

}  // namespace acx
