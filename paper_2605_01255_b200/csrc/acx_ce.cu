// Softmax cross entropy of logits = logit_scale * X W^T over a vocabulary, and its gradients, without the logits in memory:
//     lse_t = log sum_v exp(logits_tv),   loss_t = lse_t - logits_ty,
//     D = w (softmax - onehot),   dX = f D W,   dW = f D^T X,   f = scale * logit_scale / denom.
// Forward: one pass of logits tiles that leave (maximum, sum) pairs, joined per token by a small kernel.  Backward: the
// vocabulary in pieces; each piece's D (bf16) is written, used by both products, and overwritten by a later piece's.
#include <algorithm>

#include "acx_ce_gemm.cuh"
#include "acx_tmap.h"

namespace acx {
namespace {

using ce::kLn2;
using ce::kLowest;
using ce::Params;

constexpr int kTokensPerBlock = 8, kJoinThreads = 512;

__device__ __forceinline__ float dot8(uint4 a, uint4 b, float s) {
  const uint32_t x[4] = {a.x, a.y, a.z, a.w}, w[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    s = fmaf(__uint_as_float(x[i] << 16), __uint_as_float(w[i] << 16), s);
    s = fmaf(__uint_as_float(x[i] & 0xFFFF0000u), __uint_as_float(w[i] & 0xFFFF0000u), s);
  }
  return s;
}

// (m, s) <- (m, s) joined with (m1, s1): sums of 2^(x - maximum); one that holds nothing is (kLowest, 0)
__device__ __forceinline__ void join_pair(float& m, float& s, float m1, float s1) {
  const float top = fmaxf(m, m1);
  s = s * exp2f(m - top) + s1 * exp2f(m1 - top);
  m = top;
}

// Joins the (maximum, sum) pairs of 8 tokens: 16 warps; a lane has token lane & 7 and every 64th pair, eight at a time.  The
// pairs are of all words but the target.  Its logit is taken as a plain fp32 product here (two warps per token): the tensor
// core adds 16 products at a time with truncation, an error of up to 2^-24 of the logit per step and of one sign, which the
// loss of an unlikely token would show in full.  With x = log(sum over the others) - target's logit,
//     loss = log(1 + e^x) = max(x, 0) + log(1 + e^-|x|),   lse = the larger of the two + log(1 + e^-|x|),
// so that the loss of a likely token keeps its digits: it is about e^x, and a difference of lse and the target's logit would
// have the rounding of those in it.  The last block to finish adds the blocks' sums of losses and weights, in order.
// Launched behind the logits' kernel before that has finished; the products need nothing of it.
__global__ void __launch_bounds__(kJoinThreads, 3) ce_join_kernel(const float2* part, const __nv_bfloat16* __restrict__ X,
                                                       const __nv_bfloat16* __restrict__ W, const int64_t* __restrict__ targets,
                                                       const float* __restrict__ weight, int tokens, int d, int vocab, int parts, float c,
                                                       float* __restrict__ loss, float* __restrict__ lse, float2* block_sums,
                                                       uint32_t* ticket, float* __restrict__ total) {
  __shared__ float2 red[16][9];
  __shared__ float exact[16];
  __shared__ bool last;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, t0 = int(blockIdx.x) * kTokensPerBlock;
  {
    const int tt = t0 + (warp >> 1);
    const int64_t y = tt < tokens ? __ldg(targets + tt) : -1;
    float p = 0.f;
    if (y >= 0 && y < vocab) {
      const uint4* x = reinterpret_cast<const uint4*>(X + int64_t(tt) * d);
      const uint4* w = reinterpret_cast<const uint4*>(W + y * int64_t(d));
      for (int i0 = (warp & 1) * 32 + lane; i0 < d / 8; i0 += 4 * 64) {   // four vectors of each under way
        uint4 a[4], b[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const bool in = i0 + 64 * k < d / 8;
          a[k] = in ? __ldg(x + i0 + 64 * k) : make_uint4(0u, 0u, 0u, 0u);
          b[k] = in ? __ldg(w + i0 + 64 * k) : make_uint4(0u, 0u, 0u, 0u);
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) p = dot8(a[k], b[k], p);
      }
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) p += __shfl_xor_sync(0xFFFFFFFFu, p, o);
    if (lane == 0) exact[warp] = p;
  }
  wait_for_launch_before();
  let_next_launch_start();
  const int tok = lane & 7, t = t0 + tok;
  float m = kLowest, s = 0.f;
  if (t < tokens) {
    for (int q = warp * 4 + (lane >> 3); q < parts; q += 8 * 64) {   // eight pairs in flight
      float2 v[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = q + 64 * i < parts ? __ldcg(part + int64_t(q + 64 * i) * tokens + t) : make_float2(kLowest, 0.f);
#pragma unroll
      for (int i = 0; i < 8; ++i) join_pair(m, s, v[i].x, v[i].y);
    }
  }
#pragma unroll
  for (int o = 8; o <= 16; o <<= 1) join_pair(m, s, __shfl_xor_sync(0xFFFFFFFFu, m, o), __shfl_xor_sync(0xFFFFFFFFu, s, o));
  if (lane < 8) red[warp][lane] = make_float2(m, s);
  __syncthreads();
  if (warp == 0) {
    m = kLowest;
    s = 0.f;
    for (int k = lane >> 3; k < 16; k += 4) join_pair(m, s, red[k][tok].x, red[k][tok].y);
#pragma unroll
    for (int o = 8; o <= 16; o <<= 1) join_pair(m, s, __shfl_xor_sync(0xFFFFFFFFu, m, o), __shfl_xor_sync(0xFFFFFFFFu, s, o));
    float wl = 0.f, wt = 0.f;
    if (lane < 8 && t < tokens) {
      const int64_t y = __ldg(targets + t);
      const bool trained = y >= 0 && y < vocab;
      const float others = m + log2f(s), ty = trained ? (exact[2 * tok] + exact[2 * tok + 1]) * c : -INFINITY;
      // (no word possible at all: infinity minus infinity, NaN)
      const float x = others - ty, beside = log1pf(exp2f(-fabsf(x)));
      lse[t] = fmaf(x > 0.f ? others : ty, kLn2, beside);
      const float l = trained ? fmaf(fmaxf(x, 0.f), kLn2, beside) : 0.f;
      loss[t] = l;
      wt = trained ? (weight ? __ldg(weight + t) : 1.f) : 0.f;
      wl = trained ? wt * l : 0.f;
    }
#pragma unroll
    for (int o = 4; o > 0; o >>= 1) {
      wl += __shfl_xor_sync(0xFFFFFFFFu, wl, o);
      wt += __shfl_xor_sync(0xFFFFFFFFu, wt, o);
    }
    if (lane == 0 && total) {
      block_sums[blockIdx.x] = make_float2(wl, wt);
      __threadfence();
      last = atomicAdd(ticket, 1u) == gridDim.x - 1;
    }
  }
  if (!total) return;
  __syncthreads();
  if (!last) return;
  __threadfence();
  float a = 0.f, b = 0.f;
  for (int i = threadIdx.x; i < int(gridDim.x); i += kJoinThreads) {
    const float2 v = __ldcg(block_sums + i);
    a += v.x;
    b += v.y;
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    a += __shfl_xor_sync(0xFFFFFFFFu, a, o);
    b += __shfl_xor_sync(0xFFFFFFFFu, b, o);
  }
  if (lane == 0) red[warp][0] = make_float2(a, b);
  __syncthreads();
  if (warp != 0) return;
  a = lane < 16 ? red[lane][0].x : 0.f;
  b = lane < 16 ? red[lane][0].y : 0.f;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    a += __shfl_xor_sync(0xFFFFFFFFu, a, o);
    b += __shfl_xor_sync(0xFFFFFFFFu, b, o);
  }
  if (lane == 0) {
    total[0] = a;
    total[1] = b;
  }
}

// dX = f (sum over the splits + corr W[y]): what rounding D to bf16 took from the target's element, the largest of its row
// and the only one whose rounding is not averaged out, comes back here in fp32.
__global__ void __launch_bounds__(256) ce_finish_kernel(const float* acc, int splits, int64_t split_stride,
                                                        const float* corr, const int64_t* __restrict__ targets,
                                                        const __nv_bfloat16* __restrict__ W, const float* __restrict__ denom, float scale,
                                                        __nv_bfloat16* __restrict__ dX, int tokens, int d, int vocab) {
  wait_for_launch_before();
  let_next_launch_start();
  const int vecs = d / 8;
  const int64_t i = int64_t(blockIdx.x) * 256 + threadIdx.x;
  const int64_t t = i / vecs;
  if (t >= tokens) return;
  const int c = int(i - t * vecs) * 8;
  const float dn = denom ? __ldcg(denom) : 1.f, f = dn > 0.f ? scale / dn : 0.f;
  float v[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = 0.f;
  for (int s0 = 0; s0 < splits; s0 += 4) {   // four splits' loads under way, added in order
    float4 a[4], b[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const float4* p = reinterpret_cast<const float4*>(acc + (s0 + k) * split_stride + t * d + c);
      a[k] = s0 + k < splits ? __ldcg(p) : make_float4(0.f, 0.f, 0.f, 0.f);
      b[k] = s0 + k < splits ? __ldcg(p + 1) : make_float4(0.f, 0.f, 0.f, 0.f);
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      v[0] += a[k].x; v[1] += a[k].y; v[2] += a[k].z; v[3] += a[k].w;
      v[4] += b[k].x; v[5] += b[k].y; v[6] += b[k].z; v[7] += b[k].w;
    }
  }
  const int64_t y = __ldg(targets + t);
  if (y >= 0 && y < vocab) {
    const float k = __ldcg(corr + t);
    const uint4 w = __ldg(reinterpret_cast<const uint4*>(W + y * int64_t(d) + c));
    const uint32_t ww[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      v[2 * e] = fmaf(k, __uint_as_float(ww[e] << 16), v[2 * e]);
      v[2 * e + 1] = fmaf(k, __uint_as_float(ww[e] & 0xFFFF0000u), v[2 * e + 1]);
    }
  }
  uint32_t o[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(v[2 * e] * f, v[2 * e + 1] * f);
    o[e] = *reinterpret_cast<const uint32_t*>(&h);
  }
  *reinterpret_cast<uint4*>(dX + t * d + c) = make_uint4(o[0], o[1], o[2], o[3]);
}

// What rounding D to bf16 took from the targets' elements, for dW: row_add[t] = sum of corr X over the tokens with the same
// target as t, in fp32 and in the order of the tokens, where t is the first of them (row_key[t] = its target; -1 for the
// others).  A target's element is most of what its token adds to dW.  With few tokens the rounding of each would be seen in
// full (with one to sixteen weighted tokens up to 3 times the error of rounding dW alone, more than 1.5 times in one case out
// of four, 1.25 to 1.3 times at 257 to 512 tokens, where it is 1.0 times with this).  Done for up to 512 tokens; it takes 4 to
// 6 us of the 35 to 150 us of a step, and 14 us of the backward at 333 x 904 x 32003, whose products wait for it (101 -> 115
// us).  Folding it into the products' epilogue token by token took twice as
// long: targets are skewed, and a frequent word's tokens all meet one lane there.
using ce::kPutBackTokens;
__global__ void __launch_bounds__(kPutBackTokens) ce_put_back_kernel(const float* corr, const int64_t* __restrict__ targets,
                                                                     const __nv_bfloat16* __restrict__ X, int tokens, int d, int v0, int v1,
                                                                     int* __restrict__ row_key, float* __restrict__ row_add) {
  __shared__ int same[kPutBackTokens];
  __shared__ float weight[kPutBackTokens];
  __shared__ int counts[kPutBackTokens / 32];
  const int t = int(blockIdx.x), tt = int(threadIdx.x), lane = tt & 31, warp = tt >> 5;
  const int64_t y = __ldg(targets + t);
  const bool here = y >= v0 && y < v1;                     // the target is in this piece of the vocabulary
  const bool hit = here && tt < tokens && __ldg(targets + tt) == y;
  wait_for_launch_before();
  let_next_launch_start();
  if (!__syncthreads_or(here) || __syncthreads_or(hit && tt < t)) {   // not here, or another token was there before
    if (tt == 0) row_key[t] = -1;
    return;
  }
  const uint32_t hits = __ballot_sync(0xFFFFFFFFu, hit);
  if (lane == 0) counts[warp] = __popc(hits);
  __syncthreads();
  int at = __popc(hits & ((1u << lane) - 1u)), n = 0;
  for (int w = 0; w < kPutBackTokens / 32; ++w) {
    at += w < warp ? counts[w] : 0;
    n += counts[w];
  }
  if (hit) {
    same[at] = tt;
    weight[at] = __ldcg(corr + tt);
  }
  __syncthreads();
  for (int c = tt; c < d / 8; c += kPutBackTokens) {
    float s[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    for (int k0 = 0; k0 < n; k0 += 4) {
      uint4 x[4];
#pragma unroll
      for (int k = 0; k < 4; ++k)
        x[k] = k0 + k < n ? __ldg(reinterpret_cast<const uint4*>(X + int64_t(same[k0 + k]) * d) + c) : make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const float w = k0 + k < n ? weight[k0 + k] : 0.f;
        const uint32_t h[4] = {x[k].x, x[k].y, x[k].z, x[k].w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          s[2 * i] = fmaf(w, __uint_as_float(h[i] << 16), s[2 * i]);
          s[2 * i + 1] = fmaf(w, __uint_as_float(h[i] & 0xFFFF0000u), s[2 * i + 1]);
        }
      }
    }
    float4* o = reinterpret_cast<float4*>(row_add + int64_t(t) * d + 8 * c);
    o[0] = make_float4(s[0], s[1], s[2], s[3]);
    o[1] = make_float4(s[4], s[5], s[6], s[7]);
  }
  if (tt == 0) row_key[t] = int(y);
}

int ceil_div(int64_t a, int64_t b) { return int((a + b - 1) / b); }
size_t aligned(size_t bytes) { return (bytes + 1023) & ~size_t(1023); }

int pair_count() { return std::max(1, sm_count() / 2); }

template <int KIND, bool FEW>
cudaError_t launch(const CUtensorMap& ta, const CUtensorMap& tb, const CUtensorMap& ta2, const CUtensorMap& tb2, const CUtensorMap& to,
                   const CUtensorMap& to2, const CUtensorMap& to3, const Params& p, cudaStream_t st) {
  auto kernel = ce::ce_kernel<KIND, FEW>;
  static DeviceOnce once;
  if (once.needed()) {
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, ce::kSmemBytes);
    if (e != cudaSuccess) return e;
    once.done();
  }
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(unsigned(2 * std::min(p.units, pair_count())));
  cfg.blockDim = dim3(ce::kThreads);
  cfg.dynamicSmemBytes = ce::kSmemBytes;
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = 2;
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;   // see wait_first
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  const cudaError_t e = cudaLaunchKernelEx(&cfg, kernel, ta, tb, ta2, tb2, to, to2, to3, p);
  kernel_launch_counter().fetch_add(1, std::memory_order_relaxed);
  return e;
}

template <int KIND>
cudaError_t launch(bool few, const CUtensorMap& ta, const CUtensorMap& tb, const CUtensorMap& ta2, const CUtensorMap& tb2,
                   const CUtensorMap& to, const CUtensorMap& to2, const CUtensorMap& to3, const Params& p, cudaStream_t st) {
  return few ? launch<KIND, true>(ta, tb, ta2, tb2, to, to2, to3, p, st) : launch<KIND, false>(ta, tb, ta2, tb2, to, to2, to3, p, st);
}

// Up to 64 tokens: the kernels with the operands exchanged (see FEW).
bool is_few(const CeProblem& q) { return q.m <= ce::kFewTokens; }
int few_columns(const CeProblem& q) { return int(q.m + 31) & ~31; }

// Token tiles that pass over the vocabulary together: as many as have their rows of X (d wide, bf16) in 48 MB, so that X
// stays in L2 beside the tiles of W that stream by.
int token_group(int64_t d, int m_tiles) {
  const int fit = int(std::max<int64_t>(1, (int64_t(48) << 20) / (ce::kTile * d * 2)));
  const int groups = ceil_div(m_tiles, fit);
  return ceil_div(m_tiles, groups);
}

// The tensor core adds 16 products at a time to the running sum and truncates: every sum comes out too small by a share of
// its size.  While a logit builds up over d / 16 steps its running sum is on average half of it, so that the logit ends short
// by d / 16 * kTruncation of itself.  All logits of a row being short alike, the log-sum-exp would be off by that share of the
// mean logit, 2.5e-6 at d = 4096; with the logits' scale raised by it, 3e-7 is left.  How short, in 2^-23 of the logit per
// step (2048 rows): rows of N(0, 1) 0.10 to 0.135 from d = 256 to 65536, the same with 12 or 40 times the word's own row added
// 0.14 to 0.19, with one column in 64 eight times as large 0.145 to 0.16.  Rows that lose less get too much: half of the columns
// zero 0.08, 5 % of them not zero 0.02 to 0.04, sums that are exact 0.  Their logits are then long by up to kTruncation per
// step, less than what dense ones would be short by without it.
constexpr double kTruncation = 0.135 / (1 << 23);

void common(const CeProblem& q, Params* p, const int64_t* targets, const float* weight, int* status) {
  p->tokens = int(q.m);
  p->d = int(q.d);
  p->vocab = int(q.vocab);
  p->m_tiles = ceil_div(q.m, ce::kTile);
  p->group = token_group(q.d, p->m_tiles);
  p->c = float(q.logit_scale * double(ce::kLog2e) * (1.0 + kTruncation * ceil_div(q.d, 16)));
  p->targets = targets;
  p->weight = weight;
  p->status = status;
  p->wait_first = 1;
  p->few_n = few_columns(q);
}

struct FwdPlan {
  int parts, blocks;
  size_t part, sums, ticket, bytes;
};
FwdPlan fwd_plan(const CeProblem& q) {
  FwdPlan f;
  f.parts = is_few(q) ? 8 * std::min(ceil_div(q.vocab, ce::kTile), pair_count()) : ceil_div(q.vocab, ce::kGroupCols);   // see Params::part
  f.blocks = ceil_div(q.m, kTokensPerBlock);
  f.part = 0;
  f.sums = f.part + aligned(size_t(f.parts) * size_t(q.m) * sizeof(float2));
  f.ticket = f.sums + aligned(size_t(f.blocks) * sizeof(float2));
  f.bytes = f.ticket + aligned(4);
  return f;
}

// Pieces of the vocabulary, of equal size: D of one takes at most about 128 MB.  Up to three are under way at a time (see
// ce_bwd).  Backward of 8192 x 3072 x 128256 with 64 / 128 / 256 / 512 MB: 15.3 / 15.1 / 15.0 / 14.9 ms under sustained load;
// of 4096 x 896 x 151936: 3.06 / 2.97 / 2.98 / 2.95 ms.  Larger pieces are not worth their memory.
constexpr int64_t kPieceBytes = int64_t(128) << 20;
constexpr int kBuffers = 3;
struct BwdPlan {
  int piece_tiles, pieces, buffers, splits, kb_per_split, d_tiles, d_width, acc_rows;
  bool put_back;
  size_t D, D_stride, acc, corr, row_key, row_add, bytes;
};
BwdPlan bwd_plan(const CeProblem& q) {
  BwdPlan b;
  const int n_tiles = ceil_div(q.vocab, ce::kTile), m_tiles = ceil_div(q.m, ce::kTile), pairs = pair_count();
  const int fit = int(std::max<int64_t>(1, kPieceBytes / (q.m * ce::kTile * 2)));
  b.pieces = ceil_div(n_tiles, fit);
  b.piece_tiles = ceil_div(n_tiles, b.pieces);
  b.pieces = ceil_div(n_tiles, b.piece_tiles);
  b.buffers = std::min(b.pieces, kBuffers);
  b.d_tiles = ceil_div(q.d, ce::kTile);
  b.d_width = (ceil_div(q.d, b.d_tiles) + 31) & ~31;
  b.acc_rows = is_few(q) ? int(q.m) : m_tiles * ce::kTile;
  // dX is split along the piece where that lets the longest-loaded pair of CTAs finish sooner: pair c takes the units c,
  // c + pairs, ..., the tiles of dX first.  Every split costs its fp32 sums' way through memory (a unit's epilogue is worth
  // about 4 k-blocks, the last kernel's reading about one per split).
  const int piece_kb = b.piece_tiles * (ce::kTile / ce::kBK), token_kb = ceil_div(q.m, ce::kBK);
  const int64_t x1 = is_few(q) ? ceil_div(q.d, ce::kTile) : int64_t(m_tiles) * b.d_tiles, w = int64_t(b.piece_tiles) * b.d_tiles;
  double best = 1e300;
  b.kb_per_split = piece_kb;
  for (int s : {1, 2, 3, 4, 6, 8, 10, 12, 16, 20, 24, 32}) {
    if (s > 1 && piece_kb / s < 8) break;
    const int kb = ceil_div(piece_kb, s);
    const int64_t x = x1 * ceil_div(piece_kb, kb);
    double worst = 0;
    for (int c = 0; c < pairs; ++c) {
      const int64_t nx = x > c ? (x - c + pairs - 1) / pairs : 0, all = x + w > c ? (x + w - c + pairs - 1) / pairs : 0;
      worst = std::max(worst, double(nx) * (kb + 4) + double(all - nx) * (token_kb + 4));
    }
    worst += s;
    if (worst < best) { best = worst; b.kb_per_split = kb; }
  }
  b.splits = ceil_div(piece_kb, b.kb_per_split);
  b.D = 0;
  b.D_stride = aligned(size_t(q.m) * size_t(b.piece_tiles) * ce::kTile * 2);
  b.acc = b.D + size_t(b.buffers) * b.D_stride;
  b.corr = b.acc + aligned(size_t(b.splits) * size_t(b.acc_rows) * size_t(q.d) * 4);
  b.put_back = q.m <= kPutBackTokens;
  b.row_key = b.corr + aligned(size_t(q.m) * 4);
  b.row_add = b.row_key + aligned(size_t(q.m) * 4);
  b.bytes = b.row_add + (b.put_back ? aligned(size_t(q.m) * size_t(q.d) * 4) : 0);
  return b;
}

}  // namespace

size_t ce_fwd_workspace_bytes(const CeProblem& q) { return q.m == 0 ? 0 : fwd_plan(q).bytes; }
size_t ce_bwd_workspace_bytes(const CeProblem& q) { return q.m == 0 ? 0 : std::max(bwd_plan(q).bytes, fwd_plan(q).bytes); }

cudaError_t ce_fwd(const CeProblem& q, const void* X, const void* W, const int64_t* targets, const float* weight, float* loss, float* lse,
                   float* total, void* ws, int* status, cudaStream_t st) {
  const FwdPlan f = fwd_plan(q);
  uint8_t* w8 = static_cast<uint8_t*>(ws);
  Params p{};
  common(q, &p, targets, weight, status);
  p.n_tiles = ceil_div(q.vocab, ce::kTile);
  p.units = is_few(q) ? p.n_tiles : p.m_tiles * p.n_tiles;
  p.part = reinterpret_cast<float2*>(w8 + f.part);
  p.ticket = reinterpret_cast<uint32_t*>(w8 + f.ticket);
  CUtensorMap ta, tb;
  const bool few = is_few(q);
  const int token_box = few ? p.few_n / 2 : ce::kBM;
  if (!make_tmap_bf16(&ta, X, q.m, q.d, ce::kBK, token_box) || !make_tmap_bf16(&tb, W, q.vocab, q.d, ce::kBK, ce::kBM)) return cudaErrorInvalidValue;
  const cudaError_t e = launch<ce::LSE>(few, ta, tb, ta, tb, ta, ta, ta, p, st);
  if (e != cudaSuccess) return e;
  return launch_lined_up(ce_join_kernel, dim3(unsigned(f.blocks)), dim3(kJoinThreads), 0, st, static_cast<const float2*>(p.part),
                       static_cast<const __nv_bfloat16*>(X), static_cast<const __nv_bfloat16*>(W),
                       targets, weight, p.tokens, p.d, p.vocab, f.parts, q.logit_scale * ce::kLog2e, loss, lse, reinterpret_cast<float2*>(w8 + f.sums), p.ticket, total);
}

// The launches of a backward pass, L = DLOGITS and G = GRADS of a piece:
//     L0  L1  G0  L2  G1  L3  G2  ...  G(n-1)
// Two launches in the middle that follow one another need nothing of each other (D has three buffers), and each may start
// while the one before it is still at its last tiles: a launch lets the next one start only after the end of the one before
// itself, so that whatever a launch sees running beside it is its direct neighbour.  G0 thus finds L0 finished, L3 (which
// writes the buffer that G0 read) finds G0 finished, and G1 adds to sums that G0 has finished.  L0 needs the forward's
// results, and the last G follows another G, to whose sums it adds (or its own L): those two wait first.
cudaError_t ce_bwd(const CeProblem& q, const void* X, const void* W, const int64_t* targets, const float* weight, const float* lse,
                   const float* loss, const float* denom, float scale, void* dX, void* dW, void* ws, int* status, cudaStream_t st) {
  const BwdPlan b = bwd_plan(q);
  uint8_t* w8 = static_cast<uint8_t*>(ws);
  const int64_t piece_cols = int64_t(b.piece_tiles) * ce::kTile;
  float* acc = reinterpret_cast<float*>(w8 + b.acc);
  float* corr = reinterpret_cast<float*>(w8 + b.corr);
  Params p{};
  common(q, &p, targets, weight, status);
  p.lse = lse;
  p.loss = loss;
  p.corr = corr;
  p.acc = acc;
  p.ld_d = piece_cols;
  const bool put_back = b.put_back && dW;
  int* row_key = reinterpret_cast<int*>(w8 + b.row_key);
  float* row_add = reinterpret_cast<float*>(w8 + b.row_add);
  if (put_back) {
    p.row_key = row_key;
    p.row_add = row_add;
  }
  p.denom = denom;
  p.scale = scale * q.logit_scale;
  p.acc_rows = b.acc_rows;
  p.kb_per_split = b.kb_per_split;
  p.token_kb = ceil_div(q.m, ce::kBK);
  p.d_tiles = b.d_tiles;
  p.d_width = b.d_width;
  CUtensorMap xk, wk, wmn, xmn, accm, dwm, dwn, dst[kBuffers], dk[kBuffers], dmn[kBuffers];
  const bool few = is_few(q);
  const int token_box = few ? p.few_n / 2 : ce::kBM;
  if (!make_tmap_bf16(&xk, X, q.m, q.d, ce::kBK, token_box) || !make_tmap_bf16(&wk, W, q.vocab, q.d, ce::kBK, ce::kBM) ||
      !make_tmap_bf16(&wmn, W, q.vocab, q.d, 64, ce::kBK) || !make_tmap_bf16(&xmn, X, q.m, q.d, 64, ce::kBK) ||
      !make_tmap_f32(&accm, acc, int64_t(b.splits) * b.acc_rows, q.d, 32, 16) || !make_tmap_bf16(&dwm, dW ? dW : X, dW ? q.vocab : q.m, q.d, 64, 16) ||
      !make_tmap_bf16_store_sw64(&dwn, dW ? dW : X, dW ? q.vocab : q.m, q.d))
    return cudaErrorInvalidValue;
  for (int k = 0; k < b.buffers; ++k) {
    void* D = w8 + b.D + k * b.D_stride;
    if (!make_tmap_bf16(&dst[k], D, q.m, piece_cols, 64, 16) || !make_tmap_bf16(&dk[k], D, q.m, piece_cols, ce::kBK, token_box) ||
        !make_tmap_bf16(&dmn[k], D, q.m, piece_cols, 64, ce::kBK))
      return cudaErrorInvalidValue;
  }
  const int n_tiles = ceil_div(q.vocab, ce::kTile);
  auto set_piece = [&](int piece) {
    p.v0 = piece * int(piece_cols);
    p.n_tiles = std::min(b.piece_tiles, n_tiles - piece * b.piece_tiles);
  };
  auto dlogits = [&](int piece) {
    set_piece(piece);
    const CUtensorMap& out = dst[piece % kBuffers];
    p.units = few ? p.n_tiles : p.m_tiles * p.n_tiles;
    p.D = reinterpret_cast<__nv_bfloat16*>(w8 + b.D + (piece % kBuffers) * b.D_stride);
    p.wait_first = piece == 0 || put_back || few;
    return launch<ce::DLOGITS>(few, xk, wk, xk, wk, out, out, out, p, st);
  };
  auto grads = [&](int piece) {
    set_piece(piece);
    p.first_piece = piece == 0;
    p.wait_first = piece + 1 == b.pieces || put_back || few;
    p.piece_kb = p.n_tiles * (ce::kTile / ce::kBK);
    // a last piece shorter than the others may leave the last splits without a k-block: those tiles are left out
    const int splits = std::min(b.splits, ceil_div(p.piece_kb, b.kb_per_split));
    p.x_units = dX ? splits * (few ? ceil_div(q.d, ce::kTile) : p.m_tiles * b.d_tiles) : 0;
    p.units = p.x_units + (dW ? p.n_tiles * b.d_tiles : 0);
    return launch<ce::GRADS>(few, dk[piece % kBuffers], wmn, dmn[piece % kBuffers], xmn, accm, dwm, dwn, p, st);
  };
  cudaError_t e = cudaSuccess;
  if (put_back) {   // up to 512 tokens: one piece as a rule; every launch needs the one before it
    for (int piece = 0; piece < b.pieces && e == cudaSuccess; ++piece) {
      e = dlogits(piece);
      if (e == cudaSuccess)
        e = launch_lined_up(ce_put_back_kernel, dim3(unsigned(q.m)), dim3(kPutBackTokens), 0, st, static_cast<const float*>(corr), targets,
                          static_cast<const __nv_bfloat16*>(X), p.tokens, p.d, p.v0, std::min(p.vocab, p.v0 + p.n_tiles * ce::kTile), row_key,
                          row_add);
      if (e == cudaSuccess) e = grads(piece);
    }
  } else {
    e = dlogits(0);
    for (int piece = 0; piece < b.pieces && e == cudaSuccess; ++piece) {
      if (piece + 1 < b.pieces) e = dlogits(piece + 1);
      if (e == cudaSuccess) e = grads(piece);
    }
  }
  if (e != cudaSuccess || !dX) return e;
  const int64_t threads = q.m * (q.d / 8);
  return launch_lined_up(ce_finish_kernel, dim3(unsigned((threads + 255) / 256)), dim3(256), 0, st, static_cast<const float*>(acc), b.splits,
                       int64_t(b.acc_rows) * q.d, static_cast<const float*>(corr), targets, static_cast<const __nv_bfloat16*>(W), denom,
                       p.scale, static_cast<__nv_bfloat16*>(dX), p.tokens, p.d, p.vocab);
}

}  // namespace acx
