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

using ce::Params;

constexpr int kTokensPerBlock = 32;

__device__ __forceinline__ float dot8(uint4 a, uint4 b, float s) {
  const uint32_t x[4] = {a.x, a.y, a.z, a.w}, w[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    s = fmaf(__uint_as_float(x[i] << 16), __uint_as_float(w[i] << 16), s);
    s = fmaf(__uint_as_float(x[i] & 0xFFFF0000u), __uint_as_float(w[i] & 0xFFFF0000u), s);
  }
  return s;
}

// Joins the (maximum, sum) pairs of 32 tokens: 32 warps, a token per lane, every warp takes each 32nd pair.  The target's
// logit is taken again as a plain fp32 product (a warp per token): the tensor core adds 16 products at a time with
// truncation, an error of up to 2^-24 of the logit per step and of one sign, which the loss of an unlikely token would
// show in full; its term of the sum is exchanged along with it.
__global__ void __launch_bounds__(1024) ce_join_kernel(const float2* __restrict__ part, const float* __restrict__ target_logit,
                                                       const __nv_bfloat16* __restrict__ X, const __nv_bfloat16* __restrict__ W,
                                                       const int64_t* __restrict__ targets, const float* __restrict__ weight, int tokens,
                                                       int d, int vocab, int parts, float c, float* __restrict__ loss,
                                                       float* __restrict__ lse, float2* __restrict__ block_sums) {
  __shared__ float2 red[32][33];
  __shared__ float exact[32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, t0 = int(blockIdx.x) * kTokensPerBlock;
  const int t = t0 + lane;
  float m = -INFINITY, s = 0.f;
  if (t < tokens) {
    for (int q = warp; q < parts; q += 8 * 32) {   // eight pairs in flight
      float2 v[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = q + 32 * i < parts ? __ldg(part + int64_t(q + 32 * i) * tokens + t) : make_float2(-INFINITY, 0.f);
      float top = m;
#pragma unroll
      for (int i = 0; i < 8; ++i) top = fmaxf(top, v[i].x);
      s *= exp2f(m - top);
      m = top;
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (q + 32 * i < parts) s += v[i].y * exp2f(v[i].x - m);
    }
  }
  red[warp][lane] = make_float2(m, s);
  {
    const int tt = t0 + warp;
    const int64_t y = tt < tokens ? __ldg(targets + tt) : -1;
    float p = 0.f;
    if (y >= 0 && y < vocab) {
      const uint4* x = reinterpret_cast<const uint4*>(X + int64_t(tt) * d);
      const uint4* w = reinterpret_cast<const uint4*>(W + y * int64_t(d));
      for (int i = lane; i < d / 8; i += 32) p = dot8(__ldg(x + i), __ldg(w + i), p);
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) p += __shfl_xor_sync(0xFFFFFFFFu, p, o);
    if (lane == 0) exact[warp] = p * c;
  }
  __syncthreads();
  if (warp != 0) return;
  float wl = 0.f, wt = 0.f;
  if (t < tokens) {
    m = -INFINITY;
    s = 0.f;
    for (int k = 0; k < 32; ++k) m = fmaxf(m, red[k][lane].x);
    for (int k = 0; k < 32; ++k)
      if (red[k][lane].x != -INFINITY || red[k][lane].y != 0.f) s += red[k][lane].y * exp2f(red[k][lane].x - m);
    const int64_t y = __ldg(targets + t);
    const bool trained = y >= 0 && y < vocab;
    const float ty = exact[lane];
    if (trained) s += exp2f(ty - m) - exp2f(target_logit[t] - m);
    const float l2 = m + log2f(s);
    constexpr float kLn2 = 0.6931471805599453f;
    lse[t] = l2 * kLn2;
    const float l = trained ? (l2 - ty) * kLn2 : 0.f;
    loss[t] = l;
    wt = trained ? (weight ? __ldg(weight + t) : 1.f) : 0.f;
    wl = trained ? wt * l : 0.f;
  }
  if (!block_sums) return;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    wl += __shfl_xor_sync(0xFFFFFFFFu, wl, o);
    wt += __shfl_xor_sync(0xFFFFFFFFu, wt, o);
  }
  if (lane == 0) block_sums[blockIdx.x] = make_float2(wl, wt);
}

// total = (sum of w loss, sum of w): the blocks' sums in a fixed order.
__global__ void __launch_bounds__(1024) ce_total_kernel(const float2* __restrict__ block_sums, int n, float* __restrict__ total) {
  __shared__ float2 red[32];
  float a = 0.f, b = 0.f;
  for (int i = threadIdx.x; i < n; i += 1024) {
    const float2 v = block_sums[i];
    a += v.x;
    b += v.y;
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    a += __shfl_xor_sync(0xFFFFFFFFu, a, o);
    b += __shfl_xor_sync(0xFFFFFFFFu, b, o);
  }
  if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = make_float2(a, b);
  __syncthreads();
  if (threadIdx.x >= 32) return;
  a = red[threadIdx.x].x;
  b = red[threadIdx.x].y;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    a += __shfl_xor_sync(0xFFFFFFFFu, a, o);
    b += __shfl_xor_sync(0xFFFFFFFFu, b, o);
  }
  if (threadIdx.x == 0) {
    total[0] = a;
    total[1] = b;
  }
}

// dX = f (sum over the splits + corr W[y]): what rounding D to bf16 took from the target's element, the largest of its row
// and the only one whose rounding is not averaged out, comes back here in fp32.
__global__ void __launch_bounds__(256) ce_finish_kernel(const float* __restrict__ acc, int splits, int64_t split_stride,
                                                        const float* __restrict__ corr, const int64_t* __restrict__ targets,
                                                        const __nv_bfloat16* __restrict__ W, const float* __restrict__ denom, float scale,
                                                        __nv_bfloat16* __restrict__ dX, int tokens, int d, int vocab) {
  const int vecs = d / 8;
  const int64_t i = int64_t(blockIdx.x) * 256 + threadIdx.x;
  const int64_t t = i / vecs;
  if (t >= tokens) return;
  const int c = int(i - t * vecs) * 8;
  const float dn = denom ? __ldg(denom) : 1.f, f = dn > 0.f ? scale / dn : 0.f;
  float v[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = 0.f;
  for (int s = 0; s < splits; ++s) {
    const float4* p = reinterpret_cast<const float4*>(acc + s * split_stride + t * d + c);
    const float4 a = __ldg(p), b = __ldg(p + 1);
    v[0] += a.x; v[1] += a.y; v[2] += a.z; v[3] += a.w;
    v[4] += b.x; v[5] += b.y; v[6] += b.z; v[7] += b.w;
  }
  const int64_t y = __ldg(targets + t);
  if (y >= 0 && y < vocab) {
    const float k = __ldg(corr + t);
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

int ceil_div(int64_t a, int64_t b) { return int((a + b - 1) / b); }
size_t aligned(size_t bytes) { return (bytes + 1023) & ~size_t(1023); }

int pair_count() { return std::max(1, sm_count() / 2); }

template <int KIND>
cudaError_t launch(const CUtensorMap& ta, const CUtensorMap& tb, const CUtensorMap& ta2, const CUtensorMap& tb2, const CUtensorMap& to,
                   const CUtensorMap& to2, const Params& p, cudaStream_t st) {
  auto kernel = ce::ce_kernel<KIND>;
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
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = 2;
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  const cudaError_t e = cudaLaunchKernelEx(&cfg, kernel, ta, tb, ta2, tb2, to, to2, p);
  kernel_launch_counter().fetch_add(1, std::memory_order_relaxed);
  return e;
}

// Token tiles that pass over the vocabulary together: as many as have their rows of X (d wide, bf16) in 48 MB, so that X
// stays in L2 beside the tiles of W that stream by.
int token_group(int64_t d, int m_tiles) {
  const int fit = int(std::max<int64_t>(1, (int64_t(48) << 20) / (ce::kTile * d * 2)));
  const int groups = ceil_div(m_tiles, fit);
  return ceil_div(m_tiles, groups);
}

void common(const CeProblem& q, Params* p, const int64_t* targets, const float* weight, int* status) {
  p->tokens = int(q.m);
  p->d = int(q.d);
  p->vocab = int(q.vocab);
  p->m_tiles = ceil_div(q.m, ce::kTile);
  p->group = token_group(q.d, p->m_tiles);
  p->c = q.logit_scale * ce::kLog2e;
  p->targets = targets;
  p->weight = weight;
  p->status = status;
}

struct FwdPlan {
  int parts, blocks;
  size_t part, target, sums, bytes;
};
FwdPlan fwd_plan(const CeProblem& q) {
  FwdPlan f;
  f.parts = ceil_div(q.vocab, 128);
  f.blocks = ceil_div(q.m, kTokensPerBlock);
  f.part = 0;
  f.target = f.part + aligned(size_t(f.parts) * size_t(q.m) * sizeof(float2));
  f.sums = f.target + aligned(size_t(q.m) * 4);
  f.bytes = f.sums + aligned(size_t(f.blocks) * sizeof(float2));
  return f;
}

// Pieces of the vocabulary: D of one piece takes at most about 128 MB, so that much of it is still in L2 when the two
// products read it, and the pieces are of equal size.
struct BwdPlan {
  int piece_tiles, pieces, splits, kb_per_split, d_tiles, acc_rows;
  size_t D, acc, corr, bytes;
};
BwdPlan bwd_plan(const CeProblem& q) {
  BwdPlan b;
  const int n_tiles = ceil_div(q.vocab, ce::kTile), m_tiles = ceil_div(q.m, ce::kTile);
  const int fit = int(std::max<int64_t>(1, (int64_t(128) << 20) / (q.m * ce::kTile * 2)));
  b.pieces = ceil_div(n_tiles, fit);
  b.piece_tiles = ceil_div(n_tiles, b.pieces);
  b.pieces = ceil_div(n_tiles, b.piece_tiles);
  b.d_tiles = ceil_div(q.d, ce::kTile);
  b.acc_rows = m_tiles * ce::kTile;
  // dX: few tiles are split along the piece until there are about two per CTA pair (at least 8 k-blocks each)
  const int piece_kb = b.piece_tiles * (ce::kTile / ce::kBK), units = m_tiles * b.d_tiles, want = 2 * pair_count();
  const int splits = std::max(1, std::min({units >= want ? 1 : want / units, piece_kb / 8, 32}));
  b.kb_per_split = ceil_div(piece_kb, splits);
  b.splits = ceil_div(piece_kb, b.kb_per_split);
  b.D = 0;
  b.acc = b.D + aligned(size_t(q.m) * size_t(b.piece_tiles) * ce::kTile * 2);
  b.corr = b.acc + aligned(size_t(b.splits) * size_t(b.acc_rows) * size_t(q.d) * 4);
  b.bytes = b.corr + aligned(size_t(q.m) * 4);
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
  p.units = p.m_tiles * p.n_tiles;
  p.part = reinterpret_cast<float2*>(w8 + f.part);
  p.target_logit = reinterpret_cast<float*>(w8 + f.target);
  CUtensorMap ta, tb;
  if (!make_tmap_bf16(&ta, X, q.m, q.d, ce::kBK, ce::kBM) || !make_tmap_bf16(&tb, W, q.vocab, q.d, ce::kBK, ce::kBM)) return cudaErrorInvalidValue;
  cudaError_t e = launch<ce::LSE>(ta, tb, ta, tb, ta, ta, p, st);
  if (e != cudaSuccess) return e;
  float2* sums = total ? reinterpret_cast<float2*>(w8 + f.sums) : nullptr;
  ce_join_kernel<<<f.blocks, 1024, 0, st>>>(p.part, p.target_logit, static_cast<const __nv_bfloat16*>(X), static_cast<const __nv_bfloat16*>(W),
                                            targets, weight, p.tokens, p.d, p.vocab, f.parts, p.c, loss, lse, sums);
  e = launched();
  if (e != cudaSuccess || !total) return e;
  ce_total_kernel<<<1, 1024, 0, st>>>(sums, f.blocks, total);
  return launched();
}

cudaError_t ce_bwd(const CeProblem& q, const void* X, const void* W, const int64_t* targets, const float* weight, const float* lse,
                   const float* denom, float scale, void* dX, void* dW, void* ws, int* status, cudaStream_t st) {
  const BwdPlan b = bwd_plan(q);
  uint8_t* w8 = static_cast<uint8_t*>(ws);
  const int64_t piece_cols = int64_t(b.piece_tiles) * ce::kTile;
  void* D = w8 + b.D;
  float* acc = reinterpret_cast<float*>(w8 + b.acc);
  float* corr = reinterpret_cast<float*>(w8 + b.corr);
  Params p{};
  common(q, &p, targets, weight, status);
  p.lse = lse;
  p.corr = corr;
  p.denom = denom;
  p.scale = scale * q.logit_scale;
  p.acc_rows = b.acc_rows;
  p.splits = b.splits;
  p.kb_per_split = b.kb_per_split;
  p.token_kb = ceil_div(q.m, ce::kBK);
  p.d_tiles = b.d_tiles;
  CUtensorMap xk, wk, dst, dk, dmn, wmn, xmn, accm, dwm;
  if (!make_tmap_bf16(&xk, X, q.m, q.d, ce::kBK, ce::kBM) || !make_tmap_bf16(&wk, W, q.vocab, q.d, ce::kBK, ce::kBM) ||
      !make_tmap_bf16_store_sw64(&dst, D, q.m, piece_cols) || !make_tmap_bf16(&dk, D, q.m, piece_cols, ce::kBK, ce::kBM) ||
      !make_tmap_bf16(&dmn, D, q.m, piece_cols, 64, ce::kBK) || !make_tmap_bf16(&wmn, W, q.vocab, q.d, 64, ce::kBK) ||
      !make_tmap_bf16(&xmn, X, q.m, q.d, 64, ce::kBK) ||
      !make_tmap_2d(&accm, CU_TENSOR_MAP_DATA_TYPE_FLOAT32, 4, acc, int64_t(b.splits) * b.acc_rows, q.d, 16, 32, CU_TENSOR_MAP_SWIZZLE_64B) ||
      !make_tmap_bf16_store_sw64(&dwm, dW ? dW : D, q.vocab, q.d))
    return cudaErrorInvalidValue;
  const int n_tiles = ceil_div(q.vocab, ce::kTile);
  for (int piece = 0; piece < b.pieces; ++piece) {
    const int tiles = std::min(b.piece_tiles, n_tiles - piece * b.piece_tiles);
    p.v0 = piece * int(piece_cols);
    p.first_piece = piece == 0;
    p.n_tiles = tiles;
    p.units = p.m_tiles * tiles;
    cudaError_t e = launch<ce::DLOGITS>(xk, wk, xk, wk, dst, dst, p, st);
    if (e != cudaSuccess) return e;
    p.piece_kb = tiles * (ce::kTile / ce::kBK);
    // a last piece shorter than the others may leave the last splits without a k-block: those tiles are left out
    const int splits = std::min(b.splits, ceil_div(p.piece_kb, b.kb_per_split));
    p.x_units = dX ? splits * p.m_tiles * b.d_tiles : 0;
    p.units = p.x_units + (dW ? tiles * b.d_tiles : 0);
    e = launch<ce::GRADS>(dk, wmn, dmn, xmn, accm, dwm, p, st);
    if (e != cudaSuccess) return e;
  }
  if (!dX) return cudaSuccess;
  const int64_t threads = q.m * (q.d / 8);
  ce_finish_kernel<<<unsigned((threads + 255) / 256), 256, 0, st>>>(acc, b.splits, int64_t(b.acc_rows) * q.d, corr, targets,
                                                                   static_cast<const __nv_bfloat16*>(W), denom, p.scale,
                                                                   static_cast<__nv_bfloat16*>(dX), p.tokens, p.d, p.vocab);
  return launched();
}

}  // namespace acx
