// C ABI of attention, the embedding table and gradient clipping: argument checks and dispatch.
#include <algorithm>
#include <cmath>
#include <exception>
#include <vector>

#include "acx_checks.h"
#include "acx_internal.h"

namespace acx {
namespace {

acx_status validate_attn(const acx_attn_desc* d, AttnProblem* out) {
  if (!d || d->struct_size != sizeof(acx_attn_desc)) return ACX_ERR_INVALID_ARG;
  if (d->io_dtype != ACX_BF16 || (d->causal != 0 && d->causal != 1)) return ACX_ERR_INVALID_ARG;
  if (!(d->scale > 0.f) || !std::isfinite(d->scale) || !(d->softcap >= 0.f) || !std::isfinite(d->softcap)) return ACX_ERR_INVALID_ARG;
  // what the kernels take of them stays well inside fp32: scale log2(e), softcap log2(e), 2^7 scale / softcap, scale times a gradient
  constexpr double kMost = 0x1p104;
  if (d->scale > kMost || d->softcap > kMost || (d->softcap > 0.f && d->scale > kMost * d->softcap)) return ACX_ERR_INVALID_ARG;
  if (d->tokens < 0 || d->tokens > (int64_t(1) << 24) || d->docs < 1 || d->docs > (int64_t(1) << 24)) return ACX_ERR_UNSUPPORTED_SHAPE;
  if (d->heads < 1 || d->heads > 4096 || d->kv_heads < 1 || d->heads % d->kv_heads) return ACX_ERR_UNSUPPORTED_SHAPE;
  if (d->head_dim < 8 || d->head_dim > 128 || d->head_dim % 8) return ACX_ERR_UNSUPPORTED_SHAPE;
  // work items are numbered in 32 bits
  const int64_t tiles = d->tokens / 128 + (d->docs < d->tokens ? d->docs : d->tokens) + 1;
  if (tiles * d->heads > (int64_t(1) << 30)) return ACX_ERR_UNSUPPORTED_SHAPE;
  out->tokens = d->tokens;
  out->docs = d->docs;
  out->heads = d->heads;
  out->kv_heads = d->kv_heads;
  out->d = d->head_dim;
  out->causal = d->causal;
  out->scale = d->scale;
  out->softcap = d->softcap;
  return ACX_OK;
}
bool bad_heads_stride(const AttnProblem& q, int64_t ld, int heads) {
  return ld < int64_t(heads) * q.d || ld % 8 || ld > (int64_t(1) << 38);
}
AttnMatrix matrix(const void* p, int64_t ld) { return AttnMatrix{const_cast<void*>(p), ld}; }

acx_status validate_embed(const acx_embed_desc* d, EmbedProblem* out) {
  if (!d || d->struct_size != sizeof(acx_embed_desc)) return ACX_ERR_INVALID_ARG;
  if ((d->io_dtype != ACX_F32 && d->io_dtype != ACX_BF16) || (d->grad_dtype != ACX_F32 && d->grad_dtype != ACX_BF16)) return ACX_ERR_INVALID_ARG;
  if (!std::isfinite(d->scale)) return ACX_ERR_INVALID_ARG;
  if (d->tokens < 0 || d->tokens > (int64_t(1) << 28)) return ACX_ERR_UNSUPPORTED_SHAPE;
  if (d->d < 8 || d->d % 8 || d->d > (int64_t(1) << 16) || d->vocab < 1 || d->vocab > (int64_t(1) << 22)) return ACX_ERR_UNSUPPORTED_SHAPE;
  out->tokens = d->tokens;
  out->d = d->d;
  out->vocab = d->vocab;
  out->bf16 = d->io_dtype == ACX_BF16;
  out->grad_bf16 = d->grad_dtype == ACX_BF16;
  out->scale = d->scale;
  return ACX_OK;
}

// Whether a tensor that is written shares memory with another one, or with its own source other than in place: blocks work on the
// tensors in any order.
bool outputs_overlap(const acx_grad* list, int64_t count) {
  struct Range { uintptr_t begin, end; bool written; };
  std::vector<Range> ranges;
  ranges.reserve(size_t(2 * count));
  for (int64_t i = 0; i < count; ++i) {
    const acx_grad& g = list[i];
    if (g.n == 0) continue;
    const uintptr_t src = reinterpret_cast<uintptr_t>(g.src), dst = reinterpret_cast<uintptr_t>(g.dst);
    ranges.push_back(Range{dst, dst + uintptr_t(g.n) * (g.dst_dtype == ACX_BF16 ? 2 : 4), true});
    if (src != dst) ranges.push_back(Range{src, src + uintptr_t(g.n) * (g.src_dtype == ACX_BF16 ? 2 : 4), false});
  }
  std::sort(ranges.begin(), ranges.end(), [](const Range& a, const Range& b) { return a.begin < b.begin; });
  uintptr_t written_to = 0, read_to = 0;   // ends of the ranges so far
  for (const Range& r : ranges) {
    if (r.begin < written_to || (r.written && r.begin < read_to)) return true;
    uintptr_t& to = r.written ? written_to : read_to;
    to = std::max(to, r.end);
  }
  return false;
}

acx_status validate_grad(const acx_grad_desc* d, GradProblem* out) {
  if (!d || d->struct_size != sizeof(acx_grad_desc) || d->reserved != 0) return ACX_ERR_INVALID_ARG;
  if (d->tensors < 0 || d->tensors > (int64_t(1) << 24) || d->chunks < 0 || d->chunks > (int64_t(1) << 31)) return ACX_ERR_UNSUPPORTED_SHAPE;
  if (d->tensors == 0 && d->chunks > 0) return ACX_ERR_INVALID_ARG;   // no list's: a plan is asked for only where there are tensors
  out->tensors = d->tensors;
  out->chunks = d->chunks;
  return ACX_OK;
}

}  // namespace
}  // namespace acx

using namespace acx;

extern "C" {

// ---- attention -------------------------------------------------------------------------------------------------------
size_t acx_attn_workspace_bytes(const acx_attn_desc* desc, int op) {
  AttnProblem q;
  if (validate_attn(desc, &q) != ACX_OK) return 0;
  if (op == ACX_OP_ATTN_PLAN) return attn_plan_bytes(q);
  if (op == ACX_OP_ATTN_BWD) return q.tokens == 0 ? 0 : attn_bwd_workspace_bytes(q);
  return 0;
}

acx_status acx_attn_plan(const acx_attn_desc* desc, const int32_t* offsets, const int32_t* prefix, void* plan, size_t plan_bytes, void* cuda_stream) {
  AttnProblem q;
  const acx_status s = validate_attn(desc, &q);
  if (s != ACX_OK) return s;
  if (!offsets || (prefix && !q.causal)) return ACX_ERR_INVALID_ARG;
  if ((reinterpret_cast<uintptr_t>(offsets) & 3u) || (reinterpret_cast<uintptr_t>(prefix) & 3u) || misaligned(plan)) return ACX_ERR_ALIGNMENT;
  if (!plan || plan_bytes < attn_plan_bytes(q)) return ACX_ERR_WORKSPACE;
  return from_cuda(attn_plan(q, offsets, prefix, plan, static_cast<cudaStream_t>(cuda_stream)));
}

acx_status acx_attn_fwd(const acx_attn_desc* desc, const void* Q, int64_t ldq, const void* K, int64_t ldk, const void* V, int64_t ldv,
                        const float* slopes, const void* plan, size_t plan_bytes, void* O, int64_t ldo, float* lse, void* cuda_stream) {
  AttnProblem q;
  const acx_status s = validate_attn(desc, &q);
  if (s != ACX_OK) return s;
  if (bad_heads_stride(q, ldq, q.heads) || bad_heads_stride(q, ldk, q.kv_heads) || bad_heads_stride(q, ldv, q.kv_heads) ||
      bad_heads_stride(q, ldo, q.heads))
    return ACX_ERR_UNSUPPORTED_SHAPE;
  if (q.tokens == 0) return ACX_OK;
  if (any_null(Q, K, V, O)) return ACX_ERR_INVALID_ARG;
  if (any_misaligned(Q, K, V, O, plan, lse) || (reinterpret_cast<uintptr_t>(slopes) & 3u)) return ACX_ERR_ALIGNMENT;
  if (!plan || plan_bytes < attn_plan_bytes(q)) return ACX_ERR_WORKSPACE;
  int* status = device_status_ptr();
  if (!status) return ACX_ERR_CUDA;
  return from_cuda(attn_fwd(q, matrix(Q, ldq), matrix(K, ldk), matrix(V, ldv), slopes, plan, matrix(O, ldo), lse, status,
                            static_cast<cudaStream_t>(cuda_stream)));
}

acx_status acx_attn_bwd(const acx_attn_desc* desc, const void* Q, int64_t ldq, const void* K, int64_t ldk, const void* V, int64_t ldv,
                        const float* slopes, const void* plan, size_t plan_bytes, const void* O, int64_t ldo, const void* dO, int64_t lddo,
                        const float* lse, void* dQ, int64_t lddq, void* dK, int64_t lddk, void* dV, int64_t lddv, void* ws, size_t ws_bytes,
                        void* cuda_stream) {
  AttnProblem q;
  const acx_status s = validate_attn(desc, &q);
  if (s != ACX_OK) return s;
  for (int64_t ld : {ldq, ldo, lddo, lddq})
    if (bad_heads_stride(q, ld, q.heads)) return ACX_ERR_UNSUPPORTED_SHAPE;
  for (int64_t ld : {ldk, ldv, lddk, lddv})
    if (bad_heads_stride(q, ld, q.kv_heads)) return ACX_ERR_UNSUPPORTED_SHAPE;
  if (q.tokens == 0) return ACX_OK;
  if (any_null(Q, K, V, O, dO, lse, dQ, dK, dV)) return ACX_ERR_INVALID_ARG;
  if (any_misaligned(Q, K, V, O, dO, lse, dQ, dK, dV, plan, ws) || (reinterpret_cast<uintptr_t>(slopes) & 3u)) return ACX_ERR_ALIGNMENT;
  if (!plan || plan_bytes < attn_plan_bytes(q) || !ws || ws_bytes < attn_bwd_workspace_bytes(q)) return ACX_ERR_WORKSPACE;
  int* status = device_status_ptr();
  if (!status) return ACX_ERR_CUDA;
  return from_cuda(attn_bwd(q, matrix(Q, ldq), matrix(K, ldk), matrix(V, ldv), slopes, plan, matrix(O, ldo), matrix(dO, lddo), lse,
                            matrix(dQ, lddq), matrix(dK, lddk), matrix(dV, lddv), ws, status, static_cast<cudaStream_t>(cuda_stream)));
}

// ---- embedding table -------------------------------------------------------------------------------------------------
size_t acx_embed_workspace_bytes(const acx_embed_desc* desc, int op) {
  EmbedProblem q;
  if (op != ACX_OP_EMBED_BWD || validate_embed(desc, &q) != ACX_OK || q.tokens == 0) return 0;
  return embed_bwd_workspace_bytes(q);
}

acx_status acx_embed_fwd(const acx_embed_desc* desc, const int64_t* ids, const void* E, void* Y, void* cuda_stream) {
  EmbedProblem q;
  const acx_status s = validate_embed(desc, &q);
  if (s != ACX_OK) return s;
  if (q.tokens == 0) return ACX_OK;
  if (any_null(ids, E, Y)) return ACX_ERR_INVALID_ARG;
  if (any_misaligned(E, Y) || (reinterpret_cast<uintptr_t>(ids) & 7u)) return ACX_ERR_ALIGNMENT;
  return from_cuda(embed_fwd(q, ids, E, Y, static_cast<cudaStream_t>(cuda_stream)));
}

acx_status acx_embed_bwd(const acx_embed_desc* desc, const int64_t* ids, const void* dY, void* dE, float beta, void* ws, size_t ws_bytes,
                         void* cuda_stream) {
  EmbedProblem q;
  const acx_status s = validate_embed(desc, &q);
  if (s != ACX_OK) return s;
  if (!std::isfinite(beta) || !dE) return ACX_ERR_INVALID_ARG;
  if (q.tokens > 0 && any_null(ids, dY)) return ACX_ERR_INVALID_ARG;
  if (any_misaligned(dY, dE, ws) || (reinterpret_cast<uintptr_t>(ids) & 7u)) return ACX_ERR_ALIGNMENT;
  if (q.tokens > 0 && (!ws || ws_bytes < embed_bwd_workspace_bytes(q))) return ACX_ERR_WORKSPACE;
  return from_cuda(embed_bwd(q, ids, dY, dE, beta, ws, static_cast<cudaStream_t>(cuda_stream)));
}

// ---- gradient norm and clipping --------------------------------------------------------------------------------------
acx_status acx_grad_describe(const acx_grad* list, int64_t count, acx_grad_desc* desc) {
  if (!desc || count < 0 || (count > 0 && !list)) return ACX_ERR_INVALID_ARG;
  if (count > (int64_t(1) << 24)) return ACX_ERR_UNSUPPORTED_SHAPE;
  int64_t chunks = 0;
  for (int64_t i = 0; i < count; ++i) {
    const acx_grad& g = list[i];
    if ((g.src_dtype != ACX_F32 && g.src_dtype != ACX_BF16) || (g.dst_dtype != ACX_F32 && g.dst_dtype != ACX_BF16)) return ACX_ERR_INVALID_ARG;
    if (!(g.weight >= 0.f) || !std::isfinite(g.weight)) return ACX_ERR_INVALID_ARG;
    if (g.n < 0 || g.n > (int64_t(1) << 40)) return ACX_ERR_UNSUPPORTED_SHAPE;
    if (g.n == 0) continue;
    if (any_null(g.src, g.dst) || (g.src == g.dst && g.src_dtype != g.dst_dtype)) return ACX_ERR_INVALID_ARG;
    if (any_misaligned(g.src, g.dst)) return ACX_ERR_ALIGNMENT;
    chunks += (g.n + kGradChunk - 1) / kGradChunk;
  }
  if (chunks > (int64_t(1) << 31)) return ACX_ERR_UNSUPPORTED_SHAPE;
  try {
    if (outputs_overlap(list, count)) return ACX_ERR_INVALID_ARG;
  } catch (const std::exception&) {   // no memory on the host for the ranges
    return ACX_ERR_CUDA;
  }
  desc->struct_size = sizeof(acx_grad_desc);
  desc->reserved = 0;
  desc->tensors = count;
  desc->chunks = chunks;
  return ACX_OK;
}

size_t acx_grad_workspace_bytes(const acx_grad_desc* desc, int op) {
  GradProblem q;
  if (validate_grad(desc, &q) != ACX_OK) return 0;
  if (op == ACX_OP_GRAD_PLAN) return grad_plan_bytes(q);
  if (op == ACX_OP_GRAD_CLIP) return grad_clip_workspace_bytes(q);
  return 0;
}

acx_status acx_grad_plan(const acx_grad_desc* desc, const acx_grad* list, void* plan, size_t plan_bytes, void* cuda_stream) {
  GradProblem q;
  const acx_status s = validate_grad(desc, &q);
  if (s != ACX_OK) return s;
  acx_grad_desc same;
  const acx_status l = acx_grad_describe(list, q.tensors, &same);
  if (l != ACX_OK) return l;
  if (same.chunks != q.chunks) return ACX_ERR_INVALID_ARG;
  if (q.tensors == 0) return ACX_OK;
  if (misaligned(plan)) return ACX_ERR_ALIGNMENT;
  if (!plan || plan_bytes < grad_plan_bytes(q)) return ACX_ERR_WORKSPACE;
  return from_cuda(grad_plan(q, list, plan, static_cast<cudaStream_t>(cuda_stream)));
}

acx_status acx_grad_clip(const acx_grad_desc* desc, const void* plan, size_t plan_bytes, float max_norm, float* total, void* ws, size_t ws_bytes,
                         void* cuda_stream) {
  GradProblem q;
  const acx_status s = validate_grad(desc, &q);
  if (s != ACX_OK) return s;
  if (!(max_norm > 0.f) || !total) return ACX_ERR_INVALID_ARG;
  if (misaligned(plan) || misaligned(ws) || (reinterpret_cast<uintptr_t>(total) & 3u)) return ACX_ERR_ALIGNMENT;
  if ((q.tensors > 0 && (!plan || plan_bytes < grad_plan_bytes(q))) || !ws || ws_bytes < grad_clip_workspace_bytes(q)) return ACX_ERR_WORKSPACE;
  return from_cuda(grad_clip(q, plan, max_norm, total, ws, static_cast<cudaStream_t>(cuda_stream)));
}

}  // extern "C"
