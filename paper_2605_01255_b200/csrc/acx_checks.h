// What the C ABI's argument checks share.
#pragma once
#include <cuda_runtime.h>
#include <cstdint>

#include "../../include/acx.h"

namespace acx {

inline bool misaligned(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) != 0; }
template <typename... P>
bool any_misaligned(const P*... p) { return (misaligned(p) || ...); }
template <typename... P>
bool any_null(const P*... p) { return ((p == nullptr) || ...); }

inline acx_status from_cuda(cudaError_t e) { return e == cudaSuccess ? ACX_OK : ACX_ERR_CUDA; }

}  // namespace acx
