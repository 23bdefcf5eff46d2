// Internal interface between the sequence operators' C ABI (sequence_api.hip) and
// their gfx950 kernels.  The argument structures are those of winograd_crt.h,
// checked by the caller; D is the storage dtype (0 fp32, 1 fp16, 2 bf16).
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "winograd_crt.h"

namespace wg {

template <int D> hipError_t launch_gated_scan_t(const wg_gated_scan& a, hipStream_t stream);
template <int D> hipError_t launch_gated_scan_backward_t(const wg_gated_scan_backward& a, hipStream_t stream);
template <int D> hipError_t launch_gated_step_t(const wg_gated_step& a, hipStream_t stream);
size_t gated_scan_workspace(int dtype, int64_t N, int64_t L, int64_t C, bool backward);

template <int D> hipError_t launch_rms_norm_t(const wg_rms_norm& a, hipStream_t stream);
template <int D> hipError_t launch_rms_norm_backward_t(const wg_rms_norm_backward& a, hipStream_t stream);
size_t rms_norm_workspace(int dtype, int64_t N, int64_t L, int64_t C);

hipError_t launch_matvec_w4(const wg_matvec_w4& a, hipStream_t stream);
template <int D> hipError_t launch_quantize_w4_t(const wg_w4& w, const void* m, int64_t ldm, hipStream_t stream);
template <int D> hipError_t launch_dequantize_w4_t(const wg_w4& w, void* m, int64_t ldm, hipStream_t stream);
hipError_t launch_pack_w4(const wg_w4& w, const void* nibbles, const void* scales, hipStream_t stream);

template <int D> hipError_t launch_linear_attention_t(const wg_linear_attention& a, hipStream_t stream);
template <int D> hipError_t launch_linear_attention_backward_t(const wg_linear_attention_backward& a, hipStream_t stream);
template <int D> hipError_t launch_linear_attention_step_t(const wg_linear_attention_step& a, hipStream_t stream);
size_t linear_attention_workspace(int dtype, int64_t N, int64_t L, int64_t q_heads, int64_t k_heads, int64_t v_heads, int64_t H,
                                  int64_t Dk, int64_t Dv, bool backward);

template <int D> hipError_t launch_head_norm_rotate_t(const wg_head_norm_rotate& a, hipStream_t stream);
template <int D> hipError_t launch_head_norm_rotate_backward_t(const wg_head_norm_rotate_backward& a, hipStream_t stream);
size_t head_norm_rotate_workspace(int dtype, int64_t N, int64_t L, int64_t heads, int64_t D, int64_t R, bool adjacent);

}  // namespace wg
