// C ABI of the sequence operators (declared in winograd_crt.h): argument checks,
// then one call into the kernels' launchers.  No C++ exception leaves this file;
// every failure becomes a wg_status plus a thread-local message, before anything
// is launched.
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>
#include <exception>
#include <string>
#include <utility>

#include "kernels.hpp"
#include "sequence.hpp"
#include "status.hpp"
#include "winograd_crt.h"

using wg::fail;
using wg::from_hip;

namespace {

constexpr int64_t kMaxSize = int64_t(1) << 31;      // sizes are below this
constexpr int64_t kMaxElements = int64_t(1) << 40;  // and the rows of one tensor together hold at most this
constexpr int64_t kMaxReach = int64_t(1) << 58;     // elements between a tensor's first and last row

template <typename F>
wg_status guarded(F&& f) noexcept {
    try {
        return f();
    } catch (...) {
        return WG_ERR_INTERNAL;   // only building a message can throw here
    }
}

bool aligned(const void* p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

bool storage(int64_t dtype) { return dtype == WG_F32 || dtype == WG_F16 || dtype == WG_BF16; }

wg_status check_sizes(int64_t N, int64_t L, int64_t C, int64_t least_n, int64_t least_l) {
    if (N < least_n || L < least_l || C < 1 || N >= kMaxSize || L >= kMaxSize || C >= kMaxSize)
        return fail(WG_ERR_ARG, "sizes must be in range and below 2^31");
    if (N > 0 && L > 0 && (C < 8 ? 8 : C) > kMaxElements / L / N)
        return fail(WG_ERR_UNSUPPORTED, "the tensors are too large");
    return WG_OK;
}

// Rows [N][L][C] of elements of es bytes; `written`: they must not overlap.
wg_status check_rows(const wg_rows& r, const char* name, int64_t N, int64_t L, int64_t C, int64_t es, bool written) {
    if (N == 0 || L == 0) return WG_OK;   // no row is touched
    if (!r.data) return fail(WG_ERR_ARG, std::string("null tensor ") + name);
    if (!aligned(r.data, static_cast<uintptr_t>(es)))
        return fail(WG_ERR_ARG, std::string(name) + " is not aligned to its elements");
    if (r.stride_n < 0 || r.stride_l < 0 || r.stride_n > kMaxReach / N || r.stride_l > kMaxReach / L)
        return fail(WG_ERR_ARG, std::string(name) + ": strides out of range");
    if (!written) return WG_OK;
    // the two strides in ascending order: the smaller spaces the rows, the larger the runs of them
    int64_t a = r.stride_l, an = L, b = r.stride_n, bn = N;
    if (L == 1) a = C;
    if (N == 1) b = kMaxReach;
    if (a > b) {
        std::swap(a, b);
        std::swap(an, bn);
    }
    if (a < C || (bn > 1 && b < (an - 1) * a + C)) return fail(WG_ERR_ARG, std::string("rows of ") + name + " overlap");
    return WG_OK;
}

// Channels of a row that is normalised: workgroups of the gradients' sums count them.
wg_status check_row(int64_t C) {
    return C <= (int64_t(1) << 25) ? WG_OK : fail(WG_ERR_UNSUPPORTED, "rows of more than 2^25 channels");
}

// Steps and channels of a scan: the kernels count them in 32 bits, past the end too.
wg_status check_steps(int64_t L, int64_t C) {
    if (L > 0x7fff0000) return fail(WG_ERR_UNSUPPORTED, "more than 2^31 - 2^16 steps");
    return C <= (int64_t(1) << 30) ? WG_OK : fail(WG_ERR_UNSUPPORTED, "more than 2^30 channels");
}

wg_status check_f32(const void* p, const char* name, bool optional = true) {
    if (!p) return optional ? WG_OK : fail(WG_ERR_ARG, std::string("null pointer ") + name);
    if (!aligned(p, 4)) return fail(WG_ERR_ARG, std::string(name) + " is not 4-byte aligned");
    return WG_OK;
}

wg_status check_workspace(const void* ws, int64_t bytes, size_t need) {
    if (need == 0) return WG_OK;
    if (!ws || bytes < 0 || static_cast<size_t>(bytes) < need)
        return fail(WG_ERR_WORKSPACE, "workspace too small: need " + std::to_string(need) + " bytes");
    if (!aligned(ws, 16)) return fail(WG_ERR_ARG, "the workspace is not 16-byte aligned");
    return WG_OK;
}

wg_status check_w4(const wg_w4& w) {
    if (!w.codes || !w.scales) return fail(WG_ERR_ARG, "null codes or scales");
    if (!aligned(w.codes, 16) || !aligned(w.scales, 16)) return fail(WG_ERR_ARG, "codes and scales must be 16-byte aligned");
    if (w.rows < 1 || w.cols < 1 || w.rows >= kMaxSize || w.cols >= kMaxSize)
        return fail(WG_ERR_ARG, "rows and cols must be in [1, 2^31)");
    if (w.group != 32 && w.group != 64 && w.group != 128) return fail(WG_ERR_UNSUPPORTED, "group must be 32, 64 or 128");
    if ((w.rows + 15) / 16 > kMaxElements / ((w.cols + 127) / 128 * 2048))
        return fail(WG_ERR_UNSUPPORTED, "the matrix is too large");
    return WG_OK;
}

#define WG_TRY(e) do { const wg_status s_ = (e); if (s_ != WG_OK) return s_; } while (0)
#define WG_BY_DTYPE(dtype, call)                                      \
    ((dtype) == WG_F32 ? call<0> : (dtype) == WG_F16 ? call<1> : call<2>)

}  // namespace

extern "C" {

wg_status winograd_gated_scan_workspace(wg_dtype dtype, int64_t N, int64_t L, int64_t C, int backward, size_t* bytes) {
    return guarded([&]() -> wg_status {
        if (!bytes) return fail(WG_ERR_ARG, "null argument");
        if (!storage(dtype)) return fail(WG_ERR_UNSUPPORTED, "unknown dtype");
        WG_TRY(check_sizes(N, L, C, 1, 0));
        WG_TRY(check_steps(L, C));
        *bytes = wg::gated_scan_workspace(dtype, N, L, C, backward != 0);
        return WG_OK;
    });
}

wg_status winograd_gated_scan(const wg_gated_scan* a, hipStream_t stream) {
    return guarded([&]() -> wg_status {
        if (!a) return fail(WG_ERR_ARG, "null argument");
        if (!storage(a->dtype)) return fail(WG_ERR_UNSUPPORTED, "unknown dtype");
        const int64_t N = a->N, L = a->L, C = a->C, es = wg::dtype_bytes(static_cast<int>(a->dtype));
        WG_TRY(check_sizes(N, L, C, 1, 0));
        WG_TRY(check_steps(L, C));
        WG_TRY(check_rows(a->gate, "gate", N, L, C, es, false));
        WG_TRY(check_rows(a->value, "value", N, L, C, es, false));
        if (a->out_gate.data) WG_TRY(check_rows(a->out_gate, "out_gate", N, L, C, es, false));
        WG_TRY(check_rows(a->y, "y", N, L, C, es, true));
        WG_TRY(check_f32(a->h0, "h0"));
        WG_TRY(check_f32(a->lengths, "lengths"));
        WG_TRY(check_f32(a->h_last, "h_last", false));
        WG_TRY(check_f32(a->states, "states"));
        WG_TRY(check_workspace(a->workspace, a->workspace_bytes,
                               wg::gated_scan_workspace(static_cast<int>(a->dtype), N, L, C, false)));
        return from_hip(WG_BY_DTYPE(a->dtype, wg::launch_gated_scan_t)(*a, stream), "gated scan");
    });
}

wg_status winograd_gated_scan_backward(const wg_gated_scan_backward* a, hipStream_t stream) {
    return guarded([&]() -> wg_status {
        if (!a) return fail(WG_ERR_ARG, "null argument");
        if (!storage(a->dtype)) return fail(WG_ERR_UNSUPPORTED, "unknown dtype");
        const int64_t N = a->N, L = a->L, C = a->C, es = wg::dtype_bytes(static_cast<int>(a->dtype));
        WG_TRY(check_sizes(N, L, C, 1, 0));
        WG_TRY(check_steps(L, C));
        WG_TRY(check_rows(a->dy, "dy", N, L, C, es, false));
        WG_TRY(check_rows(a->gate, "gate", N, L, C, es, false));
        WG_TRY(check_rows(a->value, "value", N, L, C, es, false));
        WG_TRY(check_rows(a->dgate, "dgate", N, L, C, es, true));
        WG_TRY(check_rows(a->dvalue, "dvalue", N, L, C, es, true));
        if (a->out_gate.data) {
            WG_TRY(check_rows(a->out_gate, "out_gate", N, L, C, es, false));
            WG_TRY(check_rows(a->dout_gate, "dout_gate", N, L, C, es, true));
        }
        WG_TRY(check_f32(a->states, "states", L == 0));
        WG_TRY(check_f32(a->dh_last, "dh_last"));
        WG_TRY(check_f32(a->lengths, "lengths"));
        WG_TRY(check_f32(a->dh0, "dh0"));
        WG_TRY(check_workspace(a->workspace, a->workspace_bytes,
                               wg::gated_scan_workspace(static_cast<int>(a->dtype), N, L, C, true)));
        return from_hip(WG_BY_DTYPE(a->dtype, wg::launch_gated_scan_backward_t)(*a, stream), "gated scan's gradients");
    });
}

wg_status winograd_gated_step(const wg_gated_step* a, hipStream_t stream) {
    return guarded([&]() -> wg_status {
        if (!a) return fail(WG_ERR_ARG, "null argument");
        if (!storage(a->dtype)) return fail(WG_ERR_UNSUPPORTED, "unknown dtype");
        const int64_t es = wg::dtype_bytes(static_cast<int>(a->dtype));
        WG_TRY(check_sizes(a->N, 1, a->C, 0, 1));
        if (a->N == 0) return WG_OK;
        WG_TRY(check_rows(a->gate, "gate", a->N, 1, a->C, es, false));
        WG_TRY(check_rows(a->value, "value", a->N, 1, a->C, es, false));
        if (a->out_gate.data) WG_TRY(check_rows(a->out_gate, "out_gate", a->N, 1, a->C, es, false));
        WG_TRY(check_rows(a->y, "y", a->N, 1, a->C, es, true));
        WG_TRY(check_f32(a->h, "h", false));
        WG_TRY(check_f32(a->h_new, "h_new", false));
        return from_hip(WG_BY_DTYPE(a->dtype, wg::launch_gated_step_t)(*a, stream), "gated step");
    });
}

wg_status winograd_rms_norm(const wg_rms_norm* a, hipStream_t stream) {
    return guarded([&]() -> wg_status {
        if (!a) return fail(WG_ERR_ARG, "null argument");
        if (!storage(a->dtype)) return fail(WG_ERR_UNSUPPORTED, "unknown dtype");
        const bool quant = a->y_dtype == WG_E4M3;
        if (!quant && a->y_dtype != a->dtype) return fail(WG_ERR_UNSUPPORTED, "y_dtype must be dtype or WG_E4M3");
        if (a->group != 0 && (!quant || (a->group != 32 && a->group != 64 && a->group != 128)))
            return fail(WG_ERR_UNSUPPORTED, "group must be 0 or, for 8 bits, 32, 64 or 128");
        const int64_t N = a->N, L = a->L, C = a->C, es = wg::dtype_bytes(static_cast<int>(a->dtype));
        WG_TRY(check_sizes(N, L, C, 0, 0));
        WG_TRY(check_row(C));
        if (!std::isfinite(static_cast<float>(a->eps)) || a->eps < 0)
            return fail(WG_ERR_ARG, "eps must be finite in fp32 and not negative");
        if (N == 0 || L == 0) return WG_OK;
        WG_TRY(check_rows(a->x, "x", N, L, C, es, false));
        if (a->residual.data) WG_TRY(check_rows(a->residual, "residual", N, L, C, es, false));
        if (a->r.data) WG_TRY(check_rows(a->r, "r", N, L, C, es, true));
        WG_TRY(check_rows(a->y, "y", N, L, C, quant ? 1 : es, true));
        if (!a->weight || !aligned(a->weight, static_cast<uintptr_t>(es)))
            return fail(WG_ERR_ARG, "weight is null or not aligned to its elements");
        if (quant) WG_TRY(check_f32(a->scales, "scales", false));
        return from_hip(WG_BY_DTYPE(a->dtype, wg::launch_rms_norm_t)(*a, stream), "norm");
    });
}

wg_status winograd_rms_norm_workspace(wg_dtype dtype, int64_t N, int64_t L, int64_t C, size_t* bytes) {
    return guarded([&]() -> wg_status {
        if (!bytes) return fail(WG_ERR_ARG, "null argument");
        if (!storage(dtype)) return fail(WG_ERR_UNSUPPORTED, "unknown dtype");
        WG_TRY(check_sizes(N, L, C, 0, 0));
        WG_TRY(check_row(C));
        *bytes = wg::rms_norm_workspace(dtype, N, L, C);
        return WG_OK;
    });
}

wg_status winograd_rms_norm_backward(const wg_rms_norm_backward* a, hipStream_t stream) {
    return guarded([&]() -> wg_status {
        if (!a) return fail(WG_ERR_ARG, "null argument");
        if (!storage(a->dtype)) return fail(WG_ERR_UNSUPPORTED, "unknown dtype");
        const int64_t N = a->N, L = a->L, C = a->C, es = wg::dtype_bytes(static_cast<int>(a->dtype));
        WG_TRY(check_sizes(N, L, C, 0, 0));
        WG_TRY(check_row(C));
        if (!std::isfinite(static_cast<float>(a->eps)) || a->eps < 0)
            return fail(WG_ERR_ARG, "eps must be finite in fp32 and not negative");
        WG_TRY(check_rows(a->dy, "dy", N, L, C, es, false));
        WG_TRY(check_rows(a->r, "r", N, L, C, es, false));
        if (a->dr.data) WG_TRY(check_rows(a->dr, "dr", N, L, C, es, false));
        WG_TRY(check_rows(a->dx, "dx", N, L, C, es, true));
        if (!a->weight || !aligned(a->weight, static_cast<uintptr_t>(es)))
            return fail(WG_ERR_ARG, "weight is null or not aligned to its elements");
        WG_TRY(check_f32(a->dweight, "dweight", false));
        WG_TRY(check_workspace(a->workspace, a->workspace_bytes,
                               wg::rms_norm_workspace(static_cast<int>(a->dtype), N, L, C)));
        return from_hip(WG_BY_DTYPE(a->dtype, wg::launch_rms_norm_backward_t)(*a, stream), "norm's gradients");
    });
}

wg_status winograd_matvec_w4(const wg_matvec_w4* a, hipStream_t stream) {
    return guarded([&]() -> wg_status {
        if (!a) return fail(WG_ERR_ARG, "null argument");
        WG_TRY(check_w4(a->w));
        const bool x8 = a->x_dtype == WG_E4M3;
        if (!storage(a->x_dtype) && !x8) return fail(WG_ERR_UNSUPPORTED, "unknown x_dtype");
        if (!storage(a->y_dtype)) return fail(WG_ERR_UNSUPPORTED, "unknown y_dtype");
        if (a->M < 0 || a->M >= kMaxSize) return fail(WG_ERR_ARG, "M must be in [0, 2^31)");
        if (a->M == 0) return WG_OK;
        const int64_t K = a->w.cols, R = a->w.rows;
        const int64_t xs = x8 ? 1 : wg::dtype_bytes(static_cast<int>(a->x_dtype));
        const int64_t ys = wg::dtype_bytes(static_cast<int>(a->y_dtype));
        WG_TRY(check_sizes(1, a->M, K > R ? K : R, 1, 0));
        WG_TRY(check_rows(wg_rows{a->x, 0, a->ldx}, "x", 1, a->M, K, xs, false));
        WG_TRY(check_rows(wg_rows{a->y, 0, a->ldy}, "y", 1, a->M, R, ys, true));
        if (x8) {
            WG_TRY(check_f32(a->x_scales, "x_scales", false));
            if (a->x_groups != 1 && a->x_groups != (K + a->w.group - 1) / a->w.group)
                return fail(WG_ERR_ARG, "x_scales must be one a row or by the weights' groups");
        } else if (a->x_scales) {
            return fail(WG_ERR_ARG, "x_scales are for rows in 8 bits");
        }
        return from_hip(wg::launch_matvec_w4(*a, stream), "4-bit product");
    });
}

wg_status winograd_quantize_w4(const wg_w4* w, wg_dtype dtype, const void* m, int64_t ldm, hipStream_t stream) {
    return guarded([&]() -> wg_status {
        if (!w) return fail(WG_ERR_ARG, "null argument");
        WG_TRY(check_w4(*w));
        if (!storage(dtype)) return fail(WG_ERR_UNSUPPORTED, "unknown dtype");
        WG_TRY(check_rows(wg_rows{m, 0, ldm}, "m", 1, w->rows, w->cols, wg::dtype_bytes(dtype), false));
        return from_hip(WG_BY_DTYPE(dtype, wg::launch_quantize_w4_t)(*w, m, ldm, stream), "4-bit codes");
    });
}

wg_status winograd_pack_w4(const wg_w4* w, const void* nibbles, const void* scales, hipStream_t stream) {
    return guarded([&]() -> wg_status {
        if (!w) return fail(WG_ERR_ARG, "null argument");
        WG_TRY(check_w4(*w));
        if (!nibbles || !scales || !aligned(scales, 2)) return fail(WG_ERR_ARG, "null nibbles or scales, or scales not aligned");
        return from_hip(wg::launch_pack_w4(*w, nibbles, scales, stream), "4-bit layout");
    });
}

wg_status winograd_dequantize_w4(const wg_w4* w, wg_dtype dtype, void* m, int64_t ldm, hipStream_t stream) {
    return guarded([&]() -> wg_status {
        if (!w) return fail(WG_ERR_ARG, "null argument");
        WG_TRY(check_w4(*w));
        if (!storage(dtype)) return fail(WG_ERR_UNSUPPORTED, "unknown dtype");
        WG_TRY(check_rows(wg_rows{m, 0, ldm}, "m", 1, w->rows, w->cols, wg::dtype_bytes(dtype), true));
        return from_hip(WG_BY_DTYPE(dtype, wg::launch_dequantize_w4_t)(*w, m, ldm, stream), "4-bit weights");
    });
}

}  // extern "C"
