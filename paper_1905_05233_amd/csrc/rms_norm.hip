// The root-mean-square norm of rows with the residual's addition, its output in
// the storage type or in 8 bits with scales, and its gradients, on gfx950:
//   r = x + residual,  y = r rstd weight,  rstd = 1 / sqrt(mean(r^2) + eps)
//   dr_total = rstd (g - r rstd^2 mean(g r)) + dr  with g = dy weight,
//   dweight = sum over the rows of dy r rstd.
// Sums and statistics in fp32.
#include <hip/hip_runtime.h>

#include <cstdint>

#include "device_common.hpp"
#include "kernels.hpp"
#include "sequence.hpp"

namespace wg {

namespace {

constexpr int kNormThreads = 256;
constexpr float kFp8Max = 448.0f;            // largest value of e4m3
constexpr float kFp8Least = 0x1p-100f;       // absolute maxima below this count as this

template <typename Elem> struct NormArgs {
    int64_t N, L, C;
    wg_rows x, residual, r, y;
    const Elem* weight;
    float* scales;
    float eps;
    int64_t group;   // channels a scale covers
};

template <typename T> __device__ __forceinline__ T* row_at(const wg_rows& r, int64_t n, int64_t l) {
    return static_cast<T*>(const_cast<void*>(r.data)) + n * r.stride_n + l * r.stride_l;
}

__device__ __forceinline__ uint8_t e4m3_of(float v) {
    return static_cast<uint8_t>(__builtin_amdgcn_cvt_pk_fp8_f32(v, 0.0f, 0, false));
}

// Sum over the workgroup, the same value in every thread.
__device__ __forceinline__ float block_sum(float v, float* lds) {
    lds[threadIdx.x] = v;
    __syncthreads();
    for (int s = kNormThreads / 2; s > 0; s >>= 1) {
        if (static_cast<int>(threadIdx.x) < s) lds[threadIdx.x] += lds[threadIdx.x + s];
        __syncthreads();
    }
    const float t = lds[0];
    __syncthreads();
    return t;
}

// One workgroup per row; the row is read again for the output.
template <typename Elem, bool QUANT>
__global__ __launch_bounds__(kNormThreads) void norm_kernel(NormArgs<Elem> a) {
    using S = Storage<Elem>;
    __shared__ float lds[kNormThreads];
    for (int64_t row = blockIdx.x; row < a.N * a.L; row += gridDim.x) {
        const int64_t n = row / a.L, l = row % a.L;
        const Elem* x = row_at<const Elem>(a.x, n, l);
        const Elem* res = a.residual.data ? row_at<const Elem>(a.residual, n, l) : nullptr;
        auto sum_at = [&](int64_t c) {
            return S::to_f32(x[c]) + (res ? S::to_f32(res[c]) : 0.0f);
        };
        float ss = 0.0f;
        for (int64_t c = threadIdx.x; c < a.C; c += kNormThreads) {
            const float v = sum_at(c);
            ss = fmaf(v, v, ss);
        }
        const float rstd = 1.0f / sqrtf(block_sum(ss, lds) / static_cast<float>(a.C) + a.eps);
        if constexpr (!QUANT) {
            for (int64_t c = threadIdx.x; c < a.C; c += kNormThreads) {
                const float v = sum_at(c);
                row_at<Elem>(a.y, n, l)[c] = S::from_f32(v * rstd * S::to_f32(a.weight[c]));
                if (a.r.data) row_at<Elem>(a.r, n, l)[c] = S::from_f32(v);
            }
        } else {
            const int64_t groups = (a.C + a.group - 1) / a.group;
            for (int64_t g = 0; g < groups; ++g) {
                const int64_t end = a.C < (g + 1) * a.group ? a.C : (g + 1) * a.group;
                // as whole numbers the bit patterns of |y| ascend with it, NaN last
                uint32_t top = 0;
                for (int64_t c = g * a.group + threadIdx.x; c < end; c += kNormThreads) {
                    const uint32_t v = __float_as_uint(fabsf(sum_at(c) * rstd * S::to_f32(a.weight[c])));
                    top = v > top ? v : top;
                }
                auto* words = reinterpret_cast<uint32_t*>(lds);
                words[threadIdx.x] = top;
                __syncthreads();
                for (int s = kNormThreads / 2; s > 0; s >>= 1) {
                    if (static_cast<int>(threadIdx.x) < s && words[threadIdx.x + s] > words[threadIdx.x])
                        words[threadIdx.x] = words[threadIdx.x + s];
                    __syncthreads();
                }
                const float most = __uint_as_float(words[0]);
                __syncthreads();
                const float scale = (most < kFp8Least ? kFp8Least : most) / kFp8Max;
                const float inv = 1.0f / scale;
                for (int64_t c = g * a.group + threadIdx.x; c < end; c += kNormThreads) {
                    const float v = sum_at(c);
                    row_at<uint8_t>(a.y, n, l)[c] = e4m3_of(v * rstd * S::to_f32(a.weight[c]) * inv);
                }
                if (threadIdx.x == 0) a.scales[row * groups + g] = scale;
            }
            if (a.r.data)   // last: r may be x itself
                for (int64_t c = threadIdx.x; c < a.C; c += kNormThreads) row_at<Elem>(a.r, n, l)[c] = S::from_f32(sum_at(c));
        }
    }
}

template <typename Elem> struct NormGradArgs {
    int64_t N, L, C;
    wg_rows dy, r, dr, dx;
    const Elem* weight;
    float* dweight;
    float eps;
    float* rstd;   // workspace: one a row
};

template <typename Elem>
__global__ __launch_bounds__(kNormThreads) void norm_grad_kernel(NormGradArgs<Elem> a) {
    using S = Storage<Elem>;
    __shared__ float lds[kNormThreads];
    for (int64_t row = blockIdx.x; row < a.N * a.L; row += gridDim.x) {
        const int64_t n = row / a.L, l = row % a.L;
        const Elem* r = row_at<const Elem>(a.r, n, l);
        const Elem* dy = row_at<const Elem>(a.dy, n, l);
        float ss = 0.0f, gr = 0.0f;
        for (int64_t c = threadIdx.x; c < a.C; c += kNormThreads) {
            const float v = S::to_f32(r[c]);
            ss = fmaf(v, v, ss);
            gr = fmaf(S::to_f32(dy[c]) * S::to_f32(a.weight[c]), v, gr);
        }
        const float rstd = 1.0f / sqrtf(block_sum(ss, lds) / static_cast<float>(a.C) + a.eps);
        const float mean = block_sum(gr, lds) / static_cast<float>(a.C) * rstd * rstd;
        for (int64_t c = threadIdx.x; c < a.C; c += kNormThreads) {
            float d = rstd * (S::to_f32(dy[c]) * S::to_f32(a.weight[c]) - S::to_f32(r[c]) * mean);
            if (a.dr.data) d += S::to_f32(row_at<const Elem>(a.dr, n, l)[c]);
            row_at<Elem>(a.dx, n, l)[c] = S::from_f32(d);
        }
        if (threadIdx.x == 0) a.rstd[row] = rstd;
    }
}

// dweight, one thread per channel; ahead of the kernel above, whose dx may be dy.
template <typename Elem>
__global__ __launch_bounds__(kNormThreads) void norm_dweight_kernel(NormGradArgs<Elem> a) {
    using S = Storage<Elem>;
    const int64_t c = static_cast<int64_t>(blockIdx.x) * kNormThreads + threadIdx.x;
    if (c >= a.C) return;
    float sum = 0.0f;
    for (int64_t row = 0; row < a.N * a.L; ++row) {
        const int64_t n = row / a.L, l = row % a.L;
        sum += S::to_f32(row_at<const Elem>(a.dy, n, l)[c]) * (S::to_f32(row_at<const Elem>(a.r, n, l)[c]) * a.rstd[row]);
    }
    a.dweight[c] = sum;
}

template <typename Elem>
__global__ __launch_bounds__(kNormThreads) void norm_rstd_kernel(NormGradArgs<Elem> a) {
    using S = Storage<Elem>;
    __shared__ float lds[kNormThreads];
    for (int64_t row = blockIdx.x; row < a.N * a.L; row += gridDim.x) {
        const Elem* r = row_at<const Elem>(a.r, row / a.L, row % a.L);
        float ss = 0.0f;
        for (int64_t c = threadIdx.x; c < a.C; c += kNormThreads) ss = fmaf(S::to_f32(r[c]), S::to_f32(r[c]), ss);
        ss = block_sum(ss, lds);
        if (threadIdx.x == 0) a.rstd[row] = 1.0f / sqrtf(ss / static_cast<float>(a.C) + a.eps);
    }
}

unsigned row_blocks(int64_t rows) { return static_cast<unsigned>(rows < 65536 ? rows : 65536); }

}  // namespace

size_t rms_norm_workspace(int, int64_t N, int64_t L, int64_t) { return static_cast<size_t>((N * L + 3) / 4 * 16); }

template <int D> hipError_t launch_rms_norm_t(const wg_rms_norm& a, hipStream_t stream) {
    using Elem = typename DTypeOf<D>::type;
    const NormArgs<Elem> k{a.N, a.L, a.C, a.x, a.residual, a.r, a.y, static_cast<const Elem*>(a.weight), a.scales,
                           static_cast<float>(a.eps), a.group ? a.group : a.C};
    if (a.y_dtype == WG_E4M3) norm_kernel<Elem, true><<<row_blocks(a.N * a.L), kNormThreads, 0, stream>>>(k);
    else norm_kernel<Elem, false><<<row_blocks(a.N * a.L), kNormThreads, 0, stream>>>(k);
    return hipGetLastError();
}

template <int D> hipError_t launch_rms_norm_backward_t(const wg_rms_norm_backward& a, hipStream_t stream) {
    using Elem = typename DTypeOf<D>::type;
    const NormGradArgs<Elem> k{a.N, a.L, a.C, a.dy, a.r, a.dr, a.dx, static_cast<const Elem*>(a.weight), a.dweight,
                               static_cast<float>(a.eps), static_cast<float*>(a.workspace)};
    if (a.N * a.L > 0) norm_rstd_kernel<Elem><<<row_blocks(a.N * a.L), kNormThreads, 0, stream>>>(k);
    norm_dweight_kernel<Elem>
        <<<static_cast<unsigned>((a.C + kNormThreads - 1) / kNormThreads), kNormThreads, 0, stream>>>(k);
    if (a.N * a.L > 0) norm_grad_kernel<Elem><<<row_blocks(a.N * a.L), kNormThreads, 0, stream>>>(k);
    return hipGetLastError();
}

#define WG_NORM_INSTANCES(D)                                                       \
    template hipError_t launch_rms_norm_t<D>(const wg_rms_norm&, hipStream_t);     \
    template hipError_t launch_rms_norm_backward_t<D>(const wg_rms_norm_backward&, hipStream_t);
WG_NORM_INSTANCES(0)
WG_NORM_INSTANCES(1)
WG_NORM_INSTANCES(2)
#undef WG_NORM_INSTANCES

}  // namespace wg
