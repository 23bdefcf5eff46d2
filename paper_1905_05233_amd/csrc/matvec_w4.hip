// Products of rows with a matrix of 4-bit weights with group scales, and the
// making and unmaking of such matrices, on gfx950:
//   y[m][j] = sum_g scale[j][g] sum_(k in g) (code[j][k] - 8) x[m][k].
// The layout of codes and scales is winograd_crt.h's (wg_w4).
#include <hip/hip_runtime.h>

#include <cstdint>

#include "device_common.hpp"
#include "kernels.hpp"
#include "sequence.hpp"

namespace wg {

namespace {

constexpr int kW4Threads = 256;

struct W4 {
    uint32_t* codes;
    bf16_t* scales;
    int64_t rows, cols, groups, ktiles;
    int group;
};
W4 w4_of(const wg_w4& w) {
    return {static_cast<uint32_t*>(const_cast<void*>(w.codes)), static_cast<bf16_t*>(const_cast<void*>(w.scales)), w.rows,
            w.cols, (w.cols + w.group - 1) / w.group, (w.cols + 127) / 128, static_cast<int>(w.group)};
}

// The word with columns c .. c + 7 (c a multiple of 8) of row j.
__device__ __forceinline__ int64_t word_at(const W4& w, int64_t j, int64_t c) {
    const int64_t in = c % 128;
    return (((j / 16 * w.ktiles + c / 128) * 4 + in % 32 / 8) * 16 + j % 16) * 4 + in / 32;
}
__device__ __forceinline__ int64_t scale_at(const W4& w, int64_t j, int64_t g) { return (j / 16 * w.groups + g) * 16 + j % 16; }

__device__ __forceinline__ uint32_t pack8(const int (&code)[8]) {
    uint32_t v = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) v |= static_cast<uint32_t>(code[j]) << (4 * (j / 2) + 16 * (j % 2));
    return v << 3 | v >> 29;
}
__device__ __forceinline__ int code_of(uint32_t word, int j) {
    const uint32_t v = word >> 3 | word << 29;
    return static_cast<int>(v >> (4 * (j / 2) + 16 * (j % 2)) & 15u);
}

template <int D> struct XTypeOf { using type = typename DTypeOf<D>::type; };
template <> struct XTypeOf<3> { using type = uint8_t; };
template <typename T> __device__ __forceinline__ float x_value(T v) {
    if constexpr (sizeof(T) == 1) return __builtin_amdgcn_cvt_f32_fp8(v, 0);
    else return Storage<T>::to_f32(v);
}

// One wave per output; lanes take words of eight columns.
template <int XD, int YD>
__global__ __launch_bounds__(kW4Threads) void matvec_kernel(W4 w, int64_t M, const void* xp, int64_t ldx,
                                                            const float* xs, int64_t x_groups, void* yp, int64_t ldy) {
    using X = typename XTypeOf<XD>::type;
    using Y = typename DTypeOf<YD>::type;
    const int lane = threadIdx.x % 64;
    const int64_t waves = static_cast<int64_t>(gridDim.x) * (kW4Threads / 64);
    for (int64_t id = static_cast<int64_t>(blockIdx.x) * (kW4Threads / 64) + threadIdx.x / 64; id < M * w.rows; id += waves) {
        const int64_t m = id / w.rows, j = id % w.rows;
        const X* x = static_cast<const X*>(xp) + m * ldx;
        float sum = 0.0f;
        for (int64_t c = lane * 8; c < w.cols; c += 64 * 8) {
            const uint32_t word = w.codes[word_at(w, j, c)];
            const int64_t g = c / w.group;
            float part = 0.0f;
            for (int e = 0; e < 8 && c + e < w.cols; ++e)
                part = fmaf(static_cast<float>(code_of(word, e) - 8), x_value(x[c + e]), part);
            float s = Storage<bf16_t>::to_f32(w.scales[scale_at(w, j, g)]);
            if (XD == 3) s *= xs[m * x_groups + (x_groups == 1 ? 0 : g)];
            sum = fmaf(s, part, sum);
        }
        for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o);
        if (lane == 0) (static_cast<Y*>(yp) + m * ldy)[j] = Storage<Y>::from_f32(sum);
    }
}

// One thread per group of a row (padding rows too).
template <typename Elem>
__global__ __launch_bounds__(kW4Threads) void quantize_kernel(W4 w, const Elem* m, int64_t ldm) {
    const int64_t id = static_cast<int64_t>(blockIdx.x) * kW4Threads + threadIdx.x;
    const int64_t rows = (w.rows + 15) / 16 * 16, padded = w.ktiles * 128;
    const int64_t groups = padded / w.group;
    if (id >= rows * groups) return;
    const int64_t j = id / groups, g = id % groups;
    auto value = [&](int64_t c) {
        return j < w.rows && c < w.cols ? Storage<Elem>::to_f32(m[j * ldm + c]) : 0.0f;
    };
    float top = 0.0f;
    for (int64_t c = g * w.group; c < (g + 1) * w.group; ++c) top = fmaxf(top, fabsf(value(c)));
    const bf16_t scale = Storage<bf16_t>::from_f32(top / 7.0f);
    const float s = Storage<bf16_t>::to_f32(scale);
    if (g < w.groups) w.scales[scale_at(w, j, g)] = scale;
    for (int64_t c = g * w.group; c < (g + 1) * w.group; c += 8) {
        int code[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float q = s > 0.0f ? rintf(value(c + e) / s) : 0.0f;
            code[e] = static_cast<int>(fminf(fmaxf(q, -8.0f), 7.0f)) + 8;
        }
        w.codes[word_at(w, j, c)] = pack8(code);
    }
}

// One thread per word (of padding rows and columns too).
__global__ __launch_bounds__(kW4Threads) void pack_kernel(W4 w, const uint8_t* nibbles, const bf16_t* scales) {
    const int64_t id = static_cast<int64_t>(blockIdx.x) * kW4Threads + threadIdx.x;
    const int64_t rows = (w.rows + 15) / 16 * 16, words = w.ktiles * 16;
    if (id >= rows * words) return;
    const int64_t j = id / words, c = id % words * 8, ld = (w.cols + 1) / 2;
    int code[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const int64_t at = c + e;
        code[e] = j < w.rows && at < w.cols ? nibbles[j * ld + at / 2] >> (at % 2 * 4) & 15 : 8;
    }
    w.codes[word_at(w, j, c)] = pack8(code);
    if (c % w.group == 0 && c / w.group < w.groups) {
        const int64_t g = c / w.group;
        w.scales[scale_at(w, j, g)] = j < w.rows ? scales[j * w.groups + g] : bf16_t{0};
    }
}

template <typename Elem>
__global__ __launch_bounds__(kW4Threads) void dequantize_kernel(W4 w, Elem* m, int64_t ldm) {
    const int64_t id = static_cast<int64_t>(blockIdx.x) * kW4Threads + threadIdx.x;
    const int64_t words = (w.cols + 7) / 8;
    if (id >= w.rows * words) return;
    const int64_t j = id / words, c = id % words * 8;
    const uint32_t word = w.codes[word_at(w, j, c)];
    const float s = Storage<bf16_t>::to_f32(w.scales[scale_at(w, j, c / w.group)]);
    for (int e = 0; e < 8 && c + e < w.cols; ++e)
        m[j * ldm + c + e] = Storage<Elem>::from_f32(static_cast<float>(code_of(word, e) - 8) * s);
}

hipError_t blocks_for(int64_t threads, unsigned* blocks) {
    const int64_t b = (threads + kW4Threads - 1) / kW4Threads;
    if (b * kW4Threads > 0xffffffffLL) return hipErrorInvalidValue;
    *blocks = static_cast<unsigned>(b);
    return hipSuccess;
}

template <int XD, int YD> hipError_t matvec_t(const wg_matvec_w4& a, hipStream_t stream) {
    const int64_t waves = a.M * a.w.rows, blocks = (waves + kW4Threads / 64 - 1) / (kW4Threads / 64);
    matvec_kernel<XD, YD><<<static_cast<unsigned>(blocks < 65536 ? blocks : 65536), kW4Threads, 0, stream>>>(
        w4_of(a.w), a.M, a.x, a.ldx, a.x_scales, a.x_groups, a.y, a.ldy);
    return hipGetLastError();
}
template <int XD> hipError_t matvec_x(const wg_matvec_w4& a, hipStream_t stream) {
    return a.y_dtype == WG_F32 ? matvec_t<XD, 0>(a, stream)
                               : a.y_dtype == WG_F16 ? matvec_t<XD, 1>(a, stream) : matvec_t<XD, 2>(a, stream);
}

}  // namespace

hipError_t launch_matvec_w4(const wg_matvec_w4& a, hipStream_t stream) {
    switch (a.x_dtype) {
        case WG_F32: return matvec_x<0>(a, stream);
        case WG_F16: return matvec_x<1>(a, stream);
        case WG_BF16: return matvec_x<2>(a, stream);
        default: return matvec_x<3>(a, stream);
    }
}

template <int D> hipError_t launch_quantize_w4_t(const wg_w4& w, const void* m, int64_t ldm, hipStream_t stream) {
    using Elem = typename DTypeOf<D>::type;
    const W4 k = w4_of(w);
    unsigned blocks;
    const hipError_t e = blocks_for((w.rows + 15) / 16 * 16 * (k.ktiles * 128 / w.group), &blocks);
    if (e != hipSuccess) return e;
    quantize_kernel<Elem><<<blocks, kW4Threads, 0, stream>>>(k, static_cast<const Elem*>(m), ldm);
    return hipGetLastError();
}

template <int D> hipError_t launch_dequantize_w4_t(const wg_w4& w, void* m, int64_t ldm, hipStream_t stream) {
    using Elem = typename DTypeOf<D>::type;
    unsigned blocks;
    const hipError_t e = blocks_for(w.rows * ((w.cols + 7) / 8), &blocks);
    if (e != hipSuccess) return e;
    dequantize_kernel<Elem><<<blocks, kW4Threads, 0, stream>>>(w4_of(w), static_cast<Elem*>(m), ldm);
    return hipGetLastError();
}

hipError_t launch_pack_w4(const wg_w4& w, const void* nibbles, const void* scales, hipStream_t stream) {
    const W4 k = w4_of(w);
    unsigned blocks;
    const hipError_t e = blocks_for((w.rows + 15) / 16 * 16 * (k.ktiles * 16), &blocks);
    if (e != hipSuccess) return e;
    pack_kernel<<<blocks, kW4Threads, 0, stream>>>(k, static_cast<const uint8_t*>(nibbles),
                                                   static_cast<const bf16_t*>(scales));
    return hipGetLastError();
}

#define WG_W4_INSTANCES(D)                                                                            \
    template hipError_t launch_quantize_w4_t<D>(const wg_w4&, const void*, int64_t, hipStream_t);      \
    template hipError_t launch_dequantize_w4_t<D>(const wg_w4&, void*, int64_t, hipStream_t);
WG_W4_INSTANCES(0)
WG_W4_INSTANCES(1)
WG_W4_INSTANCES(2)
#undef WG_W4_INSTANCES

}  // namespace wg
