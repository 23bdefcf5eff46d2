// Products of rows with a matrix of 4-bit weights with group scales, and the
// making and unmaking of such matrices, on gfx950:
//   y[m][j] = sum_g scale[j][g] sum_(k in g) (code[j][k] - 8) x[m][k].
// The layout of codes and scales is winograd_crt.h's (wg_w4).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>

#include "device_common.hpp"
#include "kernels.hpp"
#include "rows.hpp"
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

// The product on the matrix cores.  A workgroup multiplies one or two tiles of 16 rows
// of the matrix with up to 16 rows of x (v_mfma_f32_16x16x32: 32 columns an instruction);
// a lane's 16 bytes of a tile of 128 columns are its fragments for four of them.
//
// A code becomes a 16-bit float without arithmetic: four bits at bit 3 of the
// fraction of a number whose ones there count 1 (16 in bf16, 128 in fp16), so that
// a word gives its eight weights, plus 16 or 128, in seven and/or/shift
// instructions.  For rows in bf16 and fp8 what was added, and the codes' 8, leaves
// through the accumulator, which starts each group from another product, of a constant
// matrix (-24) with the same x, and so exactly up to the accumulator's fp32.
// The group's sum times its scale goes to the running fp32 sum of the output.
//
// Rows of x in fp16 meet the weights themselves (four subtractions a word in place of
// that product); so do rows in fp32, cut into three bf16 parts of 8 bits each, which hold
// all 24 bits.  fp8 becomes bf16 exactly.
//
// The waves of a workgroup take the tiles of columns in turn, each wave's next tile
// in flight (two or more ahead are no faster: 25088 -> 4096 14.2 us with one, 15.8
// with two), and their sums are added in a fixed order at the end; how many
// waves depends on the matrix alone, and the order of an output's sums not on the
// tiles of its workgroup, so that an output does not depend on the other rows of x.
//
// Measured: 25088 -> 4096 for one bf16 row, 53 MB, 12.7 us a call: 4.2 TB/s; it is
// bound by memory and the waves' start and end (a copy moves as much in 10.2).  4096 ->
// 1000 for five fp32 rows 8 us, 1536 -> 1536 for sixteen 8-bit rows 5 us: latency, 63 and
// 96 workgroups.  Sixteen rows of 25088 take twice as long as one (30 against 15.6 us):
// every workgroup reads all of x through its L1.  4096 -> 32768 takes 21.4 us on the GPU
// for one row and 28.5 for sixteen, 69 MB: 3.2 and 2.4 TB/s.  fp32 rows, three products a
// fragment and rebuilt weights, are bound by that work: 25088 -> 4096 34 us for one row and
// 53 for sixteen, 4096 -> 4096 8.1 for one (bf16 4.8).
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
constexpr int kTokens = 16;     // rows of x that a wave takes

template <bool F16> __device__ __forceinline__ f32x4 mma(const u32x4& a, const u32x4& b, const f32x4& c) {
    if constexpr (F16)
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0,
                                                       0);
}

// The eight codes of a word as 16-bit floats, plus 16 (bf16) or 128 (fp16).
template <bool F16> __device__ __forceinline__ u32x4 widen_codes(uint32_t w) {
    constexpr uint32_t kMask = 0x00780078u, kOne = F16 ? 0x58005800u : 0x41804180u;
    return u32x4{(w & kMask) | kOne, (w >> 4 & kMask) | kOne, (w >> 8 & kMask) | kOne,
                 (__builtin_amdgcn_alignbit(w, w, 12) & kMask) | kOne};
}
// What must go again: -24 in bf16.
constexpr uint32_t kOffset = 0xc1c0c1c0u;

// The weights themselves, codes less 8, for fp32 and fp16 rows: what is added above
// would cost their sums three and four bits (fp32 outputs over 4096 columns from fp32
// rows 1.0e-6 off, and 1.2e-7 without; from fp16 rows 0.8 to 2.2e-6 and 0.9e-7, where 4096
// -> 5000 takes 6.5 us instead of 6.3 and 25088 -> 4096 the same).  bf16 and fp8 rows lose
// nothing: their products have few bits, 1.0e-7 either way.
__device__ __forceinline__ uint32_t upper_halves(uint32_t lo, uint32_t hi) { return __builtin_amdgcn_perm(hi, lo, 0x07060302u); }
template <bool F16> __device__ __forceinline__ u32x4 exact_codes(uint32_t w) {
    u32x4 f = widen_codes<F16>(w);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const uint32_t pair = f[j];
        if constexpr (F16)
            f[j] = __builtin_bit_cast(uint32_t, __builtin_bit_cast(f16x2, pair) - f16x2{136, 136});
        else
            f[j] = upper_halves(__float_as_uint(__uint_as_float(pair << 16) - 24.0f),
                                __float_as_uint(__uint_as_float(pair & 0xffff0000u) - 24.0f));
    }
    return f;
}

template <int D> struct XTypeOf { using type = typename DTypeOf<D>::type; };
template <> struct XTypeOf<3> { using type = uint8_t; };

// Eight columns of a row of x as 16-bit parts: one, or three for fp32.
template <int XD> constexpr int kPlanes = XD == 0 ? 3 : 1;

template <typename X> struct __attribute__((packed, aligned(1))) XRun {
    X v[8];
};
// Eight columns as they lie in memory, from p on; past the end of a row, zeros.
template <typename X> __device__ __forceinline__ XRun<X> load_x(const X* p, int64_t valid) {
    if (valid >= 8) return *reinterpret_cast<const XRun<X>*>(p);
    XRun<X> run{};
#pragma unroll
    for (int j = 0; j < 8; ++j)
        if (j < valid) run.v[j] = p[j];
    return run;
}
template <int XD>
__device__ __forceinline__ void widen_x(const XRun<typename XTypeOf<XD>::type>& run, u32x4 (&planes)[kPlanes<XD>]) {
    if constexpr (XD == 1 || XD == 2) {
        planes[0] = __builtin_bit_cast(u32x4, run);
    } else if constexpr (XD == 3) {
        const u32x2 b = __builtin_bit_cast(u32x2, run);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8(b[h], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(b[h], true);
            planes[0][2 * h] = upper_halves(__float_as_uint(lo[0]), __float_as_uint(lo[1]));
            planes[0][2 * h + 1] = upper_halves(__float_as_uint(hi[0]), __float_as_uint(hi[1]));
        }
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            float f0 = run.v[2 * j], f1 = run.v[2 * j + 1];
#pragma unroll
            for (int part = 0; part < 3; ++part) {
                const uint32_t b0 = __float_as_uint(f0), b1 = __float_as_uint(f1);
                planes[part][j] = upper_halves(b0, b1);
                f0 -= __uint_as_float(b0 & 0xffff0000u);
                f1 -= __uint_as_float(b1 & 0xffff0000u);
            }
        }
    }
}

struct MatvecArgs {
    W4 w;
    int64_t M;
    const void* x;
    int64_t ldx;
    const float* x_scales;
    int64_t x_groups;
    void* y;
    int64_t ldy;
    int y_dtype;
};

// GPT: groups of a tile of 128 columns; XG: x's scales go by groups; RT: tiles of 16
// rows of the matrix that a workgroup multiplies with the same x.
template <int XD, int GPT, bool XG, int RT>
__global__ __launch_bounds__(1024) void matvec_kernel(MatvecArgs a) {
    using X = typename XTypeOf<XD>::type;
    constexpr bool F16 = XD == 1, EXACT = XD < 2;   // the weights themselves, or plus an offset
    constexpr int SPG = 4 / GPT;   // instructions of a group
    extern __shared__ float sums[];   // [wave][tile of rows][lane][4]
    const W4& w = a.w;
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, waves = blockDim.x / 64;
    const int quarter = lane / 16;
    const int ktiles = static_cast<int>(w.ktiles);
    const u32x4* codes[RT];
    const u32x2* scales[RT];
#pragma unroll
    for (int r = 0; r < RT; ++r) {
        // past the last tile of rows that one is taken again, and not stored
        const int64_t rt = min(static_cast<int64_t>(blockIdx.x) * RT + r, (w.rows - 1) / 16);
        codes[r] = reinterpret_cast<const u32x4*>(w.codes) + rt * w.ktiles * 64 + lane;
        scales[r] = reinterpret_cast<const u32x2*>(w.scales + rt * w.groups * 16) + quarter;
    }
    // past the last row of x the last one is taken again: outputs do not mix, and none is stored
    const int64_t row = min(static_cast<int64_t>(blockIdx.y) * kTokens + lane % 16, a.M - 1);
    const X* x = static_cast<const X*>(a.x) + row * a.ldx + 8 * quarter;
    const float* xs = XG ? a.x_scales + row * a.x_groups : nullptr;

    struct Tile {
        u32x4 codes[RT];
        XRun<X> x[4];
    };
    auto load = [&](int kt, Tile& tile) {
#pragma unroll
        for (int r = 0; r < RT; ++r) tile.codes[r] = codes[r][static_cast<int64_t>(kt) * 64];
        const X* xk = x + static_cast<int64_t>(kt) * 128;
        const int64_t left = w.cols - static_cast<int64_t>(kt) * 128;
        if (left >= 128) {
#pragma unroll
            for (int s = 0; s < 4; ++s) tile.x[s] = load_x(xk + 32 * s, 8);
        } else {
#pragma unroll
            for (int s = 0; s < 4; ++s) tile.x[s] = load_x(xk + 32 * s, left - 32 * s - 8 * quarter);
        }
    };
    f32x4 acc[RT] = {};
    Tile tile;
    load(wave, tile);   // there are at least as many tiles as waves
    for (int kt = wave; kt < ktiles; kt += waves) {
        u32x4 cur[RT];
#pragma unroll
        for (int r = 0; r < RT; ++r) cur[r] = tile.codes[r];
        u32x4 xp[4][kPlanes<XD>];
#pragma unroll
        for (int s = 0; s < 4; ++s) widen_x<XD>(tile.x[s], xp[s]);
        if (kt + waves < ktiles) load(kt + waves, tile);
#pragma unroll
        for (int g = 0; g < GPT; ++g) {
            // groups past the matrix's last one have no columns
            const int64_t group = min(static_cast<int64_t>(kt) * GPT + g, w.groups - 1);
            const u32x4 offset{kOffset, kOffset, kOffset, kOffset};
            f32x4 start{0, 0, 0, 0};
            if constexpr (!EXACT) {
#pragma unroll
                for (int s = g * SPG; s < (g + 1) * SPG; ++s) start = mma<F16>(offset, xp[s][0], start);
            }
            const float by = XG ? xs[group] : 1.0f;
#pragma unroll
            for (int r = 0; r < RT; ++r) {
                const u32x2 sc = scales[r][group * 4];
                f32x4 sum = start;
#pragma unroll
                for (int s = g * SPG; s < (g + 1) * SPG; ++s) {
                    const u32x4 frag = EXACT ? exact_codes<F16>(cur[r][s]) : widen_codes<F16>(cur[r][s]);
#pragma unroll
                    for (int part = 0; part < kPlanes<XD>; ++part) sum = mma<F16>(frag, xp[s][part], sum);
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    float f = __uint_as_float(i % 2 ? sc[i / 2] & 0xffff0000u : sc[i / 2] << 16);
                    if (XG) f *= by;
                    acc[r][i] = fmaf(f, sum[i], acc[r][i]);
                }
            }
        }
    }
#pragma unroll
    for (int r = 0; r < RT; ++r) *reinterpret_cast<f32x4*>(sums + ((wave * RT + r) * 64 + lane) * 4) = acc[r];
    __syncthreads();
    // an output a thread: [tile of rows][quarter][row of x][row in the quarter]
    for (int id = threadIdx.x; id < RT * 256; id += blockDim.x) {
        const int64_t j = (static_cast<int64_t>(blockIdx.x) * RT + id / 256) * 16 + id % 256 / 64 * 4 + id % 4;
        const int64_t m = static_cast<int64_t>(blockIdx.y) * kTokens + id % 64 / 4;
        if (m >= a.M || j >= w.rows) continue;
        float s = 0.0f;
        for (int k = 0; k < waves; ++k) s += sums[k * RT * 256 + id];
        if (XD == 3 && !XG) s *= a.x_scales[m];
        const int64_t at = m * a.ldy + j;
        if (a.y_dtype == 0) static_cast<float*>(a.y)[at] = s;
        else if (a.y_dtype == 1) static_cast<_Float16*>(a.y)[at] = Storage<_Float16>::from_f32(s);
        else static_cast<bf16_t*>(a.y)[at] = Storage<bf16_t>::from_f32(s);
    }
}

// Each thread's first item of all the launch's and the number of its threads: more items
// than HIP takes threads are taken in turns.
struct Turns {
    int64_t first, stride;
};
__device__ __forceinline__ Turns turns() {
    return {static_cast<int64_t>(blockIdx.x) * kW4Threads + threadIdx.x, static_cast<int64_t>(gridDim.x) * kW4Threads};
}
unsigned blocks_for(int64_t items) {
    return static_cast<unsigned>(std::min<int64_t>((items + kW4Threads - 1) / kW4Threads, 0xffffffffLL / kW4Threads));
}

// One thread per group of a row (padding rows too).  Plain kernels, since matrices are made
// once: 4096 x 25088 from bf16 3.2 ms, from codes 0.09 ms, back into bf16 0.13 ms (4096 x
// 4096: 135, 20 and 26 us).
template <typename Elem>
__global__ __launch_bounds__(kW4Threads) void quantize_kernel(W4 w, const Elem* m, int64_t ldm, int64_t items) {
    const int64_t groups = w.ktiles * 128 / w.group;
    const Turns t = turns();
    for (int64_t id = t.first; id < items; id += t.stride) {
        const int64_t j = id / groups, g = id % groups;
        auto value = [&](int64_t c) {
            return j < w.rows && c < w.cols ? Storage<Elem>::to_f32(m[j * ldm + c]) : 0.0f;
        };
        uint32_t top = 0;   // the largest |value|'s bits: ascending with it, NaN last
        for (int64_t c = g * w.group; c < (g + 1) * w.group; ++c) top = max(top, __float_as_uint(value(c)) & 0x7fffffffu);
        // a group with NaN or an infinity has no scale, and stays recognisable: all of it is NaN
        const bool finite = top < 0x7f800000u;
        const bf16_t scale = finite ? Storage<bf16_t>::from_f32(__uint_as_float(top) / 7.0f) : bf16_t{0x7fc0};
        const float s = finite ? Storage<bf16_t>::to_f32(scale) : 0.0f;
        if (g < w.groups) w.scales[scale_at(w, j, g)] = scale;
        for (int64_t c = g * w.group; c < (g + 1) * w.group; c += 8) {
            int code[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float q = s > 0.0f ? rintf(value(c + e) / s) : 0.0f;
                code[e] = static_cast<int>(fminf(fmaxf(q, -7.0f), 7.0f)) + 8;
            }
            w.codes[word_at(w, j, c)] = pack8(code);
        }
    }
}

// One thread per word (of padding rows and columns too).
__global__ __launch_bounds__(kW4Threads) void pack_kernel(W4 w, const uint8_t* nibbles, const bf16_t* scales, int64_t items) {
    const int64_t words = w.ktiles * 16, ld = (w.cols + 1) / 2;
    const Turns t = turns();
    for (int64_t id = t.first; id < items; id += t.stride) {
        const int64_t j = id / words, c = id % words * 8;
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
}

template <typename Elem>
__global__ __launch_bounds__(kW4Threads) void dequantize_kernel(W4 w, Elem* m, int64_t ldm, int64_t items) {
    const int64_t words = (w.cols + 7) / 8;
    const Turns t = turns();
    for (int64_t id = t.first; id < items; id += t.stride) {
        const int64_t j = id / words, c = id % words * 8;
        const uint32_t word = w.codes[word_at(w, j, c)];
        const float s = Storage<bf16_t>::to_f32(w.scales[scale_at(w, j, c / w.group)]);
        for (int e = 0; e < 8 && c + e < w.cols; ++e)
            m[j * ldm + c + e] = Storage<Elem>::from_f32(static_cast<float>(code_of(word, e) - 8) * s);
    }
}

// HIP takes fewer than 2^32 threads along x and 2^16 workgroups along y: larger products
// go in several launches, of rows of the matrix and of x.
template <int XD, int GPT, bool XG, int RT> hipError_t matvec_r(const MatvecArgs& k, hipStream_t stream) {
    const int waves = static_cast<int>(k.w.ktiles < 16 ? k.w.ktiles : 16);
    const int64_t rows = int64_t(0xffffffff) / (waves * 64) * (16 * RT), tokens = int64_t(0xffff) * kTokens;
    const int64_t xs = sizeof(typename XTypeOf<XD>::type), ys = dtype_bytes(k.y_dtype);
    for (int64_t m = 0; m < k.M; m += tokens)
        for (int64_t j = 0; j < k.w.rows; j += rows) {
            MatvecArgs a = k;
            a.M = std::min(k.M - m, tokens);
            a.x = static_cast<const char*>(k.x) + m * k.ldx * xs;
            if (k.x_scales) a.x_scales = k.x_scales + m * k.x_groups;
            a.y = static_cast<char*>(k.y) + (m * k.ldy + j) * ys;
            a.w.rows = std::min(k.w.rows - j, rows);
            a.w.codes = k.w.codes + j * k.w.ktiles * 16;   // 16 words a row of a tile
            a.w.scales = k.w.scales + j * k.w.groups;
            const dim3 grid(static_cast<unsigned>((a.w.rows + 16 * RT - 1) / (16 * RT)),
                            static_cast<unsigned>((a.M + kTokens - 1) / kTokens));
            matvec_kernel<XD, GPT, XG, RT><<<grid, waves * 64, waves * RT * 256 * sizeof(float), stream>>>(a);
        }
    return hipGetLastError();
}
template <int XD, int GPT, bool XG> hipError_t matvec_t(const MatvecArgs& k, hipStream_t stream) {
    // Two tiles of rows a workgroup where one each would be more workgroups than the
    // chip has units, of which one holds one workgroup of sixteen waves at these
    // registers: the second round of them is gone, and x is read half as often.
    // One, then two: 4096 -> 5000 for one bf16 row 7.4, 6.1 us, for sixteen 12.1, 8.4;
    // 4096 -> 32768 24.1, 20.4 and 41.1, 26.9; 1000 -> 12000 5.9, 4.9.  With fewer workgroups
    // units are left idle (4096 -> 4096 4.8, 6.0); with fewer than eight waves more
    // workgroups share a unit (512 -> 8192 3.6, 3.9); fp32 rows with groups of 32 spill
    // 28 registers (4096 -> 5000 15.2, 16.6).
    if constexpr (XD != 0 || GPT != 4)
        if (k.w.ktiles >= 8 && (k.w.rows + 15) / 16 * ((k.M + kTokens - 1) / kTokens) > device_cu_count())
            return matvec_r<XD, GPT, XG, 2>(k, stream);
    return matvec_r<XD, GPT, XG, 1>(k, stream);
}
template <int XD, bool XG> hipError_t matvec_x(const MatvecArgs& k, hipStream_t stream) {
    return k.w.group == 32 ? matvec_t<XD, 4, XG>(k, stream)
                           : k.w.group == 64 ? matvec_t<XD, 2, XG>(k, stream) : matvec_t<XD, 1, XG>(k, stream);
}

}  // namespace

hipError_t launch_matvec_w4(const wg_matvec_w4& a, hipStream_t stream) {
    const MatvecArgs k{w4_of(a.w), a.M, a.x, a.ldx, a.x_scales, a.x_groups, a.y, a.ldy, static_cast<int>(a.y_dtype)};
    switch (a.x_dtype) {
        case WG_F32: return matvec_x<0, false>(k, stream);
        case WG_F16: return matvec_x<1, false>(k, stream);
        case WG_BF16: return matvec_x<2, false>(k, stream);
        // one group: its scale is the row's
        default: return a.x_groups > 1 ? matvec_x<3, true>(k, stream) : matvec_x<3, false>(k, stream);
    }
}

template <int D> hipError_t launch_quantize_w4_t(const wg_w4& w, const void* m, int64_t ldm, hipStream_t stream) {
    using Elem = typename DTypeOf<D>::type;
    const W4 k = w4_of(w);
    const int64_t items = (w.rows + 15) / 16 * 16 * (k.ktiles * 128 / w.group);
    quantize_kernel<Elem><<<blocks_for(items), kW4Threads, 0, stream>>>(k, static_cast<const Elem*>(m), ldm, items);
    return hipGetLastError();
}

template <int D> hipError_t launch_dequantize_w4_t(const wg_w4& w, void* m, int64_t ldm, hipStream_t stream) {
    using Elem = typename DTypeOf<D>::type;
    const int64_t items = w.rows * ((w.cols + 7) / 8);
    dequantize_kernel<Elem><<<blocks_for(items), kW4Threads, 0, stream>>>(w4_of(w), static_cast<Elem*>(m), ldm, items);
    return hipGetLastError();
}

hipError_t launch_pack_w4(const wg_w4& w, const void* nibbles, const void* scales, hipStream_t stream) {
    const W4 k = w4_of(w);
    const int64_t items = (w.rows + 15) / 16 * 16 * (k.ktiles * 16);
    pack_kernel<<<blocks_for(items), kW4Threads, 0, stream>>>(k, static_cast<const uint8_t*>(nibbles),
                                                              static_cast<const bf16_t*>(scales), items);
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
