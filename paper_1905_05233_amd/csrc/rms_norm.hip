// The root-mean-square norm of rows with the residual's addition, its output in
// the storage type or in 8 bits with scales, and its gradients, on gfx950:
//   r = x + residual,  y = r rstd weight,  rstd = 1 / sqrt(mean(r^2) + eps)
//   dr_total = rstd (g - r rstd^2 mean(g r)) + dr  with g = dy weight,
//   dweight = sum over the rows of dy r rstd.
// Sums and statistics in fp32.
//
// Memory bounds all of it, so a row is read once: TPR threads (2 to 1024, by the
// row's length) hold it in registers, NV runs of 16 bytes each, reduce over lanes
// (and LDS, over waves), and write.  Workgroups walk rows with the weights in
// registers; the gradients' workgroups also keep their share of dweight there and
// leave it in the workspace, [workgroup][C], which a second kernel sums in a fixed
// order.  Rows too long for that are read twice (three times by the gradients).
//
// 65536 rows of 512 bf16 with the residual into 8 bits with scales for every 128
// channels, 236 MB: 46 us in replayed graphs, 5.1 TB/s (a copy of 1 GiB 5.2), 50 a call;
// their gradients, 268 MB: 54 us for both kernels, 5.0 TB/s.  Rows that are no whole runs
// of 16 bytes start at odd addresses: 511 channels instead of 512 take 57 us instead of
// 46.  3001 rows of 1000 fp16, 24 MB: 6.3 us.  A few rows take 3.1 us, a launch's latency
// and a row's.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>

#include "device_common.hpp"
#include "kernels.hpp"
#include "rows.hpp"
#include "sequence.hpp"

namespace wg {

namespace {

constexpr int kNormThreads = 256;
constexpr float kFp8Max = 448.0f;            // largest value of e4m3
constexpr float kFp8Least = 0x1p-100f;       // absolute maxima below this count as this

// Rows [N][L][C] numbered n * L + l.
struct RowsAt {
    void* data;
    int64_t sn, sl;
};
struct RowIndex {
    int64_t L;   // 0: the rows of every tensor are evenly spaced, as one sequence
};
template <typename T> __device__ __forceinline__ T* row_at(const RowsAt& r, const RowIndex& ix, int64_t row) {
    T* p = static_cast<T*>(r.data);
    if (ix.L == 0) return p + row * r.sl;
    int64_t n, l;
    if (row >> 32 == 0 && ix.L >> 32 == 0) {
        const uint32_t q = static_cast<uint32_t>(row) / static_cast<uint32_t>(ix.L);
        n = q;
        l = static_cast<uint32_t>(row) - q * static_cast<uint32_t>(ix.L);
    } else {
        n = row / ix.L;
        l = row - n * ix.L;
    }
    return p + n * r.sn + l * r.sl;
}

template <typename Elem> struct NormArgs {
    int64_t rows, C;
    RowIndex index;
    RowsAt x, residual, r, y;
    const Elem* weight;
    float* scales;
    float eps;
    int64_t group;   // channels a scale covers
};

__device__ __forceinline__ uint8_t e4m3_of(float v) {
    return static_cast<uint8_t>(__builtin_amdgcn_cvt_pk_fp8_f32(v, 0.0f, 0, false));
}
// V values as e4m3 bytes
template <int V> __device__ __forceinline__ void store_e4m3(uint8_t* p, int valid, const float (&f)[V]) {
    uint32_t w[V / 4];
#pragma unroll
    for (int q = 0; q < V; q += 4) {
        int b = __builtin_amdgcn_cvt_pk_fp8_f32(f[q], f[q + 1], 0, false);
        b = __builtin_amdgcn_cvt_pk_fp8_f32(f[q + 2], f[q + 3], b, true);
        w[q / 4] = static_cast<uint32_t>(b);
    }
    if (valid == V) {
        __builtin_memcpy(p, w, V);
    } else {
#pragma unroll
        for (int q = 0; q < V; ++q)
            if (q < valid) p[q] = static_cast<uint8_t>(w[q / 4] >> (q % 4 * 8));
    }
}

// A scale's range: `most` is |y|'s largest bit pattern (ascending with |y|, NaN last).
__device__ __forceinline__ float scale_of(uint32_t most) {
    const float m = __uint_as_float(most);
    return (m < kFp8Least ? kFp8Least : m) / kFp8Max;
}

// Quotients by a scale: the product with 1 / s, corrected by what it leaves of y.
// Alone the product is up to 1.5 units of the last place off, which moves quotients at the
// ties of the 8-bit rounding; corrected they are exact there.  (65536 rows of 512: 45 us
// with the product alone, 46 with this, 48 with the compiler's division.)
struct ByScale {
    float inv, s;   // s 0 where it is infinite: finite values are 0 then
    __device__ __forceinline__ explicit ByScale(float scale) : inv(1.0f / scale), s(inv == 0.0f ? 0.0f : scale) {}
    __device__ __forceinline__ float operator()(float y) const {
        const float q = y * inv;
        return fmaf(-fmaf(q, s, -y), inv, q);   // in these signs -0 stays -0
    }
};

// FULL: the row's channels are whole runs.
template <typename Elem, bool FULL> __device__ __forceinline__ u32x4 load_one(const Elem* p, const RunShape& shape, int C) {
    u32x4 bits[1]{};
    const Elem* const at[1] = {p};
    if (shape.valid) load_runs<Elem, FULL, 1>(at, shape, C, bits);
    return bits[0];
}

// Reductions over a row's TPR threads; above a wave through LDS, by all threads of
// the workgroup, which then holds one row.  `slot` alternates between calls, so
// that one barrier a call is enough.
template <int TPR> struct RowReduce {
    static constexpr int kWaves = TPR > 64 ? TPR / 64 : 1;
    static __device__ __forceinline__ float sum(float v, float (*lds)[16], int slot) {
        v = lanes_sum<(TPR < 64 ? TPR : 64)>(v);
        if constexpr (kWaves > 1) {
            if (threadIdx.x % 64 == 0) lds[slot][threadIdx.x / 64] = v;
            __syncthreads();
            v = 0.0f;
#pragma unroll
            for (int w = 0; w < kWaves; ++w) v += lds[slot][w];
        }
        return v;
    }
    static __device__ __forceinline__ uint32_t max(uint32_t v, float (*lds)[16], int slot) {
        v = lanes_max<(TPR < 64 ? TPR : 64)>(v);
        if constexpr (kWaves > 1) {
            if (threadIdx.x % 64 == 0) lds[slot][threadIdx.x / 64] = __uint_as_float(v);
            __syncthreads();
            v = 0;
#pragma unroll
            for (int w = 0; w < kWaves; ++w) {
                const uint32_t o = __float_as_uint(lds[slot][w]);
                v = v > o ? v : o;
            }
        }
        return v;
    }
};

constexpr int block_of(int tpr) { return tpr > kNormThreads ? tpr : kNormThreads; }

template <typename Elem, int TPR, int NV, bool FULL, bool QUANT>
__global__ __launch_bounds__(block_of(TPR)) void norm_kernel(NormArgs<Elem> a) {
    constexpr int V = Vec<Elem>::V, ROWS = block_of(TPR) / TPR;
    __shared__ float lds[4][16];
    const int lane = threadIdx.x % TPR;
    const int C = static_cast<int>(a.C);
    RunShape shape[NV];
    float w[NV][V];
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        const int c = (j * TPR + lane) * V;
        shape[j] = run_shape<Elem>(c, C);
        Vec<Elem>::widen(load_one<Elem, FULL>(a.weight + c, shape[j], C), w[j]);
    }
    int slot = 0;
    for (int64_t row = static_cast<int64_t>(blockIdx.x) * ROWS + threadIdx.x / TPR; row < a.rows;
         row += static_cast<int64_t>(gridDim.x) * ROWS, slot ^= 2) {
        const Elem* x = row_at<const Elem>(a.x, a.index, row);
        float r[NV][V];
        u32x4 raw[NV], raw2[NV];
#pragma unroll
        for (int j = 0; j < NV; ++j) raw[j] = load_one<Elem, FULL>(x + (j * TPR + lane) * V, shape[j], C);
        if (a.residual.data) {
            const Elem* res = row_at<const Elem>(a.residual, a.index, row);
#pragma unroll
            for (int j = 0; j < NV; ++j) raw2[j] = load_one<Elem, FULL>(res + (j * TPR + lane) * V, shape[j], C);
        }
        float ss = 0.0f;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            Vec<Elem>::widen(raw[j], r[j]);
            if (a.residual.data) {
                float f[V];
                Vec<Elem>::widen(raw2[j], f);
#pragma unroll
                for (int q = 0; q < V; ++q) r[j][q] += f[q];
            }
#pragma unroll
            for (int q = 0; q < V; ++q) ss = fmaf(r[j][q], r[j][q], ss);
        }
        if (a.r.data) {
            Elem* out = row_at<Elem>(a.r, a.index, row);
#pragma unroll
            for (int j = 0; j < NV; ++j)
                if (shape[j].valid) store_run<Elem, FULL>(out + (j * TPR + lane) * V, shape[j].valid, Vec<Elem>::narrow(r[j]));
        }
        ss = RowReduce<TPR>::sum(ss, lds, slot);
        const float rstd = 1.0f / sqrtf(ss / static_cast<float>(C) + a.eps);
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
            for (int q = 0; q < V; ++q) r[j][q] = r[j][q] * rstd * w[j][q];
        if constexpr (!QUANT) {
            Elem* y = row_at<Elem>(a.y, a.index, row);
#pragma unroll
            for (int j = 0; j < NV; ++j)
                if (shape[j].valid) store_run<Elem, FULL>(y + (j * TPR + lane) * V, shape[j].valid, Vec<Elem>::narrow(r[j]));
        } else {
            uint32_t top[NV];
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                top[j] = 0;
#pragma unroll
                for (int q = 0; q < V; ++q) {   // channels past the row's end hold zeros
                    const uint32_t v = __float_as_uint(r[j][q]) & 0x7fffffffu;
                    top[j] = q < shape[j].valid && v > top[j] ? v : top[j];
                }
            }
            uint8_t* y = row_at<uint8_t>(a.y, a.index, row);
            if (a.group == a.C) {
                uint32_t m = top[0];
#pragma unroll
                for (int j = 1; j < NV; ++j) m = top[j] > m ? top[j] : m;
                m = RowReduce<TPR>::max(m, lds, slot + 1);
                const float scale = scale_of(m);
                const ByScale code(scale);
                if (lane == 0) a.scales[row] = scale;
#pragma unroll
                for (int j = 0; j < NV; ++j) {
#pragma unroll
                    for (int q = 0; q < V; ++q) r[j][q] = code(r[j][q]);
                    if (shape[j].valid) store_e4m3<V>(y + (j * TPR + lane) * V, shape[j].valid, r[j]);
                }
            } else {
                // a group is 4 to 32 adjacent threads, all of a row's waves' own
                const int per = static_cast<int>(a.group) / V;
                const int64_t groups = (a.C + a.group - 1) / a.group;
#pragma unroll
                for (int j = 0; j < NV; ++j) {
                    uint32_t m = lanes_max<4>(top[j]), o;
                    if (per > 4) o = other_half<8>(m), m = o > m ? o : m;
                    if (per > 8) o = other_half<16>(m), m = o > m ? o : m;
                    if (per > 16) o = other_half<32>(m), m = o > m ? o : m;
                    const float scale = scale_of(m);
                    const ByScale code(scale);
                    const int c = (j * TPR + lane) * V;
                    if (lane % per == 0 && shape[j].valid) a.scales[row * groups + c / static_cast<int>(a.group)] = scale;
#pragma unroll
                    for (int q = 0; q < V; ++q) r[j][q] = code(r[j][q]);
                    if (shape[j].valid) store_e4m3<V>(y + c, shape[j].valid, r[j]);
                }
            }
        }
    }
}

// Sum over a workgroup of kNormThreads, the same value in every thread.
__device__ __forceinline__ float block_sum(float v, float* lds) {
    v = lanes_sum<64>(v);
    if (threadIdx.x % 64 == 0) lds[threadIdx.x / 64] = v;
    __syncthreads();
    v = lds[0] + lds[1] + lds[2] + lds[3];
    __syncthreads();
    return v;
}

// Rows of any length, one workgroup each, read again for the output.  A plain form for
// what the registers do not hold: 300 rows of 40000 bf16 with the residual take 174 us,
// into 8 bits with a scale a row 243, with scales for every 32 channels, two barriers
// each, 1200 (a floor of 16 to 18); their gradients 275.
template <typename Elem, bool QUANT>
__global__ __launch_bounds__(kNormThreads) void norm_long_kernel(NormArgs<Elem> a) {
    using S = Storage<Elem>;
    __shared__ float lds[kNormThreads / 64];
    __shared__ uint32_t tops[kNormThreads / 64];
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const Elem* x = row_at<const Elem>(a.x, a.index, row);
        const Elem* res = a.residual.data ? row_at<const Elem>(a.residual, a.index, row) : nullptr;
        auto sum_at = [&](int64_t c) { return S::to_f32(x[c]) + (res ? S::to_f32(res[c]) : 0.0f); };
        float ss = 0.0f;
        for (int64_t c = threadIdx.x; c < a.C; c += kNormThreads) {
            const float v = sum_at(c);
            ss = fmaf(v, v, ss);
        }
        const float rstd = 1.0f / sqrtf(block_sum(ss, lds) / static_cast<float>(a.C) + a.eps);
        if constexpr (!QUANT) {
            Elem* y = row_at<Elem>(a.y, a.index, row);
            for (int64_t c = threadIdx.x; c < a.C; c += kNormThreads)
                y[c] = S::from_f32(sum_at(c) * rstd * S::to_f32(a.weight[c]));
        } else {
            uint8_t* y = row_at<uint8_t>(a.y, a.index, row);
            const int64_t groups = (a.C + a.group - 1) / a.group;
            for (int64_t g = 0; g < groups; ++g) {
                const int64_t end = min(a.C, (g + 1) * a.group);
                uint32_t top = 0;
                for (int64_t c = g * a.group + threadIdx.x; c < end; c += kNormThreads)
                    top = max(top, __float_as_uint(sum_at(c) * rstd * S::to_f32(a.weight[c])) & 0x7fffffffu);
                top = lanes_max<64>(top);
                if (threadIdx.x % 64 == 0) tops[threadIdx.x / 64] = top;
                __syncthreads();
                const float scale = scale_of(max(max(tops[0], tops[1]), max(tops[2], tops[3])));
                const ByScale code(scale);
                __syncthreads();
                for (int64_t c = g * a.group + threadIdx.x; c < end; c += kNormThreads)
                    y[c] = e4m3_of(code(sum_at(c) * rstd * S::to_f32(a.weight[c])));
                if (threadIdx.x == 0) a.scales[row * groups + g] = scale;
            }
        }
        if (a.r.data) {   // last, and every thread its own channels: r may be x itself
            Elem* r = row_at<Elem>(a.r, a.index, row);
            __syncthreads();   // channels of groups are read by other threads than these
            for (int64_t c = threadIdx.x; c < a.C; c += kNormThreads) r[c] = S::from_f32(sum_at(c));
        }
    }
}

template <typename Elem> struct NormGradArgs {
    int64_t rows, C;
    RowIndex index;
    RowsAt dy, r, dr, dx;
    const Elem* weight;
    float* dweight;
    float eps;
    float* partial;   // dweight's parts [parts][C]
    int64_t parts;
    float* rstd;      // of long rows, one a row
};

template <typename Elem, int TPR, int NV, bool FULL>
__global__ __launch_bounds__(block_of(TPR)) void norm_grad_kernel(NormGradArgs<Elem> a) {
    constexpr int V = Vec<Elem>::V, ROWS = block_of(TPR) / TPR;
    __shared__ float lds[4][16];
    __shared__ float share[ROWS > 1 ? ROWS * TPR * NV * V : 1];
    const int lane = threadIdx.x % TPR;
    const int C = static_cast<int>(a.C);
    RunShape shape[NV];
    float w[NV][V], dw[NV][V];
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        const int c = (j * TPR + lane) * V;
        shape[j] = run_shape<Elem>(c, C);
        Vec<Elem>::widen(load_one<Elem, FULL>(a.weight + c, shape[j], C), w[j]);
#pragma unroll
        for (int q = 0; q < V; ++q) dw[j][q] = 0.0f;
    }
    int slot = 0;
    for (int64_t row = static_cast<int64_t>(blockIdx.x) * ROWS + threadIdx.x / TPR; row < a.rows;
         row += static_cast<int64_t>(gridDim.x) * ROWS, slot ^= 2) {
        const Elem* rp = row_at<const Elem>(a.r, a.index, row);
        const Elem* dp = row_at<const Elem>(a.dy, a.index, row);
        u32x4 rr[NV], dd[NV], ee[NV];
#pragma unroll
        for (int j = 0; j < NV; ++j) rr[j] = load_one<Elem, FULL>(rp + (j * TPR + lane) * V, shape[j], C);
#pragma unroll
        for (int j = 0; j < NV; ++j) dd[j] = load_one<Elem, FULL>(dp + (j * TPR + lane) * V, shape[j], C);
        if (a.dr.data) {
            const Elem* ep = row_at<const Elem>(a.dr, a.index, row);
#pragma unroll
            for (int j = 0; j < NV; ++j) ee[j] = load_one<Elem, FULL>(ep + (j * TPR + lane) * V, shape[j], C);
        }
        float r[NV][V], d[NV][V];
        float ss = 0.0f, gr = 0.0f;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            Vec<Elem>::widen(rr[j], r[j]);
            Vec<Elem>::widen(dd[j], d[j]);
#pragma unroll
            for (int q = 0; q < V; ++q) {
                ss = fmaf(r[j][q], r[j][q], ss);
                gr = fmaf(d[j][q] * w[j][q], r[j][q], gr);
            }
        }
        ss = RowReduce<TPR>::sum(ss, lds, slot);
        gr = RowReduce<TPR>::sum(gr, lds, slot + 1);
        const float rstd = 1.0f / sqrtf(ss / static_cast<float>(C) + a.eps);
        const float mean = gr / static_cast<float>(C) * rstd * rstd;
        Elem* out = row_at<Elem>(a.dx, a.index, row);
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            float o[V], e[V];
            if (a.dr.data) Vec<Elem>::widen(ee[j], e);
#pragma unroll
            for (int q = 0; q < V; ++q) {
                dw[j][q] = fmaf(d[j][q], r[j][q] * rstd, dw[j][q]);
                o[q] = rstd * (d[j][q] * w[j][q] - r[j][q] * mean);
                if (a.dr.data) o[q] += e[q];
            }
            if (shape[j].valid) store_run<Elem, FULL>(out + (j * TPR + lane) * V, shape[j].valid, Vec<Elem>::narrow(o));
        }
    }
    float* part = a.partial + static_cast<int64_t>(blockIdx.x) * a.C;
    if constexpr (ROWS == 1) {
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
            for (int q = 0; q < V; ++q)
                if (q < shape[j].valid) part[(j * TPR + lane) * V + q] = dw[j][q];
    } else {
        constexpr int W = TPR * NV * V;   // channels' room of a row
        const int mine = static_cast<int>(threadIdx.x) / TPR;
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
            for (int q = 0; q < V; ++q) share[mine * W + (j * TPR + lane) * V + q] = dw[j][q];
        __syncthreads();
        for (int c = threadIdx.x; c < C; c += block_of(TPR)) {
            float s = 0.0f;
#pragma unroll
            for (int k = 0; k < ROWS; ++k) s += share[k * W + c];
            part[c] = s;
        }
    }
}

// dweight from its parts: 16 channels a workgroup, the parts over 64 threads a
// channel, eight of them in flight (1280 parts of 512 channels, 2.6 MB: 4.8 us).
__global__ __launch_bounds__(1024) void norm_parts_kernel(const float* partial, int64_t parts, int64_t C, float* dweight) {
    constexpr int kChannels = 16, kSlices = 64;
    __shared__ float lds[kSlices][kChannels + 1];
    const int64_t c = static_cast<int64_t>(blockIdx.x) * kChannels + threadIdx.x % kChannels;
    const int k = threadIdx.x / kChannels;
    float s = 0.0f;
    if (c < C)
        for (int64_t p = k; p < parts; p += 8 * kSlices) {
            float v[8];
#pragma unroll
            for (int u = 0; u < 8; ++u) v[u] = p + u * kSlices < parts ? partial[(p + u * kSlices) * C + c] : 0.0f;
#pragma unroll
            for (int u = 0; u < 8; ++u) s += v[u];
        }
    lds[k][threadIdx.x % kChannels] = s;
    __syncthreads();
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;   // a wave a channel
    s = lanes_sum<64>(lds[lane][wave]);
    const int64_t out = static_cast<int64_t>(blockIdx.x) * kChannels + wave;
    if (lane == 0 && out < C) dweight[out] = s;
}

// The gradients of rows of any length (longer than 16384 fp32 or 32768 16-bit values): 1 / sqrt of each row, dweight's parts by
// columns, then dx, which may be dy.
template <typename Elem>
__global__ __launch_bounds__(kNormThreads) void norm_rstd_kernel(NormGradArgs<Elem> a) {
    using S = Storage<Elem>;
    __shared__ float lds[kNormThreads / 64];
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const Elem* r = row_at<const Elem>(a.r, a.index, row);
        float ss = 0.0f;
        for (int64_t c = threadIdx.x; c < a.C; c += kNormThreads) ss = fmaf(S::to_f32(r[c]), S::to_f32(r[c]), ss);
        ss = block_sum(ss, lds);
        if (threadIdx.x == 0) a.rstd[row] = 1.0f / sqrtf(ss / static_cast<float>(a.C) + a.eps);
    }
}
template <typename Elem>
__global__ __launch_bounds__(kNormThreads) void norm_columns_kernel(NormGradArgs<Elem> a) {
    using S = Storage<Elem>;
    const int64_t c = static_cast<int64_t>(blockIdx.x) * kNormThreads + threadIdx.x;
    if (c >= a.C) return;
    float sum = 0.0f;
    for (int64_t row = blockIdx.y; row < a.rows; row += gridDim.y)
        sum = fmaf(S::to_f32(row_at<const Elem>(a.dy, a.index, row)[c]),
                   S::to_f32(row_at<const Elem>(a.r, a.index, row)[c]) * a.rstd[row], sum);
    a.partial[blockIdx.y * a.C + c] = sum;
}
template <typename Elem>
__global__ __launch_bounds__(kNormThreads) void norm_grad_long_kernel(NormGradArgs<Elem> a) {
    using S = Storage<Elem>;
    __shared__ float lds[kNormThreads / 64];
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const Elem* r = row_at<const Elem>(a.r, a.index, row);
        const Elem* dy = row_at<const Elem>(a.dy, a.index, row);
        const Elem* dr = a.dr.data ? row_at<const Elem>(a.dr, a.index, row) : nullptr;
        Elem* dx = row_at<Elem>(a.dx, a.index, row);
        float gr = 0.0f;
        for (int64_t c = threadIdx.x; c < a.C; c += kNormThreads)
            gr = fmaf(S::to_f32(dy[c]) * S::to_f32(a.weight[c]), S::to_f32(r[c]), gr);
        const float rstd = a.rstd[row];
        const float mean = block_sum(gr, lds) / static_cast<float>(a.C) * rstd * rstd;
        for (int64_t c = threadIdx.x; c < a.C; c += kNormThreads) {
            float d = rstd * (S::to_f32(dy[c]) * S::to_f32(a.weight[c]) - S::to_f32(r[c]) * mean);
            if (dr) d += S::to_f32(dr[c]);
            dx[c] = S::from_f32(d);
        }
    }
}

// Rows evenly spaced over all sequences in every tensor used are taken as one sequence's.
template <typename... R> RowIndex index_of(int64_t N, int64_t L, const R&... rows) {
    const bool even = N == 1 || ((!rows.data || rows.stride_n == L * rows.stride_l) && ...);
    return {even ? 0 : L};
}
RowsAt at(const wg_rows& r) { return {const_cast<void*>(r.data), r.stride_n, r.stride_l}; }

// Threads a row and 16-byte runs a thread: the fewest threads that hold the row in
// one run each up to a wave, then in two or four.
struct Shape {
    int tpr, nv;   // tpr 0: too long
};
Shape shape_of(int dtype, int64_t C) {
    const int64_t runs = (C + 16 / dtype_bytes(dtype) - 1) / (16 / dtype_bytes(dtype));
    if (runs <= 2) return {2, 1};
    if (runs <= 4) return {4, 1};
    if (runs <= 8) return {8, 1};
    if (runs <= 16) return {16, 1};
    if (runs <= 32) return {32, 1};
    if (runs <= 64) return {64, 1};
    if (runs <= 128) return {64, 2};
    if (runs <= 256) return {64, 4};
    if (runs <= 512) return {256, 2};
    if (runs <= 1024) return {256, 4};
    if (runs <= 2048) return {1024, 2};
    if (runs <= 4096) return {1024, 4};
    return {0, 0};
}
#define WG_NORM_SHAPES(X) X(2, 1) X(4, 1) X(8, 1) X(16, 1) X(32, 1) X(64, 1) X(64, 2) X(64, 4) X(256, 2) X(256, 4) X(1024, 2) X(1024, 4)

// Workgroups that walk the rows: as many as are resident at a time, by the registers
// that NV runs a thread take (the norm at most 64, 102 and 170 of them, its gradients
// 102, 170 and 256).  More would leave a second, mostly empty round: gradients of 38759
// rows of 516 bf16, 138 registers, take 83 us with four workgroups a compute unit and
// 64 with three; of 4882 rows of 4096, 51 and 44.
int64_t walkers(int64_t rows, int tpr, int per_cu) {
    const int block = block_of(tpr), per = block / tpr;
    const int64_t resident = int64_t(device_cu_count()) * std::max(1, per_cu * 256 / block);
    return std::max<int64_t>(1, std::min<int64_t>((rows + per - 1) / per, resident));
}
constexpr int norm_per_cu(int nv) { return nv == 1 ? 8 : nv == 2 ? 5 : 3; }
constexpr int grad_per_cu(int nv) { return nv == 1 ? 5 : nv == 2 ? 3 : 2; }

// The gradients' workgroups.  A few rows are one workgroup's, whose dweight is the
// whole of it: a round of rows takes some 1 us there, the second launch and its
// workspace 5 us of the host's time.
constexpr int64_t kOneRounds = 4;
int64_t grad_walkers(int64_t rows, const Shape& s) {
    return rows <= kOneRounds * (block_of(s.tpr) / s.tpr) ? 1 : walkers(rows, s.tpr, grad_per_cu(s.nv));
}
constexpr int64_t kLongBlocks = 4096, kColumnParts = 64;

}  // namespace

// dweight's parts (one part is dweight), and behind them, for long rows, the rows' 1 / sqrt.
size_t rms_norm_workspace(int dtype, int64_t N, int64_t L, int64_t C) {
    const Shape s = shape_of(dtype, C);
    const int64_t rows = N * L;
    if (s.tpr) {
        const int64_t parts = grad_walkers(rows, s);
        return parts == 1 ? 0 : static_cast<size_t>((parts * C * 4 + 15) / 16 * 16);
    }
    return static_cast<size_t>(((std::min(rows, kColumnParts) * C + rows) * 4 + 15) / 16 * 16 + 16);
}

template <int D> hipError_t launch_rms_norm_t(const wg_rms_norm& a, hipStream_t stream) {
    using Elem = typename DTypeOf<D>::type;
    const int64_t rows = a.N * a.L;
    const NormArgs<Elem> k{rows, a.C, index_of(a.N, a.L, a.x, a.residual, a.r, a.y), at(a.x), at(a.residual), at(a.r),
                           at(a.y), static_cast<const Elem*>(a.weight), a.scales, static_cast<float>(a.eps),
                           a.group && a.group < a.C ? a.group : a.C};
    const bool quant = a.y_dtype == WG_E4M3, full = a.C % Vec<Elem>::V == 0;
    const Shape s = shape_of(D, a.C);
    const unsigned blocks = static_cast<unsigned>(s.tpr ? walkers(rows, s.tpr, norm_per_cu(s.nv)) : std::min(rows, kLongBlocks));
#define WG_NORM_CASE(TPR, NV)                                                                     \
    if (s.tpr == TPR && s.nv == NV) {                                                             \
        const unsigned threads = block_of(TPR);                                                   \
        if (full && quant) norm_kernel<Elem, TPR, NV, true, true><<<blocks, threads, 0, stream>>>(k);   \
        else if (full) norm_kernel<Elem, TPR, NV, true, false><<<blocks, threads, 0, stream>>>(k);      \
        else if (quant) norm_kernel<Elem, TPR, NV, false, true><<<blocks, threads, 0, stream>>>(k);     \
        else norm_kernel<Elem, TPR, NV, false, false><<<blocks, threads, 0, stream>>>(k);         \
        return hipGetLastError();                                                                 \
    }
    WG_NORM_SHAPES(WG_NORM_CASE)
#undef WG_NORM_CASE
    if (quant) norm_long_kernel<Elem, true><<<blocks, kNormThreads, 0, stream>>>(k);
    else norm_long_kernel<Elem, false><<<blocks, kNormThreads, 0, stream>>>(k);
    return hipGetLastError();
}

template <int D> hipError_t launch_rms_norm_backward_t(const wg_rms_norm_backward& a, hipStream_t stream) {
    using Elem = typename DTypeOf<D>::type;
    const int64_t rows = a.N * a.L;
    NormGradArgs<Elem> k{rows, a.C, index_of(a.N, a.L, a.dy, a.r, a.dr, a.dx), at(a.dy), at(a.r), at(a.dr), at(a.dx),
                         static_cast<const Elem*>(a.weight), a.dweight, static_cast<float>(a.eps),
                         static_cast<float*>(a.workspace), 0, nullptr};
    const Shape s = shape_of(D, a.C);
    const unsigned column_blocks = static_cast<unsigned>((a.C + 15) / 16);
    if (s.tpr && rows > 0) {
        k.parts = grad_walkers(rows, s);
        if (k.parts == 1) k.partial = a.dweight;
        const unsigned blocks = static_cast<unsigned>(k.parts);
#define WG_NORM_CASE(TPR, NV) \
    if (s.tpr == TPR && s.nv == NV) {                                                                             \
        if (a.C % Vec<Elem>::V == 0) norm_grad_kernel<Elem, TPR, NV, true><<<blocks, block_of(TPR), 0, stream>>>(k); \
        else norm_grad_kernel<Elem, TPR, NV, false><<<blocks, block_of(TPR), 0, stream>>>(k);                     \
    }
        WG_NORM_SHAPES(WG_NORM_CASE)
#undef WG_NORM_CASE
    } else if (rows > 0) {
        k.parts = std::min(rows, kColumnParts);
        k.rstd = k.partial + k.parts * a.C;
        const unsigned blocks = static_cast<unsigned>(std::min(rows, kLongBlocks));
        norm_rstd_kernel<Elem><<<blocks, kNormThreads, 0, stream>>>(k);
        norm_columns_kernel<Elem><<<dim3(static_cast<unsigned>((a.C + kNormThreads - 1) / kNormThreads),
                                         static_cast<unsigned>(k.parts)), kNormThreads, 0, stream>>>(k);
        norm_grad_long_kernel<Elem><<<blocks, kNormThreads, 0, stream>>>(k);
    }
    if (k.partial == a.dweight) return hipGetLastError();
    norm_parts_kernel<<<column_blocks, 1024, 0, stream>>>(k.partial, k.parts, a.C, a.dweight);
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
