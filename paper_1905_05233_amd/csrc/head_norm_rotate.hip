// The root-mean-square norm of each head of queries and keys with the rotation by their
// position, and its gradients, on gfx950.  Of a head's D channels x at position p,
//   u = x / sqrt(mean(x^2) + eps) * w,
//   y: each pair (u_a, u_b) of the first R channels as (u_a cos - u_b sin, u_a sin + u_b cos)
// of the angle p f_i of pair i; channels from R on are u.  Pairs are (i, i + R/2) or
// (2 i, 2 i + 1).  Backward, with du the rotation of dy by -p and g = du w,
//   dx = rstd (g - x rstd^2 mean(g x)),   dw = sum over rows of du x rstd.
// Sums are fp32's; y and dx are rounded once.
//
// Angles: f_i / 2 pi is held as a 64-bit fraction of a turn, so that p times it modulo
// 2^64 is the turn's fraction to p 2^-65, however far the position; its top 32 bits give
// a quarter and an angle within pi / 4 of it, whose sine and cosine are their Taylor
// series (up to the 9th and 10th power: 2 10^-9 is left).
//
// A head's row is shared by 2^n lanes, each with two runs of 16 bytes: the two halves
// of V pairs, or V pairs side by side.  The lanes keep a position's sines for its
// heads.  Bound by memory: 65536 rows of 8 and 8 heads of 64 channels in bf16 take 49 us in
// the kernel, 268 MB at 5.4 TB/s, their gradients 80 (403 MB, 5.0 TB/s).  Of odd channels,
// whose last runs hold one, by the lanes' instructions: 65536 rows of 7 heads of 75, 78 us
// where their bytes cost 27; 16 bytes that end with the row, shifted, instead of the last
// run's own loads were slower (82), and so were loads ahead of the sines (gradients 105 us
// for 91, by their registers).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>

#include "device_common.hpp"
#include "kernels.hpp"
#include "rows.hpp"
#include "sequence.hpp"

namespace wg {

namespace {

constexpr int kThreads = 256;
constexpr int kPartChannels = 16;   // of a workgroup that sums the weights' gradients

template <typename Elem> struct Heads {
    Elem* p;
    int64_t sn, sl, sh;
    __device__ __forceinline__ Elem* at(int64_t n, int64_t l, int h) const { return p + n * sn + l * sl + h * sh; }
};
template <typename Elem> Heads<Elem> heads_of(const wg_heads& t) {
    return {static_cast<Elem*>(const_cast<void*>(t.data)), t.stride_n, t.stride_l, t.stride_h};
}

template <typename Elem> struct Side {      // of queries or keys
    Heads<const Elem> x, dy;
    Heads<Elem> y;                          // or dx
    const Elem* weight;
    int32_t heads;
};

template <typename Elem> struct RotateArgs {
    Side<Elem> side[2];
    int64_t rows;                           // N L
    int32_t L, D, R, adjacent, items;       // lanes of a row that hold channels
    int32_t each, chunks;                   // heads that a group of lanes takes at a position; groups a position
    const uint64_t* turns;
    const int32_t* positions;
    int64_t start;
    float eps;
    float* parts;                           // [workgroup][2][D]
};

// cos and sin of 2 pi fraction / 2^32
__device__ __forceinline__ void cos_sin(uint32_t fraction, float& c, float& s) {
    const uint32_t quarter = (fraction + 0x20000000u) >> 30;
    const float x = static_cast<float>(static_cast<int32_t>(fraction - (quarter << 30))) * 1.46291807926715968e-9f;
    const float z = x * x;
    const float sn = fmaf(x * z, fmaf(z, fmaf(z, fmaf(z, 1.0f / 362880, -1.0f / 5040), 1.0f / 120), -1.0f / 6), x);
    const float cs = fmaf(z, fmaf(z, fmaf(z, fmaf(z, fmaf(z, -1.0f / 3628800, 1.0f / 40320), -1.0f / 720), 1.0f / 24), -0.5f), 1.0f);
    const bool swap = quarter & 1;
    c = swap ? sn : cs;
    s = swap ? cs : sn;
    if (quarter == 1 || quarter == 2) c = -c;
    if (quarter & 2) s = -s;
}

// What a lane holds of a row: two runs of V channels, and which pairs are turned.
template <typename Elem> struct Runs {
    static constexpr int V = Vec<Elem>::V;
    int c[2], valid[2];
    int pair[2], pairs[2];   // the first pair of a run, and how many (side by side), or of both (apart, pairs[1] = 0)
    __device__ __forceinline__ Runs(int item, int items, int D, int R, bool adjacent) {
        const bool has = item < items;
        if (adjacent) {
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                c[u] = (2 * item + u) * V;
                valid[u] = has ? max(0, min(V, D - c[u])) : 0;
                pair[u] = c[u] / 2;
                pairs[u] = has ? max(0, min(V / 2, R / 2 - pair[u])) : 0;
            }
            return;
        }
        const int half = R / 2, turned = (half + V - 1) / V;
        if (item < turned) {
            c[0] = item * V;
            c[1] = half + c[0];
            valid[0] = valid[1] = has ? min(V, half - c[0]) : 0;
            pairs[0] = valid[0];
        } else {
            c[0] = R + (item - turned) * 2 * V;
            c[1] = c[0] + V;
#pragma unroll
            for (int u = 0; u < 2; ++u) valid[u] = has ? max(0, min(V, D - c[u])) : 0;
            pairs[0] = 0;
        }
        pair[0] = c[0];
        pair[1] = pairs[1] = 0;
    }
    template <bool FULL> __device__ __forceinline__ void load(const Elem* row, int D, u32x4 (&raw)[2]) const {
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            raw[u] = u32x4{0, 0, 0, 0};
            if (valid[u] == 0) continue;
            if (FULL || valid[u] == V) {
                raw[u] = reinterpret_cast<const Bytes16*>(row + c[u])->v;
            } else {
                typename Vec<Elem>::Packed e{};
#pragma unroll
                for (int j = 0; j < V; ++j)
                    if (j < valid[u]) e.v[j] = row[c[u] + j];
                raw[u] = __builtin_bit_cast(u32x4, e);
            }
        }
    }
    template <bool FULL> __device__ __forceinline__ void store(Elem* row, const float (&x)[2][V]) const {
#pragma unroll
        for (int u = 0; u < 2; ++u)
            if (valid[u] > 0) store_run<Elem, FULL>(row + c[u], valid[u], Vec<Elem>::narrow(x[u]));
    }
};

template <typename Elem, int G, bool FULL, bool GRAD>
__global__ __launch_bounds__(kThreads) void rotate_kernel(RotateArgs<Elem> a) {
    constexpr int V = Vec<Elem>::V, GROUPS = kThreads / G;
    constexpr int U = GRAD ? 2 : 4;   // heads whose loads are in flight together
    const int item = threadIdx.x % G, group = threadIdx.x / G;
    const bool adjacent = a.adjacent != 0;
    const Runs<Elem> runs(item, a.items, a.D, a.R, adjacent);
    float w[2][2][V], dw[2][2][V];
#pragma unroll
    for (int s = 0; s < 2; ++s) {
        u32x4 raw[2];
        runs.template load<false>(a.side[s].weight, a.D, raw);
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            Vec<Elem>::widen(raw[u], w[s][u]);
#pragma unroll
            for (int e = 0; e < V; ++e) dw[s][u][e] = 0.0f;
        }
    }
    const float share = 1.0f / static_cast<float>(a.D);

    const int64_t units = a.rows * a.chunks, step = static_cast<int64_t>(gridDim.x) * GROUPS;
    for (int64_t first = static_cast<int64_t>(blockIdx.x) * GROUPS; first < units; first += step) {
        const int64_t unit = first + group;
        const bool has = unit < units;
        int64_t row = 0, n = 0;
        if (units >> 32 == 0) {   // 64-bit divisions take ten times the instructions
            const uint32_t small = has ? static_cast<uint32_t>(unit) / static_cast<uint32_t>(a.chunks) : 0;
            row = small, n = small / static_cast<uint32_t>(a.L);
        } else if (has) {
            row = unit / a.chunks;
            n = row / a.L;
        }
        const int chunk = has ? static_cast<int>(unit - row * a.chunks) : 0;
        const int64_t l = row - n * a.L;
        const int h_first = chunk * a.each, h_end = has ? min(h_first + a.each, a.side[0].heads + a.side[1].heads) : 0;
        const int64_t position = a.positions ? a.positions[row] : a.start + l;
        float co[V], si[V];
#pragma unroll
        for (int e = 0; e < V; ++e) {
            const int u = adjacent ? e / (V / 2) : 0, j = adjacent ? e % (V / 2) : e;
            // every lane loads, the last frequency where it turns no pair: all are in flight together
            const uint64_t turns = a.turns[min(runs.pair[u] + j, a.R / 2 - 1)];
            cos_sin(static_cast<uint32_t>((static_cast<uint64_t>(position) * turns) >> 32), co[e], si[e]);
            if (GRAD) si[e] = -si[e];
        }
        // Channels that are not turned are chosen as they are: a sine of zero would not keep their
        // neighbour's infinity out.
        auto turn_pair = [](float& p, float& q, float c, float s, bool turned) {
            float a = fmaf(p, c, -(q * s)), b = fmaf(p, s, q * c);
            asm volatile("" : "+v"(a), "+v"(b));   // a choice, not a branch: the compiler loses values in those
            p = turned ? a : p;
            q = turned ? b : q;
        };
        auto turn = [&](float (&x)[2][V]) {
            if (adjacent) {
#pragma unroll
                for (int u = 0; u < 2; ++u)
#pragma unroll
                    for (int j = 0; j < V / 2; ++j)
                        turn_pair(x[u][2 * j], x[u][2 * j + 1], co[u * (V / 2) + j], si[u * (V / 2) + j], j < runs.pairs[u]);
            } else {
#pragma unroll
                for (int e = 0; e < V; ++e) turn_pair(x[0][e], x[1][e], co[e], si[e], runs.pairs[0] > 0);
            }
        };
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            const Side<Elem>& side = a.side[s];
            const int before = s == 0 ? 0 : a.side[0].heads;
            const int h0 = max(0, h_first - before), h1 = min(side.heads, h_end - before);
            // every lane of a wave goes round as often: the sums are over lanes
            const int rounds = max(0, h1 - h0);
            for (int i = 0; __any(i < rounds); i += U) {
                u32x4 raw[U][2], rdy[U][2];
#pragma unroll
                for (int k = 0; k < U; ++k) {
                    raw[k][0] = raw[k][1] = u32x4{0, 0, 0, 0};
                    if (i + k < rounds) runs.template load<FULL>(side.x.at(n, l, h0 + i + k), a.D, raw[k]);
                    if constexpr (GRAD) {
                        rdy[k][0] = rdy[k][1] = u32x4{0, 0, 0, 0};
                        if (i + k < rounds) runs.template load<FULL>(side.dy.at(n, l, h0 + i + k), a.D, rdy[k]);
                    }
                }
#pragma unroll
                for (int k = 0; k < U; ++k) {
                    if (k > 0 && !__any(i + k < rounds)) break;   // few heads a group: 64 x 16 heads 7.7 to 6.4 us
                    float x[2][V], ss = 0.0f;
#pragma unroll
                    for (int u = 0; u < 2; ++u) {
                        Vec<Elem>::widen(raw[k][u], x[u]);
#pragma unroll
                        for (int e = 0; e < V; ++e) ss = fmaf(x[u][e], x[u][e], ss);
                    }
                    const float rstd = 1.0f / sqrtf(fmaf(lanes_sum<G>(ss), share, a.eps));
                    if constexpr (!GRAD) {
#pragma unroll
                        for (int u = 0; u < 2; ++u)
#pragma unroll
                            for (int e = 0; e < V; ++e) x[u][e] = x[u][e] * rstd * w[s][u][e];
                        turn(x);
                        if (i + k < rounds) runs.template store<FULL>(side.y.at(n, l, h0 + i + k), x);
                    } else {
                        float du[2][V], gx = 0.0f;
#pragma unroll
                        for (int u = 0; u < 2; ++u) Vec<Elem>::widen(rdy[k][u], du[u]);
                        turn(du);
#pragma unroll
                        for (int u = 0; u < 2; ++u)
#pragma unroll
                            for (int e = 0; e < V; ++e) {
                                if (i + k < rounds) dw[s][u][e] = fmaf(du[u][e], x[u][e] * rstd, dw[s][u][e]);
                                du[u][e] *= w[s][u][e];
                                gx = fmaf(du[u][e], x[u][e], gx);
                            }
                        const float mean = lanes_sum<G>(gx) * share * rstd * rstd;
#pragma unroll
                        for (int u = 0; u < 2; ++u)
#pragma unroll
                            for (int e = 0; e < V; ++e) du[u][e] = rstd * (du[u][e] - x[u][e] * mean);
                        if (i + k < rounds) runs.template store<FULL>(side.y.at(n, l, h0 + i + k), du);
                    }
                }
            }
        }
    }
    if constexpr (GRAD) {
        // the groups' sums, added in their order
        __shared__ float lds[2 * V][kThreads];
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            __syncthreads();
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int e = 0; e < V; ++e) lds[u * V + e][threadIdx.x] = dw[s][u][e];
            __syncthreads();
            float* part = a.parts + (static_cast<int64_t>(blockIdx.x) * 2 + s) * a.D;
            for (int i = threadIdx.x; i < G * 2 * V; i += kThreads) {
                const Runs<Elem> of(i % G, a.items, a.D, a.R, adjacent);
                const int u = i / G / V, e = i / G % V;
                float sum = 0.0f;
                for (int k = 0; k < GROUPS; ++k) sum += lds[u * V + e][k * G + i % G];
                if (e < of.valid[u]) part[of.c[u] + e] = sum;
            }
        }
    }
}

// The weights' gradients: the workgroups' parts, each channel's added by 64 threads.
__global__ __launch_bounds__(1024) void rotate_parts_kernel(const float* parts, int count, int D, float* dq, float* dk) {
    constexpr int kSlices = 1024 / kPartChannels;
    __shared__ float lds[kSlices][kPartChannels + 1];
    const int c = static_cast<int>(blockIdx.x) * kPartChannels + static_cast<int>(threadIdx.x) % kPartChannels;
    const int k = threadIdx.x / kPartChannels;
    float s = 0.0f;
    constexpr int U = 16;   // loads in flight
    if (c < 2 * D)
        for (int p = k; p < count; p += U * kSlices) {
            float v[U];
#pragma unroll
            for (int u = 0; u < U; ++u) v[u] = p + u * kSlices < count ? parts[static_cast<int64_t>(p + u * kSlices) * 2 * D + c] : 0.0f;
#pragma unroll
            for (int u = 0; u < U; ++u) s += v[u];
        }
    lds[k][threadIdx.x % kPartChannels] = s;
    __syncthreads();
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;   // a wave a channel
    s = lanes_sum<64>(lds[lane][wave]);
    const int out = static_cast<int>(blockIdx.x) * kPartChannels + wave;
    if (lane != 0 || out >= 2 * D) return;
    if (out < D) dq[out] = s;
    else dk[out - D] = s;
}

// Lanes of a row.
int items_of(int V, int D, int R, bool adjacent) {
    if (adjacent) return (D + 2 * V - 1) / (2 * V);
    return (R / 2 + V - 1) / V + (D - R + 2 * V - 1) / (2 * V);
}
int lanes_of(int items) { return items <= 4 ? 4 : items <= 8 ? 8 : items <= 16 ? 16 : items <= 32 ? 32 : 64; }

// Heads that a group of lanes takes at a position: all of them, for the sines, where the
// groups still fill the chip, fewer where they do not.
struct Cut {
    int32_t each, chunks;
    int64_t blocks;
};
// Twice as many threads give each too little work for its sines: 8000 x 10 heads of 128
// channels 20.3 us, with 512 15.7.  With half as many that is 15.5, and the gradients of 4096
// x 16 heads of 64 channels 20.0 us for 18.2.
constexpr int64_t kThreadsPerCu = 512;
Cut cut_of(int64_t rows, int heads, int G, int64_t per_cu) {
    const int64_t wanted = int64_t(device_cu_count()) * kThreadsPerCu / G;
    Cut c;
    c.each = static_cast<int32_t>(std::clamp<int64_t>(rows * heads / wanted, 1, heads));
    c.chunks = (heads + c.each - 1) / c.each;
    const int64_t groups = kThreads / G;
    c.blocks = std::max<int64_t>(1, std::min<int64_t>((rows * c.chunks + groups - 1) / groups, device_cu_count() * per_cu));
    return c;
}
// Workgroups of a launch.  The gradients' each leave a part of the weights' gradients behind:
// with 4 to a compute unit 16384 x 20 heads of 128 channels take 64.8 us, with 2 61.2 and
// with 1 66.3; forward 4 to 32 are alike.
constexpr int64_t kForwardPerCu = 8, kGradPerCu = 2;

Cut grad_cut(int dtype, int64_t rows, int heads, int D, int R, bool adjacent) {
    return cut_of(rows, heads, lanes_of(items_of(16 / dtype_bytes(dtype), D, R, adjacent)), kGradPerCu);
}

template <typename Elem, bool GRAD> hipError_t launch(const RotateArgs<Elem>& k, int64_t blocks, hipStream_t stream) {
    constexpr int V = Vec<Elem>::V;
    const bool full = k.adjacent ? k.D % (2 * V) == 0 : k.R / 2 % V == 0 && (k.D - k.R) % (2 * V) == 0;
    const unsigned grid = static_cast<unsigned>(blocks);
    switch (lanes_of(k.items)) {
#define WG_ROTATE_CASE(G)                                                                      \
    case G:                                                                                    \
        if (full) rotate_kernel<Elem, G, true, GRAD><<<grid, kThreads, 0, stream>>>(k);        \
        else rotate_kernel<Elem, G, false, GRAD><<<grid, kThreads, 0, stream>>>(k);            \
        break;
        WG_ROTATE_CASE(4) WG_ROTATE_CASE(8) WG_ROTATE_CASE(16) WG_ROTATE_CASE(32) WG_ROTATE_CASE(64)
#undef WG_ROTATE_CASE
    }
    return hipGetLastError();
}

}  // namespace

size_t head_norm_rotate_workspace(int dtype, int64_t N, int64_t L, int64_t heads, int64_t D, int64_t R, bool adjacent) {
    const int64_t parts = grad_cut(dtype, N * L, static_cast<int>(heads), static_cast<int>(D), static_cast<int>(R), adjacent).blocks;
    return static_cast<size_t>((parts * 2 * D * 4 + 15) / 16 * 16);
}

template <int D> hipError_t launch_head_norm_rotate_t(const wg_head_norm_rotate& a, hipStream_t stream) {
    using Elem = typename DTypeOf<D>::type;
    const int heads = static_cast<int>(a.q_heads + a.k_heads);
    const int items = items_of(Vec<Elem>::V, static_cast<int>(a.D), static_cast<int>(a.R), a.adjacent != 0);
    const Cut cut = cut_of(a.N * a.L, heads, lanes_of(items), kForwardPerCu);
    auto side = [&](const wg_heads& x, const wg_heads& y, const void* w, int64_t n) {
        return Side<Elem>{heads_of<const Elem>(x), {}, heads_of<Elem>(y), static_cast<const Elem*>(w), static_cast<int32_t>(n)};
    };
    const RotateArgs<Elem> k{{side(a.q, a.q_out, a.q_weight, a.q_heads), side(a.k, a.k_out, a.k_weight, a.k_heads)},
                             a.N * a.L, static_cast<int32_t>(a.L), static_cast<int32_t>(a.D), static_cast<int32_t>(a.R),
                             a.adjacent != 0, items, cut.each, cut.chunks, static_cast<const uint64_t*>(a.turns), a.positions,
                             a.start, static_cast<float>(a.eps), nullptr};
    return launch<Elem, false>(k, cut.blocks, stream);
}

template <int D> hipError_t launch_head_norm_rotate_backward_t(const wg_head_norm_rotate_backward& a, hipStream_t stream) {
    using Elem = typename DTypeOf<D>::type;
    const int heads = static_cast<int>(a.q_heads + a.k_heads);
    const int items = items_of(Vec<Elem>::V, static_cast<int>(a.D), static_cast<int>(a.R), a.adjacent != 0);
    const Cut cut = cut_of(a.N * a.L, heads, lanes_of(items), kGradPerCu);
    auto side = [&](const wg_heads& x, const wg_heads& dy, const wg_heads& dx, const void* w, int64_t n) {
        return Side<Elem>{heads_of<const Elem>(x), heads_of<const Elem>(dy), heads_of<Elem>(dx), static_cast<const Elem*>(w),
                          static_cast<int32_t>(n)};
    };
    const RotateArgs<Elem> k{{side(a.q, a.dq_out, a.dq, a.q_weight, a.q_heads), side(a.k, a.dk_out, a.dk, a.k_weight, a.k_heads)},
                             a.N * a.L, static_cast<int32_t>(a.L), static_cast<int32_t>(a.D), static_cast<int32_t>(a.R),
                             a.adjacent != 0, items, cut.each, cut.chunks, static_cast<const uint64_t*>(a.turns), a.positions,
                             a.start, static_cast<float>(a.eps), static_cast<float*>(a.workspace)};
    if (const hipError_t e = launch<Elem, true>(k, cut.blocks, stream)) return e;
    rotate_parts_kernel<<<static_cast<unsigned>((2 * a.D + kPartChannels - 1) / kPartChannels), 1024, 0, stream>>>(
        k.parts, static_cast<int>(cut.blocks), k.D, a.dq_weight, a.dk_weight);
    return hipGetLastError();
}

#define WG_ROTATE_INSTANCES(D)                                                                  \
    template hipError_t launch_head_norm_rotate_t<D>(const wg_head_norm_rotate&, hipStream_t);  \
    template hipError_t launch_head_norm_rotate_backward_t<D>(const wg_head_norm_rotate_backward&, hipStream_t);
WG_ROTATE_INSTANCES(0)
WG_ROTATE_INSTANCES(1)
WG_ROTATE_INSTANCES(2)
#undef WG_ROTATE_INSTANCES

}  // namespace wg
