// The gated linear recurrence, its gradients and its single step on gfx950:
//   f = sigmoid(gate), i = 1 - f = sigmoid(-gate)
//   h[l] = f h[l-1] + i value[l],   y[l] = h[l] (times silu(out_gate[l]))
// and, with g[l] = dy[l] silu(out_gate[l]) and R[l] the gradient that step l hands
// to the state ahead of it,
//   R[l] = f[l] (g[l] + R[l+1])  (behind the last step: dh_last),  dh0 = R[0]
//   dvalue[l] = i (g[l] + R[l+1]),  dgate[l] = i (h[l-1] - value[l]) R[l]
//   dout_gate[l] = dy[l] h[l] silu'(out_gate[l]).
// All of it in fp32; each result is rounded once to its type.
//
// Both directions are a scan of maps s -> A s + B, which compose: a run of steps
// has A the product of its gates.  A workgroup takes 32 channels, a 64-byte run of
// 16-bit rows (128 bytes in fp32), and walks tiles of T steps.  Of a tile a thread
// holds 16 bytes of each of S steps in registers, 32 gates in all, and composes
// its steps; the composed maps of the tile's threads go through LDS, where a
// thread per (channel, 32 steps) composes them, a shift-and-compose over the 16
// lanes of a channel gives the state ahead of each 32 steps, and every thread gets
// the state ahead of its own steps.  The next tile's loads are in flight during
// that.  So rows are read once and written once, whatever the length.
//
// Where the channels do not fill the chip, the length is cut into chunks, a
// workgroup each: a first kernel composes each chunk's map (reading the gates a
// second time), the second one starts each chunk from the maps ahead of it.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>

#include "device_common.hpp"
#include "kernels.hpp"
#include "rows.hpp"
#include "sequence.hpp"

namespace wg {

namespace {

constexpr int kStepThreads = 256;
constexpr int kScanBlock = WG_SCAN_BLOCK;
constexpr int kScanChannels = 32;   // channels of a workgroup

// sigmoid(z) and sigmoid(-z), both to fp32 accuracy for any z (1 - f would lose
// the small one): with e = exp(-z) they are 1 / (1 + e) and e / (1 + e), which is 1
// where e is large (e may be infinite); NaN stays NaN.
struct Gate {
    float f, i;
};
constexpr float kLog2e = 1.44269504088896340736f;
__device__ __forceinline__ Gate gate_of(float z) {
    const float e = __builtin_amdgcn_exp2f(z * -kLog2e);
    const float f = __builtin_amdgcn_rcpf(1.0f + e);
    return {f, e > 0x1p100f ? 1.0f : e * f};
}
__device__ __forceinline__ float sigmoid_of(float o) {
    return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(o * -kLog2e));
}

template <typename Elem> struct Rows {
    Elem* p;
    int64_t sn, sl;
    __device__ __forceinline__ Elem* at(int64_t n, int64_t l) const { return p + n * sn + l * sl; }
};
template <typename Elem> Rows<Elem> rows_of(const wg_rows& r) {
    return {static_cast<Elem*>(const_cast<void*>(r.data)), r.stride_n, r.stride_l};
}

__device__ __forceinline__ int32_t steps_of(const int32_t* lengths, int64_t n, int32_t L) {
    if (!lengths) return L;
    const int32_t v = lengths[n];
    return v < 0 ? 0 : (v > L ? L : v);
}

// Where a workgroup's threads stand.  Columns are runs of V channels, numbered
// over all sequences, so that a workgroup may end one sequence and begin another.
struct Split {
    int64_t columns;        // N * runs
    uint32_t groups;        // workgroups along x that have columns
    int32_t runs;           // runs of V channels in a row, the last one maybe short
    int32_t chunk_steps;    // steps of a chunk, a multiple of the tile
    int32_t chunks;
};

// blockIdx.x -> columns: workgroups go to the eight XCDs in turn, and the two
// halves of a 128-byte line (64-byte runs of 16-bit rows) go to the same one.
template <int LANES> __device__ __forceinline__ uint32_t group_of_block(uint32_t b) {
    if (LANES == 8) return b;
    return (b / 16) * 16 + (b % 8) * 2 + b % 16 / 8;
}

// A thread's S steps of one tensor, 16 bytes each, from step l0 of a row that
// starts at `row`; steps from L on repeat the last row (they are replaced later).
template <typename Elem, bool FULL, int S>
__device__ __forceinline__ void load_steps(const Elem* row, int64_t sl, int32_t l0, int32_t L, int valid,
                                           u32x4 (&raw)[S]) {
    const bool inside = l0 + S <= L;
    const Elem* p = row + static_cast<int64_t>(inside ? l0 : min(l0, L - 1)) * sl;
    const int last = inside ? S - 1 : max(0, L - 1 - l0);
    if (FULL || valid == Vec<Elem>::V) {
#pragma unroll
        for (int k = 0; k < S; ++k)
            raw[k] = reinterpret_cast<const Bytes16*>(p + (k < last ? k : last) * sl)->v;
    } else {
#pragma unroll
        for (int k = 0; k < S; ++k) {
            const Elem* q = p + (k < last ? k : last) * sl;
            typename Vec<Elem>::Packed e{};
#pragma unroll
            for (int j = 0; j < Vec<Elem>::V; ++j)
                if (j < valid) e.v[j] = q[j];
            raw[k] = __builtin_bit_cast(u32x4, e);
        }
    }
}

// +infinity in every element: a gate that keeps the state (f = 1, i = 0)
template <typename Elem> constexpr uint32_t kKeep = 0x7f807f80u;
template <> constexpr uint32_t kKeep<float> = 0x7f800000u;
template <> constexpr uint32_t kKeep<_Float16> = 0x7c007c00u;

// LDS of a tile's composed maps: [part][segment of V][channel], a part's rows
// 4 words apart from the next one's, so that the 16 parts of 4 channels that a wave
// reads fall on different banks.
template <int T, int V> struct TileLds {
    static constexpr int kParts = T / kScanChannels;
    static constexpr int kPartWords = V * kScanChannels + 4;
    static constexpr int kWords = kParts * kPartWords;
    static __device__ __forceinline__ int at(int segment, int channel) {
        return segment / V * kPartWords + segment % V * kScanChannels + channel;
    }
};

template <int N> __device__ __forceinline__ float from_lower(float v) {   // of lane - N in rows of 16
    return __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(v), 0x110 + N, 0xf, 0xf, true));
}
template <int N> __device__ __forceinline__ float from_upper(float v) {   // of lane + N
    return __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(v), 0x100 + N, 0xf, 0xf, true));
}
template <int N, bool UP> __device__ __forceinline__ float from_part(float v) {
    if constexpr (UP) return from_lower<N>(v);
    else return from_upper<N>(v);
}

// Composes the maps of a channel's P parts (adjacent lanes), each with all parts
// ahead of it in scan order (UP: ascending).
template <int P, bool UP, int N = 1> __device__ __forceinline__ void compose_parts(int part, float& A, float& B) {
    if constexpr (N < P) {
        const float a = from_part<N, UP>(A), b = from_part<N, UP>(B);
        const bool has = UP ? part >= N : part + N < P;
        if (has) {
            B = fmaf(A, b, B);
            A *= a;
        }
        compose_parts<P, UP, 2 * N>(part, A, B);
    }
}
template <int P, bool UP> __device__ __forceinline__ float of_last_part(float v) {
    return __shfl(v, (threadIdx.x & 63) / P * P + (UP ? P - 1 : 0));
}

// The state that reaches a chunk: the maps of the `count` chunks that the scan
// meets first, from (A, B) pairs `stride` pairs apart, composed and applied to s.
// The P lanes of a channel share the work.
template <int P>
__device__ __forceinline__ float reach_chunk(const float2* maps, int64_t stride, int count, int part, float s) {
    const int each = (count + P - 1) / P;
    const int first = min(part * each, count), end = min(first + each, count);
    float A = 1.0f, B = 0.0f;
    for (int j = first; j < end; ++j) {
        const float2 m = maps[j * stride];
        B = fmaf(m.x, B, m.y);
        A *= m.x;
    }
    compose_parts<P, true>(part, A, B);
    A = of_last_part<P, true>(A);
    B = of_last_part<P, true>(B);
    return fmaf(A, s, B);
}

template <typename Elem> struct ScanArgs {
    int64_t N;
    int32_t L, C;
    Rows<const Elem> gate, value, out_gate;
    Rows<Elem> y;
    const float* h0;
    const int32_t* lengths;
    float *h_last, *states;
    float2* maps;   // [chunk][32 channels of every group]
    Split split;
};

// MAPS: only the composed maps of the chunks.
template <typename Elem, int T, int E, bool OUT, bool FULL, bool MAPS>
__global__ __launch_bounds__(T) void scan_kernel(ScanArgs<Elem> a) {
    constexpr int V = Vec<Elem>::V, LANES = kScanChannels / V, S = E / V, P = T / kScanChannels, TILE = P * E;
    using Lds = TileLds<T, V>;
    __shared__ float lds[2][2][Lds::kWords];
    const uint32_t group = group_of_block<LANES>(blockIdx.x);
    if (group >= a.split.groups) return;
    const int chunk = blockIdx.y, tid = threadIdx.x;
    const int32_t L = a.L;

    // as the owner of steps: column `lane` of the group, steps `segment * S ..` of a tile
    const int lane = tid % LANES, segment = tid / LANES;
    const int64_t column = static_cast<int64_t>(group) * LANES + lane;
    const bool has = column < a.split.columns;
    const int64_t n = has ? column / a.split.runs : 0;
    const int c0 = has ? static_cast<int>(column % a.split.runs) * V : 0;
    const int valid = has ? min(V, a.C - c0) : 0;
    const int32_t steps = has ? steps_of(a.lengths, n, L) : 0;
    const Elem* gate = a.gate.at(n, 0) + c0;
    const Elem* value = a.value.at(n, 0) + c0;
    const Elem* out_gate = OUT && !MAPS ? a.out_gate.at(n, 0) + c0 : nullptr;

    // as a scanner: one channel and one part (32 steps) of a tile
    const int channel = tid / P, part = tid % P;
    const int64_t sc = static_cast<int64_t>(group) * LANES + channel / V;
    const int64_t sn = sc / a.split.runs;
    const int schan = static_cast<int>(sc % a.split.runs) * V + channel % V;
    const bool scans = sc < a.split.columns && schan < a.C;
    const int64_t smap = static_cast<int64_t>(group) * kScanChannels + channel;
    const int64_t map_stride = static_cast<int64_t>(a.split.groups) * kScanChannels;
    const int64_t blocks = (static_cast<int64_t>(L) + kScanBlock - 1) / kScanBlock;

    // a scanner's state ahead of the tile at hand, or the map of the chunk so far
    float carry = MAPS || !scans || !a.h0 ? 0.0f : a.h0[sn * a.C + schan];
    float product = 1.0f;
    if (!MAPS && chunk > 0) carry = reach_chunk<P>(a.maps + smap, map_stride, chunk, part, carry);

    const int32_t first = chunk * a.split.chunk_steps;
    const int32_t end = static_cast<int32_t>(min(static_cast<int64_t>(first) + a.split.chunk_steps, static_cast<int64_t>(L)));
    u32x4 z[S], v[S], o[S];
    auto load = [&](int32_t t) {
        const int32_t l0 = t + segment * S;
        load_steps<Elem, FULL, S>(gate, a.gate.sl, l0, L, valid, z);
        load_steps<Elem, FULL, S>(value, a.value.sl, l0, L, valid, v);
        if (OUT && !MAPS) load_steps<Elem, FULL, S>(out_gate, a.out_gate.sl, l0, L, valid, o);
    };
    if (first < end && has) load(first);
    int buf = 0;
    for (int32_t t = first; t < end; t += TILE, buf ^= 1) {
        const int32_t l0 = t + segment * S;
        float f[S][V], b[S][V], s[S][V];
        float A[V], B[V];
#pragma unroll
        for (int q = 0; q < V; ++q) {
            A[q] = 1.0f;
            B[q] = 0.0f;
        }
#pragma unroll
        for (int k = 0; k < S; ++k) {
            if (l0 + k >= steps) {   // padding: nothing of it is used
                z[k] = u32x4{kKeep<Elem>, kKeep<Elem>, kKeep<Elem>, kKeep<Elem>};
                v[k] = u32x4{0, 0, 0, 0};
                if (OUT && !MAPS) o[k] = u32x4{0, 0, 0, 0};
            }
            float zf[V], vf[V];
            Vec<Elem>::widen(z[k], zf);
            Vec<Elem>::widen(v[k], vf);
            if constexpr (OUT && !MAPS) {
                float of[V];
                Vec<Elem>::widen(o[k], of);
#pragma unroll
                for (int q = 0; q < V; ++q) s[k][q] = of[q] * sigmoid_of(of[q]);
            }
#pragma unroll
            for (int q = 0; q < V; ++q) {
                const Gate g = gate_of(zf[q]);
                f[k][q] = g.f;
                b[k][q] = g.i * vf[q];
                A[q] *= g.f;
                B[q] = fmaf(g.f, B[q], b[k][q]);
            }
        }
        if (t + TILE < end && has) load(t + TILE);
        float* la = lds[buf][0];
        float* lb = lds[buf][1];
#pragma unroll
        for (int q = 0; q < V; q += 4) {
            const int w = Lds::at(segment, lane * V + q);
            *reinterpret_cast<float4*>(la + w) = float4{A[q], A[q + 1], A[q + 2], A[q + 3]};
            *reinterpret_cast<float4*>(lb + w) = float4{B[q], B[q + 1], B[q + 2], B[q + 3]};
        }
        __syncthreads();
        {
            float ma[V], mb[V], PA = 1.0f, PB = 0.0f;
#pragma unroll
            for (int j = 0; j < V; ++j) {
                ma[j] = la[Lds::at(part * V + j, channel)];
                mb[j] = lb[Lds::at(part * V + j, channel)];
            }
#pragma unroll
            for (int j = 0; j < V; ++j) {
                PB = fmaf(ma[j], PB, mb[j]);
                PA *= ma[j];
            }
            compose_parts<P, true>(part, PA, PB);
            if constexpr (MAPS) {
                const float ta = of_last_part<P, true>(PA), tb = of_last_part<P, true>(PB);
                carry = fmaf(ta, carry, tb);
                product *= ta;
            } else {
                // the state behind this part, and ahead of it
                const float behind = fmaf(PA, carry, PB);
                float h = from_lower<1>(behind);
                if (part == 0) h = carry;
                const int32_t block = (t + part * E) / kScanBlock;
                if (a.states && scans && part * E % kScanBlock == 0 && block < blocks)
                    a.states[(sn * blocks + block) * a.C + schan] = h;
                carry = of_last_part<P, true>(behind);
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    la[Lds::at(part * V + j, channel)] = h;
                    h = fmaf(ma[j], h, mb[j]);
                }
            }
        }
        if constexpr (!MAPS) {
            __syncthreads();
            float h[V];
#pragma unroll
            for (int q = 0; q < V; q += 4) {
                const float4 w = *reinterpret_cast<const float4*>(la + Lds::at(segment, lane * V + q));
                h[q] = w.x, h[q + 1] = w.y, h[q + 2] = w.z, h[q + 3] = w.w;
            }
            Elem* y = a.y.at(n, l0) + c0;
#pragma unroll
            for (int k = 0; k < S; ++k) {
                float out[V];
#pragma unroll
                for (int q = 0; q < V; ++q) {
                    h[q] = fmaf(f[k][q], h[q], b[k][q]);
                    out[q] = OUT ? h[q] * s[k][q] : h[q];
                }
                u32x4 bits = Vec<Elem>::narrow(out);
                if (l0 + k >= steps) bits = u32x4{0, 0, 0, 0};
                if (has && l0 + k < L) store_run<Elem, FULL>(y + k * a.y.sl, valid, bits);
            }
        }
    }
    if (part == 0 && scans) {
        if constexpr (MAPS) a.maps[chunk * map_stride + smap] = float2{product, carry};
        else if (chunk == a.split.chunks - 1) a.h_last[sn * a.C + schan] = carry;
    }
}

template <typename Elem> struct GradArgs {
    int64_t N;
    int32_t L, C;
    Rows<const Elem> dy, gate, value, out_gate;
    Rows<Elem> dgate, dvalue, dout_gate;
    const float *states, *dh_last;
    const int32_t* lengths;
    float* dh0;
    float2* maps;   // of the chunks, in the order in which the gradients' scan meets them
    Split split;
};

// The gradients: tiles from the last to the first.  A part's 32 steps are a block
// whose state the forward pass kept, so the states ahead of each thread's steps
// follow from the same composed maps without a scan over the parts.
template <typename Elem, int T, int E, bool OUT, bool FULL, bool MAPS>
__global__ __launch_bounds__(T) void scan_grad_kernel(GradArgs<Elem> a) {
    constexpr int V = Vec<Elem>::V, LANES = kScanChannels / V, S = E / V, P = T / kScanChannels, TILE = P * E;
    using Lds = TileLds<T, V>;
    __shared__ float lds[2][3][Lds::kWords];
    const uint32_t group = group_of_block<LANES>(blockIdx.x);
    if (group >= a.split.groups) return;
    const int chunk = blockIdx.y, tid = threadIdx.x;
    const int32_t L = a.L;

    const int lane = tid % LANES, segment = tid / LANES;
    const int64_t column = static_cast<int64_t>(group) * LANES + lane;
    const bool has = column < a.split.columns;
    const int64_t n = has ? column / a.split.runs : 0;
    const int c0 = has ? static_cast<int>(column % a.split.runs) * V : 0;
    const int valid = has ? min(V, a.C - c0) : 0;
    const int32_t steps = has ? steps_of(a.lengths, n, L) : 0;
    const Elem* gate = a.gate.at(n, 0) + c0;
    const Elem* value = a.value.at(n, 0) + c0;
    const Elem* dyp = a.dy.at(n, 0) + c0;
    const Elem* out_gate = OUT ? a.out_gate.at(n, 0) + c0 : nullptr;

    const int channel = tid / P, part = tid % P;
    const int64_t sc = static_cast<int64_t>(group) * LANES + channel / V;
    const int64_t sn = sc / a.split.runs;
    const int schan = static_cast<int>(sc % a.split.runs) * V + channel % V;
    const bool scans = sc < a.split.columns && schan < a.C;
    const int64_t smap = static_cast<int64_t>(group) * kScanChannels + channel;
    const int64_t map_stride = static_cast<int64_t>(a.split.groups) * kScanChannels;
    const int64_t blocks = (static_cast<int64_t>(L) + kScanBlock - 1) / kScanBlock;

    float carry = MAPS || !scans || !a.dh_last ? 0.0f : a.dh_last[sn * a.C + schan];
    float product = 1.0f;
    if (!MAPS && chunk > 0) carry = reach_chunk<P>(a.maps + smap, map_stride, chunk, part, carry);

    // chunk 0 is the last one of the sequence
    const int32_t first = (a.split.chunks - 1 - chunk) * a.split.chunk_steps;
    const int32_t end = static_cast<int32_t>(min(static_cast<int64_t>(first) + a.split.chunk_steps, static_cast<int64_t>(L)));
    const int32_t tiles = (end - first + TILE - 1) / TILE;
    u32x4 z[S], v[S], o[S], d[S];
    auto load = [&](int32_t t) {
        const int32_t l0 = t + segment * S;
        load_steps<Elem, FULL, S>(gate, a.gate.sl, l0, L, valid, z);
        load_steps<Elem, FULL, S>(dyp, a.dy.sl, l0, L, valid, d);
        if (!MAPS) load_steps<Elem, FULL, S>(value, a.value.sl, l0, L, valid, v);
        if (OUT) load_steps<Elem, FULL, S>(out_gate, a.out_gate.sl, l0, L, valid, o);
    };
    if (tiles > 0 && has) load(first + (tiles - 1) * TILE);
    int buf = 0;
    for (int32_t tile = tiles - 1; tile >= 0; --tile, buf ^= 1) {
        const int32_t t = first + tile * TILE, l0 = t + segment * S;
        // g: the gradient at a step's state from its own output; q: what times
        // the state is the output gate's gradient
        float f[S][V], i[S][V], vf[S][V], g[S][V], q[S][V];
        float A[V], B[V], R[V];
#pragma unroll
        for (int e = 0; e < V; ++e) {
            A[e] = 1.0f;
            B[e] = 0.0f;
            R[e] = 0.0f;
        }
#pragma unroll
        for (int k = 0; k < S; ++k) {
            if (l0 + k >= steps) {
                z[k] = u32x4{kKeep<Elem>, kKeep<Elem>, kKeep<Elem>, kKeep<Elem>};
                d[k] = u32x4{0, 0, 0, 0};
                if (!MAPS) v[k] = u32x4{0, 0, 0, 0};
                if (OUT) o[k] = u32x4{0, 0, 0, 0};
            }
            float zf[V], df[V];
            Vec<Elem>::widen(z[k], zf);
            Vec<Elem>::widen(d[k], df);
            if (!MAPS) Vec<Elem>::widen(v[k], vf[k]);
            if constexpr (OUT) {
                float of[V];
                Vec<Elem>::widen(o[k], of);
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    const float s = sigmoid_of(of[e]), silu = of[e] * s;
                    g[k][e] = df[e] * silu;
                    // silu' = s + silu (1 - s)
                    q[k][e] = df[e] * fmaf(silu, 1.0f - s, s);
                }
            } else {
#pragma unroll
                for (int e = 0; e < V; ++e) g[k][e] = df[e];
            }
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const Gate w = gate_of(zf[e]);
                f[k][e] = w.f;
                i[k][e] = w.i;
                A[e] *= w.f;
                if (!MAPS) B[e] = fmaf(w.f, B[e], w.i * vf[k][e]);
            }
        }
#pragma unroll
        for (int k = S - 1; k >= 0; --k)
#pragma unroll
            for (int e = 0; e < V; ++e) R[e] = f[k][e] * (g[k][e] + R[e]);
        if (tile > 0 && has) load(t - TILE);
        float* la = lds[buf][0];
        float* lb = lds[buf][1];
        float* lr = lds[buf][2];
#pragma unroll
        for (int e = 0; e < V; e += 4) {
            const int w = Lds::at(segment, lane * V + e);
            *reinterpret_cast<float4*>(la + w) = float4{A[e], A[e + 1], A[e + 2], A[e + 3]};
            if (!MAPS) *reinterpret_cast<float4*>(lb + w) = float4{B[e], B[e + 1], B[e + 2], B[e + 3]};
            *reinterpret_cast<float4*>(lr + w) = float4{R[e], R[e + 1], R[e + 2], R[e + 3]};
        }
        float h = 0.0f;   // the state ahead of this part's steps
        if (!MAPS && scans && (t + part * E) / kScanBlock < blocks)
            h = a.states[(sn * blocks + (t + part * E) / kScanBlock) * a.C + schan];
        __syncthreads();
        {
            float ma[V], mb[V], mr[V], PA = 1.0f, PR = 0.0f;
#pragma unroll
            for (int j = 0; j < V; ++j) {
                ma[j] = la[Lds::at(part * V + j, channel)];
                if (!MAPS) mb[j] = lb[Lds::at(part * V + j, channel)];
                mr[j] = lr[Lds::at(part * V + j, channel)];
            }
#pragma unroll
            for (int j = V - 1; j >= 0; --j) {
                PR = fmaf(ma[j], PR, mr[j]);
                PA *= ma[j];
            }
            compose_parts<P, false>(part, PA, PR);
            if constexpr (MAPS) {
                const float ta = of_last_part<P, false>(PA), tr = of_last_part<P, false>(PR);
                carry = fmaf(ta, carry, tr);
                product *= ta;
            } else {
                const float ahead = fmaf(PA, carry, PR);   // the gradient that leaves this part
                float r = from_upper<1>(ahead);
                if (part == P - 1) r = carry;
                carry = of_last_part<P, false>(ahead);
                if constexpr (E < kScanBlock) {
                    // the second half of a block starts where the first one ends
                    static_assert(2 * E == kScanBlock);
                    float end_state = h;
#pragma unroll
                    for (int j = 0; j < V; ++j) end_state = fmaf(ma[j], end_state, mb[j]);
                    end_state = from_lower<1>(end_state);
                    if (part % 2) h = end_state;
                }
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    lb[Lds::at(part * V + j, channel)] = h;
                    h = fmaf(ma[j], h, mb[j]);
                }
#pragma unroll
                for (int j = V - 1; j >= 0; --j) {
                    lr[Lds::at(part * V + j, channel)] = r;
                    r = fmaf(ma[j], r, mr[j]);
                }
            }
        }
        if constexpr (!MAPS) {
            __syncthreads();
            float hs[S + 1][V], r[V];
#pragma unroll
            for (int e = 0; e < V; e += 4) {
                const int w = Lds::at(segment, lane * V + e);
                const float4 x = *reinterpret_cast<const float4*>(lb + w);
                hs[0][e] = x.x, hs[0][e + 1] = x.y, hs[0][e + 2] = x.z, hs[0][e + 3] = x.w;
                const float4 y = *reinterpret_cast<const float4*>(lr + w);
                r[e] = y.x, r[e + 1] = y.y, r[e + 2] = y.z, r[e + 3] = y.w;
            }
#pragma unroll
            for (int k = 0; k < S; ++k)
#pragma unroll
                for (int e = 0; e < V; ++e) hs[k + 1][e] = fmaf(f[k][e], hs[k][e], i[k][e] * vf[k][e]);
            Elem* dz = a.dgate.at(n, l0) + c0;
            Elem* dv = a.dvalue.at(n, l0) + c0;
            Elem* dout = OUT ? a.dout_gate.at(n, l0) + c0 : nullptr;
#pragma unroll
            for (int k = S - 1; k >= 0; --k) {
                float oz[V], ov[V], oo[V];
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    const float G = g[k][e] + r[e];
                    r[e] = f[k][e] * G;
                    ov[e] = i[k][e] * G;
                    oz[e] = (i[k][e] * r[e]) * (hs[k][e] - vf[k][e]);
                    if (OUT) oo[e] = q[k][e] * hs[k + 1][e];
                }
                u32x4 bz = Vec<Elem>::narrow(oz), bv = Vec<Elem>::narrow(ov), bo{0, 0, 0, 0};
                if constexpr (OUT) bo = Vec<Elem>::narrow(oo);
                if (l0 + k >= steps) bz = bv = bo = u32x4{0, 0, 0, 0};
                if (has && l0 + k < L) {
                    store_run<Elem, FULL>(dz + k * a.dgate.sl, valid, bz);
                    store_run<Elem, FULL>(dv + k * a.dvalue.sl, valid, bv);
                    if (OUT) store_run<Elem, FULL>(dout + k * a.dout_gate.sl, valid, bo);
                }
            }
        }
    }
    if (part == 0 && scans) {
        if constexpr (MAPS) a.maps[chunk * map_stride + smap] = float2{product, carry};
        else if (a.dh0 && chunk == a.split.chunks - 1) a.dh0[sn * a.C + schan] = carry;
    }
}

template <typename Elem> struct StepArgs {
    int64_t N, C;
    Rows<const Elem> gate, value, out_gate;
    Rows<Elem> y;
    const float* h;
    float* h_new;
};

template <typename Elem>
__global__ __launch_bounds__(kStepThreads) void step_kernel(StepArgs<Elem> a) {
    using S = Storage<Elem>;
    const int64_t id = static_cast<int64_t>(blockIdx.x) * kStepThreads + threadIdx.x;
    if (id >= a.N * a.C) return;
    const int64_t n = id / a.C, c = id % a.C;
    const Gate g = gate_of(S::to_f32(a.gate.at(n, 0)[c]));
    const float h = g.f * a.h[id] + g.i * S::to_f32(a.value.at(n, 0)[c]);
    float y = h;
    if (a.out_gate.p) {
        const float o = S::to_f32(a.out_gate.at(n, 0)[c]);
        y = h * (o * sigmoid_of(o));
    }
    a.h_new[id] = h;
    a.y.at(n, 0)[c] = S::from_f32(y);
}

// How a call is cut: tiles of T steps, and chunks where the channels alone leave
// the chip idle.
struct Plan {
    Split split;
    int threads;
};
// Gates that a thread holds of a tile
constexpr int kHeld = 32, kHeldGrad = 16;
Plan plan_scan(int dtype, int64_t N, int64_t L, int64_t C, int held) {
    const int V = 16 / dtype_bytes(dtype), lanes = kScanChannels / V;
    Plan p;
    p.split.runs = static_cast<int32_t>((C + V - 1) / V);
    p.split.columns = N * p.split.runs;
    const int64_t groups = (p.split.columns + lanes - 1) / lanes;
    p.split.groups = static_cast<uint32_t>(std::min<int64_t>(groups, 0xffffffffLL));
    p.threads = L <= 4 * held ? 128 : 512;
    const int64_t tile = p.threads / kScanChannels * held, tiles = (L + tile - 1) / tile;
    int64_t chunks = std::max<int64_t>(1, std::min<int64_t>(tiles, 512 / std::max<int64_t>(1, groups)));
    if (chunks < 3) chunks = 1;
    const int64_t each = (tiles + chunks - 1) / chunks;
    p.split.chunks = static_cast<int32_t>(each ? (tiles + each - 1) / each : 1);
    p.split.chunk_steps = static_cast<int32_t>(std::max<int64_t>(each, 1) * tile);
    return p;
}
size_t maps_bytes(const Plan& p) {
    return p.split.chunks > 1 ? static_cast<size_t>(p.split.chunks) * p.split.groups * kScanChannels * sizeof(float2) : 0;
}

template <int T, typename F> hipError_t launch_tiles(const Plan& p, F&& launch) {
    const int64_t blocks = (static_cast<int64_t>(p.split.groups) + 15) / 16 * 16;
    if (blocks * T > 0xffffffffLL) return hipErrorInvalidValue;
    const unsigned x = static_cast<unsigned>(blocks), y = static_cast<unsigned>(p.split.chunks);
    return launch(dim3(x, y - 1), dim3(x, y));   // nothing reads the last chunk's map
}

template <typename Elem, int T, bool OUT, bool FULL>
hipError_t scan_t(const Plan& p, const ScanArgs<Elem>& k, hipStream_t stream) {
    return launch_tiles<T>(p, [&](dim3 ahead, dim3 grid) {
        if (p.split.chunks > 1) scan_kernel<Elem, T, kHeld, false, FULL, true><<<ahead, T, 0, stream>>>(k);
        scan_kernel<Elem, T, kHeld, OUT, FULL, false><<<grid, T, 0, stream>>>(k);
        return hipGetLastError();
    });
}
template <typename Elem, int T, bool OUT, bool FULL>
hipError_t scan_grad_t(const Plan& p, const GradArgs<Elem>& k, hipStream_t stream) {
    return launch_tiles<T>(p, [&](dim3 ahead, dim3 grid) {
        if (p.split.chunks > 1) scan_grad_kernel<Elem, T, kHeldGrad, OUT, FULL, true><<<ahead, T, 0, stream>>>(k);
        scan_grad_kernel<Elem, T, kHeldGrad, OUT, FULL, false><<<grid, T, 0, stream>>>(k);
        return hipGetLastError();
    });
}

}  // namespace

size_t gated_scan_workspace(int dtype, int64_t N, int64_t L, int64_t C, bool backward) {
    return maps_bytes(plan_scan(dtype, N, L, C, backward ? kHeldGrad : kHeld));
}

template <int D> hipError_t launch_gated_scan_t(const wg_gated_scan& a, hipStream_t stream) {
    using Elem = typename DTypeOf<D>::type;
    const Plan p = plan_scan(D, a.N, a.L, a.C, kHeld);
    const ScanArgs<Elem> k{a.N, static_cast<int32_t>(a.L), static_cast<int32_t>(a.C), rows_of<const Elem>(a.gate),
                           rows_of<const Elem>(a.value), rows_of<const Elem>(a.out_gate), rows_of<Elem>(a.y), a.h0,
                           a.lengths, a.h_last, a.states, static_cast<float2*>(a.workspace), p.split};
    const bool out = a.out_gate.data != nullptr, full = a.C % Vec<Elem>::V == 0;
#define WG_SCAN_CASE(T)                                                                                         \
    (out ? (full ? scan_t<Elem, T, true, true>(p, k, stream) : scan_t<Elem, T, true, false>(p, k, stream))       \
         : (full ? scan_t<Elem, T, false, true>(p, k, stream) : scan_t<Elem, T, false, false>(p, k, stream)))
    return p.threads == 128 ? WG_SCAN_CASE(128) : WG_SCAN_CASE(512);
#undef WG_SCAN_CASE
}

template <int D> hipError_t launch_gated_scan_backward_t(const wg_gated_scan_backward& a, hipStream_t stream) {
    using Elem = typename DTypeOf<D>::type;
    const Plan p = plan_scan(D, a.N, a.L, a.C, kHeldGrad);
    const GradArgs<Elem> k{a.N, static_cast<int32_t>(a.L), static_cast<int32_t>(a.C), rows_of<const Elem>(a.dy),
                           rows_of<const Elem>(a.gate), rows_of<const Elem>(a.value), rows_of<const Elem>(a.out_gate),
                           rows_of<Elem>(a.dgate), rows_of<Elem>(a.dvalue), rows_of<Elem>(a.dout_gate), a.states,
                           a.dh_last, a.lengths, a.dh0, static_cast<float2*>(a.workspace), p.split};
    const bool out = a.out_gate.data != nullptr, full = a.C % Vec<Elem>::V == 0;
#define WG_SCAN_CASE(T)                                                                                                   \
    (out ? (full ? scan_grad_t<Elem, T, true, true>(p, k, stream) : scan_grad_t<Elem, T, true, false>(p, k, stream))       \
         : (full ? scan_grad_t<Elem, T, false, true>(p, k, stream) : scan_grad_t<Elem, T, false, false>(p, k, stream)))
    return p.threads == 128 ? WG_SCAN_CASE(128) : WG_SCAN_CASE(512);
#undef WG_SCAN_CASE
}

template <int D> hipError_t launch_gated_step_t(const wg_gated_step& a, hipStream_t stream) {
    using Elem = typename DTypeOf<D>::type;
    const StepArgs<Elem> k{a.N, a.C, rows_of<const Elem>(a.gate), rows_of<const Elem>(a.value),
                           rows_of<const Elem>(a.out_gate), rows_of<Elem>(a.y), a.h, a.h_new};
    const int64_t blocks = (a.N * a.C + kStepThreads - 1) / kStepThreads;
    if (blocks * kStepThreads > 0xffffffffLL) return hipErrorInvalidValue;
    step_kernel<Elem><<<static_cast<unsigned>(blocks), kStepThreads, 0, stream>>>(k);
    return hipGetLastError();
}

#define WG_SCAN_INSTANCES(D)                                                                       \
    template hipError_t launch_gated_scan_t<D>(const wg_gated_scan&, hipStream_t);                 \
    template hipError_t launch_gated_scan_backward_t<D>(const wg_gated_scan_backward&, hipStream_t); \
    template hipError_t launch_gated_step_t<D>(const wg_gated_step&, hipStream_t);
WG_SCAN_INSTANCES(0)
WG_SCAN_INSTANCES(1)
WG_SCAN_INSTANCES(2)
#undef WG_SCAN_INSTANCES

}  // namespace wg
