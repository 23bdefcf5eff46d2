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
// has A the product of its gates.  A workgroup takes a group of channels and walks
// tiles of steps; of a tile a thread holds 16 bytes of each of S steps in registers,
// kHeld gates in all.  It composes its steps; the maps of the threads go through
// LDS, where a thread per (channel, kHeld steps) composes them, a
// shift-and-compose over a channel's lanes follows, and every thread gets the
// state ahead of its own steps.  The next tile's loads are in flight during that.
// Rows are read once and written once, whatever the length.
//
// Where the channels do not fill the chip, the length is cut into chunks, a
// workgroup each: a first kernel composes each chunk's map (reading the gates a
// second time), the second one starts each chunk from the maps ahead of it.
//
// What bounds it: memory, for many channels (64 x 512 x 2048 in bf16: 117 us
// forward, 4.6 TB/s; 203 us backward, 4.6 TB/s), held back where a workgroup's runs
// are 64 bytes long: a card copies those at 3.8 TB/s, runs of 128 bytes at 4.8.
// 16 x 4096 x 512, of 64-byte runs: 69 us forward (3.9 TB/s), 122 us backward (3.9).
// One sequence of 16381 x 512 reads its gates twice: 10 + 15 us, 67 MB of inputs and
// outputs (2.7 TB/s).  A few short sequences take one tile's latency.
// Times here and below are the kernels' own in replayed graphs over several sets of
// inputs, both launches of a call in chunks together.
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
// Gates that a thread holds of a tile: with 32 the gradients spill registers, and the
// forward pass of 64 x 512 x 2048 bf16 takes an eighth longer.
constexpr int kHeld = 16;

// Which form a call takes.  LANES, 16-byte runs of a group: 8 make a 128-byte run of
// channels, 4 a 64-byte one with twice as many groups.  8 where that still gives
// kFull groups (three quarters of the compute units; 64 x 512 x 2048 bf16: 117 us
// against 134 forward, 203 against 245 backward), and where the length is cut into
// chunks anyway, to as many workgroups with either.  4 in between
// (16 x 4096 x 512, 256 groups of 64 bytes, or 128 of 128 in chunks: 69 against 81 us
// forward, 122 against 138 backward; without chunks 100 and 186).  fp32 has one form.
constexpr int64_t kFull = 192;
// Chunks, where there are fewer groups than kFull: so many that there are kChunked
// workgroups (16381 x 512: 26.9 us forward and 43.7 backward; with 256 27.3 and 47.7,
// with 1024 32.8 and 47.7), and at most kMostChunks, whose maps each chunk composes
// (32768 x 64: 18.0 and 23.0 us, with 64 chunks 22.9 and 37.4, with 128 17.8 and 25.6).
// Sequences of kWalked tiles or fewer are walked: a second launch and its workspace
// cost the host 5 us.  Four tiles of 4 x 1000 x 96 fp32 take 12.9 us forward and 17.5
// backward, in chunks 10.2 and 11.2; eight tiles of the gradients cost 22.6.
constexpr int64_t kChunked = 512, kMostChunks = 256, kWalked = 4;
// Threads of a workgroup.  The gradients hold twice the values: with kGradPairs of them
// two workgroups share a compute unit (64 x 512 x 2048: 203 us, with 512 threads 211).
// More threads are better where there is one group a compute unit, for the loads in
// flight (16 x 4096 x 512: 122 us with 512, 132 with 256), and where their longer tiles
// save the second launch: training 8 x 400 x 256 bf16 takes 27 us a pass instead of 32,
// but 3 x 500 x 75 fp16, whose short runs make slow tiles, 39 instead of 32.
constexpr int kThreads = 512, kGradPairs = 256;
// Sequences of at most kShort steps take a tile of as many: 37 x 4 x 1024 fp32 takes
// 11.8 us a call (bound by the host) instead of 16.4.
constexpr int64_t kShort = 2 * kHeld;
constexpr int short_threads(int V) { return 2 * 8 * V; }
// LANES: 16-byte runs of channels of a workgroup
template <typename Elem, int LANES> constexpr int kChannels = LANES * (16 / static_cast<int>(sizeof(Elem)));

// sigmoid(z) and sigmoid(-z), each within some (|z| + 8) 2^-24 of its own size (|z| from
// the exponent's rounding; 1 - f would lose the small one): with e = exp(-z) they are
// 1 / (1 + e) and e / (1 + e), which is 1 where e is large (e may be infinite); NaN stays
// NaN.
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
    int64_t columns;      // N * runs
    int32_t runs;         // runs of V channels in a row, the last one maybe short
    int64_t first;        // group of this launch
    uint32_t groups;      // of LANES columns, of this launch
    int32_t tiles;        // of a sequence
    int32_t chunk;        // tiles of a chunk
    int32_t chunks;
};

// A thread's S steps of one tensor, 16 bytes each, from step l0 of a row that
// starts at `row`; steps from L on repeat the last row (they are replaced later).
template <typename Elem, bool FULL, int S>
__device__ __forceinline__ void load_steps(const Elem* row, int64_t sl, int32_t l0, int32_t L, const RunShape& shape, int C,
                                           u32x4 (&raw)[S]) {
    const bool inside = l0 + S <= L;
    const Elem* p = row + static_cast<int64_t>(inside ? l0 : min(l0, L - 1)) * sl;
    const int last = inside ? S - 1 : max(0, L - 1 - l0);
    const Elem* at[S];
#pragma unroll
    for (int k = 0; k < S; ++k) at[k] = p + (k < last ? k : last) * sl;
    load_runs<Elem, FULL, S>(at, shape, C, raw);
}

// +infinity in every element: a gate that keeps the state (f = 1, i = 0)
template <typename Elem> constexpr uint32_t kKeep = 0x7f807f80u;
template <> constexpr uint32_t kKeep<float> = 0x7f800000u;
template <> constexpr uint32_t kKeep<_Float16> = 0x7c007c00u;

// LDS of a tile's composed maps: [part][segment of V][channel], a part's rows
// 4 words apart from the next one's, so that the parts of a few channels that a wave
// reads fall on different banks.
template <int T, typename Elem, int LANES> struct TileLds {
    static constexpr int V = Vec<Elem>::V, kParts = T / kChannels<Elem, LANES>;
    static constexpr int kPartWords = V * kChannels<Elem, LANES> + 4;
    static constexpr int kWords = kParts * kPartWords;
    static __device__ __forceinline__ int at(int segment, int channel) {
        return segment / V * kPartWords + segment % V * kChannels<Elem, LANES> + channel;
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
// meets first, `stride` apart, composed and applied to `state`.  The P lanes of a
// channel share them in order.
template <int P>
__device__ __forceinline__ float reach_chunk(const float2* maps, int64_t stride, int count, int part, float state) {
    const int each = (count + P - 1) / P;
    const int first = min(part * each, count), end = min(first + each, count);
    float A = 1.0f, B = 0.0f;
    for (int i = first; i < end; i += 4) {
        float2 m[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) m[u] = i + u < end ? maps[(i + u) * stride] : float2{1.0f, 0.0f};
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            B = fmaf(m[u].x, B, m[u].y);
            A *= m[u].x;
        }
    }
    compose_parts<P, true>(part, A, B);
    return fmaf(of_last_part<P, true>(A), state, of_last_part<P, true>(B));
}

// Which (chunk, group) a workgroup takes, all groups of chunk 0 first.  Workgroups go
// to the eight XCDs in turn.  Where groups share lines (halves of one, for groups of 64
// bytes; any, where a row is no whole number of groups), each XCD takes a run of the
// order instead, so that a line is fetched into one L2: 12 x 4000 x 136 bf16 25 us forward
// and 40 backward, in turn 34 and 56; 16 x 4096 x 512 in groups of 64 bytes 69 and 122, in
// turn 87 and 143.  Where they do not, in turn is better (16381 x 512: 26.9 and 43.7, in
// runs 28.3 and 45.5).
struct Share {
    int64_t group;
    int chunk;   // from `chunks` on: none
};
template <int LANES> __device__ __forceinline__ Share share_of_block(const Split& split, int chunks) {
    const bool apart = LANES == 8 && split.runs % LANES == 0;
    const uint32_t id = apart ? blockIdx.x : blockIdx.x % 8 * (gridDim.x / 8) + blockIdx.x / 8;
    const uint32_t chunk = id / split.groups;
    return {split.first + (id - chunk * split.groups), chunk < static_cast<uint32_t>(chunks) ? static_cast<int>(chunk) : chunks};
}

// A thread's place as the owner of steps: its column (a run of V channels) of a
// group, its S steps of a tile.
struct Place {
    int64_t n;
    int32_t c0, steps, l0;
    RunShape shape;   // no channels: no column
};
template <typename Elem, int LANES>
__device__ __forceinline__ Place place_of(const Split& split, const int32_t* lengths, int32_t L, int32_t C, int64_t group,
                                          int32_t t) {
    constexpr int V = Vec<Elem>::V, S = kHeld / V;
    const int64_t column = group * LANES + threadIdx.x % LANES;
    const bool has = column < split.columns;
    Place p;
    if (split.columns >> 31 == 0) {   // 32-bit division
        const uint32_t q = has ? static_cast<uint32_t>(column) / static_cast<uint32_t>(split.runs) : 0;
        p.n = q;
        p.c0 = has ? (static_cast<int32_t>(column) - static_cast<int32_t>(q) * split.runs) * V : 0;
    } else {
        p.n = has ? column / split.runs : 0;
        p.c0 = has ? static_cast<int32_t>(column - p.n * split.runs) * V : 0;
    }
    p.shape = has ? run_shape<Elem>(p.c0, C) : RunShape{0, 0};
    p.steps = has ? steps_of(lengths, p.n, L) : 0;
    p.l0 = t + static_cast<int32_t>(threadIdx.x) / LANES * S;
    return p;
}
// As a scanner: one channel of the group, one part (kHeld steps) of a tile.
struct Scanner {
    int64_t n;
    int32_t c;
    bool scans;
};
template <typename Elem, int LANES>
__device__ __forceinline__ Scanner scanner_of(const Split& split, int32_t C, int64_t group, int channel) {
    constexpr int V = Vec<Elem>::V;
    const int64_t column = group * LANES + channel / V;
    Scanner s;
    if (split.columns >> 31 == 0) {
        const uint32_t q = static_cast<uint32_t>(column) / static_cast<uint32_t>(split.runs);
        s.n = q;
        s.c = (static_cast<int32_t>(column) - static_cast<int32_t>(q) * split.runs) * V + channel % V;
    } else {
        s.n = column / split.runs;
        s.c = static_cast<int32_t>(column - s.n * split.runs) * V + channel % V;
    }
    s.scans = column < split.columns && s.c < C;
    return s;
}

template <typename Elem> struct ScanArgs {
    int64_t N;
    int32_t L, C;
    Rows<const Elem> gate, value, out_gate;
    Rows<Elem> y;
    const float* h0;
    const int32_t* lengths;
    float *h_last, *states;
    float2* maps;   // of the chunks in the scan's order: [chunk][group][channel]
    Split split;
};

// MAPS: only the chunks' maps.
template <typename Elem, int T, int LANES, bool OUT, bool FULL, bool MAPS>
__global__ __launch_bounds__(T) void scan_kernel(ScanArgs<Elem> a) {
    constexpr int V = Vec<Elem>::V, S = kHeld / V, CH = kChannels<Elem, LANES>, P = T / CH, TILE = P * kHeld;
    using Lds = TileLds<T, Elem, LANES>;
    __shared__ __align__(16) float lds[2][2][Lds::kWords];
    const int tid = threadIdx.x, lane = tid % LANES, segment = tid / LANES;
    const int channel = tid / P, part = tid % P;
    const int32_t L = a.L;
    const int64_t blocks = (static_cast<int64_t>(L) + kScanBlock - 1) / kScanBlock;
    auto start_of = [&](int32_t tile) { return tile * TILE; };

    const int chunks = a.split.chunks - (MAPS ? 1 : 0);   // nothing reads the last chunk's map
    const Share share = share_of_block<LANES>(a.split, chunks);
    if (share.chunk == chunks) return;
    const int64_t group = share.group;
    const int chunk = share.chunk, end = min((chunk + 1) * a.split.chunk, a.split.tiles);
    Place at = place_of<Elem, LANES>(a.split, a.lengths, L, a.C, group, start_of(chunk * a.split.chunk));
    const Scanner sc = scanner_of<Elem, LANES>(a.split, a.C, group, channel);
    const int64_t map_stride = static_cast<int64_t>(a.split.groups) * CH;
    float2* maps = a.maps + group * CH + channel;
    // the state ahead of the tile at hand, or the map of the chunk's tiles so far
    float carry = !MAPS && sc.scans && a.h0 ? a.h0[sc.n * a.C + sc.c] : 0.0f;
    float product = 1.0f;

    u32x4 z[S], v[S], o[S];
    auto load = [&](const Place& p) {
        if (!p.shape.valid || p.l0 >= p.steps) return;   // what is not loaded is replaced
        load_steps<Elem, FULL, S>(a.gate.at(p.n, 0) + p.c0, a.gate.sl, p.l0, L, p.shape, a.C, z);
        load_steps<Elem, FULL, S>(a.value.at(p.n, 0) + p.c0, a.value.sl, p.l0, L, p.shape, a.C, v);
        if (OUT && !MAPS) load_steps<Elem, FULL, S>(a.out_gate.at(p.n, 0) + p.c0, a.out_gate.sl, p.l0, L, p.shape, a.C, o);
    };
    if (chunk * a.split.chunk < end) load(at);
    if (!MAPS && chunk > 0) carry = reach_chunk<P>(maps, map_stride, chunk, part, carry);
    for (int tile = chunk * a.split.chunk, buf = 0; tile < end; ++tile, buf ^= 1) {
        float f[S][V], b[S][V], s[S][V];
        float A[V], B[V];
#pragma unroll
        for (int q = 0; q < V; ++q) {
            A[q] = 1.0f;
            B[q] = 0.0f;
        }
#pragma unroll
        for (int k = 0; k < S; ++k) {
            if (at.l0 + k >= at.steps) {   // padding: nothing of it is used
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
        // the next tile's loads go out ahead of what follows
        const Place here = at;
        if (tile + 1 < end) {
            at.l0 = start_of(tile + 1) + segment * S;
            load(at);
        }
        const int32_t t = start_of(tile);
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
                const float ta = of_last_part<P, true>(PA);
                carry = fmaf(ta, carry, of_last_part<P, true>(PB));
                product *= ta;
                continue;
            }
            // the state behind this part, and ahead of it
            const float behind = fmaf(PA, carry, PB);
            float h = from_lower<1>(behind);
            if (part == 0) h = carry;
            const int32_t block = (t + part * kHeld) / kScanBlock;
            if (a.states && sc.scans && part * kHeld % kScanBlock == 0 && block < blocks)
                a.states[(sc.n * blocks + block) * a.C + sc.c] = h;
            carry = of_last_part<P, true>(behind);
#pragma unroll
            for (int j = 0; j < V; ++j) {
                la[Lds::at(part * V + j, channel)] = h;
                h = fmaf(ma[j], h, mb[j]);
            }
        }
        __syncthreads();
        float h[V];
#pragma unroll
        for (int q = 0; q < V; q += 4) {
            const float4 w = *reinterpret_cast<const float4*>(la + Lds::at(segment, lane * V + q));
            h[q] = w.x, h[q + 1] = w.y, h[q + 2] = w.z, h[q + 3] = w.w;
        }
        Elem* y = a.y.at(here.n, here.l0) + here.c0;
#pragma unroll
        for (int k = 0; k < S; ++k) {
            float out[V];
#pragma unroll
            for (int q = 0; q < V; ++q) {
                h[q] = fmaf(f[k][q], h[q], b[k][q]);
                out[q] = OUT ? h[q] * s[k][q] : h[q];
            }
            u32x4 bits = Vec<Elem>::narrow(out);
            if (here.l0 + k >= here.steps) bits = u32x4{0, 0, 0, 0};
            if (here.shape.valid && here.l0 + k < L) store_run<Elem, FULL>(y + k * a.y.sl, here.shape.valid, bits);
        }
    }
    if (part == 0) {
        if (MAPS) maps[chunk * map_stride] = float2{product, carry};
        else if (sc.scans && chunk == a.split.chunks - 1) a.h_last[sc.n * a.C + sc.c] = carry;
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
    float2* maps;   // of the chunks in the scan's order: [chunk][group][channel]
    Split split;
};

// The gradients: tiles from the last to the first.  The forward pass kept the
// state ahead of each block of steps, so the states ahead of each thread's steps
// follow from the same composed maps without a scan over the parts.
template <typename Elem, int T, int LANES, bool OUT, bool FULL, bool MAPS>
__global__ __launch_bounds__(T) void scan_grad_kernel(GradArgs<Elem> a) {
    constexpr int V = Vec<Elem>::V, S = kHeld / V, CH = kChannels<Elem, LANES>, P = T / CH, TILE = P * kHeld;
    static_assert(2 * kHeld == kScanBlock && P % 2 == 0);
    using Lds = TileLds<T, Elem, LANES>;
    __shared__ __align__(16) float lds[2][3][Lds::kWords];
    const int tid = threadIdx.x, lane = tid % LANES, segment = tid / LANES;
    const int channel = tid / P, part = tid % P;
    const int32_t L = a.L;
    const int64_t blocks = (static_cast<int64_t>(L) + kScanBlock - 1) / kScanBlock;
    // tiles in the scan's order: 0 is the last one of the sequence
    auto start_of = [&](int32_t tile) { return (a.split.tiles - 1 - tile) * TILE; };

    const int chunks = a.split.chunks - (MAPS ? 1 : 0);   // nothing reads the last chunk's map
    const Share share = share_of_block<LANES>(a.split, chunks);
    if (share.chunk == chunks) return;
    const int64_t group = share.group;
    const int chunk = share.chunk, end = min((chunk + 1) * a.split.chunk, a.split.tiles);
    Place at = place_of<Elem, LANES>(a.split, a.lengths, L, a.C, group, start_of(chunk * a.split.chunk));
    const Scanner sc = scanner_of<Elem, LANES>(a.split, a.C, group, channel);
    const int64_t map_stride = static_cast<int64_t>(a.split.groups) * CH;
    float2* maps = a.maps + group * CH + channel;
    // the gradient behind the tile at hand, or the map of the chunk's tiles so far
    float carry = !MAPS && sc.scans && a.dh_last ? a.dh_last[sc.n * a.C + sc.c] : 0.0f;
    float product = 1.0f;

    u32x4 z[S], v[S], o[S], d[S];
    auto load = [&](const Place& p) {
        if (!p.shape.valid || p.l0 >= p.steps) return;   // what is not loaded is replaced
        load_steps<Elem, FULL, S>(a.gate.at(p.n, 0) + p.c0, a.gate.sl, p.l0, L, p.shape, a.C, z);
        load_steps<Elem, FULL, S>(a.dy.at(p.n, 0) + p.c0, a.dy.sl, p.l0, L, p.shape, a.C, d);
        if (!MAPS) load_steps<Elem, FULL, S>(a.value.at(p.n, 0) + p.c0, a.value.sl, p.l0, L, p.shape, a.C, v);
        if (OUT) load_steps<Elem, FULL, S>(a.out_gate.at(p.n, 0) + p.c0, a.out_gate.sl, p.l0, L, p.shape, a.C, o);
    };
    if (chunk * a.split.chunk < end) load(at);
    if (!MAPS && chunk > 0) carry = reach_chunk<P>(maps, map_stride, chunk, part, carry);
    for (int tile = chunk * a.split.chunk, buf = 0; tile < end; ++tile, buf ^= 1) {
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
            if (at.l0 + k >= at.steps) {
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
        // the next tile's loads go out ahead of what follows
        const Place here = at;
        if (tile + 1 < end) {
            at.l0 = start_of(tile + 1) + segment * S;
            load(at);
        }
        const int32_t t = start_of(tile);
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
        const int32_t block = (t + part * kHeld) / kScanBlock;
        float h = 0.0f;   // the state ahead of this part's block
        if (!MAPS && sc.scans && block < blocks) h = a.states[(sc.n * blocks + block) * a.C + sc.c];
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
                const float ta = of_last_part<P, false>(PA);
                carry = fmaf(ta, carry, of_last_part<P, false>(PR));
                product *= ta;
                continue;
            }
            const float ahead = fmaf(PA, carry, PR);   // the gradient that leaves this part
            float r = from_upper<1>(ahead);
            if (part == P - 1) r = carry;
            carry = of_last_part<P, false>(ahead);
            // the second half of a block starts where the first one ends
            float half = h;
#pragma unroll
            for (int j = 0; j < V; ++j) half = fmaf(ma[j], half, mb[j]);
            half = from_lower<1>(half);
            if (part % 2) h = half;
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
        Elem* dz = a.dgate.at(here.n, here.l0) + here.c0;
        Elem* dv = a.dvalue.at(here.n, here.l0) + here.c0;
        Elem* dout = OUT ? a.dout_gate.at(here.n, here.l0) + here.c0 : nullptr;
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
            if (here.l0 + k >= here.steps) bz = bv = bo = u32x4{0, 0, 0, 0};
            if (here.shape.valid && here.l0 + k < L) {
                store_run<Elem, FULL>(dz + k * a.dgate.sl, here.shape.valid, bz);
                store_run<Elem, FULL>(dv + k * a.dvalue.sl, here.shape.valid, bv);
                if (OUT) store_run<Elem, FULL>(dout + k * a.dout_gate.sl, here.shape.valid, bo);
            }
        }
    }
    if (part == 0) {
        if (MAPS) maps[chunk * map_stride] = float2{product, carry};
        else if (sc.scans && a.dh0 && chunk == a.split.chunks - 1) a.dh0[sc.n * a.C + sc.c] = carry;
    }
}

template <typename Elem> struct StepArgs {
    int64_t N, C;
    Rows<const Elem> gate, value, out_gate;
    Rows<Elem> y;
    const float* h;
    float* h_new;
};

// One thread per channel of a sequence: 16 x 512 take 2.4 us, a launch's latency;
// 256 x 4096 bf16 4.8 us, of which 16.8 MB at a copy's rate are 3.2.
template <typename Elem>
__global__ __launch_bounds__(kStepThreads) void step_kernel(StepArgs<Elem> a) {
    using S = Storage<Elem>;
    // more states than a launch has threads: in turns
    const int64_t all = a.N * a.C, stride = static_cast<int64_t>(gridDim.x) * kStepThreads;
    for (int64_t id = static_cast<int64_t>(blockIdx.x) * kStepThreads + threadIdx.x; id < all; id += stride) {
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
}

// How a call is cut.
struct Plan {
    Split split;
    int64_t groups;
    int lanes, threads;
};
Plan plan_scan(int dtype, int64_t N, int64_t L, int64_t C, bool backward) {
    const int V = 16 / dtype_bytes(dtype);
    Plan p;
    p.split.runs = static_cast<int32_t>((C + V - 1) / V);
    p.split.columns = N * p.split.runs;
    p.lanes = dtype == kF32 || L <= kShort || p.split.columns >= 8 * kFull || p.split.columns < 4 * kFull ? 8 : 4;
    const int64_t groups = p.groups = (p.split.columns + p.lanes - 1) / p.lanes;
    p.threads = L <= kShort ? short_threads(V) : kThreads;
    const bool one_launch = C % V == 0 && L <= kWalked * (kThreads / (8 * V) * kHeld);
    if (backward && L > kShort && p.lanes == 8 && (groups >= kFull || !one_launch)) p.threads = kGradPairs;
    const int64_t tile = p.threads / (p.lanes * V) * kHeld, tiles = (L + tile - 1) / tile;
    int64_t chunks = 1;
    if (groups < kFull && tiles > kWalked) chunks = std::min<int64_t>({tiles, kChunked / groups, kMostChunks});
    const int64_t each = std::max<int64_t>(1, (tiles + chunks - 1) / chunks);
    p.split.tiles = static_cast<int32_t>(tiles);
    p.split.chunk = static_cast<int32_t>(each);
    p.split.chunks = static_cast<int32_t>(std::max<int64_t>(1, (tiles + each - 1) / each));
    return p;
}

// launch(split, workgroups of the chunks' maps, workgroups).  HIP takes fewer than 2^32
// threads: more groups than that go in several launches (they have one chunk).
template <typename F> hipError_t launch_chunks(const Plan& p, F&& launch) {
    const int64_t chunks = p.split.chunks, most = chunks > 1 ? p.groups : int64_t(0xffffffff) / p.threads / 8 * 8;
    for (int64_t first = 0; first < p.groups; first += most) {
        Split split = p.split;
        const int64_t groups = std::min(p.groups - first, most);
        split.first = first;
        split.groups = static_cast<uint32_t>(groups);
        launch(split, static_cast<unsigned>((groups * (chunks - 1) + 7) / 8 * 8), static_cast<unsigned>((groups * chunks + 7) / 8 * 8));
    }
    return hipGetLastError();
}

#define WG_SCAN_CASES(X)                                                                \
    X(4, true, true) X(4, true, false) X(4, false, true) X(4, false, false)             \
    X(8, true, true) X(8, true, false) X(8, false, true) X(8, false, false)

}  // namespace

size_t gated_scan_workspace(int dtype, int64_t N, int64_t L, int64_t C, bool backward) {
    const Plan p = plan_scan(dtype, N, L, C, backward);
    if (p.split.chunks == 1) return 0;
    return static_cast<size_t>(p.split.chunks - 1) * p.groups * p.lanes * (16 / dtype_bytes(dtype)) * sizeof(float2);
}

template <int D> hipError_t launch_gated_scan_t(const wg_gated_scan& a, hipStream_t stream) {
    using Elem = typename DTypeOf<D>::type;
    constexpr int SHORT = short_threads(Vec<Elem>::V);
    const Plan p = plan_scan(D, a.N, a.L, a.C, false);
    ScanArgs<Elem> k{a.N, static_cast<int32_t>(a.L), static_cast<int32_t>(a.C), rows_of<const Elem>(a.gate),
                     rows_of<const Elem>(a.value), rows_of<const Elem>(a.out_gate), rows_of<Elem>(a.y), a.h0,
                     a.lengths, a.h_last, a.states, static_cast<float2*>(a.workspace), p.split};
    const bool out = a.out_gate.data != nullptr, full = a.C % Vec<Elem>::V == 0;
    return launch_chunks(p, [&](const Split& split, unsigned ahead, unsigned grid) {
        k.split = split;
#define WG_SCAN_CASE(LANES, OUT, FULL)                                                                               \
    if constexpr (LANES == 8 || D != kF32)                                                                           \
        if (p.lanes == LANES && out == OUT && full == FULL) {                                                        \
            constexpr int T = kThreads;                                                                              \
            if (LANES == 8 && ahead > 0) scan_kernel<Elem, T, 8, false, FULL, true><<<ahead, T, 0, stream>>>(k);   \
            if (LANES == 8 && p.threads == SHORT) scan_kernel<Elem, SHORT, 8, OUT, FULL, false><<<grid, SHORT, 0, stream>>>(k); \
            else scan_kernel<Elem, T, LANES, OUT, FULL, false><<<grid, T, 0, stream>>>(k);                           \
        }
        WG_SCAN_CASES(WG_SCAN_CASE)
#undef WG_SCAN_CASE
    });
}

template <int D> hipError_t launch_gated_scan_backward_t(const wg_gated_scan_backward& a, hipStream_t stream) {
    using Elem = typename DTypeOf<D>::type;
    constexpr int SHORT = short_threads(Vec<Elem>::V);
    const Plan p = plan_scan(D, a.N, a.L, a.C, true);
    GradArgs<Elem> k{a.N, static_cast<int32_t>(a.L), static_cast<int32_t>(a.C), rows_of<const Elem>(a.dy),
                     rows_of<const Elem>(a.gate), rows_of<const Elem>(a.value), rows_of<const Elem>(a.out_gate),
                     rows_of<Elem>(a.dgate), rows_of<Elem>(a.dvalue), rows_of<Elem>(a.dout_gate), a.states,
                     a.dh_last, a.lengths, a.dh0, static_cast<float2*>(a.workspace), p.split};
    const bool out = a.out_gate.data != nullptr, full = a.C % Vec<Elem>::V == 0;
    return launch_chunks(p, [&](const Split& split, unsigned ahead, unsigned grid) {
        k.split = split;
#define WG_SCAN_CASE(LANES, OUT, FULL)                                                                               \
    if constexpr (LANES == 8 || D != kF32)                                                                           \
        if (p.lanes == LANES && out == OUT && full == FULL) {                                                        \
            constexpr int T = kThreads, PAIRS = kGradPairs;                                                          \
            if (LANES == 8 && ahead > 0) scan_grad_kernel<Elem, PAIRS, 8, OUT, FULL, true><<<ahead, PAIRS, 0, stream>>>(k); \
            if (LANES == 8 && p.threads == SHORT)                                                                    \
                scan_grad_kernel<Elem, SHORT, 8, OUT, FULL, false><<<grid, SHORT, 0, stream>>>(k);                   \
            else if (LANES == 8 && p.threads == PAIRS)                                                               \
                scan_grad_kernel<Elem, PAIRS, 8, OUT, FULL, false><<<grid, PAIRS, 0, stream>>>(k);                   \
            else scan_grad_kernel<Elem, T, LANES, OUT, FULL, false><<<grid, T, 0, stream>>>(k);                      \
        }
        WG_SCAN_CASES(WG_SCAN_CASE)
#undef WG_SCAN_CASE
    });
}

template <int D> hipError_t launch_gated_step_t(const wg_gated_step& a, hipStream_t stream) {
    using Elem = typename DTypeOf<D>::type;
    const StepArgs<Elem> k{a.N, a.C, rows_of<const Elem>(a.gate), rows_of<const Elem>(a.value),
                           rows_of<const Elem>(a.out_gate), rows_of<Elem>(a.y), a.h, a.h_new};
    const int64_t blocks = std::min<int64_t>((a.N * a.C + kStepThreads - 1) / kStepThreads, 0xffffffffLL / kStepThreads);
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
