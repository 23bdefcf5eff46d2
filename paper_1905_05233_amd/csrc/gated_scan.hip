// The gated linear recurrence, its gradients and its single step on gfx950:
//   f = sigmoid(gate), i = 1 - f = sigmoid(-gate)
//   h[l] = f h[l-1] + i value[l],   y[l] = h[l] (times out_gate sigmoid(out_gate))
// and, with g[l] = dy[l] silu(out_gate[l]) and G the gradient at h[l],
//   G[l] = g[l] + f[l+1] G[l+1]  (G[L-1] = g[L-1] + dh_last)
//   dvalue[l] = i G[l],  dgate[l] = f i (h[l-1] - value[l]) G[l],  dh0 = f[0] G[0]
//   dout_gate[l] = dy[l] h[l] silu'(out_gate[l]).
// All of it in fp32; each result is rounded once to its type.
#include <hip/hip_runtime.h>

#include <cstdint>

#include "device_common.hpp"
#include "kernels.hpp"
#include "sequence.hpp"

namespace wg {

namespace {

constexpr int kScanThreads = 256;
constexpr int kScanBlock = WG_SCAN_BLOCK;

// sigmoid(z) and sigmoid(-z), both to fp32 accuracy for any z (1 - f would lose
// the small one): with t = exp(-|z|) they are 1 / (1 + t) and t / (1 + t).
struct Gate {
    float f, i;
};
__device__ __forceinline__ Gate gate_of(float z) {
    const float t = __expf(-fabsf(z));
    const float big = __builtin_amdgcn_rcpf(1.0f + t), small = t * big;
    return z < 0.0f ? Gate{small, big} : Gate{big, small};
}

template <typename Elem> struct Rows {
    Elem* p;
    int64_t sn, sl;
    __device__ __forceinline__ Elem* at(int64_t n, int64_t l) const { return p + n * sn + l * sl; }
};
template <typename Elem> Rows<Elem> rows_of(const wg_rows& r) {
    return {static_cast<Elem*>(const_cast<void*>(r.data)), r.stride_n, r.stride_l};
}

template <typename Elem> struct ScanArgs {
    int64_t N, L, C;
    Rows<const Elem> gate, value, out_gate;
    Rows<Elem> y;
    const float* h0;
    const int32_t* lengths;
    float *h_last, *states;
};

__device__ __forceinline__ int64_t steps_of(const int32_t* lengths, int64_t n, int64_t L) {
    if (!lengths) return L;
    const int64_t v = lengths[n];
    return v < 0 ? 0 : (v > L ? L : v);
}

// One thread per sequence and channel, one step after the other.
template <typename Elem>
__global__ __launch_bounds__(kScanThreads) void scan_kernel(ScanArgs<Elem> a) {
    using S = Storage<Elem>;
    const int64_t id = static_cast<int64_t>(blockIdx.x) * kScanThreads + threadIdx.x;
    if (id >= a.N * a.C) return;
    const int64_t n = id / a.C, c = id % a.C, steps = steps_of(a.lengths, n, a.L);
    const int64_t blocks = (a.L + kScanBlock - 1) / kScanBlock;
    float h = a.h0 ? a.h0[id] : 0.0f;
    for (int64_t l = 0; l < a.L; ++l) {
        if (a.states && l % kScanBlock == 0) a.states[(n * blocks + l / kScanBlock) * a.C + c] = h;
        float y = 0.0f;
        if (l < steps) {
            const Gate g = gate_of(S::to_f32(a.gate.at(n, l)[c]));
            h = g.f * h + g.i * S::to_f32(a.value.at(n, l)[c]);
            y = h;
            if (a.out_gate.p) {
                const float o = S::to_f32(a.out_gate.at(n, l)[c]);
                y = h * (o * gate_of(o).f);
            }
        }
        a.y.at(n, l)[c] = S::from_f32(y);
    }
    a.h_last[id] = h;
}

template <typename Elem> struct GradArgs {
    int64_t N, L, C;
    Rows<const Elem> dy, gate, value, out_gate;
    Rows<Elem> dgate, dvalue, dout_gate;
    const float *states, *dh_last;
    const int32_t* lengths;
    float* dh0;
};

// One thread per sequence and channel, from the last block of steps to the
// first; a block's states are computed again from the one ahead of it.
template <typename Elem>
__global__ __launch_bounds__(kScanThreads) void scan_grad_kernel(GradArgs<Elem> a) {
    using S = Storage<Elem>;
    const int64_t id = static_cast<int64_t>(blockIdx.x) * kScanThreads + threadIdx.x;
    if (id >= a.N * a.C) return;
    const int64_t n = id / a.C, c = id % a.C, steps = steps_of(a.lengths, n, a.L);
    const int64_t blocks = (a.L + kScanBlock - 1) / kScanBlock;
    float G = a.dh_last ? a.dh_last[id] : 0.0f;   // the gradient at the state behind the step at hand
    for (int64_t b = blocks - 1; b >= 0; --b) {
        float before[kScanBlock];
        float h = a.states[(n * blocks + b) * a.C + c];
        for (int k = 0; k < kScanBlock; ++k) {
            const int64_t l = b * kScanBlock + k;
            before[k] = h;
            if (l < steps) {
                const Gate g = gate_of(S::to_f32(a.gate.at(n, l)[c]));
                h = g.f * h + g.i * S::to_f32(a.value.at(n, l)[c]);
            }
        }
        for (int k = kScanBlock - 1; k >= 0; --k) {
            const int64_t l = b * kScanBlock + k;
            if (l >= a.L) continue;
            float dz = 0.0f, dv = 0.0f, dout = 0.0f;
            if (l < steps) {
                const Gate g = gate_of(S::to_f32(a.gate.at(n, l)[c]));
                const float v = S::to_f32(a.value.at(n, l)[c]);
                float dy = S::to_f32(a.dy.at(n, l)[c]);
                if (a.out_gate.p) {
                    const float o = S::to_f32(a.out_gate.at(n, l)[c]);
                    const Gate s = gate_of(o);
                    const float now = g.f * before[k] + g.i * v;
                    dout = dy * now * (s.f * (1.0f + o * s.i));
                    dy *= o * s.f;
                }
                G += dy;
                dv = g.i * G;
                dz = g.f * g.i * (before[k] - v) * G;
                G *= g.f;
            }
            a.dgate.at(n, l)[c] = S::from_f32(dz);
            a.dvalue.at(n, l)[c] = S::from_f32(dv);
            if (a.out_gate.p) a.dout_gate.at(n, l)[c] = S::from_f32(dout);
        }
    }
    if (a.dh0) a.dh0[id] = G;
}

template <typename Elem> struct StepArgs {
    int64_t N, C;
    Rows<const Elem> gate, value, out_gate;
    Rows<Elem> y;
    const float* h;
    float* h_new;
};

template <typename Elem>
__global__ __launch_bounds__(kScanThreads) void step_kernel(StepArgs<Elem> a) {
    using S = Storage<Elem>;
    const int64_t id = static_cast<int64_t>(blockIdx.x) * kScanThreads + threadIdx.x;
    if (id >= a.N * a.C) return;
    const int64_t n = id / a.C, c = id % a.C;
    const Gate g = gate_of(S::to_f32(a.gate.at(n, 0)[c]));
    const float h = g.f * a.h[id] + g.i * S::to_f32(a.value.at(n, 0)[c]);
    float y = h;
    if (a.out_gate.p) {
        const float o = S::to_f32(a.out_gate.at(n, 0)[c]);
        y = h * (o * gate_of(o).f);
    }
    a.h_new[id] = h;
    a.y.at(n, 0)[c] = S::from_f32(y);
}

}  // namespace

size_t gated_scan_workspace(int, int64_t, int64_t, int64_t, bool) { return 0; }

template <int D> hipError_t launch_gated_scan_t(const wg_gated_scan& a, hipStream_t stream) {
    using Elem = typename DTypeOf<D>::type;
    const ScanArgs<Elem> k{a.N, a.L, a.C, rows_of<const Elem>(a.gate), rows_of<const Elem>(a.value),
                           rows_of<const Elem>(a.out_gate), rows_of<Elem>(a.y), a.h0, a.lengths, a.h_last, a.states};
    const int64_t blocks = (a.N * a.C + kScanThreads - 1) / kScanThreads;
    if (blocks * kScanThreads > 0xffffffffLL) return hipErrorInvalidValue;
    scan_kernel<Elem><<<static_cast<unsigned>(blocks), kScanThreads, 0, stream>>>(k);
    return hipGetLastError();
}

template <int D> hipError_t launch_gated_scan_backward_t(const wg_gated_scan_backward& a, hipStream_t stream) {
    using Elem = typename DTypeOf<D>::type;
    const GradArgs<Elem> k{a.N, a.L, a.C, rows_of<const Elem>(a.dy), rows_of<const Elem>(a.gate),
                           rows_of<const Elem>(a.value), rows_of<const Elem>(a.out_gate), rows_of<Elem>(a.dgate),
                           rows_of<Elem>(a.dvalue), rows_of<Elem>(a.dout_gate), a.states, a.dh_last, a.lengths, a.dh0};
    const int64_t blocks = (a.N * a.C + kScanThreads - 1) / kScanThreads;
    if (blocks * kScanThreads > 0xffffffffLL) return hipErrorInvalidValue;
    scan_grad_kernel<Elem><<<static_cast<unsigned>(blocks), kScanThreads, 0, stream>>>(k);
    return hipGetLastError();
}

template <int D> hipError_t launch_gated_step_t(const wg_gated_step& a, hipStream_t stream) {
    using Elem = typename DTypeOf<D>::type;
    const StepArgs<Elem> k{a.N, a.C, rows_of<const Elem>(a.gate), rows_of<const Elem>(a.value),
                           rows_of<const Elem>(a.out_gate), rows_of<Elem>(a.y), a.h, a.h_new};
    const int64_t blocks = (a.N * a.C + kScanThreads - 1) / kScanThreads;
    if (blocks * kScanThreads > 0xffffffffLL) return hipErrorInvalidValue;
    step_kernel<Elem><<<static_cast<unsigned>(blocks), kScanThreads, 0, stream>>>(k);
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
