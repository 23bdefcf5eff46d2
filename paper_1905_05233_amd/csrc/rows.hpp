// Rows of storage elements as 16-byte runs, for the sequence operators (gfx950).
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "device_common.hpp"

namespace wg {

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
// 16 bytes at any element's address: the hardware takes such accesses whole
struct __attribute__((packed, aligned(2))) Bytes16 {
    u32x4 v;
};

template <typename Elem> struct Vec {
    static constexpr int V = 16 / sizeof(Elem);
    static __device__ __forceinline__ void widen(const u32x4& b, float (&f)[V]) {
        const auto e = __builtin_bit_cast(Packed, b);
#pragma unroll
        for (int q = 0; q < V; ++q) f[q] = Storage<Elem>::to_f32(e.v[q]);
    }
    static __device__ __forceinline__ u32x4 narrow(const float (&f)[V]) {
        Packed e;
#pragma unroll
        for (int q = 0; q < V; ++q) e.v[q] = Storage<Elem>::from_f32(f[q]);
        return __builtin_bit_cast(u32x4, e);
    }
    struct Packed {
        Elem v[V];
    };
};

template <typename Elem, bool FULL>
__device__ __forceinline__ void store_run(Elem* p, int valid, const u32x4& bits) {
    if (FULL || valid == Vec<Elem>::V) {
        reinterpret_cast<Bytes16*>(p)->v = bits;
    } else {
        const auto e = __builtin_bit_cast(typename Vec<Elem>::Packed, bits);
#pragma unroll
        for (int j = 0; j < Vec<Elem>::V; ++j)
            if (j < valid) p[j] = e.v[j];
    }
}

template <typename Elem> __device__ __forceinline__ u32x4 load_run(const Elem* p, int valid) {
    if (valid == Vec<Elem>::V) return reinterpret_cast<const Bytes16*>(p)->v;
    typename Vec<Elem>::Packed e{};
#pragma unroll
    for (int j = 0; j < Vec<Elem>::V; ++j)
        if (j < valid) e.v[j] = p[j];
    return __builtin_bit_cast(u32x4, e);
}

// The value of the lane whose number differs in bit N / 2 .. (N a power of two, 2 to
// 64), for reductions whose lower bits are done: the two halves of N lanes change
// places, in mirrored order below 32.
template <int N> __device__ __forceinline__ uint32_t other_half(uint32_t v) {
    if constexpr (N == 2) return __builtin_amdgcn_update_dpp(0, v, 0xb1, 0xf, 0xf, true);         // quad_perm 1 0 3 2
    else if constexpr (N == 4) return __builtin_amdgcn_update_dpp(0, v, 0x4e, 0xf, 0xf, true);    // quad_perm 2 3 0 1
    else if constexpr (N == 8) return __builtin_amdgcn_update_dpp(0, v, 0x141, 0xf, 0xf, true);   // row_half_mirror
    else if constexpr (N == 16) return __builtin_amdgcn_update_dpp(0, v, 0x140, 0xf, 0xf, true);  // row_mirror
    else return __shfl_xor(v, N / 2);
}
// Sum over each aligned group of N lanes, in every lane.
template <int N> __device__ __forceinline__ float lanes_sum(float v) {
    if constexpr (N > 1) {
        v = lanes_sum<N / 2>(v);
        v += __uint_as_float(other_half<N>(__float_as_uint(v)));
    }
    return v;
}
template <int N> __device__ __forceinline__ uint32_t lanes_max(uint32_t v) {
    if constexpr (N > 1) {
        v = lanes_max<N / 2>(v);
        const uint32_t o = other_half<N>(v);
        v = v > o ? v : o;
    }
    return v;
}

}  // namespace wg
