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

// A run of V channels from c0 of a row of C: how many it has, and how many too many
// it would have (0 for a whole run).
struct RunShape {
    int valid, over;
};
template <typename Elem> __device__ __forceinline__ RunShape run_shape(int c0, int C) {
    constexpr int V = Vec<Elem>::V;
    return {max(0, min(V, C - c0)), max(0, c0 + V - C)};
}

// Without its first n elements, zeros behind.
template <typename Elem> __device__ __forceinline__ u32x4 drop_first(const u32x4& b, int n) {
    if (n >= Vec<Elem>::V) return u32x4{0, 0, 0, 0};
    const uint64_t lo = static_cast<uint64_t>(b[1]) << 32 | b[0], hi = static_cast<uint64_t>(b[3]) << 32 | b[2];
    const int s = n * 8 * static_cast<int>(sizeof(Elem));
    const uint64_t l = s >= 64 ? hi >> (s - 64) : s > 0 ? lo >> s | hi << (64 - s) : lo;
    const uint64_t h = s >= 64 ? 0 : hi >> s;
    return u32x4{static_cast<uint32_t>(l), static_cast<uint32_t>(l >> 32), static_cast<uint32_t>(h),
                 static_cast<uint32_t>(h >> 32)};
}

// Runs from p.  A short run is the end of its row: 16 bytes that end with the row
// are loaded and shifted (rows of fewer than V channels are loaded one by one),
// which takes the same load as the other lanes' whole runs.
template <typename Elem, bool FULL, int S>
__device__ __forceinline__ void load_runs(const Elem* const (&p)[S], const RunShape& r, int C, u32x4 (&raw)[S]) {
    constexpr int V = Vec<Elem>::V;
    if (FULL || C >= V) {
#pragma unroll
        for (int k = 0; k < S; ++k) raw[k] = reinterpret_cast<const Bytes16*>(p[k] - (FULL ? 0 : r.over))->v;
        if (!FULL && r.over > 0) {
#pragma unroll
            for (int k = 0; k < S; ++k) raw[k] = drop_first<Elem>(raw[k], r.over);
        }
    } else {
#pragma unroll
        for (int k = 0; k < S; ++k) {
            typename Vec<Elem>::Packed e{};
#pragma unroll
            for (int j = 0; j < V; ++j)
                if (j < r.valid) e.v[j] = p[k][j];
            raw[k] = __builtin_bit_cast(u32x4, e);
        }
    }
}

// Stores a run, a short one in up to three pieces.
template <typename Elem, bool FULL>
__device__ __forceinline__ void store_run(Elem* p, int valid, const u32x4& bits) {
    if (FULL || valid == Vec<Elem>::V) {
        reinterpret_cast<Bytes16*>(p)->v = bits;
        return;
    }
    constexpr int kPer8 = 8 / sizeof(Elem);
    uint64_t w = static_cast<uint64_t>(bits[1]) << 32 | bits[0];
    if (valid & kPer8) {
        __builtin_memcpy(p, &w, 8);
        p += kPer8;
        w = static_cast<uint64_t>(bits[3]) << 32 | bits[2];
    }
    if (sizeof(Elem) == 4 ? valid & 1 : valid & 2) {
        const uint32_t x = static_cast<uint32_t>(w);
        __builtin_memcpy(p, &x, 4);
        p += 4 / sizeof(Elem);
        w >>= 32;
    }
    if (sizeof(Elem) == 2 && valid & 1) {
        const uint16_t x = static_cast<uint16_t>(w);
        __builtin_memcpy(p, &x, 2);
    }
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
