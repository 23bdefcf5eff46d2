// Linear attention with a decay for each head, its gradients and its single step on
// gfx950.  With lambda = exp(log_decay) of a head and its state S [Dk][Dv],
//   S[t] = lambda S[t-1] + k[t] v[t]^T,   y[t] = scale S[t]^T q[t].
// Steps are taken in tiles of T.  Within a tile, counted from 0 and with S the state
// ahead of it,
//   y[i] = scale (lambda^(i+1) S^T q[i] + sum_(j<=i) lambda^(i-j) (q[i].k[j]) v[j])
//   S'   = lambda^T S + sum_j lambda^(T-1-j) k[j] v[j]^T,
// which are four matrix products.  The gradients are the same products again, in
// other roles: dq is linear attention of (dy, v, k), and with the steps in reverse
// dk that of (v, dy, q) and dv that of (k, q, dy), where the state of the reversed
// ones is G, the gradient at the state, for which in a tile
//   y[i] = lambda^(T-1-i) G^T q[i] + scale sum_(j>=i) lambda^(j-i) (q[i].k[j]) v[j]
//   G'   = lambda^T G + scale sum_j lambda^(j+1) k[j] v[j]^T.
// So one kernel makes all of them (a "pass"; its q, k, v are the roles above).
//
// All products are the matrix cores' bf16 ones, with sums in fp32.  A value that 8
// bits do not hold goes in as the sum of two or three bf16 parts, each the rounding
// of what the ones ahead of it leave: fp16 inputs are exact in two, fp32 ones in
// three; the state, the weights q.k and the decayed v are held in fp32 and enter in
// two parts (2^-16 of a value is left) or, for fp32 rows, three.  Products of parts
// below that are left out.  bf16 has fp32's range, so no state overflows on the way.
//
// A workgroup takes a head of a sequence and a block of v's columns, whose state stays
// in the registers of its four waves, a quarter of the columns each; q, k and v of a
// tile stand in LDS, and the weights of the tile pass through it.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>
#include <type_traits>

#include "device_common.hpp"
#include "kernels.hpp"
#include "rows.hpp"
#include "sequence.hpp"

namespace wg {

namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr int kThreads = 256;   // of the kernels beside the attention itself
constexpr size_t kLdsBytes = 160 * 1024;
constexpr float kLog2e = 1.44269504088896340736f;

// bf16 parts of an input, of the values computed in fp32 that outputs are made of, and
// of those that the state is made of, which is returned in fp32
template <typename Elem> constexpr int kParts = std::is_same_v<Elem, bf16_t> ? 1 : std::is_same_v<Elem, _Float16> ? 2 : 3;
template <typename Elem> constexpr int kSums = std::is_same_v<Elem, float> ? 3 : 2;
constexpr int kStateParts = 3;
// steps of a tile
template <typename Elem> constexpr int kTile = std::is_same_v<Elem, bf16_t> ? 64 : 32;

// Heads of one tensor: [N][L][H][D] with the channels contiguous; `per` of the
// attention's heads read each.
struct HeadsIn {
    const void* p;
    int64_t sn, sl, sh;
    int32_t per;
};
struct HeadsOut {
    void* p;
    int64_t sn, sl, sh;
    int32_t f32;   // fp32 instead of the storage type
};

// Element (i, j) of a head's state at i row + j col.
struct StateAt {
    int32_t row, col;
};

struct Pass {
    HeadsIn q, k, v;
    HeadsOut y;
    int32_t kd, vd, blocks;   // channels of q and k, of v and y; blocks of columns
    const float* s_in;        // [N][H] states (or null: zeros), and the last ones (or null)
    float* s_out;
    StateAt at;
    float in_scale, out_scale;
    int32_t reverse;
    int32_t from_segments;    // s_in holds a state for each segment, [N][H][segments]
};

struct Args {
    Pass pass[3];
    int32_t first[4];         // workgroups of a segment of each pass, added up
    int64_t N;
    int32_t L, H;
    int32_t segments, each;   // runs of `each` tiles in the order of the walk
    const float* log_decay;
    const int32_t* lengths;
    float scale;
};

__device__ __forceinline__ int32_t steps_of(const int32_t* lengths, int64_t n, int32_t L) {
    if (!lengths) return L;
    const int32_t v = lengths[n];
    return v < 0 ? 0 : (v > L ? L : v);
}

// log2(lambda); where lambda is 0 a number whose every multiple but that by 0 is a
// power that is 0 in fp32.
__device__ __forceinline__ float log2_of(float log_decay) {
    return log_decay == -__builtin_inff() ? -1e30f : log_decay * kLog2e;
}
__device__ __forceinline__ float power(float log2_decay, int n) {
    return __builtin_amdgcn_exp2f(log2_decay * static_cast<float>(n));
}
// lambda^n to fp32's last place: the state is multiplied by it once a tile, and its
// errors would add up.
__device__ __forceinline__ float exact_power(float log_decay, int n) {
    return n == 0 ? 1.0f : static_cast<float>(exp(static_cast<double>(log_decay) * n));
}

// x as the sum of bf16 parts.  What an input's rounding leaves of an infinity is made
// finite (FINITE), so that the parts stay an infinity together.
template <int P, int V, bool FINITE> struct Split {
    typedef __bf16 Run __attribute__((ext_vector_type(V)));
    Run part[P];
    __device__ __forceinline__ void of(const float (&x)[V]) {
        typedef __bf16 Pair __attribute__((ext_vector_type(2)));
        typedef uint32_t Words __attribute__((ext_vector_type(V / 2)));
#pragma unroll
        for (int e = 0; e < V; e += 2) {
            float a = x[e], b = x[e + 1];
#pragma unroll
            for (int p = 0; p < P; ++p) {
                const uint32_t w = __builtin_bit_cast(uint32_t, Pair{static_cast<__bf16>(a), static_cast<__bf16>(b)});
                Words words = __builtin_bit_cast(Words, part[p]);
                words[e / 2] = w;
                part[p] = __builtin_bit_cast(Run, words);
                if (p + 1 == P) continue;
                a -= __uint_as_float(w << 16);
                b -= __uint_as_float(w & 0xffff0000u);
                if (FINITE) {
                    a = __builtin_amdgcn_fmed3f(a, -0x1p120f, 0x1p120f);
                    b = __builtin_amdgcn_fmed3f(b, -0x1p120f, 0x1p120f);
                }
            }
        }
    }
};

// c += a b over the parts whose product is not below the last of P
template <int PA, int PB, int P>
__device__ __forceinline__ f32x4 multiply(const bf16x8 (&a)[PA], const bf16x8 (&b)[PB], f32x4 c) {
#pragma unroll
    for (int i = 0; i < PA; ++i)
#pragma unroll
        for (int j = 0; j < PB; ++j)
            if (i + j < P) c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a[i], b[j], c, 0, 0, 0);
    return c;
}

// Rows of a tile in LDS, one plane a part, in runs of 8 channels whose order changes from
// row to row: the 16 rows that a fragment reads the same run of, and the four rows and
// runs that a transposing read takes, fall on different banks.
template <int PLANES, int ROWS, int WIDTH> struct alignas(16) TileLds {
    static constexpr int kRuns = WIDTH / 8;
    uint16_t v[PLANES][ROWS][WIDTH];

    static __device__ __forceinline__ int at(int row, int c) {
        const int by4 = row >> 2 & 3;
        const int mix = kRuns >= 16 ? (row & 3) << 2 | by4 : kRuns == 8 ? (row & 2) << 1 | by4 : by4;
        return (c / 8 ^ mix) * 8 + c % 8;
    }
    // 8 channels from c of a row, as a matrix instruction takes them of its row (or
    // column) `row`: lane m + 16 g holds 8 g .. 8 g + 7 of row m
    __device__ __forceinline__ void across(int row, int c, bf16x8 (&f)[PLANES]) const {
#pragma unroll
        for (int p = 0; p < PLANES; ++p) f[p] = *reinterpret_cast<const bf16x8*>(&v[p][row][at(row, c)]);
    }
    // 8 rows from `row` of a channel: the lanes of 16 hand in the places of four
    // channels in each of four rows, and lane m gets the four rows of channel m
    __device__ __forceinline__ void down(int row, int c, bf16x8 (&f)[PLANES]) const {
        using At = __attribute__((address_space(3))) s16x4*;
#pragma unroll
        for (int p = 0; p < PLANES; ++p) {
            const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((At)(&v[p][row][at(row, c)]));
            const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((At)(&v[p][row + 4][at(row + 4, c)]));
            f[p] = __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
        }
    }
};

// A tile's rows on their way from memory: 16 bytes of U rows a thread.  Every thread
// loads, from the first row and from the end of its row's channels where it has none of
// its own; what it then holds too many is dropped on the way to LDS.
template <typename Elem, int ROWS, int WIDTH, int THREADS> struct TileLoad {
    static constexpr int V = Vec<Elem>::V, kRuns = WIDTH / V, kPer = THREADS / kRuns, U = (ROWS + kPer - 1) / kPer;
    static_assert(THREADS % kRuns == 0 && (ROWS % kPer == 0 || U == 1), "threads cover whole rows");
    u32x4 raw[U];
    const Elem* base;   // the thread's channels of the sequence's first row
    int64_t stride, own;
    int r0, over;       // its first row; channels too many

    __device__ __forceinline__ TileLoad(const Elem* p, int64_t row_stride, int c0, int D) {
        const int c = c0 + static_cast<int>(threadIdx.x) % kRuns * V;
        r0 = threadIdx.x / kRuns;
        over = max(0, c + V - D);
        stride = row_stride;
        own = r0 * stride;
        base = p + (D >= V ? c - over : 0);
    }
    // rows 0 .. live - 1 (at least one) from row t0 of the sequence
    __device__ __forceinline__ void load(int32_t t0, int live, int D) {
        const Elem* p = base + t0 * stride;
        if (D >= V) {
#pragma unroll
            for (int u = 0; u < U; ++u)
                raw[u] = reinterpret_cast<const Bytes16*>(r0 + u * kPer < live ? p + own + u * kPer * stride : p)->v;
            return;
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {   // rows shorter than 16 bytes, in pieces of 8, 4 and 2
            raw[u] = u32x4{0, 0, 0, 0};
            if (r0 + u * kPer >= live || over >= V) continue;
            const Elem* at = p + own + u * kPer * stride;
            constexpr int kPer8 = 8 / sizeof(Elem);
            uint64_t head = 0, tail = 0;
            if (D & kPer8) {
                __builtin_memcpy(&head, at, 8);
                at += kPer8;
            }
            if (sizeof(Elem) == 4 ? D & 1 : D & 2) {
                uint32_t w;
                __builtin_memcpy(&w, at, 4);
                at += 4 / sizeof(Elem);
                tail = w;
            }
            if (sizeof(Elem) == 2 && D & 1) {
                uint16_t w;
                __builtin_memcpy(&w, at, 2);
                tail |= static_cast<uint64_t>(w) << (D & 2 ? 32 : 0);
            }
            if (!(D & kPer8)) head = tail, tail = 0;
            raw[u] = u32x4{static_cast<uint32_t>(head), static_cast<uint32_t>(head >> 32), static_cast<uint32_t>(tail),
                           static_cast<uint32_t>(tail >> 32)};
        }
    }
    // what is loaded without what it holds too many; `whole`: that is nothing, for all threads
    __device__ __forceinline__ void trim(bool whole, int live, int D) {
        if (whole || D < V) return;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            raw[u] = drop_first<Elem>(raw[u], over);
            if (r0 + u * kPer >= live) raw[u] = u32x4{0, 0, 0, 0};
        }
    }
    template <int PLANES> __device__ __forceinline__ void store(TileLds<PLANES, ROWS, WIDTH>& to) const {
        const int c = static_cast<int>(threadIdx.x) % kRuns * V;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int row = r0 + u * kPer;
            if (ROWS % kPer != 0 && row >= ROWS) continue;
            if constexpr (PLANES == 1) {
                *reinterpret_cast<u32x4*>(&to.v[0][row][to.at(row, c)]) = raw[u];
            } else {
                float x[V];
                Vec<Elem>::widen(raw[u], x);
                Split<PLANES, V, true> s;
                s.of(x);
#pragma unroll
                for (int p = 0; p < PLANES; ++p)
                    *reinterpret_cast<typename Split<PLANES, V, true>::Run*>(&to.v[p][row][to.at(row, c)]) = s.part[p];
            }
        }
    }
    __device__ __forceinline__ bool finite() const {
        if constexpr (sizeof(Elem) == 4) {
            uint32_t top = 0;
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int e = 0; e < 4; ++e) top = max(top, raw[u][e] & 0x7fffffffu);
            return top < 0x7f800000u;
        } else {
            typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
            u16x2 top = {0, 0};
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    top = __builtin_elementwise_max(top, __builtin_bit_cast(u16x2, raw[u][e] & 0x7fff7fffu));
            constexpr unsigned short kInf = std::is_same_v<Elem, bf16_t> ? 0x7f80 : 0x7c00;
            return top[0] < kInf && top[1] < kInf;
        }
    }
};

template <typename Elem> __device__ __forceinline__ const Elem* heads_at(const HeadsIn& t, int64_t n, int32_t h) {
    return static_cast<const Elem*>(t.p) + n * t.sn + h / t.per * t.sh;
}

// Four values side by side, of which those below `valid` are wanted.
template <typename T> __device__ __forceinline__ void store_values(T* to, const f32x4& x, int valid) {
    struct __attribute__((packed, aligned(sizeof(T)))) Two {
        T v[2];
    };
    struct __attribute__((packed, aligned(sizeof(T)))) Four {
        T v[4];
    };
    T e[4];
#pragma unroll
    for (int r = 0; r < 4; ++r) e[r] = Storage<T>::from_f32(x[r]);
    if (valid >= 4) *reinterpret_cast<Four*>(to) = Four{e[0], e[1], e[2], e[3]};
    else {
        if (valid >= 2) *reinterpret_cast<Two*>(to) = Two{e[0], e[1]};
        if (valid == 1) to[0] = e[0];
        if (valid == 3) to[2] = e[2];
    }
}

struct None {};

// Tiles of K channels of q and k for W waves of 16 C columns each.
template <typename Elem, int K, int W, int C, bool STATES> struct Shape {
    static constexpr int T = kTile<Elem>, PI = kParts<Elem>, PS = kSums<Elem>;
    static constexpr int kColumns = 16 * C * W, kThreads = 64 * W;
    struct Steps {
        std::conditional_t<STATES, None, TileLds<PI, T, K>> q;
        TileLds<PI, T, K> k;
        TileLds<PI, T, kColumns> v;
    };
    struct Weights {
        TileLds<PS, T, T> p;
        int32_t odd[2];   // the tile (+ 1) of which v holds an infinity or NaN
    };
    // two tiles of steps, where they find room
    static constexpr int kStages = 2 * sizeof(Steps) + sizeof(Weights) <= kLdsBytes ? 2 : 1;
    struct Lds {
        Steps steps[kStages];
        std::conditional_t<STATES, None, Weights> weights;
    };
};

// A pass, or (STATES) only what its segments add to the state.  A wave's accumulators of
// the state: S[b][c], lane m + 16 g, register r holds the state at
// (32 (b / 2) + 8 g + 4 (b % 2) + r, column(c, m)), so that those of two blocks side by
// side are the 8 consecutive rows that a lane hands a matrix instruction, without a
// move.  Outputs come transposed, O[i][c] with row 16 i + m and columns
// column(c, 4 g + r): 4 C of them side by side.
template <typename Elem, int KD, int W, int CB, bool STATES>
__global__ __launch_bounds__(64 * W, 2) void attention_kernel(Args a) {
    using Sh = Shape<Elem, KD, W, CB, STATES>;
    constexpr int T = Sh::T, PI = Sh::PI, PS = Sh::PS, VB = Sh::kColumns, NT = Sh::kThreads, IB = T / 16, JS = T / 32, KS = KD / 32;
    constexpr int STAGES = Sh::kStages;
    __shared__ __align__(16) typename Sh::Lds lds;
    const int tid = threadIdx.x, wave = tid / 64, lane = tid % 64, m = lane % 16, g = lane / 16;

    const int32_t segment = blockIdx.x / static_cast<uint32_t>(a.first[3]);
    const int32_t id = blockIdx.x - segment * a.first[3];
    const int which = id >= a.first[2] ? 2 : id >= a.first[1] ? 1 : 0;
    const Pass& pass = a.pass[which];
    const uint32_t unit = id - a.first[which];
    const uint32_t head = unit / static_cast<uint32_t>(pass.blocks);
    const int32_t block = unit - head * pass.blocks, h = head % static_cast<uint32_t>(a.H);
    const int64_t n = head / static_cast<uint32_t>(a.H);
    const int32_t steps = steps_of(a.lengths, n, a.L), kd = pass.kd, vd = pass.vd, v0 = block * VB;
    const bool reverse = pass.reverse != 0, y_f32 = pass.y.f32 != 0;
    const float log_decay = a.log_decay[h], log2_decay = log2_of(log_decay);
    const float in_scale = pass.in_scale, out_scale = pass.out_scale, scale = a.scale;

    auto column = [&](int c, int i) { return CB == 1 ? 16 * wave + i : 32 * wave + 8 * (i / 4) + 4 * c + i % 4; };
    // channels that a lane hands to a transposing read, of the state's rows and columns
    auto row_chunk = [&](int b) { return 32 * (b / 2) + 8 * (m % 4) + 4 * (b % 2); };
    auto column_chunk = [&](int c) { return column(c, 4 * (m % 4)); };

    f32x4 S[KD / 16][CB];
    auto each_state = [&](auto&& f) {
#pragma unroll
        for (int b = 0; b < KD / 16; ++b)
#pragma unroll
            for (int c = 0; c < CB; ++c)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int i = 32 * (b / 2) + 8 * g + 4 * (b % 2) + r, j = v0 + column(c, m);
                    if (i < kd && j < vd) S[b][c][r] = f(S[b][c][r], i * pass.at.row + j * pass.at.col);
                }
    };
#pragma unroll
    for (int b = 0; b < KD / 16; ++b)
#pragma unroll
        for (int c = 0; c < CB; ++c) S[b][c] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    const int64_t size = static_cast<int64_t>(kd) * vd, by_segment = (static_cast<int64_t>(head) * a.segments + segment) * size;
    if (!STATES && pass.s_in) {
        const float* s = pass.s_in + (pass.from_segments ? by_segment : head * size);
        each_state([&](float, int at) { return s[at]; });
    }

    const int32_t tiles = (steps + T - 1) / T, t_first = segment * a.each, t_end = min(tiles, t_first + a.each);
    const int64_t y_sl = pass.y.sl;
    const Elem* q = heads_at<Elem>(pass.q, n, h);
    const Elem* k = heads_at<Elem>(pass.k, n, h);
    const Elem* v = heads_at<Elem>(pass.v, n, h);
    // a lane's outputs: 4 CB values side by side in row m of every 16
    const int y_valid = vd - (v0 + column(0, 4 * g));
    const int64_t y_at = n * pass.y.sn + h * pass.y.sh + m * y_sl + v0 + column(0, 4 * g);
    TileLoad<Elem, T, KD, NT> lq(q, pass.q.sl, 0, kd), lk(k, pass.k.sl, 0, kd);
    TileLoad<Elem, T, VB, NT> lv(v, pass.v.sl, v0, vd);
    const bool wide = kd == KD && vd - v0 >= VB;
    if constexpr (!STATES) {
        // weights above the diagonal are zeros that nothing writes
        for (int i = tid; i < static_cast<int>(sizeof(lds.weights) / 4); i += NT) reinterpret_cast<uint32_t*>(&lds.weights)[i] = 0;
    }

    // decays: over a tile, from the state to its steps, from its steps to the state
    float whole = 1.0f, out_decay[IB], in_decay[JS][8];
    int decays_of = 0;
    auto set_decays = [&](int live) {
        decays_of = live;
        whole = exact_power(log_decay, live);
#pragma unroll
        for (int i = 0; i < IB; ++i)
            out_decay[i] = out_scale * power(log2_decay, reverse ? max(0, live - 1 - (16 * i + m)) : 16 * i + m + 1);
#pragma unroll
        for (int s = 0; s < JS; ++s)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int j = 32 * s + 8 * g + e;
                in_decay[s][e] = in_scale * power(log2_decay, reverse ? j + 1 : max(0, live - 1 - j));
            }
    };

    // The first state is there ahead of the rounds: each of them would wait for it, and
    // for its own loads with it.
#pragma unroll
    for (int b = 0; b < KD / 16; ++b)
#pragma unroll
        for (int c = 0; c < CB; ++c) asm volatile("" : "+v"(S[b][c]));
    // a round multiplies tile t, and has tile t + 1 loaded and brought to LDS
    for (int32_t t = t_first - 1; t < t_end; ++t) {
        const int32_t next0 = (reverse ? tiles - 2 - t : t + 1) * T, t0 = reverse ? next0 + T : next0 - T;
        const bool more = t + 1 < t_end, has = t >= t_first;
        auto& now = lds.steps[t & (STAGES - 1)];
        auto& next = lds.steps[(t + 1) & (STAGES - 1)];
        if (more) {
            const int32_t live = min(T, steps - next0);
            if constexpr (!STATES) lq.load(next0, live, kd);
            lk.load(next0, live, kd);
            lv.load(next0, live, vd);
        }
        const int32_t live = min(T, steps - t0);
        f32x4 O[IB][CB];
        bf16x8 fv[JS][CB][PI];
        if (has) {
            if (live != decays_of) set_decays(live);
            if constexpr (!STATES) {
                // the weights of the tile, in blocks of 16 x 16 of the triangle
                for (int blk = wave; blk < IB * (IB + 1) / 2; blk += W) {
                    const int far = blk >= 6 ? 3 : blk >= 3 ? 2 : blk >= 1 ? 1 : 0, near = blk - far * (far + 1) / 2;
                    const int ib = reverse ? near : far, jb = reverse ? far : near;
                    f32x4 w = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                    for (int s = 0; s < KS; ++s) {
                        bf16x8 fk[PI], fq[PI];
                        now.k.across(16 * jb + m, 32 * s + 8 * g, fk);
                        now.q.across(16 * ib + m, 32 * s + 8 * g, fq);
                        w = multiply<PI, PI, PS>(fk, fq, w);
                    }
                    float x[4];
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const int i = 16 * ib + m, j = 16 * jb + 4 * g + r, d = reverse ? j - i : i - j;
                        x[r] = d < 0 ? 0.0f : w[r] * (scale * power(log2_decay, d));
                    }
                    Split<PS, 4, false> parts;
                    parts.of(x);
                    auto& to = lds.weights.p;
                    const int row = 16 * ib + m, c = 16 * jb + 4 * g;
#pragma unroll
                    for (int p = 0; p < PS; ++p) *reinterpret_cast<bf16x4*>(&to.v[p][row][to.at(row, c)]) = parts.part[p];
                }

                // what the state gives
#pragma unroll
                for (int i = 0; i < IB; ++i)
#pragma unroll
                    for (int c = 0; c < CB; ++c) O[i][c] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                for (int s = 0; s < KS; ++s) {
                    Split<PS, 8, false> fs[CB];
#pragma unroll
                    for (int c = 0; c < CB; ++c) {
                        float x[8];
#pragma unroll
                        for (int e = 0; e < 8; ++e) x[e] = S[2 * s + e / 4][c][e % 4];
                        fs[c].of(x);
                    }
#pragma unroll
                    for (int i = 0; i < IB; ++i) {
                        bf16x8 fq[PI];
                        now.q.across(16 * i + m, 32 * s + 8 * g, fq);
#pragma unroll
                        for (int c = 0; c < CB; ++c) O[i][c] = multiply<PS, PI, PS>(fs[c].part, fq, O[i][c]);
                    }
                }
#pragma unroll
                for (int i = 0; i < IB; ++i)
#pragma unroll
                    for (int c = 0; c < CB; ++c) O[i][c] *= out_decay[i];
            }

            // the state behind the tile
#pragma unroll
            for (int b = 0; b < KD / 16; ++b)
#pragma unroll
                for (int c = 0; c < CB; ++c) S[b][c] *= whole;
#pragma unroll
            for (int s = 0; s < JS; ++s) {
                Split<kStateParts, 8, false> late[CB];
#pragma unroll
                for (int c = 0; c < CB; ++c) {
                    now.v.down(32 * s + 8 * g + m / 4, column_chunk(c), fv[s][c]);
                    float x[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        float sum = 0.0f;
#pragma unroll
                        for (int p = PI - 1; p >= 0; --p) sum += static_cast<float>(fv[s][c][p][e]);
                        x[e] = sum * in_decay[s][e];
                    }
                    late[c].of(x);
                }
#pragma unroll
                for (int b = 0; b < KD / 16; ++b) {
                    bf16x8 fk[PI];
                    now.k.down(32 * s + 8 * g + m / 4, row_chunk(b), fk);
#pragma unroll
                    for (int c = 0; c < CB; ++c) S[b][c] = multiply<PI, kStateParts, kStateParts>(fk, late[c].part, S[b][c]);
                }
            }
        }
        // The next tile's rows go to LDS ahead of this one's outputs: the wait for them
        // is for every access to memory before it, stores too.
        auto stage = [&] {
            if (!more) return;
            const int32_t live = min(T, steps - next0);
            const bool whole_tile = wide && live == T;
            lk.trim(whole_tile, live, kd);
            lv.trim(whole_tile, live, vd);
            if constexpr (!STATES) {
                lq.trim(whole_tile, live, kd);
                lq.template store<PI>(next.q);
                if (!lv.finite()) lds.weights.odd[(t + 1) & 1] = t + 2;
            }
            lk.template store<PI>(next.k);
            lv.template store<PI>(next.v);
        };
        if constexpr (!STATES) __syncthreads();   // the weights
        if constexpr (STAGES == 2) stage();
        if constexpr (!STATES) {
            if (has) {
                // what the tile's own steps give
                if (lds.weights.odd[t & 1] != t + 1) {
#pragma unroll
                    for (int i = 0; i < IB; ++i)
#pragma unroll
                        for (int s = 0; s < JS; ++s) {
                            if (reverse ? 32 * s + 31 < 16 * i : 32 * s > 16 * i + 15) continue;
                            bf16x8 fp[PS];
                            lds.weights.p.across(16 * i + m, 32 * s + 8 * g, fp);
#pragma unroll
                            for (int c = 0; c < CB; ++c) O[i][c] = multiply<PI, PS, PS>(fv[s][c], fp, O[i][c]);
                        }
                } else {
                    // step by step: a weight of zero would not remove an infinity or NaN of a later v
                    auto value = [](const auto& tile, int row, int c) {
                        float sum = 0.0f;
#pragma unroll
                        for (int p = std::extent_v<std::remove_reference_t<decltype(tile.v)>> - 1; p >= 0; --p)
                            sum += __uint_as_float(static_cast<uint32_t>(tile.v[p][row][tile.at(row, c)]) << 16);
                        return sum;
                    };
#pragma unroll 1
                    for (int j = 0; j < T; ++j)
#pragma unroll
                        for (int i = 0; i < IB; ++i) {
                            const int row = 16 * i + m;
                            if (reverse ? j < row : j > row) continue;
                            const float w = value(lds.weights.p, row, j);
#pragma unroll
                            for (int c = 0; c < CB; ++c)
#pragma unroll
                                for (int r = 0; r < 4; ++r) O[i][c][r] += w * value(now.v, j, column(c, 4 * g + r));
                        }
                }
            }
        }
        if constexpr (STAGES == 1) {
            __syncthreads();
            stage();
        }
        if constexpr (!STATES) {
            if (has && y_valid > 0) {
#pragma unroll
                for (int i = 0; i < IB; ++i) {
                    if (16 * i + m >= live) continue;
                    const int64_t at = y_at + (t0 + 16 * i) * y_sl;
#pragma unroll
                    for (int c = 0; c < CB; ++c) {
                        if (y_f32) store_values<float>(static_cast<float*>(pass.y.p) + at + 4 * c, O[i][c], y_valid - 4 * c);
                        else store_values<Elem>(static_cast<Elem*>(pass.y.p) + at + 4 * c, O[i][c], y_valid - 4 * c);
                    }
                }
            }
        }
        __syncthreads();
    }

    if constexpr (STATES) {
        float* s = pass.s_out + by_segment;
        each_state([&](float x, int at) { return s[at] = x; });
    } else {
        // padding, of which each segment takes a share of rows
        const int width = min(VB, vd - v0), share = (a.L - steps + a.segments - 1) / a.segments;
        const int32_t row0 = steps + min(segment * static_cast<int64_t>(share), static_cast<int64_t>(a.L - steps));
        const int64_t values = static_cast<int64_t>(min(share, a.L - row0)) * width;
        for (int64_t i = tid; i < values; i += NT) {
            const int64_t at = n * pass.y.sn + (row0 + i / width) * y_sl + h * pass.y.sh + v0 + i % width;
            if (y_f32) static_cast<float*>(pass.y.p)[at] = 0.0f;
            else static_cast<Elem*>(pass.y.p)[at] = Storage<Elem>::from_f32(0.0f);
        }
        if (!pass.s_out) return;
        float* s = pass.s_out + head * size;
        each_state([&](float x, int at) { return s[at] = x; });
    }
}

// The states ahead of the segments from what each adds: in place, [N][H][segments] of
// `size` values, from s_in [N][H] (or null: zeros) to s_out (or null).
struct Chain {
    float* states;
    const float* s_in;
    float* s_out;
    int32_t size, reverse;
};
struct ChainArgs {
    Chain chain[2];
    int64_t heads;            // N H
    int32_t L, H, segments, each_steps, tile, blocks, of;
    const float* log_decay;
    const int32_t* lengths;
};
__global__ __launch_bounds__(kThreads) void chain_kernel(ChainArgs a) {
    constexpr int U = 8;      // segments whose loads are in flight together
    const Chain& c = a.chain[blockIdx.x % a.of];
    const uint32_t unit = blockIdx.x / a.of;
    const int64_t head = unit / a.blocks;
    const int32_t i = static_cast<int32_t>(unit % a.blocks) * kThreads + threadIdx.x;
    if (i >= c.size) return;
    const int32_t steps = steps_of(a.lengths, head / a.H, a.L), end = (steps + a.tile - 1) / a.tile * a.tile;
    const float log_decay = a.log_decay[head % a.H];
    // steps of a segment: all but the last have each_steps, but the reverse of a walk
    // begins with the tile that may be short
    auto steps_in = [&](int32_t w) {
        const int64_t from = static_cast<int64_t>(w) * a.each_steps, to = min(static_cast<int64_t>(end), from + a.each_steps);
        if (from >= end) return 0;
        return static_cast<int32_t>(c.reverse ? min(static_cast<int64_t>(steps), end - from) - (end - to)
                                              : min(static_cast<int64_t>(steps), to) - from);
    };
    const float whole = exact_power(log_decay, a.each_steps);
    float* s = c.states + head * a.segments * static_cast<int64_t>(c.size) + i;
    float run = c.s_in ? c.s_in[head * c.size + i] : 0.0f;
    for (int32_t w = 0; w < a.segments; w += U) {
        float add[U];
#pragma unroll
        for (int u = 0; u < U; ++u) add[u] = w + u < a.segments ? s[(w + u) * static_cast<int64_t>(c.size)] : 0.0f;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (w + u >= a.segments) continue;
            s[(w + u) * static_cast<int64_t>(c.size)] = run;
            const int32_t count = steps_in(w + u);
            if (count > 0) run = fmaf(count == a.each_steps ? whole : exact_power(log_decay, count), run, add[u]);
        }
    }
    if (c.s_out) c.s_out[head * c.size + i] = run;
}

// Gradients of an input that heads share: the sum over them of their parts
// [N][L][H][D] in fp32, in the order of the heads.
template <typename Elem>
__global__ __launch_bounds__(kThreads) void shared_kernel(const float* part, HeadsOut to, int64_t rows, int32_t L, int32_t heads,
                                                          int32_t per, int32_t D) {
    const int64_t all = rows * heads * D, stride = static_cast<int64_t>(gridDim.x) * kThreads;
    for (int64_t id = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x; id < all; id += stride) {
        const int64_t row = id / (heads * static_cast<int64_t>(D));
        const int32_t h = id / D % heads, d = id % D;
        const float* p = part + (row * heads + h) * per * D + d;
        float sum = 0.0f;
        for (int32_t u = 0; u < per; ++u) sum += p[static_cast<int64_t>(u) * D];
        static_cast<Elem*>(to.p)[row / L * to.sn + row % L * to.sl + h * to.sh + d] = Storage<Elem>::from_f32(sum);
    }
}

struct StepArgs {
    HeadsIn q, k, v;
    HeadsOut y;
    int64_t N;
    int32_t H, kd, vd, blocks;
    const float* log_decay;
    const float* s;
    float* s_new;
    float scale;
};

// One step: a workgroup takes 64 columns of a head's state, a thread 4 of them in every
// 16th row.  Bound by the states' memory.
constexpr int kStepColumns = 64, kStepRows = kThreads / (kStepColumns / 4);
template <typename Elem>
__global__ __launch_bounds__(kThreads) void step_kernel(StepArgs a) {
    using St = Storage<Elem>;
    __shared__ float lds[kStepRows][kStepColumns + 4];
    const int64_t units = a.N * a.H * a.blocks;
    const int c = threadIdx.x % (kStepColumns / 4) * 4, r0 = threadIdx.x / (kStepColumns / 4);
    for (int64_t unit = blockIdx.x; unit < units; unit += gridDim.x) {
        const int32_t j = static_cast<int32_t>(unit % a.blocks) * kStepColumns + c, h = unit / a.blocks % a.H;
        const int64_t n = unit / a.blocks / a.H;
        const Elem* q = heads_at<Elem>(a.q, n, h);
        const Elem* k = heads_at<Elem>(a.k, n, h);
        const Elem* v = heads_at<Elem>(a.v, n, h);
        const float keep = exact_power(a.log_decay[h], 1);
        const int valid = min(4, a.vd - j);
        float x[4], sum[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = e < valid ? St::to_f32(v[j + e]) : 0.0f;
        const int64_t at = ((n * a.H + h) * a.kd) * static_cast<int64_t>(a.vd) + j;
        for (int i = r0; i < a.kd; i += kStepRows) {
            const float ki = St::to_f32(k[i]), qi = St::to_f32(q[i]);
            const float* s = a.s + at + static_cast<int64_t>(i) * a.vd;
            float* s_new = a.s_new + at + static_cast<int64_t>(i) * a.vd;
            if (valid == 4) {
                f32x4 w = __builtin_bit_cast(f32x4, reinterpret_cast<const Bytes16*>(s)->v);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    w[e] = fmaf(keep, w[e], ki * x[e]);
                    sum[e] = fmaf(qi, w[e], sum[e]);
                }
                reinterpret_cast<Bytes16*>(s_new)->v = __builtin_bit_cast(u32x4, w);
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    if (e >= valid) continue;
                    const float w = fmaf(keep, s[e], ki * x[e]);
                    sum[e] = fmaf(qi, w, sum[e]);
                    s_new[e] = w;
                }
            }
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) lds[r0][c + e] = sum[e];
        __syncthreads();
        const int column = threadIdx.x, jj = j - c + column;
        if (column < kStepColumns && jj < a.vd) {
            float y = 0.0f;
#pragma unroll
            for (int r = 0; r < kStepRows; ++r) y += lds[r][column];
            static_cast<Elem*>(a.y.p)[n * a.y.sn + h * a.y.sh + jj] = St::from_f32(a.scale * y);
        }
        __syncthreads();
    }
}

HeadsIn heads_in(const wg_heads& t, int64_t heads, int64_t H) {
    return {t.data, t.stride_n, t.stride_l, t.stride_h, static_cast<int32_t>(H / heads)};
}
HeadsOut heads_out(const wg_heads& t) { return {const_cast<void*>(t.data), t.stride_n, t.stride_l, t.stride_h, 0}; }

// How a call is cut: the kernel's form and the segments of a sequence.
struct Cut {
    int kd, waves;            // channels of q and k and waves of a workgroup that the kernel is made for
    int32_t segments, each;   // tiles of a segment
};
// Segments, where the heads do not fill the chip: as many as make kUnits workgroups, of
// kLeast tiles at least.
constexpr int64_t kFull = 192, kUnits = 512, kLeast = 4;
constexpr int columns_of(int waves) { return 16 * waves; }
int64_t blocks_of(int vd, int waves) { return (vd + columns_of(waves) - 1) / columns_of(waves); }
Cut cut_of(int tile, int64_t N, int64_t L, int64_t H, const int (*dims)[2], int passes) {
    int kd = 0, vd = 0;
    for (int p = 0; p < passes; ++p) kd = std::max(kd, dims[p][0]), vd = std::max(vd, dims[p][1]);
    Cut c{kd <= 32 ? 32 : kd <= 64 ? 64 : kd <= 128 ? 128 : 256, vd <= 64 ? 4 : 8, 1, 1};
    int64_t units = 0;
    for (int p = 0; p < passes; ++p) units += N * H * blocks_of(dims[p][1], c.waves);
    const int64_t tiles = (L + tile - 1) / tile;
    int64_t segments = 1;
    if (units < kFull * passes && tiles >= 2 * kLeast) segments = std::min(tiles / kLeast, kUnits / units);
    segments = std::max<int64_t>(1, segments);
    c.each = static_cast<int32_t>(std::max<int64_t>(1, (tiles + segments - 1) / segments));
    c.segments = static_cast<int32_t>(std::max<int64_t>(1, (tiles + c.each - 1) / c.each));
    return c;
}
constexpr int tile_of(int dtype) { return dtype == kBF16 ? kTile<bf16_t> : kTile<float>; }

// HIP takes fewer than 2^32 threads: more sequences than that go in several launches.
hipError_t over_sequences(const Args& a, int passes, int dtype, int threads, void (*kernel)(Args), hipStream_t stream) {
    int64_t per = 0;          // workgroups of a sequence
    for (int p = 0; p < passes; ++p) per += static_cast<int64_t>(a.H) * a.pass[p].blocks;
    const int64_t most = std::max<int64_t>(1, int64_t(0x7fffff) / per);
    for (int64_t n0 = 0; n0 < a.N; n0 += most) {
        Args k = a;
        k.N = std::min(a.N - n0, most);
        if (a.lengths) k.lengths = a.lengths + n0;
        k.first[0] = 0;
        for (int p = 0; p < passes; ++p) {
            Pass& s = k.pass[p];
            const int es = dtype_bytes(dtype);
            for (HeadsIn* t : {&s.q, &s.k, &s.v}) t->p = static_cast<const char*>(t->p) + n0 * t->sn * es;
            s.y.p = static_cast<char*>(s.y.p) + n0 * s.y.sn * (s.y.f32 ? 4 : es);
            const int64_t states = n0 * a.H * s.kd * s.vd;   // with segments all sequences go in one launch
            if (s.s_in) s.s_in += states;
            if (s.s_out) s.s_out += states;
            k.first[p + 1] = k.first[p] + static_cast<int32_t>(k.N * a.H * s.blocks);
        }
        for (int p = passes; p < 3; ++p) k.first[p + 1] = k.first[p];
        kernel<<<static_cast<unsigned>(k.first[3]) * k.segments, threads, 0, stream>>>(k);
    }
    return hipGetLastError();
}

#define WG_ATTENTION_SHAPES(X) X(32, 4) X(32, 8) X(64, 4) X(64, 8) X(128, 4) X(128, 8) X(256, 4) X(256, 8)

template <typename Elem, bool STATES> hipError_t run_passes(Args& a, int passes, const Cut& cut, int dtype, hipStream_t stream) {
    for (int p = 0; p < passes; ++p) a.pass[p].blocks = static_cast<int32_t>(blocks_of(a.pass[p].vd, cut.waves));
    a.segments = cut.segments, a.each = cut.each;
#define WG_ATTENTION_CASE(K, W) \
    if (cut.kd == K && cut.waves == W) return over_sequences(a, passes, dtype, 64 * W, attention_kernel<Elem, K, W, 1, STATES>, stream);
    WG_ATTENTION_SHAPES(WG_ATTENTION_CASE)
#undef WG_ATTENTION_CASE
    return hipErrorInvalidValue;
}

// The states of `of` chains' segments: the pass that adds to each goes first.
template <typename Elem>
hipError_t run_chains(Args a, const Chain* chains, int of, const Cut& cut, int dtype, hipStream_t stream) {
    for (int c = 0; c < of; ++c) a.pass[c].s_out = chains[c].states;
    if (const hipError_t e = run_passes<Elem, true>(a, of, cut, dtype, stream)) return e;
    ChainArgs k{};
    int32_t size = 0;
    for (int c = 0; c < of; ++c) k.chain[c] = chains[c], size = std::max(size, chains[c].size);
    k.heads = a.N * a.H, k.L = a.L, k.H = a.H, k.segments = cut.segments;
    k.tile = tile_of(dtype), k.each_steps = cut.each * k.tile, k.blocks = (size + kThreads - 1) / kThreads, k.of = of;
    k.log_decay = a.log_decay, k.lengths = a.lengths;
    chain_kernel<<<static_cast<unsigned>(k.heads * k.blocks * of), kThreads, 0, stream>>>(k);
    return hipGetLastError();
}

// Bytes of the parts that an input's gradient is summed from: none where no heads share it.
size_t part_bytes(int64_t N, int64_t L, int64_t heads, int64_t H, int64_t D) {
    return heads == H ? 0 : static_cast<size_t>((N * L * H * D * 4 + 15) / 16 * 16);
}

// The passes' channels: of the attention itself, and of its gradients dq, dk and dv.
struct Dims {
    int forward[1][2], backward[3][2];
    Dims(int64_t Dk, int64_t Dv) {
        const int k = static_cast<int>(Dk), v = static_cast<int>(Dv);
        forward[0][0] = backward[2][0] = backward[0][1] = backward[1][1] = k;
        forward[0][1] = backward[2][1] = backward[0][0] = backward[1][0] = v;
    }
};
size_t segment_bytes(const Cut& c, int64_t N, int64_t H, int64_t Dk, int64_t Dv) {
    return c.segments == 1 ? 0 : static_cast<size_t>((N * H * c.segments * Dk * Dv * 4 + 15) / 16 * 16);
}

}  // namespace

#if WG_DTYPE == 0
size_t linear_attention_workspace(int dtype, int64_t N, int64_t L, int64_t q_heads, int64_t k_heads, int64_t v_heads, int64_t H,
                                  int64_t Dk, int64_t Dv, bool backward) {
    const Dims dims(Dk, Dv);
    if (!backward) return segment_bytes(cut_of(tile_of(dtype), N, L, H, dims.forward, 1), N, H, Dk, Dv);
    return 2 * segment_bytes(cut_of(tile_of(dtype), N, L, H, dims.backward, 3), N, H, Dk, Dv) +
           part_bytes(N, L, q_heads, H, Dk) + part_bytes(N, L, k_heads, H, Dk) + part_bytes(N, L, v_heads, H, Dv);
}
#endif

template <int D> hipError_t launch_linear_attention_t(const wg_linear_attention& a, hipStream_t stream) {
    using Elem = typename DTypeOf<D>::type;
    const int32_t Dk = static_cast<int32_t>(a.Dk), Dv = static_cast<int32_t>(a.Dv);
    const Dims dims(Dk, Dv);
    const Cut cut = cut_of(tile_of(D), a.N, a.L, a.heads, dims.forward, 1);
    Args k{};
    k.N = a.N, k.L = static_cast<int32_t>(a.L), k.H = static_cast<int32_t>(a.heads);
    k.log_decay = a.log_decay, k.lengths = a.lengths, k.scale = static_cast<float>(a.scale);
    k.pass[0] = Pass{heads_in(a.q, a.q_heads, a.heads), heads_in(a.k, a.k_heads, a.heads), heads_in(a.v, a.v_heads, a.heads),
                     heads_out(a.y), Dk, Dv, 0, a.s0, a.s_last, {Dv, 1}, 1.0f, k.scale, 0, 0};
    if (cut.segments > 1) {
        const Chain chain{static_cast<float*>(a.workspace), a.s0, a.s_last, Dk * Dv, 0};
        if (const hipError_t e = run_chains<Elem>(k, &chain, 1, cut, D, stream)) return e;
        k.pass[0].s_in = chain.states, k.pass[0].s_out = nullptr, k.pass[0].from_segments = 1;
    }
    return run_passes<Elem, false>(k, 1, cut, D, stream);
}

template <int D> hipError_t launch_linear_attention_backward_t(const wg_linear_attention_backward& a, hipStream_t stream) {
    using Elem = typename DTypeOf<D>::type;
    const int64_t H = a.heads;
    const int32_t Dk = static_cast<int32_t>(a.Dk), Dv = static_cast<int32_t>(a.Dv);
    const Dims dims_of(Dk, Dv);
    const Cut cut = cut_of(tile_of(D), a.N, a.L, H, dims_of.backward, 3);
    Args k{};
    k.N = a.N, k.L = static_cast<int32_t>(a.L), k.H = static_cast<int32_t>(H);
    k.log_decay = a.log_decay, k.lengths = a.lengths, k.scale = static_cast<float>(a.scale);
    const HeadsIn q = heads_in(a.q, a.q_heads, H), kk = heads_in(a.k, a.k_heads, H), v = heads_in(a.v, a.v_heads, H),
                  dy = heads_in(a.dy, H, H);
    char* ws = static_cast<char*>(a.workspace);
    const float *s_in = a.s0, *g_in = a.ds_last;
    if (cut.segments > 1) {
        const size_t bytes = segment_bytes(cut, a.N, H, Dk, Dv);
        const Chain chains[2] = {{reinterpret_cast<float*>(ws), a.s0, nullptr, Dk * Dv, 0},
                                 {reinterpret_cast<float*>(ws + bytes), a.ds_last, a.ds0, Dk * Dv, 1}};
        ws += 2 * bytes;
        k.pass[0] = Pass{q, kk, v, {}, Dk, Dv, 0, nullptr, nullptr, {Dv, 1}, 1.0f, 1.0f, 0, 0};
        k.pass[1] = Pass{kk, q, dy, {}, Dk, Dv, 0, nullptr, nullptr, {Dv, 1}, k.scale, 1.0f, 1, 0};
        if (const hipError_t e = run_chains<Elem>(k, chains, 2, cut, D, stream)) return e;
        s_in = chains[0].states, g_in = chains[1].states;
    }
    HeadsOut out[3] = {heads_out(a.dq), heads_out(a.dk), heads_out(a.dv)};
    const int64_t heads[3] = {a.q_heads, a.k_heads, a.v_heads};
    const int32_t dims[3] = {Dk, Dk, Dv};
    const float* parts[3] = {};
    for (int p = 0; p < 3; ++p) {
        if (heads[p] == H) continue;
        parts[p] = reinterpret_cast<const float*>(ws);
        ws += part_bytes(a.N, a.L, heads[p], H, dims[p]);
    }
    auto to = [&](int p) {
        if (!parts[p]) return out[p];
        return HeadsOut{const_cast<float*>(parts[p]), a.L * H * dims[p], H * dims[p], dims[p], 1};
    };
    const int32_t segmented = cut.segments > 1;
    k.pass[0] = Pass{dy, v, kk, to(0), Dv, Dk, 0, s_in, nullptr, {1, Dv}, 1.0f, k.scale, 0, segmented};
    k.pass[1] = Pass{v, dy, q, to(1), Dv, Dk, 0, g_in, nullptr, {1, Dv}, k.scale, 1.0f, 1, segmented};
    k.pass[2] = Pass{kk, q, dy, to(2), Dk, Dv, 0, g_in, segmented ? nullptr : a.ds0, {Dv, 1}, k.scale, 1.0f, 1, segmented};
    if (const hipError_t e = run_passes<Elem, false>(k, 3, cut, D, stream)) return e;
    for (int p = 0; p < 3; ++p) {
        const int64_t all = a.N * a.L * heads[p] * dims[p];
        if (!parts[p] || all == 0) continue;
        const int64_t blocks = std::min<int64_t>((all + kThreads - 1) / kThreads, 0xffffffffLL / kThreads);
        shared_kernel<Elem><<<static_cast<unsigned>(blocks), kThreads, 0, stream>>>(
            parts[p], out[p], a.N * a.L, k.L, static_cast<int32_t>(heads[p]), static_cast<int32_t>(H / heads[p]), dims[p]);
    }
    return hipGetLastError();
}

template <int D> hipError_t launch_linear_attention_step_t(const wg_linear_attention_step& a, hipStream_t stream) {
    using Elem = typename DTypeOf<D>::type;
    const int32_t blocks = static_cast<int32_t>((a.Dv + kStepColumns - 1) / kStepColumns);
    const StepArgs k{heads_in(a.q, a.q_heads, a.heads), heads_in(a.k, a.k_heads, a.heads), heads_in(a.v, a.v_heads, a.heads),
                     heads_out(a.y), a.N, static_cast<int32_t>(a.heads), static_cast<int32_t>(a.Dk), static_cast<int32_t>(a.Dv),
                     blocks, a.log_decay, a.s, a.s_new, static_cast<float>(a.scale)};
    const int64_t grid = std::min<int64_t>(a.N * a.heads * blocks, 0xffffffffLL / kThreads);
    step_kernel<Elem><<<static_cast<unsigned>(grid), kThreads, 0, stream>>>(k);
    return hipGetLastError();
}

#define WG_ATTENTION_INSTANCES(D)                                                                    \
    template hipError_t launch_linear_attention_t<D>(const wg_linear_attention&, hipStream_t);       \
    template hipError_t launch_linear_attention_backward_t<D>(const wg_linear_attention_backward&, hipStream_t); \
    template hipError_t launch_linear_attention_step_t<D>(const wg_linear_attention_step&, hipStream_t);
WG_ATTENTION_INSTANCES(WG_DTYPE)
#undef WG_ATTENTION_INSTANCES

}  // namespace wg
