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
// three; the state and the weights q.k are held in fp32 and enter in two parts (2^-16 of
// a value is left) or, for fp32 rows, three; the decayed v, of which the state is made, in
// three.  Products of parts below that are left out.  bf16 has fp32's range, so no state
// overflows on the way.
//
// A workgroup takes a head of a sequence and a block of v's columns, whose state stays in
// the registers of four or eight waves, 16 columns each, while the tiles go by; other waves
// bring q, k and v to LDS, make the tiles' weights and store their outputs (attention_kernel).
// Where the heads do not fill the chip a sequence is cut in segments (cut_of): a launch makes
// what each adds to the state, chain_kernel the states ahead of them, and a launch the outputs.
//
// Bound, for bf16 heads of 128 channels, by a tile's latency close to memory: 256 sequences
// and heads of 2048 steps take 138 us, 3.9 TB/s of the 5.1 that a copy reaches; of 64
// channels 85 us (3.2 TB/s); of 128 in fp32, where six products stand for one and every
// value is taken apart, about 400 us (2.7 TB/s at twice the bytes).  A few heads' sequences are
// bound by the start of the three launches, 4 to 8 us each, of which the code's own way to the
// compute units is a part: 16381 steps of 4 heads of 128 channels take 52 us, their bytes 13.
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
constexpr float kLeastLog = -103.972077f;   // -150 log(2), up to which a decay is 0 in fp32

// bf16 parts of an input; of the values computed in fp32 that outputs are made of, whose
// 2^-16 is small beside the outputs' rounding (2^-8 in bf16, 2^-11 in fp16: 2 of 1000 and 10 of
// 1000 outputs are rounded to the neighbour of what fp32 sums give; with three parts a tenth
// of these, at 180 us for 151 for 256 heads of 2048 steps of 128 channels, and 323 us for 187 for
// the gradients of 128 heads of 4096 steps of 64, of which LDS then has no room for two
// workgroups); and of those that the state is made of, which is returned in fp32 (two parts: 3 % less time)
template <typename Elem> constexpr int kParts = std::is_same_v<Elem, bf16_t> ? 1 : std::is_same_v<Elem, _Float16> ? 2 : 3;
template <typename Elem> constexpr int kSums = std::is_same_v<Elem, float> ? 3 : 2;
constexpr int kStateParts = 3;
// Steps of a tile: as many as find room in LDS twice.  With 32 for all bf16 the same call
// takes 150 us for 138, with 64 channels of q and k and 128 of v 161 for 101.
constexpr int tile_steps(bool bf16, int kd) { return bf16 && kd <= 128 ? 64 : 32; }

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

// log2(lambda); from -1e30 on down, infinity included, a number whose every multiple by a
// step count is finite and, but that by 0, a power that is 0 in fp32.
__device__ __forceinline__ float log2_of(float log_decay) {
    return log_decay < -1e30f ? -1e30f : log_decay * kLog2e;
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
                uint32_t w = __builtin_bit_cast(uint32_t, Pair{static_cast<__bf16>(a), static_cast<__bf16>(b)});
                asm("" : "+v"(w));   // else the compiler converts a once more for what follows
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

// c[i] += a[i] b[i] over the parts whose product is not below the last of P.  The
// accumulators take turns: a matrix instruction waits for the one ahead of it on its own.
// A and B: part p of operand i.
template <int PA, int PB, int P, int COUNT, typename A, typename B>
__device__ __forceinline__ void multiply(A&& a, B&& b, f32x4 (&c)[COUNT]) {
#pragma unroll
    for (int p = 0; p < PA; ++p)
#pragma unroll
        for (int r = 0; r < PB; ++r)
            if (p + r < P) {
#pragma unroll
                for (int i = 0; i < COUNT; ++i) c[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a(i, p), b(i, r), c[i], 0, 0, 0);
            }
}

// Rows of a tile in LDS, one plane a part, in runs of 8 channels whose order changes from
// row to row, so that every read below is free of bank conflicts: of 16 bytes a lane, for
// which lanes m + 16 g meet those of m / 4 = 0, 3 with g even and 1, 2 with g odd, and the
// other way around; of 8 bytes, for which 32 lanes meet.  A place is the byte of a lane's
// channel c in a row, from the tile's first plane on or from LDS's start on; that of a
// channel c + d, where d is a multiple of 8 of bits that c has not, is place ^ 2 d, and
// that of 16 rows on place + 32 WIDTH.
template <int PLANES, int ROWS, int WIDTH> struct alignas(512) TileLds {
    static constexpr int kRuns = WIDTH / 8, kPlane = 2 * ROWS * WIDTH;
    uint16_t v[PLANES][ROWS * WIDTH];

    static __device__ __forceinline__ int place(int row, int c) {
        const int high = row >> 3 & 1, by4 = (high ^ (row >> 2 & 1)) << 1 | high;
        const int mix = kRuns >= 16 ? (row & 3) << 2 | by4 : kRuns == 8 ? (row & 2) << 1 | by4 : by4;
        return 2 * (row * WIDTH + (c / 8 ^ mix) * 8 + c % 8);
    }
    __device__ __forceinline__ int start() const {
        return static_cast<int>(reinterpret_cast<uintptr_t>((const __attribute__((address_space(3))) uint16_t*)&v[0][0]));
    }
    template <typename T> __device__ __forceinline__ T& at(int place, int plane) {
        return *reinterpret_cast<T*>(reinterpret_cast<char*>(&v[plane][0]) + place);
    }
    __device__ __forceinline__ float value(int row, int c) const {
        float sum = 0.0f;
#pragma unroll
        for (int p = PLANES - 1; p >= 0; --p) sum += __uint_as_float(static_cast<uint32_t>(v[p][place(row, c) / 2]) << 16);
        return sum;
    }

    // Reads at places from LDS's start on; what is added to a place goes into the
    // instruction.
    template <typename T> static __device__ __forceinline__ T read(int place) {
        return *(const __attribute__((address_space(3))) T*)(static_cast<uint32_t>(place));
    }
    // the values of 4 channels side by side
    static __device__ __forceinline__ void four(int place, float (&x)[4]) {
#pragma unroll
        for (int p = PLANES - 1; p >= 0; --p) {
            const bf16x4 f = read<bf16x4>(place + p * kPlane);
#pragma unroll
            for (int e = 0; e < 4; ++e) x[e] = p == PLANES - 1 ? static_cast<float>(f[e]) : x[e] + static_cast<float>(f[e]);
        }
    }
    // 8 channels, as a matrix instruction takes them of its row (or column): lane m + 16 g
    // holds those from 8 g on of row m
    static __device__ __forceinline__ void across(int place, bf16x8 (&f)[PLANES]) {
#pragma unroll
        for (int p = 0; p < PLANES; ++p) f[p] = read<bf16x8>(place + p * kPlane);
    }
    // 8 rows of a channel: the lanes of 16 hand in the places of four channels in each of
    // four rows, and of the four rows behind them, and lane m gets the rows of channel m
    static __device__ __forceinline__ void down(int place, int behind, bf16x8 (&f)[PLANES]) {
        using At = __attribute__((address_space(3))) s16x4*;
#pragma unroll
        for (int p = 0; p < PLANES; ++p) {
            const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((At)(static_cast<uint32_t>(place + p * kPlane)));
            const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((At)(static_cast<uint32_t>(behind + p * kPlane)));
            f[p] = __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
        }
    }
};
// A place that the compiler takes to be a new one: it makes those that follow from it anew,
// by one operation each, instead of holding them in registers.
__device__ __forceinline__ int renewed(int place) {
    asm volatile("" : "+v"(place));
    return place;
}

// A tile's rows on their way from memory: 16 bytes of U rows a thread.  Every thread
// loads, from the first row and from the end of its row's channels where it has none of
// its own; what it then holds too many is dropped on the way to LDS.
template <typename Elem, int ROWS, int WIDTH, int THREADS> struct TileLoad {
    static constexpr int V = Vec<Elem>::V, kRuns = WIDTH / V, kPer = THREADS / kRuns, U = (ROWS + kPer - 1) / kPer;
    static_assert(THREADS % kRuns == 0 && (ROWS % kPer == 0 || U == 1), "threads cover whole rows");
    u32x4 raw[U];
    const Elem* base;   // the thread's channels of its first row of the sequence
    int64_t stride;
    int run, r0, over;  // its place in a row, its first row; channels too many

    __device__ __forceinline__ TileLoad(int thread, const Elem* p, int64_t row_stride, int c0, int D) {
        run = thread % kRuns * V;
        const int c = c0 + run;
        r0 = thread / kRuns;
        over = max(0, c + V - D);
        stride = row_stride;
        base = p + r0 * stride + (D >= V ? c - over : 0);
    }
    // rows 0 .. live - 1 (at least one) from row t0 of the sequence
    __device__ __forceinline__ void load(int32_t t0, int live, int D) {
        const Elem* p = base + t0 * stride;
        if (D >= V && live == ROWS && ROWS % kPer == 0) {
#pragma unroll
            for (int u = 0; u < U; ++u) raw[u] = reinterpret_cast<const Bytes16*>(p + u * kPer * stride)->v;
            return;
        }
        if (D >= V) {
            const Elem* first = p - r0 * stride;
#pragma unroll
            for (int u = 0; u < U; ++u)
                raw[u] = reinterpret_cast<const Bytes16*>(r0 + u * kPer < live ? p + u * kPer * stride : first)->v;
            return;
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {   // rows shorter than 16 bytes, in pieces of 8, 4 and 2
            raw[u] = u32x4{0, 0, 0, 0};
            if (r0 + u * kPer >= live || over >= V) continue;
            const Elem* at = p + u * kPer * stride;
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
    // SWAP: rows from 8 on of every 16 with the halves of their runs of 8 channels exchanged
    template <bool SWAP, int PLANES> __device__ __forceinline__ void store(TileLds<PLANES, ROWS, WIDTH>& to) const {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int row = r0 + u * kPer;
            if (ROWS % kPer != 0 && row >= ROWS) continue;
            const bool swap = SWAP && row & 8;
            if constexpr (PLANES == 1) {
                const u32x4 w = swap ? u32x4{raw[u][2], raw[u][3], raw[u][0], raw[u][1]} : raw[u];
                to.template at<u32x4>(to.place(row, run), 0) = w;
            } else {
                float x[V];
                Vec<Elem>::widen(raw[u], x);
                Split<PLANES, V, true> s;
                s.of(x);
#pragma unroll
                for (int p = 0; p < PLANES; ++p) {
                    if constexpr (V == 8) {
                        const u32x4 w = __builtin_bit_cast(u32x4, s.part[p]);
                        to.template at<u32x4>(to.place(row, run), p) = swap ? u32x4{w[2], w[3], w[0], w[1]} : w;
                    } else {
                        to.template at<bf16x4>(to.place(row, run) ^ (swap ? 8 : 0), p) = s.part[p];
                    }
                }
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

struct None {};

// What a workgroup holds in LDS, for tiles of K channels of q and k and W waves of 16
// columns each.
template <typename Elem, int K, int W, bool STATES> struct Shape {
    static constexpr int T = tile_steps(std::is_same_v<Elem, bf16_t>, K), PI = kParts<Elem>, PS = kSums<Elem>;
    static constexpr int kColumns = 16 * W, kPanels = T == 64 ? 3 : 1;
    struct Steps {
        std::conditional_t<STATES, None, TileLds<PI, T, K>> q;
        TileLds<PI, T, K> k;
        TileLds<PI, T, kColumns> v;
    };
    struct Own {
        // the weights in panels of 32 x 32: rows and columns 32 a .. and 32 b .. are panel a + b
        TileLds<PS, 32 * kPanels, 32> weights;
        // a tile's outputs: two tiles in the storage type, or one in fp32
        u32x4 outputs[T * kColumns / 4 * (sizeof(Elem) == 4 ? 2 : 1)];
        int32_t odd[2];                   // the tile (+ 1) of which q, k or v holds an infinity or NaN
        float whole[2];                   // the decay over a tile, and over the sequence's last one
    };
    struct Least {
        alignas(16) float in_decay[T];    // from a tile's steps to the state behind it
        std::conditional_t<STATES, None, Own> own;
    };
    // two tiles of steps, where they find room
    static constexpr int kStages = 2 * sizeof(Steps) + sizeof(Least) <= kLdsBytes ? 2 : 1;
    struct Lds : Least {
        Steps steps[kStages];
    };
    // Whether the weights' waves load and unpack q: where unpacking is what a tile waits for, with
    // inputs in several parts.  Gradients of 32 x 1024 steps of 8 heads of 64 channels in fp16 152
    // to 137 us, of 16 x 1024 of 128 in fp32 315 to 298; but of 32 x 2048 of 128 in bf16, whose
    // loads would crowd them, 411 to 432.
    static constexpr bool kOwnQ = PI > 1;
    // W waves for the state, half as many for memory and, but for STATES, as many for the
    // weights.  Twice as many of these where inputs have several parts, if a compute unit
    // holds one such workgroup: 16 x 1024 steps of 8 heads of 128 channels in fp32 152 to
    // 109 us.  In fp16 with up to 64 channels of q and k two workgroups of 8 waves do more
    // than one of 12: 64 x 1024 steps of 8 heads of 64 channels 96 and 175 us.
    static constexpr int kHelpers = W == 4 && PI > 1 && !(PI == 2 && K <= 64) ? W : W / 2;
    static constexpr int kMemory = 64 * kHelpers, kWeights = STATES ? 0 : 64 * kHelpers, kThreads = 64 * W + kMemory + kWeights;
    static constexpr int kWavesPerSimd = W == 8 ? 4 : kHelpers == W ? (STATES ? 2 : 3) : K <= 64 ? (2 * sizeof(Lds) <= kLdsBytes ? 4 : 2) : STATES && K == 128 ? 3 : 2;
};
// Where run `run` of 16 bytes of a row of outputs stands, of RUNS a row: the order changes
// from row to row.
template <int RUNS> __device__ __forceinline__ int output_at(int row, int run) { return row * RUNS + (run ^ (row & (RUNS < 16 ? RUNS - 1 : 15))); }

// A pass, or (STATES) only what its segments add to the state.  The waves of a workgroup
// have three tasks, so that some work where others wait:
//   * W hold the state, 16 columns each: they multiply it by q, add what the tile's own
//     steps give (weights times v), and bring the state over the tile; where q, k, v or the
//     state holds an infinity or NaN they go step by step instead;
//   * kHelpers (W / 2, or W) load the tile after the next and unpack the next one;
//   * as many store the last tile's outputs and make the weights (q.k, decayed) of the next; of
//     inputs in several parts they load and unpack q, too.
// Two barriers a tile: ahead of the first, tile t's outputs are made, those of tile t - 1
// leave and tile t + 1 is unpacked; ahead of the second, the state is brought over tile t
// and the weights of tile t + 1 are made.  Loads go out on both sides of the first, since
// they hold up their waves as long as the path to memory is taken.  With one stage in LDS
// the next tile's unpacking and its weights follow in turn.
//
// S[b], lane m + 16 g, register r is the state at (32 (b / 2) + 8 g + 4 (b % 2) + r,
// 16 wave + m), so that those of two blocks side by side are the 8 consecutive rows that a
// lane hands a matrix instruction, without a move.  The transposing reads of k then take 8
// bytes of every run of 16; k's rows from 8 on of every 16 stand with the halves of their
// runs in exchanged order (SWAP), so that both halves' banks are in use.  Outputs come
// transposed, O[i] with row 16 i + m and columns 16 wave + 4 g + r.
template <typename Elem, int KD, int W, bool STATES>
__global__ __launch_bounds__((Shape<Elem, KD, W, STATES>::kThreads), (Shape<Elem, KD, W, STATES>::kWavesPerSimd))
void attention_kernel(Args) {
    // the arguments where the launch left them: the compiler keeps a large copy in scratch memory
    const Args& a = *(const Args*)__builtin_amdgcn_kernarg_segment_ptr();
    using Sh = Shape<Elem, KD, W, STATES>;
    constexpr int T = Sh::T, PI = Sh::PI, PS = Sh::PS, VB = Sh::kColumns, IB = T / 16, JS = T / 32, KS = KD / 32;
    constexpr int STAGES = Sh::kStages, BLOCKS = IB * (IB + 1) / 2;
    __shared__ typename Sh::Lds lds;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x % 64, m = lane % 16, g = lane / 16;

    const int32_t segment = blockIdx.x / static_cast<uint32_t>(a.first[3]);
    const int32_t id = blockIdx.x - segment * a.first[3];
    const int which = id >= a.first[2] ? 2 : id >= a.first[1] ? 1 : 0;
    const Pass& pass = a.pass[which];
    const uint32_t unit = id - a.first[which];
    const uint32_t head = unit / static_cast<uint32_t>(pass.blocks);
    const int32_t block = unit - head * pass.blocks, h = head % static_cast<uint32_t>(a.H);
    const int64_t n = head / static_cast<uint32_t>(a.H);
    const int32_t steps = steps_of(a.lengths, n, a.L), kd = pass.kd, vd = pass.vd, v0 = block * VB;
    const bool reverse = pass.reverse != 0, y_f32 = sizeof(Elem) == 2 && pass.y.f32 != 0;
    const float log_decay = a.log_decay[h], log2_decay = log2_of(log_decay);

    // a segment's tiles, in the order of the walk
    const int32_t tiles = (steps + T - 1) / T, t_first = segment * a.each, t_end = min(tiles, t_first + a.each);
    auto row_of = [&](int32_t t) { return (reverse ? tiles - 1 - t : t) * T; };
    auto rows_of = [&](int32_t t) { return min(T, steps - row_of(t)); };
    auto stage_of = [&](int32_t t) -> auto& { return lds.steps[t & (STAGES - 1)]; };
    const bool any = t_first < t_end;

    if (wave < W) {   // the state
        f32x4 S[KD / 16];
        const int64_t size = static_cast<int64_t>(kd) * vd, by_segment = (static_cast<int64_t>(head) * a.segments + segment) * size;
        const int column = v0 + 16 * wave + m, at_column = min(column, vd - 1) * pass.at.col;
        auto row_of_state = [&](int b, int r) { return 32 * (b / 2) + 8 * g + 4 * (b % 2) + r; };
        if (!STATES && pass.s_in) {
            // every lane loads, from the last row and column where it has none: all in flight
            const float* s = pass.s_in + (pass.from_segments ? by_segment : head * size) + at_column;
#pragma unroll
            for (int b = 0; b < KD / 16; ++b)
#pragma unroll
                for (int r = 0; r < 4; ++r) S[b][r] = s[min(row_of_state(b, r), kd - 1) * pass.at.row];
#pragma unroll
            for (int b = 0; b < KD / 16; ++b)
#pragma unroll
                for (int r = 0; r < 4; ++r) S[b][r] = row_of_state(b, r) < kd && column < vd ? S[b][r] : 0.0f;
        } else {
#pragma unroll
            for (int b = 0; b < KD / 16; ++b) S[b] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        }
        auto store_state = [&](float* s) {
#pragma unroll
            for (int b = 0; b < KD / 16; ++b)
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    if (row_of_state(b, r) < kd && column < vd) s[row_of_state(b, r) * pass.at.row + at_column] = S[b][r];
        };
        using K = decltype(lds.steps[0].k);
        using V = decltype(lds.steps[0].v);
        // places of q, and of k and v for four rows and the four behind them
        const int q_own = K::place(m, 8 * g);
        int k_own[2], v_own[2];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            k_own[u] = K::place(8 * g + m / 4 + 4 * u, 8 * (m % 4)) ^ 8 * (g % 2);
            v_own[u] = V::place(8 * g + m / 4 + 4 * u, 16 * wave + 4 * (m % 4));
        }
        float whole = 1.0f, out_decay[IB];   // the decays over a tile, and from the state to its steps
        int decays_of = 0;
        auto has_infinity = [&] {            // of the wave's columns of the state
            bool found = false;
#pragma unroll
            for (int b = 0; b < KD / 16; ++b)
#pragma unroll
                for (int r = 0; r < 4; ++r) found = found || __builtin_isinf(S[b][r]);
            return __any(found) != 0;
        };
        bool infinite = !STATES && pass.s_in && has_infinity();
        // A tile by the recurrence itself, which needs of the state only the lane's own values: where
        // an infinity or NaN takes part, products with weights of zero or with lower parts would make
        // NaN of what the recurrence keeps finite or infinite.  64 steps of 128 channels take 100 us so.
        auto step_by_step = [&](const auto& now, auto& own, int32_t t, int live) {
            // all from numbers that are taken to be new ones, or registers hold it over all tiles
            const int place = renewed(lane), g = place / 16, c = 16 * wave + place % 16, rows = kd - 8 * g;
            float log_keep = log_decay;
            asm volatile("" : "+v"(log_keep));
            const float keep = expf(log_keep);
#pragma unroll 1
            for (int i = 0; i < live; ++i) {
                const int j = reverse ? live - 1 - i : i, at = K::place(j, 8 * g), swap = j >> 3 & 1;
                const float x = pass.in_scale * now.v.value(j, c);
                float sum = 0.0f;
#pragma unroll
                for (int b = 0; b < KD / 16; ++b) {
                    float fk[4], fq[4];
                    K::four(((now.k.start() + at) ^ 64 * (b / 2)) + 8 * (b % 2 ^ swap), fk);
                    K::four(((now.q.start() + at) ^ 64 * (b / 2)) + 8 * (b % 2), fq);
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        if (32 * (b / 2) + 4 * (b % 2) + r >= rows) continue;
                        const float s = reverse ? fmaf(fk[r], x, S[b][r]) : fmaf(keep, S[b][r], fk[r] * x);
                        sum = fmaf(fq[r], s, sum);
                        S[b][r] = reverse ? keep * s : s;
                    }
                    __builtin_amdgcn_sched_barrier(0);
                }
                sum += __shfl_xor(sum, 16);
                sum += __shfl_xor(sum, 32);
                const float y = pass.out_scale * sum;
                if (g != 0) continue;
                if (y_f32) {
                    reinterpret_cast<float*>(&own.outputs[output_at<VB / 4>(j, c / 4)])[c % 4] = y;
                } else {
                    constexpr int kPer = 16 / sizeof(Elem), RUNS = VB / kPer;
                    auto* run = &own.outputs[(t & 1) * T * RUNS + output_at<RUNS>(j, c / kPer)];
                    reinterpret_cast<Elem*>(run)[c % kPer] = Storage<Elem>::from_f32(y);
                }
            }
            infinite = has_infinity();
        };
        // The same for a segment's sums, in which an infinity or NaN stays: from memory, behind all
        // tiles, which costs those of other segments nothing (256 steps of 128 channels: 340 us).
        auto segment_step_by_step = [&] {
            const Elem* k = heads_at<Elem>(pass.k, n, h);
            const Elem* v = heads_at<Elem>(pass.v, n, h) + min(column, vd - 1);
            const float keep = expf(log_decay);
            const int32_t low = reverse ? t_end - 1 : t_first, high = reverse ? t_first : t_end - 1;
            const int32_t first = row_of(low), end = row_of(high) + rows_of(high);
#pragma unroll
            for (int b = 0; b < KD / 16; ++b) S[b] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 1
            for (int32_t i = 0; i < end - first; ++i) {
                const int64_t row = reverse ? end - 1 - i : first + i;
                const float x = pass.in_scale * Storage<Elem>::to_f32(v[row * pass.v.sl]);
                const int l = renewed(kd - 1);
#pragma unroll
                for (int b = 0; b < KD / 16; ++b) {
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const float kk = Storage<Elem>::to_f32(k[row * pass.k.sl + min(row_of_state(b, r), l)]);
                        S[b][r] = reverse ? keep * fmaf(kk, x, S[b][r]) : fmaf(keep, S[b][r], kk * x);
                    }
                    if (b % 4 == 3) __builtin_amdgcn_sched_barrier(0);
                }
            }
        };
        if (any) {                           // the first tile and its weights
#pragma unroll
            for (int i = 0; i < 2 * (STATES ? 0 : 1) + (STAGES == 2 ? 1 : STATES ? 2 : 3); ++i) __syncthreads();
        }
        for (int32_t t = t_first; t < t_end; ++t) {
            const auto& now = stage_of(t);
            const int live = rows_of(t);
            const int v_place[2] = {now.v.start() + v_own[0], now.v.start() + v_own[1]};
            int flag = 0;
            if constexpr (!STATES) flag = lds.own.odd[t & 1], whole = lds.own.whole[live < T];
            bool odd = false;
            if (live != decays_of) {
                decays_of = live;
                if constexpr (STATES) whole = exact_power(log_decay, live);
                const int j = threadIdx.x;
                if (j < T) lds.in_decay[j] = pass.in_scale * power(log2_decay, reverse ? j + 1 : max(0, live - 1 - j));
                if constexpr (STATES) __syncthreads();
#pragma unroll
                for (int i = 0; i < IB; ++i)
                    out_decay[i] = pass.out_scale * power(log2_decay, reverse ? max(0, live - 1 - (16 * i + m)) : 16 * i + m + 1);
            }
            if constexpr (!STATES) {
                const int q_place = now.q.start() + q_own;
                f32x4 O[IB];
#pragma unroll
                for (int i = 0; i < IB; ++i) O[i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                for (int s = 0; s < KS; ++s) {
                    Split<PS, 8, false> fs;
                    float x[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) x[e] = S[2 * s + e / 4][e % 4];
                    fs.of(x);
                    bf16x8 fq[IB][PI];
                    const int place = renewed(q_place) ^ 64 * s;
#pragma unroll
                    for (int i = 0; i < IB; ++i) now.q.across(place + 32 * i * KD, fq[i]);
                    multiply<PS, PI, PS>([&](int, int p) { return fs.part[p]; }, [&](int i, int p) { return fq[i][p]; }, O);
                }
                odd = infinite || __builtin_amdgcn_readfirstlane(flag) == t + 1;   // (behind the products: it waits for the flag)
                if (!odd) {
#pragma unroll
                    for (int i = 0; i < IB; ++i) O[i] *= out_decay[i];
                    using P = decltype(lds.own.weights);
                    const int p_place = lds.own.weights.start() + P::place(m, 8 * g);
#pragma unroll
                    for (int s = 0; s < JS; ++s) {
                        bf16x8 fv[PI];
                        now.v.down(v_place[0] + 64 * s * VB, v_place[1] + 64 * s * VB, fv);
#pragma unroll
                        for (int i = 0; i < IB; i += 2) {
                            if (reverse ? s < i / 2 : s > i / 2) continue;
                            bf16x8 fp[2][PS];
                            P::across(p_place + 64 * (i / 2 + s) * 32, fp[0]);
                            P::across(p_place + 64 * (i / 2 + s) * 32 + 32 * 32, fp[1]);
                            f32x4 pair[2] = {O[i], O[i + 1]};
                            multiply<PI, PS, PS>([&](int, int p) { return fv[p]; }, [&](int u, int p) { return fp[u][p]; }, pair);
                            O[i] = pair[0], O[i + 1] = pair[1];
                        }
                    }
                    const int c = 4 * wave + g;
                    if (y_f32) {
#pragma unroll
                        for (int i = 0; i < IB; ++i)
                            lds.own.outputs[output_at<VB / 4>(16 * i + m, c)] = __builtin_bit_cast(u32x4, O[i]);
                    } else {
                        struct alignas(4 * sizeof(Elem)) Four {
                            Elem v[4];
                        };
                        constexpr int kPer = 16 / sizeof(Four), RUNS = VB * sizeof(Elem) / 16;
#pragma unroll
                        for (int i = 0; i < IB; ++i) {
                            Four four;
                            if constexpr (std::is_same_v<Elem, bf16_t>) {   // in pairs
                                const bf16x4 e = {static_cast<__bf16>(O[i][0]), static_cast<__bf16>(O[i][1]), static_cast<__bf16>(O[i][2]),
                                                  static_cast<__bf16>(O[i][3])};
                                four = __builtin_bit_cast(Four, e);
                            } else {
#pragma unroll
                                for (int r = 0; r < 4; ++r) four.v[r] = Storage<Elem>::from_f32(O[i][r]);
                            }
                            auto* run = &lds.own.outputs[(t & 1) * T * RUNS + output_at<RUNS>(16 * i + m, c / kPer)];
                            reinterpret_cast<Four*>(run)[c % kPer] = four;
                        }
                    }
                }
            }
            if constexpr (!STATES) {
                if (odd) step_by_step(now, lds.own, t, live);
                __syncthreads();
            }
            if (!odd) {
#pragma unroll
                for (int b = 0; b < KD / 16; ++b) S[b] *= whole;
                Split<kStateParts, 8, false> late[JS];
#pragma unroll
                for (int s = 0; s < JS; ++s) {
                    bf16x8 fv[PI];
                    now.v.down(v_place[0] + 64 * s * VB, v_place[1] + 64 * s * VB, fv);
                    float x[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        float sum = static_cast<float>(fv[PI - 1][e]);
#pragma unroll
                        for (int p = PI - 2; p >= 0; --p) sum += static_cast<float>(fv[p][e]);
                        x[e] = sum * lds.in_decay[32 * s + 8 * g + e];
                    }
                    late[s].of(x);
                }
                const int k_place[2] = {now.k.start() + k_own[0], now.k.start() + k_own[1]};
#pragma unroll
                for (int b = 0; b < KD / 16; b += 2) {
                    f32x4 pair[2] = {S[b], S[b + 1]};
                    int own[2][2];
#pragma unroll
                    for (int u = 0; u < 2; ++u) own[u][0] = renewed(k_place[0]) ^ (32 * b + 8 * u), own[u][1] = renewed(k_place[1]) ^ (32 * b + 8 * u);
#pragma unroll
                    for (int s = 0; s < JS; ++s) {
                        bf16x8 fk[2][PI];
#pragma unroll
                        for (int u = 0; u < 2; ++u) now.k.down(own[u][0] + 64 * s * KD, own[u][1] + 64 * s * KD, fk[u]);
                        multiply<PI, kStateParts, kStateParts>([&](int i, int p) { return fk[i][p]; },
                                                               [&](int, int p) { return late[s].part[p]; }, pair);
                    }
                    S[b] = pair[0], S[b + 1] = pair[1];
                }
            }
            __syncthreads();
            if constexpr (STAGES == 1) {
                __syncthreads();
                if constexpr (!STATES) __syncthreads();
            }
        }
        if constexpr (STATES) {
            bool finite = true;
#pragma unroll
            for (int b = 0; b < KD / 16; ++b)
#pragma unroll
                for (int r = 0; r < 4; ++r) finite = finite && __builtin_isfinite(S[b][r]);
            if (!__all(finite)) segment_step_by_step();
            store_state(pass.s_out + by_segment);
        } else if (pass.s_out && segment == a.segments - 1) {
            store_state(pass.s_out + head * size);
        }
        return;
    }

    // a tile's outputs, whole lines of them, by NT threads
    auto put = [&](const auto& own, auto* y, int32_t t, int tid, auto threads) {
        using Out = std::remove_pointer_t<decltype(y)>;
        constexpr int V = Vec<Out>::V, RUNS = VB / V, PER = threads() / RUNS;
        const int run = tid % RUNS, valid = min(V, vd - v0 - run * V), rows = rows_of(t);
        const auto* from = own.outputs + (std::is_same_v<Out, Elem> ? (t & 1) * T * RUNS : 0);
        if (valid <= 0) return;
        y += n * pass.y.sn + h * pass.y.sh + row_of(t) * pass.y.sl + v0 + run * V;
#pragma unroll
        for (int u = 0; u < T / PER; ++u) {
            const int row = tid / RUNS + u * PER;
            if (row < rows) store_run<Out, false>(y + row * pass.y.sl, valid, from[output_at<RUNS>(row, run)]);
        }
    };

    if (STATES || wave < W + Sh::kHelpers) {   // memory
        const int tid = threadIdx.x - 64 * W;
        TileLoad<Elem, T, KD, Sh::kMemory> lq(tid, heads_at<Elem>(pass.q, n, h), pass.q.sl, 0, kd);
        TileLoad<Elem, T, KD, Sh::kMemory> lk(tid, heads_at<Elem>(pass.k, n, h), pass.k.sl, 0, kd);
        TileLoad<Elem, T, VB, Sh::kMemory> lv(tid, heads_at<Elem>(pass.v, n, h), pass.v.sl, v0, vd);
        auto load_k = [&](int32_t t) {
            if (t < t_end) lk.load(row_of(t), rows_of(t), kd);
        };
        auto load_others = [&](int32_t t) {
            if (t >= t_end) return;
            if constexpr (!STATES && !Sh::kOwnQ) lq.load(row_of(t), rows_of(t), kd);
            lv.load(row_of(t), rows_of(t), vd);
        };
        auto unpack = [&](int32_t t) {
            if (t >= t_end) return;
            const int rows = rows_of(t);
            const bool whole = kd == KD && vd - v0 >= VB && rows == T;
            auto& to = stage_of(t);
            lk.trim(whole, rows, kd);
            lk.template store<true, PI>(to.k);
            if constexpr (!STATES && !Sh::kOwnQ) {
                lq.trim(whole, rows, kd);
                lq.template store<false, PI>(to.q);
            }
            lv.trim(whole, rows, vd);
            lv.template store<false, PI>(to.v);
            if constexpr (!STATES)
                if (!lv.finite()) lds.own.odd[t & 1] = t + 1;
        };
        if (STAGES == 2 && any) {
            load_k(t_first);
            load_others(t_first);
        }
        if (!STATES && any) __syncthreads();   // the weights' waves have cleared odd
        int decays_of = 0;
        for (int32_t t = t_first - 1; t < t_end; ++t) {
            if (STATES && t >= t_first && rows_of(t) != decays_of) {   // they are set by the waves of the state
                decays_of = rows_of(t);
                __syncthreads();
            }
            if constexpr (STAGES == 2) unpack(t + 1);
            load_k(t + STAGES);
            if constexpr (!STATES)
                if (any) __syncthreads();
            load_others(t + STAGES);
            if constexpr (!STATES)
                if (y_f32 && t >= t_first) put(lds.own, static_cast<float*>(pass.y.p), t, tid, [] { return Sh::kMemory; });
            if (any) __syncthreads();
            if constexpr (STAGES == 1) {
                unpack(t + 1);
                if (any) __syncthreads();
                if constexpr (!STATES)
                    if (any) __syncthreads();
            }
        }
        if constexpr (STATES) return;
        // padding, of which each segment takes a share of rows
        const int32_t share = (a.L - steps + a.segments - 1) / a.segments;
        const int64_t row0 = min(steps + static_cast<int64_t>(segment) * share, static_cast<int64_t>(a.L));
        const int64_t row1 = min(row0 + share, static_cast<int64_t>(a.L));
        // (of parts in fp32 nothing is read there)
        constexpr int V = Vec<Elem>::V, RUNS = VB / V;
        const int run = tid % RUNS, valid = y_f32 ? 0 : min(V, vd - v0 - run * V);
        if (valid <= 0) return;
        Elem* y = static_cast<Elem*>(pass.y.p) + n * pass.y.sn + h * pass.y.sh + v0 + run * V;
        for (int64_t row = row0 + tid / RUNS; row < row1; row += Sh::kMemory / RUNS)
            store_run<Elem, false>(y + row * pass.y.sl, valid, u32x4{0, 0, 0, 0});
        return;
    }

    if constexpr (!STATES) {   // outputs and weights
        if (!any) return;
        const int tid = threadIdx.x - 64 * W - Sh::kMemory, own_wave = wave - W - Sh::kHelpers;
        const int own_place = decltype(lds.steps[0].k)::place(m, 8 * g);
        // the decays between steps of one block, of neighbouring blocks, and by 16 and 32 steps more
        const int d0 = reverse ? 4 * g - m : m - 4 * g;
        float here[4], next[4];
        const float far_by[2] = {power(log2_decay, 16), power(log2_decay, 32)};
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int d = d0 + (reverse ? r : -r);
            here[r] = a.scale * power(log2_decay, max(0, d));
            next[r] = a.scale * power(log2_decay, 16 + d);
        }
        auto weigh = [&](int32_t t) {
            if (t >= t_end) return;
            const auto& now = stage_of(t);
            const int k_place = now.k.start() + own_place, q_place = now.q.start() + own_place;
            float size = 0.0f;   // on the diagonal, where every step's q and k take part
            // in blocks of 16 x 16 of the triangle, two at a time
#pragma unroll
            for (int first = 0; first < BLOCKS; first += 2 * Sh::kHelpers) {
                constexpr int kHalf = Sh::kHelpers;
                const bool two = first + kHalf < BLOCKS;
                int ib[2], jb[2];
                bool has[2];
                f32x4 w[2];
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    const int own = first + own_wave + u * kHalf;
                    has[u] = own < BLOCKS;
                    const int blk = has[u] ? own : 0;
                    const int far = blk >= 6 ? 3 : blk >= 3 ? 2 : blk >= 1 ? 1 : 0, near = blk - far * (far + 1) / 2;
                    ib[u] = reverse ? near : far, jb[u] = reverse ? far : near;
                    w[u] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
                }
                if (!has[0]) break;
#pragma unroll
                for (int s = 0; s < KS; ++s) {
                    bf16x8 fk[2][PI], fq[2][PI];
#pragma unroll
                    for (int u = 0; u < 2; ++u) {
                        if (u == 1 && !two) continue;
                        now.k.across((k_place + 32 * jb[u] * KD) ^ 64 * s, fk[u]);
#pragma unroll
                        for (int p = 0; p < PI; ++p)   // rows whose halves are exchanged
                            if (m & 8) fk[u][p] = __builtin_shufflevector(fk[u][p], fk[u][p], 4, 5, 6, 7, 0, 1, 2, 3);
                        now.q.across((q_place + 32 * ib[u] * KD) ^ 64 * s, fq[u]);
                    }
                    if (two) {
                        multiply<PI, PI, PS>([&](int u, int p) { return fk[u][p]; }, [&](int u, int p) { return fq[u][p]; }, w);
                    } else {
                        f32x4 one[1] = {w[0]};
                        multiply<PI, PI, PS>([&](int, int p) { return fk[0][p]; }, [&](int, int p) { return fq[0][p]; }, one);
                        w[0] = one[0];
                    }
                }
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    if (!has[u] || (u == 1 && !two)) continue;
                    float x[4];
                    const int apart = reverse ? jb[u] - ib[u] : ib[u] - jb[u];
                    if (apart == 0) {
#pragma unroll
                        for (int r = 0; r < 4; ++r) {
                            x[r] = d0 + (reverse ? r : -r) < 0 ? 0.0f : w[u][r] * here[r];
                            size += fabsf(w[u][r]);
                        }
                    } else {
                        const float more = apart == 1 ? 1.0f : apart == 2 ? far_by[0] : far_by[1];
#pragma unroll
                        for (int r = 0; r < 4; ++r) x[r] = w[u][r] * (next[r] * more);
                    }
                    Split<PS, 4, false> parts;
                    parts.of(x);
                    auto& to = lds.own.weights;
                    const int row = 32 * (ib[u] / 2 + jb[u] / 2) + 16 * (ib[u] % 2) + m, c = 16 * (jb[u] % 2) + 4 * g;
#pragma unroll
                    for (int p = 0; p < PS; ++p) to.template at<bf16x4>(to.place(row, c), p) = parts.part[p];
                }
            }
            if (!__builtin_isfinite(size)) lds.own.odd[t & 1] = t + 1;
        };
        TileLoad<Elem, T, KD, Sh::kWeights> lq(tid, heads_at<Elem>(pass.q, n, h), pass.q.sl, 0, kd);
        auto load_q = [&](int32_t t) {
            if constexpr (Sh::kOwnQ)
                if (t < t_end) lq.load(row_of(t), rows_of(t), kd);
        };
        auto unpack_q = [&](int32_t t) {
            if constexpr (Sh::kOwnQ) {
                if (t >= t_end) return;
                const int rows = rows_of(t);
                lq.trim(kd == KD && rows == T, rows, kd);
                lq.template store<false, PI>(stage_of(t).q);
            }
        };
        if constexpr (STAGES == 2) load_q(t_first);
        // weights above the diagonal are zeros that nothing writes
        for (int i = tid; i < static_cast<int>(sizeof(lds.own.weights) / 4); i += Sh::kWeights)
            reinterpret_cast<uint32_t*>(&lds.own.weights)[i] = 0;
        if (tid < 2) lds.own.odd[tid] = 0;
        // (here, since its constants would take registers of the waves that hold the state)
        if (tid < 2) lds.own.whole[tid] = exact_power(log_decay, tid == 0 ? T : steps - (tiles - 1) * T);
        __syncthreads();
        for (int32_t t = t_first - 1; t < t_end; ++t) {
            if (!y_f32 && t > t_first) put(lds.own, static_cast<Elem*>(pass.y.p), t - 1, tid, [] { return Sh::kWeights; });
            if constexpr (STAGES == 2) unpack_q(t + 1);
            load_q(t + STAGES);
            __syncthreads();
            if constexpr (STAGES == 2) weigh(t + 1);
            __syncthreads();
            if constexpr (STAGES == 1) {
                unpack_q(t + 1);
                __syncthreads();
                weigh(t + 1);
                __syncthreads();
            }
        }
        if (!y_f32) put(lds.own, static_cast<Elem*>(pass.y.p), t_end - 1, tid, [] { return Sh::kWeights; });
    }
}

// The states ahead of the segments from what each but the last adds: in place,
// [N][H][segments] of `size` values, from s_in [N][H] (or null: zeros).
struct Chain {
    float* states;
    const float* s_in;
    int32_t size, reverse;
};
struct ChainArgs {
    Chain chain[2];
    int64_t heads;            // N H
    int32_t L, H, segments, each_steps, tile, blocks, of;
    const float* log_decay;
    const int32_t* lengths;
};
// A thread holds one value of a state and walks over the segments, with the loads of U in
// flight together (with 64 no faster, for all the code).  Bound by latency: 4 us for six
// segments of 39 states of 40 x 75, of which a launch takes 2.5, 9 us for 64 of 4 states of
// 128 x 128 channels.
__global__ __launch_bounds__(kThreads) void chain_kernel(ChainArgs a) {
    constexpr int U = 16;
    const Chain& c = a.chain[blockIdx.x % a.of];
    const uint32_t unit = blockIdx.x / a.of, head = unit / static_cast<uint32_t>(a.blocks);
    const int32_t i = static_cast<int32_t>(unit - head * a.blocks) * kThreads + threadIdx.x;
    const uint32_t n = head / static_cast<uint32_t>(a.H);
    const int32_t steps = steps_of(a.lengths, n, a.L), last = (steps + a.tile - 1) / a.tile * a.tile - steps;
    const float log_decay = a.log_decay[head - n * a.H];
    if (i >= c.size) return;
    const int64_t size = c.size;
    float* s = c.states + head * (a.segments * size) + i;
    float run = c.s_in ? c.s_in[head * size + i] : 0.0f;
    // Segments have each_steps, but the reverse of a walk begins with a tile that may be short,
    // the last one ends with the steps, and those behind it are empty.  Their decays are made
    // ahead of the walk: a power in every turn made 25 KB of code of it, and 13 us of those 9.
    const int64_t each = a.each_steps, end = steps + (c.reverse ? last : 0);
    const int32_t cut = static_cast<int32_t>(end / each), rest = static_cast<int32_t>(end - cut * each);
    const float whole = exact_power(log_decay, a.each_steps), at_cut = exact_power(log_decay, rest);
    const float at_first = exact_power(log_decay, max(0, static_cast<int32_t>(min(each, end)) - (c.reverse ? last : 0)));
    const int32_t adding = a.segments - 1, filled = cut + (rest > 0);
    const bool lasts = log_decay > kLeastLog;   // an infinity stays one, though its decay over a segment be 0
    for (int32_t w = 0; w < a.segments; w += U) {
        float add[U];
#pragma unroll
        for (int u = 0; u < U; ++u) add[u] = w + u < adding ? s[(w + u) * size] : 0.0f;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (w + u >= a.segments) break;
            s[(w + u) * size] = run;
            if (w + u >= min(adding, filled)) continue;
            const float decay = lasts && __builtin_isinf(run) ? 1.0f : w + u == 0 ? at_first : w + u == cut ? at_cut : whole;
            run = fmaf(decay, run, add[u]);
        }
    }
}

// Gradients of inputs that heads share: the sums over them of their parts [N][L][H][D4]
// in fp32 (D4 is D up to a multiple of 4), in the order of the heads, so that results repeat
// (atomics would not); those of padding are not there.  A thread takes four channels.  14 us for 8000 steps of 8 heads on 2
// of 128 channels: 65 MB of parts read at 4.7 TB/s.
struct Shared {
    const float* part;
    HeadsOut to;
    int32_t heads, per, D;
    int64_t first;            // of its work items among all
};
struct SharedArgs {
    Shared of[3];
    int32_t count, L;
    int64_t items;
    const int32_t* lengths;
};
template <typename Elem>
__global__ __launch_bounds__(kThreads) void shared_kernel(SharedArgs a) {
    const int64_t stride = static_cast<int64_t>(gridDim.x) * kThreads;
    for (int64_t id = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x; id < a.items; id += stride) {
        int which = 0;
        while (which + 1 < a.count && id >= a.of[which + 1].first) ++which;
        const Shared& s = a.of[which];
        const int32_t runs = (s.D + 3) / 4;
        const int64_t item = id - s.first, row_head = item / runs, row = row_head / s.heads;
        const int32_t run = static_cast<int32_t>(item - row_head * runs), h = static_cast<int32_t>(row_head - row * s.heads);
        const f32x4* p = reinterpret_cast<const f32x4*>(s.part) + row_head * s.per * runs + run;
        f32x4 sum = {0.0f, 0.0f, 0.0f, 0.0f};
        const int64_t n = row / a.L;
        if (row - n * a.L < steps_of(a.lengths, n, a.L))
            for (int32_t u = 0; u < s.per; ++u) sum += p[static_cast<int64_t>(u) * runs];
        Elem* to = static_cast<Elem*>(s.to.p) + n * s.to.sn + (row - n * a.L) * s.to.sl + h * s.to.sh + 4 * run;
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (4 * run + e < s.D) to[e] = Storage<Elem>::from_f32(sum[e]);
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
// 16th row.  Bound by the states' memory, read and written once: 2048 states of 128 x 128
// channels, 268 MB, in 55 us (4.9 TB/s); of 75 x 75, whose rows end within 16 bytes, by the
// second workgroup of a head, which has 11 columns (36 us where the bytes cost 18; by single
// values there 45).
constexpr int kStepColumns = 64, kStepRows = kThreads / (kStepColumns / 4);
// Rows of a thread whose loads are in flight together: 128 states of 128 x 128 channels take
// 6.4 us, with one row 9.0; 2048 of them 54.6, with eight 56.2.
constexpr int kStepAhead = 4;
// FULL: v's columns in whole fours, without the shifts (54.6 and 59.2 us there).
template <typename Elem, bool FULL>
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
        if (valid > 0 && (FULL || a.vd >= 4)) {
            // columns behind the last: the 16 bytes that end with the row, shifted
            const int over = FULL ? 0 : 4 - valid;
            for (int first = r0; first < a.kd; first += kStepAhead * kStepRows) {
                f32x4 w[kStepAhead];
                float ki[kStepAhead], qi[kStepAhead];
#pragma unroll
                for (int u = 0; u < kStepAhead; ++u) {   // rows behind the last are the last one's, and not used
                    const int i = min(first + u * kStepRows, a.kd - 1);
                    w[u] = __builtin_bit_cast(f32x4, reinterpret_cast<const Bytes16*>(a.s + at + static_cast<int64_t>(i) * a.vd - over)->v);
                    ki[u] = St::to_f32(k[i]);
                    qi[u] = St::to_f32(q[i]);
                }
#pragma unroll
                for (int u = 0; u < kStepAhead; ++u) {
                    const int i = first + u * kStepRows;
                    if (i >= a.kd) break;
                    if (!FULL && over > 0) w[u] = __builtin_bit_cast(f32x4, drop_first<float>(__builtin_bit_cast(u32x4, w[u]), over));
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        w[u][e] = fmaf(keep, w[u][e], ki[u] * x[e]);
                        sum[e] = fmaf(qi[u], w[u][e], sum[e]);
                    }
                    store_run<float, FULL>(a.s_new + at + static_cast<int64_t>(i) * a.vd, valid, __builtin_bit_cast(u32x4, w[u]));
                }
            }
        } else if (!FULL) {
            for (int i = r0; i < a.kd; i += kStepRows) {
                const float ki = St::to_f32(k[i]), qi = St::to_f32(q[i]);
                const float* s = a.s + at + static_cast<int64_t>(i) * a.vd;
                float* s_new = a.s_new + at + static_cast<int64_t>(i) * a.vd;
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

// A form of the kernel: the channels of q and k, and the waves that hold the state.  Eight
// where v has more than 64 columns, so that q and k are read once and their weights made once:
// 138 us instead of 254 for 256 heads of 2048 steps of 128 channels in bf16, 101 instead of
// 118 with 64 of q and k.  In fp32 and for wider heads it goes either way, and four are taken: of
// 256 channels eight make 116 to 180 us of 64 heads of 1024 steps in fp16, 205 to 269 in fp32
// and 100 to 109 in bf16, but 743 to 456 of 256 heads of 2048; in fp32 99 to 144 of 128 heads
// of 2048 steps with 32 channels of q and k and 128 of v, but 203 to 180 with 128.
struct Form {
    int kd, waves;
    bool operator==(const Form& o) const { return kd == o.kd && waves == o.waves; }
};
Form form_of(int dtype, int kd, int vd) {
    return {kd <= 32 ? 32 : kd <= 64 ? 64 : kd <= 128 ? 128 : 256, vd <= 64 || kd > 128 || dtype == kF32 ? 4 : 8};
}
constexpr int columns_of(int waves) { return 16 * waves; }
int64_t blocks_of(int vd, int waves) { return (vd + columns_of(waves) - 1) / columns_of(waves); }
// Workgroups that a compute unit holds of a form: two where LDS has room, of 8 waves that
// hold the state one, by its registers.
int64_t room_of(int dtype, const Form& f, int64_t units) { return units * (f.waves == 4 && f.kd <= (dtype == kF32 ? 0 : 64) ? 2 : 1); }

// The time of a form's tile beside the others', in eighths: of 256 heads of 2048 steps in
// bf16 4.2 us for 128 channels and 8 waves, 3.7 for 4 waves, 2.7 for 64 channels.
constexpr int64_t tile_time(const Form& f) { return f.kd > 128 ? 10 : (f.kd > 64 ? 6 : 4) + f.waves / 4; }

// How a call is cut: the forms of its passes and of the states' passes, and the segments
// of a sequence, `each` tiles of `tile` steps.
struct Cut {
    Form form[3], states;
    int tile;
    int32_t segments, each;
    double time;
};

// Segments shorten the walk where the heads do not fill the chip, and cost a pass over k
// and v for the states ahead of them.  A form's time is taken as its rounds of workgroups,
// each as many tiles long as a segment and kStart more, and the states' pass as half a tile
// for each, a launch more as kLaunch; joining the states as kJoin, more for their number and for their memory, which is
// written and read twice.  The cuts that fill half a round to kRounds rounds are compared.
// Of 128 shapes, all types, 512 to 16384 steps of 4 to 256 heads, the cut taken was 2 %
// slower on average than the best of all that were timed, and 10 of them more than 10 %.
constexpr int64_t kStart = 3, kLaunch = 2, kJoin = 4, kRounds = 4;   // in halves of a tile's time, 1.3 us
constexpr int64_t kJoinSegments = 8, kJoinBytes = 6'000'000;         // that cost one more
Cut cut_of(int dtype, int64_t N, int64_t L, int64_t H, const int (*dims)[2], int passes, bool apart, int64_t cus) {
    Cut c{};
    int kd = 0, vd = 0;
    for (int p = 0; p < passes; ++p) kd = std::max(kd, dims[p][0]), vd = std::max(vd, dims[p][1]);
    const Form joint = form_of(dtype, kd, vd);
    for (int p = 0; p < passes; ++p) c.form[p] = apart ? form_of(dtype, dims[p][0], dims[p][1]) : joint;
    c.states = c.form[passes - 1];   // dv's pass walks over the states' own channels
    c.tile = tile_steps(dtype == kBF16, c.states.kd);
    const int64_t tiles = std::max<int64_t>(1, (L + c.tile - 1) / c.tile);
    c.segments = 1, c.each = static_cast<int32_t>(tiles);
    if (N * H == 0) return c;
    auto time_of = [&](const Form& f, int64_t workgroups, double each) {
        const int64_t room = room_of(dtype, f, cus);
        return static_cast<double>((workgroups + room - 1) / room) * (each * static_cast<double>(tile_time(f)) / static_cast<double>(tile_time(joint)) + kStart);
    };
    auto passes_time = [&](int64_t segments, int64_t each) {   // those of one form go together
        double time = 0.0;
        for (int p = 0, next; p < passes; p = next) {
            int64_t workgroups = 0;
            for (next = p; next < passes && c.form[next] == c.form[p]; ++next)
                workgroups += N * H * blocks_of(dims[next][1], c.form[p].waves) * segments;
            time += time_of(c.form[p], workgroups, 2.0 * static_cast<double>(each)) + (p > 0 ? kLaunch : 0);
        }
        return time;
    };
    const int chains = std::min(passes, 2);
    const int64_t units = N * H * blocks_of(dims[passes - 1][1], c.states.waves), room = room_of(dtype, c.states, cus);
    c.time = passes_time(1, tiles);
    for (int64_t fill = room / 2; fill <= kRounds * room; fill += room / 2) {
        if (units * passes >= fill) continue;
        const int64_t share = fill / (units * passes), each = (tiles + share - 1) / share, segments = (tiles + each - 1) / each;
        if (segments == 1) continue;
        const int64_t bytes = N * H * chains * dims[0][0] * dims[0][1] * 16;   // of a segment's states
        const double time = passes_time(segments, each) + time_of(c.states, units * chains * (segments - 1), static_cast<double>(each)) +
                            static_cast<double>(kJoin + segments / kJoinSegments + segments * bytes / kJoinBytes);
        if (time < c.time) c.time = time, c.each = static_cast<int32_t>(each), c.segments = static_cast<int32_t>(segments);
    }
    return c;
}

// All passes in one form and one launch, or, where the forms' tiles are alike, each in the
// form of its own channels: gradients of 16 x 4096 steps of 8 heads of 128 and 64 channels
// in bf16 476 and 384 us, of one step of 64 of such a head 13 and 20 us.
Cut cut_of(int dtype, int64_t N, int64_t L, int64_t H, const int (*dims)[2], int passes) {
    const int64_t cus = device_cu_count();   // asked once: a call computes this twice, in some tenths of a microsecond
    const Cut joint = cut_of(dtype, N, L, H, dims, passes, false, cus);
    bool same = true;
    for (int p = 0; p < passes; ++p) {
        const Form own = form_of(dtype, dims[p][0], dims[p][1]);
        if (tile_steps(dtype == kBF16, own.kd) != joint.tile) return joint;
        same = same && own == joint.form[p];
    }
    if (same) return joint;
    const Cut apart = cut_of(dtype, N, L, H, dims, passes, true, cus);
    return apart.time < joint.time ? apart : joint;
}

// HIP takes fewer than 2^32 threads: more sequences than that go in several launches.
hipError_t over_sequences(const Args& a, int passes, int segments, int dtype, int threads, void (*kernel)(Args), hipStream_t stream) {
    int64_t per = 0;          // workgroups of a sequence
    for (int p = 0; p < passes; ++p) per += static_cast<int64_t>(a.H) * a.pass[p].blocks;
    const int64_t most = std::max<int64_t>(1, 0xffffffffLL / threads / (per * segments));
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
        kernel<<<static_cast<unsigned>(k.first[3]) * segments, threads, 0, stream>>>(k);
    }
    return hipGetLastError();
}

#define WG_ATTENTION_SHAPES(X) X(32, 4) X(32, 8) X(64, 4) X(64, 8) X(128, 4) X(128, 8) X(256, 4)

// A launch for the passes of one form that follow one another.
template <typename Elem, bool STATES> hipError_t run_passes(const Args& all, int passes, const Cut& cut, int dtype, hipStream_t stream) {
    for (int p = 0, next; p < passes; p = next) {
        const Form form = STATES ? cut.states : cut.form[p];
        Args a = all;
        a.segments = cut.segments, a.each = cut.each;
        for (next = p; next < passes && (STATES || cut.form[next] == form); ++next) {
            a.pass[next - p] = all.pass[next];
            a.pass[next - p].blocks = static_cast<int32_t>(blocks_of(all.pass[next].vd, form.waves));
        }
        hipError_t e = hipErrorInvalidValue;
#define WG_ATTENTION_CASE(K, W)                                                                                        \
    if constexpr (W == 4 || sizeof(Elem) == 2)                                                                         \
        if (form == Form{K, W})                                                                                        \
            e = over_sequences(a, next - p, STATES ? cut.segments - 1 : cut.segments, dtype,                           \
                               Shape<Elem, K, W, STATES>::kThreads, attention_kernel<Elem, K, W, STATES>, stream);
        WG_ATTENTION_SHAPES(WG_ATTENTION_CASE)
#undef WG_ATTENTION_CASE
        if (e) return e;
    }
    return hipSuccess;
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
    k.tile = cut.tile, k.each_steps = cut.each * k.tile, k.blocks = (size + kThreads - 1) / kThreads, k.of = of;
    k.log_decay = a.log_decay, k.lengths = a.lengths;
    const unsigned grid = static_cast<unsigned>(k.heads * k.blocks * of);
    chain_kernel<<<grid, kThreads, 0, stream>>>(k);
    return hipGetLastError();
}

// Bytes of the parts that an input's gradient is summed from: none where no heads share it.
size_t part_bytes(int64_t N, int64_t L, int64_t heads, int64_t H, int64_t D) {
    return heads == H ? 0 : static_cast<size_t>(N * L * H * ((D + 3) / 4)) * 16;
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
    if (!backward) return segment_bytes(cut_of(dtype, N, L, H, dims.forward, 1), N, H, Dk, Dv);
    return 2 * segment_bytes(cut_of(dtype, N, L, H, dims.backward, 3), N, H, Dk, Dv) +
           part_bytes(N, L, q_heads, H, Dk) + part_bytes(N, L, k_heads, H, Dk) + part_bytes(N, L, v_heads, H, Dv);
}
#endif

template <int D> hipError_t launch_linear_attention_t(const wg_linear_attention& a, hipStream_t stream) {
    using Elem = typename DTypeOf<D>::type;
    const int32_t Dk = static_cast<int32_t>(a.Dk), Dv = static_cast<int32_t>(a.Dv);
    const Dims dims(Dk, Dv);
    const Cut cut = cut_of(D, a.N, a.L, a.heads, dims.forward, 1);
    Args k{};
    k.N = a.N, k.L = static_cast<int32_t>(a.L), k.H = static_cast<int32_t>(a.heads);
    k.log_decay = a.log_decay, k.lengths = a.lengths, k.scale = static_cast<float>(a.scale);
    k.pass[0] = Pass{heads_in(a.q, a.q_heads, a.heads), heads_in(a.k, a.k_heads, a.heads), heads_in(a.v, a.v_heads, a.heads),
                     heads_out(a.y), Dk, Dv, 0, a.s0, a.s_last, {Dv, 1}, 1.0f, k.scale, 0, 0};
    if (cut.segments > 1) {
        const Chain chain{static_cast<float*>(a.workspace), a.s0, Dk * Dv, 0};
        if (const hipError_t e = run_chains<Elem>(k, &chain, 1, cut, D, stream)) return e;
        k.pass[0].s_in = chain.states, k.pass[0].s_out = a.s_last, k.pass[0].from_segments = 1;
    }
    return run_passes<Elem, false>(k, 1, cut, D, stream);
}

template <int D> hipError_t launch_linear_attention_backward_t(const wg_linear_attention_backward& a, hipStream_t stream) {
    using Elem = typename DTypeOf<D>::type;
    const int64_t H = a.heads;
    const int32_t Dk = static_cast<int32_t>(a.Dk), Dv = static_cast<int32_t>(a.Dv);
    const Dims dims_of(Dk, Dv);
    const Cut cut = cut_of(D, a.N, a.L, H, dims_of.backward, 3);
    Args k{};
    k.N = a.N, k.L = static_cast<int32_t>(a.L), k.H = static_cast<int32_t>(H);
    k.log_decay = a.log_decay, k.lengths = a.lengths, k.scale = static_cast<float>(a.scale);
    const HeadsIn q = heads_in(a.q, a.q_heads, H), kk = heads_in(a.k, a.k_heads, H), v = heads_in(a.v, a.v_heads, H),
                  dy = heads_in(a.dy, H, H);
    char* ws = static_cast<char*>(a.workspace);
    const float *s_in = a.s0, *g_in = a.ds_last;
    if (cut.segments > 1) {
        const size_t bytes = segment_bytes(cut, a.N, H, Dk, Dv);
        const Chain chains[2] = {{reinterpret_cast<float*>(ws), a.s0, Dk * Dv, 0},
                                 {reinterpret_cast<float*>(ws + bytes), a.ds_last, Dk * Dv, 1}};
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
        const int64_t D4 = (dims[p] + 3) / 4 * 4;
        return HeadsOut{const_cast<float*>(parts[p]), a.L * H * D4, H * D4, D4, 1};
    };
    const int32_t segmented = cut.segments > 1;
    k.pass[0] = Pass{dy, v, kk, to(0), Dv, Dk, 0, s_in, nullptr, {1, Dv}, 1.0f, k.scale, 0, segmented};
    k.pass[1] = Pass{v, dy, q, to(1), Dv, Dk, 0, g_in, nullptr, {1, Dv}, k.scale, 1.0f, 1, segmented};
    k.pass[2] = Pass{kk, q, dy, to(2), Dk, Dv, 0, g_in, a.ds0, {Dv, 1}, k.scale, 1.0f, 1, segmented};
    if (const hipError_t e = run_passes<Elem, false>(k, 3, cut, D, stream)) return e;
    SharedArgs s{};
    s.L = k.L, s.lengths = a.lengths;
    for (int p = 0; p < 3; ++p) {
        if (!parts[p]) continue;
        s.of[s.count++] = Shared{parts[p], out[p], static_cast<int32_t>(heads[p]), static_cast<int32_t>(H / heads[p]), dims[p], s.items};
        s.items += a.N * a.L * heads[p] * ((dims[p] + 3) / 4);
    }
    if (s.items > 0) {
        const int64_t blocks = std::min<int64_t>((s.items + kThreads - 1) / kThreads, 0xffffffffLL / kThreads);
        shared_kernel<Elem><<<static_cast<unsigned>(blocks), kThreads, 0, stream>>>(s);
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
    if (a.Dv % 4 == 0) step_kernel<Elem, true><<<static_cast<unsigned>(grid), kThreads, 0, stream>>>(k);
    else step_kernel<Elem, false><<<static_cast<unsigned>(grid), kThreads, 0, stream>>>(k);
    return hipGetLastError();
}

#define WG_ATTENTION_INSTANCES(D)                                                                    \
    template hipError_t launch_linear_attention_t<D>(const wg_linear_attention&, hipStream_t);       \
    template hipError_t launch_linear_attention_backward_t<D>(const wg_linear_attention_backward&, hipStream_t); \
    template hipError_t launch_linear_attention_step_t<D>(const wg_linear_attention_step&, hipStream_t);
WG_ATTENTION_INSTANCES(WG_DTYPE)
#undef WG_ATTENTION_INSTANCES

}  // namespace wg
