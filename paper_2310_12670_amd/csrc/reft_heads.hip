// Norm of queries and keys for each head, with the rotation by the row's position, and the gradients of both.  Kernels and their entry
// points (see include/reft.h).
#include "reft_calls.hpp"

#include <algorithm>

namespace reft {

// How the waves share the work on one kind of heads: units of wave_rows rows, each with row_groups groups of lanes, and one of `parts`
// parts of their heads.  Of the sizes alone, as sums are taken in this order.
struct Shares {
    uint64_t units;
    uint32_t parts, wave_rows, row_groups;                  // the last two powers of two
};

// One kind of heads: inputs, outputs, weight.
struct Side {
    const void *x, *dy, *weight;
    void *out;
    uint64_t row_x, head_x, row_dy, head_dy, row_out, head_out;
    uint32_t heads;
    Shares share;
};

struct HeadsArgs {
    Side side[2];                  // queries, keys
    const int64_t *positions;
    const float *freqs;
    uint64_t rows;
    uint32_t cols, pairs;
    float eps, inverse_cols;
    float *part;                   // [blocks][2][cols], of the backward pass
    uint8_t adjacent, weight_f32;
};

// Sine and cosine of position * frequency.  The angle is a product in 64 bits; the multiple of pi / 2 next to it leaves in two parts (Cody
// and Waite), so that the rest has fp32's bits whatever the position; the Taylor series then err by less than 2^-24 on |x| <= pi / 4.
__device__ __forceinline__ void sine_cosine(int64_t position, float freq, float *sine, float *cosine)
{
    const double angle = (double)position * (double)freq, k = rint(angle * 0.63661977236758134308);
    const float x = (float)fma(-k, 6.123233995736766036e-17, fma(-k, 1.57079632679489655800, angle)), s = x * x;
    const float sn = x + x * s * (-1.f / 6 + s * (1.f / 120 + s * (-1.f / 5040 + s * (1.f / 362880))));
    const float cs = 1.f + s * (-0.5f + s * (1.f / 24 + s * (-1.f / 720 + s * (1.f / 40320 + s * (-1.f / 3628800)))));
    const int quarter = (int)(k - 4. * floor(k * 0.25));
    const float a = quarter & 1 ? cs : sn, b = quarter & 1 ? sn : cs;
    *sine = quarter & 2 ? -a : a;
    *cosine = (quarter + 1) & 2 ? -b : b;
}

// The sum over G neighbouring lanes.
template <int G> __device__ __forceinline__ float sum_of(float v)
{
    v += __uint_as_float(paired<kSwap1>(__float_as_uint(v)));
    v += __uint_as_float(paired<kSwap2>(__float_as_uint(v)));
    v += __uint_as_float(paired<kMirror8>(__float_as_uint(v)));
    if (G > 8) v += __uint_as_float(paired<kMirror16>(__float_as_uint(v)));
    if (G > 16) v += __shfl_xor(v, 16);
    if (G > 32) v += __shfl_xor(v, 32);
    return v;
}

// To a step of fp32.  The hardware's takes numbers below 2^-126, which eps == 0 leaves room for, for zeroes.
__device__ __forceinline__ float inverse_root(float v)
{
    return v < 1.17549435e-38f ? 1.f / sqrtf(v) : __builtin_amdgcn_rsqf(v);
}

// How a lane comes to the values that its eight columns turn with: they are its own neighbours, all another lane's, or anyone's.
enum { kAdjacent, kLane, kAny };

// A pointer to memory of the GPU, for the compiler to know: one that was chosen among others it would take for any.
template <typename T> __device__ __forceinline__ T *global(T *p) { return (T *)(__attribute__((address_space(1))) T *)p; }

// The side with everything the same in all lanes.
__device__ __forceinline__ Side side_at(const HeadsArgs &a, bool keys)
{
    Side s = keys ? a.side[1] : a.side[0];
    s.x = global(s.x);
    s.dy = global(s.dy);
    s.weight = global(s.weight);
    s.out = global(s.out);
    return s;
}

// Eight values of a head, or none; WHOLE: there are no heads' ends between.
template <bool WHOLE, typename T> __device__ __forceinline__ void load_part(Eight<T> &e, const T *p, int n)
{
    e.template load<false>(p, WHOLE ? n > 0 ? 8 : 0 : n);
}
template <bool WHOLE, typename T> __device__ __forceinline__ void store_part(T *p, int n, const float v[8])
{
    if (!WHOLE) store8(p, n, v);
    else if (n > 0) store8(p, 8, v);
}

// A wave works on several rows at once, each with some of its 64 / G groups of G lanes; a group's lanes hold eight columns of a head each.
// Sines and cosines are computed once a row, one pair a lane and turn, and pass through the wave's own part of LDS, as do the partners of kAny.
template <typename T, int G, int MODE, bool WHOLE> struct Wave {
    struct __align__(16) Room {                             // so that a lane's eight values are two accesses
        float2 turn[4 * 64];                               // of a row 4 G pairs, those that do not turn with one and zero
        float values[MODE == kAny ? 64 * 8 + 1 : 1];       // and a zero
    };
    Room &room;
    const int lane, pairs;
    int c0, n, partner, pair0;                              // the lane's columns, their partners' lane (kAny: its group's place), the first one's pair
    bool lower;                                             // kLane: its columns come first in their pairs
    float cosine[8], sine[8];                               // of its columns; the sine with the partner's sign

    __device__ __forceinline__ Wave(Room &room, const HeadsArgs &a) : room(room), lane(threadIdx.x & 63), pairs((int)a.pairs)
    {
        c0 = lane % G * 8;
        n = (int)a.cols - c0;
        lower = c0 < pairs;
        const bool turns = c0 < 2 * pairs;
        partner = MODE == kAny ? lane / G * G * 8 : !turns ? lane : lower ? lane + pairs / 8 : lane - pairs / 8;
        pair0 = MODE == kAdjacent ? c0 / 2 : !turns ? pairs : lower ? c0 : c0 - pairs;
        if (MODE == kAny) room.values[64 * 8] = 0;
    }
    // The wave's lanes come together and see what the others have written; nothing moves across.  The barrier in the middle is no instruction: it
    // is what keeps the compiler from running some lanes ahead where only part of them has gone through a loop or branch before (a fence does not).
    __device__ __forceinline__ static void settle()
    {
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    }

    __device__ __forceinline__ void turn(const HeadsArgs &a, uint64_t row0, int rows, int row)
    {
        settle();
        for (int at = lane; at < rows * 4 * G; at += 64) {
            const int r = at / (4 * G), pair = at % (4 * G);
            float2 t = {1.f, 0.f};
            if (pair < pairs && row0 + r < a.rows) sine_cosine(a.positions[row0 + r], a.freqs[pair], &t.y, &t.x);
            room.turn[at] = t;
        }
        settle();
        const float2 *from = room.turn + row * 4 * G;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int c = c0 + i;
            const float2 t = from[MODE == kAdjacent ? pair0 + i / 2 : MODE == kLane ? pair0 + i : c >= 2 * pairs ? pairs : c < pairs ? c : c - pairs];
            cosine[i] = t.x;
            sine[i] = (MODE == kAdjacent ? !(i & 1) : MODE == kLane ? lower : c < pairs) ? -t.y : t.y;
        }
    }
    // All bits where column i of the lane's is one of a pair, none where it is not.
    __device__ __forceinline__ uint32_t in_pair(int i) const { return (uint32_t)((c0 + (MODE == kLane ? 0 : i) - 2 * pairs) >> 31); }
    // The values of the partners' columns.  A column that does not turn has a sine of zero; where what stands beside it or itself need be no number
    // (APART), it gets a zero as well: zero times an infinity would be a NaN.
    template <bool APART, typename E> __device__ __forceinline__ void partners(const Eight<E> &x, float v[8])
    {
        constexpr int kWords = (int)sizeof(E) / 2;
        if constexpr (MODE == kAny) {
            settle();
#pragma unroll
            for (int i = 0; i < 8; ++i) room.values[partner + c0 + i] = x[i];
            settle();
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int c = c0 + i;
                v[i] = room.values[c >= 2 * pairs ? 64 * 8 : partner + (c < pairs ? c + pairs : c - pairs)];
            }
        } else {
            Eight<E> y;
#pragma unroll
            for (int i = 0; i < kWords; ++i)
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    y.w[i][k] = MODE == kLane ? (uint32_t)__shfl((int)x.w[i][k], partner) : x.w[i][k];
                    if (APART) y.w[i][k] &= in_pair(kWords == 1 ? 2 * k : (4 * i + k) & ~1);
                }
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = y[MODE == kLane ? i : i ^ 1];
        }
    }
    __device__ __forceinline__ Eight<float> weight(const HeadsArgs &a, const Side &s)
    {
        Eight<float> w;
        if (!s.weight) {
#pragma unroll
            for (int i = 0; i < 8; ++i) w.t[i] = 1.f;
        } else if (a.weight_f32) {
            load_part<WHOLE>(w, (const float *)s.weight + c0, n);
        } else {
            Eight<T> e;
            load_part<WHOLE>(e, (const T *)s.weight + c0, n);
#pragma unroll
            for (int i = 0; i < 8; ++i) w.t[i] = e[i];
        }
        return w;
    }
};

// A unit as one of its wave's groups of lanes sees it: its row, and its heads head0 + slot, head0 + slot + step, ... of those of its row.
struct Unit {
    uint64_t row0, row;
    uint32_t head0, slot, step;
    int turn;                                               // the row's number among the unit's
    __device__ __forceinline__ Unit(const Shares &s, uint32_t number, int group)
    {
        const uint32_t bunch = s.parts == 1 ? number : number / s.parts;
        slot = group & (s.row_groups - 1);
        turn = (group - (int)slot) >> __builtin_ctz(s.row_groups);
        row0 = (uint64_t)bunch * s.wave_rows;
        row = row0 + turn;
        head0 = (number - bunch * s.parts) * s.row_groups;
        step = s.parts * s.row_groups;
    }
};

// out = rho (x (w cos) + x_partner (w_partner +- sin)), with rho = 1 / rms: the weights and angles are joined once a unit, so that a value takes a
// square, two products and rho.  Everything is read once and written once, all of a unit's next heads on their way.  Bound by HBM: 16384 rows of
// 64 + 8 heads of 128 in bf16 118 us, 5.1 TB/s (vector units busy 43 %; a lane a head's eight columns with its own sines 656 us, sines once
// a row 122, no element-wise ends 117; results through the L2 122; loads past it no different); 1024 of them 8.3 us, one 3.2.  Four heads at once in more
// registers, four waves a SIMD instead of five: 116, 10.5 and 3.3; three: 115, 9.9 and 3.3.  Five waves leave 96 registers, which all kernels keep to without a spill
// but those of at most 64 columns, no multiple of 8, with halves as pairs: they take four (4000 rows of 24 heads of 60 in bf16 15.7 -> 14.9 us,
// 16384 of 40 in f16 66 -> 67).
template <typename T, int G, int MODE, bool WHOLE> __global__ __launch_bounds__(256, sizeof(T) == 4 ? 1 : MODE == kAny && !WHOLE && G == 8 ? 4 : 5) void k_heads_forward(HeadsArgs a)
{
    typedef Wave<T, G, MODE, WHOLE> W;
    __shared__ typename W::Room room[4];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), group = (threadIdx.x & 63) / G;
    constexpr int kAhead = 2;                               // heads of a group worked on at once, and as many on their way
    W w(room[wave], a);
    const uint64_t units = a.side[0].share.units + a.side[1].share.units;
    for (uint64_t number = (uint64_t)blockIdx.x * 4 + wave; number < units; number += (uint64_t)gridDim.x * 4) {
        const bool keys = number >= a.side[0].share.units;
        const Side s = side_at(a, keys);
        const Unit u(s.share, (uint32_t)(keys ? number - a.side[0].share.units : number), group);
        const T *from = (const T *)s.x + u.row * s.row_x + (uint64_t)(u.head0 + u.slot) * s.head_x + w.c0;
        T *to = (T *)s.out + u.row * s.row_out + (uint64_t)(u.head0 + u.slot) * s.head_out + w.c0;
        const uint64_t step_x = u.step * s.head_x, step_out = u.step * s.head_out;
        const int there = u.row < a.rows ? w.n : 0;
        Eight<T> x[kAhead], next[kAhead];
        // all lanes of the wave go round as often
        auto fetch = [&](uint32_t head0) {
#pragma unroll
            for (int k = 0; k < kAhead; ++k) load_part<WHOLE>(next[k], from + k * step_x, head0 + k * u.step + u.slot < s.heads ? there : 0);
            from += kAhead * step_x;
        };
        fetch(u.head0);
        float other[8], by_own[8], by_other[8];
        const Eight<float> weight = w.weight(a, s);
        w.turn(a, u.row0, s.share.wave_rows, u.turn);
        w.template partners<true>(weight, other);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            by_own[i] = weight.t[i] * w.cosine[i];
            by_other[i] = other[i] * w.sine[i];
        }
        for (uint32_t head0 = u.head0; head0 < s.heads; head0 += u.step * kAhead, to += kAhead * step_out) {
#pragma unroll
            for (int k = 0; k < kAhead; ++k) x[k] = next[k];
            if (head0 + u.step * kAhead < s.heads) fetch(head0 + u.step * kAhead);
#pragma unroll
            for (int k = 0; k < kAhead; ++k) {
                if (k && head0 + k * u.step >= s.heads) break;
                float v[8], sum = 0;
                w.template partners<false>(x[k], other);       // of a head with an infinity all is lost
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    v[i] = x[k][i];
                    sum += v[i] * v[i];
                }
                sum = sum_of<G>(sum);
                float r = inverse_root(sum * a.inverse_cols + a.eps);
                const bool endless = !(sum < INFINITY);
                if (__builtin_expect(__any(endless), 0)) {
                    // a head that is too long: two of its values need not add up to a number, r times them are zeroes
                    const float by = endless ? r : 1.f;
                    r = endless ? 1.f : r;
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        v[i] *= by;
                        other[i] *= by;
                    }
                }
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] = r * (v[i] * by_own[i] + other[i] * by_other[i]);
                store_part<WHOLE>(to + k * step_out, head0 + k * u.step + u.slot < s.heads ? there : 0, v);
            }
        }
    }
}

// With u = dout turned back, xhat = x rho: dx = rho (u w - xhat mean(u w xhat)), dweight = sum of u xhat; both means of a head in one go over its lanes,
// of x^2 and of u w x.  16384 rows of 64 + 8 heads of 128 in bf16 184 us, 4.9 TB/s, on two waves a SIMD (queries' and keys' weights summed at once,
// which takes 16 registers more: 228; at 128 registers with four waves a SIMD: 411, spilled).
// The gradients; a lane sums its heads' part of a weight's gradient, the block adds its groups' in their order.  Queries first, then keys.
template <typename T, int G, int MODE, bool WHOLE> __global__ __launch_bounds__(256) void k_heads_backward(HeadsArgs a)
{
    typedef Wave<T, G, MODE, WHOLE> W;
    __shared__ typename W::Room room[4];
    __shared__ float fold[256 / G][G * 8];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), group = (threadIdx.x & 63) / G;
    constexpr int kAhead = 8 / sizeof(T);                   // heads of a group in flight
    W w(room[wave], a);
#pragma unroll 1
    for (int kind = 0; kind < 2; ++kind) {
        const Side s = side_at(a, kind);
        float dw[8] = {};
        const Eight<float> weight = w.weight(a, s);
        for (uint64_t number = (uint64_t)blockIdx.x * 4 + wave; number < s.share.units; number += (uint64_t)gridDim.x * 4) {
            const Unit u(s.share, (uint32_t)number, group);
            const T *from = (const T *)s.x + u.row * s.row_x + (uint64_t)(u.head0 + u.slot) * s.head_x + w.c0;
            const T *from_dy = (const T *)s.dy + u.row * s.row_dy + (uint64_t)(u.head0 + u.slot) * s.head_dy + w.c0;
            T *to = (T *)s.out + u.row * s.row_out + (uint64_t)(u.head0 + u.slot) * s.head_out + w.c0;
            const uint64_t step_x = u.step * s.head_x, step_dy = u.step * s.head_dy, step_out = u.step * s.head_out;
            const int there = u.row < a.rows ? w.n : 0;
            Eight<T> x[kAhead], dy[kAhead], next[kAhead], next_dy[kAhead];
            auto fetch = [&](uint32_t head0) {
#pragma unroll
                for (int k = 0; k < kAhead; ++k) {
                    const int n = head0 + k * u.step + u.slot < s.heads ? there : 0;
                    load_part<WHOLE>(next[k], from + k * step_x, n);
                    load_part<WHOLE>(next_dy[k], from_dy + k * step_dy, n);
                }
                from += kAhead * step_x;
                from_dy += kAhead * step_dy;
            };
            fetch(u.head0);
            w.turn(a, u.row0, s.share.wave_rows, u.turn);
            for (uint32_t head0 = u.head0; head0 < s.heads; head0 += u.step * kAhead, to += kAhead * step_out) {
#pragma unroll
                for (int k = 0; k < kAhead; ++k) {
                    x[k] = next[k];
                    dy[k] = next_dy[k];
                }
                if (head0 + u.step * kAhead < s.heads) fetch(head0 + u.step * kAhead);
#pragma unroll
                for (int k = 0; k < kAhead; ++k) {
                    if (k && head0 + k * u.step >= s.heads) break;
                    const int n = head0 + k * u.step + u.slot < s.heads ? there : 0;
                    float other[8], t[8], sum = 0, dot = 0;
                    w.template partners<true>(dy[k], other);
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const float v = x[k][i];
                        t[i] = dy[k][i] * w.cosine[i] - other[i] * w.sine[i];
                        sum += v * v;
                        dot += v * (t[i] * weight.t[i]);
                    }
                    float r = inverse_root(sum_of<G>(sum) * a.inverse_cols + a.eps);
                    r = n > 0 ? r : 0.f;                    // of zeroes that do not exist it may be infinite
                    dot = sum_of<G>(dot) * a.inverse_cols;
                    dot = r == 0 ? 0.f : r * dot;           // of a head that is too long it may be infinite
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const float xhat = x[k][i] * r;
                        dw[i] += t[i] * xhat;
                        t[i] = r * (t[i] * weight.t[i] - xhat * dot);
                    }
                    if (s.out) store_part<WHOLE>(to + k * step_out, n, t);
                }
            }
        }
        if (!a.part) continue;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 8; ++i) fold[threadIdx.x / G][w.c0 + i] = dw[i];
        __syncthreads();
        for (int c = threadIdx.x; c < (int)a.cols; c += 256) {
            float sum = 0;
            for (int g = 0; g < 256 / G; ++g) sum += fold[g][c];
            a.part[((uint64_t)blockIdx.x * 2 + kind) * a.cols + c] = sum;
        }
    }
}

// The weights' gradients: the blocks' parts in an order of their number alone, 64 interleaved sums and then those one after the other.
__global__ __launch_bounds__(1024) void k_heads_weights(const float *part, uint32_t n, uint32_t cols, float *dq, float *dk)
{
    __shared__ float sums[64][16];
    const uint32_t x = threadIdx.x & 15, y = threadIdx.x >> 4, at = blockIdx.x * 16 + x;
    float s = 0;
    if (at < 2 * cols)
#pragma unroll 8
        for (uint32_t i = y; i < n; i += 64) s += part[(uint64_t)i * 2 * cols + at];
    sums[y][x] = s;
    __syncthreads();
    if (y > 0 || at >= 2 * cols) return;
    for (int i = 1; i < 64; ++i) s += sums[i][x];
    float *out = at < cols ? dq : dk;
    if (out) out[at < cols ? at : at - cols] = s;
}

// ------------------------------------------------------------------------------------------------
// which kernel
// ------------------------------------------------------------------------------------------------
constexpr uint64_t kMaxHeadCols = 512;
static int lanes_of(uint64_t cols) { return cols <= 64 ? 8 : cols <= 128 ? 16 : cols <= 256 ? 32 : 64; }

constexpr uint64_t kWaves = 4096, kBackwardWaves = 2048, kTurns = 4, kBackwardBlocks = 512;
// Groups of lanes for a row: as many as leave each kTurns heads (16384 rows of 32 + 32 heads of 64, us with a row on a whole wave and on an
// eighth: 50 and 64; of 4 + 1 heads of 128 17 and 12), more where that fills the chip with `waves` units; then parts of the heads, for the same
// (1024 rows of 72 heads of 128, us with 4096 and 16384: 10.5 and 15; their gradient with 2048 and 4096: 17.5 and 18.7).
static Shares shares_of(uint64_t rows, uint64_t heads, uint64_t cols, uint64_t waves)
{
    Shares s = {};
    if (!heads) return s;
    const uint64_t groups = 64 / lanes_of(cols);
    s.row_groups = 1;
    while (s.row_groups < groups && (s.row_groups * 2 * kTurns <= heads || (s.row_groups < heads && (rows * s.row_groups + groups - 1) / groups < waves)))
        s.row_groups *= 2;
    s.wave_rows = (uint32_t)(groups / s.row_groups);
    const uint64_t bunches = (rows + s.wave_rows - 1) / s.wave_rows, turns = (heads + s.row_groups - 1) / s.row_groups;
    s.parts = (uint32_t)std::max<uint64_t>(1, std::min<uint64_t>(turns, waves / std::max<uint64_t>(1, bunches)));
    s.units = bunches * s.parts;
    return s;
}

// The gradients' blocks: what the chip holds at once at 176 registers (two waves a SIMD: 16384 rows of 72 heads of 128, us with 256, 512 and
// 1024 blocks 200, 178 and 185), or a wave for each row and 64 / G of its heads, which is no less than there are units.  More rows, heads or columns never
// have fewer blocks, so that a workspace serves all smaller calls.  (As few blocks as need no more rounds: 3000 rows of 72 heads 43.3 us, so 39.8; 1001
// rows of 12 heads of 80 in fp32 12.7 and 10.6, as 512 parts are added in whole loops; 2049 rows of 72 heads 35.2 and 36.0.)
static uint32_t backward_blocks(uint64_t rows, uint64_t q_heads, uint64_t k_heads, uint64_t cols)
{
    const uint64_t groups = 64 / lanes_of(cols), waves = rows * ((std::max(q_heads, k_heads) + groups - 1) / groups);
    return (uint32_t)std::min<uint64_t>((waves + 3) / 4, kBackwardBlocks);
}

template <typename T, int G, int MODE, bool WHOLE> static void launch(const HeadsArgs &a, uint32_t grid, bool back, hipStream_t s)
{
    if (back) k_heads_backward<T, G, MODE, WHOLE><<<grid, 256, 0, s>>>(a);
    else k_heads_forward<T, G, MODE, WHOLE><<<grid, 256, 0, s>>>(a);
}

template <typename T, int G> static hipError_t launch(const HeadsArgs &a, uint32_t grid, bool back, hipStream_t s)
{
    const bool whole = a.cols % 8 == 0;
    if (a.adjacent && whole) launch<T, G, kAdjacent, true>(a, grid, back, s);
    else if (a.adjacent) launch<T, G, kAdjacent, false>(a, grid, back, s);
    else if (a.pairs % 8 == 0 && whole) launch<T, G, kLane, true>(a, grid, back, s);
    else if (whole) launch<T, G, kAny, true>(a, grid, back, s);
    else launch<T, G, kAny, false>(a, grid, back, s);
    return hipGetLastError();
}

template <typename T> static hipError_t launch(const HeadsArgs &a, uint32_t grid, bool back, hipStream_t s)
{
    switch (lanes_of(a.cols)) {
    case 8: return launch<T, 8>(a, grid, back, s);
    case 16: return launch<T, 16>(a, grid, back, s);
    case 32: return launch<T, 32>(a, grid, back, s);
    default: return launch<T, 64>(a, grid, back, s);
    }
}

static hipError_t launch(const HeadsArgs &a, int dtype, uint32_t grid, bool back, hipStream_t s)
{
    return dtype == REFT_F32 ? launch<float>(a, grid, back, s) : dtype == REFT_BF16 ? launch<bf16>(a, grid, back, s) : launch<f16>(a, grid, back, s);
}

// Elements in places of their own: a row's heads one behind the other, or a head's rows.
static bool apart(const reft_heads *x, uint64_t rows, uint64_t heads, uint64_t cols)
{
    typedef unsigned __int128 wide;
    const wide rows_span = (wide)(rows - 1) * x->row + cols, heads_span = (wide)(heads - 1) * x->head + cols;
    return (heads == 1 || x->head >= cols) && (rows == 1 || x->row >= cols) &&
           (heads == 1 || rows == 1 || x->row >= heads_span || x->head >= rows_span);
}

// What both directions check of their common arguments.
static int check_heads(const char *who, uint64_t q_heads, const reft_heads *k, uint64_t k_heads, const int64_t *positions,
                       const float *freqs, uint64_t pairs, uint64_t rows, uint64_t cols, int dtype, int weight_dtype, double eps)
{
    NEED(is_float_type(dtype), REFT_EINVAL, "%s: unknown type %d", who, dtype);
    NEED(weight_dtype == dtype || weight_dtype == REFT_F32, REFT_EINVAL, "%s: the weights have the type of q or fp32", who);
    NEED(eps >= 0 && eps <= 1e30, REFT_EINVAL, "%s: eps is negative or no number", who);
    NEED(cols >= 1 && cols <= kMaxHeadCols, REFT_ESIZE, "%s: heads have 1 to %llu columns", who, (unsigned long long)kMaxHeadCols);
    NEED(pairs <= cols / 2, REFT_ESIZE, "%s: more pairs than columns", who);
    NEED(rows <= 0x7fffffff, REFT_ESIZE, "%s: too many rows", who);
    NEED(q_heads >= 1 && q_heads <= 65535 && (!k || (k_heads >= 1 && k_heads <= 65535)), REFT_ESIZE, "%s: 1 to 65535 heads of a kind", who);
    NEED(!rows || !pairs || (positions && freqs), REFT_EINVAL, "%s: pairs without positions or freqs", who);
    NEED(lies(positions, 8) && lies(freqs, 4), REFT_EINVAL, "%s: misaligned pointer", who);
    return REFT_OK;
}

static HeadsArgs heads_args(const int64_t *positions, const float *freqs, uint64_t pairs, int adjacent, uint64_t rows, uint64_t cols,
                            int weight_dtype, double eps)
{
    HeadsArgs a = {};
    a.positions = positions;
    a.freqs = freqs;
    a.rows = rows;
    a.cols = (uint32_t)cols;
    a.pairs = (uint32_t)pairs;
    a.eps = (float)eps;
    a.inverse_cols = 1.f / (float)cols;
    a.adjacent = adjacent != 0;
    a.weight_f32 = weight_dtype == REFT_F32;
    return a;
}

static Side side_of(const reft_heads *x, uint64_t rows, uint64_t heads, uint64_t cols, const void *weight, const reft_heads *dy,
                    const reft_heads *out)
{
    Side s = {};
    s.share = shares_of(rows, heads, cols, dy ? kBackwardWaves : kWaves);
    s.heads = (uint32_t)heads;
    s.weight = weight;
    s.x = x->p;
    s.row_x = x->row;
    s.head_x = x->head;
    if (dy) s.dy = dy->p, s.row_dy = dy->row, s.head_dy = dy->head;
    if (out) s.out = out->p, s.row_out = out->row, s.head_out = out->head;
    return s;
}

}  // namespace reft

using namespace reft;

extern "C" int reft_heads_forward(const reft_heads *q, uint64_t q_heads, const reft_heads *k, uint64_t k_heads, const void *q_weight,
                                  const void *k_weight, const int64_t *positions, const float *freqs, uint64_t pairs, int adjacent,
                                  uint64_t rows, uint64_t cols, int dtype, int weight_dtype, double eps, const reft_heads *q_out,
                                  const reft_heads *k_out, reft_stream stream)
{
    const char *who = "reft_heads_forward";
    if (const int rc = check_heads(who, q_heads, k, k_heads, positions, freqs, pairs, rows, cols, dtype, weight_dtype, eps)) return rc;
    NEED(q && q_out && (!k == !k_out), REFT_EINVAL, "%s: null pointer", who);
    if (!rows) return REFT_OK;
    NEED(q->p && q_out->p && (!k || (k->p && k_out->p)), REFT_EINVAL, "%s: null pointer", who);
    NEED(apart(q_out, rows, q_heads, cols) && (!k || apart(k_out, rows, k_heads, cols)), REFT_ESIZE, "%s: heads overlap", who);
    const size_t size = size_of(dtype), w_size = size_of(weight_dtype);
    NEED(lies(q->p, size) && lies(q_out->p, size) && (!k || (lies(k->p, size) && lies(k_out->p, size))) && lies(q_weight, w_size) &&
             lies(k_weight, w_size),
         REFT_EINVAL, "%s: misaligned pointer", who);
    if ((uintptr_t)stream == kCheckOnly) return REFT_OK;
    HeadsArgs a = heads_args(positions, freqs, pairs, adjacent, rows, cols, weight_dtype, eps);
    a.side[0] = side_of(q, rows, q_heads, cols, q_weight, nullptr, q_out);
    if (k) a.side[1] = side_of(k, rows, k_heads, cols, k_weight, nullptr, k_out);
    const uint64_t units = a.side[0].share.units + a.side[1].share.units;
    return launched(who, launch(a, dtype, (uint32_t)std::min<uint64_t>((units + 3) / 4, kMaxBlocks256), false, (hipStream_t)stream));
}

extern "C" uint64_t reft_heads_backward_workspace(uint64_t rows, uint64_t q_heads, uint64_t k_heads, uint64_t cols)
{
    if (!rows || !cols || cols > kMaxHeadCols || rows > 0x7fffffff || q_heads > 65535 || k_heads > 65535) return 0;
    return (uint64_t)backward_blocks(rows, q_heads, k_heads, cols) * 2 * cols * sizeof(float);
}

extern "C" int reft_heads_backward(const reft_heads *dq_out, const reft_heads *dk_out, const reft_heads *q, uint64_t q_heads,
                                   const reft_heads *k, uint64_t k_heads, const void *q_weight, const void *k_weight,
                                   const int64_t *positions, const float *freqs, uint64_t pairs, int adjacent, uint64_t rows,
                                   uint64_t cols, int dtype, int weight_dtype, double eps, const reft_heads *dq,
                                   const reft_heads *dk, float *dq_weight, float *dk_weight, void *workspace,
                                   uint64_t workspace_bytes, reft_stream stream)
{
    const char *who = "reft_heads_backward";
    if (const int rc = check_heads(who, q_heads, k, k_heads, positions, freqs, pairs, rows, cols, dtype, weight_dtype, eps)) return rc;
    NEED(q && dq_out && (!k == !dk_out) && (k || (!dk && !dk_weight)), REFT_EINVAL, "%s: null pointer", who);
    const bool sums = dq_weight || dk_weight;
    NEED(dq || dk || sums || !rows, REFT_EINVAL, "%s: no output", who);
    NEED(lies(dq_weight, 4) && lies(dk_weight, 4), REFT_EINVAL, "%s: misaligned pointer", who);
    hipStream_t s = (hipStream_t)stream;
    const uint32_t grid = backward_blocks(rows, q_heads, k ? k_heads : 0, cols);
    if (rows) {
        NEED(q->p && dq_out->p && (!k || (k->p && dk_out->p)) && (!dq || dq->p) && (!dk || dk->p), REFT_EINVAL, "%s: null pointer", who);
        NEED((!dq || apart(dq, rows, q_heads, cols)) && (!dk || apart(dk, rows, k_heads, cols)), REFT_ESIZE, "%s: heads overlap", who);
        const size_t size = size_of(dtype), w_size = size_of(weight_dtype);
        NEED(lies(q->p, size) && lies(dq_out->p, size) && (!k || (lies(k->p, size) && lies(dk_out->p, size))) && (!dq || lies(dq->p, size)) &&
                 (!dk || lies(dk->p, size)) && lies(q_weight, w_size) && lies(k_weight, w_size),
             REFT_EINVAL, "%s: misaligned pointer", who);
        if (sums) {
            NEED(workspace && lies(workspace, 16), REFT_EINVAL, "%s: no workspace, or not on 16 bytes", who);
            NEED(workspace_bytes >= (uint64_t)grid * 2 * cols * sizeof(float), REFT_ESIZE, "%s: workspace too small", who);
        }
    }
    if ((uintptr_t)stream == kCheckOnly) return REFT_OK;
    hipError_t e = hipSuccess;
    if (rows) {
        HeadsArgs a = heads_args(positions, freqs, pairs, adjacent, rows, cols, weight_dtype, eps);
        a.side[0] = side_of(q, rows, q_heads, cols, q_weight, dq_out, dq);
        if (k) a.side[1] = side_of(k, rows, k_heads, cols, k_weight, dk_out, dk);
        a.part = sums ? (float *)workspace : nullptr;
        e = launch(a, dtype, grid, true, s);
    }
    if (e == hipSuccess && sums) {
        k_heads_weights<<<(uint32_t)((2 * cols + 15) / 16), 1024, 0, s>>>((const float *)workspace, grid, (uint32_t)cols, dq_weight, dk_weight);
        e = hipGetLastError();
    }
    return launched(who, e);
}
