// Operators between the products of a feed-forward trained in 8 bits: the activation with what it keeps, its gradient from that, and the
// transpose of what is kept.  Kernels and their entry points (see include/reft.h).
#include "reft_calls.hpp"

#include <algorithm>

namespace reft {

struct EightIn {
    const uint8_t *q, *scales;
    uint64_t ld, ld_s;
};
struct EightOut {
    uint8_t *q, *scales;
    uint64_t ld, ld_s;
};

// ------------------------------------------------------------------------------------------------
// activations
// ------------------------------------------------------------------------------------------------
// exp(v): the exponent in base two is rounded, which makes it err by 1.25 |v| 2^-24 of the value; what is below 2^-126 is zero.
__device__ __forceinline__ float exp_of(float v) { return __builtin_amdgcn_exp2f(v * 1.44269504f); }

// a = act(g) and its slope.  With p = 1 / (1 + exp(-g)):
//   silu        a = g p                       slope p (1 + g (1 - p))
//   gelu        a = g P, P = erfc(-g / sqrt(2)) / 2        slope P + g exp(-g^2 / 2) / sqrt(2 pi)
//   gelu_tanh   as g p, with p = 1 / (1 + exp(-2 z)), z = sqrt(2 / pi) (g + 0.044715 g^3)       slope p + g p (1 - p) 2 z'
//   relu2       a = max(g, 0)^2               slope 2 max(g, 0)
// gelu's erfc is exp(-x^2) times a polynomial without constant term in 1 / (1 + 0.33 x), fitted to its relative error on x = 0 .. 10 (9.4e-8): the
// exponential is the one that the slope takes, and small results keep their bits.
template <int ACT> __device__ __forceinline__ void act(float g, float *a, float *slope)
{
    if constexpr (ACT == REFT_SILU) {
        const float p = __builtin_amdgcn_rcpf(1.f + exp_of(-g));
        *a = g * p;
        *slope = p * (1.f + g * (1.f - p));
    } else if constexpr (ACT == REFT_GELU) {
        const float e = exp_of(-0.5f * g * g), t = __builtin_amdgcn_rcpf(1.f + (0.33f * 0.70710678f) * fabsf(g));
        float c = -0.13535220585461186f;
        c = c * t + 0.4602624186943742f;
        c = c * t - 0.35119034921117176f;
        c = c * t + 0.4085349335117577f;
        c = c * t + 0.04720330746656776f;
        c = c * t + 0.2012288504807234f;
        c = c * t + 0.18295518349809692f;
        c = c * t + 0.1863578509843114f;
        const float tail = 0.5f * e * (c * t), p = g < 0 ? tail : 1.f - tail;
        *a = g * p;
        *slope = p + g * (e * 0.39894228f);
    } else if constexpr (ACT == REFT_GELU_TANH) {
        constexpr float k = 1.5957691216f;                  // 2 sqrt(2 / pi)
        const float s = g * g, p = __builtin_amdgcn_rcpf(1.f + exp_of(-k * (g + 0.044715f * g * s)));
        *a = g * p;
        *slope = p + g * p * (1.f - p) * (k * (1.f + 0.134145f * fminf(s, 1e4f)));      // from |g| = 10 on p (1 - p) is 0
    } else {
        const float m = g <= 0 ? 0.f : g;                   // a NaN stays one
        *a = m * m;
        *slope = 2.f * m;
    }
}

// ------------------------------------------------------------------------------------------------
// 8 bits
// ------------------------------------------------------------------------------------------------
// The conversions of fp32 from and to 8 bits take a power of two along, as a float of its exponent: 2^(e - 127) is e << 23, and with 255 all
// values are NaN.  To nearest even, as by a product with the power and a conversion (both compared over all bytes and powers).
__device__ __forceinline__ float power_of(uint32_t e) { return __uint_as_float(e << 23); }

// Eight neighbouring 8-bit values; those that do not exist are zeroes.
__device__ __forceinline__ w32x2 load8_bytes(const uint8_t *p, int n)
{
    w32x2 w = {0, 0};
    if (n >= 8) return *(const w32x2_any *)p;
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (i < n) {
            if (i < 4) w.x |= (uint32_t)p[i] << (8 * i);
            else w.y |= (uint32_t)p[i] << (8 * (i - 4));
        }
    return w;
}

typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef short s16x2 __attribute__((ext_vector_type(2)));

template <bool HIGH> __device__ __forceinline__ f32x2 widen2(uint32_t w, bool e5m2, float power)
{
    return e5m2 ? __builtin_amdgcn_cvt_scalef32_pk_f32_bf8(w, power, HIGH) : __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w, power, HIGH);
}

__device__ __forceinline__ void widen4(uint32_t w, bool e5m2, float power, float v[4])
{
    const f32x2 lo = widen2<false>(w, e5m2, power), hi = widen2<true>(w, e5m2, power);
    v[0] = lo.x, v[1] = lo.y, v[2] = hi.x, v[3] = hi.y;
}

// Four values in 8 bits.
__device__ __forceinline__ uint32_t to_four(float v0, float v1, float v2, float v3, float power, bool e5m2)
{
    s16x2 w = {0, 0};
    if (e5m2) {
        w = __builtin_amdgcn_cvt_scalef32_pk_bf8_f32(w, v0, v1, power, false);
        w = __builtin_amdgcn_cvt_scalef32_pk_bf8_f32(w, v2, v3, power, true);
    } else {
        w = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(w, v0, v1, power, false);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(w, v2, v3, power, true);
    }
    return __builtin_bit_cast(uint32_t, w);
}

__device__ __forceinline__ w32x2 to_eight_scaled(const float v[8], float power, bool e5m2)
{
    w32x2 w;
    w.x = to_four(v[0], v[1], v[2], v[3], power, e5m2);
    w.y = to_four(v[4], v[5], v[6], v[7], power, e5m2);
    return w;
}

// The larger of a magnitude and two values'; a NaN stays one, as bits larger than all numbers.
__device__ __forceinline__ float larger(float most, float a, float b)
{
    return __builtin_elementwise_maximum(__builtin_elementwise_maximum(most, fabsf(a)), fabsf(b));
}
__device__ __forceinline__ uint32_t largest_of(const float v[8])
{
    return magnitude(larger(larger(larger(larger(0.f, v[0], v[1]), v[2], v[3]), v[4], v[5]), v[6], v[7]));
}

// ------------------------------------------------------------------------------------------------
// forward
// ------------------------------------------------------------------------------------------------
struct GateForward {
    const void *g, *u;
    uint64_t ld_g, ld_u, rows, cols;
    void *y;
    uint64_t ld_y;
    EightOut y8, g8, u8;
    uint32_t words;                                         // of 512 columns in a row
    uint8_t y_e5m2, kept_e5m2;
};

// Eight of a row's values in 8 bits with the power of two of the 16 lanes' 128.  FULL: there are all of them.
template <bool FULL> __device__ __forceinline__ void leave_row(const EightOut &o, const float v[8], uint64_t row, uint64_t c, int n, bool e5m2)
{
    const uint32_t e = scale_of(max_of_16(largest_of(v)), top_of(e5m2));
    store8_bytes<true>(o.q + row * o.ld + c, FULL ? 8 : n, to_eight_scaled(v, power_of(e), e5m2));
    if ((threadIdx.x & 15) == 0) o.scales[(c / 512 * o.ld_s + row) * 4 + c / 128 % 4] = FULL || n > 0 ? (uint8_t)e : 127;
}

template <typename T, int ACT, bool FULL> __device__ __forceinline__ void gate_row(const GateForward &a, uint64_t row, uint64_t c)
{
    const int n = FULL ? 8 : c < a.cols ? (int)min(a.cols - c, (uint64_t)8) : 0;
    Eight<T> g, u;
    g.template load<false>((const T *)a.g + row * a.ld_g + c, n);
    if (a.u) u.template load<false>((const T *)a.u + row * a.ld_u + c, n);
    float v[8], y[8], slope;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        act<ACT>(g[i], &y[i], &slope);
        if (a.u) y[i] *= u[i];
    }
    if (a.y) store8((T *)a.y + row * a.ld_y + c, n, y);
    if (a.y8.q) leave_row<FULL>(a.y8, y, row, c, n, a.y_e5m2);
    if (a.g8.q) {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = g[i];
        leave_row<FULL>(a.g8, v, row, c, n, a.kept_e5m2);
    }
    if (a.u8.q) {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = u[i];
        leave_row<FULL>(a.u8, v, row, c, n, a.kept_e5m2);
    }
}

// A wave takes 512 columns of a row, 16 lanes each block of 128; waves follow each other along the rows.  Bound by HBM: 16384 x 11008 in
// bf16, silu, all three in 8 bits, 211 us, 6.0 TB/s (columns by columns, as a grid of words and rows is dealt out: 300; two rows a wave 220;
// reading past the L2 202, but 2048 x 4096 11.4 -> 13.4 and 4096 x 11008 in fp32 113 -> 121); one row of 28672 2.2 us.
template <typename T, int ACT> __global__ __launch_bounds__(256) void k_gate_forward(GateForward a)
{
    const uint32_t number = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), row = number / a.words;
    const uint64_t first = (uint64_t)(number - row * a.words) * 512, c = first + (threadIdx.x & 63) * 8;
    if (row >= a.rows) return;
    if (first + 512 <= a.cols) gate_row<T, ACT, true>(a, row, c);
    else gate_row<T, ACT, false>(a, row, c);
}

// ------------------------------------------------------------------------------------------------
// backward, and the transpose: tiles of 128 x 128 values, a thread holds 4 rows of 8 columns
// ------------------------------------------------------------------------------------------------
struct Tile {
    uint64_t row0, col0;
    uint32_t down, along, high, wide;                       // number of the tile, and of tiles
    int rows, cols;                                         // of the matrix in it
};

// Tiles go down the columns of a band, `band` of them, along it, and then to the next band.
__device__ __forceinline__ Tile tile_of(uint32_t number, uint64_t rows, uint64_t cols, uint32_t band)
{
    Tile t;
    t.high = (uint32_t)((rows + 127) / 128);
    t.wide = (uint32_t)((cols + 127) / 128);
    const uint32_t first = number / (band * t.wide) * band, in = number - first * t.wide, tall = min(t.high - first, band);
    t.along = in / tall;
    t.down = first + in - t.along * tall;
    t.row0 = (uint64_t)t.down * 128;
    t.col0 = (uint64_t)t.along * 128;
    t.rows = (int)min(rows - t.row0, (uint64_t)128);
    t.cols = (int)min(cols - t.col0, (uint64_t)128);
    return t;
}

constexpr int kTileThreads = 512, kRows = 4;               // and rows of a thread

// A thread's place in the tile: eight columns of kRows rows, of which its wave, which is the same in all lanes, has 4 kRows.  An element's
// address is one of the wave's and an offset of O bits in it.
template <typename O> struct Place {
    int lane, wave, c, r;
    __device__ __forceinline__ Place()
    {
        lane = threadIdx.x & 63;
        wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        c = (lane & 15) * 8;
        r = wave * 4 * kRows + (lane >> 4) * kRows;
    }
    // Row i of the thread's in a matrix of rows (x), scales of rows (s: words).
    template <typename E> __device__ __forceinline__ E *in(E *x, uint64_t ld, const Tile &t, int i) const
    {
        return x + (t.row0 + wave * 4 * kRows + i) * ld + t.col0 + ((O)(lane >> 4) * kRows * (O)ld + c);
    }
    template <typename E> __device__ __forceinline__ E *scale(E *s, uint64_t ld_s, const Tile &t, int i) const
    {
        return s + ((t.along / 4 * ld_s + t.row0 + wave * 4 * kRows + i) * 4 + t.along % 4) + (lane >> 4) * kRows * 4u;
    }
};

// Transposes of N tiles of values on their way out, each in 8 bits with a power of two for each of its columns.
template <int N, typename O> struct Turn {
    // Bytes of eight columns of 128 rows, and four banks more: no two of a wave's words, eight columns and four rows apart, meet.
    static constexpr int kPitch = 1024 + 16;
    __align__(16) uint8_t tile[N][16 * kPitch];
    uint32_t most[N][kTileThreads / 64][128];
    __align__(16) float power[N][128];

    // First the columns' largest magnitudes in each wave.  A step halves the lanes that hold a column and joins two columns, in
    // the halves of the wave and then in their halves; the wave's four rows of lanes end with columns 0, 2, 1, 3 and the same and four.
    __device__ __forceinline__ void look(int which, const float (&v)[kRows][8], const Place<O> &at)
    {
        uint32_t m[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) m[j] = magnitude(larger(larger(0.f, v[0][j], v[1][j]), v[2][j], v[3][j]));
#pragma unroll
        for (int j = 0; j < 8; j += 2) {
            const auto r = __builtin_amdgcn_permlane32_swap(m[j], m[j + 1], false, false);
            m[j] = max(r[0], r[1]);
        }
#pragma unroll
        for (int j = 0; j < 8; j += 4) {
            const auto r = __builtin_amdgcn_permlane16_swap(m[j], m[j + 2], false, false);
            most[which][at.wave][at.c + j + (at.lane >> 5) + 2 * (at.lane >> 4 & 1)] = max(r[0], r[1]);
        }
    }
    // Then, behind a barrier, their powers of two.
    __device__ __forceinline__ void decide(int which, int c, const EightOut &o, const Tile &t, bool e5m2)
    {
        uint32_t m = 0;
#pragma unroll
        for (int w = 0; w < kTileThreads / 64; ++w) m = max(m, most[which][w][c]);
        const uint32_t e = scale_of(m, top_of(e5m2));
        if (c < t.cols) store_scale(o.scales, o.ld_s, t.col0 + c, t.down, t.high, e);
        power[which][c] = power_of(e);
    }
    // Behind another, the bytes.
    __device__ __forceinline__ void put(int which, const float (&v)[kRows][8], bool e5m2, const Place<O> &at)
    {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            *(uint32_t *)(tile[which] + at.c / 8 * kPitch + j * 128 + at.r) = to_four(v[0][j], v[1][j], v[2][j], v[3][j], power[which][at.c + j], e5m2);
    }
    // And behind a last one whole rows of the transpose.
    template <bool FULL, bool LINES> __device__ __forceinline__ void leave(int which, const EightOut &o, const Tile &t, const Place<O> &at)
    {
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const int c0 = at.wave * 16 + k * 8, c = c0 + (at.lane >> 3), r = (at.lane & 7) * 16;
            if (!FULL && (c >= t.cols || r >= t.rows)) continue;
            const uint8_t *from = tile[which] + c0 / 8 * kPitch + (at.lane >> 3) * 128 + r;
            uint8_t *to = o.q + (t.col0 + c0) * o.ld + t.row0 + ((O)(at.lane >> 3) * (O)o.ld + r);
            if (FULL || r + 16 <= t.rows) {
                if constexpr (LINES) __builtin_nontemporal_store(*(const w32x4 *)from, (w32x4_any *)to);
                else *(w32x4_any *)to = *(const w32x4 *)from;
            } else {
                for (int i = 0; i < t.rows - r; ++i) to[i] = from[i];
            }
        }
    }
};

// Eight of a tile's row in 8 bits with the power of two of the row's 128.
template <bool FULL, bool LINES, typename O>
__device__ __forceinline__ void leave_part(const EightOut &o, const float (&v)[8], const Tile &t, const Place<O> &at, int i, bool e5m2)
{
    const uint32_t e = scale_of(max_of_16(largest_of(v)), top_of(e5m2));
    if (!FULL && at.r + i >= t.rows) return;
    if (at.c == 0) {
        uint8_t *byte = at.scale(o.scales, o.ld_s, t, i);
        *byte = (uint8_t)e;
        if (t.along + 1 == t.wide)                          // ones in the rest of the row's last word
            for (int k = 1; k < 4 - (int)(t.along % 4); ++k) byte[k] = 127;
    }
    store8_bytes<LINES>(at.in(o.q, o.ld, t, i), FULL ? 8 : t.cols - at.c, to_eight_scaled(v, power_of(e), e5m2));
}

// A thread's rows of 8-bit values, and their powers of two.
struct Rows {
    w32x2 q[kRows];
    uint32_t e[kRows];

    template <bool FULL, typename O> __device__ __forceinline__ void load(const EightIn &x, const Tile &t, const Place<O> &at)
    {
#pragma unroll
        for (int i = 0; i < kRows; ++i) {
            const int n = FULL ? 8 : at.r + i < t.rows ? t.cols - at.c : 0;
            q[i] = load8_bytes(at.in(x.q, x.ld, t, i), n);
            e[i] = FULL || n > 0 ? *at.scale(x.scales, x.ld_s, t, i) : 0;
        }
    }
    // Four of row i, the first or the last.
    __device__ __forceinline__ void widen(int i, int half, bool e5m2, float v[4]) const { widen4(q[i][half], e5m2, power_of(e[i]), v); }
};

struct GateBackward {
    const void *dy;
    uint64_t ld_dy, rows, cols;
    EightIn g8, u8;
    void *dg, *du;
    uint64_t ld_dg, ld_du;
    EightOut dg8, du8, dg8_t, du8_t, y8_t;
    uint32_t band;
    uint8_t turns;                                          // which of the last three there are
    uint8_t kept_e5m2, grad_e5m2, y_e5m2;
};

// The kernel's arguments as they lie in memory: more than the scalar registers hold, so that each is read where it is used (what is
// said here keeps the compiler from reading all of them first and holding them in vector registers).
typedef const __attribute__((address_space(4))) GateBackward *GateArgs;
__device__ __forceinline__ GateArgs gate_args()
{
    GateArgs a = (GateArgs)__builtin_amdgcn_kernarg_segment_ptr();
    asm volatile("" : "+s"(a));
    return a;
}
template <typename T> __device__ __forceinline__ T *global(T *p) { return (T *)(__attribute__((address_space(1))) T *)p; }
__device__ __forceinline__ EightIn read(const __attribute__((address_space(4))) EightIn &x)
{
    return EightIn{global(x.q), global(x.scales), x.ld, x.ld_s};
}
__device__ __forceinline__ EightOut read(const __attribute__((address_space(4))) EightOut &x)
{
    return EightOut{global(x.q), global(x.scales), x.ld, x.ld_s};
}

// The gradients at the kept values, dg = dy u act'(g) and du = dy act(g), and y = act(g) u, in every order that is asked for: what is read once
// is worked on once.  The rows' results leave while the columns' powers of two are settled, then the columns' (three tiles of fp32 in
// registers) through LDS.  16384 x 11008 in bf16, silu, all five 8-bit results, 333 to 349 us, 4.7 to 4.9 TB/s: HBM's rate explains 70 % of the
// time, the vector units' 31 instructions a value 50 %, and two blocks a compute unit (their registers allow no more) do not hide all of one
// behind the other; the rows' results alone take 218 us (5.0 TB/s), the columns' alone 292 (4.3).  At the ends of a matrix each row's loads are behind branches
// and waits of their own, one round trip to memory after the other: 1001 x 1728 14 us.  (160 registers, one block: 570 us; 128 with 55 spilled: 475; a block of 1024 that has its next tile on the way: 467.)  FULL: the tile lies within the matrix;
// E4M3: so are all 8-bit matrices, and no conversion is chosen while it runs (4096 x 4096 32 -> 28 us).
template <typename T, int ACT, bool FULL, bool E4M3, bool LINES, typename O> __device__ __forceinline__ void gate_tile(const Tile &t, Turn<3, O> &turn)
{
    const Place<O> at;
    const bool gated = gate_args()->u8.q;
    float dg[kRows][8], du[kRows][8], y[kRows][8];
    {
        Eight<T> dy[kRows];
        Rows g8, u8 = {};
        const GateArgs a = gate_args();
        const T *from = global((const T *)a->dy);
        const bool e5m2 = !E4M3 && a->kept_e5m2;
#pragma unroll
        for (int i = 0; i < kRows; ++i)
            dy[i].template load<false>(at.in(from, a->ld_dy, t, i), FULL ? 8 : at.r + i < t.rows ? t.cols - at.c : 0);
        g8.load<FULL>(read(a->g8), t, at);
        if (gated) u8.load<FULL>(read(gate_args()->u8), t, at);
#pragma unroll
        for (int i = 0; i < kRows; ++i)
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                float g[4], u[4] = {1.f, 1.f, 1.f, 1.f};
                g8.widen(i, half, e5m2, g);
                if (gated) u8.widen(i, half, e5m2, u);
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const int j = half * 4 + k;
                    float v, slope;
                    act<ACT>(g[k], &v, &slope);
                    const float d = dy[i][j];
                    dg[i][j] = d * u[k] * slope;
                    du[i][j] = d * v;
                    y[i][j] = v * u[k];
                    // here and not where they are used, behind branches, with all that they are made of held until then
                    asm volatile("" : "+v"(dg[i][j]), "+v"(du[i][j]), "+v"(y[i][j]));
                }
                __builtin_amdgcn_sched_barrier(0);          // more values under way than four would not fit the registers
            }
    }
    auto wide = [&](T *out, uint64_t ld, const float (&v)[kRows][8]) {
#pragma unroll
        for (int i = 0; i < kRows; ++i) store8(at.in(global(out), ld, t, i), FULL ? 8 : at.r + i < t.rows ? t.cols - at.c : 0, v[i]);
    };
    auto rows = [&](const EightOut &o, bool e5m2, const float (&v)[kRows][8]) {
#pragma unroll
        for (int i = 0; i < kRows; ++i) leave_part<FULL, LINES>(o, v[i], t, at, i, e5m2);
    };
    turn.look(0, dg, at);
    turn.look(1, du, at);
    turn.look(2, y, at);
    __syncthreads();
    // two waves for each of the three
    if (const GateArgs a = gate_args(); at.wave < 6 && (a->turns >> at.wave / 2 & 1)) {
        const int which = at.wave / 2;
        turn.decide(which, at.wave % 2 * 64 + at.lane, read(which == 0 ? a->dg8_t : which == 1 ? a->du8_t : a->y8_t), t,
                    !E4M3 && (which == 2 ? a->y_e5m2 : a->grad_e5m2));
    }
    if (const GateArgs a = gate_args(); a->dg) wide((T *)a->dg, a->ld_dg, dg);
    if (const GateArgs a = gate_args(); a->du) wide((T *)a->du, a->ld_du, du);
    if (const GateArgs a = gate_args(); a->dg8.q) rows(read(a->dg8), !E4M3 && a->grad_e5m2, dg);
    if (const GateArgs a = gate_args(); a->du8.q) rows(read(a->du8), !E4M3 && a->grad_e5m2, du);
    if (gate_args()->turns == 0) return;
    __syncthreads();
    if (const GateArgs a = gate_args(); a->turns & 1) turn.put(0, dg, !E4M3 && a->grad_e5m2, at);
    if (const GateArgs a = gate_args(); a->turns & 2) turn.put(1, du, !E4M3 && a->grad_e5m2, at);
    if (const GateArgs a = gate_args(); a->turns & 4) turn.put(2, y, !E4M3 && a->y_e5m2, at);
    __syncthreads();
    if (const GateArgs a = gate_args(); a->turns & 1) turn.template leave<FULL, LINES>(0, read(a->dg8_t), t, at);
    if (const GateArgs a = gate_args(); a->turns & 2) turn.template leave<FULL, LINES>(1, read(a->du8_t), t, at);
    if (const GateArgs a = gate_args(); a->turns & 4) turn.template leave<FULL, LINES>(2, read(a->y8_t), t, at);
}

__device__ __forceinline__ bool full(const Tile &t) { return t.rows == 128 && t.cols == 128; }

template <typename T, int ACT, bool LINES, typename O> __global__ __launch_bounds__(kTileThreads) void k_gate_backward(GateBackward a)
{
    __shared__ Turn<3, O> turn;
    const Tile t = tile_of(blockIdx.x, a.rows, a.cols, a.band);
    if (sizeof(O) == 8 || !full(t)) gate_tile<T, ACT, false, false, LINES>(t, turn);
    else if (a.kept_e5m2 || a.grad_e5m2 || a.y_e5m2) gate_tile<T, ACT, true, false, LINES>(t, turn);
    else gate_tile<T, ACT, true, true, LINES>(t, turn);
}

struct TransposeArgs {
    EightIn q;
    EightOut q_t;
    uint64_t rows, cols;
    uint32_t band;
    uint8_t e5m2, e5m2_t;
};

template <bool FULL, bool LINES, typename O> __device__ __forceinline__ void transpose_tile(const TransposeArgs &a, const Tile &t, Turn<1, O> &turn)
{
    const Place<O> at;
    Rows q;
    q.load<FULL>(a.q, t, at);
    float v[kRows][8];
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
        q.widen(i, 0, a.e5m2, v[i]);
        q.widen(i, 1, a.e5m2, v[i] + 4);
    }
    turn.look(0, v, at);
    __syncthreads();
    if (at.wave < 2) turn.decide(0, at.wave * 64 + at.lane, a.q_t, t, a.e5m2_t);
    __syncthreads();
    turn.put(0, v, a.e5m2_t, at);
    __syncthreads();
    turn.template leave<FULL, LINES>(0, a.q_t, t, at);
}

// Bound by HBM where large: 16384 x 8192 53 us, 5.1 TB/s (85 with the columns' maxima through shuffles and 64 reads of LDS a thread).
template <bool LINES, typename O> __global__ __launch_bounds__(kTileThreads) void k_transpose(TransposeArgs a)
{
    __shared__ Turn<1, O> turn;
    const Tile t = tile_of(blockIdx.x, a.rows, a.cols, a.band);
    if (full(t)) transpose_tile<true, LINES>(a, t, turn);
    else transpose_tile<false, LINES>(a, t, turn);
}

// ------------------------------------------------------------------------------------------------
// which kernel
// ------------------------------------------------------------------------------------------------
template <typename T> static hipError_t launch_forward(const GateForward &a, int kind, hipStream_t s)
{
    const uint32_t grid = (uint32_t)((a.rows * a.words + 3) / 4);
    if (kind == REFT_SILU) k_gate_forward<T, REFT_SILU><<<grid, 256, 0, s>>>(a);
    else if (kind == REFT_GELU) k_gate_forward<T, REFT_GELU><<<grid, 256, 0, s>>>(a);
    else if (kind == REFT_GELU_TANH) k_gate_forward<T, REFT_GELU_TANH><<<grid, 256, 0, s>>>(a);
    else k_gate_forward<T, REFT_RELU2><<<grid, 256, 0, s>>>(a);
    return hipGetLastError();
}

// Tiles of a band: neighbours in the transpose are written soon after each other.  Gradients of 16384 x 11008 in bands of 1, 8, 32 and 128 tiles, us: 384,
// 358, 354 and 393; with results in 16 bits, whose rows are wider (8192 x 11008), of 1, 8 and 32: 150, 164 and 177.  The transpose of 16384 x
// 8192 in bands of 1, 8, 32 and 128: 65, 60, 53 and 62.
constexpr uint32_t kGateBand = 8, kTransposeBand = 32;

// Results whose rows lie on cache lines, which tiles then do not share, are written past the L2.
static bool lines_of(const EightOut &o) { return !o.q || on_lines(o.q, o.ld); }
// Offsets of a wave's rows fit 32 bits.
static bool near(uint64_t ld) { return ld < (1u << 26); }

template <typename T, int ACT> static void launch_backward(const GateBackward &a, bool lines, bool far, uint32_t grid, hipStream_t s)
{
    if (far) k_gate_backward<T, ACT, false, uint64_t><<<grid, kTileThreads, 0, s>>>(a);
    else if (lines) k_gate_backward<T, ACT, true, uint32_t><<<grid, kTileThreads, 0, s>>>(a);
    else k_gate_backward<T, ACT, false, uint32_t><<<grid, kTileThreads, 0, s>>>(a);
}

template <typename T> static hipError_t launch_backward(const GateBackward &a, int kind, hipStream_t s)
{
    const uint32_t grid = (uint32_t)((a.rows + 127) / 128 * ((a.cols + 127) / 128));
    const bool lines = lines_of(a.dg8) && lines_of(a.du8) && lines_of(a.dg8_t) && lines_of(a.du8_t) && lines_of(a.y8_t);
    const bool far = !(near(a.ld_dy) && near(a.ld_dg) && near(a.ld_du) && near(a.g8.ld) && near(a.u8.ld) && near(a.dg8.ld) && near(a.du8.ld) &&
                       near(a.dg8_t.ld) && near(a.du8_t.ld) && near(a.y8_t.ld));
    if (kind == REFT_SILU) launch_backward<T, REFT_SILU>(a, lines, far, grid, s);
    else if (kind == REFT_GELU) launch_backward<T, REFT_GELU>(a, lines, far, grid, s);
    else if (kind == REFT_GELU_TANH) launch_backward<T, REFT_GELU_TANH>(a, lines, far, grid, s);
    else launch_backward<T, REFT_RELU2>(a, lines, far, grid, s);
    return hipGetLastError();
}

constexpr uint64_t kMaxTiles = 0x7fffff;                // a grid has less than 2^32 threads: blocks of 512

static bool is_act(int k) { return k >= REFT_SILU && k <= REFT_RELU2; }

// An 8-bit operand that is there.
static bool given(const reft_eight *x) { return x && x->q; }

// An 8-bit matrix [rows][cols] as it has to lie; REFT_OK also for one that is left out.
static int check_eight(const char *who, const char *name, const reft_eight *x, uint64_t rows, uint64_t cols)
{
    if (!given(x)) return REFT_OK;
    NEED(x->scales || !rows || !cols, REFT_EINVAL, "%s: %s is 8 bits without scales", who, name);
    NEED(x->ld >= cols, REFT_ESIZE, "%s: rows of %s overlap", who, name);
    NEED(x->ld_s >= rows, REFT_ESIZE, "%s: words of scales of %s overlap", who, name);
    return REFT_OK;
}

static EightIn in_of(const reft_eight *x)
{
    EightIn e = {};
    if (given(x)) e = {(const uint8_t *)x->q, (const uint8_t *)x->scales, x->ld, x->ld_s};
    return e;
}
static EightOut out_of(const reft_eight *x)
{
    EightOut e = {};
    if (given(x)) e = {(uint8_t *)x->q, (uint8_t *)x->scales, x->ld, x->ld_s};
    return e;
}

}  // namespace reft

using namespace reft;

#define CHECK_EIGHT(who, x, rows, cols)                                                           \
    do {                                                                                          \
        const int rc = check_eight(who, #x, x, rows, cols);                                       \
        if (rc != REFT_OK) return rc;                                                             \
    } while (0)

extern "C" int reft_gate_forward(const void *g, uint64_t ld_g, const void *u, uint64_t ld_u, uint64_t rows, uint64_t cols, int dtype,
                                 int act, void *y, uint64_t ld_y, const reft_eight *y8, int y_format, const reft_eight *g8,
                                 const reft_eight *u8, int kept_format, reft_stream stream)
{
    const char *who = "reft_gate_forward";
    NEED(is_float_type(dtype), REFT_EINVAL, "%s: unknown type %d", who, dtype);
    NEED(is_act(act), REFT_EINVAL, "%s: unknown activation %d", who, act);
    NEED(rows <= 0x7fffffff && cols <= 0x7fffffff, REFT_ESIZE, "%s: too many rows or columns", who);
    NEED(ld_g >= cols && (!u || ld_u >= cols) && (!y || ld_y >= cols), REFT_ESIZE, "%s: rows overlap", who);
    CHECK_EIGHT(who, y8, rows, cols);
    CHECK_EIGHT(who, g8, rows, cols);
    CHECK_EIGHT(who, u8, rows, cols);
    NEED(!given(y8) || is_eight(y_format), REFT_EINVAL, "%s: unknown 8-bit format %d of y8", who, y_format);
    NEED((!given(g8) && !given(u8)) || is_eight(kept_format), REFT_EINVAL, "%s: unknown 8-bit format %d", who, kept_format);
    if (!rows || !cols) return REFT_OK;
    NEED(y || given(y8) || given(g8) || given(u8), REFT_EINVAL, "%s: no output", who);
    NEED(u || !given(u8), REFT_EINVAL, "%s: u8 without u", who);
    NEED(g, REFT_EINVAL, "%s: null pointer", who);
    NEED((rows * ((cols + 511) / 512) + 3) / 4 <= kMaxBlocks256, REFT_ESIZE, "%s: too many values", who);
    NEED(lies(g, size_of(dtype)) && lies(u, size_of(dtype)) && lies(y, size_of(dtype)), REFT_EINVAL, "%s: misaligned pointer", who);
    if ((uintptr_t)stream == kCheckOnly) return REFT_OK;
    GateForward a;
    a.g = g;
    a.u = u;
    a.ld_g = ld_g;
    a.ld_u = ld_u;
    a.rows = rows;
    a.cols = cols;
    a.y = y;
    a.ld_y = ld_y;
    a.words = (uint32_t)((cols + 511) / 512);
    a.y8 = out_of(y8);
    a.g8 = out_of(g8);
    a.u8 = out_of(u8);
    a.y_e5m2 = y_format == REFT_E5M2;
    a.kept_e5m2 = kept_format == REFT_E5M2;
    hipStream_t s = (hipStream_t)stream;
    return launched(who, dtype == REFT_F32    ? launch_forward<float>(a, act, s)
                         : dtype == REFT_BF16 ? launch_forward<bf16>(a, act, s)
                                              : launch_forward<f16>(a, act, s));
}

extern "C" int reft_gate_backward(const void *dy, uint64_t ld_dy, const reft_eight *g8, const reft_eight *u8, int kept_format,
                                  uint64_t rows, uint64_t cols, int dtype, int act, void *dg, uint64_t ld_dg, void *du,
                                  uint64_t ld_du, const reft_eight *dg8, const reft_eight *du8, const reft_eight *dg8_t,
                                  const reft_eight *du8_t, int grad_format, const reft_eight *y8_t, int y_format,
                                  reft_stream stream)
{
    const char *who = "reft_gate_backward";
    NEED(is_float_type(dtype), REFT_EINVAL, "%s: unknown type %d", who, dtype);
    NEED(is_act(act), REFT_EINVAL, "%s: unknown activation %d", who, act);
    NEED(is_eight(kept_format), REFT_EINVAL, "%s: unknown 8-bit format %d", who, kept_format);
    NEED(rows <= 0x7fffffff && cols <= 0x7fffffff, REFT_ESIZE, "%s: too many rows or columns", who);
    NEED(ld_dy >= cols && (!dg || ld_dg >= cols) && (!du || ld_du >= cols), REFT_ESIZE, "%s: rows overlap", who);
    CHECK_EIGHT(who, g8, rows, cols);
    CHECK_EIGHT(who, u8, rows, cols);
    CHECK_EIGHT(who, dg8, rows, cols);
    CHECK_EIGHT(who, du8, rows, cols);
    CHECK_EIGHT(who, dg8_t, cols, rows);
    CHECK_EIGHT(who, du8_t, cols, rows);
    CHECK_EIGHT(who, y8_t, cols, rows);
    NEED((!given(dg8) && !given(du8) && !given(dg8_t) && !given(du8_t)) || is_eight(grad_format), REFT_EINVAL,
         "%s: unknown 8-bit format %d of the gradients", who, grad_format);
    NEED(!given(y8_t) || is_eight(y_format), REFT_EINVAL, "%s: unknown 8-bit format %d of y8_t", who, y_format);
    if (!rows || !cols) return REFT_OK;
    NEED(dg || du || given(dg8) || given(du8) || given(dg8_t) || given(du8_t) || given(y8_t), REFT_EINVAL, "%s: no output", who);
    NEED(given(u8) || (!du && !given(du8) && !given(du8_t)), REFT_EINVAL, "%s: a gradient of u without u8", who);
    NEED(dy && given(g8), REFT_EINVAL, "%s: null pointer", who);
    NEED((rows + 127) / 128 * ((cols + 127) / 128) <= kMaxTiles, REFT_ESIZE, "%s: too many values", who);
    NEED(lies(dy, size_of(dtype)) && lies(dg, size_of(dtype)) && lies(du, size_of(dtype)), REFT_EINVAL, "%s: misaligned pointer", who);
    if ((uintptr_t)stream == kCheckOnly) return REFT_OK;
    GateBackward a;
    a.dy = dy;
    a.ld_dy = ld_dy;
    a.rows = rows;
    a.cols = cols;
    a.g8 = in_of(g8);
    a.u8 = in_of(u8);
    a.dg = dg;
    a.du = du;
    a.ld_dg = dg ? ld_dg : 0;
    a.ld_du = du ? ld_du : 0;
    a.dg8 = out_of(dg8);
    a.du8 = out_of(du8);
    a.dg8_t = out_of(dg8_t);
    a.du8_t = out_of(du8_t);
    a.y8_t = out_of(y8_t);
    a.turns = (a.dg8_t.q ? 1 : 0) | (a.du8_t.q ? 2 : 0) | (a.y8_t.q ? 4 : 0);
    a.band = given(dg8) || given(du8) || given(dg8_t) || given(du8_t) ? kGateBand : 1;
    a.kept_e5m2 = kept_format == REFT_E5M2;
    a.grad_e5m2 = grad_format == REFT_E5M2;
    a.y_e5m2 = y_format == REFT_E5M2;
    hipStream_t s = (hipStream_t)stream;
    return launched(who, dtype == REFT_F32    ? launch_backward<float>(a, act, s)
                         : dtype == REFT_BF16 ? launch_backward<bf16>(a, act, s)
                                              : launch_backward<f16>(a, act, s));
}

extern "C" int reft_transpose(const reft_eight *q, int format, uint64_t rows, uint64_t cols, const reft_eight *q_t, int format_t,
                              reft_stream stream)
{
    const char *who = "reft_transpose";
    NEED(is_eight(format) && is_eight(format_t), REFT_EINVAL, "%s: unknown 8-bit format", who);
    NEED(rows <= 0x7fffffff && cols <= 0x7fffffff, REFT_ESIZE, "%s: too many rows or columns", who);
    CHECK_EIGHT(who, q, rows, cols);
    CHECK_EIGHT(who, q_t, cols, rows);
    if (!rows || !cols) return REFT_OK;
    NEED(given(q) && given(q_t), REFT_EINVAL, "%s: null pointer", who);
    NEED((rows + 127) / 128 * ((cols + 127) / 128) <= kMaxTiles, REFT_ESIZE, "%s: too many values", who);
    if ((uintptr_t)stream == kCheckOnly) return REFT_OK;
    TransposeArgs a;
    a.q = in_of(q);
    a.q_t = out_of(q_t);
    a.rows = rows;
    a.cols = cols;
    a.band = kTransposeBand;
    a.e5m2 = format == REFT_E5M2;
    a.e5m2_t = format_t == REFT_E5M2;
    const uint32_t grid = (uint32_t)((rows + 127) / 128 * ((cols + 127) / 128));
    hipStream_t s = (hipStream_t)stream;
    if (!near(q->ld) || !near(q_t->ld)) k_transpose<false, uint64_t><<<grid, kTileThreads, 0, s>>>(a);
    else if (lines_of(a.q_t)) k_transpose<true, uint32_t><<<grid, kTileThreads, 0, s>>>(a);
    else k_transpose<false, uint32_t><<<grid, kTileThreads, 0, s>>>(a);
    return launched(who, hipGetLastError());
}
