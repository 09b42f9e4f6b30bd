// Operators between the products of a feed-forward trained in 8 bits: the activation with what it keeps, its gradient from that, and the
// transpose of what is kept.  Kernels and their entry points (see include/reft.h).
#include "reft_calls.hpp"

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
// forward
// ------------------------------------------------------------------------------------------------
struct GateForward {
    const void *g, *u;
    uint64_t ld_g, ld_u, rows, cols;
    void *y;
    uint64_t ld_y;
    EightOut y8, g8, u8;
    uint8_t y_e5m2, kept_e5m2;
};

// Eight of a row's values in 8 bits with the power of two of the 16 lanes' 128.
__device__ __forceinline__ void leave_row(const EightOut &o, const float v[8], uint64_t row, uint64_t c, int n, bool e5m2)
{
    uint32_t most = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) most = max(most, magnitude(v[i]));
    const uint32_t e = scale_of(max_of_16(most), top_of(e5m2));
    store8_bytes<true>(o.q + row * o.ld + c, n, to_eight(v, inverse_of(e), e5m2));
    if ((threadIdx.x & 15) == 0) o.scales[(c / 512 * o.ld_s + row) * 4 + c / 128 % 4] = n ? (uint8_t)e : 127;
}

// A wave takes 512 columns of a row, 16 lanes each block of 128.
template <typename T, int ACT> __global__ __launch_bounds__(256) void k_gate_forward(GateForward a)
{
    const uint64_t row = (uint64_t)blockIdx.x * 4 + (threadIdx.x >> 6), c = (uint64_t)blockIdx.y * 512 + (threadIdx.x & 63) * 8;
    if (row >= a.rows) return;
    const int n = c >= a.cols ? 0 : (int)min(a.cols - c, (uint64_t)8);
    float g[8], u[8], y[8], slope;
    load8<false>((const T *)a.g + row * a.ld_g + c, n, g);
    if (a.u) load8<false>((const T *)a.u + row * a.ld_u + c, n, u);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        act<ACT>(g[i], &y[i], &slope);
        if (a.u) y[i] *= u[i];
    }
    if (a.y) store8((T *)a.y + row * a.ld_y + c, n, y);
    if (a.y8.q) leave_row(a.y8, y, row, c, n, a.y_e5m2);
    if (a.g8.q) leave_row(a.g8, g, row, c, n, a.kept_e5m2);
    if (a.u8.q) leave_row(a.u8, u, row, c, n, a.kept_e5m2);
}

// ------------------------------------------------------------------------------------------------
// backward, and the transpose: tiles of 128 x 128 values, a thread holds 4 rows of 8 columns
// ------------------------------------------------------------------------------------------------
struct Tile {
    uint64_t row0, col0;
    uint32_t down, along, high, wide;                       // number of the tile, and of tiles
    int rows, cols;                                         // of the matrix in it
};

__device__ __forceinline__ Tile tile_of(uint32_t number, uint64_t rows, uint64_t cols)
{
    Tile t;
    t.high = (uint32_t)((rows + 127) / 128);
    t.wide = (uint32_t)((cols + 127) / 128);
    t.down = number / t.wide;
    t.along = number % t.wide;
    t.row0 = (uint64_t)t.down * 128;
    t.col0 = (uint64_t)t.along * 128;
    t.rows = (int)min(rows - t.row0, (uint64_t)128);
    t.cols = (int)min(cols - t.col0, (uint64_t)128);
    return t;
}

// The factor that a scale byte stands for: 2^(e - 127), and a NaN for 255.
__device__ __forceinline__ float factor_of(uint32_t e)
{
    return __uint_as_float(e == 255 ? 0x7fc00000u : e ? e << 23 : 0x00400000u);
}

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

__device__ __forceinline__ void widen8(w32x2 w, bool e5m2, float factor, float v[8])
{
    f32x2 p[4];
    if (e5m2) {
        p[0] = __builtin_amdgcn_cvt_pk_f32_bf8((int)w.x, false);
        p[1] = __builtin_amdgcn_cvt_pk_f32_bf8((int)w.x, true);
        p[2] = __builtin_amdgcn_cvt_pk_f32_bf8((int)w.y, false);
        p[3] = __builtin_amdgcn_cvt_pk_f32_bf8((int)w.y, true);
    } else {
        p[0] = __builtin_amdgcn_cvt_pk_f32_fp8((int)w.x, false);
        p[1] = __builtin_amdgcn_cvt_pk_f32_fp8((int)w.x, true);
        p[2] = __builtin_amdgcn_cvt_pk_f32_fp8((int)w.y, false);
        p[3] = __builtin_amdgcn_cvt_pk_f32_fp8((int)w.y, true);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[2 * i] = p[i].x * factor;
        v[2 * i + 1] = p[i].y * factor;
    }
}

// Four values in 8 bits, to nearest even.
__device__ __forceinline__ uint32_t to_four(const float v[4], float inv, bool e5m2)
{
    int w = 0;
    if (e5m2) {
        w = __builtin_amdgcn_cvt_pk_bf8_f32(v[0] * inv, v[1] * inv, w, false);
        w = __builtin_amdgcn_cvt_pk_bf8_f32(v[2] * inv, v[3] * inv, w, true);
    } else {
        w = __builtin_amdgcn_cvt_pk_fp8_f32(v[0] * inv, v[1] * inv, w, false);
        w = __builtin_amdgcn_cvt_pk_fp8_f32(v[2] * inv, v[3] * inv, w, true);
    }
    return (uint32_t)w;
}

constexpr int kTileThreads = 512;

// A thread's place in the tile.
struct Place {
    int c, r;                                               // its first column and row
    __device__ __forceinline__ Place() : c((threadIdx.x & 15) * 8), r((threadIdx.x >> 4) * 4) {}
};

struct Turn {
    // LDS bytes of eight columns of 128 rows, and four banks more: no two of a wave's words, eight columns and four rows apart, meet.
    static constexpr int kPitch = 1024 + 16;
    __align__(16) uint8_t tile[16 * kPitch];
    uint32_t most[kTileThreads / 64][128];
};

// The tile's transpose in 8 bits with a power of two for each of its columns, through LDS, in whole rows.
__device__ __forceinline__ void leave_turned(const EightOut &o, const float (&v)[4][8], const Tile &t, bool e5m2, Turn &lds)
{
    const Place at;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    __syncthreads();                                        // what was here before has been read
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        uint32_t m = max(max(magnitude(v[0][j]), magnitude(v[1][j])), max(magnitude(v[2][j]), magnitude(v[3][j])));
        m = max(m, (uint32_t)__shfl_xor((int)m, 16));
        m = max(m, (uint32_t)__shfl_xor((int)m, 32));
        if (lane < 16) lds.most[wave][at.c + j] = m;
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        uint32_t m = 0;
#pragma unroll
        for (int w = 0; w < kTileThreads / 64; ++w) m = max(m, lds.most[w][at.c + j]);
        const uint32_t e = scale_of(m, top_of(e5m2));
        if (at.r == 0 && at.c + j < t.cols) store_scale(o.scales, o.ld_s, t.col0 + at.c + j, t.down, t.high, e);
        const float four[4] = {v[0][j], v[1][j], v[2][j], v[3][j]};
        *(uint32_t *)(lds.tile + at.c / 8 * Turn::kPitch + j * 128 + at.r) = to_four(four, inverse_of(e), e5m2);
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const int c = (threadIdx.x >> 3) + 64 * k, r = (threadIdx.x & 7) * 16;
        if (c >= t.cols || r >= t.rows) continue;
        const uint8_t *from = lds.tile + c / 8 * Turn::kPitch + c % 8 * 128 + r;
        uint8_t *to = o.q + (t.col0 + c) * o.ld + t.row0 + r;
        if (r + 16 <= t.rows) *(w32x4_any *)to = *(const w32x4 *)from;
        else
            for (int i = 0; i < t.rows - r; ++i) to[i] = from[i];
    }
}

// A thread's rows in 8 bits with a power of two for each row of the tile.
__device__ __forceinline__ void leave_rows(const EightOut &o, const float (&v)[4][8], const Tile &t, bool e5m2)
{
    const Place at;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        uint32_t m = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) m = max(m, magnitude(v[i][j]));
        const uint32_t e = scale_of(max_of_16(m), top_of(e5m2));
        if (at.r + i >= t.rows) continue;
        if (at.c == 0) store_scale(o.scales, o.ld_s, t.row0 + at.r + i, t.along, t.wide, e);
        store8_bytes<false>(o.q + (t.row0 + at.r + i) * o.ld + t.col0 + at.c, t.cols - at.c, to_eight(v[i], inverse_of(e), e5m2));
    }
}

__device__ __forceinline__ float factor_at(const EightIn &x, const Tile &t, int r)
{
    return factor_of(x.scales[(t.along / 4 * x.ld_s + t.row0 + r) * 4 + t.along % 4]);
}

struct GateBackward {
    const void *dy;
    uint64_t ld_dy, rows, cols;
    EightIn g8, u8;
    void *dg, *du;
    uint64_t ld_dg, ld_du;
    EightOut dg8, du8, dg8_t, du8_t, y8_t;
    uint8_t kept_e5m2, grad_e5m2, y_e5m2;
};

template <typename T, int ACT> __global__ __launch_bounds__(kTileThreads) void k_gate_backward(GateBackward a)
{
    __shared__ Turn lds;
    const Tile t = tile_of(blockIdx.x, a.rows, a.cols);
    const Place at;
    float dg[4][8], du[4][8], y[4][8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int r = at.r + i, n = r < t.rows ? t.cols - at.c : 0;
        const uint64_t row = t.row0 + r, col = t.col0 + at.c;
        float dy[8], g[8], u[8];
        load8<false>((const T *)a.dy + row * a.ld_dy + col, n, dy);
        widen8(load8_bytes(a.g8.q + row * a.g8.ld + col, n), a.kept_e5m2, n > 0 ? factor_at(a.g8, t, r) : 0.f, g);
        if (a.u8.q) widen8(load8_bytes(a.u8.q + row * a.u8.ld + col, n), a.kept_e5m2, n > 0 ? factor_at(a.u8, t, r) : 0.f, u);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            float v, slope;
            act<ACT>(g[j], &v, &slope);
            const float by_u = a.u8.q ? u[j] : 1.f;
            dg[i][j] = dy[j] * by_u * slope;
            du[i][j] = dy[j] * v;
            y[i][j] = v * by_u;
        }
        if (a.dg) store8((T *)a.dg + row * a.ld_dg + col, n, dg[i]);
        if (a.du) store8((T *)a.du + row * a.ld_du + col, n, du[i]);
    }
    if (a.dg8.q) leave_rows(a.dg8, dg, t, a.grad_e5m2);
    if (a.du8.q) leave_rows(a.du8, du, t, a.grad_e5m2);
    if (a.dg8_t.q) leave_turned(a.dg8_t, dg, t, a.grad_e5m2, lds);
    if (a.du8_t.q) leave_turned(a.du8_t, du, t, a.grad_e5m2, lds);
    if (a.y8_t.q) leave_turned(a.y8_t, y, t, a.y_e5m2, lds);
}

struct TransposeArgs {
    EightIn q;
    EightOut q_t;
    uint64_t rows, cols;
    uint8_t e5m2, e5m2_t;
};

__global__ __launch_bounds__(kTileThreads) void k_transpose(TransposeArgs a)
{
    __shared__ Turn lds;
    const Tile t = tile_of(blockIdx.x, a.rows, a.cols);
    const Place at;
    float v[4][8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int r = at.r + i, n = r < t.rows ? t.cols - at.c : 0;
        widen8(load8_bytes(a.q.q + (t.row0 + r) * a.q.ld + t.col0 + at.c, n), a.e5m2, n > 0 ? factor_at(a.q, t, r) : 0.f, v[i]);
    }
    leave_turned(a.q_t, v, t, a.e5m2_t, lds);
}

// ------------------------------------------------------------------------------------------------
// which kernel
// ------------------------------------------------------------------------------------------------
template <typename T> static hipError_t launch_forward(const GateForward &a, int kind, hipStream_t s)
{
    const dim3 grid((uint32_t)((a.rows + 3) / 4), (uint32_t)((a.cols + 511) / 512));
    if (kind == REFT_SILU) k_gate_forward<T, REFT_SILU><<<grid, 256, 0, s>>>(a);
    else if (kind == REFT_GELU) k_gate_forward<T, REFT_GELU><<<grid, 256, 0, s>>>(a);
    else if (kind == REFT_GELU_TANH) k_gate_forward<T, REFT_GELU_TANH><<<grid, 256, 0, s>>>(a);
    else k_gate_forward<T, REFT_RELU2><<<grid, 256, 0, s>>>(a);
    return hipGetLastError();
}

template <typename T> static hipError_t launch_backward(const GateBackward &a, int kind, hipStream_t s)
{
    const uint32_t grid = (uint32_t)((a.rows + 127) / 128 * ((a.cols + 127) / 128));
    if (kind == REFT_SILU) k_gate_backward<T, REFT_SILU><<<grid, kTileThreads, 0, s>>>(a);
    else if (kind == REFT_GELU) k_gate_backward<T, REFT_GELU><<<grid, kTileThreads, 0, s>>>(a);
    else if (kind == REFT_GELU_TANH) k_gate_backward<T, REFT_GELU_TANH><<<grid, kTileThreads, 0, s>>>(a);
    else k_gate_backward<T, REFT_RELU2><<<grid, kTileThreads, 0, s>>>(a);
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
    NEED(rows <= 0x7fffffff && cols <= 128 * 65535, REFT_ESIZE, "%s: too many rows or columns", who);
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
    NEED((rows + 3) / 4 * ((cols + 511) / 512) <= kMaxBlocks256, REFT_ESIZE, "%s: too many values", who);
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
    a.ld_dg = ld_dg;
    a.ld_du = ld_du;
    a.dg8 = out_of(dg8);
    a.du8 = out_of(du8);
    a.dg8_t = out_of(dg8_t);
    a.du8_t = out_of(du8_t);
    a.y8_t = out_of(y8_t);
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
    a.e5m2 = format == REFT_E5M2;
    a.e5m2_t = format_t == REFT_E5M2;
    k_transpose<<<(uint32_t)((rows + 127) / 128 * ((cols + 127) / 128)), kTileThreads, 0, (hipStream_t)stream>>>(a);
    return launched(who, hipGetLastError());
}
