// Norm of queries and keys for each head, with the rotation by the row's position, and the gradients of both.  Kernels and their entry
// points (see include/reft.h).
#include "reft_calls.hpp"

#include <algorithm>

namespace reft {

// One kind of heads: inputs, outputs, weight.
struct Side {
    const void *x, *dy, *weight;
    void *out;
    uint64_t row_x, head_x, row_dy, head_dy, row_out, head_out;
    uint32_t heads;
};

struct HeadsArgs {
    Side side[2];                  // queries, keys
    const int64_t *positions;
    const float *freqs;
    uint64_t rows;
    uint32_t cols, pairs;
    float eps;
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

// The column that column c turns with, and which pair that is; c itself and none (-1) behind the pairs.
__device__ __forceinline__ int partner_of(int c, int pairs, bool adjacent, int *pair)
{
    *pair = -1;
    if (c >= 2 * pairs) return c;
    *pair = adjacent ? c / 2 : c < pairs ? c : c - pairs;
    return adjacent ? c ^ 1 : c < pairs ? c + pairs : c - pairs;
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

template <typename T> __device__ __forceinline__ float weight_at(const HeadsArgs &a, const Side &s, int c)
{
    return !s.weight ? 1.f : a.weight_f32 ? ((const float *)s.weight)[c] : widen(((const T *)s.weight)[c]);
}

// A head belongs to G lanes with eight columns each.
template <typename T, int G> __global__ __launch_bounds__(256) void k_heads_forward(HeadsArgs a)
{
    const int cols = (int)a.cols, c0 = (threadIdx.x % G) * 8, n = cols - c0;
    const uint64_t all = a.side[0].heads + a.side[1].heads, total = a.rows * all;
    for (uint64_t unit = (uint64_t)blockIdx.x * (256 / G) + threadIdx.x / G; unit < total; unit += (uint64_t)gridDim.x * (256 / G)) {
        const uint64_t row = unit / all;
        const uint32_t number = (uint32_t)(unit % all);
        const Side &s = a.side[number >= a.side[0].heads];
        const uint32_t head = number >= a.side[0].heads ? number - a.side[0].heads : number;
        const T *x = (const T *)s.x + row * s.row_x + head * s.head_x;
        float v[8], other[8], sum = 0;
        load8<false>(x + c0, n, v);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            int pair;
            const int c = min(c0 + i, cols - 1), p = partner_of(c, a.pairs, a.adjacent, &pair);
            other[i] = widen(x[p]);
            sum += v[i] * v[i];
        }
        const float r = 1.f / sqrtf(sum_of<G>(sum) / (float)cols + a.eps);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            int pair;
            const int c = min(c0 + i, cols - 1), p = partner_of(c, a.pairs, a.adjacent, &pair);
            float sine = 0, cosine = 1;
            if (pair >= 0) sine_cosine(a.positions[row], a.freqs[pair], &sine, &cosine);
            v[i] = v[i] * r * weight_at<T>(a, s, c) * cosine + (p > c ? -sine : sine) * (other[i] * r * weight_at<T>(a, s, p));
        }
        store8((T *)s.out + row * s.row_out + head * s.head_out + c0, n, v);
    }
}

// The same for the gradients; a group of lanes sums its heads' part of the weights' gradients, the block adds its groups' in their order.
template <typename T, int G> __global__ __launch_bounds__(256) void k_heads_backward(HeadsArgs a)
{
    __shared__ float fold[256 / G][G * 8];
    const int cols = (int)a.cols, c0 = (threadIdx.x % G) * 8, n = cols - c0, group = threadIdx.x / G;
    const uint64_t all = a.side[0].heads + a.side[1].heads, total = a.rows * all;
    float dw[2][8] = {};
    for (uint64_t unit = (uint64_t)blockIdx.x * (256 / G) + group; unit < total; unit += (uint64_t)gridDim.x * (256 / G)) {
        const uint64_t row = unit / all;
        const uint32_t number = (uint32_t)(unit % all);
        const bool key = number >= a.side[0].heads;
        const Side &s = a.side[key];
        const uint32_t head = key ? number - a.side[0].heads : number;
        const T *dy = (const T *)s.dy + row * s.row_dy + head * s.head_dy;
        float x[8], t[8], w[8], sum = 0, dot = 0;
        load8<false>((const T *)s.x + row * s.row_x + head * s.head_x + c0, n, x);
        load8<false>(dy + c0, n, t);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            int pair;
            const int c = min(c0 + i, cols - 1), p = partner_of(c, a.pairs, a.adjacent, &pair);
            float sine = 0, cosine = 1;
            if (pair >= 0) sine_cosine(a.positions[row], a.freqs[pair], &sine, &cosine);
            t[i] = t[i] * cosine + (p > c ? sine : -sine) * widen(dy[p]);
            w[i] = weight_at<T>(a, s, c);
            sum += x[i] * x[i];
            dot += x[i] * (t[i] * w[i]);
        }
        const float r = 1.f / sqrtf(sum_of<G>(sum) / (float)cols + a.eps);
        dot = r * (sum_of<G>(dot) / (float)cols);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float xhat = x[i] * r;
            if (key) dw[1][i] += i < n ? t[i] * xhat : 0.f;
            else dw[0][i] += i < n ? t[i] * xhat : 0.f;
            t[i] = r * (t[i] * w[i] - xhat * dot);
        }
        if (s.out) store8((T *)s.out + row * s.row_out + head * s.head_out + c0, n, t);
    }
    if (!a.part) return;
    for (int kind = 0; kind < 2; ++kind) {
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 8; ++i) fold[group][c0 + i] = dw[kind][i];
        __syncthreads();
        for (int c = threadIdx.x; c < cols; c += 256) {
            float s = 0;
            for (int g = 0; g < 256 / G; ++g) s += fold[g][c];
            a.part[((uint64_t)blockIdx.x * 2 + kind) * cols + c] = s;
        }
    }
}

// The weights' gradients: the blocks' parts in an order of their number alone, 16 interleaved sums and then those one after the other.
__global__ __launch_bounds__(256) void k_heads_weights(const float *part, uint32_t n, uint32_t cols, float *dq, float *dk)
{
    __shared__ float sums[16][16];
    const uint32_t x = threadIdx.x & 15, y = threadIdx.x >> 4, at = blockIdx.x * 16 + x;
    float s = 0;
    if (at < 2 * cols)
        for (uint32_t i = y; i < n; i += 16) s += part[(uint64_t)i * 2 * cols + at];
    sums[y][x] = s;
    __syncthreads();
    if (y > 0 || at >= 2 * cols) return;
    for (int i = 1; i < 16; ++i) s += sums[i][x];
    float *out = at < cols ? dq : dk;
    if (out) out[at < cols ? at : at - cols] = s;
}

// ------------------------------------------------------------------------------------------------
// which kernel
// ------------------------------------------------------------------------------------------------
constexpr uint64_t kMaxHeadCols = 512;
static int lanes_of(uint64_t cols) { return cols <= 64 ? 8 : cols <= 128 ? 16 : cols <= 256 ? 32 : 64; }

// As many blocks as the chip holds at once.
static uint32_t heads_blocks(uint64_t rows, uint64_t heads, uint64_t cols)
{
    const uint64_t groups = 256 / lanes_of(cols);
    return (uint32_t)std::min<uint64_t>((rows * heads + groups - 1) / groups, 2048);
}

template <typename T> static hipError_t launch_forward(const HeadsArgs &a, hipStream_t s)
{
    const uint64_t heads = a.side[0].heads + a.side[1].heads;
    const uint32_t grid = heads_blocks(a.rows, heads, a.cols);
    switch (lanes_of(a.cols)) {
    case 8: k_heads_forward<T, 8><<<grid, 256, 0, s>>>(a); break;
    case 16: k_heads_forward<T, 16><<<grid, 256, 0, s>>>(a); break;
    case 32: k_heads_forward<T, 32><<<grid, 256, 0, s>>>(a); break;
    default: k_heads_forward<T, 64><<<grid, 256, 0, s>>>(a);
    }
    return hipGetLastError();
}

template <typename T> static hipError_t launch_backward(const HeadsArgs &a, uint32_t grid, hipStream_t s)
{
    switch (lanes_of(a.cols)) {
    case 8: k_heads_backward<T, 8><<<grid, 256, 0, s>>>(a); break;
    case 16: k_heads_backward<T, 16><<<grid, 256, 0, s>>>(a); break;
    case 32: k_heads_backward<T, 32><<<grid, 256, 0, s>>>(a); break;
    default: k_heads_backward<T, 64><<<grid, 256, 0, s>>>(a);
    }
    return hipGetLastError();
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
    a.adjacent = adjacent != 0;
    a.weight_f32 = weight_dtype == REFT_F32;
    return a;
}

static Side side_of(const reft_heads *x, uint64_t heads, const void *weight, const reft_heads *dy, const reft_heads *out)
{
    Side s = {};
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
    a.side[0] = side_of(q, q_heads, q_weight, nullptr, q_out);
    if (k) a.side[1] = side_of(k, k_heads, k_weight, nullptr, k_out);
    hipStream_t s = (hipStream_t)stream;
    return launched(who, dtype == REFT_F32    ? launch_forward<float>(a, s)
                         : dtype == REFT_BF16 ? launch_forward<bf16>(a, s)
                                              : launch_forward<f16>(a, s));
}

extern "C" uint64_t reft_heads_backward_workspace(uint64_t rows, uint64_t q_heads, uint64_t k_heads, uint64_t cols)
{
    if (!rows || !cols || cols > kMaxHeadCols || rows > 0x7fffffff || q_heads > 65535 || k_heads > 65535) return 0;
    return (uint64_t)heads_blocks(rows, q_heads + k_heads, cols) * 2 * cols * sizeof(float);
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
    const uint32_t grid = rows ? heads_blocks(rows, q_heads + (k ? k_heads : 0), cols) : 0;
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
        a.side[0] = side_of(q, q_heads, q_weight, dq_out, dq);
        if (k) a.side[1] = side_of(k, k_heads, k_weight, dk_out, dk);
        a.part = sums ? (float *)workspace : nullptr;
        e = dtype == REFT_F32    ? launch_backward<float>(a, grid, s)
            : dtype == REFT_BF16 ? launch_backward<bf16>(a, grid, s)
                                 : launch_backward<f16>(a, grid, s);
    }
    if (e == hipSuccess && sums) {
        k_heads_weights<<<(uint32_t)((2 * cols + 15) / 16), 256, 0, s>>>((const float *)workspace, grid, (uint32_t)cols, dq_weight, dk_weight);
        e = hipGetLastError();
    }
    return launched(who, e);
}
