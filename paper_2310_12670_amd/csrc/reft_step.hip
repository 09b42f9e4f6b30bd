// Operators of a training step that read and write each value once: dropout, root-mean-square norm with the
// residual's addition (forward, backward), quantization to 8 bits.  Kernels and their entry points (see include/reft.h).
#include "reft_calls.hpp"

#include <algorithm>
#include <cmath>
#include <cstring>

namespace reft {

// ------------------------------------------------------------------------------------------------
// dropout
// ------------------------------------------------------------------------------------------------
struct DropoutArgs {
    const void *x;
    void *y;
    uint64_t ld_x, ld_y;
    uint64_t cols, groups, total;  // groups of eight columns in a row, and in the matrix
    uint32_t inverse;              // floor(2^32 / groups)
    Dropout d;
};

constexpr int kDropUnroll = 4;

// y = keep ? x s : 0.  A thread takes kDropUnroll groups.  Row and group of a block's first come of one division of whole numbers,
// those of its threads of a multiplication.  Bound by HBM: 16384 x 11008 in bf16 114 us, 6.3 TB/s, and as much without a mask, so that
// the generator's ten rounds cost nothing.
template <typename T, bool STREAM> __global__ __launch_bounds__(256) void k_dropout(DropoutArgs a)
{
    const uint64_t first = (uint64_t)blockIdx.x * (256 * kDropUnroll);
    const uint64_t row0 = first / a.groups;
    const uint32_t rem = (uint32_t)(first - row0 * a.groups), groups = (uint32_t)a.groups;
    float v[kDropUnroll][8];
    uint32_t row[kDropUnroll], group[kDropUnroll];
    int n[kDropUnroll];
#pragma unroll
    for (int u = 0; u < kDropUnroll; ++u) {
        const uint32_t local = u * 256 + threadIdx.x, at = rem + local;
        uint32_t r = __umulhi(at, a.inverse);
        if (at - r * groups >= groups) ++r;                 // the rounded inverse may be one row short
        row[u] = (uint32_t)row0 + r;
        group[u] = at - r * groups;
        const uint64_t left = a.cols - (uint64_t)group[u] * 8;
        n[u] = first + local < a.total ? (int)(left < 8 ? left : 8) : 0;
        load8<STREAM>((const T *)a.x + (uint64_t)row[u] * a.ld_x + (uint64_t)group[u] * 8, n[u], v[u]);
    }
#pragma unroll
    for (int u = 0; u < kDropUnroll; ++u) {
        if (a.d.threshold) drop8(a.d, row[u], group[u], v[u]);
        store8((T *)a.y + (uint64_t)row[u] * a.ld_y + (uint64_t)group[u] * 8, n[u], v[u]);
    }
}

// ------------------------------------------------------------------------------------------------
// norm
// ------------------------------------------------------------------------------------------------
struct NormForward {
    const void *x, *residual, *weight;
    uint64_t ld_x, ld_r;
    uint32_t first, rows, cols;    // rows first .. rows - 1
    float eps;
    Dropout d;
    void *h;
    uint64_t ld_h;
    float *rstd;
    void *y;
    uint64_t ld_y;
    uint8_t *q;
    uint64_t ld_q;
    uint8_t *scales;
    uint64_t ld_s;
    uint8_t e5m2, weight_f32;
};

__device__ __forceinline__ float wave_sum(float v)
{
    v = sum_of_16(v);
    v += __shfl_xor(v, 16);
    return v + __shfl_xor(v, 32);
}

// The sum over a row's waves, added in their order.  room: a place for each wave of the block; all of the block calls.
__device__ __forceinline__ float row_sum(float v, float *room)
{
    const int waves = blockDim.x / 64;
    v = wave_sum(v);
    if (waves == 1) return v;
    float *mine = room + threadIdx.y * waves;
    if ((threadIdx.x & 63) == 0) mine[threadIdx.x / 64] = v;
    __syncthreads();
    v = 0;
    for (int i = 0; i < waves; ++i) v += mine[i];
    return v;
}

// h = residual + dropout(x), h / rms(h) weight, in 8 bits too.  A row belongs to the threads of one y (64 to 1024 of them); each holds V times eight neighbouring columns of it in registers: one
// pass over the inputs whatever the row's length.  A wave's 512 columns are four blocks of 128, 16 lanes each: one word of scales.
// Bound by HBM: 16384 x 5120 in bf16 with an fp32 residual and 8-bit output 161 us, 5.7 TB/s; one row of 8192 3.2 us.  (Fewer, wider waves:
// 171 us; blocks that loop over rows with the next one in flight: 201; reading past the L2: 173.)
template <typename T, typename R, int V> __global__ __launch_bounds__(1024) void k_norm_forward(NormForward a)
{
    __shared__ float room[16];
    const int lane = threadIdx.x & 63, first = threadIdx.x * 8, wide = blockDim.x * 8, cols = (int)a.cols;
    const uint32_t row = a.first + blockIdx.x * blockDim.y + threadIdx.y;
    const bool there = row < a.rows;
    constexpr bool kAhead = V <= 2;                          // all is asked for at once, as far as registers go
    Eight<T> x[V];
    Eight<R> r[V];
    float h[V][8], w[V][8], sum = 0;
    auto fetch = [&](int v) {
        const int c = first + v * wide, n = there ? cols - c : 0;
        x[v].template load<false>((const T *)a.x + row * a.ld_x + c, n);
        r[v].template load<false>((const R *)a.residual + row * a.ld_r + c, a.residual ? n : 0);
        if (kAhead) load8_of<T>(a.weight, a.weight_f32, c, a.weight ? n : 0, w[v]);
    };
    if (kAhead)
#pragma unroll
        for (int v = 0; v < V; ++v) fetch(v);
#pragma unroll
    for (int v = 0; v < V; ++v) {
        if (!kAhead) fetch(v);
        const int c = first + v * wide, n = there ? cols - c : 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) h[v][i] = x[v][i];
        if (a.d.threshold) drop8(a.d, row, (uint32_t)c / 8, h[v]);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            h[v][i] += r[v][i];
            sum += h[v][i] * h[v][i];
        }
        if (a.h) store8((R *)a.h + row * a.ld_h + c, n, h[v]);
    }
    const float rstd = 1.f / sqrtf(row_sum(sum, room) / (float)cols + a.eps);
    if (!there) return;
    if (a.rstd && threadIdx.x == 0) a.rstd[row] = rstd;
    if (!a.y && !a.q) return;
#pragma unroll
    for (int v = 0; v < V; ++v) {
        const int c = first + v * wide;
        if (!kAhead) load8_of<T>(a.weight, a.weight_f32, c, cols - c, w[v]);
#pragma unroll
        for (int i = 0; i < 8; ++i) w[v][i] *= h[v][i] * rstd;
        if (a.y) store8((T *)a.y + row * a.ld_y + c, cols - c, w[v]);
        if (a.q) {
            uint32_t most = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) most = max(most, magnitude(w[v][i]));
            const uint32_t e = scale_of(max_of_16(most), top_of(a.e5m2));
            store8_bytes<true>(a.q + row * a.ld_q + c, cols - c, to_eight(w[v], inverse_of(e), a.e5m2));
            const int word = c / 512;                       // the same in the whole wave
            if ((lane & 15) == 0 && word * 512 < cols)
                a.scales[(word * a.ld_s + row) * 4 + lane / 16] = c < cols ? (uint8_t)e : 127;
        }
    }
}

struct NormBackward {
    const void *dy, *dh, *h, *weight;
    const float *rstd;
    uint64_t ld_dy, ld_dh, ld_h;
    uint32_t rows, cols;
    Dropout d;
    void *dres, *dx;
    uint64_t ld_dres, ld_dx;
    float *part;                   // [blocks][cols]
    uint8_t weight_f32;
};

// Rows as above.  A block takes every so manyth row (or, of short rows, blockDim.y of them) and keeps its part of the weight's
// gradient in registers; k_sum_parts adds the blocks' parts in their order.  Of rows with eight columns a lane the next one is fetched
// while one is worked on; of wider ones the operands are read again for the second half of the work (from the L2) rather than held.
// Bound by HBM: 16384 x 8192 in bf16 with residual 228 us, 5.9 TB/s.
template <typename T, typename R, int V, bool STREAM> __global__ __launch_bounds__(1024) void k_norm_backward(NormBackward a)
{
    __shared__ float room[2][16];
    __shared__ float fold[V == 1 ? 3 * 512 : 1];
    const int first = threadIdx.x * 8, wide = blockDim.x * 8, cols = (int)a.cols;
    const uint32_t step = gridDim.x * blockDim.y;
    float dw[V][8] = {}, w[V][8];
#pragma unroll
    for (int v = 0; v < V; ++v) load8_of<T>(a.weight, a.weight_f32, first + v * wide, cols - first - v * wide, w[v]);
    Eight<T> dy[V], next_dy;
    Eight<R> h[V], dh[V], next_h, next_dh;
    float rstd, next_rstd;
    auto fetch = [&](int v, uint32_t row) {
        const int c = first + v * wide, n = row < a.rows ? cols - c : 0;
        h[v].template load<false>((const R *)a.h + row * a.ld_h + c, n);
        dy[v].template load<false>((const T *)a.dy + row * a.ld_dy + c, n);
    };
    auto fetch_dh = [&](int v, uint32_t row) {
        const int c = first + v * wide, n = row < a.rows ? cols - c : 0;
        dh[v].template load<false>((const R *)a.dh + row * a.ld_dh + c, a.dh ? n : 0);
    };
    auto fetch_next = [&](uint32_t row) {
        const int n = row < a.rows ? cols - first : 0;
        next_h.template load<STREAM>((const R *)a.h + row * a.ld_h + first, n);
        next_dy.template load<STREAM>((const T *)a.dy + row * a.ld_dy + first, n);
        next_dh.template load<STREAM>((const R *)a.dh + row * a.ld_dh + first, a.dh ? n : 0);
        next_rstd = row < a.rows ? a.rstd[row] : 0.f;
    };
    if (V == 1) fetch_next(blockIdx.x * blockDim.y + threadIdx.y);
    int half = 0;
    for (uint32_t base = blockIdx.x * blockDim.y; base < a.rows; base += step, half ^= 1) {
        const uint32_t row = base + threadIdx.y;
        const bool there = row < a.rows;
        float dot = 0;
        if (V == 1) {
            h[0] = next_h;
            dy[0] = next_dy;
            dh[0] = next_dh;
            rstd = next_rstd;
            if (base + step < a.rows) fetch_next(row + step);
        } else {
            rstd = there ? a.rstd[row] : 0.f;
        }
#pragma unroll
        for (int v = 0; v < V; ++v) {
            if (V > 1) fetch(v, row);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float part = dy[v][i] * (h[v][i] * rstd);
                dw[v][i] += part;
                dot += part * w[v][i];
            }
        }
        dot = row_sum(dot, room[half]) / (float)cols;        // this half is written again two rows on, behind another barrier
        if (!there) continue;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int c = first + v * wide;
            float o[8];
            if (V > 1) fetch(v, row), fetch_dh(v, row);
#pragma unroll
            for (int i = 0; i < 8; ++i) o[i] = dh[v][i] + rstd * (dy[v][i] * w[v][i] - h[v][i] * rstd * dot);
            if (a.dres) store8((R *)a.dres + row * a.ld_dres + c, cols - c, o);
            if (a.dx) {
                if (a.d.threshold) drop8(a.d, row, (uint32_t)c / 8, o);
                store8((T *)a.dx + row * a.ld_dx + c, cols - c, o);
            }
        }
    }
    if (!a.part) return;
    if (V == 1 && blockDim.y > 1) {                          // (64, 4) or (128, 2) threads: at most 3 times 512 sums to fold
        if (threadIdx.y > 0)
#pragma unroll
            for (int i = 0; i < 8; ++i) fold[(threadIdx.y - 1) * wide + first + i] = dw[0][i];
        __syncthreads();
        if (threadIdx.y > 0) return;
        for (uint32_t y = 1; y < blockDim.y; ++y)
#pragma unroll
            for (int i = 0; i < 8; ++i) dw[0][i] += fold[(y - 1) * wide + first + i];
    }
#pragma unroll
    for (int v = 0; v < V; ++v) {
        const int c = first + v * wide;
        store8(a.part + (uint64_t)blockIdx.x * a.cols + c, cols - c, dw[v]);
    }
}

// Rows of more than 16384 columns: nothing is held, the operands are read again for the second half (from the L2), and the weight's
// gradient, which would take all registers, is k_weight_parts'.  4096 x 65536 in bf16:
// 787 us with that, 3.4 TB/s of what has to move (1821 with all sums in registers, which spill).
template <typename T, typename R> __global__ __launch_bounds__(1024) void k_norm_backward_wide(NormBackward a)
{
    __shared__ float room[2][16];
    const int cols = (int)a.cols;
    int half = 0;
    for (uint32_t row = blockIdx.x; row < a.rows; row += gridDim.x, half ^= 1) {
        const R *h_row = (const R *)a.h + row * a.ld_h, *dh_row = (const R *)a.dh + row * a.ld_dh;
        const T *dy_row = (const T *)a.dy + row * a.ld_dy;
        const float rstd = a.rstd[row];
        float dot = 0;
#pragma unroll 2
        for (int c = threadIdx.x * 8; c < cols; c += blockDim.x * 8) {
            float h[8], dy[8], w[8];
            load8<false>(h_row + c, cols - c, h);
            load8<false>(dy_row + c, cols - c, dy);
            load8_of<T>(a.weight, a.weight_f32, c, cols - c, w);
#pragma unroll
            for (int i = 0; i < 8; ++i) dot += dy[i] * (h[i] * rstd) * w[i];
        }
        dot = row_sum(dot, room[half]) / (float)cols;
        for (int c = threadIdx.x * 8; c < cols; c += blockDim.x * 8) {
            float h[8], dy[8], w[8], o[8];
            load8<false>(h_row + c, cols - c, h);
            load8<false>(dy_row + c, cols - c, dy);
            load8<false>(dh_row + c, a.dh ? cols - c : 0, o);
            load8_of<T>(a.weight, a.weight_f32, c, cols - c, w);
#pragma unroll
            for (int i = 0; i < 8; ++i) o[i] += rstd * (dy[i] * w[i] - h[i] * rstd * dot);
            if (a.dres) store8((R *)a.dres + row * a.ld_dres + c, cols - c, o);
            if (a.dx) {
                if (a.d.threshold) drop8(a.d, row, (uint32_t)c / 8, o);
                store8((T *)a.dx + row * a.ld_dx + c, cols - c, o);
            }
        }
    }
}

// The weight's gradient alone: a block takes 512 columns and, with each of its four waves, every so manyth row.
template <typename T, typename R> __global__ __launch_bounds__(256) void k_weight_parts(NormBackward a)
{
    __shared__ float fold[3][512];
    const int c = blockIdx.x * 512 + threadIdx.x * 8, n = (int)a.cols - c;
    float dw[8] = {};
#pragma unroll 2
    for (uint32_t row = blockIdx.y * 4 + threadIdx.y; row < a.rows; row += gridDim.y * 4) {
        const float rstd = a.rstd[row];
        float h[8], dy[8];
        load8<false>((const R *)a.h + row * a.ld_h + c, n, h);
        load8<false>((const T *)a.dy + row * a.ld_dy + c, n, dy);
#pragma unroll
        for (int i = 0; i < 8; ++i) dw[i] += dy[i] * (h[i] * rstd);
    }
    if (threadIdx.y > 0)
#pragma unroll
        for (int i = 0; i < 8; ++i) fold[threadIdx.y - 1][threadIdx.x * 8 + i] = dw[i];
    __syncthreads();
    if (threadIdx.y > 0) return;
#pragma unroll
    for (int y = 0; y < 3; ++y)
#pragma unroll
        for (int i = 0; i < 8; ++i) dw[i] += fold[y][threadIdx.x * 8 + i];
    store8(a.part + (uint64_t)blockIdx.y * a.cols + c, n, dw);
}

// out[c] = sum of n rows of part, in an order that depends on n alone: 64 interleaved sums, then those one after the other.
// 256 parts of 8192 columns: 5.3 us.
__global__ __launch_bounds__(1024) void k_sum_parts(const float *part, uint32_t n, uint32_t cols, float *out)
{
    __shared__ float sums[64][16];
    const uint32_t x = threadIdx.x & 15, y = threadIdx.x >> 4, c = blockIdx.x * 16 + x;
    float s = 0;
    if (c < cols)
#pragma unroll 4
        for (uint32_t i = y; i < n; i += 64) s += part[(uint64_t)i * cols + c];
    sums[y][x] = s;
    __syncthreads();
    if (y == 0 && c < cols) {
        for (int i = 1; i < 64; ++i) s += sums[i][x];
        out[c] = s;
    }
}

// ------------------------------------------------------------------------------------------------
// quantization
// ------------------------------------------------------------------------------------------------
struct QuantizeArgs {
    const void *x;
    uint64_t ld_x, rows, cols;
    uint8_t *q, *scales, *q_t, *scales_t;
    uint64_t ld_q, ld_s, ld_qt, ld_st;
    uint8_t e5m2;
};

// A scale for each 128 columns of a row: a wave takes 512 columns of a row, 16 lanes each block.  Bound by HBM: 16384 x 8192 in bf16 77 us,
// 5.3 TB/s.
template <typename T> __global__ __launch_bounds__(256) void k_quantize_rows(QuantizeArgs a)
{
    const int lane = threadIdx.x & 63;
    const uint64_t row = (uint64_t)blockIdx.x * 4 + (threadIdx.x >> 6), c = (uint64_t)blockIdx.y * 512 + lane * 8;
    if (row >= a.rows) return;
    const int n = c >= a.cols ? 0 : (int)min(a.cols - c, (uint64_t)8);
    float v[8];
    load8<false>((const T *)a.x + row * a.ld_x + c, n, v);
    uint32_t most = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) most = max(most, magnitude(v[i]));
    const uint32_t e = scale_of(max_of_16(most), top_of(a.e5m2));
    store8_bytes<true>(a.q + row * a.ld_q + c, n, to_eight(v, inverse_of(e), a.e5m2));
    if ((lane & 15) == 0) a.scales[((uint64_t)blockIdx.y * a.ld_s + row) * 4 + lane / 16] = n ? (uint8_t)e : 127;
}

// A tile of 128 x 128 values, in registers: a thread holds 8 rows of 8 columns, so that each of its columns is 8 bytes of
// the transpose, which leaves through LDS in whole rows.  BLOCKS: one scale for the tile, else one for each row and, in the
// transpose, for each column.  LINES: the results' rows lie on cache lines, which a tile then writes whole.  Bound by HBM where large:
// 3584 x 8192 in bf16, blocks and both orders, 19.4 us, 6.0 TB/s (31 with values widened once and held in fp32).
template <typename T, bool BLOCKS, bool LINES> __global__ __launch_bounds__(256) void k_quantize_tile(QuantizeArgs a)
{
    // LDS bytes of eight columns of 128 rows.  The pitch is eight banks, so that of 16 lanes' writes those four apart meet: 12 cycles of
    // conflicts a write (3584 x 8192: 688128 in 57344 writes), beside what bounds the kernel.
    constexpr int kPitch = 1024 + 32;
    __shared__ __align__(16) uint8_t tile[16 * kPitch];
    __shared__ uint32_t most_of[4][128];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, tc = tid & 15, tr = tid >> 4;
    const uint32_t high = (uint32_t)((a.rows + 127) / 128), wide = (uint32_t)((a.cols + 127) / 128);
    const uint32_t down = blockIdx.x / wide, along = blockIdx.x % wide;
    const uint64_t row0 = (uint64_t)down * 128, col0 = (uint64_t)along * 128;
    const int rows = (int)min(a.rows - row0, (uint64_t)128), cols = (int)min(a.cols - col0, (uint64_t)128);
    Eight<T> v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i)
        v[i].template load<false>((const T *)a.x + (row0 + tr * 8 + i) * a.ld_x + col0 + tc * 8, tr * 8 + i < rows ? cols - tc * 8 : 0);
    // The values are widened anew for each use: as they lie they take half the registers.
    auto forget = [&]() {
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
            for (int k = 0; k < (int)sizeof(T) / 2; ++k) asm volatile("" : "+v"(v[i].w[k]));
    };
    const int top = top_of(a.e5m2);
    uint32_t by_col[8] = {};
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) by_col[j] = max(by_col[j], magnitude(v[i][j]));
    forget();
    uint32_t e_tile = 0;
    if constexpr (BLOCKS) {
        uint32_t m = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) m = max(m, by_col[j]);
        m = max_of_16(m);
        m = max(m, (uint32_t)__shfl_xor((int)m, 16));
        m = max(m, (uint32_t)__shfl_xor((int)m, 32));
        if (lane == 0) most_of[wave][0] = m;
        __syncthreads();
        e_tile = scale_of(max(max(most_of[0][0], most_of[1][0]), max(most_of[2][0], most_of[3][0])), top);
        if (tid == 0) {
            if (a.q) store_scale(a.scales, a.ld_s, down, along, wide, e_tile);
            if (a.q_t) store_scale(a.scales_t, a.ld_st, along, down, high, e_tile);
        }
    } else if (a.q_t) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            by_col[j] = max(by_col[j], (uint32_t)__shfl_xor((int)by_col[j], 16));
            by_col[j] = max(by_col[j], (uint32_t)__shfl_xor((int)by_col[j], 32));
            if (lane < 16) most_of[wave][tc * 8 + j] = by_col[j];
        }
    }
    if (a.q) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            uint32_t e = e_tile;
            const int r = tr * 8 + i;
            float t[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) t[j] = v[i][j];
            if constexpr (!BLOCKS) {
                uint32_t m = 0;
#pragma unroll
                for (int j = 0; j < 8; ++j) m = max(m, magnitude(t[j]));
                e = scale_of(max_of_16(m), top);
                if (tc == 0 && r < rows) store_scale(a.scales, a.ld_s, row0 + r, along, wide, e);
            }
            if (r < rows) store8_bytes<LINES>(a.q + (row0 + r) * a.ld_q + col0 + tc * 8, cols - tc * 8, to_eight(t, inverse_of(e), a.e5m2));
        }
    }
    if (!a.q_t) return;
    if constexpr (!BLOCKS) __syncthreads();
    forget();
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        uint32_t e = e_tile;
        const int c = tc * 8 + j;
        if constexpr (!BLOCKS) {
            e = scale_of(max(max(most_of[0][c], most_of[1][c]), max(most_of[2][c], most_of[3][c])), top);
            if (tr == 0 && c < cols) store_scale(a.scales_t, a.ld_st, col0 + c, down, high, e);
        }
        float t[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) t[i] = v[i][j];
        *(w32x2 *)(tile + tc * kPitch + j * 128 + tr * 8) = to_eight(t, inverse_of(e), a.e5m2);
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const int c = (tid >> 3) + 32 * k, r = (tid & 7) * 16;
        if (c >= cols || r >= rows) continue;
        const w32x4 w = *(const w32x4 *)(tile + (c / 8) * kPitch + (c % 8) * 128 + r);
        uint8_t *p = a.q_t + (col0 + c) * a.ld_qt + row0 + r;
        if (r + 16 <= rows) {
            if constexpr (LINES) __builtin_nontemporal_store(w, (w32x4_any *)p);
            else *(w32x4_any *)p = w;
        } else {
            for (int i = 0; i < rows - r; ++i) p[i] = tile[(c / 8) * kPitch + (c % 8) * 128 + r + i];
        }
    }
}

// ------------------------------------------------------------------------------------------------
// which kernel
// ------------------------------------------------------------------------------------------------
// Rows on cache lines (on_lines) are read past the L2.  (Gradient of 16384 x 8192 in bf16: 241 us kept, 227 not; dropout of 16384 x 11008: 120
// and 115.  Of other rows each line is read twice: dropout of 4096 x 5003 in fp32 31 and 38, of 16384 x 1155 16.8 and 19.7.)
template <typename T> static void launch_dropout(const DropoutArgs &a, bool lines, uint32_t blocks, hipStream_t s)
{
    if (lines) k_dropout<T, true><<<blocks, 256, 0, s>>>(a);
    else k_dropout<T, false><<<blocks, 256, 0, s>>>(a);
}

// A row's threads: as many waves as its columns fill with eight a lane, up to 16, then up to eight times eight a lane.
constexpr uint64_t kMaxCols = 65536;
constexpr uint32_t kRowsALaunch = 1u << 21;            // a grid has less than 2^32 threads, a row up to 1024
static dim3 row_threads(uint64_t cols, int v)
{
    const uint32_t waves = (uint32_t)((cols + 512 * v - 1) / (512 * v));
    return dim3(64 * waves, waves == 1 ? 4 : waves == 2 ? 2 : 1);
}
static int row_registers(uint64_t cols) { return cols <= 8192 ? 1 : cols <= 16384 ? 2 : cols <= 32768 ? 4 : 8; }

// The gradient's blocks: what the 256 compute units hold at once, at up to 16 waves each (its registers allow no more), or 12 where
// rows may lie on cache lines and fewer waves keep the memory busy.  With 16, 12 and 8 waves, us in bf16: 16384 x 2048 69, 64 and 62,
// x 5120 179 (two rounds), 152 and 152, x 1155 79, 94 and 111.  Sums are taken in an order of the sizes alone, and the
// workspace goes by them too: so a number of columns that makes whole lines of dense rows in 16 bits stands for the alignment, which is not
// looked at.  A block that has one row, where there are places for all, leaves a part as long as the row in fp32.
static uint32_t blocks_of(uint64_t rows, uint64_t cols)
{
    if (row_registers(cols) > 2) return (uint32_t)std::min<uint64_t>((rows + 3) / 4, 32);
    const dim3 t = row_threads(cols, row_registers(cols));
    const uint32_t waves = t.x * t.y / 64, room = cols % 64 ? 16 : 12;
    if (rows <= 4 * t.y) return rows ? 1 : 0;                // one block is done before a second launch would be
    return (uint32_t)std::min<uint64_t>((rows + t.y - 1) / t.y, 256 * std::max(1u, room / waves));
}

template <typename T, typename R> static hipError_t launch_forward(NormForward a, hipStream_t s)
{
    const int v = row_registers(a.cols);
    const dim3 threads = row_threads(a.cols, v);
    const uint32_t rows = a.rows;
    for (uint32_t first = 0; first < rows; first += kRowsALaunch) {
        const uint32_t n = std::min(rows - first, kRowsALaunch), grid = (n + threads.y - 1) / threads.y;
        a.first = first;
        a.rows = first + n;
        if (v == 1) k_norm_forward<T, R, 1><<<grid, threads, 0, s>>>(a);
        else if (v == 2) k_norm_forward<T, R, 2><<<grid, threads, 0, s>>>(a);
        else if (v == 4) k_norm_forward<T, R, 4><<<grid, threads, 0, s>>>(a);
        else k_norm_forward<T, R, 8><<<grid, threads, 0, s>>>(a);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

template <typename T, typename R> static hipError_t launch_backward(const NormBackward &a, uint32_t blocks, hipStream_t s)
{
    const int v = row_registers(a.cols);
    const dim3 threads = row_threads(a.cols, v);
    const bool lines = on_lines(a.dy, a.ld_dy * sizeof(T)) && on_lines(a.h, a.ld_h * sizeof(R)) && on_lines(a.dh, a.ld_dh * sizeof(R));
    if (v == 1 && lines) k_norm_backward<T, R, 1, true><<<blocks, threads, 0, s>>>(a);
    else if (v == 1) k_norm_backward<T, R, 1, false><<<blocks, threads, 0, s>>>(a);
    else if (v == 2) k_norm_backward<T, R, 2, false><<<blocks, threads, 0, s>>>(a);
    else {
        // the weight's gradient first: the others may take the place of what it reads
        if (a.part) k_weight_parts<T, R><<<dim3((a.cols + 511) / 512, blocks), dim3(64, 4), 0, s>>>(a);
        if (a.dres || a.dx) k_norm_backward_wide<T, R><<<std::min(a.rows, 512u), 1024, 0, s>>>(a);
    }
    return hipGetLastError();
}

// p in [0, 1] as a threshold of 65536; false if it is none.
static bool make_dropout(double p, uint64_t seed, uint64_t offset, Dropout *d)
{
    if (!(p >= 0 && p <= 1)) return false;
    const long t = (long)std::nearbyint(p * 65536);         // ties to even
    d->key0 = (uint32_t)seed;
    d->key1 = (uint32_t)(seed >> 32);
    d->off0 = (uint32_t)offset;
    d->off1 = (uint32_t)(offset >> 32);
    d->threshold = (uint32_t)t;
    d->scale = t >= 65536 ? 0.f : (float)(65536.0 / (double)(65536 - t));
    return true;
}

}  // namespace reft

using namespace reft;

extern "C" int reft_dropout(const void *x, uint64_t ld_x, void *y, uint64_t ld_y, uint64_t rows, uint64_t cols, int dtype,
                            double p, uint64_t seed, uint64_t offset, reft_stream stream)
{
    DropoutArgs a;
    NEED(is_float_type(dtype), REFT_EINVAL, "reft_dropout: unknown type %d", dtype);
    NEED(make_dropout(p, seed, offset, &a.d), REFT_EINVAL, "reft_dropout: p is not within [0, 1]");
    NEED(rows <= 0x7fffffff && cols <= 0x7fffffff, REFT_ESIZE, "reft_dropout: too many rows or columns");
    NEED(ld_x >= cols && ld_y >= cols, REFT_ESIZE, "reft_dropout: rows overlap");
    if (!rows || !cols) return REFT_OK;
    NEED(x && y, REFT_EINVAL, "reft_dropout: null pointer");
    NEED(lies(x, size_of(dtype)) && lies(y, size_of(dtype)), REFT_EINVAL, "reft_dropout: misaligned pointer");
    a.x = x;
    a.y = y;
    a.ld_x = ld_x;
    a.ld_y = ld_y;
    a.cols = cols;
    a.groups = (cols + 7) / 8;
    a.total = a.groups * rows;
    a.inverse = (uint32_t)std::min<uint64_t>((1ull << 32) / a.groups, 0xffffffffu);
    const uint64_t blocks = (a.total + 256 * kDropUnroll - 1) / (256 * kDropUnroll);
    NEED(blocks <= kMaxBlocks256, REFT_ESIZE, "reft_dropout: too many values");
    if ((uintptr_t)stream == kCheckOnly) return REFT_OK;
    hipStream_t s = (hipStream_t)stream;
    const bool lines = on_lines(x, ld_x * size_of(dtype));
    if (dtype == REFT_F32) launch_dropout<float>(a, lines, (uint32_t)blocks, s);
    else if (dtype == REFT_BF16) launch_dropout<bf16>(a, lines, (uint32_t)blocks, s);
    else launch_dropout<f16>(a, lines, (uint32_t)blocks, s);
    return launched("reft_dropout", hipGetLastError());
}

extern "C" int reft_norm_forward(const void *x, uint64_t ld_x, const void *residual, uint64_t ld_r, const void *weight,
                                 uint64_t rows, uint64_t cols, int dtype, int residual_dtype, int weight_dtype, double eps,
                                 double p, uint64_t seed, uint64_t offset, void *h, uint64_t ld_h, float *rstd, void *y,
                                 uint64_t ld_y, void *q, uint64_t ld_q, int format, void *scales, uint64_t ld_s,
                                 reft_stream stream)
{
    NormForward a;
    NEED(is_float_type(dtype), REFT_EINVAL, "reft_norm_forward: unknown type %d", dtype);
    NEED(residual_dtype == dtype || residual_dtype == REFT_F32, REFT_EINVAL,
         "reft_norm_forward: the residual has the type of x or fp32");
    NEED(weight_dtype == dtype || weight_dtype == REFT_F32, REFT_EINVAL, "reft_norm_forward: the weight has the type of x or fp32");
    NEED(eps >= 0 && eps <= 1e30, REFT_EINVAL, "reft_norm_forward: eps is negative or no number");
    NEED(make_dropout(p, seed, offset, &a.d), REFT_EINVAL, "reft_norm_forward: p is not within [0, 1]");
    NEED(cols >= 1 && cols <= kMaxCols, REFT_ESIZE, "reft_norm_forward: rows have 1 to %llu columns", (unsigned long long)kMaxCols);
    NEED(rows <= 0x7fffffff, REFT_ESIZE, "reft_norm_forward: too many rows");
    NEED(ld_x >= cols && (!residual || ld_r >= cols) && (!h || ld_h >= cols) && (!y || ld_y >= cols) && (!q || ld_q >= cols),
         REFT_ESIZE, "reft_norm_forward: rows overlap");
    NEED(h || rstd || y || q || !rows, REFT_EINVAL, "reft_norm_forward: no output");
    if (q) {
        NEED(is_eight(format), REFT_EINVAL, "reft_norm_forward: unknown 8-bit format %d", format);
        NEED(scales || !rows, REFT_EINVAL, "reft_norm_forward: 8 bits without scales");
        NEED(ld_s >= rows, REFT_ESIZE, "reft_norm_forward: words of scales overlap");
    }
    if (!rows) return REFT_OK;
    NEED(x && (weight || (!y && !q)), REFT_EINVAL, "reft_norm_forward: null pointer");
    NEED(lies(x, size_of(dtype)) && lies(y, size_of(dtype)) && lies(residual, size_of(residual_dtype)) &&
             lies(h, size_of(residual_dtype)) && lies(weight, size_of(weight_dtype)) && lies(rstd, 4),
         REFT_EINVAL, "reft_norm_forward: misaligned pointer");
    if ((uintptr_t)stream == kCheckOnly) return REFT_OK;
    a.x = x;
    a.residual = residual;
    a.weight = weight;
    a.ld_x = ld_x;
    a.ld_r = ld_r;
    a.rows = (uint32_t)rows;
    a.cols = (uint32_t)cols;
    a.eps = (float)eps;
    a.h = h;
    a.ld_h = ld_h;
    a.rstd = rstd;
    a.y = y;
    a.ld_y = ld_y;
    a.q = (uint8_t *)q;
    a.ld_q = ld_q;
    a.scales = (uint8_t *)scales;
    a.ld_s = ld_s;
    a.e5m2 = format == REFT_E5M2;
    a.weight_f32 = weight_dtype == REFT_F32;
    hipStream_t s = (hipStream_t)stream;
    const bool wide = residual_dtype == REFT_F32;
    return launched("reft_norm_forward", dtype == REFT_F32    ? launch_forward<float, float>(a, s)
                                         : dtype == REFT_BF16 ? (wide ? launch_forward<bf16, float>(a, s) : launch_forward<bf16, bf16>(a, s))
                                                              : (wide ? launch_forward<f16, float>(a, s) : launch_forward<f16, f16>(a, s)));
}

extern "C" uint64_t reft_norm_backward_workspace(uint64_t rows, uint64_t cols)
{
    if (rows <= 1 || !cols || cols > kMaxCols) return 0;
    return (uint64_t)blocks_of(rows, cols) * cols * sizeof(float);
}

extern "C" int reft_norm_backward(const void *dy, uint64_t ld_dy, const void *dh, uint64_t ld_dh, const void *h, uint64_t ld_h,
                                  const float *rstd, const void *weight, uint64_t rows, uint64_t cols, int dtype,
                                  int residual_dtype, int weight_dtype, double p, uint64_t seed, uint64_t offset, void *dres,
                                  uint64_t ld_dres, void *dx, uint64_t ld_dx, float *dweight, void *workspace,
                                  uint64_t workspace_bytes, reft_stream stream)
{
    NormBackward a;
    NEED(is_float_type(dtype), REFT_EINVAL, "reft_norm_backward: unknown type %d", dtype);
    NEED(residual_dtype == dtype || residual_dtype == REFT_F32, REFT_EINVAL,
         "reft_norm_backward: the residual has the type of dy or fp32");
    NEED(weight_dtype == dtype || weight_dtype == REFT_F32, REFT_EINVAL, "reft_norm_backward: the weight has the type of dy or fp32");
    NEED(make_dropout(p, seed, offset, &a.d), REFT_EINVAL, "reft_norm_backward: p is not within [0, 1]");
    NEED(cols >= 1 && cols <= kMaxCols, REFT_ESIZE, "reft_norm_backward: rows have 1 to %llu columns", (unsigned long long)kMaxCols);
    NEED(rows <= 0x7fffffff, REFT_ESIZE, "reft_norm_backward: too many rows");
    NEED((!rows || ld_dy >= cols) && (!dh || ld_dh >= cols) && (!rows || ld_h >= cols) && (!dres || ld_dres >= cols) && (!dx || ld_dx >= cols),
         REFT_ESIZE, "reft_norm_backward: rows overlap");
    NEED(dres || dx || dweight || !rows, REFT_EINVAL, "reft_norm_backward: no output");
    hipStream_t s = (hipStream_t)stream;
    const uint32_t blocks = blocks_of(rows, cols);
    if (dweight) {
        NEED(lies(dweight, 4), REFT_EINVAL, "reft_norm_backward: misaligned pointer");
        if (rows > 1) {
            NEED(workspace && lies(workspace, 16), REFT_EINVAL, "reft_norm_backward: no workspace, or not on 16 bytes");
            NEED(workspace_bytes >= reft_norm_backward_workspace(rows, cols), REFT_ESIZE, "reft_norm_backward: workspace too small");
        }
    }
    if (!rows) {
        if ((uintptr_t)stream == kCheckOnly) return REFT_OK;
        if (dweight) k_sum_parts<<<(uint32_t)((cols + 15) / 16), 1024, 0, s>>>(nullptr, 0, (uint32_t)cols, dweight);
        return launched("reft_norm_backward", hipGetLastError());
    }
    NEED(dy && h && rstd && weight, REFT_EINVAL, "reft_norm_backward: null pointer");
    NEED(lies(dy, size_of(dtype)) && lies(dx, size_of(dtype)) && lies(dh, size_of(residual_dtype)) && lies(h, size_of(residual_dtype)) &&
             lies(dres, size_of(residual_dtype)) && lies(weight, size_of(weight_dtype)) && lies(rstd, 4),
         REFT_EINVAL, "reft_norm_backward: misaligned pointer");
    if ((uintptr_t)stream == kCheckOnly) return REFT_OK;
    a.dy = dy;
    a.dh = dh;
    a.h = h;
    a.weight = weight;
    a.rstd = rstd;
    a.ld_dy = ld_dy;
    a.ld_dh = ld_dh;
    a.ld_h = ld_h;
    a.rows = (uint32_t)rows;
    a.cols = (uint32_t)cols;
    a.dres = dres;
    a.dx = dx;
    a.ld_dres = ld_dres;
    a.ld_dx = ld_dx;
    a.part = !dweight ? nullptr : blocks > 1 ? (float *)workspace : dweight;
    a.weight_f32 = weight_dtype == REFT_F32;
    const bool wide = residual_dtype == REFT_F32;
    hipError_t e = dtype == REFT_F32    ? launch_backward<float, float>(a, blocks, s)
                   : dtype == REFT_BF16 ? (wide ? launch_backward<bf16, float>(a, blocks, s) : launch_backward<bf16, bf16>(a, blocks, s))
                                        : (wide ? launch_backward<f16, float>(a, blocks, s) : launch_backward<f16, f16>(a, blocks, s));
    if (e == hipSuccess && dweight && blocks > 1) {
        k_sum_parts<<<(uint32_t)((cols + 15) / 16), 1024, 0, s>>>((const float *)workspace, blocks, a.cols, dweight);
        e = hipGetLastError();
    }
    return launched("reft_norm_backward", e);
}

template <typename T> static hipError_t launch_quantize(const QuantizeArgs &a, bool blocks, hipStream_t s)
{
    if (!blocks && !a.q_t && (a.rows + 3) / 4 <= kMaxBlocks256) {
        k_quantize_rows<T><<<dim3((uint32_t)((a.rows + 3) / 4), (uint32_t)((a.cols + 511) / 512)), 256, 0, s>>>(a);
    } else {
        // tile after tile of a row of tiles (down the columns first: 16384 x 8192 116 -> 150 us)
        const uint32_t grid = (uint32_t)((a.cols + 127) / 128 * ((a.rows + 127) / 128));
        // (lines that tiles share are joined in the L2: 4099 x 4101 36 us past it, 25 through it)
        const bool lines = (!a.q || on_lines(a.q, a.ld_q)) && (!a.q_t || on_lines(a.q_t, a.ld_qt));
        if (blocks && lines) k_quantize_tile<T, true, true><<<grid, 256, 0, s>>>(a);
        else if (blocks) k_quantize_tile<T, true, false><<<grid, 256, 0, s>>>(a);
        else if (lines) k_quantize_tile<T, false, true><<<grid, 256, 0, s>>>(a);
        else k_quantize_tile<T, false, false><<<grid, 256, 0, s>>>(a);
    }
    return hipGetLastError();
}

extern "C" int reft_quantize(const void *x, uint64_t ld_x, uint64_t rows, uint64_t cols, int dtype, int format, int blocks, void *q,
                             uint64_t ld_q, void *scales, uint64_t ld_s, void *q_t, uint64_t ld_qt, void *scales_t,
                             uint64_t ld_st, reft_stream stream)
{
    QuantizeArgs a;
    NEED(is_float_type(dtype), REFT_EINVAL, "reft_quantize: unknown type %d", dtype);
    NEED(is_eight(format), REFT_EINVAL, "reft_quantize: unknown 8-bit format %d", format);
    NEED(q || q_t || !rows || !cols, REFT_EINVAL, "reft_quantize: no output");
    NEED((!q || scales || !rows || !cols) && (!q_t || scales_t || !rows || !cols), REFT_EINVAL, "reft_quantize: 8 bits without scales");
    // the grid counts tiles, or, in its second dimension, words of columns
    NEED(rows < (1u << 26) && cols <= 128 * 65535, REFT_ESIZE, "reft_quantize: too many rows or columns");
    NEED(ld_x >= cols && (!q || ld_q >= cols) && (!q_t || ld_qt >= rows), REFT_ESIZE, "reft_quantize: rows overlap");
    NEED((!q || ld_s >= (blocks ? (rows + 127) / 128 : rows)) && (!q_t || ld_st >= (blocks ? (cols + 127) / 128 : cols)),
         REFT_ESIZE, "reft_quantize: words of scales overlap");
    if (!rows || !cols) return REFT_OK;
    NEED((rows + 127) / 128 * ((cols + 127) / 128) <= kMaxBlocks256, REFT_ESIZE, "reft_quantize: too many values");
    NEED(x, REFT_EINVAL, "reft_quantize: null pointer");
    NEED(lies(x, size_of(dtype)), REFT_EINVAL, "reft_quantize: misaligned pointer");
    if ((uintptr_t)stream == kCheckOnly) return REFT_OK;
    a.x = x;
    a.ld_x = ld_x;
    a.rows = rows;
    a.cols = cols;
    a.q = (uint8_t *)q;
    a.scales = (uint8_t *)scales;
    a.q_t = (uint8_t *)q_t;
    a.scales_t = (uint8_t *)scales_t;
    a.ld_q = ld_q;
    a.ld_s = ld_s;
    a.ld_qt = ld_qt;
    a.ld_st = ld_st;
    a.e5m2 = format == REFT_E5M2;
    hipStream_t s = (hipStream_t)stream;
    return launched("reft_quantize", dtype == REFT_F32    ? launch_quantize<float>(a, blocks, s)
                                     : dtype == REFT_BF16 ? launch_quantize<bf16>(a, blocks, s)
                                                          : launch_quantize<f16>(a, blocks, s));
}
