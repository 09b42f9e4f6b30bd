// Matrix product in 8-bit floating point with a power of two for each block of 128, on the matrix cores.
#include "reft_step.hpp"

#include <algorithm>

namespace reft {

typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

struct ProductArgs {
    const uint8_t *a, *b;          // [M][ld_a], [N][ld_b], K values of a row count
    const uint32_t *sa, *sb;       // [ceil(K / 512)][ld_sa], [..][ld_sb]: words of four blocks' scales
    uint64_t ld_a, ld_b, ld_sa, ld_sb, ld_c;
    uint32_t M, N, K;
    uint32_t b_shift;              // row n of b has scale n >> b_shift: 7 for blocks of 128 rows, else 0
    void *c;
    int c_type;
    uint32_t splits, split_steps;  // parts that K is cut into, and steps of 128 to a part (a multiple of 4)
    float *parts;                  // [splits][M][N] where there are several
};

// ---- tiles in LDS -----------------------------------------------------------------------------------------
// A row of a tile is 128 values of K: eight chunks of 16 bytes.  Chunk c of row r lies at place c ^ turn(r), so that
// neither 8 nor 16 rows that are read at one chunk meet in a bank.  Rows 16 apart are turned alike: their addresses differ by a
// constant.
__device__ __forceinline__ int turn(int r) { return (r ^ (r >> 3 & 1)) & 7; }
__device__ __forceinline__ int place(int r, int c) { return r * 128 + ((c ^ turn(r)) << 4); }

// A lane's operand of a product of 32 x 32 x 64: row lane % 32 of those from `row` (a multiple of 32) on, 32 values of
// half s of the row's 128.  Which of a half's 64 values a lane takes is the same for both operands, and the scale is the same for all.
__device__ __forceinline__ i32x8 operand(const uint8_t *tile, int row, int s, int lane)
{
    const int c = s * 4 + (lane >> 5) * 2;
    tile += row * 128;
    const w32x4 lo = *(const w32x4 *)(tile + place(lane & 31, c)), hi = *(const w32x4 *)(tile + place(lane & 31, c + 1));
    i32x8 v;
    v[0] = lo.x; v[1] = lo.y; v[2] = lo.z; v[3] = lo.w;
    v[4] = hi.x; v[5] = hi.y; v[6] = hi.z; v[7] = hi.w;
    return v;
}

// What the matrix cores multiply.  Their 8-bit products apply the scales for nothing and run at 4.5 PFLOP/s (a loop of
// independent ones), but add in fewer bits than fp32: of eight products of neighbouring k, each is cut (towards zero) where it lies
// 2^13 below the power of two of the largest one, and one further down is lost; the sums of eight are then added in fp32.  Measured, of
// normal numbers the root-mean-square error is 1.5e-5 of the result's at every K from 16 to 8192; at worst it is 7 2^-13 times
// the sum over the eights of their largest products.  Adding up outside of the matrix cores would not help, as the loss is within an
// eight.  A bf16 result's own rounding, 2^-8 of it (1.7e-3 of the norm), covers that, and takes the fast ones.  That of an f16 result,
// 2^-11, does not: where the result is f16 or fp32 (EXACT), the values are turned into bf16, which holds 8 bits times a power of
// two exactly, as long as they lie between its smallest numbers, multiples of 2^-133, and 2^128, and are multiplied at 2.2 PFLOP/s: there the cut
// lies 2^24 below the largest, with an error of 8e-8.  (us in bf16 and f16: 1 x 11008 x 4096 11.6 and 13.0, 1001 x 5120 x 1728 17.2 and
// 25.1, 8192 x 28672 x 8192 1317 and 2546.)
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

template <int F, bool EXACT> struct Operand;
template <int F> struct Operand<F, false> {
    i32x8 v;
    uint32_t scale;
    __device__ __forceinline__ void take(i32x8 bytes, uint32_t e) { v = bytes, scale = e; }
};
template <int F> struct Operand<F, true> {
    bf16x8 v[4];
    __device__ __forceinline__ void take(i32x8 bytes, uint32_t e)
    {
        e &= 255;
        const float f = __uint_as_float(e == 0 ? 0x00400000u : e == 255 ? 0x7fc00000u : e << 23);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const bf16x2 lo = F ? __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(bytes[i], f, false)
                                : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(bytes[i], f, false);
            const bf16x2 hi = F ? __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(bytes[i], f, true)
                                : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(bytes[i], f, true);
            v[i / 2][i % 2 * 4] = lo.x, v[i / 2][i % 2 * 4 + 1] = lo.y;
            v[i / 2][i % 2 * 4 + 2] = hi.x, v[i / 2][i % 2 * 4 + 3] = hi.y;
        }
    }
};

// acc[n][m] += scales * b[n][k] a[m][k]: the transposed product, so that a lane ends up with neighbouring columns of C.
template <int FA, int FB>
__device__ __forceinline__ f32x16 multiply(const Operand<FB, false> &b, const Operand<FA, false> &a, f32x16 acc)
{
    return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(b.v, a.v, acc, FB, FA, 0, (int)b.scale, 0, (int)a.scale);
}
template <int FA, int FB>
__device__ __forceinline__ f32x16 multiply(const Operand<FB, true> &b, const Operand<FA, true> &a, f32x16 acc)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(b.v[i], a.v[i], acc, 0, 0, 0);
    return acc;
}

// 16 bytes at p, of which the first n exist; the others are zero.
__device__ __forceinline__ w32x4 load16(const uint8_t *p, int n)
{
    if (n >= 16) return *(const w32x4_any *)p;
    w32x4 w = {0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < 16; ++i)
        if (i < n) w[i / 4] |= (uint32_t)p[i] << (8 * (i & 3));
    return w;
}

__device__ __forceinline__ void store1(const ProductArgs &p, uint64_t at, float v)
{
    if (p.c_type == REFT_F32) ((float *)p.c)[at] = v;
    else if (p.c_type == REFT_BF16) ((bf16 *)p.c)[at] = narrow<bf16>(v);
    else ((f16 *)p.c)[at] = narrow<f16>(v);
}

// Four neighbouring columns of a row of C, of which the first n exist.
__device__ __forceinline__ void store4(const ProductArgs &p, uint64_t at, int n, const float v[4])
{
    if (n <= 0) return;
    if (p.c_type == REFT_F32) {
        float *c = (float *)p.c + at;
        if (n >= 4) *(w32x4_any *)c = w32x4{__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])};
        else for (int i = 0; i < n; ++i) c[i] = v[i];
        return;
    }
    uint16_t t[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) t[i] = p.c_type == REFT_BF16 ? narrow<bf16>(v[i]).bits : narrow<f16>(v[i]).bits;
    uint16_t *c = (uint16_t *)p.c + at;
    if (n >= 4) *(w32x2_any *)c = w32x2{t[0] | (uint32_t)t[1] << 16, t[2] | (uint32_t)t[3] << 16};
    else for (int i = 0; i < n; ++i) c[i] = t[i];
}

// One row block of 32 x 32 results: lane holds column m = lane % 32 of the transposed tile and, of each eight rows n,
// four neighbouring ones.
__device__ __forceinline__ void store_tile(const ProductArgs &p, uint32_t m, uint32_t n0, int lane, f32x16 acc)
{
    if (m >= p.M) return;
#pragma unroll
    for (int g = 0; g < 4; ++g) {
        const uint32_t n = n0 + 8 * g + 4 * (lane >> 5);
        const float v[4] = {acc[4 * g], acc[4 * g + 1], acc[4 * g + 2], acc[4 * g + 3]};
        store4(p, m * p.ld_c + n, n < p.N ? (int)min(p.N - n, 4u) : 0, v);
    }
}

// ---- any sizes, any alignment: tiles of 128 x 128, four waves of 64 x 64 -----------------------------------------
// The next tile is loaded to registers while one is multiplied, and then written to LDS: what 16-byte copies to LDS need of alignment,
// this does not.  8192 x 4096 x 4096 to bf16: 277 us, where rows on 16 bytes take 111; 128 x 4096 x 11008, cut into 8 parts, 29 and 20.  K is multiplied in the order of k_product and cut
// into the same parts, so that where and how far apart the rows lie does not change a bit of the result.
template <int FA, int FB, bool EXACT> __global__ __launch_bounds__(256) void k_product_any(ProductArgs p)
{
    __shared__ __align__(16) uint8_t tile[2][2][128 * 128];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const uint32_t m0 = blockIdx.y * 128, n0 = blockIdx.x * 128;
    const int wm = (wave & 1) * 64, wn = (wave >> 1) * 64;
    const uint32_t all = (p.K + 127) / 128, start = blockIdx.z * p.split_steps;
    const uint32_t steps = p.splits > 1 ? min(all - start, p.split_steps) : all;        // no part is empty
    w32x4 next[2][4];
    auto load = [&](uint32_t step) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int r = (tid >> 3) + 32 * i;
            const uint32_t k = (start + step) * 128 + (tid & 7) * 16;
            const int n = k < p.K ? (int)min(p.K - k, 16u) : 0;
            next[0][i] = load16(p.a + (m0 + r) * p.ld_a + k, m0 + r < p.M ? n : 0);
            next[1][i] = load16(p.b + (n0 + r) * p.ld_b + k, n0 + r < p.N ? n : 0);
        }
    };
    auto keep = [&](int half) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int r = (tid >> 3) + 32 * i;
            *(w32x4 *)(tile[half][0] + place(r, tid & 7)) = next[0][i];
            *(w32x4 *)(tile[half][1] + place(r, tid & 7)) = next[1][i];
        }
    };
    f32x16 acc[2][2] = {};
    uint32_t sa[2] = {}, sb[2] = {};
    if (steps) {
        load(0);
        keep(0);
    }
    for (uint32_t step = 0; step < steps; ++step) {
        __syncthreads();
        const int half = step & 1;
        if (step + 1 < steps) load(step + 1);
        if (step % 4 == 0) {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                sa[i] = p.sa[(start + step) / 4 * p.ld_sa + min(m0 + wm + i * 32 + (lane & 31), p.M - 1)];
                sb[i] = p.sb[(start + step) / 4 * p.ld_sb + (min(n0 + wn + i * 32 + (lane & 31), p.N - 1) >> p.b_shift)];
            }
        }
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            Operand<FA, EXACT> a[2];
            Operand<FB, EXACT> b[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                a[i].take(operand(tile[half][0], wm + i * 32, s, lane), sa[i]);
                b[i].take(operand(tile[half][1], wn + i * 32, s, lane), sb[i]);
            }
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int j = 0; j < 2; ++j) acc[i][j] = multiply<FA, FB>(b[j], a[i], acc[i][j]);
        }
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            sa[i] >>= 8;
            sb[i] >>= 8;
        }
        if (step + 1 < steps) keep(half ^ 1);
    }
    if (p.splits > 1) {
        p.c = p.parts + (uint64_t)blockIdx.z * p.M * p.N;
        p.c_type = REFT_F32;
        p.ld_c = p.N;
    }
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j)
            store_tile(p, m0 + wm + i * 32 + (lane & 31), n0 + wn + j * 32, lane, acc[i][j]);
}

// ---- few rows of A: the weights' bytes are the bound ------------------------------------------------------------------
// A workgroup takes 16 rows of B, its waves blocks of 128 of K in turn; each lane loads its part of a product of 16 x 16 x 128 from
// memory itself (any alignment) and multiplies it with up to 16 rows of A.  The waves' sums meet in LDS and are
// added in the waves' order.  WHOLE: K is a multiple of 128.  16 waves, two blocks ahead, in 64 registers, so that two workgroups share a
// compute unit (one row, N x K = 11008 x 4096, 28672 x 8192: 11.6 and 41.1 us; 8 waves, four ahead: 17.3 and 57.3).
template <int FA, int FB, bool EXACT>
__device__ __forceinline__ f32x4 multiply16(i32x8 b, i32x8 a, f32x4 acc, uint32_t eb, uint32_t ea)
{
    if constexpr (!EXACT) {
        return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(b, a, acc, FB, FA, 0, (int)eb, 0, (int)ea);
    } else {
        Operand<FB, true> wb;
        Operand<FA, true> wa;
        wb.take(b, eb);
        wa.take(a, ea);
#pragma unroll
        for (int i = 0; i < 4; ++i) acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wb.v[i], wa.v[i], acc, 0, 0, 0);
        return acc;
    }
}

template <int FA, int FB, bool EXACT, bool WHOLE, int WAVES> __global__ __launch_bounds__(64 * WAVES, 8) void k_product_few(ProductArgs p)
{
    constexpr int kAhead = 2;
    __shared__ f32x4 sums[WAVES][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t n0 = blockIdx.x * 16, r = lane & 15, blocks = (p.K + 127) / 128;
    const uint32_t n = min(n0 + r, p.N - 1);                 // rows behind the last repeat it, and are not stored
    const bool row = r < p.M;
    const uint8_t *b = p.b + n * p.ld_b + (lane >> 4) * 32, *a = p.a + (row ? r : 0) * p.ld_a + (lane >> 4) * 32;
    const uint32_t *sb = p.sb + (n >> p.b_shift), *sa = p.sa + (row ? r : 0);
    f32x4 acc = {};
    for (uint32_t first = wave; first < blocks; first += WAVES * kAhead) {
        w32x4 vb[kAhead][2], va[kAhead][2];
        uint32_t eb[kAhead], ea[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const uint32_t block = first + u * WAVES, k = block * 128 + (lane >> 4) * 32;
            const bool there = block < blocks;                   // the same for the whole wave
            const int left = !there ? 0 : WHOLE ? 32 : k >= p.K ? 0 : (int)min(p.K - k, 32u);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                vb[u][h] = load16(b + block * 128ull + h * 16, left - h * 16);
                va[u][h] = load16(a + block * 128ull + h * 16, row ? left - h * 16 : 0);
            }
            eb[u] = there ? sb[block / 4 * p.ld_sb] >> block % 4 * 8 : 127;
            ea[u] = there && row ? sa[block / 4 * p.ld_sa] >> block % 4 * 8 : 127;
        }
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            i32x8 ob, oa;
#pragma unroll
            for (int e = 0; e < 8; ++e) ob[e] = (int)vb[u][e / 4][e % 4], oa[e] = (int)va[u][e / 4][e % 4];
            acc = multiply16<FA, FB, EXACT>(ob, oa, acc, eb[u], ea[u]);
        }
    }
    sums[wave][lane] = acc;
    __syncthreads();
    const uint32_t t = threadIdx.x;
    if (t < 256) {
        // column t % 16 of row t / 16: lane (column / 4) * 16 + row holds it, in place column % 4
        const uint32_t col = t % 16, m = t / 16;
        float v = 0;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) v += sums[w][col / 4 * 16 + m][col % 4];
        if (m < p.M && n0 + col < p.N) store1(p, m * p.ld_c + n0 + col, v);
    }
}

// ---- rows on 16 bytes: tiles in LDS that the memory system fills -------------------------------------------------
// Four waves, two by two, of MT x NT products of 32 x 32 each.  K is walked in steps of 128, with three tiles of A and two of B in LDS.
// Rows of tiles that are walked together, so that what runs at once on a die shares operands (8192 x 28672 x 8192: 4 1456 us, 8 1490, 16 1590).
constexpr int kGroup = 4;

// 16 bytes a lane from base + offset to LDS, those of a wave one after the other.  An offset of 32 bits from a base that the
// wave shares takes half the registers of addresses.
// A base that is not `there` has no bytes: the buffer's own bounds check keeps its copies from memory, but they count.
constexpr uint32_t kOutside = 0xffffffe0u;
struct Base {
    __amdgpu_buffer_rsrc_t r;
    __device__ __forceinline__ Base(const uint8_t *p, bool there)
        : r(__builtin_amdgcn_make_buffer_rsrc((void *)p, 0, __builtin_amdgcn_readfirstlane(there ? kOutside : 0), 0x00027000)) {}
};
__device__ __forceinline__ void copy_to_lds(const Base &from, uint32_t offset, uint8_t *to)
{
    __builtin_amdgcn_raw_ptr_buffer_load_lds(from.r, (__attribute__((address_space(3))) void *)to, 16, (int)offset, 0, 0, 0);
}

// For every wave: all but its last COPIES copies have arrived, what it asked LDS for is read, what it wrote is there.
template <int COPIES> __device__ __forceinline__ void meet()
{
    static_assert(COPIES < 64, "vmcnt has six bits");
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt((COPIES & 15) | (COPIES >> 4) << 14 | 0x0070);      // vmcnt(COPIES) lgkmcnt(0)
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
}

// Which tile a workgroup takes.  Workgroups are dealt to the eight dies in turn, and each die has an L2 of its own: a die gets
// tiles that follow each other.
__device__ __forceinline__ void tile_of(uint32_t id, uint32_t tiles_m, uint32_t tiles_n, uint32_t &m, uint32_t &n)
{
    const uint32_t total = tiles_m * tiles_n, each = total / 8, more = total % 8, die = id % 8;
    const uint32_t t = die * each + min(die, more) + id / 8;
    const uint32_t band = kGroup * tiles_n, first = t / band * kGroup, high = min(tiles_m - first, (uint32_t)kGroup);
    m = __builtin_amdgcn_readfirstlane(first + t % band % high);
    n = __builtin_amdgcn_readfirstlane(t % band / high);
}

// The order of a step's instructions: a product, then a few reads and copies that do not depend on it, and so on; the
// reads are done early, so that the wait for them at the step's end is none.
template <int PRODUCTS, int READS, int COPIES> __device__ __forceinline__ void interleave()
{
    constexpr int kReads = (READS * 4 + PRODUCTS * 3 - 1) / (PRODUCTS * 3), kCopies = (COPIES + PRODUCTS - 1) / PRODUCTS;
#pragma unroll
    for (int i = 0; i < PRODUCTS; ++i) {
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        if (i * kReads < READS) __builtin_amdgcn_sched_group_barrier(0x100, kReads, 0);
        if (i * kCopies < COPIES) __builtin_amdgcn_sched_group_barrier(0x010, kCopies, 0);
    }
}

// A wave's results leave in whole rows of 128 bytes, by way of 4 KB of LDS that are its own: 32 rows m of one product's columns n
// (fp32) or two products' (16 bits).
// WHOLE: all of them are C's.
template <typename T, int PARTS, bool WHOLE>
__device__ __forceinline__ void store_rows(T *to_c, uint64_t ld_c, const ProductArgs &p, uint8_t *room, uint32_t m, uint32_t n, int lane,
                                           const f32x16 *acc)
{
    constexpr uint32_t kEach = 16 / sizeof(T);
    static_assert(PARTS * 32 * sizeof(T) == 128, "a row of 128 bytes");
#pragma unroll
    for (int j = 0; j < PARTS; ++j)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const uint32_t at = (j * 32 + 8 * g + 4 * (lane >> 5)) * sizeof(T);          // of four neighbouring columns
            union { T t[4]; w32x2 w2; w32x4 w4; } u;
#pragma unroll
            for (int i = 0; i < 4; ++i) u.t[i] = narrow<T>(acc[j][4 * g + i]);
            uint8_t *to = room + place(lane & 31, at / 16) + at % 16;
            if constexpr (sizeof(T) == 4) *(w32x4 *)to = u.w4;
            else *(w32x2 *)to = u.w2;
        }
    const uint32_t col = n + (lane & 7) * kEach;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const int r = k * 8 + (lane >> 3);
        union { T t[kEach]; w32x4 w; } u;
        u.w = *(const w32x4 *)(room + place(r, lane & 7));
        if (!WHOLE && m + r >= p.M) continue;
        T *c = to_c + (m + r) * ld_c + col;
        if (WHOLE || col + kEach <= p.N) {
            *(w32x4_any *)c = u.w;
        } else {
#pragma unroll
            for (uint32_t i = 0; i < kEach; ++i)
                if (col + i < p.N) c[i] = u.t[i];
        }
    }
}

template <typename T, int MT, int NT>
__device__ __forceinline__ void store_all(T *c, uint64_t ld_c, const ProductArgs &p, uint8_t *room, uint32_t m, uint32_t n, int lane,
                                          const f32x16 (&acc)[MT][NT])
{
    constexpr int kParts = 4 / sizeof(T);
    if (m + 32 * MT <= p.M && n + 32 * NT <= p.N) {
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int j = 0; j < NT; j += kParts) store_rows<T, kParts, true>(c, ld_c, p, room, m + i * 32, n + j * 32, lane, &acc[i][j]);
    } else {
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int j = 0; j < NT; j += kParts) store_rows<T, kParts, false>(c, ld_c, p, room, m + i * 32, n + j * 32, lane, &acc[i][j]);
    }
}

// T: what is stored, into C or, of several parts of K, into a part's place.  The waves are one to a SIMD with the largest tile (its sums
// take 256 registers), so that all overlap is in the order of a wave's own instructions.  8192 x 28672 x 8192 to bf16: 1354 us, 2.84
// PFLOP/s, at 1.76 GHz (power) with the matrix cores busy 76 % of the cycles; 11008 x 4096 x 8192 to fp32: 555 us, 1.33 PFLOP/s, bound by the
// widening of operands; 1001 x 5120 x 1728 to bf16: 17.4 us, bound by the latency of 14 steps.
template <int FA, int FB, bool EXACT, typename T, int MT, int NT>
__global__ __launch_bounds__(256, MT * NT >= 16 ? 1 : 2) void k_product(ProductArgs p)
{
    constexpr int kRowsA = 64 * MT, kRowsB = 64 * NT, kCopiesA = 2 * MT, kCopiesB = 2 * NT, kCopies = kCopiesA + kCopiesB;
    constexpr int kProducts = MT * NT * (EXACT ? 4 : 1);
    // variables of their own, so that the compiler knows which copies a read has to wait for
    __shared__ __align__(16) uint8_t ta0[kRowsA * 128], ta1[kRowsA * 128], ta2[kRowsA * 128], tb0[kRowsB * 128], tb1[kRowsB * 128];
    uint8_t *const ta[3] = {ta0, ta1, ta2}, *const tb[2] = {tb0, tb1};
    constexpr bool kWhole = MT * NT >= 16;                   // K is never cut
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    uint32_t tm, tn;
    tile_of(blockIdx.x, (p.M + kRowsA - 1) / kRowsA, (p.N + kRowsB - 1) / kRowsB, tm, tn);
    const uint32_t m0 = tm * kRowsA, n0 = tn * kRowsB;
    const int wm = (wave & 1) * 32 * MT, wn = (wave >> 1) * 32 * NT;
    const uint32_t all = (p.K + 127) / 128, start = kWhole ? 0 : blockIdx.y * p.split_steps;
    const uint32_t steps = kWhole ? all : start < all ? min(all - start, p.split_steps) : 0, K = p.K - start * 128;
    // a last step that ends inside a chunk is taken by itself
    const bool cut = p.K % 16 && start + steps == all;
    const uint32_t loops = cut ? steps - 1 : steps;
    // A wave's copy fills eight rows of a tile: lane i the place i % 8 of row i / 8.  Rows behind the matrix's last repeat that.
    const uint8_t *base_a = p.a + (uint64_t)m0 * p.ld_a + (uint64_t)start * 128, *base_b = p.b + (uint64_t)n0 * p.ld_b + (uint64_t)start * 128;
    uint32_t from_a[kCopiesA], from_b[kCopiesB];
    auto chunk = [&](int i) { return (uint32_t)((lane & 7) ^ turn(i * 8 + (lane >> 3))) * 16; };
#pragma unroll
    for (int i = 0; i < kCopiesA; ++i)
        from_a[i] = min((uint32_t)((wave * kCopiesA + i) * 8 + (lane >> 3)), p.M - 1 - m0) * (uint32_t)p.ld_a + chunk(i);
#pragma unroll
    for (int i = 0; i < kCopiesB; ++i)
        from_b[i] = min((uint32_t)((wave * kCopiesB + i) * 8 + (lane >> 3)), p.N - 1 - n0) * (uint32_t)p.ld_b + chunk(i);
    // chunks behind K lie outside the buffer, and arrive as zeroes; one that holds a value of the row is memory of the row's to its end,
    // as chunks lie on 16 bytes
    auto fill_a = [&](uint32_t step, uint8_t *a) {
        const Base from(base_a + (uint64_t)step * 128, step < steps);
        const uint32_t left = K - step * 128, out0 = chunk(0) < left ? 0 : kOutside, out1 = chunk(1) < left ? 0 : kOutside;
#pragma unroll
        for (int i = 0; i < kCopiesA; ++i) copy_to_lds(from, from_a[i] | (i % 2 ? out1 : out0), a + (wave * kCopiesA + i) * 1024);
    };
    auto fill_b = [&](uint32_t step, uint8_t *b) {
        const Base from(base_b + (uint64_t)step * 128, step < steps);
        const uint32_t left = K - step * 128, out0 = chunk(0) < left ? 0 : kOutside, out1 = chunk(1) < left ? 0 : kOutside;
#pragma unroll
        for (int i = 0; i < kCopiesB; ++i) copy_to_lds(from, from_b[i] | (i % 2 ? out1 : out0), b + (wave * kCopiesB + i) * 1024);
    };
    auto read = [&](i32x8 (&a)[MT], i32x8 (&b)[NT], const uint8_t *from_a, const uint8_t *from_b, int s) {
        a[0] = operand(from_a, wm, s, lane);                 // in the order of their use
#pragma unroll
        for (int i = 0; i < NT; ++i) b[i] = operand(from_b, wn + i * 32, s, lane);
#pragma unroll
        for (int i = 1; i < MT; ++i) a[i] = operand(from_a, wm + i * 32, s, lane);
    };
    f32x16 acc[MT][NT] = {};
    uint32_t sa[MT], sb[NT], next_sa[MT], next_sb[NT];
    const uint32_t last_word = (p.K - 1) / 512;
    auto words = [&](uint32_t w) {
        w = min(start / 4 + w, last_word);
#pragma unroll
        for (int i = 0; i < MT; ++i) next_sa[i] = (p.sa + w * p.ld_sa)[min(m0 + wm + i * 32 + (lane & 31), p.M - 1)];
#pragma unroll
        for (int i = 0; i < NT; ++i) next_sb[i] = (p.sb + w * p.ld_sb)[min(n0 + wn + i * 32 + (lane & 31), p.N - 1) >> p.b_shift];
    };
    auto take_words = [&]() {
#pragma unroll
        for (int i = 0; i < MT; ++i) sa[i] = next_sa[i];
#pragma unroll
        for (int i = 0; i < NT; ++i) sb[i] = next_sb[i];
    };
    auto multiply_all = [&](const i32x8 (&ra)[MT], const i32x8 (&rb)[NT]) {
        Operand<FA, EXACT> a[MT];
        Operand<FB, EXACT> b[NT];
#pragma unroll
        for (int i = 0; i < MT; ++i) a[i].take(ra[i], sa[i]);
#pragma unroll
        for (int i = 0; i < NT; ++i) b[i].take(rb[i], sb[i]);
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int j = 0; j < NT; ++j) acc[i][j] = multiply<FA, FB>(b[j], a[i], acc[i][j]);
        // The products stay on this side of what follows: nothing else holds them, and behind it they would keep their operands'
        // registers.
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int j = 0; j < NT; ++j)
                if constexpr (kWhole) asm volatile("" : "+a"(acc[i][j]));
                else asm volatile("" : "+v"(acc[i][j]));
    };

    fill_a(0, ta0);
    fill_b(0, tb0);
    fill_a(1, ta1);
    fill_b(1, tb1);
    words(0);
    meet<0>();
    i32x8 a0[MT], b0[NT], a1[MT], b1[NT];
    read(a0, b0, ta0, tb0, 0);
    // Half a step multiplies what half a step ago was read from LDS, while the next half is read.  Between a step's halves its
    // tiles have been read by all and the next step's have arrived; the ones after those are fetched all the time, A's in a step's
    // first half (into a third place), B's in the second: a half's copies more in flight than with two places each, and no more
    // at once than the way from the L2 takes (8192 x 28672 x 8192: 1460 -> 1360 us).  A word of scales serves four steps.
    for (uint32_t step = 0; step < loops; step += 6) {
#pragma unroll
        for (int j = 0; j < 6; ++j) {
            const uint32_t at = step + j;
            if (at >= loops) break;
            if (at % 4 == 0) {
                take_words();
                words(at / 4 + 1);
            }
            __builtin_amdgcn_sched_barrier(0);
            fill_a(at + 2, ta[(j + 2) % 3]);
            read(a1, b1, ta[j % 3], tb[j % 2], 1);
            multiply_all(a0, b0);
            interleave<kProducts, 2 * (MT + NT), kCopiesA>();
            meet<kCopiesA>();
            fill_b(at + 2, tb[j % 2]);
            read(a0, b0, ta[(j + 1) % 3], tb[(j + 1) % 2], 0);
            multiply_all(a1, b1);
            interleave<kProducts, 2 * (MT + NT), kCopiesB>();
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int i = 0; i < MT; ++i) sa[i] >>= 8;
#pragma unroll
            for (int i = 0; i < NT; ++i) sb[i] >>= 8;
        }
    }
    if (cut) {                                               // what follows K in its chunk is anything: zeroed in registers
        if (loops % 4 == 0) take_words();
        const int left = (int)(K - loops * 128);
        const uint8_t *const la = loops % 3 == 0 ? ta0 : loops % 3 == 1 ? ta1 : ta2, *const lb = loops % 2 ? tb1 : tb0;
#pragma unroll 1
        for (int s = 0; s < 2; ++s) {
            read(a0, b0, la, lb, s);
            int mask[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int there = left - (s * 64 + (lane >> 5) * 32 + e * 4);          // bytes of this word
                mask[e] = there >= 4 ? -1 : there <= 0 ? 0 : (1 << 8 * there) - 1;
            }
#pragma unroll
            for (int i = 0; i < MT; ++i)
#pragma unroll
                for (int e = 0; e < 8; ++e) a0[i][e] &= mask[e];
#pragma unroll
            for (int i = 0; i < NT; ++i)
#pragma unroll
                for (int e = 0; e < 8; ++e) b0[i][e] &= mask[e];
            multiply_all(a0, b0);
        }
    }
    uint8_t *const room = (wave & 2 ? ta1 : ta0) + (wave & 1) * 4096;
    const uint32_t m = m0 + wm, n = n0 + wn;
    meet<0>();
    if (!kWhole && sizeof(T) == 4 && p.splits > 1) store_all((T *)p.parts + (uint64_t)blockIdx.y * p.M * p.N, p.N, p, room, m, n, lane, acc);
    else store_all((T *)p.c, p.ld_c, p, room, m, n, lane, acc);
}

// C from the parts of K, added in their order; four neighbouring columns a thread.  A launch more: 2 to 3 us.
template <typename T> __global__ __launch_bounds__(256) void k_add_parts(ProductArgs p)
{
    const uint32_t wide = (p.N + 3) / 4;
    const uint64_t id = (uint64_t)blockIdx.x * 256 + threadIdx.x, m = id / wide, n = id % wide * 4;
    if (m >= p.M) return;
    const int count = (int)min((uint64_t)4, p.N - n);
    float v[4] = {};
#pragma unroll 4
    for (uint32_t s = 0; s < p.splits; ++s) {
        const float *from = p.parts + ((uint64_t)s * p.M + m) * p.N + n;
        if (count == 4) {
            const w32x4 w = *(const w32x4_any *)from;
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] += __uint_as_float(w[i]);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (i < count) v[i] += from[i];
        }
    }
    T *c = (T *)p.c + m * p.ld_c + n;
    union { T t[4]; w32x2 w2; w32x4 w4; } u;
#pragma unroll
    for (int i = 0; i < 4; ++i) u.t[i] = narrow<T>(v[i]);
    if (count == 4) {
        if constexpr (sizeof(T) == 4) *(w32x4_any *)c = u.w4;
        else *(w32x2_any *)c = u.w2;
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (i < count) c[i] = u.t[i];
    }
}

// Which tiles, and into how many parts K is cut where they are too few for the 256 compute units.
struct Shape {
    int tile;                      // 0: 64 x 128, 1: 128 x 128, 2: 256 x 256
    uint32_t splits, split_steps;
};
constexpr uint64_t kMaxParts = 64ull << 20;            // bytes of the workspace

// Time goes by the tiles that fall to a compute unit, which runs two of 128 x 128 at once or one of 256 x 256; one of these takes two
// and a half times one of those, and 720 values of K more for its start and end, which nothing runs beside.  Measured, us for 128
// and 256: N x K = 11008 x 4096, M = 512 29 and 41, 768 47 and 42, 1280 61 and 50, 1536 76 and 88, 2560 113 and 101; 5120 x 13824, M =
// 1536 112 and 136, 2048 185 and 139, 3200 218 and 269; M x N = 10730 x 4416, K = 50 29 and 38, 1024 65 and 67, 2048 105 and 98.
// K is cut where there are at most half as many tiles as units (M = 128 and 512 of 4096 x 11008: 46 -> 21, 46 -> 33; cut for twice as
// many places the second takes 44).
static Shape shape_of(uint64_t M, uint64_t N, uint64_t K)
{
    Shape t;
    const uint64_t big = (M + 255) / 256 * ((N + 255) / 256), small = (M + 127) / 128 * ((N + 127) / 128), steps = (K + 127) / 128;
    t.tile = M <= 64 ? 0 : 5 * ((big + 255) / 256) * (K + 720) <= 2 * ((small + 255) / 256) * K ? 2 : 1;
    t.splits = 1;
    t.split_steps = (uint32_t)((steps + 3) / 4 * 4);
    if (M <= 16 || t.tile == 2) return t;
    const uint64_t tiles = t.tile == 0 ? (N + 127) / 128 : small;
    const uint64_t want = std::min((t.tile == 0 ? 512 : 256) / tiles, std::min(steps / 8, kMaxParts / (M * N * 4)));
    if (want < 2) return t;
    t.split_steps = (uint32_t)(((steps + want - 1) / want + 3) / 4 * 4);
    t.splits = (uint32_t)((steps + t.split_steps - 1) / t.split_steps);
    return t;
}

// Rows on 16 bytes, so that chunks are; offsets inside a tile are held in 32 bits.
static bool on_16_bytes(const ProductArgs &p)
{
    return p.K && ((uintptr_t)p.a | (uintptr_t)p.b | p.ld_a | p.ld_b) % 16 == 0 && p.ld_a < (1u << 23) && p.ld_b < (1u << 23);
}

// Which results the bits that the 8-bit matrix instructions leave out would show in (see Operand).
static bool exact(const ProductArgs &p) { return p.c_type != REFT_BF16; }

static hipError_t add_parts(const ProductArgs &p, hipStream_t s)
{
    const uint32_t blocks = (uint32_t)(((uint64_t)p.M * ((p.N + 3) / 4) + 255) / 256);
    if (p.c_type == REFT_F32) k_add_parts<float><<<blocks, 256, 0, s>>>(p);
    else if (p.c_type == REFT_BF16) k_add_parts<bf16><<<blocks, 256, 0, s>>>(p);
    else k_add_parts<f16><<<blocks, 256, 0, s>>>(p);
    return hipGetLastError();
}

template <int FA, int FB, int MT, int NT> static hipError_t launch_tiles(const ProductArgs &p, hipStream_t s)
{
    const dim3 grid((p.M + 64 * MT - 1) / (64 * MT) * ((p.N + 64 * NT - 1) / (64 * NT)), p.splits);
    if (exact(p) && (p.c_type == REFT_F32 || p.splits > 1)) {
        k_product<FA, FB, true, float, MT, NT><<<grid, 256, 0, s>>>(p);
    } else if (exact(p)) {
        k_product<FA, FB, true, f16, MT, NT><<<grid, 256, 0, s>>>(p);
    } else if (p.splits > 1) {
        if constexpr (MT * NT < 16) k_product<FA, FB, false, float, MT, NT><<<grid, 256, 0, s>>>(p);
        else return hipErrorInvalidValue;                    // shape_of cuts K for the smaller tiles only
    } else {
        k_product<FA, FB, false, bf16, MT, NT><<<grid, 256, 0, s>>>(p);
    }
    const hipError_t e = hipGetLastError();
    return e == hipSuccess && p.splits > 1 ? add_parts(p, s) : e;
}

template <int FA, int FB, bool WHOLE> static hipError_t launch_few(const ProductArgs &p, hipStream_t s)
{
    const uint32_t grid = (p.N + 15) / 16;
    if (exact(p)) k_product_few<FA, FB, true, WHOLE, 16><<<grid, 1024, 0, s>>>(p);
    else k_product_few<FA, FB, false, WHOLE, 16><<<grid, 1024, 0, s>>>(p);
    return hipGetLastError();
}

template <int FA, int FB> static hipError_t launch_product(const ProductArgs &p, hipStream_t s)
{
    if (p.M <= 16 && (p.N + 15) / 16 < (1u << 22)) return      // a grid has less than 2^32 threads
        p.K % 128 ? launch_few<FA, FB, false>(p, s) : launch_few<FA, FB, true>(p, s);
    const Shape t = shape_of(p.M, p.N, p.K);
    ProductArgs q = p;
    q.splits = t.splits;
    q.split_steps = t.split_steps;
    if (on_16_bytes(p)) {
        switch (t.tile) {
        case 2: return launch_tiles<FA, FB, 4, 4>(q, s);
        case 1: return launch_tiles<FA, FB, 2, 2>(q, s);
        default: return launch_tiles<FA, FB, 1, 2>(q, s);
        }
    }
    const dim3 grid((q.N + 127) / 128, (q.M + 127) / 128, q.splits);
    if (exact(q)) k_product_any<FA, FB, true><<<grid, 256, 0, s>>>(q);
    else k_product_any<FA, FB, false><<<grid, 256, 0, s>>>(q);
    const hipError_t e = hipGetLastError();
    return e == hipSuccess && q.splits > 1 ? add_parts(q, s) : e;
}

}  // namespace reft

using namespace reft;

extern "C" uint64_t reft_product_workspace(uint64_t M, uint64_t N, uint64_t K)
{
    if (!M || !N || !K || M > 128 * 65535 || N > 0x7fffffff || K > 0x7fffffff) return 0;
    const Shape t = shape_of(M, N, K);
    return t.splits > 1 ? t.splits * M * N * sizeof(float) : 0;
}

extern "C" int reft_product(const void *a, uint64_t ld_a, int a_format, const void *a_scales, uint64_t ld_as, const void *b,
                            uint64_t ld_b, int b_format, const void *b_scales, uint64_t ld_bs, int b_blocks, uint64_t M, uint64_t N,
                            uint64_t K, void *c, uint64_t ld_c, int c_dtype, void *workspace, uint64_t workspace_bytes,
                            reft_stream stream)
{
#define NEED(cond, code, ...)                                                                     \
    do {                                                                                          \
        if (!(cond)) return fail(code, "reft_product: " __VA_ARGS__);                             \
    } while (0)
    NEED((a_format == REFT_E4M3 || a_format == REFT_E5M2) && (b_format == REFT_E4M3 || b_format == REFT_E5M2), REFT_EINVAL,
         "unknown 8-bit format");
    NEED(c_dtype == REFT_F32 || c_dtype == REFT_BF16 || c_dtype == REFT_F16, REFT_EINVAL, "unknown type %d", c_dtype);
    // rows of tiles are counted by the grid's second dimension, all of them (of 64 x 128) by less than 2^32 threads
    NEED(M <= 128 * 65535 && N <= 0x7fffffff && K <= 0x7fffffff && (M + 63) / 64 * ((N + 127) / 128) <= 0xffffff, REFT_ESIZE,
         "a matrix is too large");
    NEED(!M || !N || (c && (!K || (a && b && a_scales && b_scales))), REFT_EINVAL, "null pointer");
    NEED(ld_c >= N && ld_a >= K && ld_b >= K, REFT_ESIZE, "rows overlap");
    NEED(ld_as >= M && ld_bs >= (b_blocks ? (N + 127) / 128 : N), REFT_ESIZE, "words of scales overlap");
    if (!M || !N) return REFT_OK;
    NEED((uintptr_t)c % (c_dtype == REFT_F32 ? 4 : 2) == 0 && (uintptr_t)a_scales % 4 == 0 && (uintptr_t)b_scales % 4 == 0, REFT_EINVAL,
         "misaligned pointer");
    const uint64_t need = reft_product_workspace(M, N, K);
    NEED(!need || (workspace && (uintptr_t)workspace % 16 == 0), REFT_EINVAL, "no workspace, or not on 16 bytes");
    NEED(workspace_bytes >= need, REFT_ESIZE, "workspace too small");
#undef NEED
    if ((uintptr_t)stream == kCheckOnly) return REFT_OK;
    ProductArgs p;
    p.a = (const uint8_t *)a;
    p.b = (const uint8_t *)b;
    p.sa = (const uint32_t *)a_scales;
    p.sb = (const uint32_t *)b_scales;
    p.ld_a = ld_a;
    p.ld_b = ld_b;
    p.ld_sa = ld_as;
    p.ld_sb = ld_bs;
    p.ld_c = ld_c;
    p.M = (uint32_t)M;
    p.N = (uint32_t)N;
    p.K = (uint32_t)K;
    p.b_shift = b_blocks ? 7 : 0;
    p.c = c;
    p.c_type = c_dtype;
    p.splits = 1;
    p.split_steps = 0;
    p.parts = (float *)workspace;
    hipStream_t s = (hipStream_t)stream;
    hipError_t e;
    if (a_format == REFT_E4M3) e = b_format == REFT_E4M3 ? launch_product<0, 0>(p, s) : launch_product<0, 1>(p, s);
    else e = b_format == REFT_E4M3 ? launch_product<1, 0>(p, s) : launch_product<1, 1>(p, s);
    if (e != hipSuccess) return fail(REFT_EHIP, "reft_product: %s", hipGetErrorString(e));
    return REFT_OK;
}
