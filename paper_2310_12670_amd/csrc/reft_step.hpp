// Shared by the operators of a training step (reft_step.hip, reft_product.hip): types, 16-byte accesses of any
// alignment, counter-based random bits, powers of two as scales.
#pragma once
#include "reft_internal.hpp"
#include "../../include/reft.h"


namespace reft {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t w32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t w32x4 __attribute__((ext_vector_type(4)));
// Rows may begin at any element: global memory is in unaligned access mode, so one wide access serves a lane
// whatever its address.
typedef w32x2 w32x2_any __attribute__((aligned(1), may_alias));
typedef w32x4 w32x4_any __attribute__((aligned(1), may_alias));

struct bf16 { uint16_t bits; };
struct f16 { uint16_t bits; };

__device__ __forceinline__ float widen(float v) { return v; }
__device__ __forceinline__ float widen(bf16 v) { return __uint_as_float((uint32_t)v.bits << 16); }
__device__ __forceinline__ float widen(f16 v) { return (float)__builtin_bit_cast(_Float16, v.bits); }

// Round to nearest, ties to even.
template <typename T> __device__ __forceinline__ T narrow(float v);
template <> __device__ __forceinline__ float narrow<float>(float v) { return v; }
template <> __device__ __forceinline__ bf16 narrow<bf16>(float v)
{
    return bf16{__builtin_bit_cast(uint16_t, (__bf16)v)};
}
template <> __device__ __forceinline__ f16 narrow<f16>(float v)
{
    return f16{__builtin_bit_cast(uint16_t, (_Float16)v)};
}

// Eight neighbouring values as they lie in memory; those that do not exist are zeroes.  STREAM: read once, so not kept in
// the caches.
template <typename T> struct Eight {
    union { w32x4 w[sizeof(T) / 2]; T t[8]; };
    template <bool STREAM> __device__ __forceinline__ void load(const T *p, int n)
    {
        if (n >= 8) {
#pragma unroll
            for (int i = 0; i < (int)sizeof(T) / 2; ++i)
                w[i] = STREAM ? __builtin_nontemporal_load((const w32x4_any *)p + i) : ((const w32x4_any *)p)[i];
        } else {
#pragma unroll
            for (int i = 0; i < (int)sizeof(T) / 2; ++i) w[i] = w32x4{0, 0, 0, 0};
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (i < n) t[i] = p[i];
        }
    }
    __device__ __forceinline__ float operator[](int i) const { return widen(t[i]); }
};

// Eight neighbouring values at p, of which the first n exist; the others read as zero.
template <bool STREAM, typename T> __device__ __forceinline__ void load8(const T *p, int n, float v[8])
{
    Eight<T> e;
    e.template load<STREAM>(p, n);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = e[i];
}

// Results are not kept in the L2: the whole of them rarely fits, and what is read beside them stays (16384 x 8192 in bf16: norm 184 ->
// 177 us, its gradient 248 -> 240; 2048 x 4096: norm 13.9 -> 12.1 us).  What reads them next is no slower by more than that gains: norm
// in 8 bits and the product of its output, us kept and past the L2: 1 x 8192 and 64 x 8192 17.4 and 17.5, 25.3 and 25.4, 512 x 4096 25.8 and
// 26.1, 2048 x 4096 49.8 and 48.0, 2048 x 8192 and 16384 x 5120 the same.
template <typename T> __device__ __forceinline__ void store8(T *p, int n, const float v[8])
{
    constexpr int kWords = 2 * sizeof(T);
    union { w32x4 w[kWords / 4]; T t[8]; } u;
#pragma unroll
    for (int i = 0; i < 8; ++i) u.t[i] = narrow<T>(v[i]);
    if (n >= 8) {
#pragma unroll
        for (int i = 0; i < kWords / 4; ++i) __builtin_nontemporal_store(u.w[i], (w32x4_any *)p + i);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < n) p[i] = u.t[i];
    }
}

// A vector of fp32 or of T.
template <typename T> __device__ __forceinline__ void load8_of(const void *p, bool f32, uint64_t at, int n, float v[8])
{
    if (f32) load8<false>((const float *)p + at, n, v);
    else load8<false>((const T *)p + at, n, v);
}

// ---- random bits: Philox4x32-10 (Salmon, Moraes, Dror, Shaw: Parallel Random Numbers: As Easy as 1, 2, 3,
// SC 2011).  128 bits from a 64-bit key and a 128-bit counter, with no state: element (r, c) of a matrix gets 16
// bits of its own whatever thread, tile or stride it is read with.  One call serves eight elements.
struct Dropout {
    uint32_t key0, key1, off0, off1;
    uint32_t threshold;            // of 65536; 0 = everything is kept, without a look at the bits
    float scale;                   // 65536 / (65536 - threshold), 0 where nothing is kept
};

__device__ __forceinline__ void drop8(const Dropout &d, uint32_t row, uint32_t group, float v[8])
{
    uint32_t c0 = group, c1 = row, c2 = d.off0, c3 = d.off1, k0 = d.key0, k1 = d.key1;
#pragma unroll
    for (int i = 0; i < 10; ++i) {
        const uint64_t a = (uint64_t)c0 * 0xD2511F53u, b = (uint64_t)c2 * 0xCD9E8D57u;
        c0 = (uint32_t)(b >> 32) ^ c1 ^ k0;
        c1 = (uint32_t)b;
        c2 = (uint32_t)(a >> 32) ^ c3 ^ k1;
        c3 = (uint32_t)a;
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    const uint32_t w[4] = {c0, c1, c2, c3};
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint32_t bits = i & 1 ? w[i >> 1] >> 16 : w[i >> 1] & 0xffff;
        v[i] = bits >= d.threshold ? v[i] * d.scale : 0.f;     // chosen, not multiplied: a dropped NaN is zero
    }
}

// ---- 8 bits with powers of two ------------------------------------------------------------------------------
// The scale of a block is the smallest power of two that brings its largest magnitude to at most the format's largest
// value, 1.75 * 2^top: its biased exponent is the magnitude's, less top, and one more where the mantissa exceeds
// 1.75, which the addition carries over.  At least 2^-126, so that factor and inverse are normal numbers.  A block
// that holds an infinity or a NaN gets 255 (NaN), and all its values become NaN.
__device__ __forceinline__ uint32_t scale_of(uint32_t amax_bits, int top)
{
    if (amax_bits >= 0x7f800000u) return 255;
    const int e = (int)((amax_bits + 0x1fffffu) >> 23) - top;
    return e < 1 ? 1 : (uint32_t)e;
}
__device__ __forceinline__ float inverse_of(uint32_t e)
{
    return e == 255 ? __uint_as_float(0x7fc00000u) : __uint_as_float((254u - e) << 23);
}

// The largest magnitude as bits: of non-negative floats the order of the bits is that of the values, and a NaN's are
// larger than all.
__device__ __forceinline__ uint32_t magnitude(float v) { return __float_as_uint(v) & 0x7fffffffu; }

// The value of the lane that a DPP control pairs this one with; all lanes take part.
template <int CONTROL> __device__ __forceinline__ uint32_t paired(uint32_t v)
{
    return (uint32_t)__builtin_amdgcn_update_dpp((int)v, (int)v, CONTROL, 0xf, 0xf, true);
}
constexpr int kSwap1 = 0xb1, kSwap2 = 0x4e, kMirror8 = 0x141, kMirror16 = 0x140;       // lanes ^ 1, ^ 2, 7 -, 15 -
// The largest of 16 neighbouring lanes' values.
__device__ __forceinline__ uint32_t max_of_16(uint32_t v)
{
    v = max(v, paired<kSwap1>(v));
    v = max(v, paired<kSwap2>(v));
    v = max(v, paired<kMirror8>(v));
    return max(v, paired<kMirror16>(v));
}
__device__ __forceinline__ float sum_of_16(float v)
{
    v += __uint_as_float(paired<kSwap1>(__float_as_uint(v)));
    v += __uint_as_float(paired<kSwap2>(__float_as_uint(v)));
    v += __uint_as_float(paired<kMirror8>(__float_as_uint(v)));
    return v + __uint_as_float(paired<kMirror16>(__float_as_uint(v)));
}

// Eight values in 8 bits, to nearest even (e5m2: the wide format).
__device__ __forceinline__ w32x2 to_eight(const float v[8], float inv, bool e5m2)
{
    float t[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) t[i] = v[i] * inv;
    int lo = 0, hi = 0;
    if (e5m2) {
        lo = __builtin_amdgcn_cvt_pk_bf8_f32(t[0], t[1], lo, false);
        lo = __builtin_amdgcn_cvt_pk_bf8_f32(t[2], t[3], lo, true);
        hi = __builtin_amdgcn_cvt_pk_bf8_f32(t[4], t[5], hi, false);
        hi = __builtin_amdgcn_cvt_pk_bf8_f32(t[6], t[7], hi, true);
    } else {
        lo = __builtin_amdgcn_cvt_pk_fp8_f32(t[0], t[1], lo, false);
        lo = __builtin_amdgcn_cvt_pk_fp8_f32(t[2], t[3], lo, true);
        hi = __builtin_amdgcn_cvt_pk_fp8_f32(t[4], t[5], hi, false);
        hi = __builtin_amdgcn_cvt_pk_fp8_f32(t[6], t[7], hi, true);
    }
    w32x2 w;
    w.x = (uint32_t)lo;
    w.y = (uint32_t)hi;
    return w;
}

template <bool STREAM> __device__ __forceinline__ void store8_bytes(uint8_t *p, int n, w32x2 w)
{
    if (n >= 8) {
        if constexpr (STREAM) __builtin_nontemporal_store(w, (w32x2_any *)p);
        else *(w32x2_any *)p = w;
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < n) p[i] = (uint8_t)((i < 4 ? w.x : w.y) >> (8 * (i & 3)));
    }
}

// The scale byte of block b of a row, and ones in the rest of its word behind the last of the `blocks` blocks.
__device__ __forceinline__ void store_scale(uint8_t *scales, uint64_t ld, uint64_t row, uint64_t b, uint64_t blocks, uint32_t e)
{
    uint8_t *word = scales + ((b / 4) * ld + row) * 4;
    word[b % 4] = (uint8_t)e;
    if (b + 1 == blocks)
        for (int i = (int)(b % 4) + 1; i < 4; ++i) word[i] = 127;
}

__device__ __forceinline__ int top_of(bool e5m2) { return e5m2 ? 15 : 8; }

}  // namespace reft
