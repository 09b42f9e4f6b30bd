// Shared by the operators' entry points: checks of arguments, and what becomes of a launch.
#pragma once
#include "reft_step.hpp"

namespace reft {

constexpr uint64_t kMaxBlocks256 = 0xffffff;            // a grid has less than 2^32 threads: blocks of 256

inline bool is_float_type(int t) { return t == REFT_F32 || t == REFT_BF16 || t == REFT_F16; }
inline bool is_eight(int t) { return t == REFT_E4M3 || t == REFT_E5M2; }
inline size_t size_of(int t) { return t == REFT_F32 ? 4 : 2; }
// Arrays of elements lie on multiples of an element.
inline bool lies(const void *p, size_t n) { return (uintptr_t)p % n == 0; }
// Rows begin on cache lines.
inline bool on_lines(const void *p, uint64_t row_bytes) { return ((uintptr_t)p | row_bytes) % 128 == 0; }

inline int launched(const char *who, hipError_t e)
{
    if (e != hipSuccess) return fail(REFT_EHIP, "%s: %s", who, hipGetErrorString(e));
    return REFT_OK;
}

}  // namespace reft

#define NEED(cond, code, ...)                                                                     \
    do {                                                                                          \
        if (!(cond)) return fail(code, __VA_ARGS__);                                              \
    } while (0)
