// What the kernels of attention over the 8-bit cache have in common.
#pragma once

#include "cache_i8.cuh"

#include <climits>
#include <type_traits>

namespace tman {
namespace {

constexpr float kLog2e = 1.4426950408889634f;

__device__ __forceinline__ float exp2_fast(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// The first token that a row at `position` sees, of a window (0: none).  The position may be negative and the window any: their difference need not be a number.
__device__ __forceinline__ int window_from(int position, int window) { return window > 0 && position >= window ? position - window + 1 : 0; }
// Four signed bytes as fp16: with the top bit turned they are 0..255, which in the low byte of 0x6400 is 1024 + that.
__device__ __forceinline__ void bytes_to_half(uint32_t w, uint32_t &lo, uint32_t &hi)
{
    const uint32_t u = w ^ 0x80808080u;
    const __half2 off = __half2half2(__ushort_as_half(0x6480));
    const uint32_t a = __byte_perm(u, 0x64646464u, 0x4140), b = __byte_perm(u, 0x64646464u, 0x4342);
    const __half2 x = __hsub2(*reinterpret_cast<const __half2 *>(&a), off), y = __hsub2(*reinterpret_cast<const __half2 *>(&b), off);
    lo = *reinterpret_cast<const uint32_t *>(&x);
    hi = *reinterpret_cast<const uint32_t *>(&y);
}

}  // namespace
}  // namespace tman
