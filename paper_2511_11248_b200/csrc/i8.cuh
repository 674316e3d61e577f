// 8-bit integers: what the token quantization, the products and the cache share.
#pragma once

#include "common.cuh"
#include "f4.cuh"                        // conversions of the two 16-bit types
#include "sm100_ptx.cuh"

namespace tman {

constexpr int kI8MaxK = 131056;          // products of two bytes, 2^14 at most, in 32-bit sums
constexpr int kI8MaxRows = 1 << 30;      // rows and channels of products, sequences: their indexes go on for a tile or a CTA's share behind the last
// Workspace: status word (kWsStatusBytes), the counters of attention, which are at rest between calls, and behind them what a call leaves lying: codes of a decode
// product, parts of attention.  So that the calls of 8-bit integers can have one workspace in turn.
constexpr int kAttendCtas = 320;         // of attention, at most
constexpr size_t kI8ScratchOff = kWsStatusBytes + kAttendCtas * sizeof(uint32_t);
static_assert(kI8ScratchOff % 256 == 0, "codes are read in 16-byte pieces");

// entry points implemented per file
tman_status launch_i8_quantize(const void *x, int ldx, int dtype, int M, int K, int8_t *a, float *row_scale, cudaStream_t s);
tman_status launch_i8_gemv(const int8_t *w, int ldw, const float *w_scale, const void *x, int ldx, void *y, int ldy, int dtype, int M, int K, int N,
                           void *ws, cudaStream_t s);
tman_status launch_i8_gemm(const int8_t *w, int ldw, const float *w_scale, const int8_t *a, const float *a_scale, void *y, int ldy, int dtype, int M,
                           int K, int N, void *ws, cudaStream_t s);
size_t      i8_workspace_bytes(int op, int M, int K);

#ifdef __CUDACC__
// What tcgen05.ld brings is there behind tcgen05.wait::ld only.  The compiler, which does not know, would be free to use it before: this says that it
// changes here.
__device__ __forceinline__ void tcgen05_loaded(uint32_t (&r)[16])
{
    asm volatile("" : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]), 
                      "+r"(r[8]), "+r"(r[9]), "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15]));
}
__device__ __forceinline__ void tcgen05_loaded(uint32_t (&r)[32])
{
    asm volatile("" : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]), 
                      "+r"(r[8]), "+r"(r[9]), "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15]), 
                      "+r"(r[16]), "+r"(r[17]), "+r"(r[18]), "+r"(r[19]), "+r"(r[20]), "+r"(r[21]), "+r"(r[22]), "+r"(r[23]), 
                      "+r"(r[24]), "+r"(r[25]), "+r"(r[26]), "+r"(r[27]), "+r"(r[28]), "+r"(r[29]), "+r"(r[30]), "+r"(r[31]));
}

// Magnitudes of two 16-bit floating-point numbers as integers, which are ordered like them; an infinity is above every number, a NaN above that.
__device__ __forceinline__ uint32_t i8_magnitudes(uint32_t pair) { return pair & 0x7FFF7FFFu; }
__device__ __forceinline__ uint32_t i8_larger(uint32_t a, uint32_t b) { return __vmaxu2(a, b); }
template <typename T> __device__ __forceinline__ uint32_t i8_infinity();
template <> __device__ __forceinline__ uint32_t i8_infinity<__half>() { return 0x7C00u; }
template <> __device__ __forceinline__ uint32_t i8_infinity<__nv_bfloat16>() { return 0x7F80u; }
template <typename T> __device__ __forceinline__ float i8_value(uint32_t bits) { return f4_to_float2<T>(bits).x; }

// The divisor of a row or page whose largest magnitude is `top` (bits): top / 127; NaN where top is none.
template <typename T> __device__ __forceinline__ float i8_scale(uint32_t top)
{
    return top >= i8_infinity<T>() ? __uint_as_float(0x7FFFFFFFu) : __fdiv_rn(i8_value<T>(top), 127.f);
}

// round(x / scale) of the quotient rounded to 32 bits, to nearest even.  Added to 2^23 + 2^22, the product with the reciprocal is rounded to an integer,
// which is in the low bits; it is off by 127 x 2^-24 at most, and the quotient's own rounding by 2^-18, so that only one next to a half needs the division; so do scales whose reciprocal
// is none (0 stands for zeros, and so does a scale that is no number).  No code is beyond 127: x is at most the scale's 127-fold.
struct I8Divisor {
    float scale, inv;
    __device__ __forceinline__ explicit I8Divisor(float s) : scale(s), inv(s >= 1e-30f ? 1.f / s : 0.f) {}
    __device__ __noinline__ static uint32_t divided(float x, float scale)
    {
        const float r = scale > 0.f ? rintf(__fdiv_rn(x, scale)) : 0.f;
        return (uint32_t)(int)fminf(fmaxf(r, -127.f), 127.f) & 0xFFu;
    }
};
// Eight codes of eight 16-bit values.
template <typename T> __device__ __forceinline__ uint2 i8_codes(const I8Divisor &d, const uint4 &v)
{
    constexpr float kMagic = 12582912.f, kNear = 0.499985f;
    const float2 p[4] = {f4_to_float2<T>(v.x), f4_to_float2<T>(v.y), f4_to_float2<T>(v.z), f4_to_float2<T>(v.w)};
    uint32_t c[8];
    float far = 0.f;                                             // how far a quotient is from its integer at most
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float x = i & 1 ? p[i >> 1].y : p[i >> 1].x, r = fmaf(x, d.inv, kMagic);
        far = fmaxf(far, fabsf(fmaf(x, d.inv, kMagic - r)));
        c[i] = __float_as_uint(r);
    }
    if (far > kNear || d.inv == 0.f) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float x = i & 1 ? p[i >> 1].y : p[i >> 1].x;
            if (d.inv == 0.f || fabsf(fmaf(x, d.inv, kMagic - __uint_as_float(c[i]))) > kNear) c[i] = I8Divisor::divided(x, d.scale);
        }
    }
    return make_uint2(__byte_perm(__byte_perm(c[0], c[1], 0x0040), __byte_perm(c[2], c[3], 0x0040), 0x5410),
                      __byte_perm(__byte_perm(c[4], c[5], 0x0040), __byte_perm(c[6], c[7], 0x0040), 0x5410));
}

// sum x (token's scale x channel's scale).  The scales' product in 32 bits where it and what it multiplies stay in range, else in 64.
__device__ __noinline__ inline float i8_scaled64(int sum, float a_scale, float w_scale) { return (float)((double)sum * (double)a_scale * (double)w_scale); }
// Two such scales have a product that i8_scaled takes in 32 bits.
__device__ __forceinline__ bool i8_ordinary(float s) { return s >= 1e-15f && s <= 1e14f; }
__device__ __forceinline__ float i8_scaled(int sum, float a_scale, float w_scale)
{
    const float s = a_scale * w_scale;
    if (fabsf(s) >= 1e-30f && fabsf(s) <= 1e28f) return (float)sum * s;
    return i8_scaled64(sum, a_scale, w_scale);
}
#endif

}  // namespace tman
