// Microscaled 4-bit floating point (e2m1 with block scales): the layout of a packed matrix and what every kernel of this path shares.
//
// A matrix of `rows` rows and K columns is cut along K into blocks of 32 or 16 values; value = e2m1 code x block scale x row scale.
//   block 32: block scale e8m0 (2^(byte - 127), 255: NaN), no row scale
//   block 16: block scale e4m3, row scale fp32
// Packed buffer (little endian), sections padded to 256 bytes:
//   header  256 bytes: "TMANF4MX", u32 version = 1, rows, K, block, u64 codes_off, scales_off, rows_off, total_bytes
//   codes   units of 256 columns (the last one 128 where that holds the rest), in each all rows, rounded up to a multiple of 8, in groups of 8.
//           A group is 8 (or 4) core matrices of the tensor cores' K-major operands without swizzle, 8 rows x 32 columns in 128 bytes: byte
//           (k%256/32)*128 + (r%8)*16 + (k%32)/2, the even k in the low half.
//   scales  the same units, in each tiles of 128 rows, in each 2 (1) x 128 / (4 block) pieces of 512 bytes: byte (r%32)*16 + (r/32%4)*4 + c is
//           the scale of block c of four: the order in which tensor memory holds the scales of 128 rows (32 lanes, a column of four bytes
//           per 32 rows).
//   rows    fp32, 128 a tile (block 16 only)
// So any rows' codes of a unit, and the scales of adjacent tiles, reach shared memory as operands by one linear bulk copy, without a tensor
// map.  K is filled up to a multiple of 128 with codes and scales of zero.
#pragma once

#include "common.cuh"
#include "f4_order.h"

#include <cuda_bf16.h>

namespace tman {

struct F4Header {
    char     magic[8];
    uint32_t version, rows, K, block;
    uint64_t codes_off, scales_off, rows_off, total_bytes;
};
constexpr uint32_t kF4Version = 1;
constexpr int kF4Half = 128;            // columns of half a unit
constexpr int kF4Tile = 128;            // rows of a tile of scales

struct F4Layout {
    int tiles, halves, height8;         // height8: all rows, rounded up to 8
    size_t codes_off, scales_off, rows_off, total;
};
__host__ __device__ constexpr int f4_scale_bytes(int block) { return block == 32 ? 512 : 1024; }      // of half a unit of a tile
__host__ __device__ inline F4Layout f4_layout(int rows, int K, int block)
{
    F4Layout L;
    L.tiles = (rows + kF4Tile - 1) / kF4Tile;
    L.halves = (K + kF4Half - 1) / kF4Half;
    L.height8 = (rows + 7) / 8 * 8;
    L.codes_off = kHeaderBytes;
    L.scales_off = L.codes_off + up256((size_t)L.halves * 64 * L.height8);
    L.rows_off = L.scales_off + (size_t)L.tiles * L.halves * f4_scale_bytes(block);
    L.total = L.rows_off + (block == 16 ? (size_t)L.tiles * kF4Tile * 4 : 0);
    return L;
}
// Byte of a code pair / of a scale, from the start of its section.
__host__ __device__ inline size_t f4_code_at(int r, int k, const F4Layout &L)
{
    const int u = k / (2 * kF4Half), wide = 2 * u + 1 < L.halves ? 1024 : 512;
    return (size_t)u * L.height8 * 128 + (size_t)(r / 8) * wide + (k % (2 * kF4Half) / 32) * 128 + (r % 8) * 16 + (k % 32) / 2;
}
__host__ __device__ inline size_t f4_scale_at(int r, int b, int block, const F4Layout &L)      // b: block along K
{
    const int per = kF4Half / block, half = b / per, u = half / 2, sb = f4_scale_bytes(block), wide = 2 * u + 1 < L.halves ? 2 : 1;
    return ((size_t)u * L.tiles * 2 + (size_t)(r / kF4Tile) * wide + half % 2) * sb + (b % per / 4) * 512 + (r % 32) * 16 + (r % kF4Tile / 32) * 4 + b % 4;
}

inline tman_status f4_check(int rows, int K, int block)
{
    if (rows < 1 || K < 1) return TMAN_ERR_SHAPE;
    if (block != 16 && block != 32) return TMAN_ERR_SHAPE;
    if (K % block != 0) return TMAN_ERR_SHAPE;
    if (rows > (1 << 30) || K > (1 << 30)) return TMAN_ERR_SHAPE;
    return TMAN_OK;
}

#ifdef __CUDACC__
// "TMAN" = 0x4E414D54, "F4MX" = 0x584D3446
__device__ inline bool f4_header_matches(const void *packed, int rows, int K, int block)
{
    const uint32_t *h = reinterpret_cast<const uint32_t *>(packed);
    return h[0] == 0x4E414D54u && h[1] == 0x584D3446u && h[2] == kF4Version && h[3] == (uint32_t)rows && h[4] == (uint32_t)K && h[5] == (uint32_t)block;
}
// The same of words that are there already.
__device__ inline bool f4_header_is(const uint4 &h, const uint2 &g, int rows, int K, int block)
{
    return h.x == 0x4E414D54u && h.y == 0x584D3446u && h.z == kF4Version && h.w == (uint32_t)rows && g.x == (uint32_t)K && g.y == (uint32_t)block;
}
// Word t (0..63) of a header.
__device__ inline uint32_t f4_header_word(int t, int rows, int K, int block, const F4Layout &L)
{
    if (t < 6) return t == 0 ? 0x4E414D54u : t == 1 ? 0x584D3446u : t == 2 ? kF4Version : t == 3 ? (uint32_t)rows : t == 4 ? (uint32_t)K : (uint32_t)block;
    if (t >= 14) return 0u;
    const uint64_t off = t < 8 ? L.codes_off : t < 10 ? L.scales_off : t < 12 ? L.rows_off : L.total;
    return (uint32_t)(off >> (32 * (t & 1)));
}

// Two e2m1 codes (the low byte) as fp16: exact.  (The byte is taken out of a 16-bit register: out of a 32-bit one that an 8-bit load filled, nvcc
// 12.9 converts zeros.)
__device__ __forceinline__ __half2 f4_pair(uint32_t byte)
{
    uint32_t h;
    asm("{\n.reg .b8 b, z;\n.reg .b16 p;\ncvt.u16.u32 p, %1;\nmov.b16 {b, z}, p;\ncvt.rn.f16x2.e2m1x2 %0, b;\n}" : "=r"(h) : "r"(byte));
    return *reinterpret_cast<__half2 *>(&h);
}
// Eight values as eight codes, the first in the lowest four bits; to nearest, ties to even, saturating.
__device__ __forceinline__ uint32_t f4_round8(const float (&v)[8])
{
    uint32_t r;
    asm("{\n.reg .b8 b0, b1, b2, b3;\n"
        "cvt.rn.satfinite.e2m1x2.f32 b0, %2, %1;\n"
        "cvt.rn.satfinite.e2m1x2.f32 b1, %4, %3;\n"
        "cvt.rn.satfinite.e2m1x2.f32 b2, %6, %5;\n"
        "cvt.rn.satfinite.e2m1x2.f32 b3, %8, %7;\n"
        "mov.b32 %0, {b0, b1, b2, b3};\n}"
        : "=r"(r) : "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7]));
    return r;
}
// A scale byte's value.
template <int BLOCK> __device__ __forceinline__ float f4_scale_value(uint32_t byte)
{
    if constexpr (BLOCK == 32) {
        if (byte == 255u) return __int_as_float(0x7FC00000);
        return __uint_as_float(byte == 0u ? 0x00400000u : byte << 23);
    } else {
        uint32_t h;
        asm("{\n.reg .b16 p;\ncvt.u16.u32 p, %1;\ncvt.rn.f16x2.e4m3x2 %0, p;\n}" : "=r"(h) : "r"(byte));
        return __low2float(*reinterpret_cast<__half2 *>(&h));
    }
}
// v >= 0 as e4m3, to nearest, ties to even, 448 at most.
__device__ __forceinline__ uint32_t f4_round_e4m3(float v)
{
    uint16_t p;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(p) : "f"(0.f), "f"(v));
    return p & 0xFFu;
}

template <typename T> __device__ __forceinline__ float2 f4_to_float2(uint32_t pair);
template <> __device__ __forceinline__ float2 f4_to_float2<__half>(uint32_t pair) { return __half22float2(*reinterpret_cast<__half2 *>(&pair)); }
template <> __device__ __forceinline__ float2 f4_to_float2<__nv_bfloat16>(uint32_t pair)
{
    return make_float2(__uint_as_float(pair << 16), __uint_as_float(pair & 0xFFFF0000u));
}
template <typename T> __device__ __forceinline__ uint32_t f4_from_float2(float a, float b);
template <> __device__ __forceinline__ uint32_t f4_from_float2<__half>(float a, float b)
{
    const __half2 h = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t *>(&h);
}
template <> __device__ __forceinline__ uint32_t f4_from_float2<__nv_bfloat16>(float a, float b)
{
    const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t *>(&h);
}
template <typename T> __device__ __forceinline__ T f4_from_float(float a);
template <> __device__ __forceinline__ __half f4_from_float<__half>(float a) { return __float2half_rn(a); }
template <> __device__ __forceinline__ __nv_bfloat16 f4_from_float<__nv_bfloat16>(float a) { return __float2bfloat16_rn(a); }
#endif

enum { kF4TypeHalf = 0, kF4TypeBf16 = 1 };

// entry points implemented per file
tman_status launch_f4_pack(const uint8_t *codes, const uint8_t *scales, const float *row_scale, int rows, int K, int block, void *packed, cudaStream_t s);
tman_status launch_f4_unpack(const void *packed, int rows, int K, int block, uint8_t *codes, uint8_t *scales, float *row_scale, uint32_t *status,
                             cudaStream_t s);
tman_status launch_f4_quantize(const void *x, int ldx, int dtype, int rows, int K, int block, void *packed, cudaStream_t s);
tman_status launch_f4_dequant(const void *packed, int rows, int K, int block, void *x, int ldx, int dtype, uint32_t *status, cudaStream_t s);
// A launch that reads `packed` as weights: whether a quantization ahead of it on s may still be writing them (call.pending), and that it was launched.
F4Order::Call f4_read_ahead(cudaStream_t s, const void *packed);
void          f4_read_behind(const F4Order::Call &call, bool launched);
size_t      f4_workspace_bytes(int op, int M, int K, int N, int block);
tman_status f4_plan(int op, int M, int K, int N, int block, int *out8);
tman_status f4_plan_for(int op, int M, int K, int N, int block, int sms, const int (&clusters)[2], int *out8);
tman_status launch_f4_gemv(const void *packed, const void *x, int ldx, void *y, int ldy, int dtype, int M, int K, int N, int block, void *ws, cudaStream_t s);
tman_status launch_f4_gemm(const void *packed, const void *a, void *y, int ldy, int dtype, int M, int K, int N, int block, void *ws, cudaStream_t s);

}  // namespace tman
