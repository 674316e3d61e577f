// Microscaled 4-bit floating point: packing and unpacking of a checkpoint's matrix, quantization of rows, dequantization.
// Memory-bound: every value is read and written once.
#include "f4.cuh"

namespace tman {

// ---- checkpoint layout <-> packed buffer -----------------------------------------------------
// codes [rows][K/2], scales [rows][K/block], row_scale [rows].  One thread moves 8 bytes of codes (16 values); the first thread of a
// block of four scales moves those.
template <int BLOCK, bool TO_PACKED>
__global__ void __launch_bounds__(256) f4_relayout_kernel(uint8_t *codes, uint8_t *scales, float *row_scale, int rows, int K, uint8_t *packed,
                                                          F4Layout L, uint32_t *status)
{
    const size_t i = (size_t)blockIdx.x * 256 + threadIdx.x;
    if constexpr (TO_PACKED) {
        if (i < 64) reinterpret_cast<uint32_t *>(packed)[i] = f4_header_word((int)i, rows, K, BLOCK, L);
    } else if (!f4_header_matches(packed, rows, K, BLOCK)) {
        if (i == 0) atomicCAS(status, 0u, (uint32_t)TMAN_ERR_BAD_PACKED);
        return;
    }
    const int pieces = L.halves * (kF4Half / 16);
    const int r = (int)(i / pieces), k = (int)(i % pieces) * 16;
    if (r >= L.tiles * kF4Tile) return;
    const int nb = K / BLOCK, b = k / BLOCK;
    if (r < L.height8) {
        uint8_t *c = packed + L.codes_off + f4_code_at(r, k, L);
        uint8_t *plain = codes + ((size_t)r * K + k) / 2;
        const bool in = r < rows && k < K;
        if constexpr (TO_PACKED) {
            uint64_t v = 0;
            if (in)
                for (int e = 0; e < 8; ++e) v |= (uint64_t)plain[e] << (8 * e);
            *reinterpret_cast<uint64_t *>(c) = v;
        } else if (in) {
            const uint64_t v = *reinterpret_cast<const uint64_t *>(c);
            for (int e = 0; e < 8; ++e) plain[e] = (uint8_t)(v >> (8 * e));
        }
    }
    if (k % (4 * BLOCK) == 0) {
        uint8_t *c = packed + L.scales_off + f4_scale_at(r, b, BLOCK, L);
        for (int e = 0; e < 4; ++e) {
            const bool in = r < rows && b + e < nb;
            if constexpr (TO_PACKED) c[e] = in ? scales[(size_t)r * nb + b + e] : 0;
            else if (in) scales[(size_t)r * nb + b + e] = c[e];
        }
    }
    if (BLOCK == 16 && k == 0) {
        float *c = reinterpret_cast<float *>(packed + L.rows_off) + r;
        if constexpr (TO_PACKED) *c = r < rows ? (row_scale ? row_scale[r] : 1.f) : 0.f;
        else if (r < rows && row_scale) row_scale[r] = *c;
    } else if (BLOCK == 32 && k == 0 && !TO_PACKED && r < rows && row_scale)
        row_scale[r] = 1.f;
}

template <bool TO_PACKED>
static tman_status launch_relayout(uint8_t *codes, uint8_t *scales, float *row_scale, int rows, int K, int block, void *packed, uint32_t *status, cudaStream_t s)
{
    const F4Layout L = f4_layout(rows, K, block);
    const size_t threads = (size_t)L.tiles * kF4Tile * L.halves * (kF4Half / 16), grid = (threads + 255) / 256;
    if (grid > 0x7FFFFFFFull) return TMAN_ERR_SHAPE;
    auto kern = block == 32 ? f4_relayout_kernel<32, TO_PACKED> : f4_relayout_kernel<16, TO_PACKED>;
    kern<<<(unsigned)grid, 256, 0, s>>>(codes, scales, row_scale, rows, K, static_cast<uint8_t *>(packed), L, status);
    return launch_status();
}

tman_status launch_f4_pack(const uint8_t *codes, const uint8_t *scales, const float *row_scale, int rows, int K, int block, void *packed, cudaStream_t s)
{
    const tman_status st = launch_relayout<true>(const_cast<uint8_t *>(codes), const_cast<uint8_t *>(scales), const_cast<float *>(row_scale), rows, K,
                                                 block, packed, nullptr, s);
    if (st == TMAN_OK) note_packed_write(s);
    return st;
}

tman_status launch_f4_unpack(const void *packed, int rows, int K, int block, uint8_t *codes, uint8_t *scales, float *row_scale, uint32_t *status,
                             cudaStream_t s)
{
    return launch_relayout<false>(codes, scales, row_scale, rows, K, block, const_cast<void *>(packed), status, s);
}

// ---- quantization of rows ----------------------------------------------------------------------
// One block's scale byte and the codes of eight of its values.  top: the largest magnitude of the block; fine: all its values are finite;
// inv_row: 1 / r, a power of two.
//   block 32: scale 2^e, e = floor(log2 top) - 2 (at least -127): x 2^-e is exact, one rounding.
//   block 16: scale s = e4m3(top / (6 r)), codes round(x / (r s)).  x / r is exact (r is a power of two), so with x of at most 11
//   significant bits and s of four the quotient x / (r s) is either exactly half way between two codes or further than 2^-11 of itself
//   from it.  x (1/s) is off by less than 2^-22 of itself, and rounding it to 17 significant bits makes the half-way cases exact again:
//   the codes are those of the exact quotient.  (top / r / 6 is a correctly rounded quotient, for the same reason.)
// A block that holds an infinity or a NaN gets the scale NaN.
template <int BLOCK>
__device__ __forceinline__ uint32_t f4_block_scale(float top, bool fine, float inv_row)
{
    if constexpr (BLOCK == 32) {
        if (!fine) return 255u;
        const int e = (int)(__float_as_uint(top) >> 23) - 2;         // biased exponent of the scale
        return (uint32_t)max(e, 0);
    } else {
        if (!fine) return 0x7Fu;
        return f4_round_e4m3(__fdiv_rn(top * inv_row, 6.f));
    }
}
template <int BLOCK>
__device__ __forceinline__ uint32_t f4_block_codes(const float (&x)[8], uint32_t scale, float inv_row)
{
    float v[8];
    if constexpr (BLOCK == 32) {
        const float inv = __uint_as_float(scale >= 254u ? 0x00400000u : (254u - scale) << 23);       // 2^(127 - byte); 2^-127 for 254
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = x[e] * inv;
    } else {
        const float s = f4_scale_value<16>(scale), inv = s > 0.f ? __frcp_rn(s) : 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = __uint_as_float((__float_as_uint(x[e] * inv_row * inv) + 0x40u) & 0xFFFFFF80u);
    }
    return f4_round8(v);
}
// The row scale of block 16: the least power of two r with m <= 2688 r (448 x 6), 2^-126 at least; 1 for a row of zeros.
__device__ __forceinline__ float f4_row_scale(float m)
{
    if (!(m > 0.f)) return 1.f;
    const uint32_t u = __float_as_uint(m);
    int e = (int)(u >> 23) - 11;                                     // (2688 = 1.3125 x 2^11)
    if ((u & 0x7FFFFFu) > 0x280000u) ++e;
    return __uint_as_float((uint32_t)max(e, 1) << 23);
}

// A CTA has one row: for block 16 its largest finite magnitude first, then eight values a thread.
template <int BLOCK, typename T>
__global__ void __launch_bounds__(256) f4_quantize_kernel(const T *x, int ldx, int rows, int K, uint8_t *packed, F4Layout L)
{
    __shared__ float red[8];
    const int r = blockIdx.x, lane = threadIdx.x & 31;
    if (r == 0 && threadIdx.x < 64) reinterpret_cast<uint32_t *>(packed)[threadIdx.x] = f4_header_word(threadIdx.x, rows, K, BLOCK, L);
    const uint4 *row = reinterpret_cast<const uint4 *>(x + (size_t)r * ldx);
    const bool real = r < rows;
    auto load = [&](int at, float (&f)[8]) {
        uint4 v = make_uint4(0u, 0u, 0u, 0u);
        if (real && at * 8 < K) v = row[at];
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float2 p = f4_to_float2<T>(w[e]);
            f[2 * e] = p.x;
            f[2 * e + 1] = p.y;
        }
    };
    float inv_row = 1.f;
    if constexpr (BLOCK == 16) {
        float m = 0.f;
        for (int at = threadIdx.x; at * 8 < K; at += 256) {
            float f[8];
            load(at, f);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float a = fabsf(f[e]);
                if (a < __int_as_float(0x7F800000)) m = fmaxf(m, a);
            }
        }
        for (int o = 16; o; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
        if (lane == 0) red[threadIdx.x >> 5] = m;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < 8; ++w) m = fmaxf(m, red[w]);
        const float rs = f4_row_scale(m);
        inv_row = __fdiv_rn(1.f, rs);
        if (threadIdx.x == 0) reinterpret_cast<float *>(packed + L.rows_off)[r] = rs;
    }
    const int vectors = L.halves * (kF4Half / 8);
    for (int at = threadIdx.x; at < (vectors + 31) / 32 * 32; at += 256) {          // (whole warps: lanes of a block exchange)
        float f[8];
        load(at, f);
        float top = 0.f;
        bool fine = true;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float a = fabsf(f[e]);
            fine = fine && a < __int_as_float(0x7F800000);
            top = fmaxf(top, a);
        }
#pragma unroll
        for (int o = BLOCK / 16; o; o >>= 1) {
            top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
            const bool other = __shfl_xor_sync(0xffffffffu, (int)fine, o) != 0;      // (every lane takes part, whatever its own verdict)
            fine = fine && other;
        }
        if (at >= vectors) continue;
        const int k = at * 8;
        const uint32_t scale = k < K ? f4_block_scale<BLOCK>(top, fine, inv_row) : 0u;
        if (r < L.height8) *reinterpret_cast<uint32_t *>(packed + L.codes_off + f4_code_at(r, k, L)) = f4_block_codes<BLOCK>(f, scale, inv_row);
        if (k % BLOCK == 0) packed[L.scales_off + f4_scale_at(r, k / BLOCK, BLOCK, L)] = (uint8_t)scale;
    }
}

template <int BLOCK, typename T>
static tman_status launch_quantize_as(const void *x, int ldx, int rows, int K, void *packed, cudaStream_t s)
{
    const F4Layout L = f4_layout(rows, K, BLOCK);
    f4_quantize_kernel<BLOCK, T><<<(unsigned)L.height8, 256, 0, s>>>(static_cast<const T *>(x), ldx, rows, K, static_cast<uint8_t *>(packed), L);
    return launch_status();
}

tman_status launch_f4_quantize(const void *x, int ldx, int dtype, int rows, int K, int block, void *packed, cudaStream_t s)
{
    if (dtype == kF4TypeHalf) return block == 32 ? launch_quantize_as<32, __half>(x, ldx, rows, K, packed, s) : launch_quantize_as<16, __half>(x, ldx, rows, K, packed, s);
    return block == 32 ? launch_quantize_as<32, __nv_bfloat16>(x, ldx, rows, K, packed, s) : launch_quantize_as<16, __nv_bfloat16>(x, ldx, rows, K, packed, s);
}

// ---- dequantization -----------------------------------------------------------------------------
template <int BLOCK, typename T>
__global__ void __launch_bounds__(256) f4_dequant_kernel(const uint8_t *packed, int rows, int K, T *x, int ldx, F4Layout L, uint32_t *status)
{
    if (!f4_header_matches(packed, rows, K, BLOCK)) {
        if (blockIdx.x == 0 && threadIdx.x == 0) atomicCAS(status, 0u, (uint32_t)TMAN_ERR_BAD_PACKED);
        return;
    }
    const int r = blockIdx.x;
    const float rs = BLOCK == 16 ? reinterpret_cast<const float *>(packed + L.rows_off)[r] : 1.f;
    for (int k = threadIdx.x * 8; k < K; k += 256 * 8) {
        const uint32_t c = *reinterpret_cast<const uint32_t *>(packed + L.codes_off + f4_code_at(r, k, L));
        const float s = f4_scale_value<BLOCK>(packed[L.scales_off + f4_scale_at(r, k / BLOCK, BLOCK, L)]) * rs;
        uint32_t w[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float2 p = __half22float2(f4_pair(c >> (8 * e)));
            w[e] = f4_from_float2<T>(p.x * s, p.y * s);
        }
        *reinterpret_cast<uint4 *>(x + (size_t)r * ldx + k) = make_uint4(w[0], w[1], w[2], w[3]);
    }
}

template <int BLOCK, typename T>
static tman_status launch_dequant_as(const void *packed, int rows, int K, void *x, int ldx, uint32_t *status, cudaStream_t s)
{
    f4_dequant_kernel<BLOCK, T><<<(unsigned)rows, 256, 0, s>>>(static_cast<const uint8_t *>(packed), rows, K, static_cast<T *>(x), ldx, f4_layout(rows, K, BLOCK), status);
    return launch_status();
}

tman_status launch_f4_dequant(const void *packed, int rows, int K, int block, void *x, int ldx, int dtype, uint32_t *status, cudaStream_t s)
{
    if (dtype == kF4TypeHalf) return block == 32 ? launch_dequant_as<32, __half>(packed, rows, K, x, ldx, status, s) : launch_dequant_as<16, __half>(packed, rows, K, x, ldx, status, s);
    return block == 32 ? launch_dequant_as<32, __nv_bfloat16>(packed, rows, K, x, ldx, status, s) : launch_dequant_as<16, __nv_bfloat16>(packed, rows, K, x, ldx, status, s);
}

}  // namespace tman
