// Products with microscaled 4-bit weights: y[m][n] = row_scale[n] sum_k x[m][k] w[n][k], x in 16 bits (decode) or 4 bits (any M).
#include "f4_stream.cuh"

namespace tman {

template <int BLOCK>
__device__ __forceinline__ float f4_value(const uint8_t *packed, const F4Layout &L, int r, int k)
{
    const uint32_t c = packed[L.codes_off + f4_code_at(r, k, L.height8, L.units)];
    const float2 p = __half22float2(f4_pair(c));
    return (k & 1 ? p.y : p.x) * f4_scale_value<BLOCK>(packed[L.scales_off + f4_scale_at(r, k / BLOCK, BLOCK, L.units)]);
}

// 64 rows x 64 channels a CTA, 4 x 4 a thread, 32 values of k at a time through shared memory.
template <int BLOCK, typename T>
__global__ void __launch_bounds__(256) f4_gemm_kernel(const uint8_t *packed, F4Layout L, const uint8_t *a, F4Layout LA, T *y, int ldy, int M, int K, int N, uint32_t *status)
{
    if (!f4_header_matches(packed, N, K, BLOCK) || !f4_header_matches(a, M, K, BLOCK)) {
        if (blockIdx.x == 0 && threadIdx.x == 0) atomicCAS(status, 0u, (uint32_t)TMAN_ERR_BAD_PACKED);
        return;
    }
    __shared__ float ta[32][65], tw[32][65];
    const int tiles_n = (N + 63) / 64, m0 = blockIdx.x / tiles_n * 64, n0 = blockIdx.x % tiles_n * 64, tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
    float acc[4][4] = {};
    for (int k0 = 0; k0 < K; k0 += 32) {
        for (int i = threadIdx.x; i < 64 * 32; i += 256) {
            const int r = i / 32, k = k0 + i % 32;
            ta[i % 32][r] = m0 + r < M && k < K ? f4_value<BLOCK>(a, LA, m0 + r, k) : 0.f;
            tw[i % 32][r] = n0 + r < N && k < K ? f4_value<BLOCK>(packed, L, n0 + r, k) : 0.f;
        }
        __syncthreads();
        for (int k = 0; k < 32; ++k)
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[i][j] = fmaf(ta[k][ty + 16 * i], tw[k][tx + 16 * j], acc[i][j]);
        __syncthreads();
    }
    for (int i = 0; i < 4; ++i)
        for (int j = 0; j < 4; ++j) {
            const int m = m0 + ty + 16 * i, n = n0 + tx + 16 * j;
            if (m >= M || n >= N) continue;
            float v = acc[i][j];
            if (BLOCK == 16) v = v * reinterpret_cast<const float *>(packed + L.rows_off)[n] * reinterpret_cast<const float *>(a + LA.rows_off)[m];
            y[(size_t)m * ldy + n] = f4_from_float<T>(v);
        }
}

size_t f4_workspace_bytes(int, int, int, int, int) { return kWsStatusBytes; }

static F4StreamParams stream_params(const void *packed, const void *a, const void *x, int ldx, void *y, int ldy, int M, int K, int N, int block, void *ws)
{
    const F4Layout L = f4_layout(N, K, block), A = f4_layout(M, K, block);
    F4StreamParams p = {};
    p.w = static_cast<const uint8_t *>(packed);
    p.a = static_cast<const uint8_t *>(a);
    p.x = x;
    p.y = y;
    p.status = static_cast<uint32_t *>(ws);
    p.w_codes = L.codes_off; p.w_scales = L.scales_off; p.w_rows = L.rows_off;
    p.a_codes = A.codes_off; p.a_scales = A.scales_off; p.a_rows = A.rows_off;
    p.M = M; p.K = K; p.N = N; p.ldx = ldx; p.ldy = ldy;
    p.units = L.units;
    p.height8 = L.height8;
    return p;
}
template <int BLOCK, typename T>
static tman_status gemm_as(const void *packed, const void *a, void *y, int ldy, int M, int K, int N, void *ws, cudaStream_t s)
{
    if (M <= kStreamMaxRows) return launch_stream<BLOCK, T, false>(stream_params(packed, a, nullptr, 0, y, ldy, M, K, N, BLOCK, ws), s);
    const long long grid = (long long)((N + 63) / 64) * ((M + 63) / 64);
    if (grid > 0x7FFFFFFFll) return TMAN_ERR_SHAPE;
    f4_gemm_kernel<BLOCK, T><<<(unsigned)grid, 256, 0, s>>>(static_cast<const uint8_t *>(packed), f4_layout(N, K, BLOCK), static_cast<const uint8_t *>(a),
                                                           f4_layout(M, K, BLOCK), static_cast<T *>(y), ldy, M, K, N, static_cast<uint32_t *>(ws));
    return launch_status();
}

tman_status launch_f4_gemv(const void *packed, const void *x, int ldx, void *y, int ldy, int dtype, int M, int K, int N, int block, void *ws, cudaStream_t s)
{
    const F4StreamParams p = stream_params(packed, nullptr, x, ldx, y, ldy, M, K, N, block, ws);
    if (dtype == kF4Half) return block == 32 ? launch_stream<32, __half, true>(p, s) : launch_stream<16, __half, true>(p, s);
    return block == 32 ? launch_stream<32, __nv_bfloat16, true>(p, s) : launch_stream<16, __nv_bfloat16, true>(p, s);
}
tman_status launch_f4_gemm(const void *packed, const void *a, void *y, int ldy, int dtype, int M, int K, int N, int block, void *ws, cudaStream_t s)
{
    if (dtype == kF4Half) return block == 32 ? gemm_as<32, __half>(packed, a, y, ldy, M, K, N, ws, s) : gemm_as<16, __half>(packed, a, y, ldy, M, K, N, ws, s);
    return block == 32 ? gemm_as<32, __nv_bfloat16>(packed, a, y, ldy, M, K, N, ws, s) : gemm_as<16, __nv_bfloat16>(packed, a, y, ldy, M, K, N, ws, s);
}

}  // namespace tman
