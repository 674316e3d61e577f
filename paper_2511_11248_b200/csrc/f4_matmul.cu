// Products with microscaled 4-bit weights: y[m][n] = row_scale[n] sum_k x[m][k] w[n][k], x in 16 bits (decode) or 4 bits (any M).
#include "f4_pair.cuh"
#include "f4_stream.cuh"

namespace tman {

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
    p.halves = L.halves;
    p.height8 = L.height8;
    return p;
}
template <int BLOCK, typename T>
static tman_status gemm_as(const void *packed, const void *a, void *y, int ldy, int M, int K, int N, void *ws, cudaStream_t s)
{
    if (stream_wins(M, N)) return launch_stream<BLOCK, T, false>(stream_params(packed, a, nullptr, 0, y, ldy, M, K, N, BLOCK, ws), s);
    const F4Layout L = f4_layout(N, K, BLOCK), A = f4_layout(M, K, BLOCK);
    F4PairParams p = {};
    p.w = static_cast<const uint8_t *>(packed);
    p.a = static_cast<const uint8_t *>(a);
    p.y = y;
    p.status = static_cast<uint32_t *>(ws);
    p.w_codes = L.codes_off; p.w_scales = L.scales_off; p.w_rows = L.rows_off;
    p.a_codes = A.codes_off; p.a_scales = A.scales_off; p.a_rows = A.rows_off;
    p.M = M; p.K = K; p.N = N; p.ldy = ldy;
    p.halves = L.halves;
    p.w_h8 = L.height8; p.a_h8 = A.height8;
    return launch_pair<BLOCK, T>(p, s);
}

tman_status launch_f4_gemv(const void *packed, const void *x, int ldx, void *y, int ldy, int dtype, int M, int K, int N, int block, void *ws, cudaStream_t s)
{
    const F4StreamParams p = stream_params(packed, nullptr, x, ldx, y, ldy, M, K, N, block, ws);
    if (dtype == kF4TypeHalf) return block == 32 ? launch_stream<32, __half, true>(p, s) : launch_stream<16, __half, true>(p, s);
    return block == 32 ? launch_stream<32, __nv_bfloat16, true>(p, s) : launch_stream<16, __nv_bfloat16, true>(p, s);
}
tman_status launch_f4_gemm(const void *packed, const void *a, void *y, int ldy, int dtype, int M, int K, int N, int block, void *ws, cudaStream_t s)
{
    if (dtype == kF4TypeHalf) return block == 32 ? gemm_as<32, __half>(packed, a, y, ldy, M, K, N, ws, s) : gemm_as<16, __half>(packed, a, y, ldy, M, K, N, ws, s);
    return block == 32 ? gemm_as<32, __nv_bfloat16>(packed, a, y, ldy, M, K, N, ws, s) : gemm_as<16, __nv_bfloat16>(packed, a, y, ldy, M, K, N, ws, s);
}

// How a call is cut; see tman_debug_f4_plan.
tman_status f4_plan_for(int op, int M, int K, int N, int block, int sms, const int (&clusters)[2], int *out8)
{
    if (op == 0 || stream_wins(M, N)) {
        const StreamPlan t = stream_plan(M, K, N, block, op == 0, sms);
        const int out[8] = {0, M, t.split, 1, t.tiles, t.tiles * t.split, t.stages, 0};
        for (int i = 0; i < 8; ++i) out8[i] = out[i];
        return TMAN_OK;
    }
    F4PairParams p = {};
    p.M = M;
    p.N = N;
    p.halves = f4_layout(N, K, block).halves;
    const long long tiles = pair_shape(p, sms / 2, clusters), pairs = tiles < sms / 2 ? tiles : sms / 2;
    if (tiles > 0x7FFFFFFF) return TMAN_ERR_SHAPE;
    const int out[8] = {1, p.nt, 1 << p.split_sh, p.tiles_m, p.tiles_n, (int)pairs << p.split_sh, block == 32 ? pair_stages<32>() : pair_stages<16>(),
                        p.rows_fastest | p.stream_y << 1};
    for (int i = 0; i < 8; ++i) out8[i] = out[i];
    return TMAN_OK;
}
tman_status f4_plan(int op, int M, int K, int N, int block, int *out8)
{
    int dev = 0, clusters[2];
    const DeviceInfo *info = device_info(&dev);
    if (!info) return TMAN_ERR_CUDA;
    if (block == 32) pair_capacity<32, __half>(dev, clusters);
    else pair_capacity<16, __half>(dev, clusters);
    return f4_plan_for(op, M, K, N, block, info->sms.load(std::memory_order_relaxed), clusters, out8);
}

}  // namespace tman
