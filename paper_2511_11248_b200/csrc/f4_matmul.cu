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
// Whether a packed x of M rows goes to CTAs that stream the weights rather than to pairs of CTAs with a tile each: by the two modelled times, and
// beyond 48 rows not with more tiles than pairs (the stream's stages are then few or its second round long).  Over the 23 shapes that the models are
// fitted to, both blocks, 1 to 64 rows, the kernel chosen takes 0.1 % more than the faster one in the mean and 6 % at most, over 11 others 0.3 % and
// 13 %.  One call in a graph of them, us, weights rotated over 300 MB, 32-value blocks, stream / pairs:
//   K x N   4096 x 1024   4096 x 4096   2048 x 8192   3584 x 4608   14336 x 4096  18944 x 3584  8192 x 8192   4096 x 14336  4096 x 28672
//   M = 16  3.3 / 6.0     4.4 / 8.5     5.3 / 6.2     5.1 / 7.9     7.7 / 14.3    9.6 / 12.5    9.8 / 12.7    7.5 / 10.2    12.9 / 14.8
//   M = 32  4.2 / 6.3     5.7 / 8.0     7.6 / 5.8     7.0 / 7.5     10.1 / 14.4   11.6 / 12.8   12.9 / 12.7   8.2 / 9.8     13.5 / 14.5
//   M = 48  5.2 / 6.3     7.6 / 8.7     10.5 / 6.5    9.2 / 8.1     12.5 / 14.6   14.1 / 12.9   16.1 / 12.8   9.6 / 10.3    14.5 / 15.0
//   M = 64  6.2 / 6.3     9.4 / 8.3     13.1 / 6.0    11.0 / 7.7    12.6 / 14.5   13.8 / 12.9   17.0 / 12.8   10.3 / 10.0   15.4 / 14.8
static bool stream_wins(int M, int K, int N, int sms, const int (&clusters)[2])
{
    const int tiles = (N + kF4Tile - 1) / kF4Tile, units = (K + 2 * kF4Half - 1) / (2 * kF4Half);
    if (M > kStreamMaxRows || (M > 48 && tiles > sms / 2)) return false;
    return stream_us(M, units, tiles, sms, clusters) <= 3.5 + 0.88 * pair_plan(M, units, (N + 255) / 256, sms / 2, clusters).us;
}
template <int BLOCK, typename T>
static tman_status gemm_as(const void *packed, const void *a, void *y, int ldy, int M, int K, int N, void *ws, cudaStream_t s)
{
    int dev = 0, clusters[2];
    const DeviceInfo *info = device_info(&dev);
    if (!info) return TMAN_ERR_CUDA;
    pair_capacity<BLOCK, T>(dev, clusters);
    if (stream_wins(M, K, N, info->sms.load(std::memory_order_relaxed), clusters)) return launch_stream<BLOCK, T, false>(stream_params(packed, a, nullptr, 0, y, ldy, M, K, N, BLOCK, ws), clusters, s);
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

template <int BLOCK, typename T>
static tman_status gemv_as(const void *packed, const void *x, int ldx, void *y, int ldy, int M, int K, int N, void *ws, cudaStream_t s)
{
    int dev = 0, clusters[2];
    if (!device_info(&dev)) return TMAN_ERR_CUDA;
    pair_capacity<BLOCK, T>(dev, clusters);
    return launch_stream<BLOCK, T, true>(stream_params(packed, nullptr, x, ldx, y, ldy, M, K, N, BLOCK, ws), clusters, s);
}

tman_status launch_f4_gemv(const void *packed, const void *x, int ldx, void *y, int ldy, int dtype, int M, int K, int N, int block, void *ws, cudaStream_t s)
{
    if (dtype == kF4TypeHalf) return block == 32 ? gemv_as<32, __half>(packed, x, ldx, y, ldy, M, K, N, ws, s) : gemv_as<16, __half>(packed, x, ldx, y, ldy, M, K, N, ws, s);
    return block == 32 ? gemv_as<32, __nv_bfloat16>(packed, x, ldx, y, ldy, M, K, N, ws, s) : gemv_as<16, __nv_bfloat16>(packed, x, ldx, y, ldy, M, K, N, ws, s);
}
tman_status launch_f4_gemm(const void *packed, const void *a, void *y, int ldy, int dtype, int M, int K, int N, int block, void *ws, cudaStream_t s)
{
    if (dtype == kF4TypeHalf) return block == 32 ? gemm_as<32, __half>(packed, a, y, ldy, M, K, N, ws, s) : gemm_as<16, __half>(packed, a, y, ldy, M, K, N, ws, s);
    return block == 32 ? gemm_as<32, __nv_bfloat16>(packed, a, y, ldy, M, K, N, ws, s) : gemm_as<16, __nv_bfloat16>(packed, a, y, ldy, M, K, N, ws, s);
}

// How a call is cut; see tman_debug_f4_plan.
tman_status f4_plan_for(int op, int M, int K, int N, int block, int sms, const int (&clusters)[2], int *out8)
{
    if (op == 0 || stream_wins(M, K, N, sms, clusters)) {
        const StreamPlan t = stream_plan(M, K, N, block, op == 0, sms, clusters);
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
