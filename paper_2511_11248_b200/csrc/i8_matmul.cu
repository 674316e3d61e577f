// 8-bit integer products: token quantization and the choice of the kernel.
#include "i8_pair.cuh"

namespace tman {
namespace {

// ---- token quantization: a row a CTA, VPT pieces of eight values a thread, read once ----------------------------------------------
template <typename T, int VPT>
__global__ void __launch_bounds__(1024) i8_quantize_kernel(const T *x, int ldx, int K, int8_t *a, float *row_scale)
{
    __shared__ uint32_t tops[32];
    const int tid = threadIdx.x, pieces = K >> 3;
    const uint4 *row = reinterpret_cast<const uint4 *>(x + (size_t)blockIdx.x * ldx);
    uint2 *out = reinterpret_cast<uint2 *>(a + (size_t)blockIdx.x * K);
    if (tid < 32) tops[tid] = 0;
    __syncthreads();
    grid_wait();
    grid_launch_next();
    uint4 v[VPT];
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
        const int at = tid + i * blockDim.x;
        v[i] = at < pieces ? ld_dependent(row + at) : make_uint4(0, 0, 0, 0);
    }
#pragma unroll
    for (int i = 0; i < VPT; ++i)
        top = i8_larger(top, i8_larger(i8_larger(i8_magnitudes(v[i].x), i8_magnitudes(v[i].y)), i8_larger(i8_magnitudes(v[i].z), i8_magnitudes(v[i].w))));
    top = __reduce_max_sync(0xffffffffu, max(top & 0xFFFFu, top >> 16));
    if ((tid & 31) == 0) tops[tid >> 5] = top;
    __syncthreads();
    top = __reduce_max_sync(0xffffffffu, tops[tid & 31]);
    const float scale = top == 0 ? 1.f : i8_scale<T>(top);
    if (tid == 0) row_scale[blockIdx.x] = scale;
    const I8Divisor d(scale);
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
        const int at = tid + i * blockDim.x;
        if (at < pieces) out[at] = i8_codes<T>(d, v[i]);
    }
}

template <typename T> tman_status quantize(const void *x, int ldx, int M, int K, int8_t *a, float *row_scale, cudaStream_t s)
{
    // Few rows: the latency of one row counts, as many threads as there are pieces.  Many: four pieces a thread, eight of long rows, so that an SM has
    // several rows in flight (8192 x 18944: four 139 us, eight 80; 777 x 3584: 5.2 and 7.0).
    const int pieces = K / 8, least = (pieces + 1023) / 1024, some = pieces >= 1024 ? 8 : 4, want = M > 2 * kGemvPlanSms && least < some ? some : least;
    const int vpt = want <= 1 ? 1 : want <= 2 ? 2 : want <= 4 ? 4 : want <= 8 ? 8 : 16;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)M);
    cfg.blockDim = dim3((unsigned)(((pieces + vpt - 1) / vpt + 31) / 32 * 32));
    cfg.stream = s;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    auto kern = vpt == 1 ? i8_quantize_kernel<T, 1> : vpt == 2 ? i8_quantize_kernel<T, 2> : vpt == 4 ? i8_quantize_kernel<T, 4> : vpt == 8 ? i8_quantize_kernel<T, 8>
                                                                                                                                         : i8_quantize_kernel<T, 16>;
    return call_status(cudaLaunchKernelEx(&cfg, kern, static_cast<const T *>(x), ldx, K, a, row_scale));
}

}  // namespace

tman_status launch_i8_quantize(const void *x, int ldx, int dtype, int M, int K, int8_t *a, float *row_scale, cudaStream_t s)
{
    return dtype == kF4TypeHalf ? quantize<__half>(x, ldx, M, K, a, row_scale, s) : quantize<__nv_bfloat16>(x, ldx, M, K, a, row_scale, s);
}

// Rows of 16 bits whose codes every CTA of the product works out itself; others are quantized by a launch of their own.  A launch costs some 1.3 us, and every
// CTA's own work grows with the rows.  In a graph, us, here / with a launch: 1 x 4096 x 4096 6.4 / 7.8, 1 x 14336 x 4096 14.0 / 15.1, 1 x 16384 x 4096 17.9 / 16.6,
// 1 x 18944 x 3584 16.8 / 17.6, 2 x 2048 x 4096 5.5 / 5.7, 2 x 4096 x 4096 7.0 / 8.0, 2 x 8192 x 4096 10.6 / 11.0, 4 x 2048 x 4096 6.3 / 5.6, 4 x 4096 x 4096
// 8.2 / 7.8, 8 x 1024 x 4096 7.7 / 4.8.
static bool i8_fused(int M, int K) { return M <= 2 && M * K <= kI8FusedValues; }

size_t i8_workspace_bytes(int op, int M, int K)
{
    return op == 0 && !i8_fused(M, K) ? kI8ScratchOff + up256((size_t)M * K) + up256(M * sizeof(float)) : kWsStatusBytes;
}

tman_status launch_i8_gemv(const int8_t *w, int ldw, const float *w_scale, const void *x, int ldx, void *y, int ldy, int dtype, int M, int K, int N,
                           void *ws, cudaStream_t s)
{
    uint8_t *w8 = static_cast<uint8_t *>(ws);
    const I8StreamParams p = {w, x, w_scale, nullptr, y, ldw, ldx, ldy, M, K, N, 0, 0};
    if (i8_fused(M, K)) return dtype == kF4TypeHalf ? launch_i8_stream<__half, false>(p, s) : launch_i8_stream<__nv_bfloat16, false>(p, s);
    int8_t *a = reinterpret_cast<int8_t *>(w8 + kI8ScratchOff);
    float *a_scale = reinterpret_cast<float *>(w8 + kI8ScratchOff + up256((size_t)M * K));
    const tman_status st = launch_i8_quantize(x, ldx, dtype, M, K, a, a_scale, s);
    if (st != TMAN_OK) return st;
    return launch_i8_gemm(w, ldw, w_scale, a, a_scale, y, ldy, dtype, M, K, N, ws, s);
}

tman_status launch_i8_gemm(const int8_t *w, int ldw, const float *w_scale, const int8_t *a, const float *a_scale, void *y, int ldy, int dtype, int M,
                           int K, int N, void *ws, cudaStream_t s)
{
    if (M <= 8) {
        const I8StreamParams p = {w, a, w_scale, a_scale, y, ldw, K, ldy, M, K, N, 0, 0};
        return dtype == kF4TypeHalf ? launch_i8_stream<__half, true>(p, s) : launch_i8_stream<__nv_bfloat16, true>(p, s);
    }
    I8PairParams p = {};
    p.w_scale = w_scale;
    p.a_scale = a_scale;
    p.y = y;
    p.status = static_cast<uint32_t *>(ws);
    p.M = M;
    p.K = K;
    p.N = N;
    p.ldy = ldy;
    return dtype == kF4TypeHalf ? launch_i8_pair<__half>(w, ldw, a, p, s) : launch_i8_pair<__nv_bfloat16>(w, ldw, a, p, s);
}

}  // namespace tman
