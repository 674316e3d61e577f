// 8-bit integer products: token quantization and the choice of the kernel.
#include "i8_pair.cuh"
#include "i8_stream.cuh"

namespace tman {
namespace {

// ---- token quantization: a row a CTA -----------------------------------------------------------------------------------------
template <typename T>
__global__ void __launch_bounds__(256) i8_quantize_kernel(const T *x, int ldx, int K, int8_t *a, float *row_scale)
{
    __shared__ uint32_t tops[8];
    const int tid = threadIdx.x, pieces = K >> 3;
    const uint4 *row = reinterpret_cast<const uint4 *>(x + (size_t)blockIdx.x * ldx);
    uint2 *out = reinterpret_cast<uint2 *>(a + (size_t)blockIdx.x * K);
    grid_wait();
    grid_launch_next();
    uint32_t top = 0;
    for (int i = tid; i < pieces; i += 256) {
        const uint4 v = ld_dependent(row + i);
        top = i8_larger(top, i8_larger(i8_larger(i8_magnitudes(v.x), i8_magnitudes(v.y)), i8_larger(i8_magnitudes(v.z), i8_magnitudes(v.w))));
    }
    top = __reduce_max_sync(0xffffffffu, max(top & 0xFFFFu, top >> 16));
    if ((tid & 31) == 0) tops[tid >> 5] = top;
    __syncthreads();
    top = __reduce_max_sync(0xffffffffu, tops[tid & 7]);
    const float scale = top == 0 ? 1.f : i8_scale<T>(top);
    if (tid == 0) row_scale[blockIdx.x] = scale;
    const I8Divisor d(scale);
    for (int i = tid; i < pieces; i += 256) out[i] = i8_codes<T>(d, ld_dependent(row + i));
}

template <typename T> tman_status quantize(const void *x, int ldx, int M, int K, int8_t *a, float *row_scale, cudaStream_t s)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)M);
    cfg.blockDim = dim3(256);
    cfg.stream = s;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return call_status(cudaLaunchKernelEx(&cfg, i8_quantize_kernel<T>, static_cast<const T *>(x), ldx, K, a, row_scale));
}

}  // namespace

tman_status launch_i8_quantize(const void *x, int ldx, int dtype, int M, int K, int8_t *a, float *row_scale, cudaStream_t s)
{
    return dtype == kF4TypeHalf ? quantize<__half>(x, ldx, M, K, a, row_scale, s) : quantize<__nv_bfloat16>(x, ldx, M, K, a, row_scale, s);
}

size_t i8_workspace_bytes(int, int, int) { return kWsStatusBytes; }

tman_status launch_i8_gemv(const int8_t *w, int ldw, const float *w_scale, const void *x, int ldx, void *y, int ldy, int dtype, int M, int K, int N,
                           void *, cudaStream_t s)
{
    const I8StreamParams p = {w, x, w_scale, nullptr, y, ldw, ldx, ldy, M, K, N, 0};
    return dtype == kF4TypeHalf ? launch_i8_stream<__half, false>(p, s) : launch_i8_stream<__nv_bfloat16, false>(p, s);
}

tman_status launch_i8_gemm(const int8_t *w, int ldw, const float *w_scale, const int8_t *a, const float *a_scale, void *y, int ldy, int dtype, int M,
                           int K, int N, void *ws, cudaStream_t s)
{
    if (M <= 8) {
        const I8StreamParams p = {w, a, w_scale, a_scale, y, ldw, K, ldy, M, K, N, 0};
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
