// Norms of query and key heads and the rotation by their position, in one pass.
//
// For each token and head: z = x / sqrt(mean(x^2) + eps) * weight (no weight: z = x), then each pair of the first `rot` values of z is turned by
// position * inv_freq[i]: pairs (i, i + rot/2), or (2i, 2i + 1).  Bound by reading and writing the heads once.
// A head is a group of 8, 16 or 32 lanes with eight values each; what a value is paired with is in the same lane or comes by a shuffle.  All in
// 32 bits, rounded once.  Angles are products of a position and a frequency, whole turns taken off, in 64 bits: in 32 a position of 100000 would
// leave 2^-8 of a turn.  A token's sines and cosines are worked out once a CTA, for all its heads.
#include "i8.cuh"

namespace tman {
namespace {

constexpr int kHeadThreads = 256, kHeadMaxWidth = 256;

struct HeadParams {
    const void *x;
    void *y;
    const void *q_weight, *k_weight;
    const int *positions;
    const float *inv_freq;
    int ldx, ldy, q_heads, k_heads, width, rot, adjacent, chunk;       // chunk: heads of a CTA
    float eps;
};

template <typename T, int LANES>
__global__ void __launch_bounds__(kHeadThreads) norm_rotate_kernel(const __grid_constant__ HeadParams p)
{
    __shared__ float2 turns[kHeadMaxWidth / 2];
    const int tid = threadIdx.x, group = tid / LANES, v = tid & (LANES - 1), token = blockIdx.x, heads = p.q_heads + p.k_heads;
    const int head0 = blockIdx.y * p.chunk, head1 = min(head0 + p.chunk, heads);
    const bool in = v * 8 < p.width;
    const T *x = static_cast<const T *>(p.x) + (size_t)token * p.ldx + v * 8;
    T *y = static_cast<T *>(p.y) + (size_t)token * p.ldy + v * 8;
    grid_wait();
    grid_launch_next();
    if (tid < p.rot / 2) {
        double a;
        {
            int pos;
            asm volatile("ld.global.s32 %0, [%1];" : "=r"(pos) : "l"(p.positions + token) : "memory");
            a = (double)pos * (double)ld_dependent(p.inv_freq + tid);
        }
        a -= rint(a * 0.15915494309189533577) * 6.283185307179586477;
        float s, c;
        sincosf((float)a, &s, &c);
        turns[tid] = make_float2(c, s);
    }
    __syncthreads();
    for (int head = head0 + group; __any_sync(0xffffffffu, head < head1); head += kHeadThreads / LANES) {
        const bool on = in && head < head1;
        uint4 raw = make_uint4(0, 0, 0, 0);
        if (on) raw = ld_dependent(reinterpret_cast<const uint4 *>(x + (size_t)head * p.width));
        float z[8];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float2 f = f4_to_float2<T>(e == 0 ? raw.x : e == 1 ? raw.y : e == 2 ? raw.z : raw.w);
            z[2 * e] = f.x;
            z[2 * e + 1] = f.y;
        }
        const T *weight = static_cast<const T *>(head < p.q_heads ? p.q_weight : p.k_weight);
        float sum = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) sum = fmaf(z[e], z[e], sum);
#pragma unroll
        for (int d = LANES / 2; d > 0; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
        if (weight && on) {
            const float r = rsqrtf(sum / (float)p.width + p.eps);
            const uint4 wr = ld_dependent(reinterpret_cast<const uint4 *>(weight + v * 8));
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float2 f = f4_to_float2<T>(e == 0 ? wr.x : e == 1 ? wr.y : e == 2 ? wr.z : wr.w);
                z[2 * e] *= r * f.x;
                z[2 * e + 1] *= r * f.y;
            }
        }
        if (p.adjacent) {
            if (v * 8 < p.rot) {
#pragma unroll
                for (int e = 0; e < 8; e += 2) {
                    const float2 c = turns[v * 4 + e / 2];
                    const float a = z[e], b = z[e + 1];
                    z[e] = a * c.x - b * c.y;
                    z[e + 1] = b * c.x + a * c.y;
                }
            }
        } else {
            const int far = p.rot >> 4;                          // lanes between the values of a pair
            const bool low = v < far, turned = v < 2 * far;
            const int from = (tid & 31 & ~(LANES - 1)) + (turned ? low ? v + far : v - far : v);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float o = __shfl_sync(0xffffffffu, z[e], from);
                if (turned) {
                    const float2 c = turns[(low ? v : v - far) * 8 + e];
                    z[e] = z[e] * c.x + (low ? -o : o) * c.y;
                }
            }
        }
        if (on)
            *reinterpret_cast<uint4 *>(y + (size_t)head * p.width) =
                make_uint4(f4_from_float2<T>(z[0], z[1]), f4_from_float2<T>(z[2], z[3]), f4_from_float2<T>(z[4], z[5]), f4_from_float2<T>(z[6], z[7]));
    }
}

template <typename T> tman_status launch(const HeadParams &p0, int tokens, cudaStream_t s)
{
    HeadParams p = p0;
    const int lanes = p.width <= 64 ? 8 : p.width <= 128 ? 16 : 32, heads = p.q_heads + p.k_heads, at_once = kHeadThreads / lanes;
    const int sms = sm_count();
    if (sms <= 0) return TMAN_ERR_CUDA;
    // few tokens: their heads are spread over CTAs
    p.chunk = tokens < 4 * sms ? at_once : heads;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)tokens, (unsigned)((heads + p.chunk - 1) / p.chunk));
    cfg.blockDim = dim3(kHeadThreads);
    cfg.stream = s;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    auto kern = lanes == 8 ? norm_rotate_kernel<T, 8> : lanes == 16 ? norm_rotate_kernel<T, 16> : norm_rotate_kernel<T, 32>;
    return call_status(cudaLaunchKernelEx(&cfg, kern, p));
}

}  // namespace

tman_status launch_norm_rotate(const void *x, int ldx, void *y, int ldy, int dtype, int T, int q_heads, int k_heads, int width, int rot, int adjacent,
                               const void *q_weight, const void *k_weight, float eps, const int *positions, const float *inv_freq, cudaStream_t s)
{
    const HeadParams p = {x, y, q_weight, k_weight, positions, inv_freq, ldx, ldy, q_heads, k_heads, width, rot, adjacent, 0, eps};
    return dtype == kF4TypeHalf ? launch<__half>(p, T, s) : launch<__nv_bfloat16>(p, T, s);
}

}  // namespace tman
