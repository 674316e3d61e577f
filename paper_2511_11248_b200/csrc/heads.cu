// Norms of query and key heads and the rotation by their position, in one pass.
//
// For each token and head: z = x / sqrt(mean(x^2) + eps) * weight (no weight: z = x), then each pair of the first `rot` values of z is turned by
// position * inv_freq[i]: pairs (i, i + rot/2), or (2i, 2i + 1).  Bound by reading and writing the heads once.
// A head is a group of 8, 16 or 32 lanes with two runs of four values each, which are each other's partners: columns 4 v .. and rot / 2 + 4 v .., or
// 8 v .. (neighbours as pairs, and what is not turned); so that no value is passed on (with eight values in a row a lane, exchanged by shuffles, instructions
// were the bound, 8191 x 32 heads of 128 45 us).  All in 32 bits, rounded once.  Angles are products of a position and a frequency, whole turns taken off, in 64 bits: in 32 a position of 100000 would
// leave 2^-8 of a turn.  Now 8191 x 32 heads take 35 us (floor 20.5), bound by instructions still.  Sines and cosines are worked out once for all heads of a token.  A CTA has so many tokens that every group has eight heads,
// all asked for at once: with one token a CTA its latency, from the position to the last store, was paid 8191 times over (8191 x 32 heads of 128
// 48 us).  Few tokens are spread over CTAs, a head a group.
#include "i8.cuh"

#include <type_traits>

namespace tman {
namespace {

constexpr int kHeadThreads = 256, kHeadHeld = 8, kHeadTurns = 1024;

struct HeadParams {
    const void *x;
    void *y;
    const void *q_weight, *k_weight;
    const int *positions;
    const float *inv_freq;
    int T, ldx, ldy, q_heads, k_heads, width, rot, adjacent, tokens, chunk;       // of a CTA: tokens, heads of each of them
    uint32_t chunk_mul;                  // 2^32 / chunk, rounded up; 0: a chunk of one
    float eps, inv_width;
};

template <typename T> __device__ __forceinline__ uint4 load_runs(const T *x, int lo, int hi)
{
    uint4 v;
    asm volatile("ld.global.v2.u32 {%0, %1}, [%2];" : "=r"(v.x), "=r"(v.y) : "l"(x + lo) : "memory");
    asm volatile("ld.global.v2.u32 {%0, %1}, [%2];" : "=r"(v.z), "=r"(v.w) : "l"(x + hi) : "memory");
    return v;
}

template <typename T, int LANES, int TURNS, bool ADJACENT>
__global__ void __launch_bounds__(kHeadThreads) norm_rotate_kernel(const __grid_constant__ HeadParams p)
{
    __shared__ float2 turns[kHeadTurns];
    constexpr int AT_ONCE = kHeadThreads / LANES;
    const int tid = threadIdx.x, group = tid / LANES, v = tid & (LANES - 1), heads = p.q_heads + p.k_heads, half = p.rot >> 1;
    const int token0 = blockIdx.x * p.tokens, tokens = min(p.tokens, p.T - token0), head0 = blockIdx.y * p.chunk, chunk = min(p.chunk, heads - head0);
    const bool in = v * 8 < p.width, far = !ADJACENT && v * 8 < p.rot, turned = v * 8 < p.rot;
    const int lo = far ? v * 4 : v * 8, hi = far ? half + v * 4 : v * 8 + 4;
    float2 wq[4], wk[4];                                         // the weights of this lane's columns
    // the group's n-th head: its token among the CTA's (none: tokens), its number
    auto head_of = [&](int n, int &token, int &head) {
        const int unit = group + n * AT_ONCE;
        token = p.chunk_mul ? (int)__umulhi((uint32_t)unit, p.chunk_mul) : unit;
        head = unit - token * p.chunk;
        if (head >= chunk || token > tokens) token = tokens;
        head += head0;
    };
    grid_wait();                         // (the rows, their positions and the output are other kernels' until here)
    grid_launch_next();
    uint4 held[TURNS];
#pragma unroll
    for (int n = 0; n < TURNS; ++n) {
        int token, head;
        head_of(n, token, head);
        held[n] = make_uint4(0, 0, 0, 0);
        if (in && token < tokens) held[n] = load_runs(static_cast<const T *>(p.x) + (size_t)(token0 + token) * p.ldx + (size_t)head * p.width, lo, hi);
    }
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const T *w = static_cast<const T *>(k ? p.k_weight : p.q_weight);
        const uint4 r = w && in ? load_runs(w, lo, hi) : make_uint4(0, 0, 0, 0);
        float2 (&to)[4] = k ? wk : wq;
        to[0] = f4_to_float2<T>(r.x);
        to[1] = f4_to_float2<T>(r.y);
        to[2] = f4_to_float2<T>(r.z);
        to[3] = f4_to_float2<T>(r.w);
    }
    for (int i = tid; i < tokens * half; i += kHeadThreads) {
        const int token = i / half, k = i - token * half;
        int pos;
        asm volatile("ld.global.s32 %0, [%1];" : "=r"(pos) : "l"(p.positions + token0 + token) : "memory");
        double a = (double)pos * (double)ld_dependent(p.inv_freq + k);
        a -= rint(a * 0.15915494309189533577) * 6.283185307179586477;
        float s, c;
        sincosf((float)a, &s, &c);
        turns[token * half + (k & 3) * (half >> 2) + (k >> 2)] = make_float2(c, s);      // (a lane reads four in a row: so that lanes next to each other do)
    }
    __syncthreads();
#pragma unroll
    for (int n = 0; n < TURNS; ++n) {
        int token, head;
        head_of(n, token, head);
        if (!__any_sync(0xffffffffu, token < tokens)) break;
        const uint32_t mask = LANES == 32 ? 0xffffffffu : ((1u << (LANES & 31)) - 1u) << (tid & 31 & ~(LANES - 1));      // the group (others of the warp may have heads without a norm)
        const bool on = in && token < tokens;
        const float2 *turn = turns + min(token, tokens - 1) * half;
        const uint4 raw = held[n];
        float z[8];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float2 f = f4_to_float2<T>(e == 0 ? raw.x : e == 1 ? raw.y : e == 2 ? raw.z : raw.w);
            z[2 * e] = f.x;
            z[2 * e + 1] = f.y;
        }
        const bool query = head < p.q_heads;
        if (query ? p.q_weight != nullptr : p.k_weight != nullptr) {
            float eps = p.eps;
            const auto squares = [&] {
                float sum = 0.f;
#pragma unroll
                for (int e = 0; e < 8; ++e) sum = fmaf(z[e], z[e], sum);
#pragma unroll
                for (int d = LANES / 2; d > 0; d >>= 1) sum += __shfl_xor_sync(mask, sum, d);
                return fmaf(sum, p.inv_width, eps);
            };
            float mean = squares();
            if constexpr (!std::is_same<T, __half>::value) {
                if (mean > 0x1p120f || mean < 0x1p-100f) {       // beyond 32 bits: of bf16 values that are very large or small
                    const float k = mean > 1.f ? 0x1p-80f : 0x1p80f;
#pragma unroll
                    for (int e = 0; e < 8; ++e) z[e] *= k;
                    eps = eps * k * k;
                    mean = squares();
                }
            }
            const float r = rsqrtf(mean);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                z[2 * e] *= r * (query ? wq[e].x : wk[e].x);
                z[2 * e + 1] *= r * (query ? wq[e].y : wk[e].y);
            }
        }
        if (turned) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {                        // pair e: values e and e + 4, or 2 e and 2 e + 1
                const float2 c = turn[e * (half >> 2) + v];
                float &a = z[ADJACENT ? 2 * e : e], &b = z[ADJACENT ? 2 * e + 1 : e + 4];
                const float x = a, y = b;
                a = x * c.x - y * c.y;
                b = y * c.x + x * c.y;
            }
        }
        if (on) {
            T *to = static_cast<T *>(p.y) + (size_t)(token0 + token) * p.ldy + (size_t)head * p.width;
            *reinterpret_cast<uint2 *>(to + lo) = make_uint2(f4_from_float2<T>(z[0], z[1]), f4_from_float2<T>(z[2], z[3]));
            *reinterpret_cast<uint2 *>(to + hi) = make_uint2(f4_from_float2<T>(z[4], z[5]), f4_from_float2<T>(z[6], z[7]));
        }
    }
}

template <typename T> tman_status launch(HeadParams p, cudaStream_t s)
{
    const int lanes = p.width <= 64 ? 8 : p.width <= 128 ? 16 : 32, heads = p.q_heads + p.k_heads, at_once = kHeadThreads / lanes;
    const int sms = sm_count();
    if (sms <= 0) return TMAN_ERR_CUDA;
    const bool many = (long long)p.T * heads >= 4ll * sms * at_once;     // (fewer: a head a group)
    const int room = many ? kHeadHeld * at_once : at_once;
    p.chunk = heads < room ? heads : room;
    p.tokens = many ? room / p.chunk : 1;
    const int fit = kHeadTurns / (p.rot > 0 ? p.rot / 2 : 1);
    if (p.tokens > fit) p.tokens = fit;
    p.chunk_mul = p.chunk == 1 ? 0u : 0xFFFFFFFFu / (uint32_t)p.chunk + 1u;
    if ((heads + p.chunk - 1) / p.chunk > 65535) return TMAN_ERR_SHAPE;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)((p.T - 1) / p.tokens + 1), (unsigned)((heads + p.chunk - 1) / p.chunk));
    cfg.blockDim = dim3(kHeadThreads);
    cfg.stream = s;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    const auto of = [&](auto l) {
        constexpr int L = decltype(l)::value;
        return p.adjacent ? many ? norm_rotate_kernel<T, L, kHeadHeld, true> : norm_rotate_kernel<T, L, 1, true>
                          : many ? norm_rotate_kernel<T, L, kHeadHeld, false> : norm_rotate_kernel<T, L, 1, false>;
    };
    auto kern = lanes == 8 ? of(std::integral_constant<int, 8>()) : lanes == 16 ? of(std::integral_constant<int, 16>()) : of(std::integral_constant<int, 32>());
    return call_status(cudaLaunchKernelEx(&cfg, kern, p));
}

}  // namespace

tman_status launch_norm_rotate(const void *x, int ldx, void *y, int ldy, int dtype, int T, int q_heads, int k_heads, int width, int rot, int adjacent,
                               const void *q_weight, const void *k_weight, float eps, const int *positions, const float *inv_freq, cudaStream_t s)
{
    const HeadParams p = {x, y, q_weight, k_weight, positions, inv_freq, T, ldx, ldy, q_heads, k_heads, width, rot, adjacent, 1, 0, 0, eps, 1.f / (float)width};
    return dtype == kF4TypeHalf ? launch<__half>(p, s) : launch<__nv_bfloat16>(p, s);
}

}  // namespace tman
