// Products of up to eight rows: y[m][n] = a_scale[m] w_scale[n] sum_k a[m][k] w[n][k], weights [N][K] in bytes.
//
// What bounds it is reading the weights once.  Every SM has a CTA with an equal share of the channels; each 64 values of k of its channels belong
// to one of 16 warps, so that a row of weights is read in runs of 1 KB by the CTA.  A lane's 16-byte pieces of two rows are the A operands of two
// mma.sync.m16n8k32 as they come (the order of k inside 64 values is the same for both operands, so it is free); the rows of a, in shared memory,
// are the columns of B, unused ones zero.  Sums of the warps meet in shared memory as integers: exact, whatever their order.
// Rows of 16 bits are quantized by every CTA itself: that spares a launch.
#pragma once

#include "i8.cuh"

namespace tman {
namespace {

constexpr int kI8Threads = 512, kI8Warps = kI8Threads / 32, kI8Batch = 4, kI8Channels = 512;
constexpr int kI8Codes = 192 * 1024;     // bytes of codes in shared memory at most (beside 16 KB of sums)

struct I8StreamParams {
    const int8_t *w;
    const void *x;                       // 16-bit rows, or codes [M][K]
    const float *w_scale, *a_scale;
    void *y;
    int ldw, ldx, ldy, M, K, N, channels;
};

__device__ __forceinline__ uint4 i8_load_weights(const int8_t *p)
{
    uint4 v;
    asm volatile("ld.global.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p) : "memory");
    return v;
}
__device__ __forceinline__ void i8_mma(int (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    asm("mma.sync.aligned.m16n8k32.row.col.s32.s8.s8.s32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+r"(c[0]), "+r"(c[1]), "+r"(c[2]), "+r"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

template <typename T, bool CODES>
__global__ void __launch_bounds__(kI8Threads, 1) i8_stream_kernel(const __grid_constant__ I8StreamParams p)
{
    extern __shared__ __align__(16) uint8_t smem[];
    __shared__ uint32_t tops[kI8Warps][8];
    __shared__ float scales[8];
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, t = lane & 3;
    const int n0 = blockIdx.x * p.channels, count = min(p.channels, p.N - n0), chunks = (p.K + 63) >> 6;
    uint8_t *codes = smem;                                       // [chunk][m][64]
    int *sums = reinterpret_cast<int *>(smem + (size_t)chunks * 64 * p.M);      // [channel][m]
    for (int i = tid; i < count * p.M; i += kI8Threads) sums[i] = 0;
    grid_wait();
    grid_launch_next();

    const int mine = (chunks - warp + kI8Warps - 1) / kI8Warps, batches = (mine + kI8Batch - 1) / kI8Batch, tiles = (count + 15) >> 4;
    const int8_t *w0 = p.w + (size_t)(n0 + g) * p.ldw + 16 * t;
    auto load = [&](uint4 (&r)[kI8Batch][2], int tile, int b) {
#pragma unroll
        for (int u = 0; u < kI8Batch; ++u) {
            const int j = b * kI8Batch + u, k = (warp + kI8Warps * j) * 64, ch = tile * 16 + g;
            const bool in = j < mine && k + 16 * t < p.K;
            r[u][0] = in && ch < count ? i8_load_weights(w0 + (size_t)(tile * 16) * p.ldw + k) : make_uint4(0, 0, 0, 0);
            r[u][1] = in && ch + 8 < count ? i8_load_weights(w0 + (size_t)(tile * 16 + 8) * p.ldw + k) : make_uint4(0, 0, 0, 0);
        }
    };
    uint4 r[2][kI8Batch][2];
    int c[4] = {0, 0, 0, 0};
    int lt = 0, lb = 0;                                          // what is loaded next
    auto load_next = [&](uint4 (&into)[kI8Batch][2]) {
        if (lt < tiles && batches > 0) load(into, lt, lb);
        if (++lb >= batches) { lb = 0; ++lt; }
    };
    load_next(r[0]);

    if constexpr (CODES) {
        const int pieces = chunks * 4;
        for (int i = tid; i < pieces * p.M; i += kI8Threads) {
            const int m = i / pieces, q = i - m * pieces;
            uint4 v = make_uint4(0, 0, 0, 0);
            if (q * 16 < p.K) v = ld_dependent(reinterpret_cast<const uint4 *>(static_cast<const int8_t *>(p.x) + (size_t)m * p.K) + q);
            *reinterpret_cast<uint4 *>(codes + ((size_t)(q >> 2) * p.M + m) * 64 + (q & 3) * 16) = v;
        }
        if (tid < p.M) scales[tid] = ld_dependent(p.a_scale + tid);
    } else {
        const T *x = static_cast<const T *>(p.x);
        const int pieces = p.K >> 3;
        uint32_t top[8];
#pragma unroll
        for (int m = 0; m < 8; ++m) {
            top[m] = 0;
            if (m < p.M)
                for (int i = tid; i < pieces; i += kI8Threads) {
                    const uint4 v = ld_dependent(reinterpret_cast<const uint4 *>(x + (size_t)m * p.ldx) + i);
                    top[m] = i8_larger(top[m], i8_larger(i8_larger(i8_magnitudes(v.x), i8_magnitudes(v.y)), i8_larger(i8_magnitudes(v.z), i8_magnitudes(v.w))));
                }
            if (m < p.M) {
                top[m] = max(top[m] & 0xFFFFu, top[m] >> 16);
                top[m] = __reduce_max_sync(0xffffffffu, top[m]);
                if (lane == 0) tops[warp][m] = top[m];
            }
        }
        __syncthreads();
        if (tid < p.M) {
            uint32_t v = 0;
            for (int i = 0; i < kI8Warps; ++i) v = max(v, tops[i][tid]);
            scales[tid] = v == 0 ? 1.f : i8_scale<T>(v);
        }
        __syncthreads();
        for (int m = 0; m < p.M; ++m) {
            const I8Divisor d(scales[m]);
            for (int i = tid; i < chunks * 8; i += kI8Threads) {
                uint2 v = make_uint2(0, 0);
                if (i < pieces) v = i8_codes<T>(d, ld_dependent(reinterpret_cast<const uint4 *>(x + (size_t)m * p.ldx) + i));
                *reinterpret_cast<uint2 *>(codes + ((size_t)(i >> 3) * p.M + m) * 64 + (i & 7) * 8) = v;
            }
        }
    }
    __syncthreads();

    auto multiply = [&](const uint4 (&v)[kI8Batch][2], int b) {
#pragma unroll
        for (int u = 0; u < kI8Batch; ++u) {
            const int j = b * kI8Batch + u;
            if (j >= mine) break;
            uint4 q = make_uint4(0, 0, 0, 0);
            if (g < p.M) q = *reinterpret_cast<const uint4 *>(codes + ((size_t)(warp + kI8Warps * j) * p.M + g) * 64 + 16 * t);
            i8_mma(c, v[u][0].x, v[u][1].x, v[u][0].y, v[u][1].y, q.x, q.y);
            i8_mma(c, v[u][0].z, v[u][1].z, v[u][0].w, v[u][1].w, q.z, q.w);
        }
    };
    auto put = [&](int tile) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int ch = tile * 16 + g + (e >> 1) * 8, m = 2 * t + (e & 1);
            if (ch < count && m < p.M) atomicAdd(sums + ch * p.M + m, c[e]);
            c[e] = 0;
        }
    };
    if (batches > 0)
        for (int tile = 0, b = 0, which = 0; tile < tiles;) {
            if (which == 0) {
                load_next(r[1]);
                multiply(r[0], b);
            } else {
                load_next(r[0]);
                multiply(r[1], b);
            }
            which ^= 1;
            if (++b == batches) {
                put(tile++);
                b = 0;
            }
        }
    __syncthreads();
    for (int i = tid; i < count * p.M; i += kI8Threads) {
        const int m = i / count, ch = i - m * count;
        static_cast<T *>(p.y)[(size_t)m * p.ldy + n0 + ch] = f4_from_float<T>(i8_scaled(sums[ch * p.M + m], scales[m], ld_dependent(p.w_scale + n0 + ch)));
    }
}

template <typename T, bool CODES>
tman_status launch_i8_stream(I8StreamParams p, cudaStream_t s)
{
    auto kern = i8_stream_kernel<T, CODES>;
    static std::atomic<bool> raised[kMaxDevices];
    int dev = 0;
    const DeviceInfo *info = device_info(&dev);
    if (!info) return TMAN_ERR_CUDA;
    const int sms = info->sms.load(std::memory_order_relaxed);
    p.channels = (p.N + sms - 1) / sms;
    if (p.channels > kI8Channels) p.channels = kI8Channels;
    // rows that fit beside their sums; more than that take more passes over the weights
    const int chunks = (p.K + 63) / 64, fit = kI8Codes / (chunks * 64), all = p.M;
    for (int m = 0; m < all; m += p.M) {
        p.M = fit < all - m ? fit : all - m;
        I8StreamParams q = p;
        q.x = CODES ? static_cast<const void *>(static_cast<const int8_t *>(p.x) + (size_t)m * p.K) : static_cast<const void *>(static_cast<const T *>(p.x) + (size_t)m * p.ldx);
        q.y = static_cast<T *>(p.y) + (size_t)m * p.ldy;
        if (CODES) q.a_scale = p.a_scale + m;
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3((unsigned)((p.N + p.channels - 1) / p.channels));
        cfg.blockDim = dim3(kI8Threads);
        cfg.dynamicSmemBytes = (size_t)chunks * 64 * q.M + (size_t)p.channels * q.M * 4;
        cfg.stream = s;
        cudaLaunchAttribute attr[1];
        attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr[0].val.programmaticStreamSerializationAllowed = 1;
        cfg.attrs = attr;
        cfg.numAttrs = 1;
        const tman_status st = launch_with_smem(kern, kI8Codes + kI8Channels * 32, dev, raised, [&] { return cudaLaunchKernelEx(&cfg, kern, q); });
        if (st != TMAN_OK) return st;
    }
    return TMAN_OK;
}

}  // namespace
}  // namespace tman
