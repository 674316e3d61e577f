// Products of up to eight rows: y[m][n] = a_scale[m] w_scale[n] sum_k a[m][k] w[n][k], weights [N][K] in bytes.
//
// What bounds it is reading the weights once.  Every SM has a CTA with an equal share of the channels, cut into units of 16 channels x 128 values of k that
// its 16 warps take in turn.  A lane's 16-byte pieces of two channels are the A operands of mma.sync.m16n8k32 as they come (the order of k inside 64
// values is the same for both operands, so it is free); the rows of a are the columns of B, unused ones zero.  Each lane copies its own pieces into its
// own places of a ring, asynchronously, so that some 190 KB an SM are under way and no barrier is needed.  Sums of the warps meet in shared memory
// as integers: exact, whatever their order.
// Codes come from global memory, a unit's as its weights are waited for.  Rows of 16 bits are quantized by every CTA itself, which spares a launch, as
// long as there are few values (i8_matmul.cu).
// In a graph, weights not in L2 (the product alone; floor): 1 x 4096 x 14336 13.7 us (9.0), 8 x 14336 x 4096 13.4 (9.0), 8 x 18944 x 3584 15.9 (10.4), 1 x 4096 x 1024 3.6:
// 4.9 TB/s with some 3 us around the stream.  Other ways: weights straight to registers, two batches of eight loads (1 x 4096 x 14336 14.9); TMA
// boxes of 64 bytes x the CTA's channels (12.4, but 4096 x 1024 5.9 and 14336 x 4096 21: the rows of a box cost two nanoseconds each); units channels
// first, the codes fetched again for each (8 x 4096 x 14336 16.4, now 14.1).
#pragma once

#include "i8.cuh"

namespace tman {
namespace {

constexpr int kI8Warps = 16, kI8Threads = 32 * kI8Warps, kI8Channels = 128, kI8Unit = 2048, kI8Slots = 6;
constexpr int kI8StreamSmem = 216 * 1024;
constexpr int kI8FusedValues = 16384, kI8FusedSlots = 4;
static_assert(kI8Warps * kI8FusedSlots * kI8Unit + kI8FusedValues + 8 * 127 + 8 * 8 * kI8Channels <= kI8StreamSmem &&
              kI8Warps * kI8Slots * kI8Unit + 8 * 8 * kI8Channels <= kI8StreamSmem, "ring, codes and sums fit");
constexpr int kI8FusedBytes = 64 * 1024; // codes in shared memory at most

struct I8StreamParams {
    const int8_t *w;
    const void *x;                       // 16-bit rows, or codes [M][K]
    const float *w_scale, *a_scale;
    void *y;
    int ldw, ldx, ldy, M, K, N, channels, groups;
};

__device__ __forceinline__ void i8_mma(int (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    asm("mma.sync.aligned.m16n8k32.row.col.s32.s8.s8.s32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+r"(c[0]), "+r"(c[1]), "+r"(c[2]), "+r"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void i8_copy16(uint32_t dst, const void *src)
{
    asm volatile("cp.async.cg.shared.global.L2::128B [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
template <int N> __device__ __forceinline__ void i8_copy_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// TILES: 16 channels at most that a group has (few: the code is short, which the first call of a kernel after others feels).
template <typename T, bool CODES, int SLOTS, int TILES>
__global__ void __launch_bounds__(kI8Threads, 1) i8_stream_kernel(const __grid_constant__ I8StreamParams p)
{
    extern __shared__ __align__(1024) uint8_t stream_smem[];
    __shared__ uint32_t tops[kI8Warps][8];
    __shared__ float scales[8];
    const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31, g = lane >> 2, t = lane & 3;
    const int n0 = blockIdx.x * p.groups * p.channels, tiles = (p.channels + 15) >> 4, blocks = (p.K + 127) >> 7;
    // A warp's units of a group: all tiles of every 16th block, and an equal part of the tiles of the blocks that are left.
    const int rounds = blocks / kI8Warps, rest = blocks % kI8Warps * tiles, rest0 = rest * warp / kI8Warps, units = rounds * tiles + rest * (warp + 1) / kI8Warps - rest0;
    const uint32_t ring = smem_u32(stream_smem) + warp * (SLOTS * kI8Unit) + lane * 16;
    const uint8_t *ring_at = stream_smem + warp * (SLOTS * kI8Unit) + lane * 16;
    uint8_t *codes = stream_smem + kI8Warps * SLOTS * kI8Unit;                              // [block][m][128]
    int *sums = reinterpret_cast<int *>(codes + (CODES ? 0 : (size_t)blocks * 128 * p.M));   // [2][channel][m]
    for (int i = tid; i < 2 * p.channels * p.M; i += kI8Threads) sums[i] = 0;

    struct Unit { int i, block, tile; };                         // the i-th of the warp's
    const int rest_block = rounds * kI8Warps + (tiles == 1 ? rest0 : rest0 / tiles), rest_tile = rest0 - (rest_block - rounds * kI8Warps) * tiles;
    const Unit first = {0, rounds > 0 ? warp : rest_block, rounds > 0 ? 0 : rest_tile};
    auto on = [&](Unit &u) {
        const bool round = u.i < rounds * tiles;
        if (++u.i == rounds * tiles) {
            u.block = rest_block;
            u.tile = rest_tile;
        } else if (++u.tile == tiles) {
            u.tile = 0;
            u.block += round ? kI8Warps : 1;
        }
    };
    Unit lu = first;                                           // what is loaded next
    int ln = n0;
    auto pieces_of = [&](auto &&take) {                          // this lane's pieces of the unit: (place, address)
        const int k = lu.block * 128 + 16 * t, ch = lu.tile * 16 + g, count = min(p.channels, p.N - ln);
        const int8_t *at = p.w + (size_t)(ln + ch) * p.ldw + k;
        if (ch < count) {
            if (k < p.K) take(0, at);
            if (k + 64 < p.K) take(1, at + 64);
        }
        if (ch + 8 < count) {
            if (k < p.K) take(2, at + (size_t)8 * p.ldw);
            if (k + 64 < p.K) take(3, at + (size_t)8 * p.ldw + 64);
        }
    };
    const int n_end = min(n0 + p.groups * p.channels, p.N);
    auto load = [&](int slot) {
        if (ln < n_end && units > 0) {
            pieces_of([&](int i, const int8_t *at) { i8_copy16(ring + slot * kI8Unit + i * 512, at); });
            on(lu);
            if (lu.i == units) {
                lu = first;
                ln += p.channels;
            }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
#pragma unroll 1
    for (int i = 0; i < SLOTS - 1 && i < units; ++i) {           // the first weights on their way to L2 before the wait for the kernel ahead
        pieces_of([](int, const int8_t *at) { asm volatile("prefetch.global.L2 [%0];" ::"l"(at)); });
        on(lu);
    }
    lu = first;
    grid_wait();
    grid_launch_next();
#pragma unroll 1
    for (int i = 0; i < SLOTS - 1; ++i) load(i);

    if constexpr (CODES) {
        if (tid < p.M) scales[tid] = ld_dependent(p.a_scale + tid);
    } else {
        const T *x = static_cast<const T *>(p.x);
        const int pieces = p.K >> 3;
#pragma unroll 1
        for (int m = 0; m < p.M; ++m) {
            uint32_t top = 0;
#pragma unroll 4
            for (int i = tid; i < pieces; i += kI8Threads) {
                const uint4 v = ld_dependent(reinterpret_cast<const uint4 *>(x + (size_t)m * p.ldx) + i);
                top = i8_larger(top, i8_larger(i8_larger(i8_magnitudes(v.x), i8_magnitudes(v.y)), i8_larger(i8_magnitudes(v.z), i8_magnitudes(v.w))));
            }
            top = __reduce_max_sync(0xffffffffu, max(top & 0xFFFFu, top >> 16));
            if (lane == 0) tops[warp][m] = top;
        }
        __syncthreads();
        if (tid < p.M) {
            uint32_t v = 0;
#pragma unroll
            for (int i = 0; i < kI8Warps; ++i) v = max(v, tops[i][tid]);
            scales[tid] = v == 0 ? 1.f : i8_scale<T>(v);
        }
        __syncthreads();
        for (int m = 0; m < p.M; ++m) {
            const I8Divisor d(scales[m]);
#pragma unroll 4
            for (int i = tid; i < blocks * 16; i += kI8Threads) {
                uint2 v = make_uint2(0, 0);
                if (i < pieces) v = i8_codes<T>(d, ld_dependent(reinterpret_cast<const uint4 *>(x + (size_t)m * p.ldx) + i));
                *reinterpret_cast<uint2 *>(codes + ((size_t)(i >> 4) * p.M + m) * 128 + (i & 15) * 8) = v;
            }
        }
    }
    __syncthreads();

    const int8_t *a = static_cast<const int8_t *>(p.x) + (size_t)min(g, p.M - 1) * p.K + 16 * t;
    auto codes_of = [&](int block, uint4 (&v)[2]) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            v[i] = make_uint4(0, 0, 0, 0);
            if constexpr (CODES) {
                if (g < p.M && block * 128 + 64 * i + 16 * t < p.K) v[i] = ld_dependent(reinterpret_cast<const uint4 *>(a + (size_t)block * 128 + 64 * i));
            } else {
                if (g < p.M) v[i] = *reinterpret_cast<const uint4 *>(codes + ((size_t)block * p.M + g) * 128 + 64 * i + 16 * t);
            }
        }
    };
    int slot = 0;
    uint4 next[2];
    Unit u = first;
    if (units > 0) codes_of(u.block, next);
    for (int group = 0, n = n0; n < n_end; ++group, n += p.channels) {
        int c[TILES][4] = {};
        for (u = first; u.i < units;) {
            // the warp's tiles of a block
            const int t0 = u.tile, t1 = min(tiles, t0 + units - u.i);
            const uint4 q0 = next[0], q1 = next[1];
            for (int i = t0; i < t1; ++i) on(u);
            codes_of(u.i < units ? u.block : first.block, next);
#pragma unroll
            for (int j = 0; j < TILES; ++j)
                if (j >= t0 && j < t1) {
                    load(slot == 0 ? SLOTS - 1 : slot - 1);
                    i8_copy_wait<SLOTS - 1>();
                    const uint4 *at = reinterpret_cast<const uint4 *>(ring_at + slot * kI8Unit);
                    const uint4 x0 = at[0], x1 = at[32], y0 = at[64], y1 = at[96];
                    i8_mma(c[j], x0.x, y0.x, x0.y, y0.y, q0.x, q0.y);
                    i8_mma(c[j], x0.z, y0.z, x0.w, y0.w, q0.z, q0.w);
                    i8_mma(c[j], x1.x, y1.x, x1.y, y1.y, q1.x, q1.y);
                    i8_mma(c[j], x1.z, y1.z, x1.w, y1.w, q1.z, q1.w);
                    if (++slot == SLOTS) slot = 0;
                }
        }
        int *sum = sums + (group & 1) * p.channels * p.M;
#pragma unroll
        for (int j = 0; j < TILES; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int ch = j * 16 + g + (e >> 1) * 8, m = 2 * t + (e & 1);
                if (ch < p.channels && m < p.M) atomicAdd(sum + ch * p.M + m, c[j][e]);
            }
        __syncthreads();
        for (int i = tid; i < p.channels * p.M; i += kI8Threads) {
            const int m = i / p.channels, ch = i - m * p.channels;
            if (n + ch < p.N)
                static_cast<T *>(p.y)[(size_t)m * p.ldy + n + ch] = f4_from_float<T>(i8_scaled(sum[ch * p.M + m], scales[m], ld_dependent(p.w_scale + n + ch)));
            sum[ch * p.M + m] = 0;
        }
    }
}

// Rows of codes, or 16-bit rows of kI8FusedValues values at most, whose codes are in shared memory (then the ring is shorter).
template <typename T, bool CODES, int TILES>
tman_status launch_i8_stream_as(I8StreamParams p, int sms, cudaStream_t s);

template <typename T, bool CODES>
tman_status launch_i8_stream(const I8StreamParams &p, cudaStream_t s)
{
    const int sms = sm_count();
    if (sms <= 0) return TMAN_ERR_CUDA;
    return (p.N + sms - 1) / sms <= 32 ? launch_i8_stream_as<T, CODES, 2>(p, sms, s) : launch_i8_stream_as<T, CODES, 8>(p, sms, s);
}

template <typename T, bool CODES, int TILES>
tman_status launch_i8_stream_as(I8StreamParams p, int sms, cudaStream_t s)
{
    constexpr int SLOTS = CODES ? kI8Slots : kI8FusedSlots;
    auto kern = i8_stream_kernel<T, CODES, SLOTS, TILES>;
    static std::atomic<bool> raised[kMaxDevices];
    int dev = 0;
    if (!device_info(&dev)) return TMAN_ERR_CUDA;
    // an equal share of the channels for every SM, in groups of at most 128
    const int share = (p.N + sms - 1) / sms;
    p.groups = (share + kI8Channels - 1) / kI8Channels;
    p.channels = (share + p.groups - 1) / p.groups;
    const long long own = (long long)p.channels * p.groups;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)((p.N + own - 1) / own));
    cfg.blockDim = dim3(kI8Threads);
    cfg.dynamicSmemBytes = (size_t)kI8Warps * SLOTS * kI8Unit + (CODES ? 0 : (size_t)(p.K + 127) / 128 * 128 * p.M) + (size_t)p.channels * p.M * 8;
    cfg.stream = s;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return launch_with_smem(kern, kI8StreamSmem, dev, raised, [&] { return cudaLaunchKernelEx(&cfg, kern, p); });
}

}  // namespace
}  // namespace tman
