// Products of many rows: y[m][n] = a_scale[m] w_scale[n] sum_k a[m][k] w[n][k], both operands in 8-bit integers on the tensor cores
// (tcgen05.mma.kind::i8, sums exact in 32 bits).
//
// A pair of CTAs (cta_group::2) has a tile of 256 channels (the rows of the tensor-core tile, 128 a CTA) x up to 256 tokens (its columns, each CTA
// loads half of them).  128 bytes of k of both operands are a stage of a ring, brought by TMA into 128-byte swizzled tiles; one thread of the pair
// issues the MMAs.  Tensor memory holds two accumulators of 256 columns, so that a tile's epilogue runs behind the next tile's MMAs.
// What bounds it: 256 x 256 x 128 products take a pair 512 clocks, in which each CTA takes 32 KB from L2; long calls by the power limit: 8192 x 4096 x 14336 295 us (3.27 POPS,
// twice the measured bf16 rate), 8192 x 18944 x 3584 340 to 355, 2048 x 4096 x 14336 79.  One round of tiles has start and epilogue around it: 777 x 3584 x 4608 15.4
// us, 7.5 of them MMAs; few tokens stream the weights: 40 x 4096 x 14336 14 to 16 (floor 9.2).
#pragma once

#include "i8_stream.cuh"

#include <type_traits>

namespace tman {
namespace {

constexpr int kI8PairThreads = 320;      // warp 0: loads, warp 1: MMAs (of the pair's first CTA), warps 2..9: epilogue
constexpr int kI8PairCols = 256, kI8PairStages = 8;
constexpr int kI8PairSmem = 222 * 1024;
constexpr uint32_t kI8PairA = 128 * 128;  // bytes of a CTA's channels in a stage
constexpr size_t kI8StreamBytes = (size_t)64 << 20;

struct I8PairParams {
    const float *w_scale, *a_scale;
    void *y;
    uint32_t *status;
    int M, K, N, ldy, nt, tiles_m, tiles_n, rows_fastest, stream_y, stages, split_sh;
};

__device__ __forceinline__ void tcgen05_mma2_i8(uint32_t d_tmem, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t accumulate)
{
    asm volatile(
        "{\n.reg .pred p;\n"
        "setp.ne.b32 p, %4, 0;\n"
        "tcgen05.mma.cta_group::2.kind::i8 [%0], %1, %2, %3, p;\n}\n"
        ::"r"(d_tmem), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accumulate) : "memory");
}
__device__ __forceinline__ void tma_prefetch_2d(const CUtensorMap *tmap, int x, int y)
{
    asm volatile("cp.async.bulk.prefetch.tensor.2d.L2.global.tile [%0, {%1, %2}];" ::"l"(reinterpret_cast<uint64_t>(tmap)), "r"(x), "r"(y) : "memory");
}

template <typename T>
__global__ void __launch_bounds__(kI8PairThreads) i8_pair_kernel(const __grid_constant__ CUtensorMap map_w, const __grid_constant__ CUtensorMap map_a,
                                                                 const __grid_constant__ I8PairParams p)
{
    extern __shared__ __align__(1024) uint8_t pair_smem[];
    __shared__ __align__(8) uint64_t full_bar[kI8PairStages], empty_bar[kI8PairStages], accf_bar[2], acce_bar[2], sums_bar;
    __shared__ uint32_t tmem_slot;
    __shared__ float token_scale[8][kI8PairCols / 2];            // of an epilogue warp's tokens
    const int warp = __shfl_sync(0xffffffffu, (int)threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
    // a cluster: the pairs with the shares of k of a tile, one tile each (split > 1), or one pair that walks over tiles
    const uint32_t crank = cluster_ctarank(), rank = crank & 1u, share = crank >> 1;
    const int worker = blockIdx.x >> (1 + p.split_sh), workers = gridDim.x >> (1 + p.split_sh), tiles = p.tiles_m * p.tiles_n, split = 1 << p.split_sh;
    const uint32_t full0 = smem_u32(full_bar), empty0 = smem_u32(empty_bar), accf0 = smem_u32(accf_bar), acce0 = smem_u32(acce_bar), ring = (smem_u32(pair_smem) + 1023u) & ~1023u;
    const uint32_t stage_bytes = kI8PairA + (uint32_t)p.nt * 64u;
    const int all_steps = (p.K + 127) >> 7, step0 = all_steps * (int)share >> p.split_sh, steps = (all_steps * (int)(share + 1) >> p.split_sh) - step0;
    const int inner = p.rows_fastest ? p.tiles_m : p.tiles_n;
    auto tile_m = [&](int tile) { return p.rows_fastest ? tile % inner : tile / inner; };
    auto tile_n = [&](int tile) { return p.rows_fastest ? tile / inner : tile % inner; };
    bool ok = true;

    if (threadIdx.x == 0) {
        for (int s = 0; s < p.stages; ++s) {
            mbar_init(full0 + 8 * s, rank == 0 ? 2 : 1);         // the first CTA's: its own copies and the word of the other's
            mbar_init(empty0 + 8 * s, 1);
        }
        for (int b = 0; b < 2; ++b) {
            mbar_init(accf0 + 8 * b, 1);
            mbar_init(acce0 + 8 * b, 16);
        }
        mbar_init(smem_u32(&sums_bar), 1);
        if (split > 1) mbar_expect_tx(smem_u32(&sums_bar), (uint32_t)p.nt * 512u);
        fence_barrier_init();
    }
    __syncthreads();
    cluster_sync_all();

    const int total = worker < tiles ? ((tiles - 1 - worker) / workers + 1) * steps : 0;       // stages of this pair
    if (warp == 0 && elect_one() && worker < tiles) {            // weights of the first stages on their way to L2 before the wait for the kernel ahead
        prefetch_tensormap(&map_w);
        prefetch_tensormap(&map_a);
        const int n0 = tile_n(worker) * 256 + (int)rank * 128;
        for (int i = 0; n0 < p.N && i < min(p.stages, steps); ++i) tma_prefetch_2d(&map_w, (step0 + i) * 128, n0);
    }
    __syncwarp();
    grid_wait();
    if (warp == 1) {
        tcgen05_alloc2(smem_u32(&tmem_slot), 512);
        tcgen05_relinquish2();
    }
    tcgen05_fence_before();
    __syncthreads();
    cluster_sync_all();                  // both CTAs hold their tensor memory
    tcgen05_fence_after();
    grid_launch_next();
    const uint32_t tmem = __shfl_sync(0xffffffffu, tmem_slot, 0);
    const bool pairs_ok = (p.N & 1) == 0 && (p.ldy & 1) == 0 && (reinterpret_cast<uintptr_t>(p.y) & 3) == 0;

    if (warp == 0) {
        const bool lead = elect_one();
        int s = 0, i = 0;
        uint32_t ph = 1;                                         // (the first pass over the ring does not wait)
        for (int tile = worker; ok && tile < tiles; tile += workers) {
            const int n0 = tile_n(tile) * 256 + (int)rank * 128, m0 = tile_m(tile) * p.nt + (int)rank * (p.nt >> 1);
            for (int step = 0; step < steps; ++step, ++i) {
                if (i >= p.stages && !warp_all(mbar_wait(empty0 + 8 * s, ph))) { ok = false; break; }
                if (lead) {
                    const uint32_t st = ring + (uint32_t)s * stage_bytes, bar = full0 + 8 * s;
                    mbar_expect_tx(bar, stage_bytes);
                    tma_load_2d(st, &map_w, (step0 + step) * 128, n0, bar);
                    tma_load_2d(st + kI8PairA, &map_a, (step0 + step) * 128, m0, bar);
                }
                __syncwarp();
                if (++s == p.stages) { s = 0; ph ^= 1u; }
            }
        }
    } else if (warp == 1 && rank != 0) {                         // tells the first CTA when this one's part of a stage is there
        const bool lead = elect_one();
        const uint32_t to = mapa_u32(full0, crank & ~1u);
        int s = 0;
        uint32_t ph = 0;
        for (int i = 0; i < total; ++i) {
            if (!warp_all(mbar_wait(full0 + 8 * s, ph))) { ok = false; break; }
            if (lead) mbar_arrive_cluster(to + 8 * s);
            __syncwarp();
            if (++s == p.stages) { s = 0; ph ^= 1u; }
        }
    } else if (warp == 1) {
        const bool lead = elect_one();
        const uint32_t idesc = (2u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(p.nt >> 3) << 17) | ((256u >> 4) << 24);
        const uint64_t op0 = make_kmajor_sw128_desc(ring);
        const uint16_t both = (uint16_t)(3u << (crank & ~1u));
        int s = 0;
        uint32_t ph = 0, ti = 0;
        for (int tile = worker; ok && tile < tiles; tile += workers, ++ti) {
            const uint32_t b = ti & 1u, acc = tmem + b * kI8PairCols;
            if (!warp_all(mbar_wait(acce0 + 8 * b, ((ti >> 1) & 1u) ^ 1u))) { ok = false; break; }
            tcgen05_fence_after();
            for (int step = 0; step < steps; ++step) {
                const uint64_t wa = op0 + (uint32_t)s * (stage_bytes >> 4), xb = wa + (kI8PairA >> 4);
                if (!warp_all(mbar_wait(full0 + 8 * s, ph))) { ok = false; break; }
                tcgen05_fence_after();
                if (lead) {
#pragma unroll
                    for (uint32_t u = 0; u < 4; ++u) tcgen05_mma2_i8(acc, wa + 2 * u, xb + 2 * u, idesc, (step | (int)u) != 0);
                    tcgen05_commit2(empty0 + 8 * s, both);
                }
                __syncwarp();
                if (++s == p.stages) { s = 0; ph ^= 1u; }
            }
            if (lead) tcgen05_commit2(accf0 + 8 * b, both);
            __syncwarp();
        }
    } else if (split == 1) {
        // ---- epilogue: a warp has 32 channels (a lane each) x half of the tile's tokens, 16 at a time; neighbouring lanes exchange every other
        // token, so that a lane stores two adjacent channels of one
        const int quad = warp & 3, half = p.nt >> 1;
        const bool odd = (lane & 1) != 0;
        const uint32_t acce_lead = mapa_u32(acce0, crank & ~1u);
        const uint64_t y_policy = p.stream_y ? policy_evict_first() : policy_evict_normal();
        uint32_t ti = 0;
        for (int tile = worker; tile < tiles; tile += workers, ++ti) {
            const uint32_t b = ti & 1u;
            const int m0 = tile_m(tile) * p.nt, n = tile_n(tile) * 256 + (int)rank * 128 + quad * 32 + lane, n2 = n & ~1;
            const int end = p.M - m0, t0 = warp >= 6 ? half : 0;
            const bool put = n2 < p.N, put1 = n2 + 1 < p.N;
            bool whole = put && put1 && pairs_ok;
            const size_t row2 = 2 * (size_t)p.ldy;
            const float w0 = ld_dependent(p.w_scale + min(n2, p.N - 1)), w1 = ld_dependent(p.w_scale + min(n2 + 1, p.N - 1));
            T *y = static_cast<T *>(p.y) + (size_t)(m0 + (odd ? 1 : 0)) * p.ldy + n2;
            const uint32_t acc = tmem + ((uint32_t)(quad * 32) << 16) + b * kI8PairCols;
            auto store16 = [&](auto whole_c, int t, const uint32_t (&r)[16]) {
                constexpr bool WHOLE = decltype(whole_c)::value;
                const float *as = token_scale[warp - 2] + (t - t0) + (odd ? 1 : 0);
                T *yt = y + (size_t)t * p.ldy;
#pragma unroll
                for (int e = 0; e < 16; e += 2) {
                    const uint32_t got = __shfl_xor_sync(0xffffffffu, odd ? r[e] : r[e + 1], 1), keep = odd ? r[e + 1] : r[e];
                    const float f = as[e];
                    float c0, c1;
                    if constexpr (WHOLE) {
                        c0 = (float)(int)(odd ? got : keep) * (f * w0);
                        c1 = (float)(int)(odd ? keep : got) * (f * w1);
                    } else {
                        c0 = i8_scaled((int)(odd ? got : keep), f, w0);
                        c1 = i8_scaled((int)(odd ? keep : got), f, w1);
                    }
                    if constexpr (WHOLE) st_policy(yt, f4_from_float2<T>(c0, c1), y_policy);
                    else if (t + e + (odd ? 1 : 0) < end && put) {
                        yt[0] = f4_from_float<T>(c0);
                        if (put1) yt[1] = f4_from_float<T>(c1);
                    }
                    yt += row2;
                }
            };
            // (the tokens' scales before the sums are there: asked for sixteen at a time behind them, 777 x 3584 x 4608 spent 6.5 us here)
            __syncwarp();
            whole = whole && i8_ordinary(w0) && i8_ordinary(w1);
            for (int i = lane; i < half; i += 32) {
                const float f = ld_dependent(p.a_scale + min(m0 + t0 + i, p.M - 1));
                token_scale[warp - 2][i] = f;
                whole = whole && i8_ordinary(f);
            }
            __syncwarp();                        // (the lanes read one another's scales)
            whole = warp_all(whole);                             // pairs of channels, scales whose products are in range
            ok = warp_all(mbar_wait(accf0 + 8 * b, (ti >> 1) & 1u));
            if (!ok) break;
            tcgen05_fence_after();
#pragma unroll 1
            for (int t = t0; t < t0 + half && t < end; t += 16) {
                uint32_t r[16];
                tcgen05_ld_32x32b_x16(acc + (uint32_t)t, r);
                tcgen05_wait_ld();
                tcgen05_loaded(r);
                if (whole && t + 16 <= end) store16(std::true_type(), t, r);
                else store16(std::false_type(), t, r);
            }
            tcgen05_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive_cluster(acce_lead + 8 * b);
        }
    }
    if (split > 1) {
        // ---- shares of a tile: column c of the tile is added up by share c / own in the CTA of the same channels; everyone sends it its sums,
        // [share][own column][channel] on the ring, which is idle everywhere once all accumulators are complete
        const int own = p.nt >> p.split_sh, m0 = tile_m(worker) * p.nt + (int)share * own, n0 = tile_n(worker) * 256 + (int)rank * 128;
        const int ch = ((int)threadIdx.x & 63) * 2, n = n0 + ch;       // two channels of each of a thread's tokens
        float w0 = 0.f, w1 = 0.f;
        if (warp >= 2) {                                         // (scales before the sums are there)
            w0 = ld_dependent(p.w_scale + min(n, p.N - 1));
            w1 = ld_dependent(p.w_scale + min(n + 1, p.N - 1));
            for (int i = lane; i < own; i += 32) token_scale[warp - 2][i] = ld_dependent(p.a_scale + min(m0 + i, p.M - 1));
            ok = warp_all(mbar_wait(accf0, 0)) && ok;
            tcgen05_fence_after();
        }
        __syncwarp();
        cluster_sync_all();
        if (warp >= 2) {
            const int quad = warp & 3, half = p.nt >> 1, t0 = warp >= 6 ? half : 0;
#pragma unroll 1
            for (int t = t0; t < t0 + half; t += 16) {           // (16 columns are of one share: nt is a multiple of 64, split 2 or 4)
                uint32_t r[16];
                tcgen05_ld_32x32b_x16(tmem + ((uint32_t)(quad * 32) << 16) + (uint32_t)t, r);
                const int to = t / own;
                const uint32_t cta = (uint32_t)to * 2u + rank, bar = mapa_u32(smem_u32(&sums_bar), cta),
                               dst = mapa_u32(ring, cta) + (uint32_t)((((int)share * own + t - to * own) * 128 + quad * 32 + lane) * 4);
                tcgen05_wait_ld();
                tcgen05_loaded(r);
#pragma unroll
                for (int e = 0; e < 16; ++e) store_cluster(dst + 512u * e, __uint_as_float(r[e]), bar);
            }
            bool all = false;
            for (int i = 0; i < 8 && !all; ++i) all = warp_all(mbar_wait(smem_u32(&sums_bar), 0));
            ok = ok && all;
            const int *sums = reinterpret_cast<const int *>(pair_smem + (ring - smem_u32(pair_smem)));
#pragma unroll 2
            for (int c = ((int)threadIdx.x - 64) >> 6; c < own; c += (kI8PairThreads - 64) / 64) {
                const int m = m0 + c;
                int v0 = 0, v1 = 0;
                for (int r = 0; r < split; ++r) {
                    const int2 v = *reinterpret_cast<const int2 *>(sums + (r * own + c) * 128 + ch);
                    v0 += v.x;
                    v1 += v.y;
                }
                if (ok && m < p.M && n < p.N) {
                    const float f = token_scale[warp - 2][c], c0 = i8_scaled(v0, f, w0), c1 = i8_scaled(v1, f, w1);
                    T *y = static_cast<T *>(p.y) + (size_t)m * p.ldy + n;
                    if (pairs_ok) *reinterpret_cast<uint32_t *>(y) = f4_from_float2<T>(c0, c1);
                    else {
                        y[0] = f4_from_float<T>(c0);
                        if (n + 1 < p.N) y[1] = f4_from_float<T>(c1);
                    }
                }
            }
        }
    }
    if (!ok) atomicCAS(p.status, 0u, (uint32_t)TMAN_ERR_TIMEOUT);
    tcgen05_fence_before();
    __syncthreads();
    cluster_sync_all();                  // nobody touches the peer's memory after this
    if (warp == 1) {
        tcgen05_fence_after();
        tcgen05_dealloc2(tmem, 512);
    }
}

// Tokens of a tile, a multiple of 32 (of 64 where shares of k are summed), and shares of k of a tile: what has the least modelled time.
struct I8PairPlan { int nt, split; double us; };
inline I8PairPlan i8_pair_plan(int M, int steps, int tiles_n, int workers, const int (&clusters)[2])      // clusters of two and of four pairs held at once
{
    I8PairPlan best = {64, 1, 1e300};
    for (int nt = 64; nt <= kI8PairCols; nt += 32) {
        const long long tiles = (long long)((M + nt - 1) / nt) * tiles_n, rounds = (tiles + workers - 1) / workers;
        const double unit = 0.12 + 0.0008 * nt, tile = 0.1 + 0.0075 * nt;
        for (int split = 1; split <= 4; split *= 2) {
            if (split > 1 && (tiles > clusters[split >> 2] || steps < 2 * split || nt % 64 != 0)) continue;
            const double us = split == 1 ? (double)rounds * steps * unit + tile : (steps + split - 1) / split * unit + tile + 2.0 + 0.004 * nt;
            if (us < best.us - 1e-9) best = {nt, split, us};
        }
    }
    return best;
}

// Clusters of `ctas` CTAs of the kernel that the current device holds at once (0: none, or the query failed).
template <typename Kernel> inline int i8_pair_clusters(Kernel kern, int ctas)
{
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)ctas;
    attr[0].val.clusterDim.y = 1;
    attr[0].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)ctas * 64);
    cfg.blockDim = dim3(kI8PairThreads);
    cfg.dynamicSmemBytes = kI8PairSmem;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    int n = 0;
    if (cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, kI8PairSmem) != cudaSuccess ||
        cudaOccupancyMaxActiveClusters(&n, kern, &cfg) != cudaSuccess) {
        (void)cudaGetLastError();
        return 0;
    }
    return n;
}

template <typename T>
tman_status launch_i8_pair(const int8_t *w, int ldw, const int8_t *a, I8PairParams p, cudaStream_t s)
{
    auto kern = i8_pair_kernel<T>;
    static std::atomic<bool> raised[kMaxDevices];
    static std::atomic<int> held[kMaxDevices][2];                // clusters of two and of four pairs, + 1 (0: not asked yet)
    int dev = 0, clusters[2];
    const DeviceInfo *info = device_info(&dev);
    const EncodeTiledFn enc = encode_fn();
    if (!info || !enc) return TMAN_ERR_CUDA;
    for (int i = 0; i < 2; ++i) {
        int n = held[dev][i].load(std::memory_order_relaxed);
        if (n == 0) held[dev][i].store(n = i8_pair_clusters(kern, 4 << i) + 1, std::memory_order_relaxed);
        clusters[i] = n - 1;
    }
    const int workers = info->sms.load(std::memory_order_relaxed) / 2;
    p.tiles_n = (int)(((long long)p.N + 255) / 256);
    const I8PairPlan plan = i8_pair_plan(p.M, (p.K + 127) / 128, p.tiles_n, workers, clusters);
    p.nt = plan.nt;
    p.split_sh = plan.split >> 1;        // 0, 1, 2
    p.tiles_m = (int)(((long long)p.M + p.nt - 1) / p.nt);
    const long long tiles = (long long)p.tiles_m * p.tiles_n;
    if (tiles > 0x7FFFFFFF - 1024) return TMAN_ERR_SHAPE;
    // Tiles are numbered so that a round of them touches the fewest bytes: rows first, it takes all of a and few channels, or the other way around.
    const long long round = tiles < workers ? tiles : workers;
    const auto bytes = [&](long long tm, long long tn) { return (double)tm * p.nt + (double)tn * 256; };
    const auto up = [](long long x, long long y) { return (x + y - 1) / y; };
    p.rows_fastest = bytes(p.tiles_m < round ? p.tiles_m : round, up(round, p.tiles_m)) < bytes(up(round, p.tiles_n), p.tiles_n < round ? p.tiles_n : round);
    p.stream_y = (size_t)p.M * p.N * 2 > kI8StreamBytes ? 1 : 0;
    const int stage = (int)kI8PairA + p.nt * 64, fit = (kI8PairSmem - 1024) / stage;
    p.stages = fit < kI8PairStages ? fit : kI8PairStages;

    CUtensorMap maps[2];
    for (int i = 0; i < 2; ++i) {
        const cuuint64_t dims[2] = {(cuuint64_t)p.K, (cuuint64_t)(i ? p.M : p.N)}, strides[1] = {(cuuint64_t)(i ? p.K : ldw)};
        const cuuint32_t box[2] = {128, (cuuint32_t)(i ? p.nt / 2 : 128)}, one[2] = {1, 1};
        if (enc(&maps[i], CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<int8_t *>(i ? a : w), dims, strides, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE,
                CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS)
            return TMAN_ERR_CUDA;
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)((2 << p.split_sh) * (tiles < workers ? tiles : workers)));
    cfg.blockDim = dim3(kI8PairThreads);
    cfg.dynamicSmemBytes = kI8PairSmem;  // (all of it: no CTA that needs tensor memory beside one of these, which hold all of that)
    cfg.stream = s;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (2u << p.split_sh);
    attr[0].val.clusterDim.y = 1;
    attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    return launch_with_smem(kern, kI8PairSmem, dev, raised, [&] { return cudaLaunchKernelEx(&cfg, kern, maps[0], maps[1], p); });
}

}  // namespace
}  // namespace tman
