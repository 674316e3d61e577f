// Products of many rows, both operands in 4 bits: y[m][n] = a_row[m] w_row[n] sum_k a[m][k] w[n][k], bound by the tensor cores.
//
// A pair of CTAs (cta_group::2) has a tile of 256 channels (the rows of the tensor-core tile, 128 a CTA) x up to 192 rows of a (its columns).
// The packed layout is the operands' layout: stages of 256 values of k reach shared memory by linear bulk copies, each CTA its own
// channels and half of the rows of a, and the scales of all of them; the scales go on to tensor memory by tcgen05.cp in front of the
// MMAs that use them, both issued by one thread of the pair.  Two accumulators of 192 columns and two sets of scales (2 x 32 columns) share
// tensor memory, so that a tile's epilogue runs behind the next tile's MMAs.
// A tile's rows of a start at a multiple of 64: in tensor memory 32 rows' scales are a column, and the scales of an operand start at an even
// column (an odd one is a misaligned address), so that a tile's scales are the first or the second half of the first 512-byte piece and on.
#pragma once

#include "f4.cuh"
#include "sm100_ptx.cuh"

namespace tman {
namespace {

constexpr int kPairThreads = 320;        // warp 0: loads, warp 1: MMAs (of the pair's first CTA), warps 2..9: epilogue
constexpr int kPairCols = 192;           // most rows of a in a tile
constexpr int kPairStages = 7;
constexpr int kPairSmem = 220 * 1024;

struct F4PairParams {
    const uint8_t *w, *a;
    void *y;
    uint32_t *status;
    size_t w_codes, w_scales, w_rows, a_codes, a_scales, a_rows;
    int M, K, N, ldy, units, w_h8, a_h8, nt, tiles_m, tiles_n, stages;
};

template <int BLOCK> struct PairStage {
    static constexpr int SB = BLOCK == 32 ? 512 : 1024, CHUNKS = SB / 512;
    static constexpr uint32_t kB = 2 * 8192, kSfa = kB + 2 * (kPairCols / 2 * 64), kSfb = kSfa + 2 * SB, kBytes = kSfb + 2 * 2 * SB;
    // (stage: [unit] channels' codes, [unit] codes of a, [unit] channels' scales, [piece][unit] scales of a)
};

template <int BLOCK, typename T>
__global__ void __launch_bounds__(kPairThreads) __cluster_dims__(2, 1, 1) f4_pair_kernel(const __grid_constant__ F4PairParams p)
{
    extern __shared__ __align__(128) uint8_t smem[];
    __shared__ __align__(8) uint64_t full_bar[kPairStages], empty_bar[kPairStages], accf_bar[2], acce_bar[2];
    __shared__ uint32_t tmem_slot;
    using St = PairStage<BLOCK>;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = cluster_ctarank();
    const int worker = blockIdx.x >> 1, workers = gridDim.x >> 1, tiles = p.tiles_m * p.tiles_n;
    const uint32_t full0 = smem_u32(full_bar), empty0 = smem_u32(empty_bar), accf0 = smem_u32(accf_bar), acce0 = smem_u32(acce_bar), ring = smem_u32(smem);
    const int steps = (p.units + 1) >> 1;
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
        fence_barrier_init();
    }
    __syncthreads();
    cluster_sync_all();

    // ---- loads of a stage --------------------------------------------------------------------------
    auto load_w = [&](int tile, int step, int s) {
        const int rt = (tile % p.tiles_n) * 2 + (int)rank, h = min(kF4Tile, p.w_h8 - rt * kF4Tile), nu = min(2, p.units - 2 * step);
        if (h <= 0) return;                                      // (channels behind the last)
        const uint32_t st = ring + s * St::kBytes, bar = full0 + 8 * s;
        const uint8_t *codes = p.w + p.w_codes + (size_t)rt * p.units * (kF4Tile * 64) + (size_t)(2 * step) * (h * 64);
        if (h == kF4Tile) bulk_load(st, codes, (uint32_t)nu * 8192u, bar);
        else for (int u = 0; u < nu; ++u) bulk_load(st + u * 8192, codes + u * (h * 64), (uint32_t)(h * 64), bar);
        bulk_load(st + St::kSfa, p.w + p.w_scales + ((size_t)rt * p.units + 2 * step) * St::SB, (uint32_t)(nu * St::SB), bar);
    };
    auto load_a = [&](int tile, int step, int s) {
        const int m0 = tile / p.tiles_n * p.nt, r0 = m0 + (int)rank * (p.nt >> 1), r1 = min(r0 + (p.nt >> 1), p.a_h8), nu = min(2, p.units - 2 * step);
        const uint32_t st = ring + s * St::kBytes, bar = full0 + 8 * s;
        for (int r = r0; r < r1;) {                              // rows of one or two tiles of the packed matrix
            const int rt = r / kF4Tile, h = min(kF4Tile, p.a_h8 - rt * kF4Tile), n = min(r1, (rt + 1) * kF4Tile) - r;
            const uint8_t *codes = p.a + p.a_codes + (size_t)rt * p.units * (kF4Tile * 64) + (size_t)(2 * step) * (h * 64) + (size_t)(r % kF4Tile) * 64;
            for (int u = 0; u < nu; ++u)
                bulk_load(st + St::kB + (uint32_t)(u * (kPairCols / 2) + r - r0) * 64u, codes + u * (h * 64), (uint32_t)(n * 64), bar);
            r += n;
        }
        const int t1 = (min(m0 + p.nt, p.a_h8) + kF4Tile - 1) / kF4Tile;
        for (int rt = m0 / kF4Tile, j = 0; rt < t1; ++rt, ++j)
            bulk_load(st + St::kSfb + j * 2 * St::SB, p.a + p.a_scales + ((size_t)rt * p.units + 2 * step) * St::SB, (uint32_t)(nu * St::SB), bar);
    };
    auto bytes_of = [&](int tile, int step) {
        const int h = min(kF4Tile, p.w_h8 - ((tile % p.tiles_n) * 2 + (int)rank) * kF4Tile), nu = min(2, p.units - 2 * step);
        const int m0 = tile / p.tiles_n * p.nt, r0 = m0 + (int)rank * (p.nt >> 1), rows = max(min(r0 + (p.nt >> 1), p.a_h8) - r0, 0);
        const int pieces = (min(m0 + p.nt, p.a_h8) + kF4Tile - 1) / kF4Tile - m0 / kF4Tile;
        return (uint32_t)(nu * ((h > 0 ? h * 64 + St::SB : 0) + rows * 64 + pieces * St::SB));
    };
    const int total = worker < tiles ? ((tiles - 1 - worker) / workers + 1) * steps : 0;       // stages of this pair
    int first = 0;
    if (warp == 0 && elect_one()) {
        // weights of the first stages before the wait for the kernel ahead: nothing that may still be running writes them
        first = min(p.stages, min(total, steps));
        for (int i = 0; i < first; ++i) {
            mbar_expect_tx(full0 + 8 * i, bytes_of(worker, i));
            load_w(worker, i, i);
        }
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
    const uint32_t tmem = tmem_slot;

    if (warp == 0) {
        if (elect_one()) {
            int s = 0, i = 0;
            uint32_t ph = 1;                                     // (the first pass over the ring does not wait)
            for (int tile = worker; ok && tile < tiles; tile += workers)
                for (int step = 0; step < steps; ++step, ++i) {
                    if (i >= first) {
                        if (!mbar_wait(empty0 + 8 * s, ph)) { ok = false; break; }
                        mbar_expect_tx(full0 + 8 * s, bytes_of(tile, step));
                        load_w(tile, step, s);
                    }
                    load_a(tile, step, s);
                    if (++s == p.stages) { s = 0; ph ^= 1u; }
                }
        }
        __syncwarp();
    } else if (warp == 1) {
        if (elect_one()) {
            int s = 0;
            uint32_t ph = 0;
            if (rank != 0) {                                     // tells the first CTA when this one's part of a stage is there
                const uint32_t lead = mapa_u32(full0, 0);
                for (int i = 0; i < total; ++i) {
                    if (!mbar_wait(full0 + 8 * s, ph)) { ok = false; break; }
                    mbar_arrive_cluster(lead + 8 * s);
                    if (++s == p.stages) { s = 0; ph ^= 1u; }
                }
            } else {
                const uint32_t id0 = f4_idesc(BLOCK, 256, p.nt, 0), id1 = f4_idesc(BLOCK, 256, p.nt, BLOCK == 32 ? 2 : 0);
                uint32_t ti = 0, set = 0;
                for (int tile = worker; ok && tile < tiles; tile += workers, ++ti) {
                    const uint32_t b = ti & 1u, acc = tmem + b * kPairCols;
                    if (!mbar_wait(acce0 + 8 * b, ((ti >> 1) & 1u) ^ 1u)) { ok = false; break; }
                    tcgen05_fence_after();
                    const int m0 = tile / p.tiles_n * p.nt, g0 = m0 / 32 % 4, pieces = (g0 + p.nt / 32 + 3) / 4;
                    for (int u = 0; u < p.units; ++u) {
                        const uint32_t st = ring + s * St::kBytes, half = (uint32_t)(u & 1);
                        if (half == 0) {
                            if (!mbar_wait(full0 + 8 * s, ph)) { ok = false; break; }
                            tcgen05_fence_after();
                        }
                        const uint32_t sfa = tmem + 2 * kPairCols + set * 32u, sfb = sfa + 4 * St::CHUNKS;
                        set ^= 1u;
#pragma unroll
                        for (int c = 0; c < St::CHUNKS; ++c) {
                            tcgen05_cp2_scales(sfa + 4 * c, make_kmajor_desc(st + St::kSfa + half * St::SB + 512 * c, 128, 128));
#pragma unroll
                            for (int j = 0; j < 2; ++j)
                                if (j < pieces)
                                    tcgen05_cp2_scales(sfb + 8 * c + 4 * j, make_kmajor_desc(st + St::kSfb + (2 * j + half) * St::SB + 512 * c, 128, 128));
                        }
                        const uint32_t wa = st + half * 8192u, xb = st + St::kB + half * (kPairCols / 2 * 64);
                        tcgen05_mma2_f4<BLOCK>(acc, make_kmajor_desc(wa, 128, 512), make_kmajor_desc(xb, 128, 512), id0, sfa, sfb + g0, u > 0);
                        tcgen05_mma2_f4<BLOCK>(acc, make_kmajor_desc(wa + 256, 128, 512), make_kmajor_desc(xb + 256, 128, 512), id1,
                                               sfa + (BLOCK == 32 ? 0 : 4), sfb + g0 + (BLOCK == 32 ? 0 : 8), 1);
                        if (half == 1 || u == p.units - 1) {
                            tcgen05_commit2_both(empty0 + 8 * s);
                            if (++s == p.stages) { s = 0; ph ^= 1u; }
                        }
                    }
                    tcgen05_commit2_both(accf0 + 8 * b);
                }
            }
        }
        __syncwarp();
    } else {
        // ---- epilogue: a warp has 32 channels (a lane each) x half of the tile's rows of a; neighbouring lanes exchange every other row, so
        // that a lane stores two adjacent channels of one row
        const bool hdr_ok = f4_header_matches(p.w, p.N, p.K, BLOCK) && f4_header_matches(p.a, p.M, p.K, BLOCK);
        if (!hdr_ok && threadIdx.x == 64 && blockIdx.x == 0) atomicCAS(p.status, 0u, (uint32_t)TMAN_ERR_BAD_PACKED);
        const int quad = warp & 3, half = ((p.nt >> 1) + 7) / 8 * 8, h0 = (warp - 2) >= 4 ? half : 0, h1 = (warp - 2) >= 4 ? p.nt : half;
        const bool odd = (lane & 1) != 0, pairs_ok = (p.N & 1) == 0 && (p.ldy & 1) == 0 && (reinterpret_cast<uintptr_t>(p.y) & 3) == 0;
        const uint32_t acce_lead = mapa_u32(acce0, 0);
        const float *a_row = reinterpret_cast<const float *>(p.a + p.a_rows), *w_row = reinterpret_cast<const float *>(p.w + p.w_rows);
        uint32_t ti = 0;
        for (int tile = worker; tile < tiles; tile += workers, ++ti) {
            const uint32_t b = ti & 1u;
            const int m0 = tile / p.tiles_n * p.nt, n = (tile % p.tiles_n) * 256 + (int)rank * 128 + quad * 32 + lane, n2 = n & ~1;
            const int end = min(h1, p.M - m0);
            const bool put = hdr_ok && n < p.N;
            const float wr = BLOCK == 16 && n < p.N ? w_row[n] : 1.f;
            const float w0 = odd ? __shfl_xor_sync(0xffffffffu, wr, 1) : wr;
            const float w1 = odd ? wr : __shfl_xor_sync(0xffffffffu, wr, 1);
            ok = warp_all(mbar_wait(accf0 + 8 * b, (ti >> 1) & 1u));
            if (!ok) break;
            tcgen05_fence_after();
            const uint32_t acc = tmem + ((uint32_t)(quad * 32) << 16) + b * kPairCols;
#pragma unroll 1
            for (int t = h0; t < end; t += 8) {
                uint32_t r[8];
                tcgen05_ld_32x32b_x8(acc + (uint32_t)t, r);
                float ar[4];
                if constexpr (BLOCK == 16) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) ar[e] = ld_dependent(a_row + min(m0 + t + 2 * e + (odd ? 1 : 0), p.M - 1));
                }
                tcgen05_wait_ld();
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const uint32_t keep = odd ? r[2 * e + 1] : r[2 * e], got = __shfl_xor_sync(0xffffffffu, odd ? r[2 * e] : r[2 * e + 1], 1);
                    float c0 = __uint_as_float(odd ? got : keep), c1 = __uint_as_float(odd ? keep : got);
                    if constexpr (BLOCK == 16) {
                        c0 *= w0 * ar[e];
                        c1 *= w1 * ar[e];
                    }
                    const int tt = t + 2 * e + (odd ? 1 : 0);
                    if (tt < end) {
                        T *y = static_cast<T *>(p.y) + (size_t)(m0 + tt) * p.ldy + n2;
                        if (pairs_ok) {
                            if (put) *reinterpret_cast<uint32_t *>(y) = f4_from_float2<T>(c0, c1);
                        } else if (hdr_ok) {
                            if (n2 < p.N) y[0] = f4_from_float<T>(c0);
                            if (n2 + 1 < p.N) y[1] = f4_from_float<T>(c1);
                        }
                    }
                }
            }
            tcgen05_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive_cluster(acce_lead + 8 * b);
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

// Rows of a in a tile: the multiple of 64 with the least modelled time, rounds of tiles x (units x time of a unit + a tile's fixed part).
inline int pair_rows(int M, int units, int tiles_n, int workers)
{
    int best = 64;
    double least = 1e300;
    for (int nt = 64; nt <= kPairCols; nt += 64) {
        const long long tiles = (long long)((M + nt - 1) / nt) * tiles_n, rounds = (tiles + workers - 1) / workers;
        const double unit = nt > 128 ? 0.00060 * nt : 0.077;
        const double us = (double)rounds * (units * unit + 0.3) + 0.005 * nt;
        if (us < least - 1e-9) { least = us; best = nt; }
    }
    return best;
}

template <int BLOCK, typename T>
tman_status launch_pair(F4PairParams p, cudaStream_t s)
{
    auto kern = f4_pair_kernel<BLOCK, T>;
    static std::atomic<bool> raised[kMaxDevices];
    int dev = 0;
    const DeviceInfo *info = device_info(&dev);
    if (!info) return TMAN_ERR_CUDA;
    const int workers = info->sms.load(std::memory_order_relaxed) / 2;
    p.tiles_n = (p.N + 255) / 256;
    p.nt = pair_rows(p.M, p.units, p.tiles_n, workers);
    p.tiles_m = (p.M + p.nt - 1) / p.nt;
    const long long tiles = (long long)p.tiles_m * p.tiles_n;
    if (tiles > 0x7FFFFFFF) return TMAN_ERR_SHAPE;
    p.stages = kPairSmem / (int)PairStage<BLOCK>::kBytes;
    if (p.stages > kPairStages) p.stages = kPairStages;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(2 * (tiles < workers ? tiles : workers)));
    cfg.blockDim = dim3(kPairThreads);
    cfg.dynamicSmemBytes = (size_t)p.stages * PairStage<BLOCK>::kBytes;
    cfg.stream = s;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = packed_write_pending(s, /*clear=*/true) ? 0 : 1;
    return launch_with_smem(kern, kPairSmem, dev, raised, [&] { return cudaLaunchKernelEx(&cfg, kern, p); });
}

}  // namespace
}  // namespace tman
