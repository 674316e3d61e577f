// Products of many rows, both operands in 4 bits: y[m][n] = a_row[m] w_row[n] sum_k a[m][k] w[n][k].
//
// A pair of CTAs (cta_group::2) has a tile of 256 channels (the rows of the tensor-core tile, 128 a CTA) x up to 256 rows of a (its columns).
// The packed layout is the operands' layout: units of 256 values of k reach shared memory by four linear bulk copies a CTA, its own
// channels, half of the rows of a, and the scales of the channels and of all the rows.  The scales go on to tensor memory by tcgen05.cp in front
// of the MMAs that use them, both issued by one thread of the pair.
// Tensor memory: two accumulators from columns 0 and 192 on, scales from 448.  Up to 192 rows of a, a tile's epilogue runs behind the next
// tile's MMAs; with 256 the accumulators share 64 columns, which the epilogue takes first: the next tile starts when it has them in
// registers.
// A tile's rows of a start at a multiple of 64: in tensor memory 32 rows' scales are a column, and the scales of an operand start at an even
// column (an odd one is a misaligned address), so that a tile's scales are the first or the second half of the first 512-byte piece and on.
#pragma once

#include "f4.cuh"
#include "sm100_ptx.cuh"

#include <type_traits>

namespace tman {
namespace {

constexpr int kPairThreads = 320;        // warp 0: loads, warp 1: MMAs (of the pair's first CTA), warps 2..9: epilogue
constexpr int kPairCols = 256;           // most rows of a in a tile
constexpr int kPairAcc1 = 192, kPairSf = 448;
constexpr int kPairStages = 6;
constexpr int kPairSmem = 222 * 1024;
constexpr double kPairSharesUs = 2.0;     // of sending and adding up the shares' sums, beside 0.004 a row
constexpr size_t kPairStreamBytes = (size_t)64 << 20;

struct F4PairParams {
    const uint8_t *w, *a;
    void *y;
    uint32_t *status;
    size_t w_codes, w_scales, w_rows, a_codes, a_scales, a_rows;
    int M, K, N, ldy, halves, w_h8, a_h8, nt, tiles_m, tiles_n, rows_fastest, stream_y, stages, split_sh;
    uint32_t tile_mul;                   // 2^32 / (the tiles that are numbered first), rounded up; 0: one, or too many tiles for it
};

template <int BLOCK> struct PairStage {
    static constexpr uint32_t SB = f4_scale_bytes(BLOCK), CHUNKS = SB / 512;
    static constexpr uint32_t kB = kF4Tile * 128, kSfa = kB + kPairCols / 2 * 128, kSfb = kSfa + 2 * SB, kBytes = kSfb + 2 * 2 * SB;
};

template <int BLOCK> constexpr int pair_stages()
{
    constexpr int n = kPairSmem / (int)PairStage<BLOCK>::kBytes;
    return n < kPairStages ? n : kPairStages;
}

template <int BLOCK, typename T>
__global__ void __launch_bounds__(kPairThreads) f4_pair_kernel(const __grid_constant__ F4PairParams p)
{
    extern __shared__ __align__(128) uint8_t smem[];
    __shared__ __align__(8) uint64_t full_bar[kPairStages], empty_bar[kPairStages], accf_bar[2], acce_bar[2], shared_bar, sums_bar;
    __shared__ uint32_t tmem_slot;
    using St = PairStage<BLOCK>;
    const int warp = __shfl_sync(0xffffffffu, (int)threadIdx.x >> 5, 0), lane = threadIdx.x & 31;      // (the shuffle tells the compiler that it is uniform)
    // a cluster: the pairs with the shares of k of a tile, one tile each (split > 1), or one pair that walks over tiles
    const uint32_t crank = cluster_ctarank(), rank = crank & 1u, share = crank >> 1;
    const int worker = blockIdx.x >> (1 + p.split_sh), workers = gridDim.x >> (1 + p.split_sh), tiles = p.tiles_m * p.tiles_n, split = 1 << p.split_sh;
    const uint32_t full0 = smem_u32(full_bar), empty0 = smem_u32(empty_bar), accf0 = smem_u32(accf_bar), acce0 = smem_u32(acce_bar),
                   shared0 = smem_u32(&shared_bar), ring = smem_u32(smem);
    const int all_steps = (p.halves + 1) >> 1, step0 = all_steps * (int)share >> p.split_sh, steps = (all_steps * (int)(share + 1) >> p.split_sh) - step0;
    const bool overlap = p.nt > kPairAcc1;                       // the two accumulators share columns
    // a tile's place among the rows and the channels (a division by a variable costs the first loads of a call a sixth of a microsecond)
    const int inner = p.rows_fastest ? p.tiles_m : p.tiles_n;
    auto outer_of = [&](int tile) { return p.tile_mul ? (int)__umulhi((uint32_t)tile, p.tile_mul) : inner == 1 ? tile : tile / inner; };
    auto tile_m = [&](int tile) { const int o = outer_of(tile); return p.rows_fastest ? tile - o * inner : o; };
    auto tile_n = [&](int tile) { const int o = outer_of(tile); return p.rows_fastest ? o : tile - o * inner; };
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
        mbar_init(shared0, 8);
        mbar_init(smem_u32(&sums_bar), 1);
        if (split > 1) mbar_expect_tx(smem_u32(&sums_bar), (uint32_t)p.nt * 512u);
        fence_barrier_init();
    }
    __syncthreads();
    cluster_sync_all();

    const int total = worker < tiles ? ((tiles - 1 - worker) / workers + 1) * steps : 0;       // stages of this pair
    // (Warps 0 and 1 walk as one and work out addresses and descriptors outside of what one lane issues, so that they sit in uniform
    // registers: 0.4 us a unit otherwise.)
    // What a tile loads: bytes of a unit (of half a unit: half of them) and where its first unit is; units are a constant distance apart.
    struct Loads {
        const uint8_t *w, *ws, *a, *as;
        uint32_t w_bytes, a_bytes, as_bytes;
    };
    auto loads_of = [&](int tile) {
        Loads l;
        const int tm = tile_m(tile), rt = tile_n(tile) * 2 + (int)rank, h = max(min(kF4Tile, p.w_h8 - rt * kF4Tile), 0);
        const int m0 = tm * p.nt, r0 = m0 + (int)rank * (p.nt >> 1), rows = max(min(p.nt >> 1, p.a_h8 - r0), 0), at = m0 / kF4Tile;
        l.w_bytes = (uint32_t)h * 128u;                          // (0: channels behind the last)
        l.a_bytes = (uint32_t)rows * 128u;
        l.as_bytes = (uint32_t)((min(m0 + p.nt, p.a_h8) + kF4Tile - 1) / kF4Tile - at) * (2u * St::SB);
        l.w = p.w + p.w_codes + (size_t)rt * (kF4Tile * 128);
        l.ws = p.w + p.w_scales + (size_t)rt * (2 * St::SB);
        l.a = p.a + p.a_codes + (size_t)r0 * 128;
        l.as = p.a + p.a_scales + (size_t)at * (2 * St::SB);
        return l;
    };
    const size_t w_step = (size_t)p.w_h8 * 128, a_step = (size_t)p.a_h8 * 128, ws_step = (size_t)((p.w_h8 + kF4Tile - 1) / kF4Tile) * (2 * St::SB),
                 as_step = (size_t)((p.a_h8 + kF4Tile - 1) / kF4Tile) * (2 * St::SB);
    // A half unit's sections are half as wide: rows (tiles) lie half as far from the section's start.
    auto load = [&](bool lead, const Loads &l, int i, int s, bool do_w, bool do_a) {
        const int step = step0 + i;
        const uint32_t sh = 2 * step + 1 < p.halves ? 0u : 1u;
        const uint32_t st = ring + (uint32_t)s * St::kBytes, bar = full0 + 8 * s;
        const uint8_t *w = p.w + p.w_codes + step * w_step + ((size_t)(l.w - (p.w + p.w_codes)) >> sh);
        const uint8_t *ws = p.w + p.w_scales + step * ws_step + ((size_t)(l.ws - (p.w + p.w_scales)) >> sh);
        const uint8_t *a = p.a + p.a_codes + step * a_step + ((size_t)(l.a - (p.a + p.a_codes)) >> sh);
        const uint8_t *as = p.a + p.a_scales + step * as_step + ((size_t)(l.as - (p.a + p.a_scales)) >> sh);
        const uint32_t wb = l.w_bytes >> sh, ab = l.a_bytes >> sh, asb = l.as_bytes >> sh, wsb = wb ? 2u * St::SB >> sh : 0u;
        if (lead) {
            if (do_w) {
                mbar_expect_tx(bar, wb + wsb + ab + asb);
                if (wb) {
                    bulk_load(st, w, wb, bar);
                    bulk_load(st + St::kSfa, ws, wsb, bar);
                }
            }
            if (do_a) {
                if (ab) bulk_load(st + St::kB, a, ab, bar);
                bulk_load(st + St::kSfb, as, asb, bar);
            }
        }
        __syncwarp();
    };
    int first = 0;
    if (warp == 0) {
        // weights of the first stages before the wait for the kernel ahead: nothing that may still be running writes them
        const bool lead = elect_one();
        first = min(p.stages, min(total, steps));
        if (first > 0) {
            const Loads l = loads_of(worker);
            for (int i = 0; i < first; ++i) load(lead, l, i, i, true, false);
        }
    }
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
    bool hdr_ok = true;
    if (warp >= 2) {
        hdr_ok = f4_header_matches(p.w, p.N, p.K, BLOCK) && f4_header_matches(p.a, p.M, p.K, BLOCK);
        if (!hdr_ok && threadIdx.x == 64 && blockIdx.x == 0) atomicCAS(p.status, 0u, (uint32_t)TMAN_ERR_BAD_PACKED);
    }
    const float *a_row = reinterpret_cast<const float *>(p.a + p.a_rows), *w_row = reinterpret_cast<const float *>(p.w + p.w_rows);
    const bool pairs_ok = (p.N & 1) == 0 && (p.ldy & 1) == 0 && (reinterpret_cast<uintptr_t>(p.y) & 3) == 0;

    if (warp == 0) {
        const bool lead = elect_one();
        int s = 0, i = 0;
        uint32_t ph = 1;                                         // (the first pass over the ring does not wait)
        for (int tile = worker; ok && tile < tiles; tile += workers) {
            const Loads l = loads_of(tile);
            for (int step = 0; step < steps; ++step, ++i) {
                if (i >= first && !warp_all(mbar_wait(empty0 + 8 * s, ph))) { ok = false; break; }
                load(lead, l, step, s, i >= first, true);
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
        const uint32_t id0 = f4_idesc(BLOCK, 256, p.nt, 0), id1 = f4_idesc(BLOCK, 256, p.nt, BLOCK == 32 ? 2 : 0);
        const uint64_t sf0 = make_kmajor_desc(ring, 128, 128);                     // (+ 1: 16 bytes)
        const uint16_t both = (uint16_t)(3u << crank);
        int s = 0;
        uint32_t ph = 0, ti = 0;
        for (int tile = worker; ok && tile < tiles; tile += workers, ++ti) {
            const uint32_t b = ti & 1u, acc = tmem + b * kPairAcc1;
            if (!warp_all(mbar_wait(acce0 + 8 * b, ((ti >> 1) & 1u) ^ 1u))) { ok = false; break; }
            if (overlap && ti > 0 && !warp_all(mbar_wait(shared0, (ti - 1) & 1u))) { ok = false; break; }
            const uint32_t g0 = (uint32_t)(tile_m(tile) * p.nt) / 32 % 4;
            const bool two = g0 + (uint32_t)p.nt / 32 > 4;           // pieces of scales of a
            for (int step = 0; step < steps; ++step) {
                const uint32_t at = (uint32_t)s * (St::kBytes >> 4), nu = 2 * (step0 + step) + 1 < p.halves ? 2u : 1u;
                const uint64_t op = make_kmajor_desc(ring, 128, nu * 512) + at, sf = sf0 + at;
                if (!warp_all(mbar_wait(full0 + 8 * s, ph))) { ok = false; break; }
                tcgen05_fence_after();
                if (lead) {
#pragma unroll
                    for (uint32_t u = 0; u < 2; ++u)
                        if (u < nu) {
                            const uint32_t sfa = tmem + kPairSf + u * 32u, sfb = sfa + 4 * St::CHUNKS;
#pragma unroll
                            for (uint32_t c = 0; c < St::CHUNKS; ++c) {
                                tcgen05_cp2_scales(sfa + 4 * c, sf + ((St::kSfa + u * St::SB + 512 * c) >> 4));
                                tcgen05_cp2_scales(sfb + 8 * c, sf + ((St::kSfb + u * St::SB + 512 * c) >> 4));
                                if (two) tcgen05_cp2_scales(sfb + 8 * c + 4, sf + ((St::kSfb + (nu + u) * St::SB + 512 * c) >> 4));
                            }
                            const uint64_t wa = op + ((u * 512) >> 4), xb = op + ((St::kB + u * 512) >> 4);
                            tcgen05_mma2_f4<BLOCK>(acc, wa, xb, id0, sfa, sfb + g0, (step | (int)u) != 0);
                            tcgen05_mma2_f4<BLOCK>(acc, wa + 16, xb + 16, id1, sfa + (BLOCK == 32 ? 0 : 4), sfb + g0 + (BLOCK == 32 ? 0 : 8), 1);
                        }
                    tcgen05_commit2(empty0 + 8 * s, both);
                }
                __syncwarp();
                if (++s == p.stages) { s = 0; ph ^= 1u; }
            }
            if (lead) tcgen05_commit2(accf0 + 8 * b, both);
            __syncwarp();
        }
    } else if (split == 1) {
        // ---- epilogue: a warp has 32 channels (a lane each) x half of the tile's rows of a, 32 at a time; neighbouring lanes exchange every
        // other row, so that a lane stores two adjacent channels of one row
        const int quad = warp & 3, half = p.nt >> 1;
        const bool second = warp >= 6, odd = (lane & 1) != 0;
        const uint32_t acce_lead = mapa_u32(acce0, crank & ~1u), shared_lead = mapa_u32(shared0, crank & ~1u);
        const uint64_t y_policy = p.stream_y ? policy_evict_first() : policy_evict_normal();
        uint32_t ti = 0;
        for (int tile = worker; tile < tiles; tile += workers, ++ti) {
            const uint32_t b = ti & 1u;
            const int m0 = tile_m(tile) * p.nt, n = tile_n(tile) * 256 + (int)rank * 128 + quad * 32 + lane, n2 = n & ~1;
            const int end = p.M - m0, t0 = second ? half : 0;
            const bool put = hdr_ok && n2 < p.N, put1 = n2 + 1 < p.N, whole = warp_all(put && put1 && pairs_ok);
            const size_t row2 = 2 * (size_t)p.ldy;
            float w0 = 1.f, w1 = 1.f;
            if constexpr (BLOCK == 16) {
                w0 = w_row[min(n2, p.N - 1)];
                w1 = w_row[min(n2 + 1, p.N - 1)];
            }
            T *y = static_cast<T *>(p.y) + (size_t)(m0 + (odd ? 1 : 0)) * p.ldy + n2;
            const uint32_t acc = tmem + ((uint32_t)(quad * 32) << 16) + b * kPairAcc1;
            // WHOLE: 32 rows of pairs of channels; else what there is of them.  (One place in the code each: a call that does one tile a pair
            // meets it with a cold instruction cache, 256 x 4096 x 14336 11.7 us with nine copies.)
            auto store32 = [&](auto whole_c, int t, const uint32_t (&r)[32]) {
                constexpr bool WHOLE = decltype(whole_c)::value;
                [[maybe_unused]] float ar = 1.f;
                if constexpr (BLOCK == 16) ar = ld_dependent(a_row + min(m0 + t + lane, p.M - 1));
                T *yt = y + (size_t)t * p.ldy;
#pragma unroll
                for (int e = 0; e < 32; e += 2) {
                    const uint32_t got = __shfl_xor_sync(0xffffffffu, odd ? r[e] : r[e + 1], 1), keep = odd ? r[e + 1] : r[e];
                    float c0 = __uint_as_float(odd ? got : keep), c1 = __uint_as_float(odd ? keep : got);
                    if constexpr (BLOCK == 16) {
                        const float f = __shfl_sync(0xffffffffu, ar, e + (odd ? 1 : 0));
                        c0 = c0 * w0 * f;        // (in turn: the scales' product may leave the range)
                        c1 = c1 * w1 * f;
                    }
                    if constexpr (WHOLE) st_policy(yt, f4_from_float2<T>(c0, c1), y_policy);
                    else if (t + e + (odd ? 1 : 0) < end && put) {
                        yt[0] = f4_from_float<T>(c0);
                        if (put1) yt[1] = f4_from_float<T>(c1);
                    }
                    yt += row2;
                }
            };
            ok = warp_all(mbar_wait(accf0 + 8 * b, (ti >> 1) & 1u));
            if (!ok) break;
            tcgen05_fence_after();
            // The columns that the next tile's accumulator has too come first: when all of them are in registers, that tile may start.
            const bool first = overlap && second == (b == 0);
            const int groups = half >> 5, g0 = first && second ? 2 : 0;      // (of 32 columns; the second warps' shared ones are their last two)
            uint32_t r[32], next[32];
#pragma unroll 1
            for (int g = 0; g < groups; ++g) {
                const int t = t0 + 32 * ((g + g0) % groups);
                if (t >= end && !first) continue;
                if (first && g == 1) {
#pragma unroll
                    for (int e = 0; e < 32; ++e) r[e] = next[e];
                } else {
                    tcgen05_ld_32x32b_x32(acc + (uint32_t)t, r);
                    if (first && g == 0) tcgen05_ld_32x32b_x32(acc + (uint32_t)t + 32u, next);
                    tcgen05_wait_ld();
                }
                if (first && g == 0) {
                    tcgen05_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive_cluster(shared_lead);
                }
                if (whole && t + 32 <= end) store32(std::true_type(), t, r);
                else if (t < end) store32(std::false_type(), t, r);
            }
            tcgen05_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive_cluster(acce_lead + 8 * b);
        }
    }
    if (split > 1) {
        // ---- shares of a tile: column c of the tile is added up by share c / own in the CTA of the same channels; everyone sends it its sums,
        // [share][own column][channel] on the ring, which is idle everywhere once all accumulators are complete
        if (warp >= 2) {
            ok = warp_all(mbar_wait(accf0, 0)) && ok;
            tcgen05_fence_after();
        }
        __syncwarp();
        cluster_sync_all();
        const int own = p.nt >> p.split_sh, m0 = tile_m(worker) * p.nt + (int)share * own, n0 = tile_n(worker) * 256 + (int)rank * 128;
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
#pragma unroll
                for (int e = 0; e < 16; ++e) store_cluster(dst + 512u * e, __uint_as_float(r[e]), bar);
            }
            bool all = false;
            for (int i = 0; i < 8 && !all; ++i) all = warp_all(mbar_wait(smem_u32(&sums_bar), 0));
            ok = ok && all;
            const float *sums = reinterpret_cast<const float *>(smem);
            for (int i = threadIdx.x - 64; i < own * 64; i += kPairThreads - 64) {
                const int c = i >> 6, ch = (i & 63) * 2, m = m0 + c, n = n0 + ch;
                float v0 = 0.f, v1 = 0.f;
                for (int r = 0; r < split; ++r) {
                    const float2 v = *reinterpret_cast<const float2 *>(sums + (r * own + c) * 128 + ch);
                    v0 += v.x;
                    v1 += v.y;
                }
                if (ok && hdr_ok && m < p.M && n < p.N) {
                    if constexpr (BLOCK == 16) {
                        const float f = ld_dependent(a_row + m);
                        v0 = v0 * w_row[n] * f;
                        v1 = v1 * w_row[min(n + 1, p.N - 1)] * f;
                    }
                    T *y = static_cast<T *>(p.y) + (size_t)m * p.ldy + n;
                    if (pairs_ok) *reinterpret_cast<uint32_t *>(y) = f4_from_float2<T>(v0, v1);
                    else {
                        y[0] = f4_from_float<T>(v0);
                        if (n + 1 < p.N) y[1] = f4_from_float<T>(v1);
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

// Rows of a in a tile, a multiple of 64, and shares of k of a tile: what has the least modelled time.  A unit takes 0.28 us with 128 rows and 0.33
// with 256 (32-value blocks; 2048 x 3584 x 18944 with 128 / 192 / 256 rows a tile: 79.7 / 61.8 / 53.2 us, 8192 x 18944 x 3584: 282 / 213 / 183).  What
// holds it there is not the products alone: in 2048 x 3584 x 18944 the tensor pipe is active 61 % of the cycles, L2 is at 39 % and sends an SM 48
// bytes a clock, DRAM is at 14 %.  Whole tiles go round the pairs; shares are for few tiles, one a cluster of pairs.
struct PairPlan { int nt, split; double us; };
inline PairPlan pair_plan(int M, int steps, int tiles_n, int workers, const int (&clusters)[2])      // clusters of two and of four pairs held at once
{
    PairPlan best = {64, 1, 1e300};
    for (int nt = 64; nt <= kPairCols; nt += 64) {
        const long long tiles = (long long)((M + nt - 1) / nt) * tiles_n, rounds = (tiles + workers - 1) / workers;
        const double unit = 0.245 + 0.00032 * nt, tile = 0.1 + 0.0075 * nt;
        for (int split = 1; split <= 4; split *= 2) {
            if (split > 1 && (tiles > clusters[split >> 2] || steps < 2 * split)) continue;
            const double us = split == 1 ? (double)rounds * (steps * unit + tile) : (steps + split - 1) / split * unit + tile + kPairSharesUs + 0.004 * nt;
            if (us < best.us - 1e-9) best = {nt, split, us};
        }
    }
    return best;
}

// Clusters of `ctas` CTAs of the kernel that the current device holds at once (0: none, or the query failed).
template <typename Kernel> inline int pair_clusters(Kernel kern, int ctas)
{
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)ctas;
    attr[0].val.clusterDim.y = 1;
    attr[0].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)ctas * 64);
    cfg.blockDim = dim3(kPairThreads);
    cfg.dynamicSmemBytes = kPairSmem;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    int n = 0;
    if (cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, kPairSmem) != cudaSuccess ||
        cudaOccupancyMaxActiveClusters(&n, kern, &cfg) != cudaSuccess) {
        (void)cudaGetLastError();
        return 0;
    }
    return n;
}

// A call's tiles: fills in what the kernel is told of them (p.M, N, halves are set), returns how many there are.
inline long long pair_shape(F4PairParams &p, int workers, const int (&clusters)[2])
{
    p.tiles_n = (p.N + 255) / 256;
    const PairPlan plan = pair_plan(p.M, (p.halves + 1) / 2, p.tiles_n, workers, clusters);
    p.nt = plan.nt;
    p.split_sh = plan.split >> 1;        // 0, 1, 2
    p.tiles_m = (p.M + p.nt - 1) / p.nt;
    const long long tiles = (long long)p.tiles_m * p.tiles_n;
    // Tiles are numbered so that a round of them touches the fewest bytes: rows first, it takes all of a and few channels, or the other way
    // around (2048 x 3584 x 18944 rows first 52.5 us, channels first 54.3; 8192 x 18944 x 3584 215 and 195).
    const long long round = tiles < workers ? tiles : workers;
    const auto bytes = [&](long long tm, long long tn) { return (double)tm * p.nt + (double)tn * 256; };
    const auto up = [](long long a, long long b) { return (a + b - 1) / b; };
    p.rows_fastest = bytes(p.tiles_m < round ? p.tiles_m : round, up(round, p.tiles_m)) < bytes(up(round, p.tiles_n), p.tiles_n < round ? p.tiles_n : round);
    const uint32_t inner = (uint32_t)(p.rows_fastest ? p.tiles_m : p.tiles_n);
    p.tile_mul = inner > 1 && tiles < 65536 ? 0xFFFFFFFFu / inner + 1u : 0u;
    // An output that does not fit L2 beside the operands leaves it early (8192 x 4096 x 14336 184 -> 172 us; 4096 x 14336 x 4096 would go 97 -> 105).
    p.stream_y = (size_t)p.M * p.N * 2 > kPairStreamBytes ? 1 : 0;
    return tiles;
}

// Clusters of two and of four pairs of the kernel that device dev, the current one, holds at once.
template <int BLOCK, typename T> inline void pair_capacity(int dev, int (&clusters)[2])
{
    static std::atomic<int> held[kMaxDevices][2];                // + 1 (0: not asked yet)
    for (int i = 0; i < 2; ++i) {
        int n = held[dev][i].load(std::memory_order_relaxed);
        if (n == 0) held[dev][i].store(n = pair_clusters(f4_pair_kernel<BLOCK, T>, 4 << i) + 1, std::memory_order_relaxed);
        clusters[i] = n - 1;
    }
}

template <int BLOCK, typename T>
tman_status launch_pair(F4PairParams p, cudaStream_t s)
{
    auto kern = f4_pair_kernel<BLOCK, T>;
    static std::atomic<bool> raised[kMaxDevices];
    int dev = 0;
    const DeviceInfo *info = device_info(&dev);
    if (!info) return TMAN_ERR_CUDA;
    int clusters[2];
    pair_capacity<BLOCK, T>(dev, clusters);
    const int workers = info->sms.load(std::memory_order_relaxed) / 2;
    const long long tiles = pair_shape(p, workers, clusters);
    if (tiles > 0x7FFFFFFF) return TMAN_ERR_SHAPE;
    p.stages = pair_stages<BLOCK>();
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)((2 << p.split_sh) * (tiles < workers ? tiles : workers)));
    cfg.blockDim = dim3(kPairThreads);
    cfg.dynamicSmemBytes = kPairSmem;    // (all of it: no CTA that needs tensor memory beside one of these, which hold all of that)
    cfg.stream = s;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (2u << p.split_sh);
    attr[0].val.clusterDim.y = 1;
    attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    const F4Order::Call call = f4_read_ahead(s, p.w);
    cfg.numAttrs = packed_write_pending(s, /*clear=*/true) || call.pending ? 1 : 2;
    const tman_status st = launch_with_smem(kern, kPairSmem, dev, raised, [&] { return cudaLaunchKernelEx(&cfg, kern, p); });
    f4_read_behind(call, st == TMAN_OK);
    return st;
}

}  // namespace
}  // namespace tman
