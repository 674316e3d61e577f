// Products of few rows with microscaled 4-bit weights, bound by the weights' bytes.
//
// y[m][n] = row_scale[n] sum_k x[m][k] w[n][k].  A CTA has 128 channels (the rows of the tensor-core tile, one per lane of tensor memory) and a
// contiguous share of the units of k; the rows of x are the tile's columns.  Weights and their scales stream through a ring of shared memory
// by linear bulk copies (the packed layout is the operands' layout), the scales go on to tensor memory by tcgen05.cp, one thread issues
// the block-scaled MMAs: no instruction touches a weight.
//
// DIGITS: x in 16 bits.  The tensor cores multiply e2m1 with e2m1, so a row of x becomes eight columns of balanced octal digits.  In a block of 16
// or 32 values with largest magnitude in [2^E, 2^(E+1)) every x is the fixed-point number 2^(E-20) X, X = round(x 2^(20-E)) < 2^21, off by
// at most 2^(E-21); X = sum_j n_j 8^j with eight digits n_j in [-4, 4], and n_j / 2 is an e2m1 value.  Column 8 m + j holds the digits n_j of
// row m, the block's scale (2^(E-2) as e8m0; as e4m3 2^E relative to a power of two of the row) is the columns' block scale, and
// x w = 16 (4) sum_j 8^(j-7) (column j): products of digits and weights are exact, sums are in fp32.  (A column counts up to twice what x
// does, -4 + 8 for 4; under 2^E the largest numbers of bf16 would leave the range there.)  Sixteen warps cut x up while the weights arrive.
//
// Otherwise: x is a packed 4-bit matrix, whose units are loaded as they are.
//
// The CTAs of a tile's shares of k form a cluster and add their sums through each other's shared memory, in the order of the shares.
//
// What bounds it, one row in a graph of calls, each after the one before, weights rotated over 300 MB (32-value blocks; the weights' bytes alone take
// 4.8 us): 4096 x 14336 7.7 us, 14336 x 4096 7.5, 4096 x 4096 4.0 of 1.4, 4096 x 1024 3.0 of 0.3; with weights in L2 6.5, 6.5, 4.2 and 3.5.
// About 3 us a call pass between the wait for the kernel ahead and the first product (x from L2, its digits) and between the last one and the
// end of the kernel; in between the weights' bytes in flight bound it (an earlier version of the kernel: rings of 74 / 111 / 220 KB a CTA 8.9 / 7.6 / 7.3 us for
// 4096 x 14336 and 9.1 / 7.2 / 8.6 for 14336 x 4096; with all of an SM's memory the next call cannot fetch its weights beside this one).  More rows
// leave a ring fewer stages: two, four and eight take 7.9, 8.4 and 10.1 us, in 16-value blocks of 14336 x 4096 8.7, 10.8 and 12.7.
// More tiles than SMs: a second CTA starts on an SM when the first has given up its right to tensor memory, which it takes behind the wait (see
// there).  So these calls cannot start early with all of their CTAs: 4096 x 20480 10.6 us, 4096 x 28672 12.4 (9.5 and 11.6 with the tensor
// memory taken ahead of the wait; behind a kernel that does not signal early the two orders are within 4 %).
// Tried and slower, on earlier versions: the weights' later units prefetched into L2 before the wait (8.6 -> 9.0), separate rings for weights and x,
// also with two tiles a CTA (7.5 -> 8.4, eight rows 9.7 -> 12.2: a second wait and commit a unit), two CTAs an SM (4096 x 4096 3.9 -> 5.6), sums
// fetched from the other CTAs between two cluster barriers instead of sent (4096 x 4096 5.2, sent and with the headers checked early 3.9).
#pragma once

#include "f4.cuh"
#include "sm100_ptx.cuh"

#include <type_traits>

namespace tman {
namespace {

constexpr int kDigitWarps = 16;
__host__ __device__ constexpr int stream_threads(bool digits) { return digits ? 64 + 32 * kDigitWarps : 192; }      // warp 0: loads, 1: MMAs, others: digits, epilogue
constexpr int kStreamMaxRows = 64;       // of a packed x
constexpr int kStreamMaxSplit = 8;
constexpr int kStreamHalfSm = 114176,      // (with 1.5 KB that are static and 1 KB of the system's)
               kStreamAllSm = 220 * 1024, kStreamLeastSmem = 57 * 1024;
constexpr int kStreamMaxStages = 12;
// Digits in shared memory: core matrices 16 bytes further apart than they are long, half units 64 bytes (mod 128), so that the stores of a warp
// (four bytes of 32 places along k) meet no bank twice.  Of an odd M the tile's last eight columns are whatever lies behind, of the second half
// unit the 576 bytes from the scales on, which a stage therefore has.
constexpr int kDigitLbo = 144, kDigitSbo = 4 * kDigitLbo;
__host__ __device__ constexpr int digit_half(int M) { return M * kDigitSbo + (M % 2 ? 0 : 64); }

struct F4StreamParams {
    const uint8_t *w, *a;                // packed weights, packed x
    const void *x;
    void *y;
    uint32_t *status;
    size_t w_codes, w_scales, w_rows, a_codes, a_scales, a_rows;
    int M, K, N, ldx, ldy, halves, height8, split, stages, stage_bytes, cols, sms;
};

template <bool DIGITS>
__host__ __device__ inline int stream_b_bytes(int M, int cols) { return DIGITS ? 2 * digit_half(M) : cols * 128; }
// Scales of a unit of x in a stage.  Of digits, at most 64 columns, the scales of 64 values of k take two of the four columns that one copy brings
// to tensor memory: two 512-byte pieces in one.
__host__ __device__ constexpr int stream_sfb_bytes(int block, bool digits) { return digits ? (block == 32 ? 640 : 1024) : 2 * f4_scale_bytes(block); }
static_assert(stream_sfb_bytes(32, true) >= kDigitSbo && stream_sfb_bytes(16, true) >= kDigitSbo, "what an odd M's last columns read lies in the stage");

// Balanced octal digits of eight numbers, as e2m1 codes: word j of the result holds digit j of number i in bits 4 i.
// y[i] = X + sum_{j<7} 4 8^j + 2 8^7, so that octal digit j of y is n_j + 4 (of the top one n_7 + 2).  Spread into nibbles, the digits are
// byte selectors into a table of eight codes.
__device__ __forceinline__ void digit_codes(const uint32_t (&y)[8], uint32_t (&out)[8])
{
    // codes of n = -4 .. 3, of an even number in the low half of a byte, of an odd one in the high half
    const uint32_t t0 = opaque_u32<0x090A0B0Cu>(), t1 = opaque_u32<0x03020100u>(), u0 = opaque_u32<0x90A0B0C0u>(), u1 = opaque_u32<0x30201000u>();
    uint32_t lo[4], hi[4];                       // of two numbers: digits 0..3 and 4..7, a byte each
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
        uint32_t v[2];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            v[e] = y[i + e] + (y[i + e] & 0x00FFF000u) * 15u;
            v[e] += (v[e] & 0x0FC00FC0u) * 3u;
            v[e] += (v[e] & 0x38383838u) + 0x20000000u;
        }
        lo[i / 2] = __byte_perm(t0, t1, v[0]) | __byte_perm(u0, u1, v[1]);
        hi[i / 2] = __byte_perm(t0, t1, v[0] >> 16) | __byte_perm(u0, u1, v[1] >> 16);
    }
    auto bytes = [](const uint32_t (&w)[4], uint32_t *o) {
        const uint32_t a = __byte_perm(w[0], w[1], 0x5140), b = __byte_perm(w[2], w[3], 0x5140);
        const uint32_t d = __byte_perm(w[0], w[1], 0x7362), e = __byte_perm(w[2], w[3], 0x7362);
        o[0] = __byte_perm(a, b, 0x5410);
        o[1] = __byte_perm(a, b, 0x7632);
        o[2] = __byte_perm(d, e, 0x5410);
        o[3] = __byte_perm(d, e, 0x7632);
    };
    bytes(lo, out);
    bytes(hi, out + 4);
}

// Row scales of weights as a power of two times what is left of them: 1 to 2, or all of what is not an ordinary number.
__device__ __forceinline__ int scale_exponent(float s)
{
    const int e = (int)(__float_as_uint(s) >> 23 & 255u);
    return e == 0 || e == 255 ? 0 : e - 127;
}
__device__ __forceinline__ float scale_rest(float s)
{
    const uint32_t u = __float_as_uint(s), e = u >> 23 & 255u;
    return e == 0u || e == 255u ? s : __uint_as_float((u & 0x807FFFFFu) | 0x3F800000u);
}
// v 2^e, e from -252 to 254: exact where the result is an ordinary number.
__device__ __forceinline__ float times_power(float v, int e)
{
    const int h = e >> 1;
    return v * __uint_as_float((uint32_t)(h + 127) << 23) * __uint_as_float((uint32_t)(e - h + 127) << 23);
}

template <int BLOCK, typename T, bool DIGITS>
__global__ void __launch_bounds__(stream_threads(DIGITS), DIGITS ? 2 : 1) f4_stream_kernel(const __grid_constant__ F4StreamParams p)
{
    extern __shared__ __align__(128) uint8_t smem[];
    __shared__ __align__(8) uint64_t full_bar[kStreamMaxStages], empty_bar[kStreamMaxStages], acc_bar, sums_bar;
    __shared__ uint32_t tmem_slot, row_top[8], bad_header;
    __shared__ float w_row[128], a_row[kStreamMaxRows];
    constexpr uint32_t SB = f4_scale_bytes(BLOCK), CHUNKS = SB / 512;
    const int warp = __shfl_sync(0xffffffffu, (int)threadIdx.x >> 5, 0), lane = threadIdx.x & 31;      // (the shuffle tells the compiler that it is uniform)
    const int rank = blockIdx.x % p.split, tile = blockIdx.x / p.split, steps = (p.halves + 1) >> 1;
    const int u0 = steps * rank / p.split, nu = steps * (rank + 1) / p.split - u0;     // units of this share
    const int b_bytes = stream_b_bytes<DIGITS>(p.M, p.cols);
    const uint32_t full0 = smem_u32(full_bar), empty0 = smem_u32(empty_bar), accf = smem_u32(&acc_bar), ring = smem_u32(smem);
    const uint32_t off_sfa = kF4Tile * 128, off_b = off_sfa + 2 * SB, off_sfb = off_b + (uint32_t)b_bytes;
    constexpr uint32_t tmem_cols = 128;      // up to 64 of sums, two sets of scales (16 each) behind them
    // Sums of a tile's shares: every CTA sends its own to the CTA that adds up a channel, [share][row][own channel] behind its ring.
    const bool push = p.split > 1;
    const int per = (128 + p.split - 1) / p.split, own0 = per * rank, own_n = min(per, 128 - own0);      // channels added up here
    bool ok = true;

    if (threadIdx.x == 0) {
        for (int s = 0; s < p.stages; ++s) {
            mbar_init(full0 + 8 * s, DIGITS ? 1 + p.M : 1);
            mbar_init(empty0 + 8 * s, 1);
        }
        mbar_init(accf, 1);
        mbar_init(smem_u32(&sums_bar), 1);
        if (push) mbar_expect_tx(smem_u32(&sums_bar), (uint32_t)(p.split * p.M * own_n) * 4u);
        fence_barrier_init();
        bad_header = 0u;
    }
    if (threadIdx.x < 8) row_top[threadIdx.x] = 0u;
    __syncthreads();
    // (Waited for before the sums are sent.)  The arrival takes 2 to 3.5 us of a CTA beside a busy one.  That holds the first loads of an early CTA back
    // until the kernel ahead needs the bandwidth less (without it 1 x 14336 x 4096 takes 8.7 us instead of 7.5), but a CTA that shares its SM with another of its
    // own grid starts late and does without, as it has no peers (1 x 4096 x 20480 12.1 -> 10.6 us).
    const bool arrive = push || (int)blockIdx.x < p.sms;
    if (arrive) cluster_arrive();

    // (Warps 0 and 1 walk as one, one lane issues: addresses and descriptors in uniform registers.)
    if (warp == 0) {
        const bool lead = elect_one();
        const int w_tiles = (p.height8 + kF4Tile - 1) / kF4Tile, a_h8 = (p.M + 7) / 8 * 8;
        const uint32_t wb_full = (uint32_t)min(kF4Tile, p.height8 - tile * kF4Tile) * 128u, ab_full = DIGITS ? 0u : (uint32_t)a_h8 * 128u;
        auto load = [&](int i, int s, bool do_w, bool do_a) {
            const int u = u0 + i;
            const uint32_t sh = 2 * u + 1 < p.halves ? 0u : 1u;  // a half unit's sections are half as wide
            const uint8_t *w = p.w + p.w_codes + (size_t)u * p.height8 * 128 + ((size_t)tile * (kF4Tile * 128) >> sh);
            const uint8_t *ws = p.w + p.w_scales + (size_t)u * w_tiles * (2 * SB) + ((size_t)tile * (2 * SB) >> sh);
            const uint8_t *a = p.a + p.a_codes + (size_t)u * a_h8 * 128, *as = p.a + p.a_scales + (size_t)u * (2 * SB);
            const uint32_t wb = wb_full >> sh, ab = ab_full >> sh, sb = 2 * SB >> sh, st = ring + (uint32_t)(s * p.stage_bytes), bar = full0 + 8 * s;
            if (lead) {
                if (do_w) {
                    mbar_expect_tx(bar, DIGITS ? wb + sb : wb + ab + 2 * sb);
                    bulk_load(st, w, wb, bar);
                    bulk_load(st + off_sfa, ws, sb, bar);
                }
                if (do_a) {
                    bulk_load(st + off_b, a, ab, bar);
                    bulk_load(st + off_sfb, as, sb, bar);
                }
            }
            __syncwarp();
        };
        // weights of the first stages before the wait for the kernel ahead: nothing that may still be running writes them
        const int first = min(nu, p.stages);
        for (int i = 0; i < first; ++i) load(i, i, true, false);
        if constexpr (!DIGITS) {
            grid_wait();
            for (int i = 0; i < first; ++i) load(i, i, false, true);
        }
        int s = 0;
        uint32_t ph = 0;
        for (int i = first; i < nu; ++i) {
            if (!warp_all(mbar_wait(empty0 + 8 * s, ph))) { ok = false; break; }
            load(i, s, true, !DIGITS);
            if (++s == p.stages) { s = 0; ph ^= 1u; }
        }
    } else if (warp == 1) {
        // Tensor memory is taken behind the wait for the kernel ahead, which may be one that signals before it takes its own (each would wait for
        // the other), and before the signal to the next.
        grid_wait();
        tcgen05_alloc(smem_u32(&tmem_slot), tmem_cols);
        tcgen05_relinquish();
        grid_launch_next();
        __syncwarp();
        const uint32_t tmem = __shfl_sync(0xffffffffu, *const_cast<volatile uint32_t *>(&tmem_slot), 0);
        const bool lead = elect_one();
        const uint32_t id0 = f4_idesc(BLOCK, 128, p.cols, 0), id1 = f4_idesc(BLOCK, 128, p.cols, BLOCK == 32 ? 2 : 0);
        const uint64_t sf0 = make_kmajor_desc(ring, 128, 128);                     // (+ 1: 16 bytes)
        const uint32_t b_half = DIGITS ? (uint32_t)digit_half(p.M) : 512u, b_chunk = DIGITS ? kDigitLbo : 128;
        int s = 0;
        uint32_t ph = 0;
        for (int i = 0; i < nu; ++i) {
            const uint32_t at = (uint32_t)(s * p.stage_bytes) >> 4, two = 2 * (u0 + i) + 1 < p.halves ? 2u : 1u;
            const uint64_t wd = make_kmajor_desc(ring, 128, two * 512) + at, sf = sf0 + at;
            const uint64_t xd = make_kmajor_desc(ring + off_b, b_chunk, DIGITS ? kDigitSbo : two * 512) + at;
            if (!warp_all(mbar_wait(full0 + 8 * s, ph))) { ok = false; break; }
            tcgen05_fence_after();
            if (lead) {
                // (scales of both halves, then the products: the scales' copies follow one another)
                const uint32_t sfa = tmem + (uint32_t)p.cols, sfb = sfa + 8u;
#pragma unroll
                for (uint32_t u = 0; u < 2; ++u)
                    if (u < two)
#pragma unroll
                        for (uint32_t c = 0; c < CHUNKS; ++c) {
                            tcgen05_cp_scales(sfa + 16 * u + 4 * c, sf + ((off_sfa + u * SB + 512 * c) >> 4));
                            if constexpr (!DIGITS) tcgen05_cp_scales(sfb + 16 * u + 4 * c, sf + ((off_sfb + u * SB + 512 * c) >> 4));
                            else if (c == 0 && (BLOCK == 16 || u == 0)) tcgen05_cp_scales(sfb + 16 * u, sf + ((off_sfb + 512 * u) >> 4));
                        }
#pragma unroll
                for (uint32_t u = 0; u < 2; ++u)
                    if (u < two) {
                        const uint64_t wa = wd + ((u * 512) >> 4), xb = xd + ((u * b_half) >> 4);
                        const uint32_t fb = DIGITS && BLOCK == 32 ? sfb + 2 * u : sfb + 16 * u;
                        tcgen05_mma_f4<BLOCK>(tmem, wa, xb, id0, sfa + 16 * u, fb, (i | (int)u) != 0);
                        tcgen05_mma_f4<BLOCK>(tmem, wa + 16, xb + ((2 * b_chunk) >> 4), id1, sfa + 16 * u + (BLOCK == 32 ? 0 : 4),
                                              fb + (BLOCK == 32 ? 0 : DIGITS ? 2 : 4), 1);
                    }
                tcgen05_commit(empty0 + 8 * s);
            }
            __syncwarp();
            if (++s == p.stages) { s = 0; ph ^= 1u; }
        }
        if (lead) tcgen05_commit(accf);
        __syncwarp();
    } else {
        const int pt = threadIdx.x - 64;
        // The weights' header and row scales: asked for before the wait, like the weights, and looked at when the products are under way.  Past the
        // L1, which an early launch does not empty of what an earlier call left there.
        uint4 head0 = make_uint4(0u, 0u, 0u, 0u);
        uint2 head1 = make_uint2(0u, 0u);
        float row_scale = 0.f;
        if (pt == 0) {
            head0 = __ldcg(reinterpret_cast<const uint4 *>(p.w));
            head1 = __ldcg(reinterpret_cast<const uint2 *>(p.w + 16));
        }
        if (BLOCK == 16 && pt < 128 && tile * 128 + pt < p.N) row_scale = __ldcg(reinterpret_cast<const float *>(p.w + p.w_rows) + tile * 128 + pt);
        grid_wait();
        if constexpr (!DIGITS) {
            if (pt == 32 && !f4_header_matches(p.a, p.M, p.K, BLOCK)) bad_header = 1u;
            if (BLOCK == 16 && pt < p.M) a_row[pt] = ld_dependent(reinterpret_cast<const float *>(p.a + p.a_rows) + pt);
        } else {
            const T *x = static_cast<const T *>(p.x);
            const int l16 = lane & 15;
            // A warp has a row, and of its units every `teams`-th; a lane eight of a unit's 256 values.  A wait for a free slot names its turn by parity
            // alone: it holds only where the turn before is known to have passed.  So a warp's units lie at most a round of the ring
            // apart: the unit before, whose slot's turn it has waited for, is at least as late.
            const int all_teams = kDigitWarps / p.M, teams = min(all_teams, p.stages), team = (warp - 2) / p.M, m = (warp - 2) - team * p.M;
            const uint4 *xm = reinterpret_cast<const uint4 *>(x + (size_t)m * p.ldx) + lane;
            auto fetch = [&](int i) {
                const int at = (u0 + i) * (2 * kF4Half / 8);
                return i < nu && at + lane < p.K / 8 ? ld_dependent(xm + at) : make_uint4(0u, 0u, 0u, 0u);
            };
            auto top_of = [](uint32_t t, const uint4 &v) {
                return __vmaxu2(t, __vmaxu2(__vmaxu2(v.x & 0x7FFF7FFFu, v.y & 0x7FFF7FFFu), __vmaxu2(v.z & 0x7FFF7FFFu, v.w & 0x7FFF7FFFu)));
            };
            uint4 next = make_uint4(0u, 0u, 0u, 0u);
            if (team < all_teams) next = fetch(team);
            if constexpr (BLOCK == 16) {
                // the largest magnitude of each row of this share of k (of a row that holds an infinity or a NaN: whatever comes out); every value is
                // asked for once a CTA: all CTAs read the same few lines
                if (team < all_teams) {
                    uint32_t t = top_of(0u, next);
#pragma unroll 4
                    for (int i = team + all_teams; i < nu; i += all_teams) t = top_of(t, fetch(i));
                    t = __reduce_max_sync(0xffffffffu, max(t & 0xFFFFu, t >> 16));
                    if (lane == 0) atomicMax(&row_top[m], t);
                }
                asm volatile("bar.sync 1, %0;" ::"n"(32 * kDigitWarps) : "memory");
            }
            int s = team;
            uint32_t ph = 1;                                     // (the first round of the ring does not wait)
            for (int i = team; i < nu && team < teams; i += teams, s += teams) {
                if (s >= p.stages) { s -= p.stages; ph ^= 1u; }
                const uint4 cur = next;
                next = fetch(i + teams);
                const uint32_t w[4] = {cur.x, cur.y, cur.z, cur.w};
                float f[8];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float2 v = f4_to_float2<T>(w[e]);
                    f[2 * e] = v.x;
                    f[2 * e + 1] = v.y;
                }
                // the block's largest magnitude as a bit pattern (they order like the values, infinities and NaN above all others), its exponent
                uint32_t t2 = top_of(0u, cur);
#pragma unroll
                for (int o = BLOCK / 16; o; o >>= 1) t2 = __vmaxu2(t2, __shfl_xor_sync(0xffffffffu, t2, o));
                const uint32_t eb = __float_as_uint(f4_to_float2<T>(max(t2 & 0xFFFFu, t2 >> 16)).x) >> 23;
                uint32_t byte;                                   // the block's scale
                int e2;                                          // E + 127
                if constexpr (BLOCK == 32) {
                    e2 = max((int)eb, std::is_same<T, __half>::value ? 103 : 3);
                    byte = eb == 255u ? 255u : (uint32_t)e2 - 2u;
                } else {
                    const uint32_t rt = row_top[m];
                    // the row's power of two, + 127 (at least 2^-111: bf16's smallest numbers are then off by 2^-141 at most, a 2^-8 of the least of them)
                    const int r2 = max((int)(__float_as_uint(f4_to_float2<T>(rt).x) >> 23) - 8, 16);
                    e2 = min(max((int)eb, r2 - 9), r2 + 8);
                    const int d = e2 - r2;                       // -9 .. 8
                    byte = eb == 255u ? 0x7Fu : d >= -6 ? (uint32_t)(d + 7) << 3 : 1u << (d + 9);
                }
                // X + bias in the low 23 bits of 2^23 + X + bias
                constexpr float kMagic = 8388608.f + 4.f * 299593.f + 2.f * 2097152.f;      // 299593 = (8^7 - 1) / 7
                uint32_t yb[8];
                if constexpr (std::is_same<T, __half>::value) {
                    const float mul = __uint_as_float((uint32_t)(127 + 20 + 127 - e2) << 23);           // 2^(20 - E), E >= -24
#pragma unroll
                    for (int e = 0; e < 8; ++e) yb[e] = __float_as_uint(fmaf(f[e], mul, kMagic)) - 0x4B000000u;
                } else {
                    const int q = 147 - e2, qa = q >> 1;                                              // E down to -126: in two factors
                    const float ma = __uint_as_float((uint32_t)(127 + qa) << 23), mb = __uint_as_float((uint32_t)(127 + q - qa) << 23);
#pragma unroll
                    for (int e = 0; e < 8; ++e) yb[e] = __float_as_uint(fmaf(f[e] * ma, mb, kMagic)) - 0x4B000000u;
                }
                uint32_t d[8];
                digit_codes(yb, d);
                // four blocks' scales: lanes of a block 4 (2) apart, four blocks in 16 (8) lanes
                uint32_t word = byte << (BLOCK == 32 ? 2 * (lane & 12) : 4 * (lane & 6));
                word |= __shfl_xor_sync(0xffffffffu, word, BLOCK / 8);
                word |= __shfl_xor_sync(0xffffffffu, word, BLOCK / 4);
                ok = warp_all(mbar_wait(empty0 + 8 * s, ph));
                if (!ok) break;
                uint8_t *st = smem + (size_t)s * p.stage_bytes;
                if (lane < 16 || 2 * (u0 + i) + 1 < p.halves) {
                    uint8_t *b = st + off_b + (lane >> 4) * digit_half(p.M) + m * kDigitSbo + (l16 >> 2) * kDigitLbo + (l16 & 3) * 4;
#pragma unroll
                    for (int e = 0; e < 8; ++e) *reinterpret_cast<uint32_t *>(b + e * 16) = d[e];
                    if (BLOCK == 16 || l16 < 8) {
                        const int t = 8 * m + (l16 & 7);
                        *reinterpret_cast<uint32_t *>(st + off_sfb + (BLOCK == 32 ? (lane >> 4) * 8 : (lane >> 4) * 512 + (l16 >> 3) * 8) + (t & 31) * 16 +
                                                      (t >> 5) * 4) = word;
                    }
                }
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                __syncwarp();
                if (lane == 0) mbar_arrive(full0 + 8 * s);
            }
        }
        if (pt == 0 && !f4_header_is(head0, head1, p.N, p.K, BLOCK)) bad_header = 1u;
        if (BLOCK == 16 && pt < 128) w_row[pt] = row_scale;
    }

    // ---- epilogue: warps 2..5, a channel a lane -------------------------------------------------
    tcgen05_fence_before();
    __syncthreads();                     // row scales and the rest in shared memory are there; roles are done
    if (arrive) cluster_wait();
    tcgen05_fence_after();
    const uint32_t tmem = __shfl_sync(0xffffffffu, tmem_slot, 0);
    const bool hdr_ok = bad_header == 0u;
    if (!hdr_ok && threadIdx.x == 64 && blockIdx.x == 0) atomicCAS(p.status, 0u, (uint32_t)TMAN_ERR_BAD_PACKED);
    T *y = static_cast<T *>(p.y);
    const float *sums = reinterpret_cast<const float *>(smem + (size_t)p.stages * p.stage_bytes);
    if (warp >= 2 && warp < 6) {
        ok = warp_all(mbar_wait(accf, 0)) && ok;
        tcgen05_fence_after();
        const int ch = (warp & 3) * 32 + lane, n = tile * 128 + ch;
        const uint32_t acc = tmem + ((uint32_t)((warp & 3) * 32) << 16);
        const bool put = ok && hdr_ok && n < p.N;
        const float wr = BLOCK == 16 ? w_row[ch] : 1.f;
        // (Digits' sums are of x over a power of two of the row.  That, and the power of two in the weights' row scale, come back in one step: in turn
        // they may leave the range where their product does not.  Powers of two change no rounding.)
        [[maybe_unused]] const int w_exp = scale_exponent(wr);
        const int to = ch / per;
        const uint32_t to_sums = mapa_u32(smem_u32(sums), (uint32_t)to) + (uint32_t)((rank * p.M) * per + ch - to * per) * 4u, to_bar = mapa_u32(smem_u32(&sums_bar), (uint32_t)to);
        auto give = [&](int m, float v) {
            if (push) store_cluster(to_sums + (uint32_t)(m * per) * 4u, v, to_bar);
            else if (put) y[(size_t)m * p.ldy + n] = f4_from_float<T>(BLOCK == 16 ? (DIGITS ? v * scale_rest(wr) : v * wr * a_row[m]) : v);
        };
        if constexpr (DIGITS) {
#pragma unroll 1
            for (int m = 0; m < p.M; ++m) {
                uint32_t r[8];
                tcgen05_ld_32x32b_x8(acc + 8 * m, r);
                tcgen05_wait_ld();
                float v = __uint_as_float(r[0]);
#pragma unroll
                for (int e = 1; e < 8; ++e) v = fmaf(v, 0.125f, __uint_as_float(r[e]));
                if constexpr (BLOCK == 16) v = times_power(v, max((int)(__float_as_uint(f4_to_float2<T>(row_top[m]).x) >> 23) - 8, 16) - 127 + 2 + w_exp);
                else v *= 16.f;
                give(m, v);
            }
        } else {
#pragma unroll 1
            for (int m = 0; m < p.M; m += 16) {
                uint32_t r[16];
                tcgen05_ld_32x32b_x16(acc + m, r);
                tcgen05_wait_ld();
#pragma unroll
                for (int e = 0; e < 16; ++e)
                    if (m + e < p.M) give(m + e, __uint_as_float(r[e]));
            }
        }
    }
    if (push && warp >= 2 && warp < 6) {
        // (Every CTA sends its sums, whatever its own waits say, within their limit of a second each: waited for several times as
        // long, so that no CTA is gone when sums for it arrive.)
        bool all = false;
        for (int i = 0; i < 8 && !all; ++i) all = warp_all(mbar_wait(smem_u32(&sums_bar), 0));
        ok = ok && all;
        for (int i = threadIdx.x - 64; i < p.M * own_n; i += 128) {
            const int m = i / own_n, c = i - m * own_n, n = tile * 128 + own0 + c;
            float v = 0.f;
            for (int r = 0; r < p.split; ++r) v += sums[(r * p.M + m) * per + c];
            if constexpr (BLOCK == 16) v = DIGITS ? v * scale_rest(w_row[own0 + c]) : v * w_row[own0 + c] * a_row[m];
            if (ok && hdr_ok && n < p.N) y[(size_t)m * p.ldy + n] = f4_from_float<T>(v);
        }
    }
    if (!ok) atomicCAS(p.status, 0u, (uint32_t)TMAN_ERR_TIMEOUT);
    tcgen05_fence_before();
    __syncthreads();
    if (warp == 1) {
        tcgen05_fence_after();
        tcgen05_dealloc(tmem, tmem_cols);
    }
}

// Clusters of `split` CTAs that the device holds at once with an SM for each CTA; `clusters`: of four and of eight.
inline int stream_fit(int split, int sms, const int (&clusters)[2])
{
    return split <= 2 ? sms / split : split < 7 ? clusters[0] * 4 / split : clusters[1];
}
// Shares of k: as many as give every SM a CTA at most (4096 x 4096, one row: four shares 3.9 us, eight, two CTAs an SM, 5.6), in clusters that fit so: a CTA
// that shares its SM starts late (see above).
inline int stream_split(int tiles, int units, int sms, const int (&clusters)[2])      // units of 256
{
    int best = 1;
    for (int s = 2; s <= kStreamMaxSplit && units >= s; ++s)
        if (tiles <= stream_fit(s, sms, clusters)) best = s;
    return best;
}

// Modelled time of a packed x of M rows here, beside what the weights' bytes cost either kernel.  A row costs its stores, a unit its loads, and in
// shares the sums of the own channels are added up row by row.
inline double stream_us(int M, int units, int tiles, int sms, const int (&clusters)[2])
{
    const int split = stream_split(tiles, units, sms, clusters), share = (units + split - 1) / split, rounds = (tiles * split + sms - 1) / sms;
    return 1.5 + 0.045 * M + 0.225 * share * rounds + (split > 1 ? 0.23 * M / split : 0.0);
}

struct StreamPlan { int tiles, cols, split, stages, stage_bytes, smem; };
inline StreamPlan stream_plan(int M, int K, int N, int block, bool digits, int sms, const int (&clusters)[2])
{
    StreamPlan t;
    const int halves = (K + kF4Half - 1) / kF4Half, steps = (halves + 1) / 2;
    t.tiles = (N + kF4Tile - 1) / kF4Tile;
    t.cols = digits ? (M + 1) / 2 * 16 : (M + 15) / 16 * 16;
    t.split = stream_split(t.tiles, steps, sms, clusters);
    const int b_bytes = digits ? stream_b_bytes<true>(M, t.cols) : stream_b_bytes<false>(M, t.cols);
    t.stage_bytes = (kF4Tile * 128 + 2 * f4_scale_bytes(block) + stream_sfb_bytes(block, digits) + b_bytes + 127) / 128 * 128;
    // Half an SM's shared memory, so that the next call's CTAs fill their rings beside this one's; all of it where half holds fewer than three stages
    // beside the sums (64 rows of 32-value blocks: 14336 x 4096 15.5 us with two stages, 12.7 with seven; 28672 x 4096 23.6 and 17.4), or, of a packed
    // x, fewer than four without them.
    const int sums = t.split > 1 ? (128 + 8) * M * 4 : 0;
    const int budget = t.stage_bytes * 3 + sums <= kStreamHalfSm && (digits || t.stage_bytes * 4 <= kStreamHalfSm) ? kStreamHalfSm : kStreamAllSm;
    t.stages = (budget - sums) / t.stage_bytes;
    if (t.stages > kStreamMaxStages) t.stages = kStreamMaxStages;
    const int share = (steps + t.split - 1) / t.split;
    if (t.stages > share) t.stages = share;
    // (at least a quarter of an SM's, so that no more CTAs share an SM than its tensor memory has room for: CTAs of a cluster wait for one another,
    // which one that waits for tensor memory must not hold up)
    t.smem = t.stages * t.stage_bytes + sums;
    if (t.smem < kStreamLeastSmem) t.smem = kStreamLeastSmem;
    return t;
}

template <int BLOCK, typename T, bool DIGITS>
tman_status launch_stream(F4StreamParams p, const int (&clusters)[2], cudaStream_t s)
{
    auto kern = f4_stream_kernel<BLOCK, T, DIGITS>;
    static std::atomic<bool> raised[kMaxDevices];
    int dev = 0;
    const DeviceInfo *info = device_info(&dev);
    if (!info) return TMAN_ERR_CUDA;
    p.sms = info->sms.load(std::memory_order_relaxed);
    const StreamPlan plan = stream_plan(p.M, p.K, p.N, BLOCK, DIGITS, p.sms, clusters);
    p.cols = plan.cols;
    p.split = plan.split;
    p.stages = plan.stages;
    p.stage_bytes = plan.stage_bytes;
    if ((long long)plan.tiles * p.split > 0x7FFFFFFF) return TMAN_ERR_SHAPE;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(plan.tiles * p.split));
    cfg.blockDim = dim3((unsigned)stream_threads(DIGITS));
    cfg.dynamicSmemBytes = (size_t)plan.smem;
    cfg.stream = s;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)p.split;
    attr[0].val.clusterDim.y = 1;
    attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    // (also a cluster of one: without the attribute the next call's CTAs do not spread over the SMs, 1 x 3584 x 18944 7.1 -> 8.9 us)
    cfg.attrs = attr;
    const F4Order::Call call = f4_read_ahead(s, p.w);
    cfg.numAttrs = packed_write_pending(s, /*clear=*/true) || call.pending ? 1 : 2;
    const tman_status st = launch_with_smem(kern, kStreamAllSm, dev, raised, [&] { return cudaLaunchKernelEx(&cfg, kern, p); });
    f4_read_behind(call, st == TMAN_OK);
    return st;
}

}  // namespace
}  // namespace tman
