// Attention over the 8-bit cache for many new tokens of a sequence.
//
// What bounds it is the exponential function (16 a clock and SM) and the tensor cores, which take as long.  A CTA has up to 256 rows (new tokens x
// query heads of one key head) in two tiles of 128 (one where heads are wide), and walks over the keys 64 at a time.  Four warps bring keys and
// values from the cache, make fp16 of the bytes and lay them out as the tensor cores' operands; one thread issues the MMAs (scores: rows x keys; output:
// rows x columns, both in tensor memory); four warps a tile of rows, a thread a row, do the softmax.  A tile of rows has two buffers of
// scores: while one is worked on, the other is filled, so that the softmax warps need not wait for the tensor cores.
// A score is (q . code) x (key page's scale) x scale; probabilities carry the value page's scale, p' = 2^(s + log2 vs - M), so that codes are what they are
// multiplied with, and the row's sum is that of p' / vs, of p' as fp16 holds it: what the rounding takes from a probability it takes from the sum too, so that one
// that counts for nearly all is not off (with sums ahead of the rounding it was, by up to 2^-12, since M need not be the maximum).  Pages whose values are small
// beside others' may count for much in the sum and be far down in fp16's range: theirs are added up ahead of the rounding.  1 / vs is relative to a power of two
// that follows the largest vs, so that values of any size have their sum in range; the maximum does not see pages of zeros, whose vs is taken as very small.
// Probabilities go back to tensor memory over the scores, as the A operand of the second product.  M
// is the maximum so far and raised, and the output so far scaled, only when a score is above it by more than 10: p' is at most 2^10, rows seldom
// raise it after their first keys, and one pass over the scores is enough; one that finds such a score is made again behind the raise.
// 2 x 2048 new tokens over 4096, 32 heads of 128 (floor 87): scores twice from tensor memory and a wait for both products in turn 274 us; with one pass, keys
// 128 at a time, 197 (two threads a row instead of one made no difference); keys 64 at a time 190, a tile in 2250 clocks;
// with sums of the rounded probabilities, this, 197.
#pragma once

#include "attend.cuh"

namespace tman {
namespace {

template <int D> struct PromptShape {
    static constexpr int kKeys = 64, kTiles = D <= 128 ? 2 : 1, kSoft = 4 * kTiles, kLoad = 4, kStages = D <= 128 ? 4 : D <= 192 ? 3 : 2;
    static constexpr int kThreads = 32 * (kSoft + kLoad + kTiles), kRows = 128 * kTiles;
    static constexpr int kQ = kRows * D * 2, kKv = kKeys * D * 2, kSmem = kQ + 2 * kStages * kKv + 1024;
    static constexpr int kScore = 0, kOut = 2 * kTiles * kKeys;  // columns of tensor memory
    static constexpr int kConsts = 8;                            // tiles whose pages' scales are kept: the loads are up to kStages + 1 ahead of the softmax
    static_assert(kOut + kTiles * D <= 512 && kSmem <= 227 * 1024 && kStages + 2 <= kConsts, "it fits");
};

struct PromptParams {
    CacheSeqs c;
    const void *q;
    void *y;
    int ldq, ldy, group, window, least;  // least: rows (tokens x group) that a sequence must have to be done here
    float scale;
};

constexpr float kPromptSmall = 0.125f;   // scales of values below this much of the largest are small
constexpr float kPromptLeast = 0x1p-64f; // relative to 2^unit: smaller ones, and zero, count as this
constexpr int kPromptMargin = 16;        // a scale that is larger than 2^unit by 2^this raises the unit
constexpr float kPromptSlack = 10.f;     // a score above the maximum so far by this much raises it

// Two fp16 numbers added to two sums in 32 bits.
__device__ __forceinline__ void add_halves(float &lo, float &hi, uint32_t pair)
{
    asm("{\n.reg .f16 a, b;\nmov.b32 {a, b}, %2;\nadd.rn.f32.f16 %0, a, %0;\nadd.rn.f32.f16 %1, b, %1;\n}" : "+f"(lo), "+f"(hi) : "r"(pair));
}
__device__ __forceinline__ void fence_async_shared() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

template <typename T, int D>
__global__ void __launch_bounds__(PromptShape<D>::kThreads, 1) attend_prompt_kernel(const __grid_constant__ PromptParams p)
{
    using Sh = PromptShape<D>;
    constexpr int KT = Sh::kKeys, RT = Sh::kTiles, GROUPS = KT / 16, NS = Sh::kStages;
    extern __shared__ __align__(1024) uint8_t prompt_smem[];
    __shared__ __align__(8) uint64_t q_bar, k_full[NS], k_empty[NS], v_full[NS], v_empty[NS], s_full[RT][2], p_full[RT][2], o_full[RT], all_bar[RT];
    __shared__ uint32_t tmem_slot;
    // of 16 keys: scale of the keys, log2 of the values' scale, its reciprocal times 2^unit (negative: sums ahead of the rounding), unit
    __shared__ float4 page_consts[Sh::kConsts][GROUPS];
    __shared__ int found[2], sums[Sh::kThreads / 32 + 1];
    const CacheSeqs &c = p.c;
    const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31, page_mask = (1 << c.page_sh) - 1;
    const uint32_t base = (smem_u32(prompt_smem) + 1023u) & ~1023u;
    uint8_t *smem = prompt_smem + (base - smem_u32(prompt_smem));
    const uint32_t qs = base, ks = base + Sh::kQ, vs = ks + NS * Sh::kKv;
    if (tid == 0) {
        mbar_init(smem_u32(&q_bar), 4 * RT);
        for (int i = 0; i < NS; ++i) {
            mbar_init(smem_u32(&k_full[i]), Sh::kLoad);
            mbar_init(smem_u32(&v_full[i]), Sh::kLoad);
            mbar_init(smem_u32(&k_empty[i]), RT);
            mbar_init(smem_u32(&v_empty[i]), RT);
        }
        for (int r = 0; r < RT; ++r) {
            for (int i = 0; i < 2; ++i) {
                mbar_init(smem_u32(&s_full[r][i]), 1);
                mbar_init(smem_u32(&p_full[r][i]), 4);
            }
            mbar_init(smem_u32(&o_full[r]), 1);
            mbar_init(smem_u32(&all_bar[r]), 1);
        }
        found[0] = -1;
        fence_barrier_init();
    }
    grid_wait();
    // ---- blocks of rows, counted over the sequences: which one is this CTA's.  A sequence's last rows, which see the most keys, come first.
    const int head = blockIdx.x % c.heads, index = blockIdx.x / c.heads;
    {
        const int per = (c.S + Sh::kThreads - 1) / Sh::kThreads, s0 = min(tid * per, c.S), s1 = min(s0 + per, c.S);
        auto blocks_of = [&](int s) {
            const CacheSeq q = cache_seq(c, s);
            const int rows = q.rows * p.group;
            return rows < p.least ? 0 : (rows + Sh::kRows - 1) / Sh::kRows;
        };
        int mine = 0;
        for (int s = s0; s < s1; ++s) mine += blocks_of(s);
        int upto = mine;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const int o = __shfl_up_sync(0xffffffffu, upto, d);
            if (lane >= d) upto += o;
        }
        if (lane == 31) sums[warp] = upto;
        __syncthreads();
        for (int w = 0; w < warp; ++w) upto += sums[w];
        int before = upto - mine;
        if (index >= before && index < upto)
            for (int s = s0; s < s1; ++s) {
                const int n = blocks_of(s);
                if (index < before + n) {
                    found[0] = s;
                    found[1] = n - 1 - (index - before);
                    break;
                }
                before += n;
            }
        __syncthreads();
    }
    const int seq = found[0];
    if (seq < 0) return;                                         // (all threads; a block that exits lets the next kernel start)
    const CacheSeq q = cache_seq(c, seq);
    const int row0 = found[1] * Sh::kRows, rows = min(q.rows * p.group - row0, Sh::kRows), pos0 = q.len - q.rows;
    const int first = pos0 + row0 / p.group, last = pos0 + (row0 + rows - 1) / p.group;      // positions of the first and the last row
    const int hi = max(last + 1, 0), lo = window_from(first, p.window);
    const int tile0 = lo / KT, tiles = max((hi + KT - 1) / KT - tile0, 1), active = RT == 2 && rows > 128 ? 2 : 1;       // tiles of keys, of rows
    if (warp == Sh::kSoft + Sh::kLoad) {
        tcgen05_alloc(smem_u32(&tmem_slot), 512);
        tcgen05_relinquish();
    }
    tcgen05_fence_before();
    __syncthreads();
    tcgen05_fence_after();
    grid_launch_next();
    const uint32_t tmem = __shfl_sync(0xffffffffu, tmem_slot, 0);
    bool ok = true;

    if (warp < Sh::kSoft) {
        // ---- softmax: a thread has a row
        const int r = warp >> 2, local = (warp & 3) * 32 + lane, row = r * 128 + local;
        if (r >= active) {
            if (lane == 0) mbar_arrive(smem_u32(&q_bar));
        } else {
            const bool real = row < rows;
            const int rho = row0 + min(row, rows - 1), token = rho / p.group;
            const size_t head_at = (size_t)(head * p.group + rho % p.group) * D;
            const T *src = static_cast<const T *>(p.q) + (size_t)(q.row + token) * p.ldq + head_at;
            float f = 1.f;
            if constexpr (!std::is_same<T, __half>::value) {     // a bf16 row into fp16's range by a power of two
                uint32_t top = 0;
                for (int i = 0; i < D / 8; ++i) {
                    const uint4 v = ld_dependent(reinterpret_cast<const uint4 *>(src) + i);
                    top = i8_larger(top, i8_larger(i8_larger(i8_magnitudes(v.x), i8_magnitudes(v.y)), i8_larger(i8_magnitudes(v.z), i8_magnitudes(v.w))));
                }
                top = max(top & 0xFFFFu, top >> 16);
                f = top == 0 || top >= i8_infinity<T>() ? 1.f : __uint_as_float((uint32_t)(127 + min(141 - (int)(top >> 7), 100)) << 23);
            }
#pragma unroll 4
            for (int i = 0; i < D / 8; ++i) {
                uint4 v = make_uint4(0, 0, 0, 0);
                if (real) v = ld_dependent(reinterpret_cast<const uint4 *>(src) + i);
                if constexpr (!std::is_same<T, __half>::value) {
                    const float2 a = f4_to_float2<T>(v.x), b = f4_to_float2<T>(v.y), d = f4_to_float2<T>(v.z), e = f4_to_float2<T>(v.w);
                    v = make_uint4(f4_from_float2<__half>(a.x * f, a.y * f), f4_from_float2<__half>(b.x * f, b.y * f), f4_from_float2<__half>(d.x * f, d.y * f),
                                   f4_from_float2<__half>(e.x * f, e.y * f));
                }
                *reinterpret_cast<uint4 *>(smem + (r * (D / 64) + (i >> 3)) * 16384 + local * 128 + (((i & 7) ^ (local & 7)) << 4)) = v;
            }
            fence_async_shared();
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&q_bar));

            const float rf = p.scale * kLog2e / f;
            const int limit = pos0 + token, low = window_from(limit, p.window);
            const int least_limit = __reduce_min_sync(0xffffffffu, limit), most_low = __reduce_max_sync(0xffffffffu, low);
            const uint32_t at = tmem + ((uint32_t)((warp & 3) * 32) << 16), out = at + Sh::kOut + r * D;
            float M = -INFINITY, l = 0.f, unit = 0.f;
            for (int j = 0; j < tiles; ++j) {
                const int k0 = (tile0 + j) * KT;
                const bool plain = k0 + KT - 1 <= least_limit && k0 >= most_low;
                const int upto = limit - k0, from = low - k0;      // columns that this row sees
                const float4 *consts = page_consts[j & (Sh::kConsts - 1)];
                const uint32_t score = at + Sh::kScore + (r * 2 + (j & 1)) * KT;
                ok = warp_all(mbar_wait(smem_u32(&s_full[r][j & 1]), (j >> 1) & 1));
                if (!ok) break;
                tcgen05_fence_after();
                uint32_t h[KT / 2];
                float sum;
#pragma unroll 1
                for (bool raise = j == 0;; raise = true) {
                    if (raise) {                                 // the maximum first
                        float mx = -INFINITY;
#pragma unroll 1
                        for (int i = 0; i < GROUPS; ++i) {
                            uint32_t z[16];
                            tcgen05_ld_32x32b_x16(score + 16u * i, z);
                            const float4 cc = consts[i];
                            const float f = cc.x * rf;
                            tcgen05_wait_ld();
                            tcgen05_loaded(z);
#pragma unroll
                            for (int e = 0; e < 16; ++e) mx = fmaxf(mx, 16 * i + e <= upto && 16 * i + e >= from ? fmaf(__uint_as_float(z[e]), f, cc.y) : -INFINITY);
                        }
                        const float next = mx > M + kPromptSlack || M == -INFINITY ? fmaxf(mx, M) : M;
                        const float g = next == M ? 1.f : exp2_fast(M - next);
                        const float now = consts[0].w, larger = j > 0 ? now - unit : 0.f;      // (l is in units of 2^-(M + unit))
                        unit = now;
                        l *= exp2_fast(fminf((next == M ? 0.f : M - next) + larger, 126.f));
                        l = l > 0x1p126f ? 0x1p126f : l;
                        M = next;
                        if (j > 0) {                             // (behind the product of the tile before)
                            ok = warp_all(mbar_wait(smem_u32(&o_full[r]), (j - 1) & 1));
                            if (!ok) break;
                            tcgen05_fence_after();
#pragma unroll 1
                            for (int i = 0; i < D; i += 16) {
                                uint32_t z[16];
                                tcgen05_ld_32x32b_x16(out + (uint32_t)i, z);
                                tcgen05_wait_ld();
                                tcgen05_loaded(z);
#pragma unroll
                                for (int e = 0; e < 16; ++e) z[e] = __float_as_uint(__uint_as_float(z[e]) * g);
                                tcgen05_st_32x32b_x16(out + (uint32_t)i, z);
                            }
                        }
                    }
                    const float Mu = M == -INFINITY ? 0.f : M;
                    float mx = -INFINITY, now = 0.f;
                    sum = 0.f;
                    uint32_t z[2][32];
                    tcgen05_ld_32x32b_x32(score, z[0]);
                    tcgen05_ld_32x32b_x32(score + 32u, z[1]);
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        float4 c0, c1;
                        asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(c0.x), "=f"(c0.y), "=f"(c0.z), "=f"(c0.w) : "r"(smem_u32(consts + 2 * i)) : "memory");
                        asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(c1.x), "=f"(c1.y), "=f"(c1.z), "=f"(c1.w) : "r"(smem_u32(consts + 2 * i + 1)) : "memory");
                        now = c1.w;
                        const float f0 = c0.x * rf, f1 = c1.x * rf, b0 = c0.y - Mu, b1 = c1.y - Mu;
                        if (i == 0) tcgen05_wait_ld();
                        tcgen05_loaded(z[i]);
                        float x[32];
#pragma unroll
                        for (int e = 0; e < 32; ++e) x[e] = fmaf(__uint_as_float(z[i][e]), e < 16 ? f0 : f1, e < 16 ? b0 : b1);
                        if (!plain) {
#pragma unroll
                            for (int e = 0; e < 32; ++e) x[e] = 32 * i + e <= upto && 32 * i + e >= from ? x[e] : -INFINITY;
                        }
#pragma unroll
                        for (int half = 0; half < 2; ++half) {
                            float s0 = 0.f, s1 = 0.f;
                            const float inverse = half == 0 ? c0.z : c1.z;
                            const auto add16 = [&](auto as_rounded) {
#pragma unroll
                                for (int e = 16 * half; e < 16 * half + 16; e += 2) {
                                    mx = fmaxf(mx, fmaxf(x[e], x[e + 1]));
                                    const float u = exp2_fast(x[e]), v = exp2_fast(x[e + 1]);
                                    h[16 * i + e / 2] = f4_from_float2<__half>(u, v);
                                    if constexpr (decltype(as_rounded)::value) add_halves(s0, s1, h[16 * i + e / 2]);
                                    else { s0 += u; s1 += v; }
                                }
                            };
                            if (inverse >= 0.f) add16(std::true_type()); else add16(std::false_type());
                            sum = fmaf(s0 + s1, fabsf(inverse), sum);
                        }
                        asm volatile("" : "+f"(sum), "+f"(mx));          // (added up here: put off, the values would stay in registers)
                    }
                    // (once: what the maximum was taken of is rounded apart from this by less than a unit)
                    if (raise || !__any_sync(0xffffffffu, mx > kPromptSlack || (M == -INFINITY && mx != -INFINITY) || now != unit)) break;
                }
                if (!ok) break;
                l += sum;
#pragma unroll
                for (int i = 0; i < KT / 2; i += 16) tcgen05_st_32x32b_x16(score + (uint32_t)i, *reinterpret_cast<uint32_t(*)[16]>(h + i));
                tcgen05_wait_st();
                tcgen05_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_u32(&p_full[r][j & 1]));
            }
            if (ok) {
                ok = warp_all(mbar_wait(smem_u32(&all_bar[r]), 0));
                tcgen05_fence_after();
                const int e = (int)unit >> 1;
                const float f1 = __uint_as_float((uint32_t)(127 + e) << 23), f2 = l == 0.f ? 0.f : __uint_as_float((uint32_t)(127 + (int)unit - e) << 23) / l;      // 2^unit / l
                T *dst = static_cast<T *>(p.y) + (size_t)(q.row + token) * p.ldy + head_at;
#pragma unroll 1
                for (int i = 0; ok && i < D; i += 16) {
                    uint32_t z[16];
                    tcgen05_ld_32x32b_x16(out + (uint32_t)i, z);
                    tcgen05_wait_ld();
                    tcgen05_loaded(z);
                    if (real) {
                        uint32_t h[8];
#pragma unroll
                        for (int e = 0; e < 8; ++e) h[e] = f4_from_float2<T>(__uint_as_float(z[2 * e]) * f1 * f2, __uint_as_float(z[2 * e + 1]) * f1 * f2);
                        *reinterpret_cast<uint4 *>(dst + i) = make_uint4(h[0], h[1], h[2], h[3]);
                        *reinterpret_cast<uint4 *>(dst + i + 8) = make_uint4(h[4], h[5], h[6], h[7]);
                    }
                }
            }
        }
    } else if (warp < Sh::kSoft + Sh::kLoad) {
        // ---- keys and values: a warp has every fourth 16 tokens of a tile
        constexpr int MINE = GROUPS / Sh::kLoad, PIECES = D / 32;
        const int w = warp - Sh::kSoft, g = lane >> 2, t = lane & 3;
        const uint8_t *codes = c.cache + (size_t)head * 2 * D * (page_mask + 1) + lane * 16;
        const size_t page_bytes = (size_t)c.heads * 2 * D * (page_mask + 1);
        const float *scales = reinterpret_cast<const float *>(c.cache + c.scales_off) + head * 2;
        // Lane i looks up the page of group i of a tile, a tile before its codes and scales are asked for.
        int id = -1, next_id = -1;
        float key_scale = 0.f, value_scale = 0.f, top = 0.f;      // top: the largest scale of values so far
        int unit = -150;                                         // (below any scale)
        float2 to_unit = make_float2(0x1p75f, 0x1p75f);          // 2^-unit
        float small = 0.f;
        auto look = [&](int j) {
            const int token = (tile0 + j) * KT + 16 * (lane & (GROUPS - 1));
            return j < tiles && lane < GROUPS && token < hi ? cache_page(c, seq, token >> c.page_sh) : -1;
        };
        uint4 kr[MINE][PIECES], vr[MINE][PIECES];
        auto fetch = [&](int j) {
            id = next_id;
            next_id = look(j + 1);
            key_scale = value_scale = 0.f;
            if (id >= 0) {
                key_scale = ld_dependent(scales + (size_t)id * c.heads * 2);
                value_scale = ld_dependent(scales + (size_t)id * c.heads * 2 + 1);
            }
#pragma unroll
            for (int n = 0; n < MINE; ++n) {
                const int step = w + n * Sh::kLoad, at = __shfl_sync(0xffffffffu, id, step), token = (tile0 + j) * KT + 16 * step;
                const uint8_t *k = codes + (at < 0 ? 0 : at) * page_bytes + (size_t)(token & page_mask) * D, *v = k + (size_t)D * (page_mask + 1);
#pragma unroll
                for (int i = 0; i < PIECES; ++i) kr[n][i] = at >= 0 ? ld_dependent(reinterpret_cast<const uint4 *>(k + i * 512)) : make_uint4(0, 0, 0, 0);
#pragma unroll
                for (int i = 0; i < PIECES; ++i) vr[n][i] = at >= 0 ? ld_dependent(reinterpret_cast<const uint4 *>(v + i * 512)) : make_uint4(0, 0, 0, 0);
            }
        };
        next_id = look(0);
        fetch(0);
        int s = 0;
        uint32_t ph = 1;                                         // (the first turn of the rings does not wait)
        for (int j = 0; j < tiles; ++j) {
            if (j >= NS && !warp_all(mbar_wait(smem_u32(&k_empty[s]), ph))) { ok = false; break; }
            float most = lane < GROUPS && id >= 0 && value_scale == value_scale ? value_scale : 0.f;
            most = __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(most)));
            if (most > top) {
                top = most;
                const int e = (int)floorf(__log2f(top));
                if (e >= unit + kPromptMargin) {
                    unit = e;
                    to_unit = make_float2(__uint_as_float((uint32_t)(127 - (e >> 1)) << 23), __uint_as_float((uint32_t)(127 - (e - (e >> 1))) << 23));
                }
                small = top * to_unit.x * to_unit.y * kPromptSmall;
            }
            if (w == 0 && lane < GROUPS) {
                const bool none = value_scale != value_scale;    // values that are none: in the scores, whose masked ones do not count
                const float v = fmaxf(none ? 0.f : value_scale * to_unit.x * to_unit.y, kPromptLeast), sign = value_scale > 0.f && v >= small ? 1.f : -1.f;
                page_consts[j & (Sh::kConsts - 1)][lane] =
                    make_float4(id < 0 ? 0.f : none ? value_scale : key_scale, id < 0 ? -INFINITY : (float)unit + __log2f(v), id < 0 ? 0.f : sign / v, (float)unit);
            }
            uint8_t *kt = smem + Sh::kQ + s * Sh::kKv, *vt = smem + Sh::kQ + (NS + s) * Sh::kKv;
#pragma unroll
            for (int n = 0; n < MINE; ++n)
#pragma unroll
                for (int i = 0; i < PIECES; ++i) {               // piece 2 p + h: token 8 h + g, columns 64 p + 16 t ..
                    const int row = (w + n * Sh::kLoad) * 16 + (i & 1) * 8 + g;
                    const uint4 u = kr[n][i];
                    uint32_t h[8];
                    bytes_to_half(u.x, h[0], h[1]);
                    bytes_to_half(u.y, h[2], h[3]);
                    bytes_to_half(u.z, h[4], h[5]);
                    bytes_to_half(u.w, h[6], h[7]);
                    uint8_t *at = kt + (i >> 1) * (KT * 128) + row * 128;
                    *reinterpret_cast<uint4 *>(at + (((2 * t) ^ g) << 4)) = make_uint4(h[0], h[1], h[2], h[3]);
                    *reinterpret_cast<uint4 *>(at + (((2 * t + 1) ^ g) << 4)) = make_uint4(h[4], h[5], h[6], h[7]);
                }
            fence_async_shared();
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&k_full[s]));
            if (j >= NS && !warp_all(mbar_wait(smem_u32(&v_empty[s]), ph))) { ok = false; break; }
#pragma unroll
            for (int n = 0; n < MINE; ++n) {
                const int step = w + n * Sh::kLoad;
                uint8_t *atom = vt + (step >> 2) * (D * 128) + g * 128 + 4 * t;
                const uint32_t lo = ((2 * (step & 3)) ^ g) << 4, hi2 = ((2 * (step & 3) + 1) ^ g) << 4;
#pragma unroll
                for (int i = 0; i < PIECES; ++i)                 // bytes 4 e ..: column 8 (4 i + e) + g, tokens 2t, 2t + 1, 2t + 8, 2t + 9
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        uint32_t h0, h1;
                        bytes_to_half(e == 0 ? vr[n][i].x : e == 1 ? vr[n][i].y : e == 2 ? vr[n][i].z : vr[n][i].w, h0, h1);
                        *reinterpret_cast<uint32_t *>(atom + (4 * i + e) * 1024 + lo) = h0;
                        *reinterpret_cast<uint32_t *>(atom + (4 * i + e) * 1024 + hi2) = h1;
                    }
            }
            fence_async_shared();
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&v_full[s]));
            if (j + 1 < tiles) fetch(j + 1);
            if (++s == NS) { s = 0; ph ^= 1u; }
        }
    } else {
        // ---- MMAs, a warp for each tile of rows (one for both spent its time between waits: 200 us).  Scores of tile j go to buffer j & 1, behind the
        // product that read the probabilities of tile j - 2 there: the tensor cores work in the order of issue.
        // (Addresses and descriptors are worked out by the whole warp, outside of what one lane issues, so that they sit in uniform registers.)
        const int r = warp - Sh::kSoft - Sh::kLoad;
        const bool lead = elect_one(), twice = active < RT;      // (the word of the tile of rows that is not there)
        constexpr uint32_t score_desc = 1u << 4 | (uint32_t)(KT >> 3) << 17 | (128u >> 4) << 24, out_desc = 1u << 4 | (uint32_t)(D >> 3) << 17 | (128u >> 4) << 24;
        const uint64_t qd = make_kmajor_sw128_desc(qs) + (uint32_t)r * (D / 64) * (16384 / 16), kd = make_kmajor_sw128_desc(ks), vd = make_kmajor_sw128_desc(vs);
        const uint32_t score = tmem + Sh::kScore + r * 2 * KT, out = tmem + Sh::kOut + r * D;
        const uint32_t sf = smem_u32(&s_full[r][0]), pf = smem_u32(&p_full[r][0]), of = smem_u32(&o_full[r]);
        int sk = 0, sv = 0;                                      // stages of the next tile of keys, of values
        uint32_t pk = 0, pv = 0;
        auto scores = [&](int j) {                               // keys of tile j
            ok = warp_all(mbar_wait(smem_u32(&k_full[sk]), pk));
            if (!ok) return;
            tcgen05_fence_after();
            const uint64_t kj = kd + (uint32_t)sk * (Sh::kKv / 16);
            const uint32_t to = score + (j & 1) * KT, full = sf + (j & 1) * 8, empty = smem_u32(&k_empty[sk]);
            if (lead) {
#pragma unroll
                for (uint32_t i = 0; i < D / 16; ++i)
                    tcgen05_mma_f16(to, qd + ((i >> 2) * 16384 + (i & 3) * 32) / 16, kj + ((i >> 2) * (KT * 128) + (i & 3) * 32) / 16, score_desc, i != 0);
                tcgen05_commit(full);
                tcgen05_commit(empty);
                if (twice) tcgen05_commit(empty);
            }
            __syncwarp();
            if (++sk == NS) { sk = 0; pk ^= 1u; }
        };
        if (r < active) {
            ok = warp_all(mbar_wait(smem_u32(&q_bar), 0));
            tcgen05_fence_after();
            for (int j = 0; ok && j < 2 && j < tiles; ++j) scores(j);
            for (int j = 0; ok && j < tiles; ++j) {
                ok = warp_all(mbar_wait(smem_u32(&v_full[sv]), pv) && mbar_wait(pf + (j & 1) * 8, (j >> 1) & 1));
                if (!ok) break;
                tcgen05_fence_after();
                const uint64_t vj = vd + (uint32_t)sv * (Sh::kKv / 16);
                const uint32_t from = score + (j & 1) * KT, empty = smem_u32(&v_empty[sv]);
                if (lead) {
#pragma unroll
                    for (uint32_t i = 0; i < KT / 16; ++i) tcgen05_mma_f16_ts(out, from + i * 8, vj + i * 2, out_desc, i == 0 ? (uint32_t)j : 1u);
                    tcgen05_commit(empty);
                    if (twice) tcgen05_commit(empty);
                    tcgen05_commit(of);
                    if (j + 1 == tiles) tcgen05_commit(smem_u32(&all_bar[r]));
                }
                __syncwarp();
                if (j + 2 < tiles) scores(j + 2);
                if (++sv == NS) { sv = 0; pv ^= 1u; }
            }
        }
    }
    if (!ok) atomicCAS(c.status, 0u, (uint32_t)TMAN_ERR_TIMEOUT);
    tcgen05_fence_before();
    __syncthreads();
    if (warp == Sh::kSoft + Sh::kLoad) {
        tcgen05_fence_after();
        tcgen05_dealloc(tmem, 512);
    }
}

template <typename T, int D> tman_status launch_prompt(const PromptParams &p, cudaStream_t s)
{
    using Sh = PromptShape<D>;
    auto kern = attend_prompt_kernel<T, D>;
    static std::atomic<bool> raised[kMaxDevices];
    int dev = 0;
    if (!device_info(&dev)) return TMAN_ERR_CUDA;
    // blocks of rows: a sequence of n rows has at most n / kRows + 1, and n / least
    const long long rows = (long long)p.c.T * p.group;
    const long long most = rows / Sh::kRows + (rows / p.least < p.c.S ? rows / p.least : p.c.S);
    if (most * p.c.heads > INT32_MAX) return TMAN_ERR_SHAPE;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(most * p.c.heads));
    cfg.blockDim = dim3(Sh::kThreads);
    cfg.dynamicSmemBytes = Sh::kSmem;
    cfg.stream = s;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return launch_with_smem(kern, Sh::kSmem, dev, raised, [&] { return cudaLaunchKernelEx(&cfg, kern, p); });
}

}  // namespace
}  // namespace tman
