// Attention over the 8-bit cache: for every new token and query head softmax(scale q . k) v over the keys up to the token, or the last `window` of
// them, in one pass with a running maximum and sum.
//
// What bounds few new tokens is reading the cache once.  The rows that share a key head (new tokens x query heads of it) are the 16 rows of an MMA
// tile; keys are its columns.  A warp takes 16 keys and values at a time, in the cache's own order (cache_i8.cuh): a ring of asynchronous copies, each
// lane's pieces its own, so that no barrier is needed; bytes become fp16 by one permutation and one subtraction for two, exactly.
// The work, in steps of 16 tokens over all sequences, row tiles and heads, is dealt to the CTAs in equal runs; within a CTA the warps take steps in
// turn.  Warps join their sums in shared memory.  A run that ends inside of a head's tokens leaves them in the workspace, and the last of the CTAs
// that share the head adds them up, in their order.
// Scores are products of 16-bit queries and codes, 32-bit sums, times the key page's scale.  Probabilities meet the values as fp16 numbers
// p x (scale of the value page), relative to the largest of those so far: each off by 2^-12 of itself, or 2^-25 of that largest one.  Sums and maxima are
// held in 32 bits.  A bf16 query row is brought into fp16 by a power of two, exact down to 2^-38 of its largest value.
// Measured: 32 sequences of 9830 to 32768 tokens, 28 heads on 4 of 128, 145 us in a graph (floor 108): 4.9 TB/s over the call, some 8 us of it start and end; one of
// 500 tokens 9.1, the chain from lengths to pages to keys to sums.
#include "attend_prompt.cuh"

namespace tman {
namespace {

// Rows of a sequence from which the kernel for prompts takes it.  Here every 16 rows read the keys again, and all of that is spread over all CTAs; there up to 256 rows
// read them once, but one CTA walks over all of a key head's.  32 heads on 8 of 128, us in a graph, here / there:
//   rows      8 x 512     8 x 4096    8 x 32768   1 x 512     1 x 4096    1 x 32768 tokens
//   32        12 / 17     42 / 94     207 / 682   11 / 17     16 / 74     39 / 665
//   64        20 / 17     71 / 94     392 / 682   11 / 17     22 / 74     65 / 666
//   128       37 / 18     128 / 95    761 / 684   14 / 18     29 / 75     113 / 666
//   256       74 / 24     245 / 107   1539 / 749  17 / 24     46 / 91     205 / 734
//   512       162 / 25    497 / 104   3440 / 732  34 / 24     83 / 92     394 / 719
// The line is right for several sequences of some hundred tokens; where there are fewer (sequences x key heads) than multiprocessors it comes too soon.
constexpr int kPromptRows = 64;
constexpr int kItemCost = 48;            // steps that beginning and ending a head are worth
constexpr int kShortSteps = 96;          // heads of so few steps are not cut
constexpr uint32_t kNoneYet = 0x7FA5A5A5u;      // what tman_workspace_init writes: a counter at rest

template <int D> struct AttendShape {
    static constexpr int kWarps = D <= 128 ? 12 : 8, kThreads = 32 * kWarps, kStages = D == 64 ? 6 : D == 128 ? 4 : 3;
    static constexpr int kStep = 32 * D, kRing = kStages * kStep, kQ = 32 * D, kSmem = kWarps * kRing + kQ;
    static constexpr int kSumRow = D + 8;     // floats from a row of a warp's sums to the next: rows start at different banks
    static_assert(kRing >= 16 * kSumRow * 4, "a warp's sums fit its ring");
};

struct AttendParams {
    CacheSeqs c;
    const void *q;
    void *y;
    float *parts;
    uint32_t *counters;
    int ldq, ldy, group, window, least;  // group: query heads of a key head; sequences of `least` rows (tokens x group) and more are done elsewhere
    uint32_t group_mul;                  // 2^32 / group, rounded up; 0: a group of one
    float scale;
};

__device__ __forceinline__ void mma_f16(float (&c)[4], const uint4 &a, uint32_t b0, uint32_t b1)
{
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a.x), "r"(a.y), "r"(a.z), "r"(a.w), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void copy16(uint32_t dst, const void *src)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void copy_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// Tokens of the first n rows (n and the group are below 2^16).
__device__ __forceinline__ int token_of(const AttendParams &p, int n) { return p.group_mul ? (int)__umulhi((uint32_t)n, p.group_mul) : n; }

// The keys that a tile of rows sees: tokens [lo, hi), and steps of 16 of them, one at least.
struct TileKeys { int first, lo, hi, step0, steps; };            // first: position of the tile's first token
__device__ __forceinline__ TileKeys tile_keys(const AttendParams &p, const CacheSeq &q, int tile)
{
    TileKeys k;
    const int rows = q.rows * p.group, i0 = token_of(p, tile * kAttendRows), i1 = token_of(p, min(tile * kAttendRows + kAttendRows - 1, rows - 1));
    k.first = q.len - q.rows + i0;
    k.hi = max(q.len - q.rows + i1 + 1, 0);
    k.lo = window_from(k.first, p.window);
    k.step0 = k.lo >> 4;
    k.steps = max(((k.hi + 15) >> 4) - k.step0, 1);
    return k;
}
__device__ __forceinline__ int tiles_of(const AttendParams &p, const CacheSeq &q)
{
    const int rows = q.rows * p.group;
    return rows >= p.least ? 0 : (rows + kAttendRows - 1) / kAttendRows;
}

template <typename T, int D>
__global__ void __launch_bounds__(AttendShape<D>::kThreads, 1) attend_kernel(const __grid_constant__ AttendParams p)
{
    using Sh = AttendShape<D>;
    constexpr int W = Sh::kWarps, NT = D / 8, PIECES = D / 32;      // tiles of columns of the output, pieces of a lane
    extern __shared__ __align__(128) uint8_t smem[];
    __shared__ int before[Sh::kThreads + 1];                     // steps of the sequences in front of thread t's
    __shared__ CacheSeq known[Sh::kThreads];                     // the sequence of thread t, if each has one
    __shared__ float row_factor[16], warp_max[W][16], warp_lmax[W][16], warp_sum[W][16], share_of[W][16], row_max[16], row_lmax[16], row_sum[16];
    __shared__ uint32_t last_flag;
    const CacheSeqs &c = p.c;
    const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31, g = lane >> 2, t = lane & 3, page_mask = (1 << c.page_sh) - 1;
    uint4 *qs = reinterpret_cast<uint4 *>(smem + W * Sh::kRing);
    const uint32_t ring = smem_u32(smem) + warp * Sh::kRing + lane * 16;
    const uint8_t *ring_at = smem + warp * Sh::kRing + lane * 16;
    grid_wait();
    grid_launch_next();

    const int per = (c.S + Sh::kThreads - 1) / Sh::kThreads;
    auto units_of = [&](const CacheSeq &q) {
        int n = 0;
#pragma unroll 1
        for (int i = 0; i < tiles_of(p, q); ++i) n += tile_keys(p, q, i).steps + kItemCost;
        return n * c.heads;
    };
    {
        int mine = 0;
#pragma unroll 1
        for (int s = min(tid * per, c.S); s < min(tid * per + per, c.S); ++s) {
            const CacheSeq q = cache_seq(c, s);
            if (per == 1) known[tid] = q;
            mine += units_of(q);
        }
        int upto = mine;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const int o = __shfl_up_sync(0xffffffffu, upto, d);
            if (lane >= d) upto += o;
        }
        if (lane == 31) warp_sum[0][warp] = __int_as_float(upto);
        __syncthreads();
#pragma unroll
        for (int w = 0; w < W; ++w) upto += w < warp ? __float_as_int(warp_sum[0][w]) : 0;
        before[tid + 1] = upto;
        if (tid == 0) before[0] = 0;
        __syncthreads();
    }
    const int total = before[Sh::kThreads];                      // (below 2^31: checked by the host)
    int run = total / (int)gridDim.x + (total % (int)gridDim.x != 0);
    run = max((run + W - 1) / W, 1) * W;

    // Sequence, head and tile of a unit, by all threads alike.
    struct Item { int s, head, tile, at; CacheSeq q; TileKeys k; };      // at: unit of its first step
    auto item_of = [&](int u) {
        int lo = 0, hi = min(Sh::kThreads, c.S);
#pragma unroll 1
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (before[mid] <= u) lo = mid; else hi = mid;
        }
        Item it;
        it.at = before[lo];
        it.s = lo * per;
        if (per == 1) it.q = known[lo];
        else {
#pragma unroll 1
            for (;; ++it.s) {
                it.q = cache_seq(c, it.s);
                const int n = units_of(it.q);
                if (u < it.at + n) break;
                it.at += n;
            }
        }
        const int tiles = tiles_of(p, it.q);
        it.tile = 0;
        it.k = tile_keys(p, it.q, 0);
        int one = it.k.steps + kItemCost;
#pragma unroll 1
        for (int i = 1; i < tiles; ++i) one += tile_keys(p, it.q, i).steps + kItemCost;
        it.head = (u - it.at) / one;
        it.at += it.head * one;
#pragma unroll 1
        while (u >= it.at + kItemCost + it.k.steps) {
            it.at += kItemCost + it.k.steps;
            it.k = tile_keys(p, it.q, ++it.tile);
        }
        it.at += kItemCost;
        return it;
    };
    // The first turn finds where the runs of this CTA and of the next begin (lanes 0 and 1): a short head belongs to the CTA that its first step
    // falls to.
    int u = 0, end = 0;
#pragma unroll 1
    for (int turn = 0;; ++turn) {
        const long long from = ((long long)blockIdx.x + (lane & 1)) * run;
        const int at_u = turn > 0 ? u : from < total ? (int)from : total;
        Item it = {};
        if (at_u < total) it = item_of(at_u);
        if (turn == 0) {
            const int begin = at_u < total && at_u > it.at && it.k.steps <= kShortSteps ? it.at + it.k.steps : at_u;
            u = __shfl_sync(0xffffffffu, begin, 0);
            end = __shfl_sync(0xffffffffu, begin, 1);
            if (u >= end) break;
            continue;
        }
        const int s0 = max(u - it.at, 0), s1 = min(it.k.steps, end - it.at);       // steps of this run
        const bool whole = s0 == 0 && s1 == it.k.steps;
        const int rows = min(kAttendRows, it.q.rows * p.group - it.tile * kAttendRows);
        u = it.at + it.k.steps;
        if (s1 <= s0) break;                                     // (the run ends in front of the head's first step)

        // ---- the warp's first copies
        const uint8_t *codes = c.cache + (size_t)it.head * 2 * D * (page_mask + 1);
        const size_t page_bytes = (size_t)c.heads * 2 * D * (page_mask + 1);
        const float *scales = reinterpret_cast<const float *>(c.cache + c.scales_off) + it.head * 2;
        // Lane i looks up page and scales of the warp's step 32 b + i, for two b at a time.
        struct Look { int id; float ks, vs; };
        auto look = [&](int b) {
            Look l = {-1, -1.f, 0.f};                            // (scale -1: masked)
            const int step = s0 + warp + (32 * b + lane) * W, token = (it.k.step0 + step) * 16;
            if (step < s1 && token < it.k.hi) {
                l.id = cache_page(c, it.s, token >> c.page_sh);
                if (l.id >= 0) {
                    const float *f = scales + (size_t)l.id * c.heads * 2;
                    l.ks = ld_dependent(f);
                    l.vs = ld_dependent(f + 1);
                    if (l.vs != l.vs) {                          // values that are none: in the scores, whose masked ones do not count
                        l.ks = l.vs;
                        l.vs = 1.f;
                    }
                }
            }
            return l;
        };
        int looked = 0;                                          // b of `now`
        Look now = look(0), next = {-1, -1.f, 0.f};
        const int mine = s1 - s0 > warp ? (s1 - s0 - warp + W - 1) / W : 0;      // steps of this warp
        auto fetch = [&](int i, int slot) {                      // the warp's step i into a slot of the ring
            if (i < mine) {
                const int id = __shfl_sync(0xffffffffu, (i >> 5) == looked ? now.id : next.id, i & 31);
                if (id >= 0) {
                    const int token = (it.k.step0 + s0 + warp + i * W) * 16;
                    const uint8_t *k = codes + id * page_bytes + (size_t)(token & page_mask) * D + lane * 16, *v = k + (size_t)D * (page_mask + 1);
                    const uint32_t dst = ring + slot * Sh::kStep;
#pragma unroll
                    for (int j = 0; j < PIECES; ++j) copy16(dst + j * 512, k + j * 512);
#pragma unroll
                    for (int j = 0; j < PIECES; ++j) copy16(dst + 16 * D + j * 512, v + j * 512);
                }
            }
            copy_commit();
        };
        // Queries on their way: rows warp and warp + W of the tile.
        constexpr int QR = (16 + W - 1) / W, QW = (D / 4 + 31) / 32;
        uint2 raw[QR][QW];
#pragma unroll
        for (int a = 0; a < QR; ++a) {
            const int r = warp + a * W, rho = it.tile * kAttendRows + min(r, rows - 1), i = token_of(p, rho);
            const T *src = static_cast<const T *>(p.q) + (size_t)(it.q.row + i) * p.ldq + (size_t)(it.head * p.group + rho - i * p.group) * D;
#pragma unroll
            for (int b = 0; b < QW; ++b) {
                raw[a][b] = make_uint2(0, 0);
                if (r < rows && lane + 32 * b < D / 4)
                    asm volatile("ld.global.v2.u32 {%0, %1}, [%2];" : "=r"(raw[a][b].x), "=r"(raw[a][b].y) : "l"(reinterpret_cast<const uint2 *>(src) + lane + 32 * b) : "memory");
            }
        }
#pragma unroll 1
        for (int i = 0; i < Sh::kStages - 1; ++i) fetch(i, i);

        // ---- queries as A operands, zero behind the last row: columns 64 i + 16 t + 4 j of row r in step 4 i + j of k, lane 4 (r % 8) + t, words r / 8 and r / 8 + 2
#pragma unroll
        for (int a = 0; a < QR; ++a) {
            const int r = warp + a * W;
            if (r >= 16) break;
            float f = 1.f;
            if constexpr (!std::is_same<T, __half>::value) {
                uint32_t top = 0;
#pragma unroll
                for (int b = 0; b < QW; ++b) top = i8_larger(top, i8_larger(i8_magnitudes(raw[a][b].x), i8_magnitudes(raw[a][b].y)));
                top = __reduce_max_sync(0xffffffffu, max(top & 0xFFFFu, top >> 16));
                // largest value in [2^e, 2^(e + 1)), e = top / 128 - 127
                f = top == 0 || top >= i8_infinity<T>() ? 1.f : __uint_as_float((uint32_t)(127 + min(141 - (int)(top >> 7), 100)) << 23);
            }
            if (lane == 0) row_factor[r] = p.scale * kLog2e / f;
#pragma unroll
            for (int b = 0; b < QW; ++b) {
                const int i = lane + 32 * b;
                if (i >= D / 4) break;
                uint2 h = raw[a][b];
                if constexpr (!std::is_same<T, __half>::value) {
                    const float2 x = f4_to_float2<T>(h.x), y = f4_to_float2<T>(h.y);
                    h = make_uint2(f4_from_float2<__half>(x.x * f, x.y * f), f4_from_float2<__half>(y.x * f, y.y * f));
                }
                uint32_t *at = reinterpret_cast<uint32_t *>(qs + ((i >> 4) * 4 + (i & 3)) * 32 + (r & 7) * 4 + ((i >> 2) & 3)) + (r >> 3);
                at[0] = h.x;
                at[2] = h.y;
            }
        }
        __syncthreads();

        const float rf0 = row_factor[g], rf1 = row_factor[g + 8];
        auto limit_of = [&](int r) { return it.q.len - it.q.rows + token_of(p, it.tile * kAttendRows + min(r, rows - 1)); };
        const int lim0 = limit_of(g), lim1 = limit_of(g + 8);
        const int low0 = window_from(lim0, p.window), low1 = window_from(lim1, p.window);
        const int all_from = p.window > 0 ? it.k.hi - p.window : 0;      // tokens [all_from, first] are seen by every row
        float o[NT][4];
#pragma unroll
        for (int i = 0; i < NT; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) o[i][e] = 0.f;
        float m0 = -INFINITY, m1 = -INFINITY, lm0 = -INFINITY, lm1 = -INFINITY, l0 = 0.f, l1 = 0.f;

        auto take = [&](int step, int slot, float2 sc) {
            const uint8_t *at = ring_at + slot * Sh::kStep;
            const int token = (it.k.step0 + step) * 16;
            float z[2][4];
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int e = 0; e < 4; ++e) z[h][e] = 0.f;
#pragma unroll
            for (int i = 0; i < D / 64; ++i)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const uint4 w = *reinterpret_cast<const uint4 *>(at + (2 * i + h) * 512);
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        uint32_t b0, b1;
                        bytes_to_half(j == 0 ? w.x : j == 1 ? w.y : j == 2 ? w.z : w.w, b0, b1);
                        mma_f16(z[h], qs[(4 * i + j) * 32 + lane], b0, b1);
                    }
                }
            const float f0 = sc.x * rf0, f1 = sc.x * rf1, lv = __log2f(sc.y);
            const bool plain = token + 15 <= it.k.first && token >= all_from && sc.x != -1.f;
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int key = token + 8 * h + 2 * t + (e & 1);
                    z[h][e] *= e < 2 ? f0 : f1;
                    if (!plain && !(key <= (e < 2 ? lim0 : lim1) && key >= (e < 2 ? low0 : low1) && sc.x != -1.f)) z[h][e] = -INFINITY;
                }
            // sums of probabilities, of this lane's columns and relative to their own maximum
            const float a0 = fmaxf(fmaxf(z[0][0], z[0][1]), fmaxf(z[1][0], z[1][1])), a1 = fmaxf(fmaxf(z[0][2], z[0][3]), fmaxf(z[1][2], z[1][3]));
            const float n0 = fmaxf(lm0, a0), n1 = fmaxf(lm1, a1), u0 = n0 == -INFINITY ? 0.f : n0, u1 = n1 == -INFINITY ? 0.f : n1;
            l0 = l0 * exp2_fast(lm0 - u0) + (exp2_fast(z[0][0] - u0) + exp2_fast(z[0][1] - u0)) + (exp2_fast(z[1][0] - u0) + exp2_fast(z[1][1] - u0));
            l1 = l1 * exp2_fast(lm1 - u1) + (exp2_fast(z[0][2] - u1) + exp2_fast(z[0][3] - u1)) + (exp2_fast(z[1][2] - u1) + exp2_fast(z[1][3] - u1));
            lm0 = n0;
            lm1 = n1;
            // p x scale of the values, relative to the largest of the row
            float x0 = a0 + lv, x1 = a1 + lv;
            x0 = fmaxf(x0, __shfl_xor_sync(0xffffffffu, x0, 1));
            x1 = fmaxf(x1, __shfl_xor_sync(0xffffffffu, x1, 1));
            x0 = fmaxf(m0, fmaxf(x0, __shfl_xor_sync(0xffffffffu, x0, 2)));
            x1 = fmaxf(m1, fmaxf(x1, __shfl_xor_sync(0xffffffffu, x1, 2)));
            if (__any_sync(0xffffffffu, x0 != m0 || x1 != m1)) {
                const float r0 = x0 == m0 ? 1.f : exp2_fast(m0 - x0), r1 = x1 == m1 ? 1.f : exp2_fast(m1 - x1);
                m0 = x0;
                m1 = x1;
#pragma unroll
                for (int i = 0; i < NT; ++i) {
                    o[i][0] *= r0;
                    o[i][1] *= r0;
                    o[i][2] *= r1;
                    o[i][3] *= r1;
                }
            }
            const float v0 = lv - (m0 == -INFINITY ? 0.f : m0), v1 = lv - (m1 == -INFINITY ? 0.f : m1);
            uint4 a;
            a.x = f4_from_float2<__half>(exp2_fast(z[0][0] + v0), exp2_fast(z[0][1] + v0));
            a.y = f4_from_float2<__half>(exp2_fast(z[0][2] + v1), exp2_fast(z[0][3] + v1));
            a.z = f4_from_float2<__half>(exp2_fast(z[1][0] + v0), exp2_fast(z[1][1] + v0));
            a.w = f4_from_float2<__half>(exp2_fast(z[1][2] + v1), exp2_fast(z[1][3] + v1));
#pragma unroll
            for (int i = 0; i < PIECES; ++i) {
                const uint4 w = *reinterpret_cast<const uint4 *>(at + 16 * D + i * 512);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    uint32_t b0, b1;
                    bytes_to_half(j == 0 ? w.x : j == 1 ? w.y : j == 2 ? w.z : w.w, b0, b1);
                    mma_f16(o[4 * i + j], a, b0, b1);
                }
            }
        };
        for (int i = 0, slot = 0; i < mine; ++i) {
            if ((i & 31) == 0) next = look((i >> 5) + 1);
            fetch(i + Sh::kStages - 1, slot == 0 ? Sh::kStages - 1 : slot - 1);
            copy_wait<Sh::kStages - 1>();
            take(s0 + warp + i * W, slot, make_float2(__shfl_sync(0xffffffffu, now.ks, i & 31), __shfl_sync(0xffffffffu, now.vs, i & 31)));
            if (++slot == Sh::kStages) slot = 0;
            if ((i & 31) == 31) {
                now = next;
                ++looked;
            }
        }
        copy_wait<0>();

        // ---- the warps' sums; a row's probabilities are spread over four lanes
#pragma unroll
        for (int d = 1; d < 4; d <<= 1) {
            const float b0 = __shfl_xor_sync(0xffffffffu, lm0, d), b1 = __shfl_xor_sync(0xffffffffu, lm1, d);
            const float k0 = __shfl_xor_sync(0xffffffffu, l0, d), k1 = __shfl_xor_sync(0xffffffffu, l1, d);
            const float n0 = fmaxf(lm0, b0), n1 = fmaxf(lm1, b1);
            l0 = n0 == -INFINITY ? l0 + k0 : l0 * exp2_fast(lm0 - n0) + k0 * exp2_fast(b0 - n0);
            l1 = n1 == -INFINITY ? l1 + k1 : l1 * exp2_fast(lm1 - n1) + k1 * exp2_fast(b1 - n1);
            lm0 = n0;
            lm1 = n1;
        }
        if (t == 0) {
            warp_max[warp][g] = m0;
            warp_max[warp][g + 8] = m1;
            warp_lmax[warp][g] = lm0;
            warp_lmax[warp][g + 8] = lm1;
            warp_sum[warp][g] = l0;
            warp_sum[warp][g + 8] = l1;
        }
        float *os = reinterpret_cast<float *>(smem + warp * Sh::kRing);
#pragma unroll
        for (int i = 0; i < NT; ++i) {
            *reinterpret_cast<float2 *>(os + g * Sh::kSumRow + 8 * i + 2 * t) = make_float2(o[i][0], o[i][1]);
            *reinterpret_cast<float2 *>(os + (g + 8) * Sh::kSumRow + 8 * i + 2 * t) = make_float2(o[i][2], o[i][3]);
        }
        __syncthreads();
        const int first_cta = it.at / run, cells = rows * (D / 4);
        if (tid < W * 16) {
            const int w = tid >> 4, r = tid & 15;
            float m = -INFINITY, lm = -INFINITY, l = 0.f;
#pragma unroll
            for (int i = 0; i < W; ++i) {
                m = fmaxf(m, warp_max[i][r]);
                lm = fmaxf(lm, warp_lmax[i][r]);
            }
            share_of[w][r] = exp2_fast(warp_max[w][r] - (m == -INFINITY ? 0.f : m));
            if (w == 0) {
                const float ul = lm == -INFINITY ? 0.f : lm;
#pragma unroll
                for (int i = 0; i < W; ++i) l += warp_sum[i][r] * exp2_fast(warp_lmax[i][r] - ul);
                row_max[r] = m;
                row_lmax[r] = lm;
                row_sum[r] = l;
            }
        }
        __syncthreads();
        // y of four columns from their sums, relative to row_max, and the row's probabilities, relative to row_lmax
        auto store = [&](int r, int col, float4 v) {
            const int rho = it.tile * kAttendRows + r, i = token_of(p, rho);
            const float m = row_max[r], lm = row_lmax[r], l = row_sum[r];
            // (half of the exponent at a time: values may be so small that all of it is below the least number)
            const float f1 = exp2_fast(0.5f * ((m == -INFINITY ? 0.f : m) - (lm == -INFINITY ? 0.f : lm))), f2 = l == 0.f ? 0.f : f1 / l;
            v = make_float4(v.x * f1, v.y * f1, v.z * f1, v.w * f1);
            T *at = static_cast<T *>(p.y) + (size_t)(it.q.row + i) * p.ldy + (size_t)(it.head * p.group + rho - i * p.group) * D + col;
            *reinterpret_cast<uint2 *>(at) = make_uint2(f4_from_float2<T>(v.x * f2, v.y * f2), f4_from_float2<T>(v.z * f2, v.w * f2));
        };
        float *part = p.parts + ((size_t)blockIdx.x * 2 + (s0 == 0 ? 1 : 0)) * (kAttendRows * (D + 4));
#pragma unroll 1
        for (int i = tid; i < cells; i += Sh::kThreads) {
            const int r = i / (D / 4);
            float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int w = 0; w < W; ++w) {
                const float4 x = *reinterpret_cast<const float4 *>(smem + w * Sh::kRing + (r * Sh::kSumRow + i % (D / 4) * 4) * 4);
                const float f = share_of[w][r];
                v = make_float4(fmaf(x.x, f, v.x), fmaf(x.y, f, v.y), fmaf(x.z, f, v.z), fmaf(x.w, f, v.w));
            }
            if (whole) store(r, i % (D / 4) * 4, v);
            else __stcg(reinterpret_cast<float4 *>(part) + i, v);
        }
        if (!whole) {
            if (tid < rows) {
                __stcg(part + 16 * D + tid, row_max[tid]);
                __stcg(part + 16 * D + 16 + tid, row_lmax[tid]);
                __stcg(part + 16 * D + 32 + tid, row_sum[tid]);
            }
            const int pieces = (it.at + it.k.steps - 1) / run - first_cta + 1;
            __threadfence();
            __syncthreads();
            if (tid == 0) {
                const uint32_t was = atomicAdd(p.counters + first_cta, 1u) - kNoneYet;
                last_flag = was == (uint32_t)pieces - 1u;
                if (last_flag) atomicExch(p.counters + first_cta, kNoneYet);
                __threadfence();
            }
            __syncthreads();
            if (last_flag) {
                // ---- all parts of the head, in their order: first what each counts for, then the sums
                auto part_of = [&](int i) { return p.parts + ((size_t)(first_cta + i) * 2 + (i == 0 ? 1 : 0)) * (kAttendRows * (D + 4)); };
                float *pm = reinterpret_cast<float *>(smem), *plm = pm + kAttendCtas * 16, *pl = plm + kAttendCtas * 16;
                float4 *sums = reinterpret_cast<float4 *>(pl + kAttendCtas * 16);
                for (int i = tid; i < pieces * 16; i += Sh::kThreads) {
                    const int k = i >> 4, r = i & 15;
                    if (r < rows) {
                        const float *at = part_of(k) + 16 * D + r;
                        pm[i] = __ldcg(at);
                        plm[i] = __ldcg(at + 16);
                        pl[i] = __ldcg(at + 32);
                    }
                }
                __syncthreads();
                for (int r = warp; r < rows; r += W) {
                    float m = -INFINITY, lm = -INFINITY, l = 0.f;
                    for (int k = lane; k < pieces; k += 32) {
                        m = fmaxf(m, pm[k * 16 + r]);
                        lm = fmaxf(lm, plm[k * 16 + r]);
                    }
#pragma unroll
                    for (int d = 16; d > 0; d >>= 1) {
                        m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, d));
                        lm = fmaxf(lm, __shfl_xor_sync(0xffffffffu, lm, d));
                    }
                    const float um = m == -INFINITY ? 0.f : m, ul = lm == -INFINITY ? 0.f : lm;
                    for (int k = lane; k < pieces; k += 32) {
                        l += pl[k * 16 + r] * exp2_fast(plm[k * 16 + r] - ul);
                        pm[k * 16 + r] = exp2_fast(pm[k * 16 + r] - um);
                    }
#pragma unroll
                    for (int d = 16; d > 0; d >>= 1) l += __shfl_xor_sync(0xffffffffu, l, d);
                    if (lane == 0) {
                        row_max[r] = m;
                        row_lmax[r] = lm;
                        row_sum[r] = l;
                    }
                }
                __syncthreads();
                // (few cells: several threads share the parts of one)
                const int teams = cells * 4 <= Sh::kThreads ? 4 : cells * 2 <= Sh::kThreads ? 2 : 1;
#pragma unroll 1
                for (int i = tid; i < cells * teams; i += Sh::kThreads) {
                    const int cell = i % cells, team = i / cells, r = cell / (D / 4);
                    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 8
                    for (int k = team; k < pieces; k += teams) {
                        const float4 x = __ldcg(reinterpret_cast<const float4 *>(part_of(k)) + cell);
                        const float f = pm[k * 16 + r];
                        v = make_float4(fmaf(x.x, f, v.x), fmaf(x.y, f, v.y), fmaf(x.z, f, v.z), fmaf(x.w, f, v.w));
                    }
                    if (teams == 1) store(r, cell % (D / 4) * 4, v);
                    else sums[i] = v;
                }
                if (teams > 1) {
                    __syncthreads();
                    if (tid < cells) {
                        float4 v = sums[tid];
                        for (int k = 1; k < teams; ++k) {
                            const float4 x = sums[k * cells + tid];
                            v = make_float4(v.x + x.x, v.y + x.y, v.z + x.z, v.w + x.w);
                        }
                        store(tid / (D / 4), tid % (D / 4) * 4, v);
                    }
                }
            }
        }
        __syncthreads();
        if (u >= end) break;
    }
}

template <typename T, int D> tman_status launch(AttendParams p, cudaStream_t s)
{
    auto kern = attend_kernel<T, D>;
    static std::atomic<bool> raised[kMaxDevices];
    int dev = 0;
    const DeviceInfo *info = device_info(&dev);
    if (!info) return TMAN_ERR_CUDA;
    const int sms = info->sms.load(std::memory_order_relaxed);
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(sms < kAttendCtas ? sms : kAttendCtas));
    cfg.blockDim = dim3(AttendShape<D>::kThreads);
    cfg.dynamicSmemBytes = AttendShape<D>::kSmem;
    cfg.stream = s;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return launch_with_smem(kern, AttendShape<D>::kSmem, dev, raised, [&] { return cudaLaunchKernelEx(&cfg, kern, p); });
}

template <typename T, int D> tman_status launch_both(AttendParams p, cudaStream_t s)
{
    // Sequences of many rows go to the kernel for prompts, where the call has room for one; which do is known on the device only.
    if (p.least == kPromptRows) {
        const PromptParams q = {p.c, p.q, p.y, p.ldq, p.ldy, p.group, p.window, kPromptRows, p.scale};
        const tman_status st = launch_prompt<T, D>(q, s);
        if (st != TMAN_OK) return st;
    }
    return launch<T, D>(p, s);
}

template <typename T> tman_status launch_width(const AttendParams &p, cudaStream_t s)
{
    switch (p.c.width) {
        case 64: return launch_both<T, 64>(p, s);
        case 128: return launch_both<T, 128>(p, s);
        case 192: return launch_both<T, 192>(p, s);
        default: return launch_both<T, 256>(p, s);
    }
}

}  // namespace

tman_status launch_attend_i8(const CacheSeqs &c, const void *q, int ldq, void *y, int ldy, int dtype, int q_heads, float scale, int window, void *ws,
                             cudaStream_t s)
{
    uint8_t *w8 = static_cast<uint8_t *>(ws);
    const int group = q_heads / c.heads;
    const long long rows = c.starts ? (long long)c.T * group : group;
    const bool prompts = c.starts && rows >= kPromptRows;
    // steps are counted in 32 bits
    const long long steps = ((long long)c.ldt << c.page_sh) / 16 + kItemCost, tiles = ((prompts ? kPromptRows : rows) + kAttendRows - 1) / kAttendRows;
    if (tiles * steps > INT32_MAX || tiles * steps * c.heads > INT32_MAX || tiles * steps * c.heads * c.S > INT32_MAX) return TMAN_ERR_UNSUPPORTED;
    const AttendParams p = {c, q, y, reinterpret_cast<float *>(w8 + kI8ScratchOff), reinterpret_cast<uint32_t *>(w8 + kWsStatusBytes),
                            ldq, ldy, group, window, prompts ? kPromptRows : INT_MAX, group == 1 ? 0u : 0xFFFFFFFFu / (uint32_t)group + 1u, scale};
    return dtype == kF4TypeHalf ? launch_width<__half>(p, s) : launch_width<__nv_bfloat16>(p, s);
}

}  // namespace tman
