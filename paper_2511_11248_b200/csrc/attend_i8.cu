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
#include "attend_prompt.cuh"

namespace tman {
namespace {

constexpr int kPromptRows = 64;          // rows of a sequence from which the kernel for prompts takes it
constexpr int kShortSteps = 96;          // heads of so few steps are not cut
constexpr uint32_t kNoneYet = 0x7FA5A5A5u;      // what tman_workspace_init writes: a counter at rest

template <int D> struct AttendShape {
    static constexpr int kWarps = D <= 128 ? 12 : 8, kThreads = 32 * kWarps, kStages = D == 64 ? 6 : D == 128 ? 4 : 3;
    static constexpr int kStep = 32 * D, kRing = kStages * kStep, kQ = 32 * D, kSmem = kWarps * kRing + kQ;
    static_assert(kRing >= 16 * D * 4, "a warp's sums fit its ring");
};

struct AttendParams {
    CacheSeqs c;
    const void *q;
    void *y;
    float *parts;
    uint32_t *counters;
    int ldq, ldy, group, window, least;  // group: query heads of a key head; sequences of `least` rows (tokens x group) and more are done elsewhere
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

// The keys that a tile of rows sees: tokens [lo, hi), and steps of 16 of them, one at least.
struct TileKeys { int first, lo, hi, step0, steps; };            // first: position of the tile's first token
__device__ __forceinline__ TileKeys tile_keys(const AttendParams &p, const CacheSeq &q, int tile)
{
    TileKeys k;
    const int rows = q.rows * p.group, i0 = tile * kAttendRows / p.group, i1 = min(tile * kAttendRows + kAttendRows - 1, rows - 1) / p.group;
    k.first = q.len - q.rows + i0;
    k.hi = max(q.len - q.rows + i1 + 1, 0);
    k.lo = p.window > 0 ? max(k.first - p.window + 1, 0) : 0;
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
    __shared__ long long before[Sh::kThreads + 1];               // steps of the sequences in front of thread t's
    __shared__ CacheSeq known[Sh::kThreads];                     // the sequence of thread t, if each has one
    __shared__ long long place[4];
    __shared__ float row_factor[16], warp_max[W][16], warp_lmax[W][16], warp_sum[W][16];
    __shared__ uint32_t last_flag;
    const CacheSeqs &c = p.c;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, t = lane & 3, page_mask = (1 << c.page_sh) - 1;
    uint4 *qs = reinterpret_cast<uint4 *>(smem + W * Sh::kRing);
    const uint32_t ring = smem_u32(smem) + warp * Sh::kRing + lane * 16;
    const uint8_t *ring_at = smem + warp * Sh::kRing + lane * 16;
    grid_wait();
    grid_launch_next();

    const int per = (c.S + Sh::kThreads - 1) / Sh::kThreads;
    auto seq_of = [&](int s) { return per == 1 ? known[s] : cache_seq(c, s); };
    auto units_of = [&](const CacheSeq &q) -> long long {
        long long n = 0;
        for (int i = 0; i < tiles_of(p, q); ++i) n += tile_keys(p, q, i).steps;
        return n * c.heads;
    };
    {
        long long mine = 0;
        for (int s = min(tid * per, c.S); s < min(tid * per + per, c.S); ++s) {
            const CacheSeq q = cache_seq(c, s);
            if (per == 1) known[tid] = q;
            mine += units_of(q);
        }
        long long upto = mine;
        for (int d = 1; d < 32; d <<= 1) {
            const long long o = __shfl_up_sync(0xffffffffu, upto, d);
            if (lane >= d) upto += o;
        }
        before[tid + 1] = upto;
        __syncthreads();
        long long add = 0;
        for (int w = 0; w < warp; ++w) add += before[w * 32 + 32];
        __syncthreads();
        before[tid + 1] = upto + add;
        if (tid == 0) before[0] = 0;
        __syncthreads();
    }
    const long long total = before[Sh::kThreads];
    long long run = (total + gridDim.x - 1) / gridDim.x;
    run = max((run + W - 1) / W, 1ll) * W;

    // Sequence, head and tile of a unit, by all threads alike.
    struct Item { int s, head, tile; long long at; CacheSeq q; TileKeys k; };
    auto item_of = [&](long long u) {
        int lo = 0, hi = Sh::kThreads;
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (before[mid] <= u) lo = mid; else hi = mid;
        }
        Item it;
        it.at = before[lo];
        it.s = lo * per;
        for (;;) {
            const long long n = per > 1 ? units_of(cache_seq(c, it.s)) : before[lo + 1] - before[lo];
            if (u < it.at + n) break;
            it.at += n;
            ++it.s;
        }
        it.q = seq_of(it.s);
        const int tiles = tiles_of(p, it.q);
        long long one = 0;
        if (tiles > 1)
            for (int i = 0; i < tiles; ++i) one += tile_keys(p, it.q, i).steps;
        else one = tile_keys(p, it.q, 0).steps;
        it.head = (int)((u - it.at) / one);
        it.at += it.head * one;
        it.tile = 0;
        for (;;) {
            it.k = tile_keys(p, it.q, it.tile);
            if (u < it.at + it.k.steps) break;
            it.at += it.k.steps;
            ++it.tile;
        }
        return it;
    };
    // Where the runs of the CTAs begin: a short head belongs to the CTA that its first step falls to.
    auto begin_of = [&](long long cta) {
        const long long u = cta * run;
        if (u >= total || u <= 0) return u <= 0 ? 0ll : total;
        const Item it = item_of(u);
        return it.at != u && it.k.steps <= kShortSteps ? it.at + it.k.steps : u;
    };
    if (tid < 2) place[tid] = begin_of((long long)blockIdx.x + tid);
    __syncthreads();
    const long long begin = place[0], end = place[1];

    for (long long u = begin; u < end;) {
        const Item it = item_of(u);
        const int s0 = (int)(u - it.at), s1 = (int)min((long long)it.k.steps, end - it.at);       // steps of this run
        const bool whole = s0 == 0 && s1 == it.k.steps;
        const int rows = min(kAttendRows, it.q.rows * p.group - it.tile * kAttendRows);
        u = it.at + s1;

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
#pragma unroll
        for (int i = 0; i < Sh::kStages - 1; ++i) fetch(i, i);

        // ---- queries: rows of the tile as A operands, zero behind the last
        if (warp < 16) {
            for (int r = warp; r < 16; r += W) {
                const int rho = it.tile * kAttendRows + r;
                uint32_t top = 0;
                const T *src = static_cast<const T *>(p.q) + (size_t)(it.q.row + rho / p.group) * p.ldq + (size_t)(it.head * p.group + rho % p.group) * D;
                float f = 1.f;
                if constexpr (!std::is_same<T, __half>::value) {
                    if (r < rows)
                        for (int i = lane; i < D / 8; i += 32) {
                            const uint4 v = ld_dependent(reinterpret_cast<const uint4 *>(src) + i);
                            top = i8_larger(top, i8_larger(i8_larger(i8_magnitudes(v.x), i8_magnitudes(v.y)), i8_larger(i8_magnitudes(v.z), i8_magnitudes(v.w))));
                        }
                    top = __reduce_max_sync(0xffffffffu, max(top & 0xFFFFu, top >> 16));
                    const int e = (int)(top >> 7) - 127;          // largest value in [2^e, 2^(e + 1))
                    f = top == 0 || top >= i8_infinity<T>() ? 1.f : __uint_as_float((uint32_t)(127 + min(14 - e, 100)) << 23);
                }
                if (lane == 0) row_factor[r] = p.scale * kLog2e / f;
                // columns 64 i + 16 t + 4 j of row r: step 4 i + j of k, lane 4 (r % 8) + t, words (r / 8) and (r / 8) + 2
                for (int i = lane; i < D / 4; i += 32) {
                    uint2 h = make_uint2(0, 0);
                    if (r < rows) {
                        uint2 raw;
                        asm volatile("ld.global.v2.u32 {%0, %1}, [%2];" : "=r"(raw.x), "=r"(raw.y) : "l"(reinterpret_cast<const uint2 *>(src) + i) : "memory");
                        if constexpr (std::is_same<T, __half>::value) h = raw;
                        else {
                            const float2 a = f4_to_float2<T>(raw.x), b = f4_to_float2<T>(raw.y);
                            h = make_uint2(f4_from_float2<__half>(a.x * f, a.y * f), f4_from_float2<__half>(b.x * f, b.y * f));
                        }
                    }
                    const int step = (i >> 4) * 4 + (i & 3), l = (r & 7) * 4 + ((i >> 2) & 3);
                    uint32_t *at = reinterpret_cast<uint32_t *>(qs + step * 32 + l) + (r >> 3);
                    at[0] = h.x;
                    at[2] = h.y;
                }
            }
        }
        __syncthreads();

        const float rf0 = row_factor[g], rf1 = row_factor[g + 8];
        auto limit_of = [&](int r) { return it.q.len - it.q.rows + (it.tile * kAttendRows + min(r, rows - 1)) / p.group; };
        const int lim0 = limit_of(g), lim1 = limit_of(g + 8);
        const int low0 = p.window > 0 ? lim0 - p.window + 1 : INT_MIN, low1 = p.window > 0 ? lim1 - p.window + 1 : INT_MIN;
        const int all_from = p.window > 0 ? it.k.hi - p.window : INT_MIN;       // tokens [all_from, first] are seen by every row
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
            *reinterpret_cast<float2 *>(os + g * D + 8 * i + 2 * t) = make_float2(o[i][0], o[i][1]);
            *reinterpret_cast<float2 *>(os + (g + 8) * D + 8 * i + 2 * t) = make_float2(o[i][2], o[i][3]);
        }
        __syncthreads();
        const long long first_cta = it.at / run;
        float *part = p.parts + ((size_t)blockIdx.x * 2 + (s0 == 0 ? 1 : 0)) * (kAttendRows * (D + 4));
        // y of (row, column) from sums relative to `m`, probabilities relative to `lm`
        auto store = [&](int r, int col, float v, float m, float lm, float l) {
            const int rho = it.tile * kAttendRows + r;
            const float out = l == 0.f ? 0.f : v * exp2_fast((m == -INFINITY ? 0.f : m) - (lm == -INFINITY ? 0.f : lm)) / l;
            static_cast<T *>(p.y)[(size_t)(it.q.row + rho / p.group) * p.ldy + (size_t)(it.head * p.group + rho % p.group) * D + col] = f4_from_float<T>(out);
        };
        for (int i = tid; i < rows * D; i += Sh::kThreads) {
            const int r = i / D, col = i % D;
            float m = -INFINITY, lm = -INFINITY;
#pragma unroll
            for (int w = 0; w < W; ++w) {
                m = fmaxf(m, warp_max[w][r]);
                lm = fmaxf(lm, warp_lmax[w][r]);
            }
            const float um = m == -INFINITY ? 0.f : m, ul = lm == -INFINITY ? 0.f : lm;
            float v = 0.f, l = 0.f;
#pragma unroll
            for (int w = 0; w < W; ++w) {
                v += reinterpret_cast<const float *>(smem + w * Sh::kRing)[i] * exp2_fast(warp_max[w][r] - um);
                l += warp_sum[w][r] * exp2_fast(warp_lmax[w][r] - ul);
            }
            if (whole) store(r, col, v, m, lm, l);
            else {
                __stcg(part + i, v);
                if (col == 0) {
                    __stcg(part + 16 * D + r, m);
                    __stcg(part + 16 * D + 16 + r, lm);
                    __stcg(part + 16 * D + 32 + r, l);
                }
            }
        }
        if (!whole) {
            const int pieces = (int)((it.at + it.k.steps - 1) / run - first_cta) + 1;
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
                auto part_of = [&](int i) { return p.parts + ((size_t)(first_cta + i) * 2 + (i == 0 ? 1 : 0)) * (kAttendRows * (D + 4)); };
                for (int i = tid; i < rows * D; i += Sh::kThreads) {
                    const int r = i / D, col = i % D;
                    float m = -INFINITY, lm = -INFINITY, v = 0.f, l = 0.f;
                    for (int k = 0; k < pieces; ++k) {
                        m = fmaxf(m, __ldcg(part_of(k) + 16 * D + r));
                        lm = fmaxf(lm, __ldcg(part_of(k) + 16 * D + 16 + r));
                    }
                    const float um = m == -INFINITY ? 0.f : m, ul = lm == -INFINITY ? 0.f : lm;
                    for (int k = 0; k < pieces; ++k) {
                        v += __ldcg(part_of(k) + i) * exp2_fast(__ldcg(part_of(k) + 16 * D + r) - um);
                        l += __ldcg(part_of(k) + 16 * D + 32 + r) * exp2_fast(__ldcg(part_of(k) + 16 * D + 16 + r) - ul);
                    }
                    store(r, col, v, m, lm, l);
                }
            }
        }
        __syncthreads();
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
    if (p.c.starts && (long long)p.c.T * p.group >= kPromptRows) {
        p.least = kPromptRows;
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
    const AttendParams p = {c, q, y, reinterpret_cast<float *>(w8 + kWsStatusBytes + kAttendCtas * 4), reinterpret_cast<uint32_t *>(w8 + kWsStatusBytes),
                            ldq, ldy, q_heads / c.heads, window, INT_MAX, scale};
    return dtype == kF4TypeHalf ? launch_width<__half>(p, s) : launch_width<__nv_bfloat16>(p, s);
}

}  // namespace tman
