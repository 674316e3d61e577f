// The 8-bit cache: appending tokens and reading them back.
#include "cache_i8.cuh"

namespace tman {
namespace {

constexpr int kCacheThreads = 128;

// Which of the things that the sequences have in turn, `of(s)` of them each, is number `index`: found[0] is its sequence (-1: there are fewer),
// found[1] its place in it.  All threads.
template <typename Of> __device__ __forceinline__ void find_in_sequences(int S, int index, int (&found)[2], int (&warps)[kCacheThreads / 32], const Of &of)
{
    const int tid = threadIdx.x, lane = tid & 31, per = (S + kCacheThreads - 1) / kCacheThreads, s0 = min(tid * per, S), s1 = min(s0 + per, S);
    int mine = 0;
    for (int s = s0; s < s1; ++s) mine += of(s);
    int upto = mine;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const int o = __shfl_up_sync(0xffffffffu, upto, d);
        if (lane >= d) upto += o;
    }
    if (lane == 31) warps[tid >> 5] = upto;
    if (tid == 0) found[0] = -1;
    __syncthreads();
    for (int w = 0; w < (tid >> 5); ++w) upto += warps[w];
    int before = upto - mine;
    if (index >= before && index < upto) {
        int s = s0;
        if (per > 1)
            for (int n; index >= before + (n = of(s)); ++s) before += n;
        found[0] = s;
        found[1] = index - before;
    }
    __syncthreads();
}
// Steps of 2^sh tokens that a sequence's rows lie in; none of one whose rows are more than its tokens (the status word says so).
__device__ __forceinline__ int steps_of(const CacheSeqs &c, int s, int sh)
{
    const CacheSeq q = cache_seq(c, s);
    if (q.rows > q.len) {
        atomicCAS(c.status, 0u, (uint32_t)TMAN_ERR_INDEX);
        return 0;
    }
    return q.rows == 0 ? 0 : ((q.len - 1) >> sh) - ((q.len - q.rows) >> sh) + 1;
}

// ---- append: a CTA has one page that changes, one head, keys or values ----------------------------------------------------------
// scale = max(old scale, max|new| / 127); codes that are there already become round(code x old / scale), new ones round(x / scale).  The page's
// codes are put together in shared memory and leave as they came, in 16-byte pieces.
// Bound by latency for few tokens (what sequence, what page, what maximum, one behind the other) and by reading the rows for many: a thread takes
// eight columns of four tokens whose codes are neighbours in the cache (cache_i8.cuh), so that values need no byte stores, and keeps the first it takes
// in registers between the maximum and the codes (pages of more than 4096 values are read twice).
struct AppendParams {
    CacheSeqs c;
    const void *k, *v;
    int ldk, ldv;
};

template <typename T>
__global__ void __launch_bounds__(kCacheThreads) append_kernel(const __grid_constant__ AppendParams p)
{
    extern __shared__ __align__(16) uint8_t tiles[];
    __shared__ int found[2], warps[kCacheThreads / 32];
    __shared__ uint32_t tops[kCacheThreads / 32];
    const CacheSeqs &c = p.c;
    const int tid = threadIdx.x, lane = tid & 31, head = blockIdx.y, values = blockIdx.z, page = 1 << c.page_sh, width = c.width;
    grid_wait();
    grid_launch_next();
    find_in_sequences(c.S, blockIdx.x, found, warps, [&](int s) { return steps_of(c, s, c.page_sh); });
    const int s = found[0];
    if (s < 0) return;
    const CacheSeq q = cache_seq(c, s);
    const int first = q.len - q.rows, at = (first >> c.page_sh) + found[1], id = cache_page(c, s, at);
    if (id < 0) return;
    const int r0 = max(first - (at << c.page_sh), 0), r1 = min(q.len - (at << c.page_sh), page);      // new tokens of the page
    const int ld = values ? p.ldv : p.ldk, pieces = width >> 3;
    const T *x = static_cast<const T *>(values ? p.v : p.k) + (ptrdiff_t)(q.row + (at << c.page_sh) - first) * ld + (size_t)head * width;
    uint8_t *codes = c.cache + (((size_t)id * c.heads + head) * 2 + values) * page * width;
    float *scale_at = reinterpret_cast<float *>(c.cache + c.scales_off) + ((size_t)id * c.heads + head) * 2 + values;
    const int end = (r1 + 15) >> 4, words = end * width;         // tiles, and their 16-byte pieces
    const int quads = (end - (r0 >> 4)) * 4 * pieces;            // quadruples of rows in tiles with new ones x pieces of eight columns
    // quadruple i: tokens 2 t, 2 t + 1, 2 t + 8, 2 t + 9 of a tile
    auto rows_of = [&](int i, int &row, int &piece) {
        piece = i % pieces;
        const int n = i / pieces;
        row = ((r0 >> 4) + (n >> 2)) * 16 + (n & 3) * 2;
    };
    auto row_in = [&](int row, int e) { const int r = row + (e >> 1) * 8 + (e & 1); return r >= r0 && r < r1; };
    auto load = [&](int row, int piece, int e) {
        return row_in(row, e) ? ld_dependent(reinterpret_cast<const uint4 *>(x + (ptrdiff_t)(row + (e >> 1) * 8 + (e & 1)) * ld) + piece) : make_uint4(0, 0, 0, 0);
    };
    uint4 held[4];
    int row = 0, piece = 0;
    rows_of(tid, row, piece);
#pragma unroll
    for (int e = 0; e < 4; ++e) held[e] = tid < quads ? load(row, piece, e) : make_uint4(0, 0, 0, 0);
    uint4 *st = reinterpret_cast<uint4 *>(tiles);
    for (int i = tid; i < words; i += kCacheThreads) st[i] = r0 > 0 ? ld_dependent(reinterpret_cast<const uint4 *>(codes) + i) : make_uint4(0, 0, 0, 0);
    const float old = r0 > 0 ? ld_dependent(scale_at) : 0.f;
    uint32_t top = 0;
    uint4 v[4] = {held[0], held[1], held[2], held[3]};
#pragma unroll 1
    for (int i = tid;;) {
#pragma unroll
        for (int e = 0; e < 4; ++e) top = i8_larger(top, i8_larger(i8_larger(i8_magnitudes(v[e].x), i8_magnitudes(v[e].y)), i8_larger(i8_magnitudes(v[e].z), i8_magnitudes(v[e].w))));
        if ((i += kCacheThreads) >= quads) break;
        rows_of(i, row, piece);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = load(row, piece, e);
    }
    top = __reduce_max_sync(0xffffffffu, max(top & 0xFFFFu, top >> 16));
    if (lane == 0) tops[tid >> 5] = top;
    __syncthreads();
    top = __reduce_max_sync(0xffffffffu, tops[lane & (kCacheThreads / 32 - 1)]);
    const float fresh = i8_scale<T>(top), scale = old != old ? old : fresh <= old ? old : fresh;       // (a NaN of either stays)
    const float ratio = scale > 0.f ? __fdiv_rn(old, scale) : 0.f;
    if (r0 > 0 && scale != old) {                                // codes that are there already
        for (int i = tid; i < r0 * width; i += kCacheThreads) {
            const int r = i / width, col = i % width, tile = (r >> 4) * 16 * width;
            uint8_t *b = tiles + tile + (values ? cache_value_at(r & 15, col) : cache_key_at(r & 15, col));
            *b = (uint8_t)(int8_t)(int)rintf((float)(int8_t)*b * ratio);
        }
    }
    const I8Divisor d(scale);
#pragma unroll 1
    for (int i = tid; i < quads; i += kCacheThreads) {
        rows_of(i, row, piece);
        uint2 u[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) u[e] = i8_codes<T>(d, i == tid ? held[e] : load(row, piece, e));
        uint8_t *tile = tiles + (row >> 4) * 16 * width;
        if (!values) {
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (row_in(row, e)) *reinterpret_cast<uint2 *>(tile + cache_key_at((row & 15) + (e >> 1) * 8 + (e & 1), piece * 8)) = u[e];
        } else {
            // the four tokens' bytes of a column are a word: all of it where all four are new
            const bool all = row_in(row, 0) && row_in(row, 3);
#pragma unroll
            for (int col = 0; col < 8; ++col) {
                const uint32_t sel = (col & 3) | (4 + (col & 3)) << 4;
                const uint32_t lo = __byte_perm(col < 4 ? u[0].x : u[0].y, col < 4 ? u[1].x : u[1].y, sel), hi = __byte_perm(col < 4 ? u[2].x : u[2].y, col < 4 ? u[3].x : u[3].y, sel);
                const uint32_t word = __byte_perm(lo, hi, 0x5410);
                uint8_t *to = tile + cache_value_at(row & 15, piece * 8 + col);
                if (all) *reinterpret_cast<uint32_t *>(to) = word;
                else
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (row_in(row, e)) to[e] = (uint8_t)(word >> (8 * e));
            }
        }
    }
    __syncthreads();
    const int begin = r0 > 0 && scale == old ? (r0 >> 4) * width : 0;
    for (int i = begin + tid; i < words; i += kCacheThreads) reinterpret_cast<uint4 *>(codes)[i] = st[i];
    if (tid == 0) *scale_at = scale;
}

// ---- read: tokens back in 16 bits; a CTA has the 16 tokens of a tile and one head ---------------------------------------------------
// Pieces come as they lie in the cache and are turned into rows in shared memory.
struct ReadParams {
    CacheSeqs c;
    void *k, *v;
    int ldk, ldv;
};

template <typename T>
__global__ void __launch_bounds__(kCacheThreads) read_cache_kernel(const __grid_constant__ ReadParams p)
{
    extern __shared__ __align__(16) uint8_t tiles[];             // [keys, values][16 tokens][width + 8]
    __shared__ int found[2], warps[kCacheThreads / 32];
    const CacheSeqs &c = p.c;
    const int tid = threadIdx.x, head = blockIdx.y, width = c.width, pitch = width + 8, page = 1 << c.page_sh;
    T *rows = reinterpret_cast<T *>(tiles);
    grid_wait();
    grid_launch_next();
    find_in_sequences(c.S, blockIdx.x, found, warps, [&](int s) { return steps_of(c, s, 4); });
    const int s = found[0];
    if (s < 0) return;
    const CacheSeq q = cache_seq(c, s);
    const int first = q.len - q.rows, token0 = ((first >> 4) + found[1]) * 16, id = cache_page(c, s, token0 >> c.page_sh);
    if (id < 0) return;
    const size_t at = ((size_t)id * c.heads + head) * 2;
    const uint8_t *tile = c.cache + at * page * width + (token0 & (page - 1)) * width;
    const float *scales = reinterpret_cast<const float *>(c.cache + c.scales_off) + at;
    const float ks = ld_dependent(scales), vs = ld_dependent(scales + 1);
#pragma unroll 2
    for (int i = tid; i < 2 * width; i += kCacheThreads) {       // pieces of keys, then of values
        const bool values = i >= width;
        const int j = values ? i - width : i, piece = j >> 5, g = (j & 31) >> 2, t = j & 3;
        const uint4 u = ld_dependent(reinterpret_cast<const uint4 *>(tile + (values ? (size_t)page * width : 0)) + j);
        const uint32_t w[4] = {u.x, u.y, u.z, u.w};
        const float f = values ? vs : ks;
        if (!values) {
            uint32_t h[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) h[e] = f4_from_float2<T>((float)(int8_t)(w[e >> 1] >> (16 * (e & 1))) * f, (float)(int8_t)(w[e >> 1] >> (16 * (e & 1) + 8)) * f);
            uint4 *to = reinterpret_cast<uint4 *>(rows + ((piece & 1) * 8 + g) * pitch + (piece >> 1) * 64 + t * 16);
            to[0] = make_uint4(h[0], h[1], h[2], h[3]);
            to[1] = make_uint4(h[4], h[5], h[6], h[7]);
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e)
#pragma unroll
                for (int b = 0; b < 4; ++b)
                    rows[(16 + 2 * t + (b >> 1) * 8 + (b & 1)) * pitch + (4 * piece + e) * 8 + g] = f4_from_float<T>((float)(int8_t)(w[e] >> (8 * b)) * f);
        }
    }
    __syncthreads();
    const int pieces = width >> 3, r0 = max(first - token0, 0), r1 = min(q.len - token0, 16);
    for (int i = tid; i < 32 * pieces; i += kCacheThreads) {
        const int r = i / pieces, j = i % pieces, values = r >> 4, token = r & 15;
        if (token < r0 || token >= r1) continue;
        const size_t row = (size_t)(q.row + token0 + token - first);
        T *out = (values ? static_cast<T *>(p.v) + row * p.ldv : static_cast<T *>(p.k) + row * p.ldk) + (size_t)head * width;
        reinterpret_cast<uint4 *>(out)[j] = *reinterpret_cast<const uint4 *>(rows + r * pitch + j * 8);
    }
}

template <typename Kernel, typename Params> tman_status launch(Kernel kern, const Params &p, dim3 grid, size_t smem, cudaStream_t s)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(kCacheThreads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return call_status(cudaLaunchKernelEx(&cfg, kern, p));
}

}  // namespace

tman_status launch_append_i8(const CacheSeqs &c, const void *k, int ldk, const void *v, int ldv, int dtype, cudaStream_t s)
{
    const AppendParams p = {c, k, v, ldk, ldv};
    // pages that change: a sequence of n rows has at most n / page + 2, and n, of them
    const long long most = ((long long)c.T >> c.page_sh) + 2ll * c.S;
    const dim3 grid((unsigned)(most < c.T ? most : c.T), (unsigned)c.heads, 2);
    const size_t smem = (size_t)c.width << c.page_sh;
    return dtype == kF4TypeHalf ? launch(append_kernel<__half>, p, grid, smem, s) : launch(append_kernel<__nv_bfloat16>, p, grid, smem, s);
}

tman_status launch_read_cache_i8(const CacheSeqs &c, void *k, int ldk, void *v, int ldv, int dtype, cudaStream_t s)
{
    const ReadParams p = {c, k, v, ldk, ldv};
    const long long most = ((long long)c.T >> 4) + 2ll * c.S;    // (tiles, as above)
    const dim3 grid((unsigned)(most < c.T ? most : c.T), (unsigned)c.heads);
    const size_t smem = (size_t)32 * (c.width + 8) * 2;
    return dtype == kF4TypeHalf ? launch(read_cache_kernel<__half>, p, grid, smem, s) : launch(read_cache_kernel<__nv_bfloat16>, p, grid, smem, s);
}

}  // namespace tman
