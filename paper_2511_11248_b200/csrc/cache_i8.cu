// The 8-bit cache: appending tokens and reading them back.
#include "cache_i8.cuh"

namespace tman {
namespace {

constexpr int kCacheThreads = 128;

// ---- append: a CTA has one page that changes, one head, keys or values ----------------------------------------------------------
// scale = max(old scale, max|new| / 127); codes that are there already become round(code x old / scale), new ones round(x / scale).  The page's
// codes are put together in shared memory and leave as they came, in 16-byte pieces.
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
    // pages that change, counted over the sequences: which one is this CTA's
    {
        const int per = (c.S + kCacheThreads - 1) / kCacheThreads, s0 = min(tid * per, c.S), s1 = min(s0 + per, c.S);
        auto pages_of = [&](int s) {
            const CacheSeq q = cache_seq(c, s);
            if (q.rows > q.len) {
                atomicCAS(c.status, 0u, (uint32_t)TMAN_ERR_INDEX);
                return 0;
            }
            return q.rows == 0 ? 0 : ((q.len - 1) >> c.page_sh) - ((q.len - q.rows) >> c.page_sh) + 1;
        };
        int mine = 0;
        for (int s = s0; s < s1; ++s) mine += pages_of(s);
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
        if ((int)blockIdx.x >= before && (int)blockIdx.x < upto)
            for (int s = s0; s < s1; ++s) {
                const int n = pages_of(s);
                if ((int)blockIdx.x < before + n) {
                    found[0] = s;
                    found[1] = (int)blockIdx.x - before;
                    break;
                }
                before += n;
            }
        __syncthreads();
    }
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
    uint4 *st = reinterpret_cast<uint4 *>(tiles);
    for (int i = tid; i < words; i += kCacheThreads) st[i] = r0 > 0 ? ld_dependent(reinterpret_cast<const uint4 *>(codes) + i) : make_uint4(0, 0, 0, 0);
    const float old = r0 > 0 ? ld_dependent(scale_at) : 0.f;
    uint32_t top = 0;
    for (int i = tid; i < (r1 - r0) * pieces; i += kCacheThreads) {
        const int r = r0 + i / pieces, j = i % pieces;
        const uint4 v = ld_dependent(reinterpret_cast<const uint4 *>(x + (ptrdiff_t)r * ld) + j);
        top = i8_larger(top, i8_larger(i8_larger(i8_magnitudes(v.x), i8_magnitudes(v.y)), i8_larger(i8_magnitudes(v.z), i8_magnitudes(v.w))));
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
    for (int i = tid; i < (r1 - r0) * pieces; i += kCacheThreads) {
        const int r = r0 + i / pieces, j = i % pieces;
        const uint2 v = i8_codes<T>(d, ld_dependent(reinterpret_cast<const uint4 *>(x + (ptrdiff_t)r * ld) + j));
        uint8_t *tile = tiles + (r >> 4) * 16 * width;
        if (!values) *reinterpret_cast<uint2 *>(tile + cache_key_at(r & 15, j * 8)) = v;
        else {
#pragma unroll
            for (int e = 0; e < 8; ++e) tile[cache_value_at(r & 15, j * 8 + e)] = (uint8_t)((e < 4 ? v.x : v.y) >> (8 * (e & 3)));
        }
    }
    __syncthreads();
    const int begin = r0 > 0 && scale == old ? (r0 >> 4) * width : 0;
    for (int i = begin + tid; i < words; i += kCacheThreads) reinterpret_cast<uint4 *>(codes)[i] = st[i];
    if (tid == 0) *scale_at = scale;
}

// ---- read: tokens back in 16 bits ------------------------------------------------------------------------------------------------
struct ReadParams {
    CacheSeqs c;
    void *k, *v;
    int ldk, ldv;
};

// The sequence that row `row` belongs to: the last one that starts at or before it, if its rows reach so far.
__device__ __forceinline__ int sequence_of(const CacheSeqs &c, int row)
{
    if (!c.starts) return row < c.S ? row : -1;
    int lo = 0, hi = c.S;                                        // starts[lo] <= row < starts[hi]
    if (ld_dependent(c.starts) > row || ld_dependent(c.starts + c.S) <= row) return -1;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (ld_dependent(c.starts + mid) <= row) lo = mid; else hi = mid;
    }
    return lo;
}

template <typename T>
__global__ void __launch_bounds__(kCacheThreads) read_cache_kernel(const __grid_constant__ ReadParams p)
{
    const CacheSeqs &c = p.c;
    const int row = blockIdx.x, pieces = c.width >> 3, page = 1 << c.page_sh;
    grid_wait();
    grid_launch_next();
    if (row == 0)                                                // (what no row is found by is reported all the same)
        for (int i = threadIdx.x; i < c.S; i += kCacheThreads) {
            const CacheSeq q = cache_seq(c, i);
            if (q.rows > q.len) atomicCAS(c.status, 0u, (uint32_t)TMAN_ERR_INDEX);
        }
    const int s = sequence_of(c, row);
    if (s < 0) return;
    const CacheSeq q = cache_seq(c, s);
    if (row < q.row || row >= q.row + q.rows) return;
    const int pos = q.len - q.rows + row - q.row;
    if (pos < 0) return;
    const int id = cache_page(c, s, pos >> c.page_sh), r = pos & (page - 1);
    if (id < 0) return;
    const float *scales = reinterpret_cast<const float *>(c.cache + c.scales_off) + (size_t)id * c.heads * 2;
    for (int i = threadIdx.x; i < c.heads * 2 * pieces; i += kCacheThreads) {
        const int h2 = i / pieces, j = i % pieces, values = h2 & 1;
        const uint8_t *tile = c.cache + ((size_t)id * c.heads * 2 + h2) * page * c.width + (r >> 4) * 16 * c.width;
        const float scale = ld_dependent(scales + h2);
        float z[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const uint8_t *b = tile + (values ? cache_value_at(r & 15, j * 8 + e) : cache_key_at(r & 15, j * 8 + e));
            z[e] = (float)*reinterpret_cast<const volatile int8_t *>(b) * scale;
        }
        T *out = values ? static_cast<T *>(p.v) + (size_t)row * p.ldv : static_cast<T *>(p.k) + (size_t)row * p.ldk;
        *reinterpret_cast<uint4 *>(out + (h2 >> 1) * c.width + j * 8) =
            make_uint4(f4_from_float2<T>(z[0], z[1]), f4_from_float2<T>(z[2], z[3]), f4_from_float2<T>(z[4], z[5]), f4_from_float2<T>(z[6], z[7]));
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
    const dim3 grid((unsigned)c.T);
    return dtype == kF4TypeHalf ? launch(read_cache_kernel<__half>, p, grid, 0, s) : launch(read_cache_kernel<__nv_bfloat16>, p, grid, 0, s);
}

}  // namespace tman
