// Microscaled 4-bit floating point: packing and unpacking of a checkpoint's matrix, quantization of rows, dequantization.
// Memory-bound: every value is read and written once.
#include "f4.cuh"
#include "sm100_ptx.cuh"

#include <type_traits>

namespace tman {

// ---- checkpoint layout <-> packed buffer -----------------------------------------------------
// codes [rows][K/2], scales [rows][K/block], row_scale [rows].  One thread moves 8 bytes of codes (16 values); the first thread of a
// block of four scales moves those.
template <int BLOCK, bool TO_PACKED>
__global__ void __launch_bounds__(256) f4_relayout_kernel(uint8_t *codes, uint8_t *scales, float *row_scale, int rows, int K, uint8_t *packed,
                                                          F4Layout L, bool vec, uint32_t *status)
{
    const size_t i = (size_t)blockIdx.x * 256 + threadIdx.x;
    if constexpr (TO_PACKED) {
        if (i < 64) reinterpret_cast<uint32_t *>(packed)[i] = f4_header_word((int)i, rows, K, BLOCK, L);
    } else if (!f4_header_matches(packed, rows, K, BLOCK)) {
        if (i == 0) atomicCAS(status, 0u, (uint32_t)TMAN_ERR_BAD_PACKED);
        return;
    }
    const int pieces = L.halves * (kF4Half / 16);
    const int r = (int)(i / pieces), k = (int)(i % pieces) * 16;
    if (r >= L.tiles * kF4Tile) return;
    const int nb = K / BLOCK, b = k / BLOCK;
    if (r < L.height8) {
        uint8_t *c = packed + L.codes_off + f4_code_at(r, k, L);
        uint8_t *plain = codes + ((size_t)r * K + k) / 2;
        const bool in = r < rows && k < K;
        if constexpr (TO_PACKED) {
            uint64_t v = 0;
            if (in && vec) v = *reinterpret_cast<const uint64_t *>(plain);
            else if (in)
                for (int e = 0; e < 8; ++e) v |= (uint64_t)plain[e] << (8 * e);
            *reinterpret_cast<uint64_t *>(c) = v;
        } else if (in) {
            const uint64_t v = *reinterpret_cast<const uint64_t *>(c);
            if (vec) *reinterpret_cast<uint64_t *>(plain) = v;
            else for (int e = 0; e < 8; ++e) plain[e] = (uint8_t)(v >> (8 * e));
        }
    }
    if (k % (4 * BLOCK) == 0) {
        uint8_t *c = packed + L.scales_off + f4_scale_at(r, b, BLOCK, L);
        for (int e = 0; e < 4; ++e) {
            const bool in = r < rows && b + e < nb;
            if constexpr (TO_PACKED) c[e] = in ? scales[(size_t)r * nb + b + e] : 0;
            else if (in) scales[(size_t)r * nb + b + e] = c[e];
        }
    }
    if (BLOCK == 16 && k == 0) {
        float *c = reinterpret_cast<float *>(packed + L.rows_off) + r;
        if constexpr (TO_PACKED) *c = r < rows ? (row_scale ? row_scale[r] : 1.f) : 0.f;
        else if (r < rows && row_scale) row_scale[r] = *c;
    } else if (BLOCK == 32 && k == 0 && !TO_PACKED && r < rows && row_scale)
        row_scale[r] = 1.f;
}

template <bool TO_PACKED>
static tman_status launch_relayout(uint8_t *codes, uint8_t *scales, float *row_scale, int rows, int K, int block, void *packed, uint32_t *status, cudaStream_t s)
{
    const F4Layout L = f4_layout(rows, K, block);
    const size_t threads = (size_t)L.tiles * kF4Tile * L.halves * (kF4Half / 16), grid = (threads + 255) / 256;
    if (grid > 0x7FFFFFFFull) return TMAN_ERR_SHAPE;
    auto kern = block == 32 ? f4_relayout_kernel<32, TO_PACKED> : f4_relayout_kernel<16, TO_PACKED>;
    kern<<<(unsigned)grid, 256, 0, s>>>(codes, scales, row_scale, rows, K, static_cast<uint8_t *>(packed), L, (reinterpret_cast<uintptr_t>(codes) & 7) == 0, status);
    return launch_status();
}

tman_status launch_f4_pack(const uint8_t *codes, const uint8_t *scales, const float *row_scale, int rows, int K, int block, void *packed, cudaStream_t s)
{
    const tman_status st = launch_relayout<true>(const_cast<uint8_t *>(codes), const_cast<uint8_t *>(scales), const_cast<float *>(row_scale), rows, K,
                                                 block, packed, nullptr, s);
    if (st == TMAN_OK) note_packed_write(s);
    return st;
}

tman_status launch_f4_unpack(const void *packed, int rows, int K, int block, uint8_t *codes, uint8_t *scales, float *row_scale, uint32_t *status,
                             cudaStream_t s)
{
    return launch_relayout<false>(codes, scales, row_scale, rows, K, block, const_cast<void *>(packed), status, s);
}

// ---- quantization of rows ----------------------------------------------------------------------
// The kernels let their successor start once their predecessor has ended, so that a product behind them fetches its weights meanwhile; what they
// write is read only behind the successor's wait.  Unless it is the successor's weights: such a product is launched in plain stream order
// (f4_read_ahead).  (An earlier quantization has ended when a later one has let anything start.)

// One block's scale byte and the codes of eight of its values.  top: the largest magnitude of the block; fine: all its values are finite;
// inv_row: 1 / r, a power of two.
//   block 32: scale 2^e, e = floor(log2 top) - 2 (at least -127): x 2^-e is exact, one rounding.
//   block 16: scale s = e4m3(top / (6 r)), codes round(x / (r s)).  Both quotients of numbers of few significant bits (x and top at most 11, s
//   four, 6 two; r is a power of two) are either exactly half way between two values of the target, or further than 2^-11 of themselves
//   from it.  A product with the reciprocal is off by less than 2^-21; the reciprocal is taken 2^-18 too large and the product cut to
//   17 significant bits, which brings the half-way cases to exactly half way and the others across no border: the roundings are those of
//   the exact quotients.  (Correctly rounded divisions and a rounding in two operations: 2048 x 14336 30.1 us instead of 19.8.)
// A block that holds an infinity or a NaN gets the scale NaN.
constexpr float kAbove = 1.f + 0x1p-18f;
__device__ __forceinline__ float cut17(float v) { return __uint_as_float(__float_as_uint(v) & 0xFFFFFF80u); }
template <int BLOCK>
__device__ __forceinline__ uint32_t f4_block_scale(float top, bool fine, float inv_row)
{
    if constexpr (BLOCK == 32) {
        if (!fine) return 255u;
        const int e = (int)(__float_as_uint(top) >> 23) - 2;         // biased exponent of the scale
        return (uint32_t)max(e, 0);
    } else
        return fine ? f4_round_e4m3(cut17(top * inv_row * (kAbove / 6.f))) : 0x7Fu;
}
template <int BLOCK, typename T>
__device__ __forceinline__ uint32_t f4_block_codes(const float (&x)[8], uint32_t scale, float inv_row)
{
    float v[8];
    if constexpr (BLOCK == 32) {
        const float inv = __uint_as_float(scale >= 254u ? 0x00400000u : (254u - scale) << 23);       // 2^(127 - byte); 2^-127 for 254
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = x[e] * inv;
    } else {
        // (bf16's 1 / (r s) may leave the range: in two factors)
        constexpr bool ONE = std::is_same<T, __half>::value;
        const float s = f4_scale_value<16>(scale), inv = scale ? __fdividef(kAbove, s) * (ONE ? inv_row : 1.f) : 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = cut17((ONE ? x[e] : x[e] * inv_row) * inv);
    }
    return f4_round8(v);
}
// The row scale of block 16: the least power of two r with m <= 2688 r (448 x 6), 2^-126 at least; 1 for a row of zeros.
__device__ __forceinline__ float f4_row_scale(float m)
{
    if (!(m > 0.f)) return 1.f;
    const uint32_t u = __float_as_uint(m);
    int e = (int)(u >> 23) - 11;                                     // (2688 = 1.3125 x 2^11)
    if ((u & 0x7FFFFFu) > 0x280000u) ++e;
    return __uint_as_float((uint32_t)max(e, 1) << 23);
}

// Where a row's scale is known (block 32 has none): eight rows, a group of the packed layout, a CTA.  A warp takes 8 rows x 32 columns at a time,
// lane 4 r + q eight values of row r, so that its codes are 128 contiguous bytes, and V such chunks, four of them half a unit.
constexpr int kRowsWarps = 8;

// Largest magnitudes of two packed pairs of T, as bit patterns: they order like the values, infinities and NaN above all others.
__device__ __forceinline__ uint32_t top_pair(uint32_t a, uint32_t b) { return __vmaxu2(a & 0x7FFF7FFFu, b & 0x7FFF7FFFu); }
template <typename T> constexpr uint32_t kInfBits = std::is_same<T, __half>::value ? 0x7C00u : 0x7F80u;
// Of t and eight values: the larger halves of words, NaN above all.
template <typename T> __device__ __forceinline__ uint32_t top_of(uint32_t t, const uint4 &v)
{
    using T2 = typename std::conditional<std::is_same<T, __half>::value, __half2, __nv_bfloat162>::type;
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
    T2 p[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) p[e] = __habs2(*reinterpret_cast<const T2 *>(&w[e]));
    const T2 m = __hmax2_nan(__hmax2_nan(p[0], p[1]), __hmax2_nan(p[2], p[3]));
    return __vmaxu2(t, *reinterpret_cast<const uint32_t *>(&m));
}
// The largest finite one of eight values.
template <typename T> __device__ __forceinline__ uint32_t finite_top(const uint4 &v)
{
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
    uint32_t t = 0u;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const uint32_t lo = w[e] & 0x7FFFu, hi = w[e] >> 16 & 0x7FFFu;
        t = max(t, max(lo < kInfBits<T> ? lo : 0u, hi < kInfBits<T> ? hi : 0u));
    }
    return t;
}

template <int BLOCK, typename T, int V>
__global__ void __launch_bounds__(32 * kRowsWarps) f4_quantize_kernel(const T *x, int ldx, int rows, int K, uint8_t *packed, const __grid_constant__ F4Layout L, int parts)
{
    grid_wait();
    grid_launch_next();                  // (see f4_read_ahead)
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, r = lane >> 2, q = lane & 3;
    const int part = blockIdx.x % parts, g = blockIdx.x / parts, row = g * 8 + r;
    if (blockIdx.x == 0 && threadIdx.x < 64) reinterpret_cast<uint32_t *>(packed)[threadIdx.x] = f4_header_word(threadIdx.x, rows, K, BLOCK, L);
    const int chunks = L.halves * 4, c0 = (part * kRowsWarps + warp) * V;      // this warp's chunks of 32 columns
    const uint4 *src = reinterpret_cast<const uint4 *>(x + (size_t)min(row, rows - 1) * ldx);
    uint4 v[V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const int k = (c0 + i) * 32 + q * 8;
        v[i] = make_uint4(0u, 0u, 0u, 0u);
        if (row < rows && k < K) v[i] = ld_dependent(src + k / 8);
    }
    float inv_row = 1.f;
    if constexpr (BLOCK == 16) inv_row = __uint_as_float((254u << 23) - __float_as_uint(reinterpret_cast<const float *>(packed + L.rows_off)[min(row, rows - 1)]));
    uint32_t word = 0u;                          // scales of a half unit (block 16: of two chunks)
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const int c = c0 + i;
        if (c >= chunks) break;
        const uint32_t w[4] = {v[i].x, v[i].y, v[i].z, v[i].w};
        const uint32_t t2 = __vmaxu2(top_pair(w[0], w[1]), top_pair(w[2], w[3]));
        uint32_t top = max(t2 & 0xFFFFu, t2 >> 16);
        top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
        if constexpr (BLOCK == 32) top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
        const uint32_t scale = c * 32 + q * 8 < K ? f4_block_scale<BLOCK>(f4_to_float2<T>(top).x, top < kInfBits<T>, inv_row) : 0u;
        float f[8];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float2 p = f4_to_float2<T>(w[e]);
            f[2 * e] = p.x;
            f[2 * e + 1] = p.y;
        }
        const uint32_t codes = f4_block_codes<BLOCK, T>(f, scale, inv_row);
        const int wide = (c | 7) < chunks ? 1024 : 512;
        *reinterpret_cast<uint32_t *>(packed + L.codes_off + (size_t)(c >> 3) * L.height8 * 128 + (size_t)g * wide + (c & 7) * 128 + lane * 4) = codes;
        if constexpr (BLOCK == 32) {
            word |= scale << (8 * (i & 3));
            if ((i & 3) == 3) {
                if (q == 0 && row < rows) *reinterpret_cast<uint32_t *>(packed + L.scales_off + f4_scale_at(row, c - 3, 32, L)) = word;
                word = 0u;
            }
        } else {
            // lanes q = 0 and 2 have the chunk's two scales, the first and the second byte of a pair
            const uint32_t other = __shfl_xor_sync(0xffffffffu, scale, 2);
            word |= (scale | other << 8) << (16 * (i & 1));
            if ((i & 1) == 1) {
                if (q == 0 && row < rows) *reinterpret_cast<uint32_t *>(packed + L.scales_off + f4_scale_at(row, 2 * (c - 1), 16, L)) = word;
                word = 0u;
            }
        }
    }
}

// Block 16: the row's largest magnitude comes first.  A CTA has a row, a warp a unit of 256 columns at a time, a lane V times eight values, which
// stay in registers between the two.  Neither its bytes nor the issue of its operations (113 to 128 instructions for eight values) bound it alone:
// 2048 x 14336 takes 17.3 to 20.4 us of 11.5, issue slots used 71 % while CTAs run and 57 % of all cycles, 3.46 waves of CTAs, whose loads,
// maximum and codes follow one another; 8192 x 18944 84 to 98 of 60.7, 72 % and 68 %, DRAM at 51 %.  (Rows in shared memory, brought by bulk
// copies while the pair before is worked on: 2048 x 14336 24.7 us, 8192 x 18944 115; two rows a CTA in registers 19.8 and 123; two
// passes, the second from L2, 26.7 and 127; eight rows a cluster of CTAs with the maxima through distributed shared memory 37.4 and 188.)
template <typename T, int V, int THREADS>
__global__ void __launch_bounds__(THREADS) f4_quantize16_kernel(const T *x, int ldx, int rows, int K, uint8_t *packed, const __grid_constant__ F4Layout L)
{
    constexpr int WARPS = THREADS / 32;
    __shared__ uint32_t tops[WARPS];
    grid_wait();
    grid_launch_next();                  // (see f4_read_ahead)
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, row = blockIdx.x;
    if (blockIdx.x == 0 && threadIdx.x < 64) reinterpret_cast<uint32_t *>(packed)[threadIdx.x] = f4_header_word(threadIdx.x, rows, K, 16, L);
    const uint4 *src = reinterpret_cast<const uint4 *>(x + (size_t)row * ldx) + threadIdx.x;
    const int vectors = K / 8;
    uint4 v[V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
        v[i] = make_uint4(0u, 0u, 0u, 0u);
        if (i * THREADS + (int)threadIdx.x < vectors) v[i] = ld_dependent(src + i * THREADS);
    }
    uint32_t t = 0u;
#pragma unroll
    for (int i = 0; i < V; ++i) t = top_of<T>(t, v[i]);
    t = __reduce_max_sync(0xffffffffu, max(t & 0xFFFFu, t >> 16));
    if (t >= kInfBits<T>) {                                      // an infinity or a NaN: the finite values' only
        t = 0u;
#pragma unroll
        for (int i = 0; i < V; ++i) t = max(t, finite_top<T>(v[i]));
        t = __reduce_max_sync(0xffffffffu, t);
    }
    if (lane == 0) tops[warp] = t;
    __syncthreads();
    t = __reduce_max_sync(0xffffffffu, lane < WARPS ? tops[lane] : 0u);
    const float rs = f4_row_scale(f4_to_float2<T>(t).x), inv_row = __uint_as_float((254u << 23) - __float_as_uint(rs));      // 1 / 2^n
    if (threadIdx.x == 0) reinterpret_cast<float *>(packed + L.rows_off)[row] = rs;
    const int units = (L.halves + 1) / 2, lone = L.halves & 1 ? units - 1 : -1;      // (lone: half a unit)
    const size_t code_step = (size_t)WARPS * L.height8 * 128, scale_step = (size_t)WARPS * L.tiles * (2 * f4_scale_bytes(16));
    uint8_t *codes = packed + L.codes_off + (size_t)warp * L.height8 * 128 + (size_t)(row >> 3) * 1024 + (row & 7) * 16 + (lane >> 2) * 128 + (lane & 3) * 4;
    uint8_t *scales = packed + L.scales_off + ((size_t)warp * L.tiles + (row >> 7)) * (2 * f4_scale_bytes(16)) + (row & 31) * 16 + (row >> 5 & 3) * 4 + (lane >> 3) * 512;
#pragma unroll
    for (int i = 0; i < V; ++i, codes += code_step, scales += scale_step) {
        const int u = i * WARPS + warp;
        if (u >= units) break;
        if (u == lone) {
            codes -= (size_t)(row >> 3) * 512;
            scales -= (size_t)(row >> 7) * f4_scale_bytes(16);
        }
        uint32_t bt = top_of<T>(0u, v[i]);
        bt = __vmaxu2(bt, __shfl_xor_sync(0xffffffffu, bt, 1));
        bt = max(bt & 0xFFFFu, bt >> 16);
        const uint32_t scale = i * THREADS + (int)threadIdx.x < vectors ? f4_block_scale<16>(f4_to_float2<T>(bt).x, bt < kInfBits<T>, inv_row) : 0u;
        const uint32_t w[4] = {v[i].x, v[i].y, v[i].z, v[i].w};
        float f[8];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float2 p = f4_to_float2<T>(w[e]);
            f[2 * e] = p.x;
            f[2 * e + 1] = p.y;
        }
        const uint32_t c = f4_block_codes<16, T>(f, scale, inv_row);
        uint32_t word = scale | __shfl_xor_sync(0xffffffffu, scale, 2) << 8;      // (in the first lane of eight: four blocks' scales)
        word |= __shfl_xor_sync(0xffffffffu, word, 4) << 16;
        if (lane < 16 || u != lone) {
            *reinterpret_cast<uint32_t *>(codes) = c;
            if ((lane & 7) == 0) *reinterpret_cast<uint32_t *>(scales) = word;
        }
    }
}

// Row scales of rows too long for a CTA, which are read twice.
template <typename T>
__global__ void __launch_bounds__(32 * kRowsWarps) f4_row_scales_kernel(const T *x, int ldx, int K, uint8_t *packed, const __grid_constant__ F4Layout L)
{
    __shared__ uint32_t tops[kRowsWarps];
    grid_wait();
    grid_launch_next();                  // (see f4_read_ahead)
    const uint4 *src = reinterpret_cast<const uint4 *>(x + (size_t)blockIdx.x * ldx);
    uint32_t top = 0u;
    for (int i = threadIdx.x; i < K / 8; i += 32 * kRowsWarps) top = max(top, finite_top<T>(ld_dependent(src + i)));
    top = __reduce_max_sync(0xffffffffu, top);
    if ((threadIdx.x & 31) == 0) tops[threadIdx.x >> 5] = top;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int w = 1; w < kRowsWarps; ++w) top = max(top, tops[w]);
        reinterpret_cast<float *>(packed + L.rows_off)[blockIdx.x] = f4_row_scale(f4_to_float2<T>(top).x);
    }
}

// A launch that may start while the kernel ahead drains (the kernels wait for it before they read or write).
template <typename... P, typename... A>
static tman_status launch_rows(void (*kern)(P...), long long grid, int threads, cudaStream_t s, A... args)
{
    if (grid > 0x7FFFFFFFll) return TMAN_ERR_SHAPE;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)grid);
    cfg.blockDim = dim3((unsigned)threads);
    cfg.stream = s;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return call_status(cudaLaunchKernelEx(&cfg, kern, static_cast<P>(args)...));
}

template <int BLOCK, typename T>
static tman_status launch_quantize_as(const void *xv, int ldx, int rows, int K, void *pv, cudaStream_t s)
{
    const F4Layout L = f4_layout(rows, K, BLOCK);
    const T *x = static_cast<const T *>(xv);
    uint8_t *packed = static_cast<uint8_t *>(pv);
    const int sms = sm_count();
    if (sms == 0) return TMAN_ERR_CUDA;
    const long long groups = L.height8 / 8, few = 2 * sms;       // (below two CTAs an SM, more and smaller ones)
    const auto parts = [&](int v) { return (L.halves * 4 + kRowsWarps * v - 1) / (kRowsWarps * v); };      // CTAs along K
    if constexpr (BLOCK == 16) {
        const int units = (L.halves + 1) / 2;                    // (few rows: more warps a row)
        if (rows < few && units <= 32) return launch_rows(f4_quantize16_kernel<T, 1, 1024>, rows, 1024, s, x, ldx, rows, K, packed, L);
        if (rows < few && units <= 96) return launch_rows(f4_quantize16_kernel<T, 3, 1024>, rows, 1024, s, x, ldx, rows, K, packed, L);
        if (units <= 8) return launch_rows(f4_quantize16_kernel<T, 1, 256>, rows, 256, s, x, ldx, rows, K, packed, L);
        if (units <= 16) return launch_rows(f4_quantize16_kernel<T, 2, 256>, rows, 256, s, x, ldx, rows, K, packed, L);
        if (units <= 32) return launch_rows(f4_quantize16_kernel<T, 4, 256>, rows, 256, s, x, ldx, rows, K, packed, L);
        if (units <= 56) return launch_rows(f4_quantize16_kernel<T, 7, 256>, rows, 256, s, x, ldx, rows, K, packed, L);
        if (units <= 80) return launch_rows(f4_quantize16_kernel<T, 10, 256>, rows, 256, s, x, ldx, rows, K, packed, L);
        if (units <= 128) return launch_rows(f4_quantize16_kernel<T, 16, 256>, rows, 256, s, x, ldx, rows, K, packed, L);
        const tman_status st = launch_rows(f4_row_scales_kernel<T>, rows, 32 * kRowsWarps, s, x, ldx, K, packed, L);
        if (st != TMAN_OK) return st;
        return launch_rows(f4_quantize_kernel<BLOCK, T, 8>, groups * parts(8), 32 * kRowsWarps, s, x, ldx, rows, K, packed, L, parts(8));
    } else {
        if (groups * parts(8) >= few) return launch_rows(f4_quantize_kernel<BLOCK, T, 8>, groups * parts(8), 32 * kRowsWarps, s, x, ldx, rows, K, packed, L, parts(8));
        return launch_rows(f4_quantize_kernel<BLOCK, T, 4>, groups * parts(4), 32 * kRowsWarps, s, x, ldx, rows, K, packed, L, parts(4));
    }
}

// All kernels that write a packed matrix and let their successor start: argument `at` is the matrix.
struct F4Quantizer { const void *kernel; int at; };
template <typename T> static bool quantizer_writes(const cudaKernelNodeParams &node, const void *packed)
{
    static const F4Quantizer all[] = {
        {(const void *)f4_quantize_kernel<32, T, 4>, 4},     {(const void *)f4_quantize_kernel<32, T, 8>, 4},     {(const void *)f4_quantize_kernel<16, T, 8>, 4},
        {(const void *)f4_quantize16_kernel<T, 1, 1024>, 4}, {(const void *)f4_quantize16_kernel<T, 3, 1024>, 4}, {(const void *)f4_quantize16_kernel<T, 1, 256>, 4},
        {(const void *)f4_quantize16_kernel<T, 2, 256>, 4},  {(const void *)f4_quantize16_kernel<T, 4, 256>, 4},  {(const void *)f4_quantize16_kernel<T, 7, 256>, 4},
        {(const void *)f4_quantize16_kernel<T, 10, 256>, 4}, {(const void *)f4_quantize16_kernel<T, 16, 256>, 4}, {(const void *)f4_row_scales_kernel<T>, 3}};
    for (const F4Quantizer &q : all)
        if (node.func == q.kernel) return *static_cast<const void *const *>(node.kernelParams[q.at]) == packed;
    return false;
}

static F4Order g_f4_order;

F4Order::Call f4_read_ahead(cudaStream_t s, const void *packed)
{
    return g_f4_order.ahead(s, packed, [](const cudaKernelNodeParams &node, const void *w) { return quantizer_writes<__half>(node, w) || quantizer_writes<__nv_bfloat16>(node, w); });
}
void f4_read_behind(const F4Order::Call &call, bool launched) { g_f4_order.behind(call, launched); }

tman_status launch_f4_quantize(const void *x, int ldx, int dtype, int rows, int K, int block, void *packed, cudaStream_t s)
{
    F4Order::Call call;
    if (!g_f4_order.begin(s, packed, call)) return TMAN_ERR_CUDA;
    tman_status st;
    if (dtype == kF4TypeHalf) st = block == 32 ? launch_quantize_as<32, __half>(x, ldx, rows, K, packed, s) : launch_quantize_as<16, __half>(x, ldx, rows, K, packed, s);
    else st = block == 32 ? launch_quantize_as<32, __nv_bfloat16>(x, ldx, rows, K, packed, s) : launch_quantize_as<16, __nv_bfloat16>(x, ldx, rows, K, packed, s);
    g_f4_order.end(call, st == TMAN_OK);
    return st;
}

// ---- dequantization -----------------------------------------------------------------------------
// The same groups and lanes: a warp reads a unit's 1024 bytes of eight rows and writes 64 bytes of each row at a time.
template <int BLOCK, typename T>
__global__ void __launch_bounds__(32 * kRowsWarps) f4_dequant_kernel(const uint8_t *packed, int rows, int K, T *x, int ldx, const __grid_constant__ F4Layout L, int parts,
                                                                     uint32_t *status)
{
    grid_wait();
    grid_launch_next();                  // (see f4_read_ahead)
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, r = lane >> 2, q = lane & 3;
    const int part = blockIdx.x % parts, g = blockIdx.x / parts, row = g * 8 + r, u = part * kRowsWarps + warp;      // unit
    const int chunks = min(8, L.halves * 4 - u * 8);
    if (chunks <= 0) return;
    const uint32_t *codes = reinterpret_cast<const uint32_t *>(packed + L.codes_off + (size_t)u * L.height8 * 128 + (size_t)g * (chunks * 128)) + lane;
    const uint32_t *scales = reinterpret_cast<const uint32_t *>(packed + L.scales_off + f4_scale_at(min(row, rows - 1), u * (2 * kF4Half / BLOCK), BLOCK, L));
    constexpr int WORDS = BLOCK == 32 ? 2 : 4;                   // of scales of a unit, 512 bytes apart
    uint32_t c[8], w[WORDS];
#pragma unroll
    for (int i = 0; i < 8; ++i) c[i] = i < chunks ? codes[i * 32] : 0u;
#pragma unroll
    for (int i = 0; i < WORDS; ++i) w[i] = i < chunks * WORDS / 8 ? scales[i * 128] : 0u;
    const float rs = BLOCK == 16 ? reinterpret_cast<const float *>(packed + L.rows_off)[min(row, rows - 1)] : 1.f;
    if (!f4_header_matches(packed, rows, K, BLOCK)) {
        if (blockIdx.x == 0 && threadIdx.x == 0) atomicCAS(status, 0u, (uint32_t)TMAN_ERR_BAD_PACKED);
        return;
    }
    if (row >= rows) return;
    T *out = x + (size_t)row * ldx + u * (2 * kF4Half) + q * 8;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int k = u * (2 * kF4Half) + i * 32 + q * 8;
        if (k >= K) break;
        const uint32_t byte = BLOCK == 32 ? w[i >> 2] >> (8 * (i & 3)) & 0xFFu : w[i >> 1] >> (16 * (i & 1) + 8 * (q >> 1)) & 0xFFu;
        const float s = f4_scale_value<BLOCK>(byte) * rs;
        uint32_t o[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float2 p = __half22float2(f4_pair(c[i] >> (8 * e)));
            o[e] = f4_from_float2<T>(p.x * s, p.y * s);
        }
        *reinterpret_cast<uint4 *>(out + i * 32) = make_uint4(o[0], o[1], o[2], o[3]);
    }
}

template <int BLOCK, typename T>
static tman_status launch_dequant_as(const void *packed, int rows, int K, void *x, int ldx, uint32_t *status, cudaStream_t s)
{
    const F4Layout L = f4_layout(rows, K, BLOCK);
    const int parts = ((L.halves + 1) / 2 + kRowsWarps - 1) / kRowsWarps;
    return launch_rows(f4_dequant_kernel<BLOCK, T>, (long long)(L.height8 / 8) * parts, 32 * kRowsWarps, s, static_cast<const uint8_t *>(packed), rows, K, static_cast<T *>(x), ldx, L, parts, status);
}

tman_status launch_f4_dequant(const void *packed, int rows, int K, int block, void *x, int ldx, int dtype, uint32_t *status, cudaStream_t s)
{
    if (dtype == kF4TypeHalf) return block == 32 ? launch_dequant_as<32, __half>(packed, rows, K, x, ldx, status, s) : launch_dequant_as<16, __half>(packed, rows, K, x, ldx, status, s);
    return block == 32 ? launch_dequant_as<32, __nv_bfloat16>(packed, rows, K, x, ldx, status, s) : launch_dequant_as<16, __nv_bfloat16>(packed, rows, K, x, ldx, status, s);
}

}  // namespace tman
