// A paged cache of keys and values in 8 bits.
//
// A page holds `page` consecutive tokens (16, 32, 64 or 128) of one sequence; for every key head it has codes of keys, codes of values, and one
// scale for each: a key or value is code x scale, codes in [-127, 127].
//   codes    [pages][heads][2: keys, values][page / 16] tiles of 16 tokens x width bytes
//   scales   fp32 [pages][heads][2], behind the codes padded to 256 bytes
// A tile is laid out as the attention's warps take it: 16-byte pieces, piece i of lane l at (32 i + l) * 16, so that a warp's loads are whole
// lines and a lane's bytes are its operands of mma.sync.m16n8k16, without an exchange.  With lane l = 4 g + t:
//   keys     piece 2 p + h: token 8 h + g, columns 64 p + 16 t .. + 15
//   values   piece j / 4, bytes 4 (j % 4) ..: column 8 j + g of tokens 2t, 2t + 1, 2t + 8, 2t + 9
#pragma once

#include "i8.cuh"

namespace tman {

// What all sequences' calls have in common.
struct CacheSeqs {
    uint8_t *cache;
    const int *table, *lens, *starts;    // pages of sequence s: table[s * ldt ..]; its rows: starts[s] .. starts[s + 1] - 1 (NULL: row s)
    uint32_t *status;
    size_t scales_off;
    int pages, page_sh, heads, width, ldt, S, T;
};

inline size_t cache_scales_off(int pages, int page, int heads, int width) { return up256((size_t)pages * heads * 2 * page * width); }
inline size_t cache_bytes(int pages, int page, int heads, int width) { return cache_scales_off(pages, page, heads, width) + (size_t)pages * heads * 8; }

constexpr int kAttendRows = 16;          // rows of a tile
inline size_t attend_slot_bytes(int width) { return (size_t)kAttendRows * (width + 4) * 4; }
inline size_t attend_workspace_bytes(int width) { return kI8ScratchOff + 2 * kAttendCtas * attend_slot_bytes(width); }

tman_status launch_append_i8(const CacheSeqs &c, const void *k, int ldk, const void *v, int ldv, int dtype, cudaStream_t s);
tman_status launch_read_cache_i8(const CacheSeqs &c, void *k, int ldk, void *v, int ldv, int dtype, cudaStream_t s);
tman_status launch_attend_i8(const CacheSeqs &c, const void *q, int ldq, void *y, int ldy, int dtype, int q_heads, float scale, int window, void *ws,
                             cudaStream_t s);
tman_status launch_norm_rotate(const void *x, int ldx, void *y, int ldy, int dtype, int T, int q_heads, int k_heads, int width, int rot, int adjacent,
                               const void *q_weight, const void *k_weight, float eps, const int *positions, const float *inv_freq, cudaStream_t s);

#ifdef __CUDACC__
__device__ __forceinline__ int ld_dependent(const int *p)
{
    int v;
    asm volatile("ld.global.s32 %0, [%1];" : "=r"(v) : "l"(p) : "memory");
    return v;
}

// Byte of (token, column) in a tile.
__device__ __forceinline__ uint32_t cache_key_at(int token, int column)
{
    return (uint32_t)((((column >> 6) * 2 + (token >> 3)) * 32 + (token & 7) * 4 + ((column >> 4) & 3)) * 16 + (column & 15));
}
__device__ __forceinline__ uint32_t cache_value_at(int token, int column)
{
    return (uint32_t)(((column >> 5) * 32 + (column & 7) * 4 + ((token & 7) >> 1)) * 16 + ((column >> 3) & 3) * 4 + (token >> 3) * 2 + (token & 1));
}

// Rows of sequence s, its tokens.  A sequence whose numbers cannot be (rows outside of [0, T), more tokens than its table has pages for, a
// negative length) has no rows, and the status word says so.
struct CacheSeq { int row, rows, len; };
__device__ __forceinline__ CacheSeq cache_seq(const CacheSeqs &c, int s)
{
    CacheSeq q;
    q.row = c.starts ? ld_dependent(c.starts + s) : s;
    q.rows = c.starts ? ld_dependent(c.starts + s + 1) - q.row : 1;
    q.len = ld_dependent(c.lens + s);
    if (q.row < 0 || q.rows < 0 || q.row > c.T - q.rows || q.len < 0 || q.len > (long long)c.ldt << c.page_sh) {
        atomicCAS(c.status, 0u, (uint32_t)TMAN_ERR_INDEX);
        q.rows = 0;
    }
    return q;
}
// Page `i` of sequence s; -1, and the status word says so, where the table holds none of the cache's.
__device__ __forceinline__ int cache_page(const CacheSeqs &c, int s, int i)
{
    const int id = ld_dependent(c.table + (size_t)s * c.ldt + i);
    if ((unsigned)id < (unsigned)c.pages) return id;
    atomicCAS(c.status, 0u, (uint32_t)TMAN_ERR_INDEX);
    return -1;
}
#endif

}  // namespace tman
