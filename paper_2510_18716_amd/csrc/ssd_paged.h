// What the kernels of the paged cache share: the pool as they see it, slot to address, and the checks of a config.
#pragma once

#include "ssd_device.h"

namespace ssd {

// Everything a kernel needs to find a row.  Strides in bytes.
struct PagedGeom {
    int64_t page_stride, head_stride, row_stride;
    const int32_t *block_table;
    const int32_t *seq_len;
    const int32_t *seq_pos;          // may be seq_len
    int32_t n_seqs, n_kv, page_size, n_pages, max_blocks;
    int32_t max_len;                 // min(caller's bound, max_blocks * page_size)
    int32_t page_log2;               // log2 of page_size, or -1 where it is no power of two
    int32_t share;                   // log2 of the heads whose entries of a page share a cache line of the tables
};

static __device__ __forceinline__ int clamp_len(const PagedGeom &g, int b) {
    const int n = g.seq_len[b];
    return n < 0 ? 0 : n > g.max_len ? g.max_len : n;
}

// Block and place of a slot, by a shift where the page size allows it.
static __device__ __forceinline__ void split_slot(const PagedGeom &g, int slot, int &block, int &place) {
    if (g.page_log2 >= 0) {
        block = slot >> g.page_log2;
        place = slot & (g.page_size - 1);
    } else {
        block = (int)((unsigned)slot / (unsigned)g.page_size);
        place = slot - block * g.page_size;
    }
}

// The page a slot lies in, or -1 where the table names none.  slot < max_blocks * page_size.
static __device__ __forceinline__ int page_of(const PagedGeom &g, int b, int block) {
    const int p = g.block_table[(size_t)b * (size_t)g.max_blocks + (size_t)block];
    return (unsigned)p < (unsigned)g.n_pages ? p : -1;
}
static __device__ __forceinline__ int64_t row_offset(const PagedGeom &g, int page, int kv, int place) {
    return (int64_t)page * g.page_stride + (int64_t)kv * g.head_stride + (int64_t)place * g.row_stride;
}
static __device__ __forceinline__ int64_t table_index(const PagedGeom &g, int page, int kv, int place) {
    return ((int64_t)page * g.n_kv + kv) * g.page_size + place;
}

// The sequence and key head of a workgroup of a grid (heads, sequences).  Workgroups go to the eight XCDs in turn.  Where a page's entries of one
// head are less than a cache line, the heads that share one go to the same XCD, or two would read and write every line of the tables (one eviction from each
// of 256 units of 8000 rows in pages of 16 28.7 -> 20.3 us, of 16000 105 -> 64, in pages of one row 186 -> 83; 32 unequal prompts 45.1 -> 45.9; attention with
// weights over 4096 units of 640 rows 250 -> 237; the second launch of the attention gains nothing).
static __device__ __forceinline__ void unit_of(const PagedGeom &g, int &kv, int &b) {
    kv = blockIdx.x;
    b = blockIdx.y;
    if (g.share == 0) return;
    const unsigned heads = (unsigned)g.n_kv, i = blockIdx.y * heads + blockIdx.x, round = 8u << g.share;
    if (i < (unsigned)g.n_seqs * heads / round * round) {
        const unsigned unit = ((i / round * 8 + (i & 7)) << g.share) + (i >> 3 & ((1u << g.share) - 1));
        b = (int)(unit / heads);
        kv = (int)(unit - (unsigned)b * heads);
    }
}

// Inclusive sum over the lanes of a wave: rows of 16 by shifts, then the last lane of a row to the rows behind it.
template <int CTRL, int ROWS> static __device__ __forceinline__ uint32_t dpp_add(uint32_t v) {
    return v + (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, ROWS, 0xF, false);
}
static __device__ __forceinline__ uint32_t wave_scan(uint32_t v) {
    v = dpp_add<0x111, 0xF>(v);
    v = dpp_add<0x112, 0xF>(v);
    v = dpp_add<0x114, 0xF>(v);
    v = dpp_add<0x118, 0xF>(v);
    v = dpp_add<0x142, 0xA>(v);
    return dpp_add<0x143, 0xC>(v);
}
static __device__ __forceinline__ uint32_t wave_sum(uint32_t v) { return (uint32_t)__builtin_amdgcn_readlane((int)wave_scan(v), 63); }
// Or over the lanes of a wave, the same way (bits may come in twice).
template <int CTRL, int ROWS> static __device__ __forceinline__ uint32_t dpp_or(uint32_t v) {
    return v | (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, ROWS, 0xF, false);
}
static __device__ __forceinline__ uint32_t wave_or(uint32_t v) {
    v = dpp_or<0x111, 0xF>(v);
    v = dpp_or<0x112, 0xF>(v);
    v = dpp_or<0x114, 0xF>(v);
    v = dpp_or<0x118, 0xF>(v);
    v = dpp_or<0x142, 0xA>(v);
    return (uint32_t)__builtin_amdgcn_readlane((int)dpp_or<0x143, 0xC>(v), 63);
}

// Checks of the config (with the error text set), then the geometry; max_len <= 0 selects the table's reach.
int check_paged(const ssd_paged_config *c);
PagedGeom paged_geom(const ssd_paged_config *c, const int32_t *block_table, const int32_t *seq_len, const int32_t *seq_pos, int max_len);
int check_max_len(const ssd_paged_config *c, int max_len);
static inline int paged_reach(const ssd_paged_config *c, int max_len) {
    const int64_t all = (int64_t)c->max_blocks * c->page_size;
    return max_len > 0 && max_len < all ? max_len : (int)all;
}
static inline size_t paged_esize(const ssd_paged_config *c) { return c->dtype == SSD_F32 ? 4 : 2; }
static inline size_t round256(size_t n) { return (n + 255) / 256 * 256; }

}  // namespace ssd
