// ssd_paged_decode_attn, ssd_paged_decode_step: attention of one new token per sequence over the sequence's pages.
//
// What it computes, per (sequence, key / value head) and its G query heads:  s[j, h] = scale k[j].q[h],  p = softmax over j,
// o[h] = sum_j p[j, h] v[j],  and on request the probabilities, summed over the G heads, onto the rows' accumulated weights.
//
// What bounds it: the rows of K and V come from memory once, 4 G flops for every two or four bytes.  The vector units would
// keep up with G = 1 or 2 only; both products run on the matrix cores, with the heads padded to 16 (at G = 1 a sixteenth of their results
// is used, and they are still idle most of the time).
//
// How: a wave takes tiles of 32 rows (fp32: 16).  S = K Q^T has the rows of K as its first operand, so that a tile's logits lie
// with a head in the lane's place and eight rows in its registers (four); the same registers are the second operand of V^T P, if the rows of V
// are taken in the order the lanes hold them.  So the probabilities never leave their lane.  V^T's operand wants eight rows' elements of
// one column in a lane; a lane loads 16 bytes of each of its eight rows and transposes the 8 x 8 block in registers, 32 byte permutations for
// 16 KB of rows.  Maximum and sum of the softmax are kept in fp32 along the way (one pass), the sum by its lane until the end.
//
// K of the next tile is requested when the last product with K has read its registers, V when V's has: a wave has one of the two in
// flight at any time and the registers hold one tile, which lets three waves share a SIMD (four where rows have 64 elements).
//
// A workgroup's four waves take the tiles of its rows in turn and meet in LDS.  The rows' part of the block table is brought into LDS first, as
// byte offsets, so that no row's address waits for memory.  Who takes which rows stands at "who works on what"; units that more than one workgroup
// had a part of are joined by a second launch, which also brings their weights up to date, from logits that the first one left in memory.
//
// Measured (bf16, rows of 128; time of the call, share of the K and V bytes alone): 4 sequences of 30000 to 131072 rows, 32 query heads on 8: 184 to
// 192 us, 6.2 to 6.5 TB/s (a plain read reaches 6.1 to 7.0).  128 sequences of 64 to 640 rows, 32 heads: 92 to 95 us, 5.6 to 5.8 TB/s; with weights 99 to
// 102.  128 sequences of 10 to 8000 rows, 32 query heads on 4: 67 us, 4.8 TB/s; with weights and the new rows 87 -- the logits are 6 % of the bytes and,
// written among the reads, cost 16 us (batches of them in LDS, other orders in memory and the hints on the stores change nothing).
// fp32, rows of 64, 48 sequences of 0 to 5000 rows with weights: 37 us, 3.3 TB/s.
#include "ssd_paged_attn.h"

namespace ssd {

// Where a lane finds its rows of a tile.  K: rows lane % 16 (and + 16); V and the logits: rows 4 g .. 4 g + 3 (and + 16), g = lane / 16.
// Rows that do not exist (past the end, or of a block without a page) get an address all the same -- the pool's first row -- and a zero
// bit in `there`.
template <bool BF16, bool QUADS> struct TileRows {
    static constexpr int SUB = BF16 ? 2 : 1;                       // groups of 16 rows
    static constexpr int NV = QUADS ? SUB : 4 * SUB;
    int64_t k[SUB];
    int64_t v[NV];                                                 // QUADS: four rows of a page from here on
    uint32_t there;                                                // bit 4 t + i: row 16 t + 4 g + i

    struct Seen {
        uint32_t there;
        __device__ __forceinline__ bool all() const { return __all(there == (1u << 4 * SUB) - 1u); }
        __device__ __forceinline__ bool has(int e) const { return there >> e & 1; }
    };
    __device__ __forceinline__ Seen seen(int) const { return Seen{there}; }
};

// One row's byte offset in the pool, negative if it does not exist.  x: row of the chunk.
static __device__ __forceinline__ int64_t row_at(const PagedAttnArgs &a, const Stage &st, int x) {
    const int y = (x < st.rows ? x : st.rows - 1) + st.lead;
    const int block = block_of(a, y), place = y - block * a.g.page_size;
    return st.pages[block] + (int64_t)place * a.g.row_stride;      // a block without a page: NO_PAGE, far below zero
}

template <bool BF16, bool QUADS>
static __device__ __forceinline__ void find_k(const PagedAttnArgs &a, const Stage &st, int first, int lane, TileRows<BF16, QUADS> &t) {
#pragma unroll
    for (int s = 0; s < TileRows<BF16, QUADS>::SUB; ++s) {
        const int64_t k = row_at(a, st, first + 16 * s + (lane & 15));
        t.k[s] = k < 0 ? 0 : k;
    }
}

template <bool BF16, bool QUADS>
static __device__ __forceinline__ void find_v(const PagedAttnArgs &a, const Stage &st, int first, int lane, TileRows<BF16, QUADS> &t) {
    t.there = 0;
#pragma unroll
    for (int s = 0; s < TileRows<BF16, QUADS>::SUB; ++s) {
        const int x = first + 16 * s + 4 * (lane >> 4);
        if constexpr (QUADS) {                                     // the chunk's first row and the page size are multiples of four
            const int64_t v = row_at(a, st, x < st.rows ? x : (st.rows - 1) & ~3);
            t.v[s] = v < 0 ? 0 : v;
            const int left = v < 0 ? 0 : st.rows - x;
#pragma unroll
            for (int i = 0; i < 4; ++i) t.there |= i < left ? 1u << (4 * s + i) : 0u;
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int64_t v = row_at(a, st, x + i);
                t.v[4 * s + i] = v < 0 ? 0 : v;
                t.there |= v >= 0 && x + i < st.rows ? 1u << (4 * s + i) : 0u;
            }
        }
    }
}

// Makes an address wait for a result, for the compiler: requests that it moves up across the products that still read the registers they
// are to fill need a second set of them, which then goes to scratch memory (attn over 290000 rows 0.2 -> 0.54 ms).
static __device__ __forceinline__ void after(int64_t &address, float result) { asm volatile("" : "+v"(address) : "v"(result)); }
template <bool BF16, bool QUADS> static __device__ __forceinline__ void hold_k(TileRows<BF16, QUADS> &t, float result) {
#pragma unroll
    for (int s = 0; s < TileRows<BF16, QUADS>::SUB; ++s) after(t.k[s], result);
}
template <bool BF16, bool QUADS> static __device__ __forceinline__ void hold_v(TileRows<BF16, QUADS> &t, float result) {
#pragma unroll
    for (int i = 0; i < TileRows<BF16, QUADS>::NV; ++i) after(t.v[i], result);
}

// Requests of a tile's rows; a step's newest row (from last_row on) comes from where the call has it.
template <typename Step, bool BF16, bool QUADS, typename TT>
static __device__ __forceinline__ void request_k(Step, const PagedAttnArgs &a, const TileRows<BF16, QUADS> &at, TT &tl, int first, int last_row,
                                                 const char *k_new, int lane) {
#pragma unroll
    for (int s = 0; s < TileRows<BF16, QUADS>::SUB; ++s) {
        const char *row = a.k_pages + at.k[s];
        if (Step::value && first + 16 * s + (lane & 15) >= last_row) row = k_new;
        tl.load_k(s, row, lane);
    }
}
template <typename Step, bool BF16, bool QUADS, typename TT>
static __device__ __forceinline__ void request_v(Step, const PagedAttnArgs &a, const TileRows<BF16, QUADS> &at, TT &tl, int first, int last_row,
                                                 const char *v_new, int lane) {
#pragma unroll
    for (int i = 0; i < TT::ROWS / 4; ++i) {
        const char *row = a.v_pages + (QUADS ? at.v[i / 4] + (i % 4) * a.g.row_stride : at.v[i]);
        if (Step::value && first + 16 * (i / 4) + 4 * (lane >> 4) + i % 4 >= last_row) row = v_new;
        tl.load_v(i, row, lane);
    }
}

// ---- a tile's operands and products, by element type --------------------------------------------------------------

template <typename T, int D> struct Tile;

template <int D_> struct Tile<bf16_t, D_> {
    typedef bf16_t elem;
    static constexpr bool MX = false, TABLE = false;
    static constexpr int RESIDENT = 3, EXTRA = 1, ENTRIES = 0;
    typedef int entry_t;
    static __device__ __forceinline__ int head(int r) { return r; }
    static __device__ __forceinline__ bool writes(int) { return true; }
    template <bool QUADS> using Rows = TileRows<true, QUADS>;
    static constexpr int D = D_, ROWS = 32, STEPS = D / 32;                // STEPS: 64-byte pieces of a row of K
    static constexpr int VB = D / 8;                               // bytes of a row of V in a lane: 16 or 8
    static constexpr int NV = D / 16, NO = NV;                     // tiles of V^T P
    static __device__ __forceinline__ void finish(f32x4 (&)[NO]) {}
    typedef uint32_t vrow_t __attribute__((ext_vector_type(VB / 4)));
    u32x4_nt_t k[2][STEPS];
    vrow_t v[8];
    struct Q { bf16x8 x[STEPS]; };

    static __device__ __forceinline__ void load_q(const char *row, int lane, Q &q) {
#pragma unroll
        for (int s = 0; s < STEPS; ++s) q.x[s] = *reinterpret_cast<const bf16x8 *>(row + 64 * s + 16 * (lane >> 4));
    }
    __device__ __forceinline__ void load_k(int sub, const char *row, int lane) {
#pragma unroll
        for (int s = 0; s < STEPS; ++s)
            k[sub][s] = __builtin_nontemporal_load(reinterpret_cast<const u32x4_nt_t *>(row + 64 * s + 16 * (lane >> 4)));
    }
    __device__ __forceinline__ void load_v(int i, const char *row, int lane) {
        v[i] = __builtin_nontemporal_load(reinterpret_cast<const vrow_t *>(row + VB * (lane & 15)));
    }
    __device__ __forceinline__ void zero_v(int i) { v[i] = vrow_t(0); }
    __device__ __forceinline__ void logits(const Q &q, float (&z)[8]) const {
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            f32x4 c = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int s = 0; s < STEPS; ++s) c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, k[t][s]), q.x[s], c, 0, 0, 0);
#pragma unroll
            for (int i = 0; i < 4; ++i) z[4 * t + i] = c[i];
        }
    }
    // o[j] += column d = NV m + j of V, times p.  The probabilities go in as a bf16 and what it leaves out as another: 15 bits of each or more,
    // for the sum as good as fp32, at eight products more that the matrix cores have time for.  Both terms have to be above zero where p is, or an infinite
    // element of V would give 0 * inf or inf - inf: so the first is rounded from a 256th less than p, and leaves out 2^-15 to 2^-7 of it.  That holds
    // for p down to 2^-100; the second has to be a normal number.
    __device__ __forceinline__ void accumulate(const float (&p)[8], f32x4 (&o)[NV]) const {
        bf16x8 hi, lo;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            hi[i] = (__bf16)(p[i] * (1.f - 0x1p-8f));
            lo[i] = (__bf16)(p[i] - (float)hi[i]);
        }
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            uint32_t w[4];
#pragma unroll
            for (int e = 0; e < 4; ++e)
                w[e] = __builtin_amdgcn_perm(v[2 * e + 1][j / 2], v[2 * e][j / 2], j & 1 ? 0x07060302u : 0x05040100u);
            const bf16x8 col = __builtin_bit_cast(bf16x8, *reinterpret_cast<u32x4_nt_t *>(w));
            o[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(col, hi, o[j], 0, 0, 0);
            o[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(col, lo, o[j], 0, 0, 0);
        }
    }
    // column of o[j][i] in lane
    static __device__ __forceinline__ int column(int j, int i, int lane) { return NV * (4 * (lane >> 4) + i) + j; }
};

template <int D_> struct Tile<float, D_> {
    typedef float elem;
    static constexpr bool MX = false, TABLE = false;
    static constexpr int RESIDENT = 3, EXTRA = 1, ENTRIES = 0;
    typedef int entry_t;
    static __device__ __forceinline__ int head(int r) { return r; }
    static __device__ __forceinline__ bool writes(int) { return true; }
    template <bool QUADS> using Rows = TileRows<false, QUADS>;
    static constexpr int D = D_, ROWS = 16, STEPS = D / 16;
    static constexpr int HALVES = D / 64, NV = D / 16, NO = NV;
    static __device__ __forceinline__ void finish(f32x4 (&)[NO]) {}
    u32x4_nt_t k[1][STEPS];
    u32x4_nt_t v[4][HALVES];
    struct Q { f32x4 x[STEPS]; };

    static __device__ __forceinline__ void load_q(const char *row, int lane, Q &q) {
#pragma unroll
        for (int s = 0; s < STEPS; ++s) q.x[s] = *reinterpret_cast<const f32x4 *>(row + 64 * s + 16 * (lane >> 4));
    }
    __device__ __forceinline__ void load_k(int sub, const char *row, int lane) {
#pragma unroll
        for (int s = 0; s < STEPS; ++s)
            k[sub][s] = __builtin_nontemporal_load(reinterpret_cast<const u32x4_nt_t *>(row + 64 * s + 16 * (lane >> 4)));
    }
    __device__ __forceinline__ void load_v(int i, const char *row, int lane) {
#pragma unroll
        for (int h = 0; h < HALVES; ++h) v[i][h] = __builtin_nontemporal_load(reinterpret_cast<const u32x4_nt_t *>(row + 256 * h + 16 * (lane & 15)));
    }
    __device__ __forceinline__ void zero_v(int i) {
#pragma unroll
        for (int h = 0; h < HALVES; ++h) v[i][h] = u32x4_nt_t(0);
    }
    __device__ __forceinline__ void logits(const Q &q, float (&z)[4]) const {
        f32x4 c = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int s = 0; s < STEPS; ++s)
#pragma unroll
            for (int e = 0; e < 4; ++e) c = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(k[0][s][e]), q.x[s][e], c, 0, 0, 0);
#pragma unroll
        for (int i = 0; i < 4; ++i) z[i] = c[i];
    }
    __device__ __forceinline__ void accumulate(const float (&p)[4], f32x4 (&o)[NV]) const {
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < NV; ++j) o[j] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(v[i][j / 4][j % 4]), p[i], o[j], 0, 0, 0);
    }
    static __device__ __forceinline__ int column(int j, int i, int lane) { return 64 * (j / 4) + 4 * (4 * (lane >> 4) + i) + j % 4; }
};

template <typename T, int D> static hipError_t launch_tiles(const PagedAttnArgs &a, const PagedShape &sh, bool step, hipStream_t s) {
    return a.g.page_size % 4 == 0 ? launch_paged_attn<Tile<T, D>, true>(a, sh, step, s) : launch_paged_attn<Tile<T, D>, false>(a, sh, step, s);
}

static TileShape tile_shape(const ssd_paged_config *c) { return {c->dtype == SSD_BF16 ? 32 : 16, c->head_dim == 64 ? 1024 : 768, 0}; }

static int paged_attend(const AttendCall &c, hipStream_t s) {
    clear_error();
    int rc = check_paged(c.cfg);
    if (rc != SSD_OK) return rc;
    PagedAttnArgs a;
    PagedShape shape;
    if ((rc = attend_args(c, tile_shape(c.cfg), 8 * (int)paged_esize(c.cfg), a, shape)) != SSD_OK) return rc;
    hipError_t e;
    if (c.cfg->dtype == SSD_BF16) e = c.cfg->head_dim == 128 ? launch_tiles<bf16_t, 128>(a, shape, c.step, s) : launch_tiles<bf16_t, 64>(a, shape, c.step, s);
    else e = c.cfg->head_dim == 128 ? launch_tiles<float, 128>(a, shape, c.step, s) : launch_tiles<float, 64>(a, shape, c.step, s);
    return e == hipSuccess ? SSD_OK : hip_fail(e, "paged attention launch");
}

}  // namespace ssd

using namespace ssd;

extern "C" size_t ssd_paged_workspace_bytes(const ssd_paged_config *cfg, int max_len, int with_weights) {
    clear_error();
    if (check_paged(cfg) != SSD_OK || check_max_len(cfg, max_len) != SSD_OK) return 0;
    return paged_scratch(cfg, paged_shape(cfg, max_len, tile_shape(cfg)), with_weights != 0).all;
}

extern "C" int ssd_paged_decode_attn(const ssd_paged_config *cfg, const void *q, const void *k_pages, const void *v_pages,
                                     const float *weight_in, float *weight_out, const int32_t *block_table, const int32_t *seq_len, void *out,
                                     float *lse, int max_len, void *workspace, size_t workspace_bytes, void *stream) {
    return paged_attend({cfg, q, nullptr, nullptr, const_cast<void *>(k_pages), const_cast<void *>(v_pages), nullptr, weight_in, weight_out, block_table, seq_len,
                         nullptr, out, lse, max_len, workspace, workspace_bytes, false},
                        static_cast<hipStream_t>(stream));
}

extern "C" int ssd_paged_decode_step(const ssd_paged_config *cfg, const void *q, const void *k_new, const void *v_new, void *k_pages,
                                     void *v_pages, int32_t *pos, const float *weight_in, float *weight_out, const int32_t *block_table,
                                     const int32_t *seq_len, const int32_t *seq_pos, void *out, float *lse, int max_len, void *workspace,
                                     size_t workspace_bytes, void *stream) {
    return paged_attend({cfg, q, k_new, v_new, k_pages, v_pages, pos, weight_in, weight_out, block_table, seq_len, seq_pos, out, lse, max_len, workspace,
                         workspace_bytes, true},
                        static_cast<hipStream_t>(stream));
}
