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
#include "ssd_paged.h"

namespace ssd {

struct PagedAttnArgs {
    PagedGeom g;
    const char *q, *k_pages, *v_pages;
    const char *k_new, *v_new;   // step: the newest row, from here instead of the pool
    char *k_dst, *v_dst;
    int32_t *pos;
    const float *weight_in;
    float *weight_out;
    char *out;
    float *lse;
    float *z;                 // logits (base 2) [n_seqs, n_heads, z_stride]; LATER only (see Weights)
    float *lse2;              // [n_seqs, n_heads] lse (base 2) of units that one workgroup completed; LATER only
    float *part_o;            // [2 * workgroups, heads of a tile, D] sums of a unit's part, relative to its maximum
    uint2 *parts;             // [n_seqs, n_kv, q_tiles] where a unit's first part lies, how many workgroups share it; only where rows are dealt
    float2 *part_ml;          // [2 * workgroups, heads of a tile] its maximum (base 2) and sum
    int64_t q_stride, new_stride;   // bytes
    int64_t z_stride;         // rows, a multiple of a round
    int n_heads, group, q_tiles;
    int tile_heads;           // min(group, 16)
    int workgroups;           // 0: a workgroup takes a whole unit
    int by_length;            // then: the longest sequences first
    int stage;                // rows whose part of the block table is in LDS at a time: a multiple of a round
    uint32_t page_magic, single;   // ceil(2^32 / page_size) and 0, or 0 and 1 where that is 2^32
    float scale;              // softmax scale * log2 e
};

// entries of the block table that a workgroup has in LDS
static constexpr int blocks_of(int waves) { return 256 * waves; }
static constexpr int HEADS = 16;                                   // heads of a tile
static constexpr int64_t NO_PAGE = -(1ll << 62);
static constexpr float LN2 = 0.6931471805599453f;

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef f32x4 f32x4_any __attribute__((aligned(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

// block of a row: x / page_size for x < 2^16 (a chunk's rows and what lies before them in its first page), page_size <= 2^15:
// the rounded-up reciprocal is exact while x * page_size < 2^32.  For pages of one row it is 0 and `single` 1.
static __device__ __forceinline__ int block_of(const PagedAttnArgs &a, int x) {
    return (int)(__umulhi((uint32_t)x, a.page_magic) + __umul24((uint32_t)x, a.single));
}

// Where a lane finds its rows of a tile.  K: rows lane % 16 (and + 16); V and the logits: rows 4 g .. 4 g + 3 (and + 16), g = lane / 16.
// Rows that do not exist (past the end, or of a block without a page) get an address all the same -- the pool's first row -- and a zero
// bit in `there`.
template <bool BF16, bool QUADS> struct TileRows {
    static constexpr int SUB = BF16 ? 2 : 1;                       // groups of 16 rows
    static constexpr int NV = QUADS ? SUB : 4 * SUB;
    int64_t k[SUB];
    int64_t v[NV];                                                 // QUADS: four rows of a page from here on
    uint32_t there;                                                // bit 4 t + i: row 16 t + 4 g + i
};

// One row's byte offset in the pool, negative if it does not exist.  x: row of the chunk.
static __device__ __forceinline__ int64_t row_at(const PagedAttnArgs &a, const int64_t *pages, int lead, int rows, int x) {
    const int y = (x < rows ? x : rows - 1) + lead;
    const int block = block_of(a, y), place = y - block * a.g.page_size;
    return pages[block] + (int64_t)place * a.g.row_stride;         // a block without a page: NO_PAGE, far below zero
}

template <bool BF16, bool QUADS>
static __device__ __forceinline__ void find_k(const PagedAttnArgs &a, const int64_t *pages, int lead, int rows, int first, int lane,
                                              TileRows<BF16, QUADS> &t) {
#pragma unroll
    for (int s = 0; s < TileRows<BF16, QUADS>::SUB; ++s) {
        const int64_t k = row_at(a, pages, lead, rows, first + 16 * s + (lane & 15));
        t.k[s] = k < 0 ? 0 : k;
    }
}

template <bool BF16, bool QUADS>
static __device__ __forceinline__ void find_v(const PagedAttnArgs &a, const int64_t *pages, int lead, int rows, int first, int lane,
                                              TileRows<BF16, QUADS> &t) {
    t.there = 0;
#pragma unroll
    for (int s = 0; s < TileRows<BF16, QUADS>::SUB; ++s) {
        const int x = first + 16 * s + 4 * (lane >> 4);
        if constexpr (QUADS) {                                     // the chunk's first row and the page size are multiples of four
            const int64_t v = row_at(a, pages, lead, rows, x < rows ? x : (rows - 1) & ~3);
            t.v[s] = v < 0 ? 0 : v;
            const int left = v < 0 ? 0 : rows - x;
#pragma unroll
            for (int i = 0; i < 4; ++i) t.there |= i < left ? 1u << (4 * s + i) : 0u;
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int64_t v = row_at(a, pages, lead, rows, x + i);
                t.v[4 * s + i] = v < 0 ? 0 : v;
                t.there |= v >= 0 && x + i < rows ? 1u << (4 * s + i) : 0u;
            }
        }
    }
}

// Makes an address wait for a result, for the compiler: requests that it moves up across the products that still read the registers they
// are to fill need a second set of them, which then goes to scratch memory (attn over 290000 rows 0.2 -> 0.54 ms).
static __device__ __forceinline__ void after(int64_t &address, float result) { asm volatile("" : "+v"(address) : "v"(result)); }

// ---- a tile's operands and products, by element type --------------------------------------------------------------

template <typename T, int D> struct Tile;

template <int D> struct Tile<bf16_t, D> {
    static constexpr bool BF16 = true;
    static constexpr int ROWS = 32, STEPS = D / 32;                // STEPS: 64-byte pieces of a row of K
    static constexpr int VB = D / 8;                               // bytes of a row of V in a lane: 16 or 8
    static constexpr int NV = D / 16;                              // tiles of V^T P
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

template <int D> struct Tile<float, D> {
    static constexpr bool BF16 = false;
    static constexpr int ROWS = 16, STEPS = D / 16;
    static constexpr int HALVES = D / 64, NV = D / 16;
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

template <typename T> static __device__ __forceinline__ void store_out(char *out, int64_t i, float x) {
    if constexpr (sizeof(T) == 4) reinterpret_cast<float *>(out)[i] = x;
    else reinterpret_cast<uint16_t *>(out)[i] = (uint16_t)f32_to_bf16_bits(x);
}

// ---- who works on what -------------------------------------------------------------------------------------------------
//
// A unit is a (sequence, key / value head, tile of query heads); its rows are counted in rounds of WAVES tiles.  All units' rounds, in the order
// sequence, head, row, are dealt to the workgroups in runs of equal cost, so that the chip is evenly loaded whatever the lengths are: a
// workgroup finishes one unit, goes through some and begins another.  The lengths are known on the device only; every wave adds them
// up for itself, 64 sequences (or runs of them) at a time, and finds its place by a ballot.  A unit in more than one workgroup leaves parts
// for the second launch; a workgroup leaves at most two, the one it begins with and the one it ends with.  Who has a unit's first round notes where
// its parts are.

static __device__ __forceinline__ int rounds_of(int n, int round) { return n == 0 ? 1 : (n + round - 1) / round; }

// What a unit costs besides its rounds, in rounds: its queries, its part of the block table and the meeting of its waves, 4 us against 3 to 6 for a
// round (128 sequences of 10 to 8000 rows with weights: counted as none 98 us, as one round 88, two 89, three 91; 48 of up to 5000, fp32: 39.8, 38.5, 39.6,
// 40.8; one of 5000 rows 14.1 and 15.2).
static constexpr int EXTRA = 1;
static __device__ __forceinline__ uint32_t cost_of(int n, int round) { return (uint32_t)rounds_of(n, round) + EXTRA; }

static __device__ __forceinline__ uint32_t uniform(uint32_t v) { return (uint32_t)__builtin_amdgcn_readfirstlane((int)v); }

// The runs: a cost of `all` over at most `most` workgroups, none below two where there are 256 workgroups without.
struct Runs {
    uint32_t q, rem;
    __device__ __forceinline__ Runs(uint32_t q_, uint32_t rem_) : q(q_), rem(rem_) {}
    static __device__ __forceinline__ Runs of(uint32_t all, uint32_t most) {
        uint32_t w = all / 2 > 256 ? all / 2 : 256;
        w = w < most ? w : most;
        w = w < all ? w : all;
        return Runs(all / w, all % w);
    }
    __device__ __forceinline__ uint32_t start(uint32_t w) const { return w * q + (w < rem ? w : rem); }
    __device__ __forceinline__ uint32_t owner(uint32_t r) const {
        const uint32_t longer = rem * (q + 1);
        return r < longer ? r / (q + 1) : rem + (r - longer) / q;
    }
};

// Rows j .. j + 3 (j < n, a multiple of four) in the tables: where they are, negative past n and where no page is named, and their weights so far.
struct Entries {
    int64_t at[4];
    float w[4];
};
// page(block): the block's page, or a negative number
template <bool QUADS, typename Page>
static __device__ __forceinline__ Entries entries_of(const PagedAttnArgs &a, int kv, int j, int n, const Page &page) {
    Entries x;
    int block, place;
    split_slot(a.g, j, block, place);
    if constexpr (QUADS) {                                         // four places of one page
        const int p = page(block);
        const int64_t i = table_index(a.g, p < 0 ? 0 : p, kv, place);
        const f32x4 w = *reinterpret_cast<const f32x4_any *>(a.weight_in + i);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            x.at[e] = p >= 0 && j + e < n ? i + e : -1;
            x.w[e] = w[e];
        }
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int p = j + e < n ? page(block) : -1;
            x.at[e] = p < 0 ? -1 : table_index(a.g, p, kv, place);
            x.w[e] = a.weight_in[p < 0 ? 0 : x.at[e]];
            if (++place == a.g.page_size) {
                place = 0;
                ++block;
            }
        }
    }
    return x;
}

// p: what is added; newest: the row without a weight so far, or -1.
template <bool QUADS> static __device__ __forceinline__ void add_weights(const PagedAttnArgs &a, int j, int n, Entries x, const f32x4 &p, int newest) {
#pragma unroll
    for (int e = 0; e < 4; ++e) x.w[e] = (j + e == newest ? 0.f : x.w[e]) + p[e];
    if (QUADS && j + 4 <= n) {
        if (x.at[0] >= 0) *reinterpret_cast<f32x4_any *>(a.weight_out + x.at[0]) = f32x4{x.w[0], x.w[1], x.w[2], x.w[3]};
        return;
    }
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if (x.at[e] >= 0) a.weight_out[x.at[e]] = x.w[e];
}

// Four rows' probabilities, summed over heads; z: the first head's logits of theirs, the others' `stride` apart.
template <typename I> static __device__ __forceinline__ f32x4 probabilities(const float *z, I stride, const float *lse2, int heads) {
    f32x4 p = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 8
    for (int h = 0; h < heads; ++h) {
        const f32x4 x = *reinterpret_cast<const f32x4 *>(z + h * stride);
#pragma unroll
        for (int e = 0; e < 4; ++e) p[e] += fast_exp2(x[e] - lse2[h]);
    }
    return p;
}

// The arguments, to be read from their segment again: what one phase of the kernel needs of them does not have to stay in scalar
// registers through the others (there are too few: they would be kept in vector registers' lanes, and those in scratch memory).
static __device__ __forceinline__ const PagedAttnArgs &arguments() {
    typedef const PagedAttnArgs __attribute__((address_space(4))) *args_t;
    args_t p = (args_t)__builtin_amdgcn_kernarg_segment_ptr();
    asm volatile("" : "+s"(p));
    return *(const PagedAttnArgs *)p;
}

// The sequence of rank `rank` by length, the longest first, equal ones in their order; n_seqs <= 64 * PER.  Every lane has PER lengths; the length
// of that rank is found bit by bit from ballots.
template <int PER> static __device__ __forceinline__ int by_length(const PagedAttnArgs &a, int rank, int lane) {
    int len[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) len[i] = 64 * i + lane < a.g.n_seqs ? clamp_len(a.g, 64 * i + lane) : -1;
    int t = 0, above = 0;                                           // the length so far, sequences that are longer
    for (int bit = 1 << (31 - __clz(a.g.max_len)); bit; bit >>= 1) {
        int c = 0;
#pragma unroll
        for (int i = 0; i < PER; ++i) c += (int)__popcll(__ballot((len[i] & ~(bit - 1)) == (t | bit)));
        if (above + c > rank) t |= bit;
        else above += c;
    }
    int left = rank - above;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const unsigned long long m = __ballot(len[i] == t);
        const int c = (int)__popcll(m);
        if (left < c) return 64 * i + kth_set_bit(m, 0, left);
        left -= c;
    }
    return 0;
}

// What becomes of a tile's logits: nothing more, or they wait for the softmax's sum, in memory for the second launch or in LDS for the end of this one.
enum Weights { NONE, LATER, HERE };

// grid = (workgroups), or (kv heads * tiles of query heads, sequences) where a workgroup takes a whole unit
template <typename T, int D, bool QUADS, bool STEP, Weights WEIGHTS, int WAVES>
__global__ __launch_bounds__(64 * WAVES, 3) void paged_attn_kernel(PagedAttnArgs) {
    typedef Tile<T, D> TT;
    constexpr int NZ = TT::ROWS / 4;                                // logits of a lane
    constexpr int ROUND = WAVES * TT::ROWS;
    constexpr int LD = D + 4;                                       // row of the merge area
    __shared__ int64_t pages[blocks_of(WAVES)];
    __shared__ float sm_ml[WAVES][HEADS][2];
    __shared__ float sm_lse[HEADS];
    __shared__ uint32_t sm_runs[2];
    __shared__ int32_t page_ids[WEIGHTS == HERE ? blocks_of(WAVES) : 1];
    extern __shared__ __align__(16) float sm_o[];                   // [WAVES][tile_heads][LD], then (HERE) logits [tile_heads][z_stride + 4]

    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, r = lane & 15, g = lane >> 4;
    int b, n, ht, t;                                                // sequence, its rows, head tile, round of the unit
    uint32_t left;                                                  // rounds of the run
    {
    const PagedAttnArgs &a = arguments();
    const uint32_t K = (uint32_t)(a.g.n_kv * a.q_tiles);
    if (a.workgroups == 0) {
        int rank = (int)blockIdx.y;
        if constexpr (WEIGHTS == HERE) unit_of(a.g, ht, rank);
        else ht = (int)((blockIdx.x + blockIdx.y) % K);
        b = a.by_length ? by_length<2>(a, rank, lane) : rank;
        t = 0;
        n = clamp_len(a.g, b);
        left = (uint32_t)rounds_of(n, ROUND);
    } else {
        uint32_t before = 0, r0;                                    // rounds of one head of the sequences before b; first of the run
        if (a.g.n_seqs <= 256) {                                    // every lane has four lengths, and nothing is read twice
            int len[4];
            uint32_t mine = 0;
#pragma unroll
            for (int i = 0; i < 4; ++i) len[i] = a.g.seq_len[64 * i + lane < a.g.n_seqs ? 64 * i + lane : a.g.n_seqs - 1];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                len[i] = len[i] < 0 ? 0 : len[i] > a.g.max_len ? a.g.max_len : len[i];
                mine += 64 * i + lane < a.g.n_seqs ? cost_of(len[i], ROUND) : 0u;
            }
            const uint32_t all = uniform(wave_sum(mine)) * K;
            const Runs runs = Runs::of(all, (uint32_t)a.workgroups);
            r0 = runs.start(blockIdx.x);
            const uint32_t r1 = runs.start(blockIdx.x + 1);
            if (r0 >= r1 || r0 >= all) return;
            left = r1 - r0;
            if (threadIdx.x == 0) {
                sm_runs[0] = runs.q;
                sm_runs[1] = runs.rem;
            }
            const uint32_t at = r0 / K;                             // in rounds of one head
            b = -1;
            n = 0;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (b >= 0 || 64 * i >= a.g.n_seqs) continue;
                const uint32_t up = wave_scan(64 * i + lane < a.g.n_seqs ? cost_of(len[i], ROUND) : 0u) + before;
                const int k = (int)__popcll(__ballot(up <= at));
                if (k < 64) {
                    b = 64 * i + k;
                    n = __builtin_amdgcn_readlane(len[i], k);
                }
                before = k > 0 ? (uint32_t)__builtin_amdgcn_readlane((int)up, k - 1) : before;
            }
        } else {
            const int run = (a.g.n_seqs + 63) / 64;                 // sequences of a lane
            uint32_t mine = 0;
            for (int i = 0; i < run; ++i) {
                const int seq = lane * run + i;
                if (seq < a.g.n_seqs) mine += cost_of(clamp_len(a.g, seq), ROUND);
            }
            const uint32_t upto = wave_scan(mine);
            const uint32_t all = (uint32_t)__builtin_amdgcn_readlane((int)upto, 63) * K;
            const Runs runs = Runs::of(all, (uint32_t)a.workgroups);
            r0 = runs.start(blockIdx.x);
            const uint32_t r1 = runs.start(blockIdx.x + 1);
            if (r0 >= r1 || r0 >= all) return;
            left = r1 - r0;
            if (threadIdx.x == 0) {
                sm_runs[0] = runs.q;
                sm_runs[1] = runs.rem;
            }
            const uint32_t at = r0 / K;
            const int l = (int)__popcll(__ballot(upto <= at));
            before = l == 0 ? 0 : (uint32_t)__builtin_amdgcn_readlane((int)upto, l - 1);
            b = l * run;
            for (int i0 = 0;; i0 += 64) {                           // the run's sequences, 64 at a time
                const int seq = l * run + i0 + lane;
                const bool ours = i0 + lane < run && seq < a.g.n_seqs;
                const uint32_t up = wave_scan(ours ? cost_of(clamp_len(a.g, seq), ROUND) : 0u) + before;
                const int k = (int)__popcll(__ballot(up <= at));
                if (k < 64) {
                    b = l * run + i0 + k;
                    if (k > 0) before = (uint32_t)__builtin_amdgcn_readlane((int)up, k - 1);
                    break;
                }
                before = (uint32_t)__builtin_amdgcn_readlane((int)up, 63);
            }
            n = clamp_len(a.g, b);
        }
        const uint32_t tb = uniform(cost_of(n, ROUND)), into = r0 - before * K;
        ht = (int)(into / tb);
        t = (int)(into - (uint32_t)ht * tb) - EXTRA;
        if (t < 0) {                                                // the run begins with what the unit costs besides
            if (left <= (uint32_t)-t) return;
            left -= (uint32_t)-t;
            t = 0;
        }
    }
    }
    b = (int)uniform((uint32_t)b);
    ht = (int)uniform((uint32_t)ht);
    t = (int)uniform((uint32_t)t);
    left = uniform(left);
    n = (int)uniform((uint32_t)n);

    for (bool first_unit = true;; first_unit = false) {
        const PagedAttnArgs &a = arguments();
        const int kv = ht / a.q_tiles, qt = ht - kv * a.q_tiles;
        const int heads = a.group - qt * HEADS < HEADS ? a.group - qt * HEADS : HEADS, head0 = kv * a.group + qt * HEADS;
        const int rounds = rounds_of(n, ROUND);
        const int take = (uint32_t)(rounds - t) < left ? rounds - t : (int)left;
        const int begin = t * ROUND, end = begin + take * ROUND < n ? begin + take * ROUND : n;
        const bool whole = take == rounds;                          // this workgroup writes the outputs
        const bool newest = STEP && end == n && n > 0 && a.g.seq_len[b] == n;      // the row of this call is among them
        const char *k_new = nullptr, *v_new = nullptr;
        if (STEP && newest) {
            k_new = a.k_new + (int64_t)b * a.new_stride + (int64_t)kv * (D * sizeof(T));
            v_new = a.v_new + (int64_t)b * a.new_stride + (int64_t)kv * (D * sizeof(T));
        }
        typename TT::Q q;
        TT::load_q(a.q + (int64_t)b * a.q_stride + (int64_t)(head0 + (r < heads ? r : 0)) * (D * sizeof(T)), lane, q);
        // the unit's logits; lanes without a head are out of the buffer's bounds, and what they store is dropped
        __amdgpu_buffer_rsrc_t z_unit;
        uint32_t z_lane = 0;
        if constexpr (WEIGHTS == LATER) {
            float *at = a.z + ((int64_t)b * a.n_heads + head0) * a.z_stride;
            z_unit = __builtin_amdgcn_make_buffer_rsrc(at, 0, (int)(4u * (uint32_t)heads * (uint32_t)a.z_stride), 0x00027000);
            z_lane = r < heads ? 4u * ((uint32_t)r * (uint32_t)a.z_stride + 4u * (uint32_t)g) : 0x80000000u;
        }

        float m = NEG_BIG, l = 0.f;
        f32x4 o[TT::NV];
#pragma unroll
        for (int j = 0; j < TT::NV; ++j) o[j] = f32x4{0.f, 0.f, 0.f, 0.f};

        for (int row0 = begin; row0 < end;) {
            const PagedAttnArgs &a = arguments();
            const int rows = end - row0 < a.stage ? end - row0 : a.stage;
            int block0, lead;
            split_slot(a.g, row0, block0, lead);
            const int blocks = block_of(a, rows - 1 + lead) + 1;
            __syncthreads();                                        // the last stage's entries, and a unit's merge area, have been read
            for (int i = threadIdx.x; i < blocks; i += 64 * WAVES) {
                const int page = page_of(a.g, b, block0 + i);
                if constexpr (WEIGHTS == HERE) page_ids[i] = page;
                pages[i] = page < 0 ? NO_PAGE : (int64_t)page * a.g.page_stride + (int64_t)kv * a.g.head_stride;
            }
            __syncthreads();
            const int last_row = newest && row0 + rows == n ? rows - 1 : 0x7fffffff;

            TT tl;
            TileRows<TT::BF16, QUADS> at;
            auto request_k = [&](int first) {
#pragma unroll
                for (int s = 0; s < at.SUB; ++s) {
                    const char *row = a.k_pages + at.k[s];
                    if (STEP && first + 16 * s + r >= last_row) row = k_new;
                    tl.load_k(s, row, lane);
                }
            };
            auto request_v = [&](int first) {
#pragma unroll
                for (int i = 0; i < NZ; ++i) {
                    const char *row = a.v_pages + (QUADS ? at.v[i / 4] + (i % 4) * a.g.row_stride : at.v[i]);
                    if (STEP && first + 16 * (i / 4) + 4 * g + i % 4 >= last_row) row = v_new;
                    tl.load_v(i, row, lane);
                }
            };
            // One tile: its products and softmax step.  LAST: no tile follows.  Outside the last one every request is made without a condition,
            // or the compiler would wait for all that is in flight wherever it waits for anything.
            auto tile = [&](int first, auto last) {
                constexpr bool LAST = decltype(last)::value;
                const int next = first + ROUND;
                float z[NZ];
                tl.logits(q, z);
                const uint32_t there = at.there;
                if constexpr (!LAST) {
                    find_k(a, pages, lead, rows, next, lane, at);
#pragma unroll
                    for (int s = 0; s < at.SUB; ++s) after(at.k[s], z[NZ - 1]);
                    request_k(next);
                }
#pragma unroll
                for (int e = 0; e < NZ; ++e) z[e] *= a.scale;
                if constexpr (WEIGHTS == HERE) {
                    if (r < heads)
#pragma unroll
                        for (int e = 0; e < NZ; e += 4)
                            *reinterpret_cast<f32x4 *>(sm_o + WAVES * heads * LD + r * ((int)a.z_stride + 4) + row0 + first + 4 * e + 4 * g) =
                                f32x4{z[e], z[e + 1], z[e + 2], z[e + 3]};
                }
                if constexpr (WEIGHTS == LATER)
#pragma unroll
                    for (int e = 0; e < NZ; e += 4)
                        __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4_nt_t, f32x4{z[e], z[e + 1], z[e + 2], z[e + 3]}), z_unit,
                                                               (int)(z_lane + 4u * (uint32_t)(row0 + first + 4 * e)), 0, 0);
                const bool all = __all(there == (1u << NZ) - 1u);
                if (!all) {
#pragma unroll
                    for (int e = 0; e < NZ; ++e) z[e] = there >> e & 1 ? z[e] : NEG_BIG;
                }
                float top = m;
#pragma unroll
                for (int e = 0; e < NZ; ++e) top = fmaxf(top, z[e]);
                {
                    float x, y;
                    rows_pair(top, x, y);
                    top = fmaxf(x, y);
                    halves_pair(top, x, y);
                    top = fmaxf(x, y);
                }
                if (__any(top > m)) {                               // a larger logit: what is summed so far shrinks
                    const float f = fast_exp2(m - top);
                    l *= f;
#pragma unroll
                    for (int j = 0; j < TT::NV; ++j) o[j] *= f;
                    m = top;
                }
                float p[NZ];
#pragma unroll
                for (int e = 0; e < NZ; ++e) p[e] = fast_exp2(z[e] - m);
                if (!all) {                                         // rows that do not exist: neither their p nor their V may count
#pragma unroll
                    for (int e = 0; e < NZ; ++e)
                        if (!(there >> e & 1)) {
                            p[e] = 0.f;
                            tl.zero_v(e);
                        }
                }
#pragma unroll
                for (int e = 0; e < NZ; ++e) l += p[e];
                tl.accumulate(p, o);
                if constexpr (!LAST) {
                    find_v(a, pages, lead, rows, next, lane, at);
#pragma unroll
                    for (int i = 0; i < at.NV; ++i) after(at.v[i], o[TT::NV - 1][0]);
                    request_v(next);
                    asm volatile("" ::: "memory");                  // or the requests would move to the loop's head, behind K's
                }
            };
            const int tiles = (rows + TT::ROWS - 1) / TT::ROWS;
            if (wave < tiles) {
                int first = wave * TT::ROWS;
                find_k(a, pages, lead, rows, first, lane, at);
                request_k(first);
                find_v(a, pages, lead, rows, first, lane, at);
                request_v(first);
                asm volatile("" ::: "memory");
#pragma unroll 1
                for (int i = wave; i + WAVES < tiles; i += WAVES, first += ROUND) tile(first, std::false_type{});
                tile(first, std::true_type{});
            }
            row0 += rows;
        }

        {
        const PagedAttnArgs &a = arguments();
        // the newest row goes where it belongs
        if (STEP && newest && qt == 0 && wave == 0) {
            int block, place;
            split_slot(a.g, n - 1, block, place);
            const int page = page_of(a.g, b, block);
            if (page >= 0) {
                constexpr int FR = D * (int)sizeof(T) / 16;
                if (lane < 2 * FR) {
                    const bool v = lane >= FR;
                    const int sub = (v ? lane - FR : lane) * 16;
                    *reinterpret_cast<uint4 *>((v ? a.v_dst : a.k_dst) + row_offset(a.g, page, kv, place) + sub) =
                        *reinterpret_cast<const uint4 *>((v ? v_new : k_new) + sub);
                }
                if (lane == 0 && a.pos) a.pos[table_index(a.g, page, kv, place)] = a.g.seq_pos[b] - 1;
            }
        }

        // HERE: a thread's four rows (a unit has no more of them than the workgroup has threads), their weights so far on their way while the waves meet
        const int j = 4 * (int)threadIdx.x;
        Entries entries;
        if constexpr (WEIGHTS == HERE)
            if (j < n) entries = entries_of<QUADS>(a, kv, j, n, [&](int block) { return page_ids[block]; });
        // the waves' states meet
        {
            float x, y;
            rows_pair(l, x, y);
            l = x + y;
            halves_pair(l, x, y);
            l = x + y;
        }
        if (!first_unit) __syncthreads();                           // a unit without rows passes no other barrier
        const int active = end - begin > (WAVES - 1) * TT::ROWS ? WAVES : end - begin > TT::ROWS ? (end - begin + TT::ROWS - 1) / TT::ROWS : 1;
        if (r < heads && wave < active) {                           // the others have had no tile
            if (g == 0) {
                sm_ml[wave][r][0] = m;
                sm_ml[wave][r][1] = l;
            }
            float *dst = sm_o + (wave * heads + r) * LD;
#pragma unroll
            for (int j = 0; j < TT::NV; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) dst[TT::column(j, e, lane)] = o[j][e];
        }
        __syncthreads();
        const int64_t slot = 2 * (int64_t)blockIdx.x + (first_unit ? 0 : 1);
        for (int i = threadIdx.x; i < heads * D; i += 64 * WAVES) {
            const int h = i / D, d = i % D;
            float top = sm_ml[0][h][0], sum = 0.f, acc = 0.f;
#pragma unroll
            for (int w = 1; w < WAVES; ++w)
                if (w < active) top = fmaxf(top, sm_ml[w][h][0]);
#pragma unroll
            for (int w = 0; w < WAVES; ++w) {
                if (w >= active) break;
                const float f = fast_exp2(sm_ml[w][h][0] - top);
                sum = fmaf(sm_ml[w][h][1], f, sum);
                acc = fmaf(sm_o[(w * heads + h) * LD + d], f, acc);
            }
            const int64_t bh = (int64_t)b * a.n_heads + head0 + h;
            if (whole) {
                store_out<T>(a.out, bh * D + d, sum == 0.f ? 0.f : acc / sum);
                if (d == 0) {
                    const float lse = top + __builtin_amdgcn_logf(sum);
                    if (a.lse) a.lse[bh] = sum == 0.f ? -INFINITY : lse * LN2;
                    if (WEIGHTS == LATER) a.lse2[bh] = sum == 0.f ? INFINITY : lse;
                    if (WEIGHTS == HERE) sm_lse[h] = sum == 0.f ? INFINITY : lse;
                }
            } else {
                a.part_o[(slot * a.tile_heads + h) * D + d] = acc;
                if (d == 0) a.part_ml[slot * a.tile_heads + h] = make_float2(top, sum);
            }
        }
        if constexpr (WEIGHTS == HERE) {
            __syncthreads();
            if (j < n)
                add_weights<QUADS>(a, j, n, entries, probabilities(sm_o + WAVES * heads * LD + j, (int)a.z_stride + 4, sm_lse, heads), newest ? n - 1 : -1);
            return;
        }
        if (a.workgroups && t == 0 && threadIdx.x == 0) {           // where the parts of a unit lie is told by who has its first round
            uint32_t count = 1;
            if (!whole) {
                const Runs runs{sm_runs[0], sm_runs[1]};
                count = runs.owner(runs.start(blockIdx.x + 1) + (uint32_t)(rounds - take) - 1) - blockIdx.x + 1;
            }
            a.parts[(int64_t)b * (a.g.n_kv * a.q_tiles) + ht] = make_uint2((uint32_t)slot, count);
        }
        left -= (uint32_t)take;
        if (left <= EXTRA) return;
        left -= EXTRA;
        t = 0;
        if (++ht == a.g.n_kv * a.q_tiles) {
            ht = 0;
            ++b;
            n = clamp_len(a.g, b);
        }
        }
        __syncthreads();
    }
}

// Maximum over the lanes of a wave.
static __device__ __forceinline__ float wave_max(float v) {
    v = fmaxf(v, dpp_f<0xB1>(v));
    v = fmaxf(v, dpp_f<0x4E>(v));
    v = fmaxf(v, dpp_f<0x141>(v));
    v = fmaxf(v, dpp_f<0x140>(v));
    return across_groups_max<16>(v);
}

// What the first launch leaves open: joins the parts of units that several workgroups share (blockIdx.z < head_blocks; a query head takes a
// wave, or the whole workgroup where WIDE), and brings the rows' weights up to date (the workgroups beyond, 1024 rows at a time).
// grid = (kv heads, sequences, head_blocks + a few)
template <typename T, int D, bool QUADS, bool WIDE>
__global__ __launch_bounds__(256) void paged_join_kernel(PagedAttnArgs a, int step, int head_blocks) {
    constexpr int FR = D / 4, PW = 64 / FR, NW = WIDE ? 4 : 1;      // 16-byte pieces of a part's sums; parts a wave reads side by side; waves
    __shared__ float red[2][4];
    __shared__ f32x4 sums[4][FR];
    __shared__ float2 ml_lds[4][HEADS];
    extern __shared__ float lse2[];                                 // [group]
    const int kv = blockIdx.x, b = blockIdx.y, tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int n = clamp_len(a.g, b);
    // the workgroups that share a unit, and where the first one's part lies
    struct Parts { uint32_t slot0, count; };
    auto parts_of = [&](int tile) {
        if (a.workgroups == 0) return Parts{0, 1};
        const uint2 p = a.parts[((int64_t)b * a.g.n_kv + kv) * a.q_tiles + tile];
        return Parts{uniform(p.x), uniform(p.y)};
    };
    auto slot = [&](const Parts &p, uint32_t c) { return (int64_t)(c == 0 ? p.slot0 : (p.slot0 & ~1u) + 2 * c) * a.tile_heads; };

    if ((int)blockIdx.z < head_blocks) {
        const int head = WIDE ? (int)blockIdx.z : (int)blockIdx.z * 4 + wave, w = WIDE ? wave : 0;
        if (head >= a.group) return;
        const int h = head % HEADS;
        const Parts p = parts_of(head / HEADS);
        if (p.count == 1) return;
        const int64_t bh = (int64_t)b * a.n_heads + kv * a.group + head;
        float top = NEG_BIG, sum = 0.f;
        for (uint32_t c = w * 64 + lane; c < p.count; c += 64 * NW) top = fmaxf(top, a.part_ml[slot(p, c) + h].x);
        top = wave_max(top);
        if constexpr (WIDE) {
            if (lane == 0) red[0][w] = top;
            __syncthreads();
            top = fmaxf(fmaxf(red[0][0], red[0][1]), fmaxf(red[0][2], red[0][3]));
        }
        f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
        for (uint32_t c = w * PW + lane / FR; c < p.count; c += PW * NW) {
            const int64_t at = slot(p, c) + h;
            const float2 x = a.part_ml[at];
            const float f = fast_exp2(x.x - top);
            sum = fmaf(x.y, f, sum);
            acc += f * *reinterpret_cast<const f32x4 *>(a.part_o + at * D + 4 * (lane % FR));
        }
        if constexpr (PW == 4) {
            sum = across_groups_sum<16>(sum);
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[e] = across_groups_sum<16>(acc[e]);
        } else {
            float x, y;
            halves_pair(sum, x, y);
            sum = x + y;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                halves_pair(acc[e], x, y);
                acc[e] = x + y;
            }
        }
        if constexpr (WIDE) {
            if (lane == 0) red[1][w] = sum;
            if (lane < FR) sums[w][lane] = acc;
            __syncthreads();
            if (w > 0) return;
            sum = (red[1][0] + red[1][1]) + (red[1][2] + red[1][3]);
            acc = (sums[0][lane % FR] + sums[1][lane % FR]) + (sums[2][lane % FR] + sums[3][lane % FR]);
        }
        if (lane < FR)
#pragma unroll
            for (int e = 0; e < 4; ++e) store_out<T>(a.out, bh * D + 4 * lane + e, sum == 0.f ? 0.f : acc[e] / sum);
        if (lane == 0 && a.lse) a.lse[bh] = sum == 0.f ? -INFINITY : (top + __builtin_amdgcn_logf(sum)) * LN2;
        return;
    }
    const int first = ((int)blockIdx.z - head_blocks) * 1024;
    if (first >= n) return;
    int j = first + 4 * tid;                                       // the tables' entries are on their way while the lse are found
    Entries entries;
    const auto page = [&](int block) { return page_of(a.g, b, block); };
    if (j < n) entries = entries_of<QUADS>(a, kv, j, n, page);
    // the heads' lse: a lane takes a head of the tile and every sixteenth part
    for (int tile = 0; tile < a.q_tiles; ++tile) {
        const int h0 = tile * HEADS, h = lane & 15, heads = a.group - h0 < HEADS ? a.group - h0 : HEADS;
        const Parts p = parts_of(tile);
        if (p.count == 1) {
            if (tid < heads) lse2[h0 + tid] = a.lse2[(int64_t)b * a.n_heads + kv * a.group + h0 + tid];
            continue;
        }
        float top = NEG_BIG, sum = 0.f;
#pragma unroll 4
        for (uint32_t c = tid >> 4; c < p.count; c += 16) {
            const float2 x = a.part_ml[slot(p, c) + (h < heads ? h : 0)];
            const float up = fmaxf(top, x.x);
            sum = sum * fast_exp2(top - up) + x.y * fast_exp2(x.x - up);
            top = up;
        }
        const float most = across_groups_max<16>(top);
        sum = across_groups_sum<16>(sum * fast_exp2(top - most));
        __syncthreads();
        if (lane < 16) ml_lds[wave][h] = make_float2(most, sum);
        __syncthreads();
        if (tid < heads) {
            top = fmaxf(fmaxf(ml_lds[0][tid].x, ml_lds[1][tid].x), fmaxf(ml_lds[2][tid].x, ml_lds[3][tid].x));
            sum = 0.f;
#pragma unroll
            for (int i = 0; i < 4; ++i) sum += ml_lds[i][tid].y * fast_exp2(ml_lds[i][tid].x - top);
            lse2[h0 + tid] = sum == 0.f ? INFINITY : top + __builtin_amdgcn_logf(sum);
        }
    }
    __syncthreads();
    const int newest = step && a.g.seq_len[b] == n ? n - 1 : -1;
    const float *z0 = a.z + ((int64_t)b * a.n_heads + kv * a.group) * a.z_stride;
    while (j < n) {
        add_weights<QUADS>(a, j, n, entries, probabilities(z0 + j, a.z_stride, lse2, a.group), newest);
        j += ((int)gridDim.z - head_blocks) * 1024;
        if (j < n) entries = entries_of<QUADS>(a, kv, j, n, page);
    }
}

// ---- launch shapes ---------------------------------------------------------------------------------------------------

struct PagedShape {
    int waves, round, q_tiles, tile_heads, workgroups, stage;
    bool by_length, here;     // here: a unit's weights are brought up to date by its own workgroup, from logits in LDS
    int64_t reach;            // rows, in whole rounds
    size_t lds;               // where the waves meet
};

static PagedShape paged_shape(const ssd_paged_config *c, int max_len) {
    PagedShape s;
    const int reach = paged_reach(c, max_len), group = c->n_heads / c->n_kv_heads;
    const int tile = c->dtype == SSD_BF16 ? 32 : 16;
    s.q_tiles = (group + HEADS - 1) / HEADS;
    s.tile_heads = group < HEADS ? group : HEADS;
    const int64_t units = (int64_t)c->n_seqs * c->n_kv_heads * s.q_tiles, rounds = (reach + 4 * tile - 1) / (4 * tile);
    s.reach = rounds * 4 * tile;
    // A unit of few rounds is taken whole: one launch instead of two (8 units of 400 rows 8.5 us whole and 11.0 dealt, 256 12.9 and 18.8, 128 of 640 13.9
    // and 16.7, 32 12.2 and 11.5); with more rounds only where units are many (256 of 1000 rows 24.5 and 28.6, of 10 to 1000 18.5 and 16.6, 1024 85 and 92, 38 and
    // 34; 128 of 1000 19.7 and 21.0, of 10 to 1000 17.7 and 13.3; 512 of 2048 84 and 91, of 10 to 2048 44 and 29; all with 16 key heads, two query heads each; weights
    // change little), and where 32 bits would not hold the sums.
    const bool plain = rounds <= 5 || (units >= 256 && rounds <= 8) || units * (rounds + EXTRA) >= 1ll << 31;
    // Very short units, many of them: a wave each (2048 of 128 rows 25.6 us and 29.0 with four waves, of 256 45 and 47; 512 of 128 10.3 and 9.3).
    s.waves = units >= 1024 && rounds <= 2 ? 1 : 4;
    s.round = s.waves * tile;
    // 256 compute units, four or three workgroups each; twice as many are no better (128 sequences of 10 to 8000 rows 67 and 69 us, with weights 87 and 87, of 1195 rows
    // 63.5 and 66.7; fp32 of 64 elements, 48 of up to 5000 rows, 37.4 and 39.8, with three each 38)
    const int64_t resident = c->head_dim == 64 ? 1024 : 768;
    s.workgroups = plain ? 0 : (int)(units * rounds < resident ? units * rounds : resident);
    // Where not all units are resident at once a late long one would run on alone; ranking costs every workgroup a microsecond (32 heads of 64 to 640
    // rows, 64 sequences 54 us in their order and 50 by length, 128 96 and 95, of 10 to 1000 rows 94 and 89; 256 168 and 173, 16 17.3 and 19.0).
    s.by_length = plain && s.waves == 4 && units > 1024 && c->n_seqs <= 128;
    // a stage's blocks: its rows and what lies before them in the first one; block_of allows 2^16 rows
    const int64_t most = (int64_t)(blocks_of(s.waves) - 1) * c->page_size;
    s.stage = (int)((most < 8192 ? most : 8192) / s.round * s.round);
    s.lds = (size_t)s.waves * s.tile_heads * (c->head_dim + 4) * sizeof(float);
    // The weights are brought up to date by the unit's own workgroup, from logits in LDS (up to 66 KB), where it takes one tile of heads (2 sequences of
    // 64 to 97 rows, 16 heads 6.5 us, by a second launch 10.2; 128 of 64 to 640 rows, 32 heads 100 and 103, 256 query heads on 32 111 and 130, on 16 with
    // up to 500 rows 89 and 103; 64 of 1000 rows, 32 heads 192 and 187).
    s.here = plain && s.q_tiles == 1 && s.reach <= s.stage && s.reach <= 256 * s.waves;
    return s;
}

struct PagedScratch { size_t z, lse2, o, ml, parts, all; };

static PagedScratch paged_scratch(const ssd_paged_config *c, const PagedShape &s, bool weights) {
    PagedScratch w;
    const size_t bh = (size_t)c->n_seqs * c->n_heads, parts = (size_t)2 * s.workgroups * s.tile_heads;
    w.z = weights && !s.here ? round256(bh * s.reach * sizeof(float)) : 0;
    w.lse2 = weights && !s.here ? round256(bh * sizeof(float)) : 0;
    w.o = round256(parts * c->head_dim * sizeof(float));
    w.ml = round256(parts * sizeof(float2));
    w.parts = s.workgroups ? round256((size_t)c->n_seqs * c->n_kv_heads * s.q_tiles * sizeof(uint2)) : 0;
    w.all = w.z + w.lse2 + w.o + w.ml + w.parts;
    return w;
}

template <typename T, int D, bool QUADS, int WAVES> static void launch_paged_rows(const PagedAttnArgs &a, const PagedShape &sh, bool step, hipStream_t s) {
    const bool weights = a.weight_out != nullptr;
    const dim3 wg(64 * WAVES), grid = sh.workgroups ? dim3((unsigned)sh.workgroups) : dim3((unsigned)(a.g.n_kv * sh.q_tiles), (unsigned)a.g.n_seqs);
    const auto go = [&](auto kernel, size_t lds) { hipLaunchKernelGGL(kernel, grid, wg, (unsigned)lds, s, a); };
    const size_t here = sh.lds + (size_t)a.tile_heads * (a.z_stride + 4) * sizeof(float);
    if (!weights) go(step ? paged_attn_kernel<T, D, QUADS, true, NONE, WAVES> : paged_attn_kernel<T, D, QUADS, false, NONE, WAVES>, sh.lds);
    else if (sh.here) go(step ? paged_attn_kernel<T, D, QUADS, true, HERE, WAVES> : paged_attn_kernel<T, D, QUADS, false, HERE, WAVES>, here);
    else go(step ? paged_attn_kernel<T, D, QUADS, true, LATER, WAVES> : paged_attn_kernel<T, D, QUADS, false, LATER, WAVES>, sh.lds);
}

template <typename T, int D, bool QUADS> static hipError_t launch_paged_attn(const PagedAttnArgs &a, const PagedShape &sh, bool step, hipStream_t s) {
    const bool weights = a.weight_out != nullptr;
    if (sh.waves == 1) launch_paged_rows<T, D, QUADS, 1>(a, sh, step, s);
    else launch_paged_rows<T, D, QUADS, 4>(a, sh, step, s);
    if (!sh.workgroups && (!weights || sh.here)) return hipGetLastError();
    const int64_t units = (int64_t)a.g.n_seqs * a.g.n_kv;
    const bool wide = units * a.group < 1024;
    const int head_blocks = !sh.workgroups ? 0 : wide ? a.group : (a.group + 3) / 4;
    int64_t pieces = weights ? (sh.reach + 1023) / 1024 : 0;
    const int64_t enough = 4096 / units + 1;
    if (pieces > enough) pieces = enough;
    const dim3 join((unsigned)a.g.n_kv, (unsigned)a.g.n_seqs, (unsigned)(head_blocks + pieces));
    const size_t lse = (size_t)a.group * sizeof(float);
    if (wide) hipLaunchKernelGGL((paged_join_kernel<T, D, QUADS, true>), join, dim3(256), lse, s, a, step ? 1 : 0, head_blocks);
    else hipLaunchKernelGGL((paged_join_kernel<T, D, QUADS, false>), join, dim3(256), lse, s, a, step ? 1 : 0, head_blocks);
    return hipGetLastError();
}

template <typename T, int D> static hipError_t launch_paged_attn(const PagedAttnArgs &a, const PagedShape &sh, bool step, hipStream_t s) {
    return a.g.page_size % 4 == 0 ? launch_paged_attn<T, D, true>(a, sh, step, s) : launch_paged_attn<T, D, false>(a, sh, step, s);
}

static int paged_attend(const ssd_paged_config *cfg, const void *q, const void *k_new, const void *v_new, void *k_pages, void *v_pages, int32_t *pos,
                        const float *weight_in, float *weight_out, const int32_t *block_table, const int32_t *seq_len, const int32_t *seq_pos,
                        void *out, float *lse, int max_len, void *workspace, size_t workspace_bytes, bool step, hipStream_t s) {
    clear_error();
    int rc = check_paged(cfg);
    if (rc != SSD_OK) return rc;
    if ((rc = check_max_len(cfg, max_len)) != SSD_OK) return rc;
    if (!q || !k_pages || !v_pages || !out) return fail(SSD_ERR_INVALID_ARG, "q, k_pages, v_pages or out is NULL");
    if (step && (!k_new || !v_new)) return fail(SSD_ERR_INVALID_ARG, "k_new or v_new is NULL");
    if (!aligned(q, 16) || !aligned(k_pages, 16) || !aligned(v_pages, 16) || !aligned(out, 16) || !aligned(k_new, 16) || !aligned(v_new, 16))
        return fail(SSD_ERR_INVALID_ARG, "q, k_new, v_new, k_pages, v_pages and out must be 16-byte aligned");
    if (!block_table || !seq_len) return fail(SSD_ERR_INVALID_ARG, "block_table or seq_len is NULL");
    if ((weight_in == nullptr) != (weight_out == nullptr)) return fail(SSD_ERR_INVALID_ARG, "weight_in and weight_out are given both or neither");
    if (!aligned(block_table, 4) || !aligned(seq_len, 4) || !aligned(seq_pos, 4) || !aligned(pos, 4) || !aligned(weight_in, 4) ||
        !aligned(weight_out, 4) || !aligned(lse, 4))
        return fail(SSD_ERR_INVALID_ARG, "tables must be aligned to their elements");
    const PagedShape shape = paged_shape(cfg, max_len);
    const PagedScratch parts = paged_scratch(cfg, shape, weight_out != nullptr);
    const size_t need = parts.all;
    if (need > 0 && (!workspace || !aligned(workspace, 256) || workspace_bytes < need))
        return fail(SSD_ERR_INVALID_ARG, "workspace of %zu bytes, 256-byte aligned, needed; %zu given", need, workspace_bytes);
    PagedAttnArgs a;
    a.g = paged_geom(cfg, block_table, seq_len, seq_pos, max_len);
    a.q = static_cast<const char *>(q);
    a.k_pages = static_cast<const char *>(k_pages);
    a.v_pages = static_cast<const char *>(v_pages);
    a.weight_in = weight_in;
    a.weight_out = weight_out;
    a.out = static_cast<char *>(out);
    a.lse = lse;
    char *ws = static_cast<char *>(workspace);
    a.z = reinterpret_cast<float *>(ws);
    a.lse2 = reinterpret_cast<float *>(ws + parts.z);
    a.part_o = reinterpret_cast<float *>(ws + parts.z + parts.lse2);
    a.part_ml = reinterpret_cast<float2 *>(ws + parts.z + parts.lse2 + parts.o);
    a.parts = reinterpret_cast<uint2 *>(ws + parts.z + parts.lse2 + parts.o + parts.ml);
    a.k_new = static_cast<const char *>(k_new);
    a.v_new = static_cast<const char *>(v_new);
    a.k_dst = static_cast<char *>(k_pages);
    a.v_dst = static_cast<char *>(v_pages);
    a.pos = pos;
    a.new_stride = (cfg->new_stride ? cfg->new_stride : (int64_t)cfg->n_kv_heads * cfg->head_dim) * (int64_t)paged_esize(cfg);
    a.z_stride = shape.reach;
    a.q_tiles = shape.q_tiles;
    a.tile_heads = shape.tile_heads;
    a.workgroups = shape.workgroups;
    a.by_length = shape.by_length;
    a.stage = shape.stage;
    a.single = cfg->page_size == 1;
    a.page_magic = (uint32_t)((0xffffffffull + (unsigned)cfg->page_size) / (unsigned)cfg->page_size);
    a.q_stride = (cfg->q_stride ? cfg->q_stride : (int64_t)cfg->n_heads * cfg->head_dim) * (int64_t)paged_esize(cfg);
    a.n_heads = cfg->n_heads;
    a.group = cfg->n_heads / cfg->n_kv_heads;
    a.scale = LOG2E * (cfg->softmax_scale != 0.f ? cfg->softmax_scale : 1.f / sqrtf((float)cfg->head_dim));
    hipError_t e;
    if (cfg->dtype == SSD_BF16) e = cfg->head_dim == 128 ? launch_paged_attn<bf16_t, 128>(a, shape, step, s) : launch_paged_attn<bf16_t, 64>(a, shape, step, s);
    else e = cfg->head_dim == 128 ? launch_paged_attn<float, 128>(a, shape, step, s) : launch_paged_attn<float, 64>(a, shape, step, s);
    return e == hipSuccess ? SSD_OK : hip_fail(e, "paged attention launch");
}

}  // namespace ssd

using namespace ssd;

extern "C" size_t ssd_paged_workspace_bytes(const ssd_paged_config *cfg, int max_len, int with_weights) {
    clear_error();
    if (check_paged(cfg) != SSD_OK || check_max_len(cfg, max_len) != SSD_OK) return 0;
    return paged_scratch(cfg, paged_shape(cfg, max_len), with_weights != 0).all;
}

extern "C" int ssd_paged_decode_attn(const ssd_paged_config *cfg, const void *q, const void *k_pages, const void *v_pages,
                                     const float *weight_in, float *weight_out, const int32_t *block_table, const int32_t *seq_len, void *out,
                                     float *lse, int max_len, void *workspace, size_t workspace_bytes, void *stream) {
    return paged_attend(cfg, q, nullptr, nullptr, const_cast<void *>(k_pages), const_cast<void *>(v_pages), nullptr, weight_in, weight_out,
                        block_table, seq_len, nullptr, out, lse, max_len, workspace, workspace_bytes, false, static_cast<hipStream_t>(stream));
}

extern "C" int ssd_paged_decode_step(const ssd_paged_config *cfg, const void *q, const void *k_new, const void *v_new, void *k_pages,
                                     void *v_pages, int32_t *pos, const float *weight_in, float *weight_out, const int32_t *block_table,
                                     const int32_t *seq_len, const int32_t *seq_pos, void *out, float *lse, int max_len, void *workspace,
                                     size_t workspace_bytes, void *stream) {
    return paged_attend(cfg, q, k_new, v_new, k_pages, v_pages, pos, weight_in, weight_out, block_table, seq_len, seq_pos, out, lse, max_len,
                        workspace, workspace_bytes, true, static_cast<hipStream_t>(stream));
}
