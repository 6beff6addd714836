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
// flight at any time and the registers hold one tile, which lets three waves share a SIMD.
//
// A workgroup of four waves takes a piece ("chunk") of a sequence; its waves take the chunk's tiles in turn and meet in LDS.  Where a sequence can
// be longer than a chunk a second launch joins the chunks; otherwise the workgroup writes the outputs.  The chunk's part of the block table
// is brought into LDS once, as byte offsets, so that no row's address waits for memory.
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
    float *z;                 // logits (base 2) [n_seqs, n_heads, z_stride]; only where weights are wanted
    float *part_o;            // [n_seqs, n_heads, n_split, D] sums of a chunk, relative to its maximum
    float2 *part_ml;          // [n_seqs, n_heads, n_split] maximum (base 2) and sum of a chunk
    int64_t q_stride, new_stride;   // bytes
    int64_t z_stride;         // rows, a multiple of the chunk
    int n_heads, group, q_tiles;
    int chunk, n_split;
    uint32_t page_magic, single;   // ceil(2^32 / page_size) and 0, or 0 and 1 where that is 2^32
    float scale;              // softmax scale * log2 e
};

static constexpr int WAVES = 4;
static constexpr int CHUNK_MAX = 1024;
static constexpr int HEADS = 16;                                   // heads of a tile
static constexpr int64_t NO_PAGE = -(1ll << 62);
static constexpr float LN2 = 0.6931471805599453f;

typedef float f32x4 __attribute__((ext_vector_type(4)));
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
    // o[j] += column d = NV m + j of V, times p.  The probabilities go in as a bf16 and what it leaves out as another: 16 bits of each, as
    // good as fp32 for the sum, at eight products more that the matrix cores have time for.
    __device__ __forceinline__ void accumulate(const float (&p)[8], f32x4 (&o)[NV]) const {
        bf16x8 hi, lo;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            hi[i] = (__bf16)p[i];
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

// Which piece a workgroup takes.
struct Piece { int b, chunk, head_tile; };
static __device__ __forceinline__ Piece piece_of() {
    const unsigned z = blockIdx.z;
    return {(int)((blockIdx.y + z) % gridDim.y), (int)z, (int)((blockIdx.x + z) % gridDim.x)};
}

template <typename T, int D, bool QUADS, bool STEP, bool WEIGHTS>
__global__ __launch_bounds__(64 * WAVES, 3) void paged_attn_kernel(PagedAttnArgs a) {
    typedef Tile<T, D> TT;
    constexpr int NZ = TT::ROWS / 4;                                // logits of a lane
    constexpr int LD = D + 4;                                       // row of the merge area
    __shared__ int64_t pages[CHUNK_MAX + 1];
    __shared__ float sm_ml[WAVES][HEADS][2];
    __shared__ float sm_lse[HEADS];
    extern __shared__ float sm_o[];                                 // [WAVES][heads][LD]

    const Piece pc = piece_of();
    const int b = pc.b, kv = pc.head_tile / a.q_tiles, qt = pc.head_tile - kv * a.q_tiles;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, r = lane & 15, g = lane >> 4;
    const int n = clamp_len(a.g, b);
    const int row0 = pc.chunk * a.chunk;
    const int heads = a.group - qt * HEADS < HEADS ? a.group - qt * HEADS : HEADS, head0 = kv * a.group + qt * HEADS;
    const bool whole = n <= a.chunk && a.q_tiles == 1;              // this workgroup writes the outputs
    if (row0 >= n) {
        if (n == 0 && row0 == 0 && whole) {                         // a sequence without rows
            for (int i = threadIdx.x; i < heads * D; i += 64 * WAVES) store_out<T>(a.out, ((int64_t)b * a.n_heads + head0) * D + i, 0.f);
            if (a.lse && (int)threadIdx.x < heads) a.lse[(int64_t)b * a.n_heads + head0 + threadIdx.x] = -INFINITY;
        }
        return;
    }
    const int rows = n - row0 < a.chunk ? n - row0 : a.chunk;
    int block0, lead;
    split_slot(a.g, row0, block0, lead);
    const int blocks = block_of(a, rows - 1 + lead) + 1;
    for (int i = threadIdx.x; i < blocks; i += 64 * WAVES) {
        const int page = page_of(a.g, b, block0 + i);
        pages[i] = page < 0 ? NO_PAGE : (int64_t)page * a.g.page_stride + (int64_t)kv * a.g.head_stride;
    }
    typename TT::Q q;
    TT::load_q(a.q + (int64_t)b * a.q_stride + (int64_t)(head0 + (r < heads ? r : 0)) * (D * sizeof(T)), lane, q);
    __syncthreads();

    // step: the sequence's last row, if it lies here
    const bool newest = STEP && a.g.seq_len[b] == n && row0 + rows == n;
    const char *k_new = nullptr, *v_new = nullptr;
    if (STEP && newest) {
        k_new = a.k_new + (int64_t)b * a.new_stride + (int64_t)kv * (D * sizeof(T));
        v_new = a.v_new + (int64_t)b * a.new_stride + (int64_t)kv * (D * sizeof(T));
    }
    const char *kp = a.k_pages, *vp = a.v_pages;

    float m = NEG_BIG, l = 0.f;
    f32x4 o[TT::NV];
#pragma unroll
    for (int j = 0; j < TT::NV; ++j) o[j] = f32x4{0.f, 0.f, 0.f, 0.f};

    TT t;
    TileRows<TT::BF16, QUADS> at;
    auto request_k = [&](int first) {
#pragma unroll
        for (int s = 0; s < at.SUB; ++s) {
            const char *row = kp + at.k[s];
            if (STEP && newest && first + 16 * s + r >= rows - 1) row = k_new;
            t.load_k(s, row, lane);
        }
    };
    auto request_v = [&](int first) {
#pragma unroll
        for (int i = 0; i < NZ; ++i) {
            const char *row = vp + (QUADS ? at.v[i / 4] + (i % 4) * a.g.row_stride : at.v[i]);
            if (STEP && newest && first + 16 * (i / 4) + 4 * g + i % 4 >= rows - 1) row = v_new;
            t.load_v(i, row, lane);
        }
    };
    const int tiles = (rows + TT::ROWS - 1) / TT::ROWS;
    float *zrow = WEIGHTS ? a.z + ((int64_t)b * a.n_heads + head0 + (r < heads ? r : 0)) * a.z_stride + row0 : nullptr;
    // One tile: its products and softmax step.  LAST: no tile follows.  Outside the last one every request is made without a condition, or
    // the compiler would wait for all that is in flight wherever it waits for anything.
    auto tile = [&](int first, auto last) {
        constexpr bool LAST = decltype(last)::value;
        const int next = first + WAVES * TT::ROWS;
        float z[NZ];
        t.logits(q, z);
        const uint32_t there = at.there;
        if constexpr (!LAST) {
            find_k(a, pages, lead, rows, next, lane, at);
#pragma unroll
            for (int s = 0; s < at.SUB; ++s) after(at.k[s], z[NZ - 1]);
            request_k(next);
        }
#pragma unroll
        for (int e = 0; e < NZ; ++e) z[e] *= a.scale;
        if constexpr (WEIGHTS)                                      // lanes without a head repeat the first head's: the same values
#pragma unroll
            for (int e = 0; e < NZ; e += 4) *reinterpret_cast<f32x4 *>(zrow + first + 4 * e + 4 * g) = f32x4{z[e], z[e + 1], z[e + 2], z[e + 3]};
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
        if (__any(top > m)) {                                       // a larger logit: what is summed so far shrinks
            const float f = fast_exp2(m - top);
            l *= f;
#pragma unroll
            for (int j = 0; j < TT::NV; ++j) o[j] *= f;
            m = top;
        }
        float p[NZ];
#pragma unroll
        for (int e = 0; e < NZ; ++e) p[e] = fast_exp2(z[e] - m);
        if (!all) {                                                 // rows that do not exist: neither their p nor their V may count
#pragma unroll
            for (int e = 0; e < NZ; ++e)
                if (!(there >> e & 1)) {
                    p[e] = 0.f;
                    t.zero_v(e);
                }
        }
#pragma unroll
        for (int e = 0; e < NZ; ++e) l += p[e];
        t.accumulate(p, o);
        if constexpr (!LAST) {
            find_v(a, pages, lead, rows, next, lane, at);
#pragma unroll
            for (int i = 0; i < at.NV; ++i) after(at.v[i], o[TT::NV - 1][0]);
            request_v(next);
            asm volatile("" ::: "memory");                          // or the requests would move to the loop's head, behind K's
        }
    };
    if (wave < tiles) {
        int first = wave * TT::ROWS;
        find_k(a, pages, lead, rows, first, lane, at);
        request_k(first);
        find_v(a, pages, lead, rows, first, lane, at);
        request_v(first);
        asm volatile("" ::: "memory");
#pragma unroll 1
        for (int i = wave; i + WAVES < tiles; i += WAVES, first += WAVES * TT::ROWS) tile(first, std::false_type{});
        tile(first, std::true_type{});
    }

    // the newest row goes where it belongs
    if (STEP && newest && qt == 0 && wave == 0) {
        const int64_t to = row_at(a, pages, lead, rows, rows - 1);
        if (to >= 0) {
            constexpr int FR = D * (int)sizeof(T) / 16;
            if (lane < 2 * FR) {
                const bool v = lane >= FR;
                const int sub = (v ? lane - FR : lane) * 16;
                *reinterpret_cast<uint4 *>((v ? a.v_dst : a.k_dst) + to + sub) = *reinterpret_cast<const uint4 *>((v ? v_new : k_new) + sub);
            }
            if (lane == 0 && a.pos) {
                int block, place;
                split_slot(a.g, n - 1, block, place);
                a.pos[table_index(a.g, page_of(a.g, b, block), kv, place)] = a.g.seq_pos[b] - 1;
            }
        }
    }

    // the waves' states meet
    {
        float x, y;
        rows_pair(l, x, y);
        l = x + y;
        halves_pair(l, x, y);
        l = x + y;
    }
    if (r < heads) {
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
    for (int i = threadIdx.x; i < heads * D; i += 64 * WAVES) {
        const int h = i / D, d = i % D;
        float top = sm_ml[0][h][0], sum = 0.f, acc = 0.f;
#pragma unroll
        for (int w = 1; w < WAVES; ++w) top = fmaxf(top, sm_ml[w][h][0]);
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
            const float f = fast_exp2(sm_ml[w][h][0] - top);
            sum = fmaf(sm_ml[w][h][1], f, sum);
            acc = fmaf(sm_o[(w * heads + h) * LD + d], f, acc);
        }
        const int64_t bh = (int64_t)b * a.n_heads + head0 + h;
        if (whole) {
            store_out<T>(a.out, bh * D + d, sum == 0.f ? 0.f : acc / sum);
            if (d == 0) {
                const float lse = sum == 0.f ? -INFINITY : top + __builtin_amdgcn_logf(sum);
                if (a.lse) a.lse[bh] = lse * LN2;
                sm_lse[h] = sum == 0.f ? INFINITY : lse;
            }
        } else {
            a.part_o[(bh * a.n_split + pc.chunk) * D + d] = acc;
            if (d == 0) a.part_ml[bh * a.n_split + pc.chunk] = make_float2(top, sum);
        }
    }
    if (!WEIGHTS || !whole) return;
    __syncthreads();
    for (int j = threadIdx.x; j < rows; j += 64 * WAVES) {
        const int block = block_of(a, j + lead), place = j + lead - block * a.g.page_size;
        if (pages[block] < 0) continue;
        const float *z = a.z + ((int64_t)b * a.n_heads + head0) * a.z_stride + j;
        float p = 0.f;
        for (int h = 0; h < heads; ++h) p += fast_exp2(z[(int64_t)h * a.z_stride] - sm_lse[h]);
        const int64_t i = table_index(a.g, page_of(a.g, b, block0 + block), kv, place);
        a.weight_out[i] = (STEP && newest && j == rows - 1 ? 0.f : a.weight_in[i]) + p;
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

// Joins the chunks of a (sequence, query head): blockIdx.z < group.  The workgroups beyond bring the weights of 1024 rows each up to date.
// Sequences of one chunk are complete already.
// grid = (kv heads, sequences, group + pieces of 1024 rows)
template <typename T, int D>
__global__ __launch_bounds__(256) void paged_join_kernel(PagedAttnArgs a, int step) {
    constexpr int FR = D / 4, PAR = 256 / FR;                       // 16-byte pieces of a chunk's sums, chunks read side by side
    constexpr int SEG = 512;                                        // chunks whose factors are in LDS at a time
    __shared__ float factor[SEG];
    __shared__ float red[8];
    __shared__ f32x4 part[PAR][FR];
    extern __shared__ float lse2[];                                 // [group]
    const int kv = blockIdx.x, b = blockIdx.y, tid = threadIdx.x;
    const int n = clamp_len(a.g, b), chunks = (n + a.chunk - 1) / a.chunk;
    if (chunks == 1 && a.q_tiles == 1) return;
    if ((int)blockIdx.z < a.group) {
        const int64_t bh = (int64_t)b * a.n_heads + kv * a.group + blockIdx.z;
        const float2 *ml = a.part_ml + bh * a.n_split;
        const float *po = a.part_o + bh * a.n_split * D + 4 * (tid % FR);
        float top = NEG_BIG, sum = 0.f;
        for (int c = tid; c < chunks; c += 256) top = fmaxf(top, ml[c].x);
        top = wave_max(top);
        if ((tid & 63) == 0) red[tid >> 6] = top;
        __syncthreads();
        top = fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]));
        f32x4 acc = {0.f, 0.f, 0.f, 0.f};
        for (int c0 = 0; c0 < chunks; c0 += SEG) {
            const int end = chunks - c0 < SEG ? chunks - c0 : SEG;
            __syncthreads();
            for (int c = tid; c < end; c += 256) {
                const float2 x = ml[c0 + c];
                factor[c] = fast_exp2(x.x - top);
                sum = fmaf(x.y, factor[c], sum);
            }
            __syncthreads();
#pragma unroll 4
            for (int c = tid / FR; c < end; c += PAR) acc += factor[c] * *reinterpret_cast<const f32x4 *>(po + (int64_t)(c0 + c) * D);
        }
        sum = across_groups_sum<16>(group_sum<16>(sum));
        if ((tid & 63) == 0) red[4 + (tid >> 6)] = sum;
        part[tid / FR][tid % FR] = acc;
        __syncthreads();
        sum = (red[4] + red[5]) + (red[6] + red[7]);
        if (tid < D) {
            float x = 0.f;
#pragma unroll
            for (int i = 0; i < PAR; ++i) x += reinterpret_cast<const float *>(part[i])[tid];
            store_out<T>(a.out, bh * D + tid, sum == 0.f ? 0.f : x / sum);
        }
        if (tid == 0 && a.lse) a.lse[bh] = sum == 0.f ? -INFINITY : (top + __builtin_amdgcn_logf(sum)) * LN2;
        return;
    }
    const int j0 = ((int)blockIdx.z - a.group) * 1024;
    if (j0 >= n) return;
    for (int h = tid >> 6; h < a.group; h += 4) {                   // a wave sums a head's chunks
        const float2 *ml = a.part_ml + ((int64_t)b * a.n_heads + kv * a.group + h) * a.n_split;
        float top = NEG_BIG, sum = 0.f;
        for (int c = tid & 63; c < chunks; c += 64) top = fmaxf(top, ml[c].x);
        top = wave_max(top);
        for (int c = tid & 63; c < chunks; c += 64) sum += ml[c].y * fast_exp2(ml[c].x - top);
        sum = across_groups_sum<16>(group_sum<16>(sum));
        if ((tid & 63) == 0) lse2[h] = sum == 0.f ? INFINITY : top + __builtin_amdgcn_logf(sum);
    }
    __syncthreads();
    const int end = n - j0 < 1024 ? n : j0 + 1024;
    for (int j = j0 + tid; j < end; j += 256) {
        int block, place;
        split_slot(a.g, j, block, place);
        const int page = page_of(a.g, b, block);
        if (page < 0) continue;
        const float *z = a.z + ((int64_t)b * a.n_heads + kv * a.group) * a.z_stride + j;
        float p = 0.f;
        for (int h = 0; h < a.group; ++h) p += fast_exp2(z[(int64_t)h * a.z_stride] - lse2[h]);
        const int64_t i = table_index(a.g, page, kv, place);
        a.weight_out[i] = (step && j == a.g.seq_len[b] - 1 ? 0.f : a.weight_in[i]) + p;
    }
}

// ---- launch shapes ---------------------------------------------------------------------------------------------------

struct PagedShape {
    int q_tiles, chunk, n_split;
    bool whole;
};

// Rows of a chunk: as many as leave the chip enough workgroups, 128 (a tile for each wave) to 1024.
static PagedShape paged_shape(const ssd_paged_config *c, int max_len) {
    PagedShape s;
    const int reach = paged_reach(c, max_len), group = c->n_heads / c->n_kv_heads;
    s.q_tiles = (group + HEADS - 1) / HEADS;
    const int64_t units = (int64_t)c->n_seqs * c->n_kv_heads * s.q_tiles;
    s.chunk = CHUNK_MAX;
    while (s.chunk > 128 && units * ((reach + s.chunk - 1) / s.chunk) < 8192) s.chunk /= 2;
    s.n_split = (reach + s.chunk - 1) / s.chunk;
    s.whole = s.n_split == 1 && s.q_tiles == 1;

    return s;
}

struct PagedScratch { size_t z, o, ml, all; };

static PagedScratch paged_scratch(const ssd_paged_config *c, const PagedShape &s, bool weights) {
    PagedScratch w;
    const size_t bh = (size_t)c->n_seqs * c->n_heads;
    w.z = weights ? round256(bh * s.n_split * s.chunk * sizeof(float)) : 0;
    w.o = s.whole ? 0 : round256(bh * s.n_split * c->head_dim * sizeof(float));
    w.ml = s.whole ? 0 : round256(bh * s.n_split * sizeof(float2));
    w.all = w.z + w.o + w.ml;
    return w;
}

template <typename T, int D, bool QUADS> static hipError_t launch_paged_attn(const PagedAttnArgs &a, const PagedShape &sh, bool step, hipStream_t s) {
    const int heads = a.group < HEADS ? a.group : HEADS;
    const size_t lds = (size_t)WAVES * heads * (D + 4) * sizeof(float);
    const dim3 grid((unsigned)(a.g.n_kv * sh.q_tiles), (unsigned)a.g.n_seqs, (unsigned)sh.n_split);
    const dim3 wg(64 * WAVES);
    if (step && a.weight_out) hipLaunchKernelGGL((paged_attn_kernel<T, D, QUADS, true, true>), grid, wg, lds, s, a);
    else if (step) hipLaunchKernelGGL((paged_attn_kernel<T, D, QUADS, true, false>), grid, wg, lds, s, a);
    else if (a.weight_out) hipLaunchKernelGGL((paged_attn_kernel<T, D, QUADS, false, true>), grid, wg, lds, s, a);
    else hipLaunchKernelGGL((paged_attn_kernel<T, D, QUADS, false, false>), grid, wg, lds, s, a);
    if (!sh.whole) {
        const unsigned pieces = a.weight_out ? (unsigned)(a.g.max_len + 1023) / 1024 : 0;
        hipLaunchKernelGGL((paged_join_kernel<T, D>), dim3((unsigned)a.g.n_kv, (unsigned)a.g.n_seqs, (unsigned)a.group + pieces), dim3(256),
                           (size_t)a.group * sizeof(float), s, a, step ? 1 : 0);
    }
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
    a.z = parts.z ? reinterpret_cast<float *>(ws) : nullptr;
    a.part_o = reinterpret_cast<float *>(ws + parts.z);
    a.part_ml = reinterpret_cast<float2 *>(ws + parts.z + parts.o);
    a.k_new = static_cast<const char *>(k_new);
    a.v_new = static_cast<const char *>(v_new);
    a.k_dst = static_cast<char *>(k_pages);
    a.v_dst = static_cast<char *>(v_pages);
    a.pos = pos;
    a.new_stride = (cfg->new_stride ? cfg->new_stride : (int64_t)cfg->n_kv_heads * cfg->head_dim) * (int64_t)paged_esize(cfg);
    a.z_stride = (int64_t)shape.n_split * shape.chunk;
    a.q_tiles = shape.q_tiles;
    a.chunk = shape.chunk;
    a.n_split = shape.n_split;

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
