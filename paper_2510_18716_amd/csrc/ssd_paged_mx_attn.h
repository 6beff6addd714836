// The attention over a paged cache held in 8 or 4 bits: a tile's operands from codes and scales.
//
// Both products run on the matrix cores in bf16, which holds every element of either format exactly; the conversion multiplies by the block's scale on the
// way (one instruction for two elements).  The cores' own products of scaled blocks (v_mfma_scale_f32_16x16x128_f8f6f4, q in two terms of eight bits) would save the conversion
// of K, but their sums are off by up to 2^-13 of sum |q k|, measured, where those of bf16 are fp32's.
// A lane's part of a row of K is a run of D / 4 elements, so that with rows of 128 it has one block and one scale; q is laid out alike.
// V: D / 16 columns of eight rows in a lane.  fp32 calls split q into three bf16 terms and the probabilities too (24 bits of both); bf16 calls take q as it is
// and probabilities in two terms.
//
// With four bits a row's bytes are so few that instructions bound the kernel as soon as memory: 199 vector instructions for 32 rows of 128 elements (all of a
// launch's over its tiles), 64 of them conversions.  4 sequences of 30000 to 131072 rows, 32 query heads on 8: 58 us with the second launch, 5.4 TB/s; 128 of 64 to 640 rows of
// 32 heads with weights 43 us, 3.5 TB/s: there the units' beginnings, a length, block table entries and rows one after the other, are half the time.  What was there before: V turned by
// byte permutations (32 instructions), addresses added lane by lane (14), logits scaled on their own (8), the workgroup's page addresses looked up in LDS: 63 and 51 us.
// Tried and taken back then: tiles of 64 rows (70 and 57 us: the registers do not hold them; rows of 64 elements, which they hold, gain nothing), tiles that pass
// through LDS by direct loads (64 and 51).
#pragma once

#include "ssd_mx.h"
#include "ssd_paged_attn.h"

namespace ssd {

// Where a tile's rows lie.  Every wave looks up its own tiles' pages, a chunk of them at a time.  GROUP: rows that are neighbours in one page from a multiple of GROUP on
// (16, 4 or 1, by the page size).  With 16 a group's address is the same for all lanes: found in scalar registers, the lanes' part of it never changes.  With fewer
// the groups' addresses are in LDS, in a place of the wave's own.
struct MxEntry {
    int64_t row, scales;                                           // bytes from the pools' and the scales' beginnings; row -1: no page
};

template <int SUB, int SB, int GROUP> struct MxRows {
    static constexpr int LDS = 128, PER_TILE = 16 * SUB / GROUP, TILES = LDS / PER_TILE, NV = 4 * SUB / (GROUP == 4 ? 4 : 1);
    const MxEntry *entries;                                        // of the tile to come
    int64_t k[SUB], ks[SUB], v[NV], vs[NV];
    uint32_t there;                                                // bit 4 t + i: row 16 t + 4 g + i

    template <int WAVES> __device__ __forceinline__ void begin(const PagedAttnArgs &a, const Stage &st, int wave, int lane, MxEntry *own) {
#pragma unroll
        for (int i = lane; i < LDS; i += 64) {
            const int x = (wave + i / PER_TILE * WAVES) * (16 * SUB) + i % PER_TILE * GROUP;
            int block, place;
            split_slot(a.g, st.begin + (x < st.rows ? x : 0), block, place);
            const int page = page_of(a.g, st.b, block);
            own[i] = page < 0 || x >= st.rows ? MxEntry{-1, 0} : MxEntry{row_offset(a.g, page, st.kv, place), table_index(a.g, page, st.kv, place) * SB};
        }
        entries = own;
    }
    struct Seen {
        uint32_t there;
        __device__ __forceinline__ bool all() const { return __all(there == (1u << 4 * SUB) - 1u); }
        __device__ __forceinline__ bool has(int e) const { return there >> e & 1; }
    };
    __device__ __forceinline__ Seen seen(int) const { return Seen{there}; }
};

template <int SUB, int SB> struct MxRows<SUB, SB, 16> {
    static constexpr int TILES = 64 / SUB, LDS = 1;                // tiles of a chunk
    // A lane has 16 rows of the wave's tiles in this chunk: lane SUB k + s group s of tile k.  Byte offset in the pool (the upper half below zero: no page), and
    // first place in the tables by 16.
    uint32_t low, group;
    int high, next;                                                // next: the lane of the tile to come
    int64_t off[SUB], soff[SUB];                                   // that tile's: bytes from the pools' and the scales' beginnings
    int left[SUB];                                                 // rows there are from a group's first on

    template <int WAVES> __device__ __forceinline__ void begin(const PagedAttnArgs &a, const Stage &st, int wave, int lane, MxEntry *) {
        const int x = (wave + lane / SUB * WAVES) * (16 * SUB) + lane % SUB * 16;
        int block, place;
        split_slot(a.g, st.begin + (x < st.rows ? x : 0), block, place);
        const int page = page_of(a.g, st.b, block);
        const int64_t at = row_offset(a.g, page, st.kv, place);
        low = (uint32_t)at;
        high = page < 0 ? -1 : (int)(at >> 32);
        group = ((uint32_t)page * (uint32_t)a.g.n_kv + (uint32_t)st.kv) * (uint32_t)(a.g.page_size / 16) + (uint32_t)place / 16;
        next = 0;
    }
    struct Seen {
        int left[SUB], own;                                        // own: the lane's first row in a group
        __device__ __forceinline__ bool all() const {
            bool x = true;
#pragma unroll
            for (int s = 0; s < SUB; ++s) x = x && left[s] >= 16;
            return x;
        }
        __device__ __forceinline__ bool has(int e) const { return own + e % 4 < left[e / 4]; }
    };
    __device__ __forceinline__ Seen seen(int lane) const {
        Seen x;
#pragma unroll
        for (int s = 0; s < SUB; ++s) x.left[s] = left[s];
        x.own = 4 * (lane >> 4);
        return x;
    }
};

template <int SUB, int SB>
static __device__ __forceinline__ void find_k(const PagedAttnArgs &, const Stage &st, int first, int, MxRows<SUB, SB, 16> &t) {
#pragma unroll
    for (int s = 0; s < SUB; ++s) {
        const int high = __builtin_amdgcn_readlane(t.high, t.next + s);
        const uint32_t low = (uint32_t)__builtin_amdgcn_readlane((int)t.low, t.next + s), group = (uint32_t)__builtin_amdgcn_readlane((int)t.group, t.next + s);
        t.off[s] = high < 0 ? 0 : (int64_t)((uint64_t)(uint32_t)high << 32 | low);
        t.soff[s] = high < 0 ? 0 : (int64_t)((uint64_t)group * (16 * SB));
        t.left[s] = high < 0 ? 0 : st.rows - first - 16 * s;
    }
    t.next += SUB;
}
template <int SUB, int SB>
static __device__ __forceinline__ void find_v(const PagedAttnArgs &, const Stage &, int, int, MxRows<SUB, SB, 16> &) {}

template <int SUB, int SB, int GROUP>
static __device__ __forceinline__ void find_k(const PagedAttnArgs &a, const Stage &, int, int lane, MxRows<SUB, SB, GROUP> &t) {
#pragma unroll
    for (int s = 0; s < SUB; ++s) {
        const int r = 16 * s + (lane & 15);
        const MxEntry e = t.entries[r / GROUP];
        t.k[s] = (e.row < 0 ? 0 : e.row) + (int64_t)((uint32_t)(r % GROUP) * (uint64_t)a.g.row_stride);
        t.ks[s] = e.scales + r % GROUP * SB;
    }
}
template <int SUB, int SB, int GROUP>
static __device__ __forceinline__ void find_v(const PagedAttnArgs &, const Stage &st, int first, int lane, MxRows<SUB, SB, GROUP> &t) {
    typedef MxRows<SUB, SB, GROUP> R;
    t.there = 0;
#pragma unroll
    for (int i = 0; i < R::NV; ++i) {
        const int r = GROUP == 4 ? 16 * i + 4 * (lane >> 4) : 16 * (i / 4) + 4 * (lane >> 4) + i % 4;
        const MxEntry e = t.entries[r / GROUP];
        t.v[i] = e.row < 0 ? 0 : e.row;
        t.vs[i] = e.scales;
        const int left = e.row < 0 ? 0 : st.rows - first - r;
#pragma unroll
        for (int x = 0; x < (GROUP == 4 ? 4 : 1); ++x) t.there |= x < left ? 1u << (GROUP == 4 ? 4 * i + x : i) : 0u;
    }
    t.entries += R::PER_TILE;                                       // K's were found before
}

// Requests wait for the product that has read the registers they fill (as with plain rows).
template <int SUB, int SB> static __device__ __forceinline__ void hold_k(MxRows<SUB, SB, 16> &t, float result) {
#pragma unroll
    for (int s = 0; s < SUB; ++s) asm volatile("" : "+s"(t.off[s]), "+s"(t.soff[s]) : "v"(result));
}
template <int SUB, int SB> static __device__ __forceinline__ void hold_v(MxRows<SUB, SB, 16> &t, float result) { hold_k(t, result); }
template <int SUB, int SB, int GROUP> static __device__ __forceinline__ void hold_k(MxRows<SUB, SB, GROUP> &t, float result) {
#pragma unroll
    for (int s = 0; s < SUB; ++s) asm volatile("" : "+v"(t.k[s]), "+v"(t.ks[s]) : "v"(result));
}
template <int SUB, int SB, int GROUP> static __device__ __forceinline__ void hold_v(MxRows<SUB, SB, GROUP> &t, float result) {
#pragma unroll
    for (int i = 0; i < MxRows<SUB, SB, GROUP>::NV; ++i) asm volatile("" : "+v"(t.v[i]), "+v"(t.vs[i]) : "v"(result));
}

template <int N> struct Words { typedef uint32_t type __attribute__((ext_vector_type(N))); };
template <> struct Words<1> { typedef uint32_t type; };
template <> struct Words<8> { typedef uint32_t type __attribute__((ext_vector_type(8), aligned(16))); };

// The upper 16 bits of x as a bf16 (rounded toward zero), and what they leave out, exactly.  An infinity leaves nothing.
static __device__ __forceinline__ uint32_t take_upper(float &x) {
    const uint32_t u = __float_as_uint(x), hi = u & 0xffff0000u;
    x = (u & 0x7fffffffu) == 0x7f800000u ? 0.f : x - __uint_as_float(hi);
    return hi >> 16;
}

// Waves of a SIMD: fp32 rows of 128 elements need more registers than three leave (q in three terms).
static constexpr int mx_resident(bool f32, int d) { return f32 && d == 128 ? 2 : 3; }

// HT: heads of a tile, 4, 8 or 16.  The matrix cores' sixteen columns hold COPIES = 16 / HT columns for a head.  With two, one takes the even elements of a
// pair (V's columns 2 c), the other the odd ones: a pair is the operand as it comes from the conversion, two neighbouring places of the sum, and a copy has its
// probability in one of them and nothing in the other.  So V is not turned at all, and the sums take half the registers.  With four (bf16 calls) two more take
// the probabilities' second term.
template <typename T, int D_, int BITS_, int GROUP, int HT> struct MxTile {
    typedef T elem;
    static constexpr bool MX = true, TABLE = true, QUADS = GROUP >= 4;
    static constexpr int RESIDENT = mx_resident(sizeof(T) == 4, D_), EXTRA = BITS_ == 4 ? 3 : 2, ENTRIES = GROUP == 16 ? 0 : 128;
    typedef MxEntry entry_t;
    static constexpr int D = D_, BITS = BITS_, SB = D / 32;        // SB: bytes of a row's scales
    static constexpr int SUB = 2, ROWS = 16 * SUB;
    static constexpr int STEPS = D / 32, NV = D / 16, KE = D / 4;  // KE: elements of a row of K in a lane
    static constexpr int KW = KE * BITS / 32, VB = NV * BITS / 8;  // dwords of those; bytes of a row of V in a lane
    static constexpr int QT = sizeof(T) == 4 ? 3 : 1, PT = sizeof(T) == 4 ? 3 : 2;      // terms of q and of the probabilities
    static constexpr int COPIES = 16 / HT, NO = COPIES == 1 ? NV : NV / 2;
    static_assert(COPIES < 4 || PT == 2, "four copies have two terms");
    static __device__ __forceinline__ int head(int r) { return r % HT; }
    static __device__ __forceinline__ bool writes(int r) { return r < 2 * HT; }
    template <bool> using Rows = MxRows<SUB, SB, GROUP>;
    static constexpr int TILES = MxRows<SUB, SB, GROUP>::TILES;
    typedef typename Words<KW>::type krow_t;
    typedef std::conditional_t<VB == 2, uint16_t, typename Words<VB == 8 ? 2 : 1>::type> vrow_t;
    typedef std::conditional_t<SB == 2, uint16_t, uint32_t> one_t;  // of one

    krow_t k[SUB];
    uint32_t ks[SUB];
    vrow_t v[4 * SUB];
    uint32_t vs[QUADS ? SUB : 4 * SUB];                            // V's scales: QUADS of row 4 g + lane % 4 of a group, else of row i
    struct Q { bf16x8 x[QT][STEPS]; };

    static __device__ __forceinline__ int odd(int lane) { return (lane & 15) / HT & 1; }
    static __device__ __forceinline__ bool second(int lane) { return (lane & 15) / (2 * HT) & 1; }
    template <typename X> static __device__ __forceinline__ X load(const char *p) { return __builtin_nontemporal_load(reinterpret_cast<const X *>(p)); }

    static __device__ __forceinline__ void load_q(const char *row, int lane, Q &q) {
#pragma unroll
        for (int s = 0; s < STEPS; ++s) {
            const char *p = row + (KE * (lane >> 4) + 8 * s) * sizeof(T);
            if constexpr (QT == 1) {
                q.x[0][s] = *reinterpret_cast<const bf16x8 *>(p);
            } else {
                const f32x4 lo = *reinterpret_cast<const f32x4 *>(p), hi = *reinterpret_cast<const f32x4 *>(p + 16);
                uint32_t w[QT][8];
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    float x = e < 4 ? lo[e % 4] : hi[e % 4];
                    w[0][e] = take_upper(x);
                    w[1][e] = take_upper(x);
                    w[2][e] = __float_as_uint(x) >> 16;
                    if (x != x) w[2][e] = 0x7fc0u;                 // NaN, whose upper half alone may be an infinity's
                }
#pragma unroll
                for (int t = 0; t < QT; ++t) {
                    const u32x4_nt_t d = {w[t][0] | w[t][1] << 16, w[t][2] | w[t][3] << 16, w[t][4] | w[t][5] << 16, w[t][6] | w[t][7] << 16};
                    q.x[t][s] = __builtin_bit_cast(bf16x8, d);
                }
            }
        }
    }

    __device__ __forceinline__ void load_k(int s, const char *row, const char *scales, int lane) {
        k[s] = load<krow_t>(row + (uint32_t)(lane >> 4) * (KE * BITS / 8));
        ks[s] = (uint32_t)*reinterpret_cast<const uint8_t *>(scales + (uint32_t)(lane >> 4) * KE / 32);
    }

    __device__ __forceinline__ void logits(const Q &q, float (&z)[4 * SUB]) const {
#pragma unroll
        for (int t = 0; t < SUB; ++t) {
            const float scale = __uint_as_float(ks[t] << 23);
            f32x4 c = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int s = 0; s < STEPS; ++s) {
                u32x4_nt_t w;
#pragma unroll
                for (int i = 0; i < 4; ++i) w[i] = BITS == 4 ? pair(k[t][s], scale, i) : pair(k[t][2 * s + i / 2], scale, i % 2);
#pragma unroll
                for (int m = QT - 1; m >= 0; --m) c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, w), q.x[m][s], c, 0, 0, 0);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) z[4 * t + i] = c[i];
        }
    }

    static __device__ __forceinline__ uint32_t pair(uint32_t codes, float scale, int i) {
        return i == 0 ? mx_pair<BITS, 0>(codes, scale)
               : i == 1 ? mx_pair<BITS, 1>(codes, scale)
               : i == 2 ? mx_pair<BITS, BITS == 4 ? 2 : 1>(codes, scale)
                        : mx_pair<BITS, BITS == 4 ? 3 : 1>(codes, scale);
    }

    // Scale of row i in the lane's block of V, the byte (lane % 16) NV / 32 of the row's; four neighbouring lanes have four rows'.
    __device__ __forceinline__ float v_scale(int i, int lane) const {
        const uint32_t block = (uint32_t)(lane & 15) * NV / 32;
        uint32_t w;
        if constexpr (QUADS) {
            const int x = (int)vs[i / 4];
            w = (uint32_t)(i % 4 == 0 ? __builtin_amdgcn_update_dpp(0, x, 0x00, 0xF, 0xF, true) : i % 4 == 1 ? __builtin_amdgcn_update_dpp(0, x, 0x55, 0xF, 0xF, true)
                           : i % 4 == 2 ? __builtin_amdgcn_update_dpp(0, x, 0xAA, 0xF, 0xF, true) : __builtin_amdgcn_update_dpp(0, x, 0xFF, 0xF, 0xF, true));
        } else {
            w = vs[i];
        }
        w &= 0xffu << 8 * block;
        return __uint_as_float(__builtin_amdgcn_alignbit(w, w, 8 * block + 9));        // the byte to the exponent's place
    }
    // A row that does not exist: neither its codes nor a scale that is NaN may count.
    __device__ __forceinline__ void zero_v(int i) {
        v[i] = vrow_t(0);
        if constexpr (!QUADS) vs[i] = 0;
        else if ((int)(threadIdx.x & 3) == i % 4) vs[i / 4] = 0;
    }

    // x less one of two bf16 (`which`: -1 in its place, 0 in the other's), exactly: the upper half of x, so that what is left has fewer bits.
    static __device__ __forceinline__ float less(float x, uint32_t two, uint32_t which) {
        return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2_t, two), __builtin_bit_cast(bf16x2_t, which), x, false);
    }
    __device__ __forceinline__ uint32_t v_pair(int i, int c, float scale) const {
        if constexpr (VB == 8) return pair(v[i][c / 2], scale, c % 2);
        else return pair((uint32_t)v[i], scale, c);
    }

    // Sums of V's columns times p.  The probabilities go in as terms of bf16, each the upper half of what the one before leaves: 16 bits of each (two terms) or 24 (three, which
    // leave nothing).  The second of two is rounded: cut off, it would leave out up to 2^-15 of every probability, all on one side, where the sum of the softmax has them
    // whole; half a step added to its bits does it, since no p is below zero (eight of 200 vector instructions of a tile; nothing in the times).
    __device__ __forceinline__ void accumulate(const float (&p)[4 * SUB], f32x4 (&o)[NO]) const {
        const int lane = threadIdx.x & 63;
        if constexpr (COPIES == 1) {
            // -1 as the lower and as the upper of two bf16, from registers: as a constant the lower one is encoded as the fp32 number -1, which is the upper
            uint32_t lower = 0x0000bf80u, upper = 0xbf800000u;
            asm("" : "+s"(lower), "+s"(upper));
#pragma unroll
            for (int t = 0; t < SUB / 2; ++t) {
                bf16x8 term[PT];
                float rest[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) rest[i] = p[8 * t + i];
#pragma unroll
                for (int m = 0; m < PT; ++m) {
                    u32x4_nt_t d;
                    if (m == 1 && PT == 2) {
#pragma unroll
                        for (int i = 0; i < 8; ++i) term[m][i] = (__bf16)rest[i];
                        continue;
                    }
#pragma unroll
                    for (int i = 0; i < 8; i += 2) {
                        const uint32_t two = __builtin_amdgcn_perm(__float_as_uint(rest[i + 1]), __float_as_uint(rest[i]), 0x07060302u);
                        d[i / 2] = two;
                        rest[i] = less(rest[i], two, lower);
                        rest[i + 1] = less(rest[i + 1], two, upper);
                    }
                    term[m] = __builtin_bit_cast(bf16x8, d);
                }
                float scale[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) scale[i] = v_scale(8 * t + i, lane);
#pragma unroll
                for (int c = 0; c < NV / 2; ++c) {
                    uint32_t x[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i) x[i] = v_pair(8 * t + i, c, scale[i]);
#pragma unroll
                    for (int half = 0; half < 2; ++half) {
                        u32x4_nt_t w;
#pragma unroll
                        for (int e = 0; e < 4; ++e) w[e] = __builtin_amdgcn_perm(x[2 * e + 1], x[2 * e], half ? 0x07060302u : 0x05040100u);
#pragma unroll
                        for (int m = PT - 1; m >= 0; --m)
                            o[2 * c + half] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, w), term[m], o[2 * c + half], 0, 0, 0);
                    }
                }
            }
        } else {
            constexpr int TERMS = COPIES == 4 ? 1 : PT;
            const uint32_t take = odd(lane) ? 0x07060c0cu : 0x0c0c0706u;        // the upper half of a number, in the copy's place
            const uint32_t which = odd(lane) ? 0xbf800000u : 0x0000bf80u, less_first = second(lane) ? 0xffff0000u : 0u;
            const uint32_t half = COPIES == 4 ? (second(lane) ? 0x8000u : 0u) : PT == 2 ? 0x8000u : 0u;       // of the last term's step
#pragma unroll
            for (int t = 0; t < SUB; ++t) {
                u32x4_nt_t term[TERMS];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    float x = p[4 * t + i];
                    if constexpr (COPIES == 4) x -= __uint_as_float(__float_as_uint(x) & less_first);
#pragma unroll
                    for (int m = 0; m < TERMS; ++m) {
                        const uint32_t two = __builtin_amdgcn_perm(__float_as_uint(x) + (m + 1 == TERMS ? half : 0u), 0u, take);
                        term[m][i] = two;
                        if (m + 1 < TERMS) x = less(x, two, which);
                    }
                }
                float scale[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) scale[i] = v_scale(4 * t + i, lane);
#pragma unroll
                for (int c = 0; c < NV / 2; ++c) {
                    u32x4_nt_t w;
#pragma unroll
                    for (int i = 0; i < 4; ++i) w[i] = v_pair(4 * t + i, c, scale[i]);
#pragma unroll
                    for (int m = TERMS - 1; m >= 0; --m)
                        o[c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, w), __builtin_bit_cast(bf16x8, term[m]), o[c], 0, 0, 0);
                }
            }
        }
    }
    // The copies' terms meet.
    static __device__ __forceinline__ void finish(f32x4 (&o)[NO]) {
        if constexpr (COPIES == 4) {
#pragma unroll
            for (int j = 0; j < NO; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) o[j][e] += dpp_f<0x128>(o[j][e]);      // eight lanes on
        }
    }
    // column of o[j][i] in lane
    static __device__ __forceinline__ int column(int j, int i, int lane) { return NV * (4 * (lane >> 4) + i) + (COPIES == 1 ? j : 2 * j + odd(lane)); }

    // A step's newest row: its codes into the pool, by the wave that is about to read it (of every workgroup that does: all write the same).  A wave's loads are in
    // order with the stores before them.
    static constexpr int SLICES = D / 8;                           // lanes of a row, eight elements each: K's, then V's
    struct Newest { Eight<T> x; };
    static __device__ __forceinline__ Newest load_newest(const char *k_new, const char *v_new, int lane) {
        const char *row = lane & SLICES ? v_new : k_new;
        return {load_eight<T>(row + (lane & (SLICES - 1)) * 8 * (int)sizeof(T))};
    }
    static __device__ __forceinline__ void put_newest(const Newest &x, const PagedAttnArgs &a, int b, int kv, int n, int lane) {
        const int slice = lane & (SLICES - 1);
        const bool is_v = lane & SLICES;
        int block, place;
        split_slot(a.g, n - 1, block, place);
        const int page = page_of(a.g, b, block);
        const uint32_t byte = mx_scale_of<BITS>(quad_max(largest_of<T>(x.x)));
        const Codes<BITS> c = mx_encode<BITS, T>(x.x, byte);
        if (page >= 0 && lane < 2 * SLICES) {
            *reinterpret_cast<Codes<BITS> *>((is_v ? a.v_dst : a.k_dst) + row_offset(a.g, page, kv, place) + slice * BITS) = c;
            const int64_t entry = table_index(a.g, page, kv, place);
            if (slice % 4 == 0) (is_v ? a.v_scales : a.k_scales)[entry * SB + slice / 4] = (uint8_t)byte;
            if (lane == 0 && a.pos) a.pos[entry] = a.g.seq_pos[b] - 1;
        }
        asm volatile("" ::: "memory");
    }
};

// Bytes at base + more + own, base and more being the same for all lanes: through a buffer, whose address is in scalar registers (as a pointer the compiler adds
// it lane by lane, 14 of 250 vector instructions).  NT: read once.
static __device__ __forceinline__ __amdgpu_buffer_rsrc_t mx_buffer(const void *base) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void *>(base), 0, -1, 0x00027000);
}
template <typename X, int NT> static __device__ __forceinline__ X mx_load(__amdgpu_buffer_rsrc_t from, uint32_t own, uint32_t more) {
    if constexpr (sizeof(X) == 32) {
        const u32x4_nt_t lo = mx_load<u32x4_nt_t, NT>(from, own, more), hi = mx_load<u32x4_nt_t, NT>(from, own + 16, more);
        return X{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
    } else if constexpr (sizeof(X) == 16) {
        return __builtin_bit_cast(X, __builtin_amdgcn_raw_buffer_load_b128(from, (int)own, (int)more, NT));
    } else if constexpr (sizeof(X) == 8) {
        return __builtin_bit_cast(X, __builtin_amdgcn_raw_buffer_load_b64(from, (int)own, (int)more, NT));
    } else if constexpr (sizeof(X) == 4) {
        return __builtin_bit_cast(X, __builtin_amdgcn_raw_buffer_load_b32(from, (int)own, (int)more, NT));
    } else {
        return (X)__builtin_amdgcn_raw_buffer_load_b16(from, (int)own, (int)more, NT);
    }
}
template <typename Step, typename TT, int SUB, int SB>
static __device__ __forceinline__ void request_k(Step, const PagedAttnArgs &a, const MxRows<SUB, SB, 16> &at, TT &tl, int, int, const char *, int lane) {
    const uint32_t r = (uint32_t)lane & 15, g = (uint32_t)lane >> 4, own = r * (uint32_t)a.g.row_stride + g * (TT::KE * TT::BITS / 8);
#pragma unroll
    for (int s = 0; s < SUB; ++s) {
        tl.k[s] = mx_load<typename TT::krow_t, 2>(mx_buffer(a.k_pages + at.off[s]), own, 0);
        tl.ks[s] = __builtin_amdgcn_raw_buffer_load_b8(mx_buffer(a.k_scales + at.soff[s]), (int)(r * SB + g * TT::KE / 32), 0, 0);
    }
}
template <typename Step, typename TT, int SUB, int SB>
static __device__ __forceinline__ void request_v(Step, const PagedAttnArgs &a, const MxRows<SUB, SB, 16> &at, TT &tl, int, int, const char *, int lane) {
    const uint32_t g = (uint32_t)lane >> 4, own = 4 * g * (uint32_t)a.g.row_stride + ((uint32_t)lane & 15) * TT::VB;
#pragma unroll
    for (int s = 0; s < SUB; ++s) {
        const __amdgpu_buffer_rsrc_t from = mx_buffer(a.v_pages + at.off[s]);
#pragma unroll
        for (int i = 0; i < 4; ++i) tl.v[4 * s + i] = mx_load<typename TT::vrow_t, 2>(from, own, (uint32_t)i * (uint32_t)a.g.row_stride);
        tl.vs[s] = mx_load<typename TT::one_t, 0>(mx_buffer(a.v_scales + at.soff[s]), (4 * g + (lane & 3)) * SB, 0);
    }
}
template <typename Step, typename TT, int SUB, int SB, int GROUP>
static __device__ __forceinline__ void request_k(Step, const PagedAttnArgs &a, const MxRows<SUB, SB, GROUP> &at, TT &tl, int, int, const char *, int lane) {
#pragma unroll
    for (int s = 0; s < SUB; ++s) tl.load_k(s, a.k_pages + at.k[s], reinterpret_cast<const char *>(a.k_scales) + at.ks[s], lane);
}
template <typename Step, typename TT, int SUB, int SB, int GROUP>
static __device__ __forceinline__ void request_v(Step, const PagedAttnArgs &a, const MxRows<SUB, SB, GROUP> &at, TT &tl, int, int, const char *, int lane) {
#pragma unroll
    for (int i = 0; i < 4 * SUB; ++i) {
        const char *row = a.v_pages + (GROUP == 4 ? at.v[i / 4] + i % 4 * a.g.row_stride : at.v[i]);
        tl.v[i] = TT::template load<typename TT::vrow_t>(row + ((uint32_t)lane & 15) * TT::VB);
    }
#pragma unroll
    for (int i = 0; i < MxRows<SUB, SB, GROUP>::NV; ++i)
        tl.vs[i] = *reinterpret_cast<const typename TT::one_t *>(a.v_scales + at.vs[i] + (GROUP == 4 ? (lane & 3) * SB : 0));
}

// Rows that are neighbours in a page: 16 (at distances that fit 32 bits), 4 (up to eight query heads on a key head: there are no tiles of sixteen for it) or 1.
static inline int mx_group(const ssd_paged_config *c) {
    if (c->page_size % 16 == 0 && 16 * (c->row_stride ? c->row_stride : (int64_t)c->head_dim) < 1ll << 31) return 16;
    return c->page_size % 4 == 0 && c->n_heads / c->n_kv_heads <= 8 ? 4 : 1;
}
static inline TileShape mx_tile_shape(const ssd_paged_config *c) {
    const int group = mx_group(c);
    return {32, 256 * mx_resident(c->dtype == SSD_F32, c->head_dim), group == 16 ? 32 : group == 4 ? 16 : 4};
}

template <typename T, int BITS> hipError_t launch_mx_attn(const PagedAttnArgs &a, const PagedShape &sh, int d, int group, bool step, hipStream_t s);

#ifdef SSD_MX_ONLY
template <typename T, int D, int BITS> static hipError_t launch_mx_rows(const PagedAttnArgs &a, const PagedShape &sh, int group, bool step, hipStream_t s) {
    if (group == 1) return launch_paged_attn<MxTile<T, D, BITS, 1, 16>, false>(a, sh, step, s);
    if (group == 4) return launch_paged_attn<MxTile<T, D, BITS, 4, 8>, true>(a, sh, step, s);
    if constexpr (sizeof(T) == 2)
        if (a.group <= 4) return launch_paged_attn<MxTile<T, D, BITS, 16, 4>, true>(a, sh, step, s);
    if (a.group <= 8) return launch_paged_attn<MxTile<T, D, BITS, 16, 8>, true>(a, sh, step, s);
    return launch_paged_attn<MxTile<T, D, BITS, 16, 16>, true>(a, sh, step, s);
}
template <typename T, int BITS> hipError_t launch_mx_attn(const PagedAttnArgs &a, const PagedShape &sh, int d, int group, bool step, hipStream_t s) {
    return d == 128 ? launch_mx_rows<T, 128, BITS>(a, sh, group, step, s) : launch_mx_rows<T, 64, BITS>(a, sh, group, step, s);
}
template hipError_t launch_mx_attn<SSD_MX_ONLY>(const PagedAttnArgs &, const PagedShape &, int, int, bool, hipStream_t);
#endif

}  // namespace ssd
