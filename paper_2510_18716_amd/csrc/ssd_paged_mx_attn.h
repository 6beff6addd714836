// The attention over a paged cache held in 8 or 4 bits: a tile's operands from codes and scales.
//
// Both products run on the matrix cores in bf16, which holds every element of either format exactly; the conversion multiplies by the block's scale on the
// way (one instruction for two elements).  A lane's part of a row of K is a run of D / 4 elements, so that with rows of 128 it has one block and one scale;
// q is laid out alike.  V as in the tiles of plain rows: D / 16 columns of eight rows in a lane, turned by byte permutations after the conversion.
// fp32 calls split q into three bf16 terms and the probabilities too (24 bits of both); bf16 calls take q as it is and probabilities in two terms.
#pragma once

#include "ssd_mx.h"
#include "ssd_paged_attn.h"

namespace ssd {

// Where a tile's rows lie.  P16: the page size is a multiple of 16, so that 16 rows are neighbours in one page, and a group's address is the same for all
// lanes: found in scalar registers, the lanes' part of it never changes.
template <int SUB, int SB, bool P16> struct MxRows;

template <int SUB, int SB> struct MxRows<SUB, SB, true> {
    int64_t off[SUB], soff[SUB];                                   // bytes from the pools' and the scales' beginnings
    int left[SUB];                                                 // rows there are from the group's first on
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

template <int SUB, int SB> struct MxRows<SUB, SB, false> {
    int64_t k[SUB], ks[SUB], v[4 * SUB], vs[4 * SUB];
    uint32_t there;                                                // bit 4 t + i: row 16 t + 4 g + i
    struct Seen {
        uint32_t there;
        __device__ __forceinline__ bool all() const { return __all(there == (1u << 4 * SUB) - 1u); }
        __device__ __forceinline__ bool has(int e) const { return there >> e & 1; }
    };
    __device__ __forceinline__ Seen seen(int) const { return Seen{there}; }
};

template <int SUB, int SB>
static __device__ __forceinline__ void find_k(const PagedAttnArgs &a, const Stage &st, int first, int, MxRows<SUB, SB, true> &t) {
#pragma unroll
    for (int s = 0; s < SUB; ++s) {
        const int x = first + 16 * s, y = (x < st.rows ? x : (st.rows - 1) & ~15) + st.lead;
        const int block = block_of(a, y), place = y - block * a.g.page_size;
        const int id = __builtin_amdgcn_readfirstlane(st.ids[block]), page = id < 0 ? 0 : id;
        t.off[s] = row_offset(a.g, page, st.kv, place);
        t.soff[s] = table_index(a.g, page, st.kv, place) * SB;
        t.left[s] = id < 0 ? 0 : st.rows - x;
    }
}
template <int SUB, int SB>
static __device__ __forceinline__ void find_v(const PagedAttnArgs &, const Stage &, int, int, MxRows<SUB, SB, true> &) {}

// A row's offsets in the pool and the scales; rows that do not exist get the pool's first row and `false`.
static __device__ __forceinline__ bool mx_row_at(const PagedAttnArgs &a, const Stage &st, int x, int64_t &row, int64_t &entry) {
    const int y = (x < st.rows ? x : st.rows - 1) + st.lead;
    const int block = block_of(a, y), place = y - block * a.g.page_size, id = st.ids[block];
    row = id < 0 ? 0 : row_offset(a.g, id, st.kv, place);
    entry = id < 0 ? 0 : table_index(a.g, id, st.kv, place);
    return id >= 0 && x < st.rows;
}
template <int SUB, int SB>
static __device__ __forceinline__ void find_k(const PagedAttnArgs &a, const Stage &st, int first, int lane, MxRows<SUB, SB, false> &t) {
#pragma unroll
    for (int s = 0; s < SUB; ++s) {
        int64_t entry;
        mx_row_at(a, st, first + 16 * s + (lane & 15), t.k[s], entry);
        t.ks[s] = entry * SB;
    }
}
template <int SUB, int SB>
static __device__ __forceinline__ void find_v(const PagedAttnArgs &a, const Stage &st, int first, int lane, MxRows<SUB, SB, false> &t) {
    t.there = 0;
#pragma unroll
    for (int i = 0; i < 4 * SUB; ++i) {
        int64_t entry;
        const bool is = mx_row_at(a, st, first + 16 * (i / 4) + 4 * (lane >> 4) + i % 4, t.v[i], entry);
        t.vs[i] = entry * SB;
        t.there |= is ? 1u << i : 0u;
    }
}

// Requests wait for the product that has read the registers they fill (as with plain rows).
template <int SUB, int SB> static __device__ __forceinline__ void hold_k(MxRows<SUB, SB, true> &t, float result) {
#pragma unroll
    for (int s = 0; s < SUB; ++s) asm volatile("" : "+s"(t.off[s]), "+s"(t.soff[s]) : "v"(result));
}
template <int SUB, int SB> static __device__ __forceinline__ void hold_v(MxRows<SUB, SB, true> &t, float result) { hold_k(t, result); }
template <int SUB, int SB> static __device__ __forceinline__ void hold_k(MxRows<SUB, SB, false> &t, float result) {
#pragma unroll
    for (int s = 0; s < SUB; ++s) asm volatile("" : "+v"(t.k[s]), "+v"(t.ks[s]) : "v"(result));
}
template <int SUB, int SB> static __device__ __forceinline__ void hold_v(MxRows<SUB, SB, false> &t, float result) {
#pragma unroll
    for (int i = 0; i < 4 * SUB; ++i) asm volatile("" : "+v"(t.v[i]), "+v"(t.vs[i]) : "v"(result));
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

template <typename T, int D_, int BITS_, bool P16> struct MxTile {
    typedef T elem;
    static constexpr bool MX = true;
    static constexpr int D = D_, BITS = BITS_, SB = D / 32;        // SB: bytes of a row's scales
    static constexpr int SUB = 2, ROWS = 16 * SUB;
    static constexpr int STEPS = D / 32, NV = D / 16, KE = D / 4;  // KE: elements of a row of K in a lane
    static constexpr int KW = KE * BITS / 32, VB = NV * BITS / 8;  // dwords of those; bytes of a row of V in a lane
    static constexpr int QT = sizeof(T) == 4 ? 3 : 1, PT = sizeof(T) == 4 ? 3 : 2;      // terms of q and of the probabilities
    template <bool QUADS> using Rows = MxRows<SUB, SB, P16>;
    typedef typename Words<KW>::type krow_t;
    typedef std::conditional_t<VB == 2, uint16_t, typename Words<VB == 8 ? 2 : 1>::type> vrow_t;
    typedef typename Words<SB>::type four_t;                       // scales of four rows
    typedef std::conditional_t<SB == 2, uint16_t, uint32_t> one_t;  // of one

    krow_t k[SUB];
    uint32_t ks[SUB];
    vrow_t v[4 * SUB];
    std::conditional_t<P16, four_t, one_t> vs[P16 ? SUB : 4 * SUB];
    struct Q { bf16x8 x[QT][STEPS]; };

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
    __device__ __forceinline__ uint32_t word(const krow_t &x, int i) const {
        if constexpr (KW == 1) return x;
        else return x[i];
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
                for (int i = 0; i < 4; ++i) w[i] = BITS == 4 ? pair(word(k[t], s), scale, i) : pair(word(k[t], 2 * s + i / 2), scale, i % 2);
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

    // Scale of row i in the lane's block of V.
    __device__ __forceinline__ float v_scale(int i, int lane) const {
        const uint32_t block = (uint32_t)(lane & 15) * NV / 32;
        uint32_t w, at = 8 * block;
        if constexpr (P16) {
            if constexpr (SB == 4) {
                w = vs[i / 4][i % 4];
            } else {
                w = vs[i / 4][i % 4 / 2];
                at += 16 * (i % 2);
            }
        } else {
            w = vs[i];
        }
        return __uint_as_float(__builtin_amdgcn_ubfe(w, at, 8) << 23);
    }
    // A row that does not exist: neither its codes nor a scale that is NaN may count.
    __device__ __forceinline__ void zero_v(int i) {
        v[i] = vrow_t(0);
        if constexpr (!P16) vs[i] = 0;
        else if constexpr (SB == 4) vs[i / 4][i % 4] = 0;
        else vs[i / 4][i % 4 / 2] &= i % 2 ? 0x0000ffffu : 0xffff0000u;
    }

    // o[j] += column d = NV m + j of V, times p.  The probabilities go in as terms of bf16, each the upper half of what the one before leaves; the last
    // one of two is rounded: 16 bits of each or more (2^-17), of three 24.
    __device__ __forceinline__ void accumulate(const float (&p)[4 * SUB], f32x4 (&o)[NV]) const {
        const int lane = threadIdx.x & 63;
#pragma unroll
        for (int t = 0; t < SUB / 2; ++t) {
            bf16x8 term[PT];
            {
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
                    for (int i = 0; i < 8; i += 2) d[i / 2] = __builtin_amdgcn_perm(__float_as_uint(rest[i + 1]), __float_as_uint(rest[i]), 0x07060302u);
                    term[m] = __builtin_bit_cast(bf16x8, d);
#pragma unroll
                    for (int i = 0; i < 8; ++i) rest[i] -= __uint_as_float(__float_as_uint(rest[i]) & 0xffff0000u);
                }
            }
            float scale[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) scale[i] = v_scale(8 * t + i, lane);
#pragma unroll
            for (int c = 0; c < NV / 2; ++c) {
                uint32_t x[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    if constexpr (VB == 8) x[i] = pair(v[8 * t + i][c / 2], scale[i], c % 2);
                    else x[i] = pair((uint32_t)v[8 * t + i], scale[i], c);
                }
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
    }
    static __device__ __forceinline__ int column(int j, int i, int lane) { return NV * (4 * (lane >> 4) + i) + j; }

    // A step's newest row: its codes into the pool, by every workgroup that is about to read it (all write the same).
    static __device__ __forceinline__ void put_newest(const PagedAttnArgs &a, int b, int kv, int n, const char *k_new, const char *v_new) {
        constexpr int PARTS = D / 8;
        const int tid = (int)threadIdx.x, part = tid & (PARTS - 1);
        if (tid >= 2 * PARTS) return;
        const bool is_v = tid >= PARTS;
        const Eight<T> x = load_eight<T>((is_v ? v_new : k_new) + part * 8 * (int)sizeof(T));
        int block, place;
        split_slot(a.g, n - 1, block, place);
        const int page = page_of(a.g, b, block);
        const uint32_t byte = mx_scale_of<BITS>(quad_max(largest_of<T>(x)));
        const Codes<BITS> c = mx_encode<BITS, T>(x, byte);
        if (page < 0) return;
        char *to = (is_v ? a.v_dst : a.k_dst) + row_offset(a.g, page, kv, place) + part * BITS;
#pragma unroll
        for (int i = 0; i < BITS / 4; ++i) reinterpret_cast<uint32_t *>(to)[i] = c.c[i];
        const int64_t entry = table_index(a.g, page, kv, place);
        if (part % 4 == 0) (is_v ? a.v_scales : a.k_scales)[entry * SB + part / 4] = (uint8_t)byte;
        if (tid == 0 && a.pos) a.pos[entry] = a.g.seq_pos[b] - 1;
    }
};

template <typename Step, typename TT, int SUB, int SB>
static __device__ __forceinline__ void request_k(Step, const PagedAttnArgs &a, const MxRows<SUB, SB, true> &at, TT &tl, int, int, const char *, int lane) {
    const uint32_t r = (uint32_t)lane & 15, own = r * (uint32_t)a.g.row_stride;
#pragma unroll
    for (int s = 0; s < SUB; ++s) tl.load_k(s, a.k_pages + at.off[s] + own, reinterpret_cast<const char *>(a.k_scales) + at.soff[s] + r * SB, lane);
}
template <typename Step, typename TT, int SUB, int SB>
static __device__ __forceinline__ void request_v(Step, const PagedAttnArgs &a, const MxRows<SUB, SB, true> &at, TT &tl, int, int, const char *, int lane) {
    const uint32_t g = (uint32_t)lane >> 4, own = 4 * g * (uint32_t)a.g.row_stride + ((uint32_t)lane & 15) * TT::VB;
#pragma unroll
    for (int s = 0; s < SUB; ++s) {
#pragma unroll
        for (int i = 0; i < 4; ++i) tl.v[4 * s + i] = TT::template load<typename TT::vrow_t>(a.v_pages + at.off[s] + i * a.g.row_stride + own);
        tl.vs[s] = *reinterpret_cast<const typename TT::four_t *>(reinterpret_cast<const char *>(a.v_scales) + at.soff[s] + g * (4 * SB));
    }
}
template <typename Step, typename TT, int SUB, int SB>
static __device__ __forceinline__ void request_k(Step, const PagedAttnArgs &a, const MxRows<SUB, SB, false> &at, TT &tl, int, int, const char *, int lane) {
#pragma unroll
    for (int s = 0; s < SUB; ++s) tl.load_k(s, a.k_pages + at.k[s], reinterpret_cast<const char *>(a.k_scales) + at.ks[s], lane);
}
template <typename Step, typename TT, int SUB, int SB>
static __device__ __forceinline__ void request_v(Step, const PagedAttnArgs &a, const MxRows<SUB, SB, false> &at, TT &tl, int, int, const char *, int lane) {
#pragma unroll
    for (int i = 0; i < 4 * SUB; ++i) {
        tl.v[i] = TT::template load<typename TT::vrow_t>(a.v_pages + at.v[i] + ((uint32_t)lane & 15) * TT::VB);
        tl.vs[i] = *reinterpret_cast<const typename TT::one_t *>(a.v_scales + at.vs[i]);
    }
}

static inline bool mx_sixteen(const PagedGeom &g) { return g.page_size % 16 == 0 && g.row_stride < 1 << 26; }

template <typename T, int BITS> hipError_t launch_mx_attn(const PagedAttnArgs &a, const PagedShape &sh, int d, bool step, hipStream_t s);

#ifdef SSD_MX_ONLY
template <typename T, int BITS> hipError_t launch_mx_attn(const PagedAttnArgs &a, const PagedShape &sh, int d, bool step, hipStream_t s) {
    const bool p16 = mx_sixteen(a.g);
    if (d == 128) return p16 ? launch_paged_attn<MxTile<T, 128, BITS, true>, true>(a, sh, step, s) : launch_paged_attn<MxTile<T, 128, BITS, false>, false>(a, sh, step, s);
    return p16 ? launch_paged_attn<MxTile<T, 64, BITS, true>, true>(a, sh, step, s) : launch_paged_attn<MxTile<T, 64, BITS, false>, false>(a, sh, step, s);
}
template hipError_t launch_mx_attn<SSD_MX_ONLY>(const PagedAttnArgs &, const PagedShape &, int, bool, hipStream_t);
#endif

}  // namespace ssd
