// ssd_paged_evict: each (sequence, kv head) of a paged cache is cut to its budget; the rows of the largest accumulated attention weight
// stay (the top-M rule of Algorithm 1, sinks and recent tokens protected as in Sec. 3.3).
//
// Selection.  The key of the last row that stays is found by a descent over the keys' bits: the weight first, then the position; whole-number
// compares, so the set is exact.  Up to 16384 rows a unit is one workgroup's, whose threads keep their rows' keys in registers, so that the tables
// are read once.  Up to 256 rows that is one wave, which descends bit by bit (a ballot counts); above, ten bits a step by a histogram in LDS,
// beginning at the first bit in which the keys differ.  Every thread ranks its free slots below n' and its kept rows above by one scan over
// the workgroup.  A longer unit is cut into slices (the section "long units").
// Slots whose block has no page hold no row and can take none: they are left out of the competition, and so are their places below n'.
// Movement.  A kept row above n' goes to the free slot of its own rank, in 16-byte fragments: by the unit's workgroup where units are many,
// by a launch with more workgroups per unit otherwise.
//
// Measured (8 key heads, rows of 256 bytes in pages of 16 and 64): 32 sequences of 500 to 8192 rows to 1024, 46 us, of which selection takes the first 13 (latency: tables,
// three histograms, ranks) and the rows, all units' at once, 24 at 4.9 TB/s read and written, and 9 are not accounted for; 2 sequences of 70001 and 100000 rows to 16000, 96 us, rows 48 at 4.4 TB/s and
// five launches of 7 to 10; one of 129 rows in 512 units 4.5 us, launch and latency.
#include "ssd_paged.h"

namespace ssd {

struct PagedEvictArgs {
    PagedGeom g;
    char *k_pages, *v_pages;
    const int32_t *budget, *pos_in;
    const float *weight_in;
    int32_t *pos_out;
    float *weight_out;
    int32_t *len_out;
    int32_t *moves;          // per unit: count, then cap free slots, then cap slots to move from
    int n_sink, recent;
    int cap;
    int lpr_log2;
};

static __host__ __device__ inline int64_t moves_of(int cap, int64_t unit) { return unit * (2 * (int64_t)cap + 1); }

// Larger is better.  Weights: NaN below everything, -0 as +0, the rest by their bits turned into an ascending order.
static __device__ __forceinline__ uint32_t weight_key(float w) {
    const uint32_t u = __float_as_uint(w);
    if ((u & 0x7fffffffu) > 0x7f800000u) return 0;
    if (u << 1 == 0) return 0x80000000u;
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}
static __device__ __forceinline__ uint32_t pos_key(int pos) { return ~((uint32_t)pos ^ 0x80000000u); }

struct Four {
    float w[4];
    int pos[4];
    uint32_t there;                                                // bits: rows whose block has a page
};

// Weights and positions of rows j .. j + 3 (those below n).
static __device__ __forceinline__ Four table_rows(const PagedEvictArgs &a, int b, int kv, int j, int n) {
    typedef float f4 __attribute__((ext_vector_type(4), aligned(4)));
    typedef int i4 __attribute__((ext_vector_type(4), aligned(4)));
    Four r;
    int block, place;
    split_slot(a.g, j, block, place);
    if (place + 4 <= a.g.page_size) {
        const int page = page_of(a.g, b, block);
        const int64_t i = table_index(a.g, page < 0 ? 0 : page, kv, place);
        const f4 w = *reinterpret_cast<const f4 *>(a.weight_in + i);
        const i4 p = *reinterpret_cast<const i4 *>(a.pos_in + i);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            r.w[e] = w[e];
            r.pos[e] = p[e];
        }
        r.there = page < 0 ? 0u : 15u;
        return r;
    }
    r.there = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        r.w[e] = 0.f;
        r.pos[e] = 0;
        if (j + e < n) {
            split_slot(a.g, j + e, block, place);
            const int page = page_of(a.g, b, block);
            if (page >= 0) {
                const int64_t i = table_index(a.g, page, kv, place);
                r.w[e] = a.weight_in[i];
                r.pos[e] = a.pos_in[i];
                r.there |= 1u << e;
            }
        }
    }
    return r;
}

// Rows from[i] to slots to[i]: K and V of a row by neighbouring threads, MOVES rows of a thread on their way at a time (past the end it repeats
// the last row, which writes the same again); move_entries: the tables' entries, a thread each.  No load is under a condition: the compiler would wait for
// everything in flight.
template <int MOVES, typename I>
static __device__ __forceinline__ void move_rows(const PagedEvictArgs &a, int b, int kv, const I *to, const I *from, int count, int thread,
                                                 int threads) {
    const int lanes = 2 << a.lpr_log2, lane = thread & (lanes - 1), step = threads / lanes;
    const bool v = lane >> a.lpr_log2;
    char *pool = (v ? a.v_pages : a.k_pages) + (int64_t)kv * a.g.head_stride + (int64_t)(lane & ((1 << a.lpr_log2) - 1)) * 16;
    for (int i0 = thread / lanes; i0 < count; i0 += MOVES * step) {
        int tp[MOVES], fp[MOVES], tpage[MOVES], fpage[MOVES];
#pragma unroll
        for (int m = 0; m < MOVES; ++m) {
            const int i = i0 + m * step < count ? i0 + m * step : count - 1;
            int block;
            split_slot(a.g, to[i], block, tp[m]);
            tpage[m] = page_of(a.g, b, block);
            split_slot(a.g, from[i], block, fp[m]);
            fpage[m] = page_of(a.g, b, block);
        }
        u32x4_nt_t x[MOVES];
#pragma unroll
        for (int m = 0; m < MOVES; ++m)
            x[m] = __builtin_nontemporal_load(
                reinterpret_cast<const u32x4_nt_t *>(pool + (int64_t)(fpage[m] < 0 ? 0 : fpage[m]) * a.g.page_stride + (int64_t)fp[m] * a.g.row_stride));
#pragma unroll
        for (int m = 0; m < MOVES; ++m)
            if (tpage[m] >= 0 && fpage[m] >= 0) *reinterpret_cast<u32x4_nt_t *>(pool + (int64_t)tpage[m] * a.g.page_stride + (int64_t)tp[m] * a.g.row_stride) = x[m];
    }
}

template <typename I>
static __device__ __forceinline__ void move_entries(const PagedEvictArgs &a, int b, int kv, const I *to, const I *from, int count, int thread,
                                                    int threads) {
    for (int i = thread; i < count; i += threads) {
        int block, tp, fp;
        split_slot(a.g, to[i], block, tp);
        const int tpage = page_of(a.g, b, block);
        split_slot(a.g, from[i], block, fp);
        const int fpage = page_of(a.g, b, block);
        if (tpage < 0 || fpage < 0) continue;
        const int64_t t = table_index(a.g, tpage, kv, tp), f = table_index(a.g, fpage, kv, fp);
        a.weight_out[t] = a.weight_in[f];
        a.pos_out[t] = a.pos_in[f];
    }
}

// ---- the descent ---------------------------------------------------------------------------------------------------------

static constexpr int BITS = 10, BINS = 1 << BITS;

// Bits in which the rows that compete differ, and how many rows are protected.
struct Spread {
    uint32_t safe, any_w, not_all_w, any_p, not_all_p;             // any: some row has the bit, not_all: some row lacks it
    __device__ __forceinline__ void add(uint32_t w, uint32_t p, bool in) {
        any_w |= in ? w : 0;
        not_all_w |= in ? ~w : 0;
        any_p |= in ? p : 0;
        not_all_p |= in ? ~p : 0;
    }
};

// The last row that stays: rows with a larger key stay, of those with the same key the first `ties` in slot order.
struct Last {
    uint32_t w, p;
    int ties;                                                      // 2^31 - 1: all of them
};

template <int THREADS> struct DescentLds {
    uint32_t hist[2][BINS];
    uint32_t red[5][THREADS / 64];
    int found[3];
};

// each(f): f(weight key, position key) for this thread's competing rows.  left: places among them, 1 .. their number.  Both histograms are
// clear on entry.
template <int THREADS, typename Each>
static __device__ __forceinline__ Last descend(DescentLds<THREADS> &lds, const Spread &sp, int left, const Each &each) {
    const int tid = threadIdx.x, lane = tid & 63;
    const uint32_t dw = sp.any_w & sp.not_all_w, dp = sp.any_p & sp.not_all_p;
    int bits = dw ? 32 - __clz((int)dw) : 0;                       // open bits of the key at hand
    uint32_t ref = bits == 32 ? 0 : sp.any_w >> bits << bits;      // (above them any row's bits are every row's)
    uint32_t w_done = ref;
    bool on_pos = false, whole = false;
    for (int level = 0;; ++level) {
        if (bits == 0) {
            if (on_pos) break;
            w_done = ref;
            on_pos = true;
            bits = dp ? 32 - __clz((int)dp) : 0;
            ref = bits == 32 ? 0 : sp.any_p >> bits << bits;
            if (bits == 0) break;
        }
        const int take = bits < BITS ? bits : BITS, shift = bits - take;
        const uint32_t mask = (1u << take) - 1;
        uint32_t *h = lds.hist[level & 1];
        each([&](uint32_t w, uint32_t p) {
            const uint32_t key = on_pos ? p : w;
            if ((!on_pos || w == w_done) && (bits == 32 || (key ^ ref) >> bits == 0)) atomicAdd(&h[key >> shift & mask], 1u);
        });
        __syncthreads();
        // the digit in which the place falls: one wave adds up the bins from the top while the others clear the next step's
        if (tid < 64) {
            constexpr int PER = BINS / 64;
            uint32_t bin[PER], sum = 0;
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                bin[i] = h[BINS - 1 - (lane * PER + i)];
                sum += bin[i];
            }
            const uint32_t upto = wave_scan(sum);
            const int l = __ffsll((unsigned long long)__ballot(upto >= (uint32_t)left)) - 1;
            uint32_t above = upto - sum;
            int digit = -1;
            uint32_t in_bin = 0;
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                const bool here = digit < 0 && above + bin[i] >= (uint32_t)left;
                digit = here ? BINS - 1 - (lane * PER + i) : digit;
                in_bin = here ? bin[i] : in_bin;
                above += digit < 0 ? bin[i] : 0;
            }
            if (lane == l) {
                lds.found[0] = digit;
                lds.found[1] = (int)above;
                lds.found[2] = (int)in_bin;
            }
        }
        if (THREADS == 64 || tid >= 64)
            for (int i = THREADS == 64 ? tid : tid - 64; i < BINS; i += THREADS == 64 ? 64 : THREADS - 64) lds.hist[(level & 1) ^ 1][i] = 0;
        __syncthreads();
        ref |= (uint32_t)lds.found[0] << shift;
        left -= lds.found[1];
        bits = shift;
        whole = lds.found[2] == left;                              // all of them stay: nothing below needs looking at
        if (whole) break;
    }
    Last r;
    r.w = on_pos ? w_done : ref;
    r.p = on_pos ? ref : 0;
    r.ties = whole ? 0x7fffffff : left;
    return r;
}

// The same for the rows of one wave, bit by bit: how many rows have the bits found so far and a one in the next.
template <typename Count>
static __device__ __forceinline__ Last descend_wave(const Spread &sp, int left, int rows, const Count &count) {
    const uint32_t dw = sp.any_w & sp.not_all_w, dp = sp.any_p & sp.not_all_p;
    Last r;
    r.w = sp.any_w & ~dw;
    r.p = 0;
    // rows: with the bits so far; `left` of them stay
    for (uint32_t open = dw; open;) {
        const uint32_t bit = 0x80000000u >> __clz((int)open), try_w = r.w | bit;
        open &= ~bit;
        const int ones = count([&](uint32_t w, uint32_t) { return ((w ^ try_w) & ~open) == 0; });
        if (ones >= left) {
            r.w = try_w;
            rows = ones;
        } else {
            left -= ones;
            rows -= ones;
        }
        if (rows == left) {
            r.ties = 0x7fffffff;
            return r;
        }
    }
    r.p = sp.any_p & ~dp;
    for (uint32_t open = dp; open;) {
        const uint32_t bit = 0x80000000u >> __clz((int)open), try_p = r.p | bit;
        open &= ~bit;
        const int ones = count([&](uint32_t w, uint32_t p) { return w == r.w && ((p ^ try_p) & ~open) == 0; });
        if (ones >= left) {
            r.p = try_p;
            rows = ones;
        } else {
            left -= ones;
            rows -= ones;
        }
        if (rows == left) {
            r.ties = 0x7fffffff;
            return r;
        }
    }
    r.ties = left;
    return r;
}

// Where few rows go: they are taken out one by one.  keys: this thread's; compete: which of them do; gone: the bits of rows that go are set.
// The least key goes; of equal ones the highest slot (threads have consecutive rows).
// Lines where the descent takes as long: 256 units of 200 rows, 12 evictions 8.8 and 11.2 us, 24 12.6 and 10.0; of 2000, 8 15.4 and 18.2, 16 23.3 and 19.9; of 8000, 4 35.6
// and 38.6, 6 40.5 and 39.0.
static constexpr int few(int threads) { return threads == 64 ? 16 : threads == 256 ? 8 : 4; }
template <int THREADS, int KEYS>
static __device__ __forceinline__ uint32_t take_least(const uint32_t (&wk)[KEYS], const uint32_t (&pk)[KEYS], uint32_t compete, int rows,
                                                      unsigned long long (&least)[2][THREADS / 64], int (&owner)[2][THREADS / 64]) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    uint32_t gone = 0;
    for (int i = 0; i < rows; ++i) {
        unsigned long long m = ~0ull;
        int at = 0;
#pragma unroll
        for (int k = 0; k < KEYS; ++k) {
            const unsigned long long key = (unsigned long long)wk[k] << 32 | pk[k];
            const bool less = ((compete & ~gone) >> k & 1) && key <= m;
            m = less ? key : m;
            at = less ? k : at;
        }
        unsigned long long all = wave_min_u64(m);
        const bool any = (compete & ~gone) != 0;
        int last = 63 - __clzll((long long)(__ballot(any && m == all) | 1));  // the highest lane that has it
        bool ours = true;
        if constexpr (THREADS > 64) {
            const bool some = __any(any);                          // of the whole wave: not inside the branch
            if (lane == 0) {
                least[i & 1][wave] = all;
                owner[i & 1][wave] = some;
            }
            __syncthreads();
            int w = -1;
#pragma unroll
            for (int x = 0; x < THREADS / 64; ++x)
                if (owner[i & 1][x] && (w < 0 || least[i & 1][x] <= all)) {
                    w = x;
                    all = least[i & 1][x];
                }
            ours = w == wave;
        }
        if (ours && lane == last) gone |= 1u << at;
    }
    return gone;
}

// 2: stays, 1: has the last row's keys, 0: goes.  Where the descent ended early the open bits of the last keys are 0 and everything
// at or above them stays.
static __device__ __forceinline__ int standing(const Last &l, uint32_t w, uint32_t p) {
    if (w != l.w) return w > l.w ? 2 : 0;
    return p > l.p ? 2 : p == l.p ? 1 : 0;
}

// The tables' entries of rows j .. j + 3 below `stay`, from the old tables to the new.
static __device__ __forceinline__ void copy_entries(const PagedEvictArgs &a, int b, int kv, int j, int stay) {
    typedef float f4 __attribute__((ext_vector_type(4), aligned(4)));
    typedef int i4 __attribute__((ext_vector_type(4), aligned(4)));
    int block, place;
    split_slot(a.g, j, block, place);
    if (place + 4 <= a.g.page_size && j + 4 <= stay) {
        const int page = page_of(a.g, b, block);
        if (page < 0) return;
        const int64_t i = table_index(a.g, page, kv, place);
        *reinterpret_cast<f4 *>(a.weight_out + i) = *reinterpret_cast<const f4 *>(a.weight_in + i);
        *reinterpret_cast<i4 *>(a.pos_out + i) = *reinterpret_cast<const i4 *>(a.pos_in + i);
        return;
    }
    for (int e = 0; e < 4 && j + e < stay; ++e) {
        split_slot(a.g, j + e, block, place);
        const int page = page_of(a.g, b, block);
        if (page < 0) continue;
        const int64_t i = table_index(a.g, page, kv, place);
        a.pos_out[i] = a.pos_in[i];
        a.weight_out[i] = a.weight_in[i];
    }
}

static __device__ __forceinline__ int stay_of(const PagedEvictArgs &a, int b, int n) {
    const int want = a.budget[b] < 0 ? 0 : a.budget[b];
    return n < want ? n : want;
}
static __device__ __forceinline__ bool is_safe(const PagedEvictArgs &a, int64_t total, int pos) {
    return pos < a.n_sink || (int64_t)pos >= total - a.recent;
}

// ---- units of one workgroup ----------------------------------------------------------------------------------------------

// A thread has KEYS consecutive rows.  grid = (kv heads, sequences)
template <int THREADS, int KEYS>
__global__ __launch_bounds__(THREADS) void paged_select_kernel(PagedEvictArgs a, int move_here) {
    constexpr int NW = THREADS / 64, HALF = THREADS * KEYS / 2;
    __shared__ DescentLds<THREADS> lds;
    __shared__ uint16_t free_slots[HALF], move_slots[HALF];        // if the rows move here: at most half of them do
    __shared__ unsigned long long least[2][NW];
    __shared__ int owner[2][NW];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    int kv, b;
    unit_of(a.g, kv, b);
    const int n = clamp_len(a.g, b), stay = stay_of(a, b, n);
    const bool copy = a.pos_out != a.pos_in;
    const int64_t total = a.g.seq_pos[b];
    int32_t *list = a.moves + moves_of(a.cap, (int64_t)b * a.g.n_kv + kv);
    if (kv == 0 && tid == 0 && a.len_out) a.len_out[b] = stay;
    if (n == stay) {
        if (tid == 0 && !move_here) list[0] = 0;
        if (copy)
            for (int j = 4 * tid; j < stay; j += 4 * THREADS) copy_entries(a, b, kv, j, stay);
        return;
    }
    const int j0 = tid * KEYS;
    uint32_t wk[KEYS], pk[KEYS], safe = 0, in = 0;                 // keys; bits: protected, below n and with a page
#pragma unroll
    for (int k = 0; k < KEYS; k += 4) {
        if (j0 + k < n) {
            const Four r = table_rows(a, b, kv, j0 + k, n);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                wk[k + e] = weight_key(r.w[e]);
                pk[k + e] = pos_key(r.pos[e]);
                safe |= is_safe(a, total, r.pos[e]) ? 1u << (k + e) : 0u;
                in |= j0 + k + e < n && (r.there >> e & 1) ? 1u << (k + e) : 0u;
            }
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) wk[k + e] = pk[k + e] = 0;
        }
    }
    safe &= in;
    // the tables' entries of slots below n'; those of free slots are written again with the rows that move there
    if (copy)
#pragma unroll
        for (int k = 0; k < KEYS; k += 4)
            if (j0 + k < stay) copy_entries(a, b, kv, j0 + k, stay);
    if (THREADS > 64) {
        for (int i = tid; i < 2 * BINS; i += THREADS) (&lds.hist[0][0])[i] = 0;
    }

    // protected rows and slots without a page, at most 16384 of either
    const int mine = n - j0 < 0 ? 0 : n - j0 < KEYS ? n - j0 : KEYS, below = stay - j0 < 0 ? 0 : stay - j0 < KEYS ? stay - j0 : KEYS;
    const uint32_t low = (1u << below) - 1;                        // the thread's slots below n'
    uint32_t counts = wave_sum((uint32_t)__popc(safe) | (uint32_t)(mine - __popc(in)) << 16);
    if (NW > 1) {
        if (lane == 0) lds.red[0][wave] = counts;
        __syncthreads();
        counts = 0;
#pragma unroll
        for (int i = 0; i < NW; ++i) counts += lds.red[0][i];
    }
    const int safe_rows = (int)(counts & 0xffff), rows = n - (int)(counts >> 16);
    int places = stay;                                             // slots below n' that can hold a row
    if (rows < n) {
        uint32_t c = wave_sum((uint32_t)__popc(in & low));
        if (NW > 1) {
            if (lane == 0) lds.red[1][wave] = c;
            __syncthreads();
            c = 0;
#pragma unroll
            for (int i = 0; i < NW; ++i) c += lds.red[1][i];
            __syncthreads();                                       // the line is written again
        }
        places = (int)c;
    }
    // protected rows, if they leave places for others; else they alone compete
    const bool among_safe = safe_rows >= places;
    const int left = among_safe ? places : places - safe_rows;
    const uint32_t compete = among_safe ? safe : in & ~safe;
    uint32_t kept = among_safe ? 0 : safe, tie = 0;
    Last last = {0, 0, 0};
    const int go = (among_safe ? safe_rows : rows - safe_rows) - left;     // of those that compete
    if (left > 0 && go <= few(THREADS)) {
        kept |= compete & ~take_least<THREADS, KEYS>(wk, pk, compete, go, least, owner);
    } else if (left > 0) {
        Spread sp = {0, 0, 0, 0, 0};
#pragma unroll
        for (int k = 0; k < KEYS; ++k) sp.add(wk[k], pk[k], compete >> k & 1);
        sp.any_w = wave_or(sp.any_w);
        sp.not_all_w = wave_or(sp.not_all_w);
        sp.any_p = wave_or(sp.any_p);
        sp.not_all_p = wave_or(sp.not_all_p);
        if constexpr (NW == 1) {
            last = descend_wave(sp, left, among_safe ? safe_rows : rows - safe_rows, [&](auto f) {
                int c = 0;
#pragma unroll
                for (int k = 0; k < KEYS; ++k) c += (int)__popcll(__ballot((compete >> k & 1) && f(wk[k], pk[k])));
                return c;
            });
        } else {
            if (lane == 0) {
                lds.red[1][wave] = sp.any_w;
                lds.red[2][wave] = sp.not_all_w;
                lds.red[3][wave] = sp.any_p;
                lds.red[4][wave] = sp.not_all_p;
            }
            __syncthreads();
#pragma unroll
            for (int i = 0; i < NW; ++i) {
                sp.any_w |= lds.red[1][i];
                sp.not_all_w |= lds.red[2][i];
                sp.any_p |= lds.red[3][i];
                sp.not_all_p |= lds.red[4][i];
            }
            last = descend<THREADS>(lds, sp, left, [&](auto f) {
#pragma unroll
                for (int k = 0; k < KEYS; ++k)
                    if (compete >> k & 1) f(wk[k], pk[k]);
            });
        }
#pragma unroll
        for (int k = 0; k < KEYS; ++k) {
            const int st = standing(last, wk[k], pk[k]);
            kept |= (compete >> k & 1) && st == 2 ? 1u << k : 0u;
            tie |= (compete >> k & 1) && st == 1 ? 1u << k : 0u;
        }
        if (last.ties == 0x7fffffff) {
            kept |= tie;
        } else {                                                   // the lowest slots of those with the last keys
            const uint32_t c = (uint32_t)__popc(tie), up = wave_scan(c);
            uint32_t before = up - c;
            if (NW > 1) {
                if (lane == 63) lds.red[0][wave] = up;
                __syncthreads();
#pragma unroll
                for (int i = 0; i < NW; ++i) before += i < wave ? lds.red[0][i] : 0;
            }
#pragma unroll
            for (int k = 0; k < KEYS; ++k)
                if (tie >> k & 1) {
                    kept |= (int)before < last.ties ? 1u << k : 0u;
                    ++before;
                }
        }
    }

    // where slots become free, which rows move
    const uint32_t free_bits = in & low & ~kept, move_bits = kept & ~low;
    const uint32_t c = (uint32_t)__popc(free_bits) | (uint32_t)__popc(move_bits) << 16, up = wave_scan(c);
    uint32_t before = up - c, all = (uint32_t)__builtin_amdgcn_readlane((int)up, 63);
    if (NW > 1) {
        if (lane == 63) lds.red[1][wave] = up;
        __syncthreads();
        all = 0;
#pragma unroll
        for (int i = 0; i < NW; ++i) {
            before += i < wave ? lds.red[1][i] : 0;
            all += lds.red[1][i];
        }
    }
    uint32_t f = before & 0xffff, m = before >> 16;
    const int moves = (int)(all >> 16);
#pragma unroll
    for (int k = 0; k < KEYS; ++k) {
        if (free_bits >> k & 1) {
            if (move_here) free_slots[f] = (uint16_t)(j0 + k);
            else list[1 + f] = j0 + k;
            ++f;
        }
        if (move_bits >> k & 1) {
            if (move_here) move_slots[m] = (uint16_t)(j0 + k);
            else list[1 + a.cap + m] = j0 + k;
            ++m;
        }
    }
    if (!move_here) {
        if (tid == 0) list[0] = moves;
    } else if (moves > 0) {
        __syncthreads();
        move_entries(a, b, kv, free_slots, move_slots, moves, tid, THREADS);
        if (moves <= THREADS / (2 << a.lpr_log2)) move_rows<1>(a, b, kv, free_slots, move_slots, moves, tid, THREADS);
        else move_rows<8>(a, b, kv, free_slots, move_slots, moves, tid, THREADS);
    }
}

// ---- long units ------------------------------------------------------------------------------------------------------------
//
// The rows below n' and those above are cut into slices of equally many rows, a workgroup each; a unit's own workgroup works in between.
//   1 slices: how many rows have which upper 12 bits of their weight, protected ones and others apart; slots without a page
//   2 unit:   the bin in which the last place falls, and how many rows of a slice are above it and in it
//   3 slices: the rows in the bin, in slot order, into one list (the memory of the moves, which come later), with their keys
//   4 unit:   the descent among those; where each slice's free slots and moving rows begin in the lists
//   5 slices: the lists
//   6 as everywhere: the rows move
static constexpr int TOP = 12, TOP_BINS = 1 << TOP, SLICES = 62;
static constexpr int ST = 1024;                                    // threads of a slice
static constexpr int PICK = 6144;                                  // candidates whose keys fit in LDS

// What step 2 and 4 leave for a unit's slices.
struct SliceInfo {
    int32_t kept, in_bin, first;                                   // rows above the bin, in it, and where the latter begin in the list
    int32_t at;                                                    // where its free slots, or its moving rows, begin in the lists
    int32_t safe;                                                  // protected rows
    int32_t gone;                                                  // slots without a page
};
struct UnitInfo {
    int32_t among_safe, bin, left, candidates;
    uint32_t last_w, last_p;
    int32_t last_slot, pad;
    SliceInfo slice[SLICES + 2];
};

struct SliceArgs {
    PagedEvictArgs e;
    uint32_t *hist;                                                // [units, slices + 2, 2, TOP_BINS]
    UnitInfo *info;                                                // [units]
    int slices;
    // the first candidates' keys, where the unit's histograms were
    __device__ __forceinline__ uint32_t *keys(int64_t unit) const { return hist + unit * (slices + 2) * 2 * TOP_BINS; }
};
static_assert(PICK <= 3 * TOP_BINS, "a unit has three slices' histograms or more");

struct Slices {
    int rows, low, count;                                          // rows of a slice, slices below n', all of them
    __device__ __forceinline__ Slices(int n, int stay, int slices) {
        rows = ((n + slices - 1) / slices + 3) & ~3;
        low = (stay + rows - 1) / rows;
        count = low + (n - stay + rows - 1) / rows;
    }
    __device__ __forceinline__ int begin(int s, int stay) const { return s < low ? s * rows : stay + (s - low) * rows; }
    __device__ __forceinline__ int end(int s, int n, int stay) const {
        const int e = begin(s, stay) + rows, most = s < low ? stay : n;
        return e < most ? e : most;
    }
    __device__ __forceinline__ int of(int slot, int stay) const { return slot < stay ? slot / rows : low + (slot - stay) / rows; }
};

__global__ __launch_bounds__(ST) void slice_count_kernel(SliceArgs s) {
    const PagedEvictArgs &a = s.e;
    __shared__ uint32_t hist[2][TOP_BINS];
    __shared__ uint32_t red[2][ST / 64];
    const int kv = blockIdx.y, b = blockIdx.z, tid = threadIdx.x;
    const int n = clamp_len(a.g, b), stay = stay_of(a, b, n);
    const Slices sl(n > 0 ? n : 1, stay, s.slices);
    if (n == stay || (int)blockIdx.x >= sl.count) return;
    const int64_t total = a.g.seq_pos[b], unit = (int64_t)b * a.g.n_kv + kv;
    for (int i = tid; i < 2 * TOP_BINS / 4; i += ST) reinterpret_cast<uint4 *>(&hist[0][0])[i] = make_uint4(0, 0, 0, 0);
    __syncthreads();
    const int end = sl.end((int)blockIdx.x, n, stay);
    uint32_t safe = 0, gone = 0;
    for (int j = sl.begin((int)blockIdx.x, stay) + 4 * tid; j < end; j += 4 * ST) {
        const Four r = table_rows(a, b, kv, j, end);
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (j + e < end) {
                if (!(r.there >> e & 1)) {
                    ++gone;
                    continue;
                }
                const bool sf = is_safe(a, total, r.pos[e]);
                safe += sf;
                atomicAdd(&hist[sf][weight_key(r.w[e]) >> (32 - TOP)], 1u);
            }
    }
    safe = wave_sum(safe);
    gone = wave_sum(gone);
    if ((tid & 63) == 0) {
        red[0][tid >> 6] = safe;
        red[1][tid >> 6] = gone;
    }
    __syncthreads();
    safe = gone = 0;
#pragma unroll
    for (int i = 0; i < ST / 64; ++i) {
        safe += red[0][i];
        gone += red[1][i];
    }
    if (tid == 0) {
        s.info[unit].slice[blockIdx.x].safe = (int32_t)safe;
        s.info[unit].slice[blockIdx.x].gone = (int32_t)gone;
    }
    uint4 *out = reinterpret_cast<uint4 *>(s.hist + (unit * (s.slices + 2) + blockIdx.x) * 2 * TOP_BINS);
    // the protected rows' half only where there are such rows
    for (int i = tid; i < (safe ? 2 : 1) * TOP_BINS / 4; i += ST) out[i] = *reinterpret_cast<const uint4 *>(&hist[0][0] + 4 * i);
}

__global__ __launch_bounds__(1024) void slice_bin_kernel(SliceArgs s) {
    const PagedEvictArgs &a = s.e;
    __shared__ uint32_t red[16];
    __shared__ int found[5], safe_of[SLICES + 2];
    __shared__ SliceInfo info[SLICES + 2];
    const int kv = blockIdx.x, b = blockIdx.y, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int n = clamp_len(a.g, b), stay = stay_of(a, b, n);
    if (kv == 0 && tid == 0 && a.len_out) a.len_out[b] = stay;
    if (n == stay) return;
    const Slices sl(n, stay, s.slices);
    const int64_t unit = (int64_t)b * a.g.n_kv + kv;
    const uint32_t *hist = s.hist + unit * (s.slices + 2) * 2 * TOP_BINS;
    UnitInfo *u = s.info + unit;
    uint32_t gone = 0;                                             // of slice tid
    if (tid < 64) {
        const uint32_t c = tid < sl.count ? (uint32_t)u->slice[tid].safe : 0;
        gone = tid < sl.count ? (uint32_t)u->slice[tid].gone : 0;
        safe_of[tid] = (int)c;
        const uint32_t all = wave_sum(c), low = wave_sum(tid < sl.low ? gone : 0u);
        if (tid == 0) {
            found[2] = (int)all;
            found[4] = stay - (int)low;
        }
    }
    if (tid == 0) {
        found[0] = TOP_BINS;                                       // no place to compete for: nothing is in or above this bin
        found[1] = 0;
        found[3] = 0;
    }
    __syncthreads();
    const int safe_rows = found[2], places = found[4], k = safe_rows >= places;       // k = 1: protected rows alone compete
    const uint32_t left = (uint32_t)(k ? places : places - safe_rows);
    // a thread has PER bins, counted from the top
    constexpr int PER = TOP_BINS / 1024;
    static_assert(PER == 4, "bins are read four at a time");
    const int bin = TOP_BINS - PER * (tid + 1);
    uint32_t h[PER] = {0, 0, 0, 0};
    if (!k) {
        constexpr int AT = 16;                                     // slices on their way at a time
        for (int i0 = 0; i0 < sl.count; i0 += AT) {
            uint4 x[AT];
#pragma unroll
            for (int i = 0; i < AT; ++i)
                x[i] = *reinterpret_cast<const uint4 *>(hist + (int64_t)(i0 + i < sl.count ? i0 + i : sl.count - 1) * 2 * TOP_BINS + bin);
#pragma unroll
            for (int i = 0; i < AT; ++i) {
                const bool real = i0 + i < sl.count;
                h[0] += real ? x[i].w : 0;
                h[1] += real ? x[i].z : 0;
                h[2] += real ? x[i].y : 0;
                h[3] += real ? x[i].x : 0;
            }
        }
    } else {
        for (int i = 0; i < sl.count; ++i)
            if (safe_of[i] > 0) {
                const uint4 x = *reinterpret_cast<const uint4 *>(hist + ((int64_t)i * 2 + 1) * TOP_BINS + bin);
                h[0] += x.w;
                h[1] += x.z;
                h[2] += x.y;
                h[3] += x.x;
            }
    }
    const uint32_t mine = h[0] + h[1] + h[2] + h[3], up = wave_scan(mine);
    if (lane == 63) red[wave] = up;
    __syncthreads();
    uint32_t above = up - mine;
#pragma unroll
    for (int i = 0; i < 16; ++i) above += i < wave ? red[i] : 0;
    if (above == 0 && mine > 0) found[3] = bin + PER;              // no row is in this bin or above it
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        if (left > 0 && above < left && above + h[i] >= left) {
            found[0] = bin + PER - 1 - i;
            found[1] = (int)(left - above);
        }
        above += h[i];
    }
    __syncthreads();
    const int at = found[0];
    // a wave per slice: what it has above the bin and in it
    for (int i = wave; i < sl.count; i += 16) {
        const uint32_t *row = hist + ((int64_t)i * 2 + k) * TOP_BINS;
        const bool any = !k || safe_of[i] > 0;
        uint32_t over = 0;
        if (any)
            for (int x = (at & ~3) + lane * 4; x < found[3]; x += 256) {
                const uint4 v = *reinterpret_cast<const uint4 *>(row + x);
                over += (x > at ? v.x : 0) + (x + 1 > at ? v.y : 0) + (x + 2 > at ? v.z : 0) + (x + 3 > at ? v.w : 0);
            }
        over = wave_sum(over);
        if (lane == 0) info[i] = SliceInfo{(int32_t)over + (k ? 0 : safe_of[i]), any && at < TOP_BINS ? (int32_t)row[at] : 0, 0, 0, 0, 0};
    }
    __syncthreads();
    if (tid < 64) {
        const uint32_t c = tid < sl.count ? (uint32_t)info[tid].in_bin : 0, up = wave_scan(c);
        if (tid < sl.count) u->slice[tid] = SliceInfo{info[tid].kept, info[tid].in_bin, (int32_t)(up - c), 0, safe_of[tid], (int32_t)gone};
        if (tid == 63) {
            u->among_safe = k;
            u->bin = at;
            u->left = found[1];
            u->candidates = (int32_t)up;
        }
    }
}

// A slice's rows 4 * ST at a time, four a thread: body(first row of the thread, its rows or none) between barriers of its own.
template <typename Body>
static __device__ __forceinline__ void slice_rows(const PagedEvictArgs &a, int b, int kv, int begin, int end, const Body &body) {
    Four r[2];
    int j = begin + 4 * (int)threadIdx.x;
    if (j < end) r[0] = table_rows(a, b, kv, j, end);
    for (int base = begin; base < end; base += 4 * ST, j += 4 * ST) {
        if (j + 4 * ST < end) r[1] = table_rows(a, b, kv, j + 4 * ST, end);       // on its way while these are ranked
        body(j, r[0]);
        r[0] = r[1];
    }
}

__global__ __launch_bounds__(ST) void slice_gather_kernel(SliceArgs s) {
    const PagedEvictArgs &a = s.e;
    __shared__ uint32_t red[2][ST / 64];
    const int kv = blockIdx.y, b = blockIdx.z, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int n = clamp_len(a.g, b), stay = stay_of(a, b, n);
    const Slices sl(n > 0 ? n : 1, stay, s.slices);
    if (n == stay || (int)blockIdx.x >= sl.count) return;
    const int64_t total = a.g.seq_pos[b], unit = (int64_t)b * a.g.n_kv + kv;
    const UnitInfo *u = s.info + unit;
    if (u->slice[blockIdx.x].in_bin == 0) return;
    int32_t *out = a.moves + moves_of(a.cap, unit) + 1;
    uint32_t *keys = s.keys(unit);
    int first = u->slice[blockIdx.x].first;
    const bool among_safe = u->among_safe != 0;
    const uint32_t bin = (uint32_t)u->bin;
    int parity = 0;
    const int end = sl.end((int)blockIdx.x, n, stay);
    slice_rows(a, b, kv, sl.begin((int)blockIdx.x, stay), end, [&](int j, const Four &r) {
        uint32_t bits = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e)
            bits |= j + e < end && (r.there >> e & 1) && is_safe(a, total, r.pos[e]) == among_safe && weight_key(r.w[e]) >> (32 - TOP) == bin ? 1u << e : 0u;
        const uint32_t c = (uint32_t)__popc(bits), up = wave_scan(c);
        if (lane == 63) red[parity][wave] = up;
        __syncthreads();
        int at = first + (int)(up - c);
#pragma unroll
        for (int i = 0; i < ST / 64; ++i) {
            at += i < wave ? (int)red[parity][i] : 0;
            first += (int)red[parity][i];
        }
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (bits >> e & 1) {
                out[at] = j + e;
                if (at < PICK) {
                    keys[at] = weight_key(r.w[e]);
                    keys[PICK + at] = pos_key(r.pos[e]);
                }
                ++at;
            }
        parity ^= 1;
    });
}

__global__ __launch_bounds__(1024) void slice_pick_kernel(SliceArgs s) {
    const PagedEvictArgs &a = s.e;
    __shared__ DescentLds<1024> lds;
    __shared__ uint32_t cw[PICK], cp[PICK];
    __shared__ int kept[SLICES + 2];
    __shared__ int last_slot;
    const int kv = blockIdx.x, b = blockIdx.y, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int n = clamp_len(a.g, b), stay = stay_of(a, b, n);
    const int64_t unit = (int64_t)b * a.g.n_kv + kv;
    int32_t *list = a.moves + moves_of(a.cap, unit);
    if (n == stay) {
        if (tid == 0) list[0] = 0;
        return;
    }
    const Slices sl(n, stay, s.slices);
    UnitInfo *u = s.info + unit;
    const int count = u->candidates, left = u->left;
    for (int i = tid; i < 2 * BINS; i += 1024) (&lds.hist[0][0])[i] = 0;
    if (tid < SLICES + 2) kept[tid] = 0;
    if (tid == 0) last_slot = 0x7fffffff;
    auto row = [&](int i, uint32_t &w, uint32_t &p) {              // candidate i's keys
        if (i < PICK) {
            w = cw[i];
            p = cp[i];
            return;
        }
        int block, place;
        split_slot(a.g, list[1 + i], block, place);
        const int page = page_of(a.g, b, block);                   // a candidate's block has one
        const int64_t at = table_index(a.g, page < 0 ? 0 : page, kv, place);
        w = weight_key(a.weight_in[at]);
        p = pos_key(a.pos_in[at]);
    };
    const uint32_t *keys = s.keys(unit);
#pragma unroll
    for (int i = tid; i < PICK; i += 1024)
        if (i < count) {
            cw[i] = keys[i];
            cp[i] = keys[PICK + i];
        }
    __syncthreads();
    Last last = {~0u, ~0u, 0};
    if (left > 0) {
        Spread sp = {0, 0, 0, 0, 0};
        for (int i = tid; i < count; i += 1024) {
            uint32_t w, p;
            row(i, w, p);
            sp.add(w, p, true);
        }
        sp.any_w = wave_or(sp.any_w);
        sp.not_all_w = wave_or(sp.not_all_w);
        sp.any_p = wave_or(sp.any_p);
        sp.not_all_p = wave_or(sp.not_all_p);
        if (lane == 0) {
            lds.red[1][wave] = sp.any_w;
            lds.red[2][wave] = sp.not_all_w;
            lds.red[3][wave] = sp.any_p;
            lds.red[4][wave] = sp.not_all_p;
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            sp.any_w |= lds.red[1][i];
            sp.not_all_w |= lds.red[2][i];
            sp.any_p |= lds.red[3][i];
            sp.not_all_p |= lds.red[4][i];
        }
        last = descend<1024>(lds, sp, left, [&](auto f) {
            for (int i = tid; i < count; i += 1024) {
                uint32_t w, p;
                row(i, w, p);
                f(w, p);
            }
        });
        if (last.ties != 0x7fffffff) {                             // the slot of the last of the equals that stay: candidates are in slot order
            int before = 0;
            for (int base = 0; base < count; base += 1024) {
                const int i = base + tid;
                uint32_t w = 0, p = 0;
                if (i < count) row(i, w, p);
                const bool tie = i < count && standing(last, w, p) == 1;
                const uint32_t up = wave_scan(tie);
                __syncthreads();
                if (lane == 63) lds.red[0][wave] = up;
                __syncthreads();
                int at = before + (int)up;
#pragma unroll
                for (int x = 0; x < 16; ++x) {
                    at += x < wave ? (int)lds.red[0][x] : 0;
                    before += (int)lds.red[0][x];
                }
                if (tie && at == last.ties) last_slot = list[1 + i];
            }
        }
    }
    __syncthreads();
    const int ls = last_slot;
    if (left > 0)
        for (int i = tid; i < count; i += 1024) {
            uint32_t w, p;
            row(i, w, p);
            const int st = standing(last, w, p), slot = list[1 + i];
            if (st == 2 || (st == 1 && slot <= ls)) atomicAdd(&kept[sl.of(slot, stay)], 1);
        }
    __syncthreads();
    if (tid < 64) {
        const int begin = sl.begin(tid, stay), rows = tid < sl.count ? sl.end(tid, n, stay) - begin - u->slice[tid].gone : 0;
        const int k = tid < sl.count ? u->slice[tid].kept + kept[tid] : 0;
        const uint32_t free_here = tid < sl.low ? (uint32_t)(rows - k) : 0, move_here = tid >= sl.low ? (uint32_t)k : 0;
        const uint32_t f = wave_scan(free_here), m = wave_scan(move_here);
        if (tid < sl.count) u->slice[tid].at = (int32_t)(tid < sl.low ? f - free_here : m - move_here);
        if (tid == 63) {
            u->last_w = last.w;
            u->last_p = last.p;
            u->last_slot = ls;
            list[0] = (int32_t)m;
        }
    }
}

__global__ __launch_bounds__(ST) void slice_list_kernel(SliceArgs s) {
    const PagedEvictArgs &a = s.e;
    __shared__ uint32_t red[2][ST / 64];
    const int kv = blockIdx.y, b = blockIdx.z, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int n = clamp_len(a.g, b), stay = stay_of(a, b, n);
    const Slices sl(n > 0 ? n : 1, stay, s.slices);
    if ((int)blockIdx.x >= sl.count) return;
    const int begin = sl.begin((int)blockIdx.x, stay), end = sl.end((int)blockIdx.x, n, stay);
    const bool low = (int)blockIdx.x < sl.low;
    if (low && a.pos_out != a.pos_in)
        for (int j = begin + 4 * tid; j < end; j += 4 * ST) copy_entries(a, b, kv, j, end);
    if (n == stay) return;
    const int64_t total = a.g.seq_pos[b], unit = (int64_t)b * a.g.n_kv + kv;
    const UnitInfo *u = s.info + unit;
    const bool among_safe = u->among_safe != 0, any_left = u->left > 0;
    const uint32_t bin = (uint32_t)u->bin;
    const Last last = {u->last_w, u->last_p, 0};
    const int last_slot = u->last_slot;
    int32_t *out = a.moves + moves_of(a.cap, unit) + 1 + (low ? 0 : a.cap) + u->slice[blockIdx.x].at;
    int parity = 0;
    slice_rows(a, b, kv, begin, end, [&](int j, const Four &r) {
        uint32_t bits = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const uint32_t w = weight_key(r.w[e]);
            bool kept;
            if (is_safe(a, total, r.pos[e]) != among_safe) {
                kept = !among_safe;
            } else if (!any_left || w >> (32 - TOP) != bin) {
                kept = any_left && w >> (32 - TOP) > bin;
            } else {
                const int st = standing(last, w, pos_key(r.pos[e]));
                kept = st == 2 || (st == 1 && j + e <= last_slot);
            }
            bits |= j + e < end && (r.there >> e & 1) && kept != low ? 1u << e : 0u;
        }
        const uint32_t c = (uint32_t)__popc(bits), up = wave_scan(c);
        if (lane == 63) red[parity][wave] = up;
        __syncthreads();
        uint32_t at = up - c, all = 0;
#pragma unroll
        for (int i = 0; i < ST / 64; ++i) {
            at += i < wave ? red[parity][i] : 0;
            all += red[parity][i];
        }
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (bits >> e & 1) out[at++] = j + e;
        out += all;
        parity ^= 1;
    });
}

// grid = (kv heads, sequences, ENTRIES + workgroups per unit): the first ones bring the tables' entries
static constexpr int ENTRIES = 4;
__global__ __launch_bounds__(256) void paged_move_kernel(PagedEvictArgs a) {
    const int kv = blockIdx.x, b = blockIdx.y, z = (int)blockIdx.z - ENTRIES, tid = threadIdx.x;
    const int32_t *list = a.moves + moves_of(a.cap, (int64_t)b * a.g.n_kv + kv);
    if (z < 0) move_entries(a, b, kv, list + 1, list + 1 + a.cap, list[0], (int)blockIdx.z * 256 + tid, ENTRIES * 256);
    else move_rows<2>(a, b, kv, list + 1, list + 1 + a.cap, list[0], z * 256 + tid, ((int)gridDim.z - ENTRIES) * 256);
}

// ---- launch shapes and memory ------------------------------------------------------------------------------------------------

struct EvictShape {
    int cap, slices;                                               // slices: 0 where a unit is one workgroup's
    bool move_here;                                                // the unit's workgroup moves its rows, from lists in LDS
    size_t moves, hist, info;
};

static EvictShape evict_shape(const ssd_paged_config *c, int max_len) {
    EvictShape s;
    const int reach = paged_reach(c, max_len);
    const int64_t units = (int64_t)c->n_seqs * c->n_kv_heads;
    s.cap = reach / 2 + 1;
    s.slices = 0;
    if (reach > 16384) {
        const int64_t rows = (reach + 4095) / 4096, share = 2048 / units + 1;
        s.slices = (int)(rows < share ? rows : share);
        if (s.slices > SLICES) s.slices = SLICES;
    }
    // Rows move by the unit's workgroup, which saves a launch, where units fill the chip (one eviction from each of 64 units of 2000 rows 7.5 us here and 9.2 by a launch, 1000 32.9 and
    // 17.0; 128 units 39 and 28, 256 42.6 and 43.4, of 8000 rows to 4000 137 and 156); with few rows, from 128 units on (one of 129 rows 6.3 and 8.2, 100 of 250 stay 16.7 and 14.0).
    s.move_here = units >= (reach <= 256 ? 128 : 256) && !s.slices;
    s.moves = s.move_here ? 0 : round256((size_t)moves_of(s.cap, units) * 4);
    s.hist = s.slices ? (size_t)units * (s.slices + 2) * 2 * TOP_BINS * 4 : 0;
    s.info = s.slices ? round256((size_t)units * sizeof(UnitInfo)) : 0;
    return s;
}

}  // namespace ssd

using namespace ssd;

extern "C" size_t ssd_paged_evict_workspace_bytes(const ssd_paged_config *cfg, int max_len) {
    clear_error();
    if (check_paged(cfg) != SSD_OK || check_max_len(cfg, max_len) != SSD_OK) return 0;
    const EvictShape s = evict_shape(cfg, max_len);
    return s.moves + s.hist + s.info;
}

extern "C" int ssd_paged_evict(const ssd_paged_config *cfg, void *k_pages, void *v_pages, const int32_t *block_table, const int32_t *seq_len,
                               const int32_t *seq_pos, const int32_t *budget, int n_sink, int recent, const int32_t *pos_in, int32_t *pos_out,
                               const float *weight_in, float *weight_out, int32_t *seq_len_out, int max_len, void *workspace,
                               size_t workspace_bytes, void *stream) {
    clear_error();
    int rc = check_paged(cfg);
    if (rc != SSD_OK) return rc;
    if ((rc = check_max_len(cfg, max_len)) != SSD_OK) return rc;
    if (!k_pages || !v_pages || !aligned(k_pages, 16) || !aligned(v_pages, 16))
        return fail(SSD_ERR_INVALID_ARG, "k_pages and v_pages must be given, 16-byte aligned");
    if (!block_table || !seq_len || !budget) return fail(SSD_ERR_INVALID_ARG, "block_table, seq_len or budget is NULL");
    if (!pos_in || !pos_out || !weight_in || !weight_out) return fail(SSD_ERR_INVALID_ARG, "pos_in, pos_out, weight_in or weight_out is NULL");
    if ((pos_in == pos_out) != (weight_in == weight_out)) return fail(SSD_ERR_INVALID_ARG, "both tables are updated in place, or neither");
    if (seq_len_out && (seq_len_out == seq_len || seq_len_out == seq_pos || seq_len_out == budget))
        return fail(SSD_ERR_INVALID_ARG, "seq_len_out must not be seq_len, seq_pos or budget");
    if (n_sink < 0 || recent < 0) return fail(SSD_ERR_INVALID_ARG, "n_sink=%d and recent=%d must be >= 0", n_sink, recent);
    const void *all[] = {block_table, seq_len, seq_pos, budget, pos_in, pos_out, weight_in, weight_out, seq_len_out};
    for (const void *x : all)
        if (!aligned(x, 4)) return fail(SSD_ERR_INVALID_ARG, "tables must be aligned to their elements");
    const EvictShape shape = evict_shape(cfg, max_len);
    const size_t need = shape.moves + shape.hist + shape.info;
    if (need > 0 && (!workspace || !aligned(workspace, 256) || workspace_bytes < need))
        return fail(SSD_ERR_INVALID_ARG, "workspace of %zu bytes, 256-byte aligned, needed; %zu given", need, workspace_bytes);
    PagedEvictArgs a;
    a.g = paged_geom(cfg, block_table, seq_len, seq_pos, max_len);
    a.k_pages = static_cast<char *>(k_pages);
    a.v_pages = static_cast<char *>(v_pages);
    a.budget = budget;
    a.pos_in = pos_in;
    a.weight_in = weight_in;
    a.pos_out = pos_out;
    a.weight_out = weight_out;
    a.len_out = seq_len_out;
    a.moves = static_cast<int32_t *>(workspace);
    a.n_sink = n_sink;
    a.recent = recent;
    a.cap = shape.cap;
    a.lpr_log2 = __builtin_ctz((unsigned)((size_t)cfg->head_dim * paged_esize(cfg) / 16));
    hipStream_t s = static_cast<hipStream_t>(stream);
    const dim3 units((unsigned)a.g.n_kv, (unsigned)a.g.n_seqs);
    const int64_t n_units = (int64_t)units.x * units.y;
    const int reach = a.g.max_len;
    const int move_here = shape.move_here;
    // A wave, 256 or 1024 threads per unit: the next larger take 15.6 us instead of 11.5 (12 of 200 rows, 64 units), 18.0 and 17.0 (half of 2000 rows, 32 units; 39.5 and 42.6 with 256), 38.7 and
    // 32.0 (half of 8000); slices from 8192 rows on 38.1 and 29.2 (one of 16000 rows, 32 units; 346 and 305 for half of them, 256).
    if (shape.slices) {
        SliceArgs sa;
        sa.e = a;
        char *ws = static_cast<char *>(workspace);
        sa.hist = reinterpret_cast<uint32_t *>(ws + shape.moves);
        sa.info = reinterpret_cast<UnitInfo *>(ws + shape.moves + shape.hist);
        sa.slices = shape.slices;
        const dim3 slices((unsigned)shape.slices + 2, units.x, units.y);
        hipLaunchKernelGGL(slice_count_kernel, slices, dim3(ST), 0, s, sa);
        hipLaunchKernelGGL(slice_bin_kernel, units, dim3(1024), 0, s, sa);
        hipLaunchKernelGGL(slice_gather_kernel, slices, dim3(ST), 0, s, sa);
        hipLaunchKernelGGL(slice_pick_kernel, units, dim3(1024), 0, s, sa);
        hipLaunchKernelGGL(slice_list_kernel, slices, dim3(ST), 0, s, sa);
    } else if (reach <= 256) hipLaunchKernelGGL((paged_select_kernel<64, 4>), units, dim3(64), 0, s, a, move_here);
    else if (reach <= 2048) hipLaunchKernelGGL((paged_select_kernel<256, 8>), units, dim3(256), 0, s, a, move_here);
    else if (reach <= 8192) hipLaunchKernelGGL((paged_select_kernel<1024, 8>), units, dim3(1024), 0, s, a, move_here);
    else hipLaunchKernelGGL((paged_select_kernel<1024, 16>), units, dim3(1024), 0, s, a, move_here);
    if (!move_here) {
        const int64_t pieces = (a.cap + 31) / 32, enough = 4096 / n_units + 1;
        hipLaunchKernelGGL(paged_move_kernel, dim3(units.x, units.y, (unsigned)(ENTRIES + (pieces < enough ? pieces : enough))), dim3(256), 0, s, a);
    }
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? SSD_OK : hip_fail(e, "paged eviction launch");
}
