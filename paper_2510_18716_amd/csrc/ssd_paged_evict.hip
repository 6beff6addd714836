// ssd_paged_evict: each (sequence, kv head) of a paged cache is cut to its budget; the rows of the largest accumulated attention weight
// stay (the top-M rule of Algorithm 1, sinks and recent tokens protected as in Sec. 3.3).
//
// A unit's selection is one workgroup's: the key of the last row that stays is found by a descent over the keys' bits (weight first,
// then position; whole-number compares, so the set is exact), eight bits a step by a histogram in LDS, beginning at the first bit in which the
// weights differ.  Up to 16384 rows a thread keeps its rows' keys in registers, and the tables are read once; longer units are read anew for every
// step, eleven bits each.  Then every thread ranks its free slots below n' and its kept rows above by one scan over the workgroup, and the rows
// move, in 16-byte fragments: by the same workgroup where units are many, by a second launch with more workgroups per unit otherwise.
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

struct Four { float w[4]; int pos[4]; };

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
            r.w[e] = page < 0 ? __uint_as_float(0x7fc00000u) : w[e];
            r.pos[e] = page < 0 ? 0 : p[e];
        }
        return r;
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        r.w[e] = __uint_as_float(0x7fc00000u);
        r.pos[e] = 0;
        if (j + e < n) {
            split_slot(a.g, j + e, block, place);
            const int page = page_of(a.g, b, block);
            if (page >= 0) {
                const int64_t i = table_index(a.g, page, kv, place);
                r.w[e] = a.weight_in[i];
                r.pos[e] = a.pos_in[i];
            }
        }
    }
    return r;
}

static __device__ __forceinline__ uint32_t wave_sum(uint32_t v) {
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) v += (uint32_t)__shfl_xor((int)v, o);
    return v;
}
static __device__ __forceinline__ uint32_t wave_scan(uint32_t v) {
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const uint32_t w = (uint32_t)__shfl_up((int)v, o);
        v += lane >= o ? w : 0;
    }
    return v;
}

// Rows from[i] to slots to[i], i = first, first + step, ..; K and V of a row by neighbouring threads, their table entries by the first of them.
// A thread has MOVES rows' loads in flight at each of the three stages (list, block table, row); past the end it repeats the last row, which
// writes the same again.
static constexpr int MOVES = 8;
static __device__ __forceinline__ void move_rows(const PagedEvictArgs &a, int b, int kv, const int32_t *to, const int32_t *from, int count, int thread,
                                                 int threads) {
    const int lanes = 2 << a.lpr_log2, lane = thread & (lanes - 1), step = threads / lanes;
    const bool v = lane >> a.lpr_log2;
    const int64_t sub = (int64_t)kv * a.g.head_stride + (int64_t)(lane & ((1 << a.lpr_log2) - 1)) * 16;
    char *pool = (v ? a.v_pages : a.k_pages) + sub;
    for (int i0 = thread / lanes; i0 < count; i0 += MOVES * step) {
        int t[MOVES], f[MOVES], tp[MOVES], fp[MOVES], pages[2][MOVES];
#pragma unroll
        for (int m = 0; m < MOVES; ++m) {
            const int i = i0 + m * step < count ? i0 + m * step : count - 1;
            t[m] = to[i];
            f[m] = from[i];
        }
#pragma unroll
        for (int m = 0; m < MOVES; ++m) {
            int block;
            split_slot(a.g, t[m], block, tp[m]);
            pages[0][m] = page_of(a.g, b, block);
            split_slot(a.g, f[m], block, fp[m]);
            pages[1][m] = page_of(a.g, b, block);
        }
        u32x4_nt_t x[MOVES];
        float w[MOVES];
        int p[MOVES];
#pragma unroll
        for (int m = 0; m < MOVES; ++m) {
            const int page = pages[1][m] < 0 ? 0 : pages[1][m];
            x[m] = __builtin_nontemporal_load(reinterpret_cast<const u32x4_nt_t *>(pool + (int64_t)page * a.g.page_stride + (int64_t)fp[m] * a.g.row_stride));
            if (lane == 0) {
                const int64_t i = table_index(a.g, page, kv, fp[m]);
                w[m] = a.weight_in[i];
                p[m] = a.pos_in[i];
            }
        }
#pragma unroll
        for (int m = 0; m < MOVES; ++m)
            if (pages[0][m] >= 0 && pages[1][m] >= 0) {
                *reinterpret_cast<u32x4_nt_t *>(pool + (int64_t)pages[0][m] * a.g.page_stride + (int64_t)tp[m] * a.g.row_stride) = x[m];
                if (lane == 0) {
                    const int64_t i = table_index(a.g, pages[0][m], kv, tp[m]);
                    a.weight_out[i] = w[m];
                    a.pos_out[i] = p[m];
                }
            }
    }
}

// KEYS: rows whose keys a thread keeps, consecutive ones; 0: none, the tables are read again for every step.  grid = (kv heads, sequences)
template <int THREADS, int KEYS>
__global__ __launch_bounds__(THREADS) void paged_select_kernel(PagedEvictArgs a, int move_here) {
    constexpr int NW = THREADS / 64, BITS = KEYS ? 8 : 11, BINS = 1 << BITS, LEVELS = 2 * ((32 + BITS - 1) / BITS);
    constexpr int HISTS = KEYS ? LEVELS : 1;                        // one histogram per step, or one that is cleared in between
    __shared__ uint32_t hist[HISTS][BINS];
    __shared__ uint32_t red[3][NW];
    const int kv = blockIdx.x, b = blockIdx.y, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int n = clamp_len(a.g, b);
    const int want = a.budget[b] < 0 ? 0 : a.budget[b];
    const int stay = n < want ? n : want;
    const bool copy = a.pos_out != a.pos_in;
    const int64_t total = a.g.seq_pos[b];
    int32_t *list = a.moves + moves_of(a.cap, (int64_t)b * a.g.n_kv + kv);
    if (kv == 0 && tid == 0 && a.len_out) a.len_out[b] = stay;
    if (n == stay && !copy) {
        if (tid == 0) list[0] = 0;
        return;
    }
    for (int i = tid; i < HISTS * BINS; i += THREADS) (&hist[0][0])[i] = 0;

    // what a thread looks at: its own rows in registers, or all rows of the unit with stride THREADS * 4, read again
    uint32_t wk[KEYS ? KEYS : 1], pk[KEYS ? KEYS : 1], safe_bits = 0;
    auto is_safe = [&](int pos) { return pos < a.n_sink || (int64_t)pos >= total - a.recent; };
    if constexpr (KEYS > 0) {
#pragma unroll
        for (int k = 0; k < KEYS; k += 4) {
            const int j = tid * KEYS + k;
            if (j < n) {
                const Four r = table_rows(a, b, kv, j, n);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    wk[k + e] = weight_key(r.w[e]);
                    pk[k + e] = pos_key(r.pos[e]);
                    safe_bits |= is_safe(r.pos[e]) ? 1u << (k + e) : 0u;
                }
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e) wk[k + e] = pk[k + e] = 0;
            }
        }
    }
    auto each = [&](auto f) {                                      // f(weight key, position key, safe)
        if constexpr (KEYS > 0) {
#pragma unroll
            for (int k = 0; k < KEYS; ++k)
                if (tid * KEYS + k < n) f(wk[k], pk[k], (safe_bits >> k & 1) != 0);
        } else {
#pragma unroll 2
            for (int j = 4 * tid; j < n; j += 4 * THREADS) {
                const Four r = table_rows(a, b, kv, j, n);
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (j + e < n) f(weight_key(r.w[e]), pos_key(r.pos[e]), is_safe(r.pos[e]));
            }
        }
    };

    // which rows compete and for how many places; the bits in which the weights of each kind differ
    uint32_t last_w = 0, last_p = 0;                               // keys of the last row that stays
    int ties = 0;                                                  // how many rows with just these keys stay
    bool among_safe = false, compete = false;
    if (stay < n && stay > 0) {
        uint32_t safe_rows = 0, or_s = 0, and_s = ~0u, or_o = 0, and_o = ~0u;
        each([&](uint32_t w, uint32_t, bool safe) {
            safe_rows += safe;
            or_s |= safe ? w : 0;
            and_s &= safe ? w : ~0u;
            or_o |= safe ? 0 : w;
            and_o &= safe ? ~0u : w;
        });
        safe_rows = wave_sum(safe_rows);
        if (lane == 0) red[0][wave] = safe_rows;
        __syncthreads();
        safe_rows = 0;
#pragma unroll
        for (int i = 0; i < NW; ++i) safe_rows += red[0][i];
        among_safe = (int)safe_rows >= stay;
        int left = among_safe ? stay : stay - (int)safe_rows;
        compete = left > 0;
        uint32_t any = among_safe ? or_s : or_o, every = among_safe ? and_s : and_o;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            any |= (uint32_t)__shfl_xor((int)any, o);
            every &= (uint32_t)__shfl_xor((int)every, o);
        }
        if (lane == 0) {
            red[1][wave] = any;
            red[2][wave] = every;
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < NW; ++i) {
            any |= red[1][i];
            every &= red[2][i];
        }
        const uint32_t differ = any ^ every;
        int bits = differ ? 32 - __clz((int)differ) : 0;           // bits of the weight still open
        last_w = bits == 32 ? 0 : every >> bits << bits;
        bool on_pos = bits == 0, whole = false;
        if (on_pos) bits = 32;
        for (int level = 0; compete && !whole; ++level) {
            const int take = bits < BITS ? bits : BITS, shift = bits - take;
            uint32_t *h = hist[KEYS ? level : 0];
            const uint32_t mask = (1u << take) - 1;
            each([&](uint32_t w, uint32_t p, bool safe) {
                const uint32_t key = on_pos ? p : w, ref = on_pos ? last_p : last_w;
                const bool in = safe == among_safe && (!on_pos || w == last_w) && (bits == 32 || key >> bits == ref >> bits);
                if (in) atomicAdd(&h[key >> shift & mask], 1u);
            });
            __syncthreads();
            // the digit in which the place falls: every wave adds up the bins from the top, BINS / 64 a lane
            constexpr int PER = BINS / 64;
            uint32_t sum = 0, mine[PER];
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                mine[i] = h[BINS - 1 - (lane * PER + i)];
                sum += mine[i];
            }
            const uint32_t upto = wave_scan(sum);
            const int l = __ffsll((unsigned long long)__ballot(upto >= (uint32_t)left)) - 1;
            uint32_t above = upto - sum, in_bin = 0;
            int digit = 0;
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                const bool here = above < (uint32_t)left && above + mine[i] >= (uint32_t)left;
                if (here && in_bin == 0) {
                    digit = BINS - 1 - (lane * PER + i);
                    in_bin = mine[i];
                }
                if (in_bin == 0) above += mine[i];
            }
            digit = __builtin_amdgcn_readlane(digit, l);
            above = (uint32_t)__builtin_amdgcn_readlane((int)above, l);
            in_bin = (uint32_t)__builtin_amdgcn_readlane((int)in_bin, l);
            left -= (int)above;
            if (on_pos) last_p |= (uint32_t)digit << shift;
            else last_w |= (uint32_t)digit << shift;
            bits = shift;
            whole = (int)in_bin == left;                           // all of them stay: nothing below needs looking at
            if (bits == 0) {
                if (on_pos) break;
                on_pos = true;
                bits = 32;
            }
            if constexpr (KEYS == 0) {
                if (!whole) {
                    __syncthreads();
                    for (int i = tid; i < BINS; i += THREADS) hist[0][i] = 0;
                    __syncthreads();
                }
            }
        }
        ties = whole ? n : left;
    }
    // Rows above the last one's keys stay; so do those equal to them while there are ties left.  Where the descent ended early, the bits
    // below are 0 in the last keys, and everything at or above them stays.
    auto level_of = [&](uint32_t w, uint32_t p) {                  // 2: stays, 1: equal, 0: goes
        if (w != last_w) return w > last_w ? 2 : 0;
        return p > last_p ? 2 : p == last_p ? 1 : 0;
    };

    // who stays, where slots become free, which rows move
    constexpr int HAVE = KEYS ? KEYS : 4;
    uint32_t seen_tie = 0, seen_free = 0, seen_move = 0;
    for (int base = 0; base < n; base += THREADS * HAVE) {
        const int j0 = base + tid * HAVE;
        uint32_t kept = 0, tie = 0;
        Four r;
        if constexpr (KEYS == 0) {
            if (j0 < n) r = table_rows(a, b, kv, j0, n);
        }
#pragma unroll
        for (int k = 0; k < HAVE; ++k) {
            if (j0 + k >= n) continue;
            bool safe;
            uint32_t w, p;
            if constexpr (KEYS > 0) {
                safe = safe_bits >> k & 1;
                w = wk[k];
                p = pk[k];
            } else {
                safe = is_safe(r.pos[k]);
                w = weight_key(r.w[k]);
                p = pos_key(r.pos[k]);
            }
            int lv = stay == n ? 2 : stay == 0 ? 0 : safe != among_safe ? (safe ? 2 : 0) : compete ? level_of(w, p) : 0;
            kept |= lv == 2 ? 1u << k : 0u;
            tie |= lv == 1 ? 1u << k : 0u;
        }
        if (stay < n) {
            if (ties >= n) {
                kept |= tie;
            } else {                                               // equal keys: the lowest slots
                const uint32_t c = (uint32_t)__popc(tie), up = wave_scan(c);
                __syncthreads();
                if (lane == 63) red[0][wave] = up;
                __syncthreads();
                uint32_t before = seen_tie + up - c;
#pragma unroll
                for (int i = 0; i < NW; ++i) {
                    before += i < wave ? red[0][i] : 0;
                    seen_tie += red[0][i];
                }
#pragma unroll
                for (int k = 0; k < HAVE; ++k)
                    if (tie >> k & 1) {
                        kept |= (int)before < ties ? 1u << k : 0u;
                        ++before;
                    }
            }
            const int below = stay - j0 < 0 ? 0 : stay - j0 < HAVE ? stay - j0 : HAVE, there = n - j0 < 0 ? 0 : n - j0 < HAVE ? n - j0 : HAVE;
            const uint32_t low = below == 32 ? ~0u : (1u << below) - 1, in = there == 32 ? ~0u : (1u << there) - 1;
            const uint32_t free_bits = in & low & ~kept, move_bits = kept & ~low;
            const uint32_t c = (uint32_t)__popc(free_bits) | (uint32_t)__popc(move_bits) << 16, up = wave_scan(c);
            __syncthreads();
            if (lane == 63) red[1][wave] = up;
            __syncthreads();
            uint32_t before = up - c, all = 0;
#pragma unroll
            for (int i = 0; i < NW; ++i) {
                before += i < wave ? red[1][i] : 0;
                all += red[1][i];
            }
            uint32_t f = seen_free + (before & 0xffff), m = seen_move + (before >> 16);
            seen_free += all & 0xffff;
            seen_move += all >> 16;
#pragma unroll
            for (int k = 0; k < HAVE; ++k) {
                if (free_bits >> k & 1) list[1 + f++] = j0 + k;
                if (move_bits >> k & 1) list[1 + a.cap + m++] = j0 + k;
            }
        }
        // the tables' entries of slots below n'; those of free slots are written again with the rows that move there
        if (copy) {
            typedef float f4 __attribute__((ext_vector_type(4), aligned(4)));
            typedef int i4 __attribute__((ext_vector_type(4), aligned(4)));
#pragma unroll
            for (int k = 0; k < HAVE; k += 4) {
                const int j = j0 + k;
                int block, place;
                if (j >= stay) continue;
                split_slot(a.g, j, block, place);
                const int page = page_of(a.g, b, block);
                const int64_t i = table_index(a.g, page, kv, place);
                if (place + 4 <= a.g.page_size && j + 4 <= stay) {
                    if (page < 0) continue;
                    *reinterpret_cast<f4 *>(a.weight_out + i) = *reinterpret_cast<const f4 *>(a.weight_in + i);
                    *reinterpret_cast<i4 *>(a.pos_out + i) = *reinterpret_cast<const i4 *>(a.pos_in + i);
                } else {
                    for (int e = 0; e < 4 && j + e < stay; ++e) {
                        split_slot(a.g, j + e, block, place);
                        const int pg = page_of(a.g, b, block);
                        if (pg < 0) continue;
                        const int64_t at = table_index(a.g, pg, kv, place);
                        a.pos_out[at] = a.pos_in[at];
                        a.weight_out[at] = a.weight_in[at];
                    }
                }
            }
        }
    }
    if (tid == 0) list[0] = (int32_t)seen_move;
    if (move_here && seen_move > 0) {
        __syncthreads();
        move_rows(a, b, kv, list + 1, list + 1 + a.cap, (int)seen_move, tid, THREADS);
    }
}

// grid = (kv heads, sequences, workgroups per unit)
__global__ __launch_bounds__(256) void paged_move_kernel(PagedEvictArgs a) {
    const int kv = blockIdx.x, b = blockIdx.y;
    const int32_t *list = a.moves + moves_of(a.cap, (int64_t)b * a.g.n_kv + kv);
    move_rows(a, b, kv, list + 1, list + 1 + a.cap, list[0], (int)(blockIdx.z * 256 + threadIdx.x), (int)gridDim.z * 256);
}

static int evict_cap(const ssd_paged_config *c, int max_len) { return paged_reach(c, max_len) / 2 + 1; }

}  // namespace ssd

using namespace ssd;

extern "C" size_t ssd_paged_evict_workspace_bytes(const ssd_paged_config *cfg, int max_len) {
    clear_error();
    if (check_paged(cfg) != SSD_OK || check_max_len(cfg, max_len) != SSD_OK) return 0;
    return round256((size_t)moves_of(evict_cap(cfg, max_len), (int64_t)cfg->n_seqs * cfg->n_kv_heads) * 4);
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
    if (seq_len_out == seq_len) return fail(SSD_ERR_INVALID_ARG, "seq_len_out must not be seq_len");
    if (n_sink < 0 || recent < 0) return fail(SSD_ERR_INVALID_ARG, "n_sink=%d and recent=%d must be >= 0", n_sink, recent);
    const void *all[] = {block_table, seq_len, seq_pos, budget, pos_in, pos_out, weight_in, weight_out, seq_len_out};
    for (const void *x : all)
        if (!aligned(x, 4)) return fail(SSD_ERR_INVALID_ARG, "tables must be aligned to their elements");
    const size_t need = ssd_paged_evict_workspace_bytes(cfg, max_len);
    if (!workspace || !aligned(workspace, 256) || workspace_bytes < need)
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
    a.cap = evict_cap(cfg, max_len);
    a.lpr_log2 = __builtin_ctz((unsigned)((size_t)cfg->head_dim * paged_esize(cfg) / 16));
    hipStream_t s = static_cast<hipStream_t>(stream);
    const dim3 units((unsigned)a.g.n_kv, (unsigned)a.g.n_seqs);
    const int64_t n_units = (int64_t)units.x * units.y;
    const int move_here = n_units >= 128;
    const int reach = a.g.max_len;
    if (reach <= 256) hipLaunchKernelGGL((paged_select_kernel<64, 4>), units, dim3(64), 0, s, a, move_here);
    else if (reach <= 2048) hipLaunchKernelGGL((paged_select_kernel<256, 8>), units, dim3(256), 0, s, a, move_here);
    else if (reach <= 8192) hipLaunchKernelGGL((paged_select_kernel<1024, 8>), units, dim3(1024), 0, s, a, move_here);
    else if (reach <= 16384) hipLaunchKernelGGL((paged_select_kernel<1024, 16>), units, dim3(1024), 0, s, a, move_here);
    else hipLaunchKernelGGL((paged_select_kernel<1024, 0>), units, dim3(1024), 0, s, a, move_here);
    if (!move_here) {
        const int64_t pieces = (a.cap + 31) / 32, enough = 2048 / n_units + 1;
        hipLaunchKernelGGL(paged_move_kernel, dim3(units.x, units.y, (unsigned)(pieces < enough ? pieces : enough)), dim3(256), 0, s, a);
    }
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? SSD_OK : hip_fail(e, "paged eviction launch");
}
