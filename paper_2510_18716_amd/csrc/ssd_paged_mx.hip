// ssd_paged_mx_append: new tokens' rows into the pages of a cache held in 8 or 4 bits, quantised on the way.  ssd_paged_mx_read: rows of the cache back
// in the calls' type.
//
// Both are bound by HBM, the wide side by far: 256 bytes of bf16 for 64 + 4 of codes and scales.  A lane has eight elements, 16 bytes (fp32: 32) on the wide side and 4 or
// 8 on the narrow one; the four lanes of a block find its largest element by two lane exchanges.  Scales meet in LDS and leave with the tables' entries, a
// page's places by neighbouring threads.  22500 tokens of 32 heads of 128 elements (369 MB of bf16) into four bits and back 162 us, 5.8 TB/s read and written (a
// plain copy 5.45); 557 MB from eight bits 103 us, 5.4.  A few tokens: 3.5 us each way, launch and dependent loads.
#include "ssd_mx.h"
#include "ssd_paged_mx.h"

namespace ssd {

struct MxRowsArgs {
    PagedGeom g;
    char *k_pages, *v_pages;
    uint8_t *k_scales, *v_scales;
    char *k, *v;             // the rows outside the cache
    const int32_t *start;    // a sequence's first row there, or NULL: one each
    const int32_t *first;    // read: its slot, or NULL: 0
    const float *weight_new;
    int32_t *pos;
    float *weight;
    int64_t stride;          // bytes from a token's row to the next's
    int n;
    int tokens_log2, lanes_log2;
};

static constexpr int STARTS = 1024;      // sequences whose first rows fit in LDS
static constexpr int TOKENS = 64;

// A workgroup takes a few consecutive tokens; a thread per token finds where it is in the cache.
struct Spots {
    int64_t row[TOKENS];     // byte offset of its place in the pool (head 0), negative: none
    int64_t entry[TOKENS];   // index of its entry in the tables (head 0)
    int32_t pos[TOKENS];
    int32_t starts[STARTS + 1];
};

// First token of a workgroup.  Workgroups go to the eight XCDs in turn; four neighbours' tokens go to one, as their rows and scales share cache lines (22500 tokens of 32
// heads of 128 elements written in four bits and read back in their order 172 us, by twos 166, fours 162, sixteens 165, the whole grid in eight runs 162, which costs reading
// 557 MB 103 -> 108; in eight bits, one line to a row, nothing changes).
static __device__ __forceinline__ int first_token(const MxRowsArgs &a) {
    const unsigned i = blockIdx.x;
    constexpr unsigned RUN = 4;
    if (i >= gridDim.x / (8 * RUN) * (8 * RUN)) return (int)(i << a.tokens_log2);
    return (int)((i / (8 * RUN) * (8 * RUN) + (i & 7) * RUN + (i >> 3) % RUN) << a.tokens_log2);
}

template <bool READ> static __device__ __forceinline__ void find_spots(const MxRowsArgs &a, int row0, Spots &sm) {
    const int tid = threadIdx.x, tokens = 1 << a.tokens_log2, row = row0 + tid;
    const bool in_lds = a.start && a.g.n_seqs <= STARTS;
    if (in_lds) {
        for (int i = tid; i <= a.g.n_seqs; i += 256) sm.starts[i] = a.start[i];
        __syncthreads();
    }
    if (tid < tokens) {
        int64_t at = -1, entry = 0;
        int p = 0;
        if (row < a.n) {
            int b = row, begin = row, count = 1;
            if (a.start) {
                const auto start = [&](int i) { return in_lds ? sm.starts[i] : a.start[i]; };
                b = sequence_of(a.g, row, start);
                begin = start(b);
                count = start(b + 1) - begin;
            }
            if (row >= begin && row - begin < count) {
                const int64_t from = READ ? (a.first ? a.first[b] : 0) : (int64_t)a.g.seq_len[b] - count, slot = from + (row - begin);
                if (slot >= 0 && slot < clamp_len(a.g, b)) {
                    int block, place;
                    split_slot(a.g, (int)slot, block, place);
                    const int page = page_of(a.g, b, block);
                    if (page >= 0) {
                        at = row_offset(a.g, page, 0, place);
                        entry = table_index(a.g, page, 0, place);
                        if (!READ) p = a.g.seq_pos[b] - count + (row - begin);
                    }
                }
            }
        }
        sm.row[tid] = at;
        sm.entry[tid] = entry;
        sm.pos[tid] = p;
    }
    __syncthreads();
}

// A thread's share of a workgroup's tokens: the q-th fragment of eight elements.
struct Share {
    int i, f;                // token, fragment of its heads
    __device__ __forceinline__ Share(const MxRowsArgs &a, int q, int lane, int per_token) {
        const int t = q / per_token;
        i = ((int)threadIdx.x >> a.lanes_log2) + (t << (8 - a.lanes_log2));
        f = lane + ((q - t * per_token) << a.lanes_log2);
    }
};

template <typename T, int D, int BITS> __global__ __launch_bounds__(256) void mx_append_kernel(MxRowsArgs a) {
    constexpr int PARTS = D / 8, SB = D / 32, U = 2;
    typedef std::conditional_t<SB == 4, uint32_t, uint16_t> scales_t;
    __shared__ Spots sm;
    extern __shared__ __align__(16) uint8_t sm_scale[];     // [K and V][kv heads][tokens][SB]
    const int tid = threadIdx.x, tokens = 1 << a.tokens_log2, row0 = first_token(a);
    const int lane = tid & ((1 << a.lanes_log2) - 1), step = 1 << a.lanes_log2, frags = a.g.n_kv * PARTS, per_token = (frags + step - 1) >> a.lanes_log2;
    const int mine = ((tokens + (256 >> a.lanes_log2) - 1) >> (8 - a.lanes_log2)) * per_token;
    // what a thread reads is on its way two fragments ahead, the first ones while the tokens' places are looked up
    Eight<T> k[U], v[U];
    const auto load = [&](int q) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const Share x(a, q + u, lane, per_token);
            const int row = row0 + x.i;
            const int64_t from = (int64_t)(row < a.n ? row : a.n - 1) * a.stride + (int64_t)(x.f < frags ? x.f : 0) * (8 * (int)sizeof(T));
            k[u] = load_eight<T>(a.k + from);
            v[u] = load_eight<T>(a.v + from);
        }
    };
    load(0);
    find_spots<false>(a, row0, sm);
    for (int q = 0; q < mine; q += U) {
        Eight<T> k0[U], v0[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            k0[u] = k[u];
            v0[u] = v[u];
        }
        if (q + U < mine) load(q + U);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const Share x(a, q + u, lane, per_token);
            if (q + u >= mine || x.i >= tokens || x.f >= frags || sm.row[x.i] < 0) continue;       // the same for the four lanes of a block
            const int kv = x.f / PARTS, part = x.f % PARTS;
            const int64_t to = sm.row[x.i] + (int64_t)kv * a.g.head_stride + part * BITS;
            const auto put = [&](char *pool, const Eight<T> &e, int which) {
                const uint32_t byte = mx_scale_of<BITS>(quad_max(largest_of<T>(e)));
                const Codes<BITS> c = mx_encode<BITS, T>(e, byte);
                *reinterpret_cast<Codes<BITS> *>(pool + to) = c;
                if (part % 4 == 0) sm_scale[(((size_t)which * a.g.n_kv + kv) * tokens + x.i) * SB + part / 4] = (uint8_t)byte;
            };
            put(a.k_pages, k0[u], 0);
            put(a.v_pages, v0[u], 1);
        }
    }
    __syncthreads();
    const int i = tid & (tokens - 1);
    if (sm.row[i] < 0) return;
    for (int kv = tid >> a.tokens_log2; kv < a.g.n_kv; kv += 256 >> a.tokens_log2) {
        const int64_t entry = sm.entry[i] + (int64_t)kv * a.g.page_size;
        const scales_t *s = reinterpret_cast<const scales_t *>(sm_scale);
        reinterpret_cast<scales_t *>(a.k_scales)[entry] = s[(size_t)kv * tokens + i];
        reinterpret_cast<scales_t *>(a.v_scales)[entry] = s[((size_t)a.g.n_kv + kv) * tokens + i];
        if (a.pos) a.pos[entry] = sm.pos[i];
        if (a.weight) a.weight[entry] = a.weight_new ? a.weight_new[(int64_t)(row0 + i) * a.g.n_kv + kv] : 0.f;
    }
}

// ONCE: the rows written are so many that whoever reads them next finds few of them in the memory-side cache, and are not to push one another out of it.
template <typename T, int D, int BITS, bool ONCE> __global__ __launch_bounds__(256) void mx_read_kernel(MxRowsArgs a) {
    constexpr int PARTS = D / 8, SB = D / 32, U = 4;
    __shared__ Spots sm;
    const int tid = threadIdx.x, tokens = 1 << a.tokens_log2, row0 = first_token(a);
    const int lane = tid & ((1 << a.lanes_log2) - 1), step = 1 << a.lanes_log2, frags = a.g.n_kv * PARTS, per_token = (frags + step - 1) >> a.lanes_log2;
    const int mine = ((tokens + (256 >> a.lanes_log2) - 1) >> (8 - a.lanes_log2)) * per_token;
    find_spots<true>(a, row0, sm);
    for (int q = 0; q < mine; q += U) {
        Codes<BITS> k[U], v[U];
        uint32_t ks[U], vs[U];
        bool is[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {                        // no load is under a condition: what does not exist is the pool's first row
            const Share x(a, q + u, lane, per_token);
            is[u] = q + u < mine && x.i < tokens && x.f < frags;
            const int i = is[u] ? x.i : 0, kv = is[u] ? x.f / PARTS : 0, part = x.f % PARTS;
            const int64_t at = sm.row[i];
            is[u] = is[u] && at >= 0;
            const int64_t from = (is[u] ? at + (int64_t)kv * a.g.head_stride : 0) + part * BITS;
            const int64_t scale = (is[u] ? sm.entry[i] + (int64_t)kv * a.g.page_size : 0) * SB + part / 4;
            k[u] = *reinterpret_cast<const Codes<BITS> *>(a.k_pages + from);
            v[u] = *reinterpret_cast<const Codes<BITS> *>(a.v_pages + from);
            ks[u] = a.k_scales[scale];
            vs[u] = a.v_scales[scale];
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (!is[u]) continue;
            const Share x(a, q + u, lane, per_token);
            const int64_t to = (int64_t)(row0 + x.i) * a.stride + (int64_t)x.f * (8 * (int)sizeof(T));
            const auto put = [&](char *p, const Eight<T> &e) {
#pragma unroll
                for (int j = 0; j < (int)sizeof(T) / 2; ++j) {
                    if constexpr (ONCE) __builtin_nontemporal_store(e.r[j], reinterpret_cast<u32x4_nt_t *>(p) + j);
                    else reinterpret_cast<u32x4_nt_t *>(p)[j] = e.r[j];
                }
            };
            put(a.k + to, mx_decode<BITS, T>(k[u], ks[u]));
            put(a.v + to, mx_decode<BITS, T>(v[u], vs[u]));
        }
    }
}

static int launch_mx_rows(const ssd_paged_config *c, int format, MxRowsArgs &a, bool read, hipStream_t s) {
    const int64_t e = (int64_t)paged_esize(c);
    a.stride = (c->new_stride ? c->new_stride : (int64_t)c->n_kv_heads * c->head_dim) * e;
    const int frags = c->n_kv_heads * c->head_dim / 8;
    a.lanes_log2 = 4;
    while (a.lanes_log2 < 8 && 1 << a.lanes_log2 < frags) ++a.lanes_log2;
    // 64 KB of rows to a workgroup that writes the cache, 32 to one that reads it, if that leaves 1024 of them (22500 tokens of 32 heads written in 32, 64 and 128 KB, read back in 32, in 64, 16 where
    // they were written in 128: 174, 171 and 179 us; 557 MB read in 16, 32, 64 and 128 KB 107, 103, 107 and 110)
    a.tokens_log2 = 0;
    while (1 << a.tokens_log2 < TOKENS && ((int64_t)frags * 8 * e) << a.tokens_log2 < (read ? 16384 : 32768) && a.n >> a.tokens_log2 > 1024) ++a.tokens_log2;
    const dim3 grid((unsigned)(((int64_t)a.n + (1 << a.tokens_log2) - 1) >> a.tokens_log2));
    const unsigned lds = read ? 0 : (unsigned)(2 * c->n_kv_heads * (c->head_dim / 32)) << a.tokens_log2;
    // 367 MB: 114 us with ordinary stores, 103 with the hint; 146 MB: 60 and 53; 45 MB: 33.5 either way
    const bool once = (int64_t)a.n * frags * 16 * e > 64 << 20;
    const auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(256), lds, s, a); };
    const auto by_bits = [&](auto t, auto d) {
        typedef decltype(t) T;
        constexpr int D = decltype(d)::value;
        if (read && once) format == SSD_MXFP8 ? go(mx_read_kernel<T, D, 8, true>) : go(mx_read_kernel<T, D, 4, true>);
        else if (read) format == SSD_MXFP8 ? go(mx_read_kernel<T, D, 8, false>) : go(mx_read_kernel<T, D, 4, false>);
        else format == SSD_MXFP8 ? go(mx_append_kernel<T, D, 8>) : go(mx_append_kernel<T, D, 4>);
    };
    const auto by_row = [&](auto t) {
        if (c->head_dim == 128) by_bits(t, std::integral_constant<int, 128>());
        else by_bits(t, std::integral_constant<int, 64>());
    };
    if (c->dtype == SSD_BF16) by_row(bf16_t());
    else by_row(float());
    const hipError_t err = hipGetLastError();
    return err == hipSuccess ? SSD_OK : hip_fail(err, read ? "paged read launch" : "paged append launch");
}

// What both calls ask of their arguments.
static int check_mx_rows(const ssd_paged_config *cfg, int format, const MxRowsArgs &a, const int32_t *block_table, const int32_t *seq_len,
                         const int32_t *seq_pos, const char *rows) {
    int rc = check_mx(cfg, format);
    if (rc != SSD_OK) return rc;
    if (!a.k_pages || !a.v_pages || (a.n != 0 && (!a.k || !a.v))) return fail(SSD_ERR_INVALID_ARG, "k_pages, v_pages or %s is NULL", rows);
    if (!aligned(a.k_pages, 16) || !aligned(a.v_pages, 16) || !aligned(a.k, 16) || !aligned(a.v, 16))
        return fail(SSD_ERR_INVALID_ARG, "k_pages, v_pages and %s must be 16-byte aligned", rows);
    if ((rc = check_mx_scales(a.k_scales, a.v_scales)) != SSD_OK) return rc;
    if (!block_table || !seq_len) return fail(SSD_ERR_INVALID_ARG, "block_table or seq_len is NULL");
    const void *all[] = {block_table, seq_len, seq_pos, a.pos, a.weight, a.start, a.first, a.weight_new};
    for (const void *x : all)
        if (!aligned(x, 4)) return fail(SSD_ERR_INVALID_ARG, "tables must be aligned to their elements");
    if (a.n < 0) return fail(SSD_ERR_INVALID_ARG, "%d rows: must be >= 0", a.n);
    if (!a.start && a.n != cfg->n_seqs) return fail(SSD_ERR_INVALID_ARG, "%d rows without their starts must be n_seqs=%d", a.n, cfg->n_seqs);
    return SSD_OK;
}

}  // namespace ssd

using namespace ssd;

extern "C" int ssd_paged_mx_append(const ssd_paged_config *cfg, int format, void *k_pages, void *v_pages, uint8_t *k_scales, uint8_t *v_scales, int32_t *pos,
                                   float *weight, const int32_t *block_table, const int32_t *seq_len, const int32_t *seq_pos, const void *k_new,
                                   const void *v_new, const int32_t *new_start, int n_new, const float *weight_new, void *stream) {
    clear_error();
    MxRowsArgs a = {};
    a.k_pages = static_cast<char *>(k_pages);
    a.v_pages = static_cast<char *>(v_pages);
    a.k_scales = k_scales;
    a.v_scales = v_scales;
    a.k = static_cast<char *>(const_cast<void *>(k_new));
    a.v = static_cast<char *>(const_cast<void *>(v_new));
    a.start = new_start;
    a.weight_new = weight_new;
    a.pos = pos;
    a.weight = weight;
    a.n = n_new;
    const int rc = check_mx_rows(cfg, format, a, block_table, seq_len, seq_pos, "k_new or v_new");
    if (rc != SSD_OK || n_new == 0) return rc;
    a.g = paged_geom(cfg, block_table, seq_len, seq_pos, 0, format);
    return launch_mx_rows(cfg, format, a, false, static_cast<hipStream_t>(stream));
}

extern "C" int ssd_paged_mx_read(const ssd_paged_config *cfg, int format, const void *k_pages, const void *v_pages, const uint8_t *k_scales,
                                 const uint8_t *v_scales, const int32_t *block_table, const int32_t *seq_len, const int32_t *row_start, int n_rows,
                                 const int32_t *first_slot, void *k_out, void *v_out, void *stream) {
    clear_error();
    MxRowsArgs a = {};
    a.k_pages = static_cast<char *>(const_cast<void *>(k_pages));
    a.v_pages = static_cast<char *>(const_cast<void *>(v_pages));
    a.k_scales = const_cast<uint8_t *>(k_scales);
    a.v_scales = const_cast<uint8_t *>(v_scales);
    a.k = static_cast<char *>(k_out);
    a.v = static_cast<char *>(v_out);
    a.start = row_start;
    a.first = first_slot;
    a.n = n_rows;
    const int rc = check_mx_rows(cfg, format, a, block_table, seq_len, nullptr, "k_out or v_out");
    if (rc != SSD_OK || n_rows == 0) return rc;
    a.g = paged_geom(cfg, block_table, seq_len, nullptr, 0, format);
    return launch_mx_rows(cfg, format, a, true, static_cast<hipStream_t>(stream));
}
