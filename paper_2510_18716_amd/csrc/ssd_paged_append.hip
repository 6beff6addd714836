// ssd_paged_append: new tokens' K and V rows into the pages of a cache of unequal lengths, with their entries in the tables.
// Also the checks that every call on such a cache shares.
//
// Pure data movement, bound by HBM: a row is a run of adjacent lanes, 16 bytes each, on both sides.  22500 tokens of 16 KB (prompts of 64
// requests, 32 heads of 128, bf16): 145 us, 5.1 TB/s read and written, where a plain copy reaches 5.4.  One token for each of 8 sequences: 3.7 us, launch
// and four dependent loads (first row, length, block table, the row itself, which is requested first).
#include <cmath>

#include "ssd_paged.h"

namespace ssd {

int check_paged(const ssd_paged_config *c, int bits) {
    if (!c) return fail(SSD_ERR_INVALID_ARG, "config is NULL");
    if (c->n_seqs < 1 || c->n_seqs > 65535) return fail(SSD_ERR_INVALID_ARG, "n_seqs=%d outside 1..65535", c->n_seqs);
    if (c->n_kv_heads < 1 || c->n_kv_heads > 1024) return fail(SSD_ERR_INVALID_ARG, "n_kv_heads=%d outside 1..1024", c->n_kv_heads);
    if (c->n_heads < 1 || c->n_heads > 1024 || c->n_heads % c->n_kv_heads != 0)
        return fail(SSD_ERR_INVALID_ARG, "n_heads=%d must be a multiple of n_kv_heads=%d, at most 1024", c->n_heads, c->n_kv_heads);
    if (c->head_dim != 64 && c->head_dim != 128) return fail(SSD_ERR_INVALID_ARG, "head_dim=%d, supported: 64, 128", c->head_dim);
    if (c->dtype != SSD_F32 && c->dtype != SSD_BF16) return fail(SSD_ERR_INVALID_ARG, "dtype=%d is neither SSD_F32 nor SSD_BF16", c->dtype);
    if (c->page_size < 1 || c->page_size > 32768) return fail(SSD_ERR_INVALID_ARG, "page_size=%d outside 1..32768", c->page_size);
    if (c->n_pages < 1) return fail(SSD_ERR_INVALID_ARG, "n_pages=%d must be >= 1", c->n_pages);
    if (c->max_blocks < 1 || (int64_t)c->max_blocks * c->page_size > (1ll << 25))
        return fail(SSD_ERR_INVALID_ARG, "max_blocks=%d must be >= 1, with max_blocks * page_size at most 2^25", c->max_blocks);
    if (!(c->softmax_scale >= 0.f) || !std::isfinite(c->softmax_scale)) return fail(SSD_ERR_INVALID_ARG, "softmax_scale must be finite and >= 0");
    for (int i = 0; i < 3; ++i)
        if (c->reserved[i] != 0) return fail(SSD_ERR_INVALID_ARG, "reserved[%d] must be 0", i);
    const int64_t unit = 16 / (int64_t)paged_esize(c), pool_unit = bits ? 128 / bits : unit, most = 1ll << 50;
    const bool none = c->page_stride == 0 && c->head_stride == 0 && c->row_stride == 0;
    const int64_t st[3] = {c->page_stride, c->head_stride, c->row_stride};
    for (int i = 0; i < 3 && !none; ++i)
        if (st[i] < c->head_dim || st[i] % pool_unit != 0 || st[i] > most / ((int64_t)c->n_pages + c->n_kv_heads + c->page_size))
            return fail(SSD_ERR_INVALID_ARG, "page_stride, head_stride and row_stride are all 0, or multiples of 16 bytes of at least head_dim elements");
    if (c->q_stride != 0 && (c->q_stride < (int64_t)c->n_heads * c->head_dim || c->q_stride % unit != 0 || c->q_stride > most / 65536))
        return fail(SSD_ERR_INVALID_ARG, "q_stride must be 0 or a multiple of 16 bytes of at least n_heads * head_dim elements");
    if (c->new_stride != 0 && (c->new_stride < (int64_t)c->n_kv_heads * c->head_dim || c->new_stride % unit != 0 || c->new_stride > most >> 31))
        return fail(SSD_ERR_INVALID_ARG, "new_stride must be 0 or a multiple of 16 bytes of at least n_kv_heads * head_dim elements");
    return SSD_OK;
}

int check_max_len(const ssd_paged_config *c, int max_len) {
    if (max_len < 0 || max_len > (int64_t)c->max_blocks * c->page_size)
        return fail(SSD_ERR_INVALID_ARG, "max_len=%d outside 0..max_blocks * page_size", max_len);
    return SSD_OK;
}

PagedGeom paged_geom(const ssd_paged_config *c, const int32_t *block_table, const int32_t *seq_len, const int32_t *seq_pos, int max_len, int bits) {
    PagedGeom g;
    const int64_t b = bits ? bits : 8 * (int64_t)paged_esize(c);
    const bool dense = c->page_stride == 0;
    g.row_stride = (dense ? c->head_dim : c->row_stride) * b / 8;
    g.head_stride = dense ? g.row_stride * c->page_size : c->head_stride * b / 8;
    g.page_stride = dense ? g.head_stride * c->n_kv_heads : c->page_stride * b / 8;
    g.block_table = block_table;
    g.seq_len = seq_len;
    g.seq_pos = seq_pos ? seq_pos : seq_len;
    g.n_seqs = c->n_seqs;
    g.n_kv = c->n_kv_heads;
    g.page_size = c->page_size;
    g.n_pages = c->n_pages;
    g.max_blocks = c->max_blocks;
    g.max_len = paged_reach(c, max_len);
    g.page_log2 = (c->page_size & (c->page_size - 1)) == 0 ? __builtin_ctz((unsigned)c->page_size) : -1;
    g.share = c->page_size >= 32 ? 0 : c->page_size >= 16 ? 1 : c->page_size >= 8 ? 2 : 3;
    return g;
}

struct PagedAppendArgs {
    PagedGeom g;
    char *k_pages, *v_pages;
    const char *k_new, *v_new;
    const float *weight_new;
    int32_t *pos;
    float *weight;
    const int32_t *new_start;
    int64_t new_stride;      // bytes
    int n_new;
    int lpr_log2;            // 16-byte fragments per row: 8, 16 or 32
    int tokens_log2;         // tokens of a workgroup: 1 .. 64
    int lanes_log2;          // threads that share a token: 16 .. 256
};

static constexpr int STARTS = 1024;      // sequences whose first rows fit in LDS
static constexpr int TOKENS = 64;

// ONCE: the rows written are more than the memory-side cache holds, and are not to push one another out of it.
// A workgroup writes a few consecutive tokens.  First a thread per token finds the token's sequence, by bisection in LDS, and its place; then
// the rows are copied, a token's 16-byte fragments by neighbouring threads; the tables come last, a page's places by neighbouring threads.
template <bool ONCE>
__global__ __launch_bounds__(256) void paged_append_kernel(PagedAppendArgs a) {
    __shared__ int32_t starts[STARTS + 1];
    __shared__ int64_t sm_row[TOKENS];                       // byte offset of the token's place in the pool (head 0), negative: none
    __shared__ int64_t sm_entry[TOKENS];                     // index of its entry in the tables (head 0)
    __shared__ int32_t sm_pos[TOKENS];
    const int tid = threadIdx.x, tokens = 1 << a.tokens_log2;
    const int row0 = (int)blockIdx.x << a.tokens_log2;
    const int lane = tid & ((1 << a.lanes_log2) - 1), step = 1 << a.lanes_log2;
    const int frags = a.g.n_kv << a.lpr_log2;                // of K; as many of V
    // a thread's first fragments are on their way while the places are looked up
    const int i0 = tid >> a.lanes_log2;
    const bool any = i0 < tokens && row0 + i0 < a.n_new && lane < frags;
    u32x4_nt_t k0, v0;
    if (any) {
        const int64_t from = (int64_t)(row0 + i0) * a.new_stride + (int64_t)lane * 16;
        k0 = __builtin_nontemporal_load(reinterpret_cast<const u32x4_nt_t *>(a.k_new + from));
        v0 = __builtin_nontemporal_load(reinterpret_cast<const u32x4_nt_t *>(a.v_new + from));
    }
    const bool in_lds = a.new_start && a.g.n_seqs <= STARTS;
    if (in_lds) {
        for (int i = tid; i <= a.g.n_seqs; i += 256) starts[i] = a.new_start[i];
        __syncthreads();
    }
    if (tid < tokens) {
        const int row = row0 + tid;
        int64_t at = -1, entry = 0;
        int p = 0;
        if (row < a.n_new) {
            int b = row, first = row, count = 1;
            if (a.new_start) {
                b = sequence_of(a.g, row, [&](int i) { return in_lds ? starts[i] : a.new_start[i]; });
                first = in_lds ? starts[b] : a.new_start[b];
                count = (in_lds ? starts[b + 1] : a.new_start[b + 1]) - first;
            }
            if (row >= first && row - first < count) {
                const int64_t slot = (int64_t)a.g.seq_len[b] - count + (row - first);
                if (slot >= 0 && slot < clamp_len(a.g, b)) {
                    int block, place;
                    split_slot(a.g, (int)slot, block, place);
                    const int page = page_of(a.g, b, block);
                    if (page >= 0) {
                        at = row_offset(a.g, page, 0, place);
                        entry = table_index(a.g, page, 0, place);
                        p = a.g.seq_pos[b] - count + (row - first);
                    }
                }
            }
        }
        sm_row[tid] = at;
        sm_entry[tid] = entry;
        sm_pos[tid] = p;
    }
    __syncthreads();
    auto put = [](char *p, const u32x4_nt_t &x) {
        if constexpr (ONCE) __builtin_nontemporal_store(x, reinterpret_cast<u32x4_nt_t *>(p));
        else *reinterpret_cast<u32x4_nt_t *>(p) = x;
    };
    auto place_of = [&](int f) { return (int64_t)(f >> a.lpr_log2) * a.g.head_stride + (int64_t)(f & ((1 << a.lpr_log2) - 1)) * 16; };
    if (any && sm_row[i0] >= 0) {
        const int64_t to = sm_row[i0] + place_of(lane);
        put(a.k_pages + to, k0);
        put(a.v_pages + to, v0);
    }
    for (int i = i0; i < tokens; i += 256 >> a.lanes_log2) {
        const int64_t at = sm_row[i];
        if (at < 0) continue;
        const int64_t from = (int64_t)(row0 + i) * a.new_stride;
#pragma unroll 4
        for (int f = i == i0 ? lane + step : lane; f < frags; f += step) {
            const int64_t to = at + place_of(f);
            const u32x4_nt_t k = __builtin_nontemporal_load(reinterpret_cast<const u32x4_nt_t *>(a.k_new + from + (int64_t)f * 16));
            const u32x4_nt_t v = __builtin_nontemporal_load(reinterpret_cast<const u32x4_nt_t *>(a.v_new + from + (int64_t)f * 16));
            put(a.k_pages + to, k);
            put(a.v_pages + to, v);
        }
    }
    if (!a.pos && !a.weight) return;
    const int i = tid & (tokens - 1);
    if (sm_row[i] < 0) return;
    for (int kv = tid >> a.tokens_log2; kv < a.g.n_kv; kv += 256 >> a.tokens_log2) {
        const int64_t entry = sm_entry[i] + (int64_t)kv * a.g.page_size;
        if (a.pos) a.pos[entry] = sm_pos[i];
        if (a.weight) a.weight[entry] = a.weight_new ? a.weight_new[(int64_t)(row0 + i) * a.g.n_kv + kv] : 0.f;
    }
}

static int launch_paged_append(const ssd_paged_config *c, void *k_pages, void *v_pages, int32_t *pos, float *weight, const int32_t *block_table,
                               const int32_t *seq_len, const int32_t *seq_pos, const void *k_new, const void *v_new, const int32_t *new_start,
                               int n_new, const float *weight_new, hipStream_t s) {
    PagedAppendArgs a;
    a.g = paged_geom(c, block_table, seq_len, seq_pos, 0);
    a.k_pages = static_cast<char *>(k_pages);
    a.v_pages = static_cast<char *>(v_pages);
    a.k_new = static_cast<const char *>(k_new);
    a.v_new = static_cast<const char *>(v_new);
    a.weight_new = weight_new;
    a.pos = pos;
    a.weight = weight;
    a.new_start = new_start;
    const int64_t e = (int64_t)paged_esize(c);
    a.new_stride = (c->new_stride ? c->new_stride : (int64_t)c->n_kv_heads * c->head_dim) * e;
    a.n_new = n_new;
    a.lpr_log2 = __builtin_ctz((unsigned)(c->head_dim * e / 16));
    const int frags = c->n_kv_heads << a.lpr_log2;
    a.lanes_log2 = 4;
    while (a.lanes_log2 < 8 && 1 << a.lanes_log2 < frags) ++a.lanes_log2;
    // 32 KB a workgroup, if that leaves 1024 of them (22500 tokens of 16 KB: 2 tokens 154 us, 16 163; of 4 KB: 2 36.8, 8 34.5; 128000 of 512 bytes: 2 95, 16 27.5)
    a.tokens_log2 = 0;
    while (1 << a.tokens_log2 < TOKENS && ((int64_t)frags * 32) << a.tokens_log2 < 32768 && n_new >> a.tokens_log2 > 1024) ++a.tokens_log2;
    const int64_t blocks = ((int64_t)n_new + (1 << a.tokens_log2) - 1) >> a.tokens_log2;
    // 369 MB: 153 us with ordinary stores, 145 with the hint; 93 MB: 33.5 and 36.3
    if ((int64_t)n_new * frags * 32 > 256ll << 20) hipLaunchKernelGGL((paged_append_kernel<true>), dim3((unsigned)blocks), dim3(256), 0, s, a);
    else hipLaunchKernelGGL((paged_append_kernel<false>), dim3((unsigned)blocks), dim3(256), 0, s, a);
    const hipError_t err = hipGetLastError();
    return err == hipSuccess ? SSD_OK : hip_fail(err, "paged append launch");
}

}  // namespace ssd

using namespace ssd;

extern "C" int ssd_paged_append(const ssd_paged_config *cfg, void *k_pages, void *v_pages, int32_t *pos, float *weight,
                                const int32_t *block_table, const int32_t *seq_len, const int32_t *seq_pos, const void *k_new,
                                const void *v_new, const int32_t *new_start, int n_new, const float *weight_new, void *stream) {
    clear_error();
    const int rc = check_paged(cfg);
    if (rc != SSD_OK) return rc;
    if (!k_pages || !v_pages || !k_new || !v_new) return fail(SSD_ERR_INVALID_ARG, "k_pages, v_pages, k_new or v_new is NULL");
    if (!aligned(k_pages, 16) || !aligned(v_pages, 16) || !aligned(k_new, 16) || !aligned(v_new, 16))
        return fail(SSD_ERR_INVALID_ARG, "k_pages, v_pages, k_new and v_new must be 16-byte aligned");
    if (!block_table || !seq_len) return fail(SSD_ERR_INVALID_ARG, "block_table or seq_len is NULL");
    if (!aligned(block_table, 4) || !aligned(seq_len, 4) || !aligned(seq_pos, 4) || !aligned(pos, 4) || !aligned(weight, 4) ||
        !aligned(new_start, 4) || !aligned(weight_new, 4))
        return fail(SSD_ERR_INVALID_ARG, "tables must be aligned to their elements");
    if (n_new < 0) return fail(SSD_ERR_INVALID_ARG, "n_new=%d must be >= 0", n_new);
    if (!new_start && n_new != cfg->n_seqs) return fail(SSD_ERR_INVALID_ARG, "n_new=%d without new_start must be n_seqs=%d", n_new, cfg->n_seqs);
    if (n_new == 0) return SSD_OK;
    return launch_paged_append(cfg, k_pages, v_pages, pos, weight, block_table, seq_len, seq_pos, k_new, v_new, new_start, n_new, weight_new,
                               static_cast<hipStream_t>(stream));
}
