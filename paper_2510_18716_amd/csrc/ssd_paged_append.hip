// ssd_paged_append: new tokens' K and V rows into the pages of a cache of unequal lengths, with their entries in the tables.
// Also the checks that every call on such a cache shares.
//
// Pure data movement: one lane moves one 16-byte fragment, so a row is a run of adjacent lanes on both sides.
#include <cmath>

#include "ssd_paged.h"

namespace ssd {

int check_paged(const ssd_paged_config *c) {
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
    const int64_t unit = 16 / (int64_t)paged_esize(c), most = 1ll << 50;
    const bool none = c->page_stride == 0 && c->head_stride == 0 && c->row_stride == 0;
    const int64_t st[3] = {c->page_stride, c->head_stride, c->row_stride};
    for (int i = 0; i < 3 && !none; ++i)
        if (st[i] < c->head_dim || st[i] % unit != 0 || st[i] > most / ((int64_t)c->n_pages + c->n_kv_heads + c->page_size))
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

PagedGeom paged_geom(const ssd_paged_config *c, const int32_t *block_table, const int32_t *seq_len, const int32_t *seq_pos, int max_len) {
    PagedGeom g;
    const int64_t e = (int64_t)paged_esize(c);
    const bool dense = c->page_stride == 0;
    g.row_stride = (dense ? c->head_dim : c->row_stride) * e;
    g.head_stride = dense ? g.row_stride * c->page_size : c->head_stride * e;
    g.page_stride = dense ? g.head_stride * c->n_kv_heads : c->page_stride * e;
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
};

// grid = (blocks over a token's heads and fragments, tokens)
__global__ __launch_bounds__(256) void paged_append_kernel(PagedAppendArgs a) {
    const int t = (int)(blockIdx.x * 256 + threadIdx.x);
    const int kv = t >> (a.lpr_log2 + 1);
    for (int row = (int)blockIdx.y; row < a.n_new; row += (int)gridDim.y) {
        int b = row, first = row, count = 1;
        if (a.new_start) {
            int lo = 0, hi = a.g.n_seqs;           // the last sequence that begins at or before the row
            while (hi - lo > 1) {
                const int mid = (lo + hi) / 2;
                if (a.new_start[mid] <= row) lo = mid;
                else hi = mid;
            }
            b = lo;
            first = a.new_start[b];
            count = a.new_start[b + 1] - first;
        }
        if (kv >= a.g.n_kv || row < first || row - first >= count) continue;
        const int n = clamp_len(a.g, b);
        const int64_t slot64 = (int64_t)a.g.seq_len[b] - count + (row - first);
        if (slot64 < 0 || slot64 >= n) continue;
        int block, place;
        split_slot(a.g, (int)slot64, block, place);
        const int page = page_of(a.g, b, block);
        if (page < 0) continue;
        const bool v = (t >> a.lpr_log2) & 1;
        const int64_t sub = (int64_t)(t & ((1 << a.lpr_log2) - 1)) * 16;
        const char *src = (v ? a.v_new : a.k_new) + (int64_t)row * a.new_stride + (((int64_t)kv << a.lpr_log2) * 16 + sub);
        *reinterpret_cast<uint4 *>((v ? a.v_pages : a.k_pages) + row_offset(a.g, page, kv, place) + sub) = *reinterpret_cast<const uint4 *>(src);
        if (!v && sub == 0) {
            const int64_t i = table_index(a.g, page, kv, place);
            if (a.pos) a.pos[i] = a.g.seq_pos[b] - count + (row - first);
            if (a.weight) a.weight[i] = a.weight_new ? a.weight_new[(int64_t)row * a.g.n_kv + kv] : 0.f;
        }
    }
}

int launch_paged_append(const ssd_paged_config *c, void *k_pages, void *v_pages, int32_t *pos, float *weight, const int32_t *block_table,
                        const int32_t *seq_len, const int32_t *seq_pos, int max_len, const void *k_new, const void *v_new,
                        const int32_t *new_start, int n_new, const float *weight_new, hipStream_t s) {
    PagedAppendArgs a;
    a.g = paged_geom(c, block_table, seq_len, seq_pos, max_len);
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
    const unsigned per_token = (unsigned)c->n_kv_heads << (a.lpr_log2 + 1);
    hipLaunchKernelGGL(paged_append_kernel, dim3((per_token + 255) / 256, n_new < 65535 ? n_new : 65535), dim3(256), 0, s, a);
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
    return launch_paged_append(cfg, k_pages, v_pages, pos, weight, block_table, seq_len, seq_pos, 0, k_new, v_new, new_start, n_new, weight_new,
                               static_cast<hipStream_t>(stream));
}
