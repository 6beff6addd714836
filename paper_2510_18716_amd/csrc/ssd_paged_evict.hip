// ssd_paged_evict: each (sequence, kv head) of a paged cache is cut to its budget; the rows of the largest accumulated attention weight
// stay (the top-M rule of Algorithm 1, sinks and recent tokens protected as in Sec. 3.3).
//
// Two launches.  Selection: one workgroup per unit finds the key of the last row that stays by a radix descent over the keys
// (weight, position) -- integer compares, so the set is exact -- and lists the slots that become free below n' and the kept rows
// above, both in slot order.  Movement: the rows of the lists, 16-byte fragments.
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

// Larger is better: the weight, then the lower position.
static __device__ __forceinline__ unsigned long long evict_key(float w, int pos) {
    uint32_t u = __float_as_uint(w);
    if ((u & 0x7fffffffu) > 0x7f800000u) u = 0;                                   // NaN: below everything
    else if (u == 0x80000000u) u = 0x80000000u;                                   // -0 as +0
    else u = u & 0x80000000u ? ~u : u | 0x80000000u;
    return (unsigned long long)u << 32 | (uint32_t)~((uint32_t)pos ^ 0x80000000u);
}

struct EvictRow { unsigned long long key; bool safe; };

static __device__ __forceinline__ EvictRow evict_row(const PagedEvictArgs &a, int b, int kv, int j, int total) {
    int block, place;
    split_slot(a.g, j, block, place);
    const int page = page_of(a.g, b, block);
    float w = __uint_as_float(0x7fc00000u);
    int pos = 0;
    if (page >= 0) {
        const int64_t i = table_index(a.g, page, kv, place);
        w = a.weight_in[i];
        pos = a.pos_in[i];
    }
    return {evict_key(w, pos), pos < a.n_sink || (int64_t)pos >= (int64_t)total - a.recent};
}

// Position of this thread among those of the workgroup whose flag is set, and how many there are.
static __device__ __forceinline__ int block_rank(bool flag, uint32_t *lds, int &all) {
    const unsigned long long m = __ballot(flag);
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    __syncthreads();
    if (lane == 0) lds[wave] = (uint32_t)__popcll(m);
    __syncthreads();
    int before = 0;
    all = 0;
    for (int i = 0; i < (int)(blockDim.x >> 6); ++i) {
        if (i < wave) before += (int)lds[i];
        all += (int)lds[i];
    }
    return before + __popcll(m & ((1ull << lane) - 1));
}

__global__ __launch_bounds__(1024) void paged_select_kernel(PagedEvictArgs a) {
    __shared__ uint32_t hist[256];
    __shared__ uint32_t lds[16];
    __shared__ int found[3];
    const int kv = blockIdx.x, b = blockIdx.y, tid = threadIdx.x;
    const int n = clamp_len(a.g, b);
    const int want = a.budget[b] < 0 ? 0 : a.budget[b];
    const int stay = n < want ? n : want;
    int32_t *list = a.moves + moves_of(a.cap, (int64_t)b * a.g.n_kv + kv);
    if (kv == 0 && tid == 0 && a.len_out) a.len_out[b] = stay;
    const bool copy = a.pos_out != a.pos_in;
    const int total = a.g.seq_pos[b];
    int count = 0, all;

    // which rows compete, and for how many places
    int safe_rows = 0;
    if (stay < n)
        for (int j0 = 0; j0 < n; j0 += 1024) {
            const int j = j0 + tid;
            block_rank(j < n && evict_row(a, b, kv, j, total).safe, lds, all);
            safe_rows += all;
        }
    const bool among_safe = safe_rows >= stay;
    int left = among_safe ? stay : stay - safe_rows;

    // the key of the last row that stays, and how many of its equals
    unsigned long long last = 0;
    int ties = 0;
    if (stay < n && left > 0) {
        int shift = 64;
        while (shift > 0) {
            shift -= 8;
            for (int i = tid; i < 256; i += 1024) hist[i] = 0;
            __syncthreads();
            for (int j = tid; j < n; j += 1024) {
                const EvictRow r = evict_row(a, b, kv, j, total);
                if (r.safe == among_safe && (shift == 56 || r.key >> (shift + 8) == last >> (shift + 8)))
                    atomicAdd(&hist[(int)(r.key >> shift) & 255], 1u);
            }
            __syncthreads();
            if (tid == 0) {
                int above = 0, digit = 255;
                while (digit > 0 && above + (int)hist[digit] < left) above += (int)hist[digit--];
                found[0] = digit;
                found[1] = above;
                found[2] = (int)hist[digit];
            }
            __syncthreads();
            last |= (unsigned long long)found[0] << shift;
            left -= found[1];
            ties = left;
            const bool whole = found[2] == left;
            __syncthreads();
            if (whole) {                       // all of them stay: nothing below needs looking at
                ties = n;
                break;
            }
        }
    }

    int n_free = 0, n_move = 0, n_tie = 0;
    for (int j0 = 0; j0 < n && (stay < n || copy); j0 += 1024) {
        const int j = j0 + tid;
        bool kept = j < n;
        if (stay < n) {
            const EvictRow r = evict_row(a, b, kv, j < n ? j : n - 1, total);
            const bool competes = j < n && r.safe == among_safe && stay > 0 && (among_safe || stay > safe_rows);
            const bool tie = competes && r.key == last;
            const int rank = n_tie + block_rank(tie, lds, all);
            n_tie += all;
            kept = j < n && ((r.safe && !among_safe) || (competes && (r.key > last || (tie && rank < ties))));
            const int f = n_free + block_rank(j < stay && !kept, lds, all);
            n_free += all;
            if (j < stay && !kept) list[1 + f] = j;
            const int m = n_move + block_rank(j >= stay && kept, lds, all);
            n_move += all;
            if (j >= stay && kept) list[1 + a.cap + m] = j;
        }
        if (copy && kept && j < stay) {
            int block, place;
            split_slot(a.g, j, block, place);
            const int page = page_of(a.g, b, block);
            if (page >= 0) {
                const int64_t i = table_index(a.g, page, kv, place);
                a.pos_out[i] = a.pos_in[i];
                a.weight_out[i] = a.weight_in[i];
            }
        }
    }
    count = n_move;
    if (tid == 0) list[0] = count;
}

// grid = (pieces of the list, kv heads, sequences)
__global__ __launch_bounds__(256) void paged_move_kernel(PagedEvictArgs a) {
    const int kv = blockIdx.y, b = blockIdx.z;
    const int32_t *list = a.moves + moves_of(a.cap, (int64_t)b * a.g.n_kv + kv);
    const int count = list[0], lanes = 2 << a.lpr_log2;          // a row of K and one of V
    const int per = 256 / lanes, lane = threadIdx.x & (lanes - 1);
    const bool v = lane >> a.lpr_log2;
    const int64_t sub = (int64_t)(lane & ((1 << a.lpr_log2) - 1)) * 16;
    char *pool = v ? a.v_pages : a.k_pages;
    for (int i = (int)blockIdx.x * per + (int)threadIdx.x / lanes; i < count; i += (int)gridDim.x * per) {
        const int to = list[1 + i], from = list[1 + a.cap + i];
        int tb, tp, fb, fp;
        split_slot(a.g, to, tb, tp);
        split_slot(a.g, from, fb, fp);
        const int tpage = page_of(a.g, b, tb), fpage = page_of(a.g, b, fb);
        if (tpage < 0 || fpage < 0) continue;
        *reinterpret_cast<uint4 *>(pool + row_offset(a.g, tpage, kv, tp) + sub) =
            *reinterpret_cast<const uint4 *>(pool + row_offset(a.g, fpage, kv, fp) + sub);
        if (lane == 0) {
            const int64_t t = table_index(a.g, tpage, kv, tp), f = table_index(a.g, fpage, kv, fp);
            a.pos_out[t] = a.pos_in[f];
            a.weight_out[t] = a.weight_in[f];
        }
    }
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
    hipLaunchKernelGGL(paged_select_kernel, units, dim3(1024), 0, s, a);
    const unsigned pieces = (unsigned)(a.cap + 127) / 128;
    hipLaunchKernelGGL(paged_move_kernel, dim3(pieces < 256 ? pieces : 256, units.x, units.y), dim3(256), 0, s, a);
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? SSD_OK : hip_fail(e, "paged eviction launch");
}
