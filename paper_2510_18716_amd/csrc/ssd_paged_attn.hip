// ssd_paged_decode_attn, ssd_paged_decode_step: attention of one new token per sequence over the sequence's pages.
//
// Three launches: every row's logits into the workspace, the softmax and the weighted sum of V per (sequence, query head), the
// probabilities onto the accumulated weights per row.
#include "ssd_paged.h"

namespace ssd {

struct PagedAttnArgs {
    PagedGeom g;
    const char *q, *k_pages, *v_pages;
    const float *weight_in;
    float *weight_out;
    char *out;
    float *lse;
    float *z;                 // [n_seqs, n_heads, max_len] logits, then probabilities
    const int32_t *pos;
    int64_t q_stride;         // bytes
    int n_heads, group;
    float scale;
    int step;                 // the newest row has no weight yet
};

template <typename T, int D>
__global__ __launch_bounds__(256) void paged_logits_kernel(PagedAttnArgs a) {
    const int h = blockIdx.y, b = blockIdx.z, kv = h / a.group;
    const int n = clamp_len(a.g, b);
    const T *q = reinterpret_cast<const T *>(a.q + (int64_t)b * a.q_stride) + h * D;
    for (int j = (int)(blockIdx.x * 256 + threadIdx.x); j < n; j += (int)gridDim.x * 256) {
        int block, place;
        split_slot(a.g, j, block, place);
        const int page = page_of(a.g, b, block);
        float z = -INFINITY;
        if (page >= 0) {
            const char *k = a.k_pages + row_offset(a.g, page, kv, place);
            z = 0.f;
            for (int i = 0; i < D; i += Elem<T>::VEC)
                z += Elem<T>::dot(Elem<T>::load_q(*reinterpret_cast<const uint4 *>(q + i)), *reinterpret_cast<const uint4 *>(k + i * sizeof(T)));
            z *= a.scale;
        }
        a.z[((int64_t)b * a.n_heads + h) * a.g.max_len + j] = z;
    }
}

template <bool MAX> static __device__ float block_reduce(float v, float *lds) {
    for (int o = 32; o > 0; o >>= 1) {
        const float w = __shfl_xor(v, o);
        v = MAX ? fmaxf(v, w) : v + w;
    }
    __syncthreads();
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    return MAX ? fmaxf(fmaxf(lds[0], lds[1]), fmaxf(lds[2], lds[3])) : lds[0] + lds[1] + lds[2] + lds[3];
}

template <typename T, int D>
__global__ __launch_bounds__(256) void paged_sum_kernel(PagedAttnArgs a) {
    __shared__ float lds[4];
    __shared__ float part[256 / D][D];
    const int h = blockIdx.x, b = blockIdx.y, kv = h / a.group;
    const int n = clamp_len(a.g, b);
    float *z = a.z + ((int64_t)b * a.n_heads + h) * a.g.max_len;
    float top = -INFINITY;
    for (int j = threadIdx.x; j < n; j += 256) top = fmaxf(top, z[j]);
    top = block_reduce<true>(top, lds);
    float sum = 0.f;
    if (top > -INFINITY)
        for (int j = threadIdx.x; j < n; j += 256) sum += expf(z[j] - top);
    sum = block_reduce<false>(sum, lds);
    const bool none = n == 0 || top == -INFINITY;
    for (int j = threadIdx.x; j < n; j += 256) z[j] = none ? 0.f : expf(z[j] - top) / sum;
    __syncthreads();
    const int e = threadIdx.x % D, lane = threadIdx.x / D;
    float acc = 0.f;
    for (int j = lane; j < n; j += 256 / D) {
        int block, place;
        split_slot(a.g, j, block, place);
        const int page = page_of(a.g, b, block);
        if (page < 0) continue;
        const T *v = reinterpret_cast<const T *>(a.v_pages + row_offset(a.g, page, kv, place));
        float x;
        if constexpr (sizeof(T) == 4) x = v[e];
        else x = __uint_as_float((uint32_t)v[e].bits << 16);
        acc = fmaf(z[j], x, acc);
    }
    part[lane][e] = acc;
    __syncthreads();
    if (lane == 0) {
        for (int i = 1; i < 256 / D; ++i) acc += part[i][e];
        T *o = reinterpret_cast<T *>(a.out) + ((int64_t)b * a.n_heads + h) * D;
        if constexpr (sizeof(T) == 4) o[e] = acc;
        else o[e].bits = (uint16_t)f32_to_bf16_bits(acc);
    }
    if (threadIdx.x == 0 && a.lse) a.lse[(int64_t)b * a.n_heads + h] = none ? -INFINITY : top + logf(sum);
}

__global__ __launch_bounds__(256) void paged_weight_kernel(PagedAttnArgs a) {
    const int kv = blockIdx.y, b = blockIdx.z;
    const int n = clamp_len(a.g, b);
    for (int j = (int)(blockIdx.x * 256 + threadIdx.x); j < n; j += (int)gridDim.x * 256) {
        int block, place;
        split_slot(a.g, j, block, place);
        const int page = page_of(a.g, b, block);
        if (page < 0) continue;
        const int64_t i = table_index(a.g, page, kv, place);
        float w = a.step && j == a.g.seq_len[b] - 1 ? 0.f : a.weight_in[i];
        float p = 0.f;
        for (int h = kv * a.group; h < (kv + 1) * a.group; ++h) p += a.z[((int64_t)b * a.n_heads + h) * a.g.max_len + j];
        a.weight_out[i] = w + p;
    }
}

template <typename T, int D> static hipError_t launch_paged_attn(const PagedAttnArgs &a, hipStream_t s) {
    const unsigned blocks = (unsigned)(a.g.max_len + 255) / 256;
    hipLaunchKernelGGL((paged_logits_kernel<T, D>), dim3(blocks, a.n_heads, a.g.n_seqs), dim3(256), 0, s, a);
    hipLaunchKernelGGL((paged_sum_kernel<T, D>), dim3(a.n_heads, a.g.n_seqs), dim3(256), 0, s, a);
    if (a.weight_out) hipLaunchKernelGGL(paged_weight_kernel, dim3(blocks, a.g.n_kv, a.g.n_seqs), dim3(256), 0, s, a);
    return hipGetLastError();
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
    const size_t need = ssd_paged_workspace_bytes(cfg, max_len, weight_out != nullptr);
    if (need > 0 && (!workspace || !aligned(workspace, 256) || workspace_bytes < need))
        return fail(SSD_ERR_INVALID_ARG, "workspace of %zu bytes, 256-byte aligned, needed; %zu given", need, workspace_bytes);
    if (step) {
        rc = launch_paged_append(cfg, k_pages, v_pages, pos, nullptr, block_table, seq_len, seq_pos, max_len, k_new, v_new, nullptr, cfg->n_seqs,
                                 nullptr, s);
        if (rc != SSD_OK) return rc;
    }
    PagedAttnArgs a;
    a.g = paged_geom(cfg, block_table, seq_len, seq_pos, max_len);
    a.q = static_cast<const char *>(q);
    a.k_pages = static_cast<const char *>(k_pages);
    a.v_pages = static_cast<const char *>(v_pages);
    a.weight_in = weight_in;
    a.weight_out = weight_out;
    a.out = static_cast<char *>(out);
    a.lse = lse;
    a.z = static_cast<float *>(workspace);
    a.pos = pos;
    a.q_stride = (cfg->q_stride ? cfg->q_stride : (int64_t)cfg->n_heads * cfg->head_dim) * (int64_t)paged_esize(cfg);
    a.n_heads = cfg->n_heads;
    a.group = cfg->n_heads / cfg->n_kv_heads;
    a.scale = cfg->softmax_scale != 0.f ? cfg->softmax_scale : 1.f / sqrtf((float)cfg->head_dim);
    a.step = step;
    hipError_t e;
    if (cfg->dtype == SSD_BF16) e = cfg->head_dim == 128 ? launch_paged_attn<bf16_t, 128>(a, s) : launch_paged_attn<bf16_t, 64>(a, s);
    else e = cfg->head_dim == 128 ? launch_paged_attn<float, 128>(a, s) : launch_paged_attn<float, 64>(a, s);
    return e == hipSuccess ? SSD_OK : hip_fail(e, "paged attention launch");
}

}  // namespace ssd

using namespace ssd;

extern "C" size_t ssd_paged_workspace_bytes(const ssd_paged_config *cfg, int max_len, int with_weights) {
    (void)with_weights;
    clear_error();
    if (check_paged(cfg) != SSD_OK || check_max_len(cfg, max_len) != SSD_OK) return 0;
    return round256((size_t)cfg->n_seqs * cfg->n_heads * paged_reach(cfg, max_len) * sizeof(float));
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
