// ssd_paged_mx_decode_attn, ssd_paged_mx_decode_step: attention of one new token per sequence over pages held in 8 or 4 bits.
#include "ssd_paged_mx.h"
#include "ssd_paged_mx_attn.h"

namespace ssd {

static int mx_attend(const AttendCall &c, int format, uint8_t *k_scales, uint8_t *v_scales, hipStream_t s) {
    clear_error();
    int rc = check_mx(c.cfg, format);
    if (rc != SSD_OK || (rc = check_mx_scales(k_scales, v_scales)) != SSD_OK) return rc;
    PagedAttnArgs a;
    PagedShape shape;
    if ((rc = attend_args(c, mx_tile_shape(c.cfg), format, a, shape)) != SSD_OK) return rc;
    a.k_scales = k_scales;
    a.v_scales = v_scales;
    const int d = c.cfg->head_dim;
    const int group = mx_group(c.cfg);
    hipError_t e;
    if (c.cfg->dtype == SSD_BF16) e = format == SSD_MXFP8 ? launch_mx_attn<bf16_t, 8>(a, shape, d, group, c.step, s) : launch_mx_attn<bf16_t, 4>(a, shape, d, group, c.step, s);
    else e = format == SSD_MXFP8 ? launch_mx_attn<float, 8>(a, shape, d, group, c.step, s) : launch_mx_attn<float, 4>(a, shape, d, group, c.step, s);
    return e == hipSuccess ? SSD_OK : hip_fail(e, "paged attention launch");
}

}  // namespace ssd

using namespace ssd;

extern "C" size_t ssd_paged_mx_workspace_bytes(const ssd_paged_config *cfg, int format, int max_len, int with_weights) {
    clear_error();
    if (check_mx(cfg, format) != SSD_OK || check_max_len(cfg, max_len) != SSD_OK) return 0;
    return paged_scratch(cfg, paged_shape(cfg, max_len, mx_tile_shape(cfg)), with_weights != 0).all;
}

extern "C" int ssd_paged_mx_decode_attn(const ssd_paged_config *cfg, int format, const void *q, const void *k_pages, const void *v_pages,
                                        const uint8_t *k_scales, const uint8_t *v_scales, const float *weight_in, float *weight_out,
                                        const int32_t *block_table, const int32_t *seq_len, void *out, float *lse, int max_len, void *workspace,
                                        size_t workspace_bytes, void *stream) {
    return mx_attend({cfg, q, nullptr, nullptr, const_cast<void *>(k_pages), const_cast<void *>(v_pages), nullptr, weight_in, weight_out, block_table, seq_len,
                      nullptr, out, lse, max_len, workspace, workspace_bytes, false},
                     format, const_cast<uint8_t *>(k_scales), const_cast<uint8_t *>(v_scales), static_cast<hipStream_t>(stream));
}

extern "C" int ssd_paged_mx_decode_step(const ssd_paged_config *cfg, int format, const void *q, const void *k_new, const void *v_new, void *k_pages,
                                        void *v_pages, uint8_t *k_scales, uint8_t *v_scales, int32_t *pos, const float *weight_in, float *weight_out,
                                        const int32_t *block_table, const int32_t *seq_len, const int32_t *seq_pos, void *out, float *lse, int max_len,
                                        void *workspace, size_t workspace_bytes, void *stream) {
    return mx_attend({cfg, q, k_new, v_new, k_pages, v_pages, pos, weight_in, weight_out, block_table, seq_len, seq_pos, out, lse, max_len, workspace,
                      workspace_bytes, true},
                     format, k_scales, v_scales, static_cast<hipStream_t>(stream));
}
