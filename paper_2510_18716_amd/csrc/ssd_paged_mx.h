// What the calls on a paged cache held in 8 or 4 bits share on the host: their checks.
#pragma once

#include "ssd_paged.h"

namespace ssd {

// The config with the pool's strides in elements of the format, whose bits `format` is.
static inline int check_mx(const ssd_paged_config *c, int format) {
    if (format != SSD_MXFP8 && format != SSD_MXFP4) return fail(SSD_ERR_INVALID_ARG, "format=%d is neither SSD_MXFP8 nor SSD_MXFP4", format);
    return check_paged(c, format);
}
static inline int check_mx_scales(const void *k_scales, const void *v_scales) {
    if (!k_scales || !v_scales || !aligned(k_scales, 16) || !aligned(v_scales, 16))
        return fail(SSD_ERR_INVALID_ARG, "k_scales and v_scales must be given, 16-byte aligned");
    return SSD_OK;
}

}  // namespace ssd
