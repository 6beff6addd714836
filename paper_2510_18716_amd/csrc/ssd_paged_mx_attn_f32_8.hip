// The attention over a paged cache held in 8 bits, kernels of f32 calls.
#define SSD_MX_ONLY float, 8
#include "ssd_paged_mx_attn.h"
