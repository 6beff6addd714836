// The attention over a paged cache held in 4 bits, kernels of f32 calls.
#define SSD_MX_ONLY float, 4
#include "ssd_paged_mx_attn.h"
