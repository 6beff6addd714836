// The attention over a paged cache held in 4 bits, kernels of bf16 calls.
#define SSD_MX_ONLY bf16_t, 4
#include "ssd_paged_mx_attn.h"
