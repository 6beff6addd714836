// The attention over a paged cache held in 8 bits, kernels of bf16 calls.
#define SSD_MX_ONLY bf16_t, 8
#include "ssd_paged_mx_attn.h"
