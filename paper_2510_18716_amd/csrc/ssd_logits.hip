// ssd_logits_process: guidance, bias, penalties for repeated tokens, temperature and grammar mask, from a step's logits to those a
// token is sampled from.
//
// One workgroup takes a piece of a row's vocabulary.  How often the row's tokens fall into the piece is counted in LDS (whole-number
// atomics: their order does not matter), one count per entry with the highest bit for "seen at all"; then the piece's logits go
// through once.
#include <cmath>

#include "ssd_device.h"

namespace ssd {

struct LogitsArgs {
    const void *logits;
    float *out;
    int64_t logits_stride, out_stride;   // elements
    ssd_logits_params p;
    int V, guided;
    float gamma;
};

static constexpr int PIECE = 8192;
static constexpr uint32_t SEEN = 0x80000000u;

static __device__ __forceinline__ float widen1(const float *p, int64_t i) { return p[i]; }
static __device__ __forceinline__ float widen1(const bf16_t *p, int64_t i) { return __uint_as_float((uint32_t)p[i].bits << 16); }

template <typename T>
__global__ __launch_bounds__(256) void logits_kernel(LogitsArgs a) {
#pragma clang fp contract(off)
    __shared__ uint32_t count[PIECE];
    const int i = blockIdx.y, v0 = blockIdx.x * PIECE;
    const int len = a.V - v0 < PIECE ? a.V - v0 : PIECE;
    const bool told = a.p.tokens != nullptr;
    if (told) {
        for (int j = threadIdx.x; j < len; j += 256) count[j] = 0;
        __syncthreads();
        int64_t n = a.p.n_tokens[i];
        n = n < 0 ? 0 : n > a.p.token_stride ? a.p.token_stride : n;
        const int64_t n_prompt = a.p.n_prompt ? a.p.n_prompt[i] : 0;
        const int32_t *tok = a.p.tokens + (int64_t)i * a.p.token_stride;
        for (int64_t j = threadIdx.x; j < n; j += 256) {
            const unsigned at = (unsigned)tok[j] - (unsigned)v0;
            if (at < (unsigned)len) {
                if (j >= n_prompt) atomicAdd(&count[at], 1u);
                atomicOr(&count[at], SEEN);
            }
        }
        __syncthreads();
    }
    const float rep0 = a.p.repetition ? a.p.repetition[i] : 1.f, temp0 = a.p.temperature ? a.p.temperature[i] : 1.f;
    const float rep = rep0 > 0.f ? rep0 : 1.f, temp = temp0 > 0.f ? temp0 : 1.f;
    const float presence = a.p.presence ? a.p.presence[i] : 0.f, frequency = a.p.frequency ? a.p.frequency[i] : 0.f;
    const T *c = static_cast<const T *>(a.logits) + (a.guided ? 2 : 1) * (int64_t)i * a.logits_stride;
    const T *u = c + a.logits_stride;
    const float *bias = a.p.bias ? a.p.bias + (int64_t)i * a.p.bias_stride : nullptr;
    const uint32_t *mask = a.p.mask ? a.p.mask + (int64_t)i * a.p.mask_stride : nullptr;
    float *o = a.out + (int64_t)i * a.out_stride;
    for (int j = threadIdx.x; j < len; j += 256) {
        const int v = v0 + j;
        float x = widen1(c, v);
        if (a.guided) x = x + a.gamma * (x - widen1(u, v));
        if (bias) x = x + bias[v];
        const uint32_t n = told ? count[j] : 0;
        if (n) {
            x = x > 0.f ? x / rep : x * rep;
            const uint32_t times = n & ~SEEN;
            x = x - (frequency * (float)times + (times ? presence : 0.f));
        }
        x = x / temp;
        if (mask && !((mask[v >> 5] >> (v & 31)) & 1u)) x = -INFINITY;
        o[v] = x;
    }
}

}  // namespace ssd

using namespace ssd;

extern "C" int ssd_logits_process(const void *logits, int n_rows, int V, int dtype, int64_t logits_stride, int guided, float gamma,
                                  const ssd_logits_params *params, float *out, int64_t out_stride, void *stream) {
    clear_error();
    if (!logits || !out || !params) return fail(SSD_ERR_INVALID_ARG, "logits, params or out is NULL");
    if (!aligned(logits, 16) || !aligned(out, 16)) return fail(SSD_ERR_INVALID_ARG, "logits and out must be 16-byte aligned");
    if (n_rows < 1 || n_rows > 65535) return fail(SSD_ERR_INVALID_ARG, "n_rows=%d outside 1..65535", n_rows);
    if (V < 1 || V > (1 << 24)) return fail(SSD_ERR_INVALID_ARG, "V=%d outside 1..2^24", V);
    if (dtype != SSD_F32 && dtype != SSD_BF16) return fail(SSD_ERR_INVALID_ARG, "bad dtype");
    if (guided != 0 && guided != 1) return fail(SSD_ERR_INVALID_ARG, "guided is 0 or 1");
    if (guided && !std::isfinite(gamma)) return fail(SSD_ERR_INVALID_ARG, "gamma must be finite");
    if (logits_stride == 0) logits_stride = V;
    if (out_stride == 0) out_stride = V;
    const int64_t most = 1ll << 40;
    if (logits_stride < V || out_stride < V || logits_stride > most || out_stride > most)
        return fail(SSD_ERR_INVALID_ARG, "logits_stride and out_stride are 0 or at least V");
    const ssd_logits_params &p = *params;
    if ((p.tokens == nullptr) != (p.n_tokens == nullptr)) return fail(SSD_ERR_INVALID_ARG, "tokens and n_tokens are given both or neither");
    if (p.tokens && (p.token_stride < 0 || p.token_stride > 0x7fffffff)) return fail(SSD_ERR_INVALID_ARG, "token_stride outside 0..2^31-1");
    if (p.bias && p.bias_stride != 0 && (p.bias_stride < V || p.bias_stride > most)) return fail(SSD_ERR_INVALID_ARG, "bias_stride is 0 or at least V");
    if (p.mask && p.mask_stride != 0 && (p.mask_stride < (V + 31) / 32 || p.mask_stride > most))
        return fail(SSD_ERR_INVALID_ARG, "mask_stride is 0 or at least ceil(V / 32)");
    const void *all[] = {p.tokens, p.n_tokens, p.n_prompt, p.repetition, p.presence, p.frequency, p.temperature, p.bias, p.mask};
    for (const void *x : all)
        if (!aligned(x, 4)) return fail(SSD_ERR_INVALID_ARG, "params must be aligned to their elements");
    const bool in_place = static_cast<const void *>(out) == logits;
    if (in_place && (dtype != SSD_F32 || guided || logits_stride != out_stride))
        return fail(SSD_ERR_INVALID_ARG, "out may be logits only where these are fp32, not guided, and the strides agree");
    LogitsArgs a;
    a.logits = logits;
    a.out = out;
    a.logits_stride = logits_stride;
    a.out_stride = out_stride;
    a.p = p;
    a.V = V;
    a.guided = guided;
    a.gamma = gamma;
    const dim3 grid((unsigned)(V + PIECE - 1) / PIECE, (unsigned)n_rows);
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (dtype == SSD_F32) hipLaunchKernelGGL((logits_kernel<float>), grid, dim3(256), 0, s, a);
    else hipLaunchKernelGGL((logits_kernel<bf16_t>), grid, dim3(256), 0, s, a);
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? SSD_OK : hip_fail(e, "logits launch");
}
