// ssd_logits_process: guidance, bias, penalties for repeated tokens, temperature and grammar mask, from a step's logits to those a
// token is sampled from.
//
// One workgroup takes a piece of a row's vocabulary.  Its logits are requested first, into registers; while they travel, the row's
// tokens that fall into the piece are counted in LDS (whole-number atomics: their order does not matter), one count per entry with the highest bit for
// "seen at all"; then the piece goes through once, 16 bytes of logits at a time.  Bound by HBM (the logits in, 4 bytes out each); the tokens are read
// by every piece of the row, from L2.  256 rows of 128257 in fp32 with 1000 to 8000 tokens, shared bias and masks: 64 to 66 us, 4.1 TB/s (56 with short
// histories, where a copy would take 50; 72 without the non-temporal hint on the stores; pieces of 4096 and 16384 and a bias held in registers gain
// nothing).  64 guided rows of 16384 in bf16: 4.5 to 5.3 us, the launch and two dependent loads.
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

static constexpr uint32_t SEEN = 0x80000000u;

typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef f32x4_t f32x4_any_t __attribute__((aligned(4)));
typedef uint32_t u32x4_any2_t __attribute__((ext_vector_type(4), aligned(2)));
typedef int32_t i32x4_any_t __attribute__((ext_vector_type(4), aligned(4)));

// VEC logits from any element's address; past `there` of them: 0, not read.
template <typename T> static __device__ __forceinline__ uint4 load_logits(const T *p, int there) {
    constexpr int VEC = Elem<T>::VEC;
    if (there >= VEC) {
        const u32x4_any2_t x = __builtin_nontemporal_load(reinterpret_cast<const u32x4_any2_t *>(p));
        return make_uint4(x.x, x.y, x.z, x.w);
    }
    uint4 r = make_uint4(0, 0, 0, 0);
    uint32_t *w = reinterpret_cast<uint32_t *>(&r);
#pragma unroll
    for (int e = 0; e < VEC; ++e)
        if (e < there) {
            if constexpr (VEC == 4) w[e] = __float_as_uint(reinterpret_cast<const float *>(p)[e]);
            else w[e / 2] |= (uint32_t)reinterpret_cast<const uint16_t *>(p)[e] << (16 * (e & 1));
        }
    return r;
}

// what an array that is not given stands for: repetition, presence, frequency, temperature
__device__ const float logits_defaults[4] = {1.f, 0.f, 0.f, 1.f};

// grid = (pieces, rows)
template <typename T, int THREADS, int GROUPS>
__global__ __launch_bounds__(THREADS) void logits_kernel(LogitsArgs a) {
#pragma clang fp contract(off)
    constexpr int VEC = Elem<T>::VEC, PIECE = THREADS * GROUPS * VEC;
    __shared__ __align__(16) uint32_t count[PIECE];
    const int i = blockIdx.y, v0 = (int)blockIdx.x * PIECE, tid = threadIdx.x;
    const T *c = static_cast<const T *>(a.logits) + (a.guided ? 2 : 1) * (int64_t)i * a.logits_stride;
    const T *u = c + a.logits_stride;
    const float *bias = a.p.bias ? a.p.bias + (int64_t)i * a.p.bias_stride : nullptr;
    const uint32_t *mask = a.p.mask ? a.p.mask + (int64_t)i * a.p.mask_stride : nullptr;

    // all four at once, before anything waits
    const float rep0 = *(a.p.repetition ? a.p.repetition + i : logits_defaults), presence = *(a.p.presence ? a.p.presence + i : logits_defaults + 1);
    const float frequency = *(a.p.frequency ? a.p.frequency + i : logits_defaults + 2);
    const float temp0 = *(a.p.temperature ? a.p.temperature + i : logits_defaults + 3);
    const bool told = a.p.tokens != nullptr;
    int64_t n = told ? a.p.n_tokens[i] : 0;
    const int64_t n_prompt = told && a.p.n_prompt ? a.p.n_prompt[i] : 0;
    uint4 cr[GROUPS], ur[GROUPS];
    uint32_t allowed[GROUPS];
#pragma unroll
    for (int g = 0; g < GROUPS; ++g) {
        const int v = v0 + (g * THREADS + tid) * VEC;
        cr[g] = load_logits(c + v, a.V - v);
        if (a.guided) ur[g] = load_logits(u + v, a.V - v);
        allowed[g] = mask && v < a.V ? mask[v >> 5] >> (v & 31) : ~0u;      // a group lies in one word
    }
    if (told) {
#pragma unroll
        for (int j = 0; j < PIECE / 4; j += THREADS) *reinterpret_cast<uint4 *>(&count[4 * (j + tid)]) = make_uint4(0, 0, 0, 0);
        __syncthreads();
        n = n < 0 ? 0 : n > a.p.token_stride ? a.p.token_stride : n;
        const int32_t *tok = a.p.tokens + (int64_t)i * a.p.token_stride;
        auto one = [&](int t, int64_t j) {
            const unsigned at = (unsigned)t - (unsigned)v0;
            if (at < (unsigned)PIECE && t < a.V) {
                if (j >= n_prompt) atomicAdd(&count[at], 1u);
                atomicOr(&count[at], SEEN);
            }
        };
        int64_t j = 4 * tid;
#pragma unroll 4
        for (; j + 4 <= n; j += 4 * THREADS) {
            const i32x4_any_t t = *reinterpret_cast<const i32x4_any_t *>(tok + j);
#pragma unroll
            for (int e = 0; e < 4; ++e) one(t[e], j + e);
        }
        for (int e = 0; e < 4 && j + e < n; ++e) one(tok[j + e], j + e);
        __syncthreads();
    }
    const float rep = rep0 > 0.f ? rep0 : 1.f, temp = temp0 > 0.f ? temp0 : 1.f;
    // the reciprocal in two factors, 1 and a normal number: one that overflows would make NaN of 0, one below the normal numbers has fewer bits
    const float part = temp < 0x1p-126f ? 0x1p64f : temp > 0x1p126f ? 0x1p-64f : 1.f, cool = 1.f / (temp * part);
    float *o = a.out + (int64_t)i * a.out_stride;
#pragma unroll
    for (int g = 0; g < GROUPS; ++g) {
        const int at = (g * THREADS + tid) * VEC, v = v0 + at;
        if (v >= a.V) break;
        float x[VEC], y[VEC];
        Elem<T>::unpack(cr[g], x);
        if (a.guided) {
            Elem<T>::unpack(ur[g], y);
#pragma unroll
            for (int e = 0; e < VEC; ++e) x[e] = x[e] + a.gamma * (x[e] - y[e]);
        }
        const bool full = v + VEC <= a.V;
        if (bias) {
#pragma unroll
            for (int e = 0; e < VEC; e += 4) {
                f32x4_t w = {0.f, 0.f, 0.f, 0.f};
                if (full) w = *reinterpret_cast<const f32x4_any_t *>(bias + v + e);
                else
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        if (v + e + k < a.V) w[k] = bias[v + e + k];
#pragma unroll
                for (int k = 0; k < 4; ++k) x[e + k] = x[e + k] + w[k];
            }
        }
        if (told) {
            uint32_t n[VEC], any = 0;
#pragma unroll
            for (int e = 0; e < VEC; e += 4) *reinterpret_cast<uint4 *>(&n[e]) = *reinterpret_cast<const uint4 *>(&count[at + e]);
#pragma unroll
            for (int e = 0; e < VEC; ++e) any |= n[e];
            if (any) {
#pragma unroll
                for (int e = 0; e < VEC; ++e)
                    if (n[e]) {
                        x[e] = x[e] > 0.f ? x[e] / rep : x[e] * rep;
                        const uint32_t times = n[e] & ~SEEN;
                        x[e] = x[e] - (frequency * (float)times + (times ? presence : 0.f));
                    }
            }
        }
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
            x[e] = x[e] * cool * part;
            x[e] = allowed[g] >> e & 1 ? x[e] : -INFINITY;
        }
        if (full) {
#pragma unroll
            for (int e = 0; e < VEC; e += 4)                       // written once, and more than L2 holds where it counts
                __builtin_nontemporal_store((f32x4_any_t)f32x4_t{x[e], x[e + 1], x[e + 2], x[e + 3]}, reinterpret_cast<f32x4_any_t *>(o + v + e));
        } else {
#pragma unroll
            for (int e = 0; e < VEC; ++e)
                if (v + e < a.V) o[v + e] = x[e];
        }
    }
}

template <typename T> static void launch_logits(const LogitsArgs &a, int n_rows, hipStream_t s) {
    const int64_t large = 8192, small = 2048;
    // large pieces read a row's tokens less often, small ones fill the chip (256 rows of 128257 70 us and 88, 32 13.1 and 14.5, 8 8.7 and 8.3)
    if ((int64_t)n_rows * ((a.V + large - 1) / large) >= 512) {
        constexpr int G = 16 / Elem<T>::VEC;
        hipLaunchKernelGGL((logits_kernel<T, 512, G>), dim3((unsigned)((a.V + large - 1) / large), (unsigned)n_rows), dim3(512), 0, s, a);
    } else {
        constexpr int G = 8 / Elem<T>::VEC;
        hipLaunchKernelGGL((logits_kernel<T, 256, G>), dim3((unsigned)((a.V + small - 1) / small), (unsigned)n_rows), dim3(256), 0, s, a);
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
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (dtype == SSD_F32) launch_logits<float>(a, n_rows, s);
    else launch_logits<bf16_t>(a, n_rows, s);
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? SSD_OK : hip_fail(e, "logits launch");
}
