// ssd_rope_axes: heads of tokens turned by positions with one to four axes.
//
// Pair i of a token's heads turns by the angle pos[axis[i]] * inv_freq[i].  The angle's revolutions are found in 64 bits: the product and what its rounding
// left out (it has up to 55 bits) are divided by 2 pi with the quotient's rounding made up for, so that positions of 2^31 lose nothing; then the fraction of a quarter
// turn that is left is at most pi / 4, where the series of sine and cosine up to r^11 and r^10 are below 2^-28 off.
//
// Bound by HBM: every element read once and written once.  A token's angles serve all its heads: they are found once per workgroup, into LDS.  22500 tokens of 40 heads of 128
// elements (bf16) 75 us, 6.1 TB/s read and written; 4611 of 32 heads 16.2 us, 4.7; 16 tokens 3.4 us on the device, launch and latency.  (The first elements requested before
// the angles are found: 87 and 16.7 us.)
#include <cmath>

#include "ssd_device.h"

namespace ssd {

struct RopeArgs {
    const char *x;
    char *out;
    const int32_t *pos;      // [axes, n]
    const uint8_t *axis;     // [pairs], or NULL: 0
    const float *inv_freq;   // [pairs]
    int64_t x_stride, out_stride;   // bytes
    int n, heads, d, pairs, axes;
    int tokens;              // of a workgroup
    float sign;              // -1: turned back
};

// (cos, sin) of pos * f.  Products and sums stay apart: r less its whole turns, taken from x * C in one step, would have what `low` adds already.
static __device__ __forceinline__ float2 turn_of(int pos, float f, float sign) {
#pragma clang fp contract(off)
    const double x = (double)pos * (double)f, rest = __builtin_fma((double)pos, (double)f, -x);
    constexpr double C = 0x1.45f306dc9c883p-3, C2 = -0x1.6b01ec5417056p-57;        // 1 / (2 pi) in two parts
    const double r = x * C, low = __builtin_fma(x, C, -r) + __builtin_fma(x, C2, rest * C);
    const double quarter = (r - __builtin_rint(r)) * 4.0, q0 = __builtin_rint(quarter), part = (quarter - q0) + low * 4.0, q1 = __builtin_rint(part);
    const float t = (float)((part - q1) * 0x1.921fb54442d18p+0), t2 = t * t;     // at most pi / 4
    float s = __builtin_fmaf(t2, -2.50521084e-8f, 2.75573192e-6f);
    s = __builtin_fmaf(t2, s, -1.98412698e-4f);
    s = __builtin_fmaf(t2, s, 8.33333333e-3f);
    s = __builtin_fmaf(t2, s, -1.66666667e-1f);
    s = __builtin_fmaf(t2 * t, s, t);
    float c = __builtin_fmaf(t2, -2.75573192e-7f, 2.48015873e-5f);
    c = __builtin_fmaf(t2, c, -1.38888889e-3f);
    c = __builtin_fmaf(t2, c, 4.16666667e-2f);
    c = __builtin_fmaf(t2, c, -0.5f);
    c = __builtin_fmaf(t2, c, 1.f);
    const int k = ((int)q0 + (int)q1) & 3;
    const float cs = k & 1 ? s : c, sn = k & 1 ? c : s;
    return make_float2(k == 1 || k == 2 ? -cs : cs, sign * (k & 2 ? -sn : sn));
}

// N neighbouring elements.  Two may lie anywhere (interleaved pairs in rows at odd addresses).
template <typename T, int N> struct alignas(N == 2 ? sizeof(T) : sizeof(T) * N) Wide { T e[N]; };

template <typename T> static __device__ __forceinline__ float to_f32(T x) {
    if constexpr (sizeof(T) == 4) return x;
    else return __uint_as_float((uint32_t)x.bits << 16);
}
template <typename T> static __device__ __forceinline__ T from_f32(float x) {
    if constexpr (sizeof(T) == 4) return x;
    else return T{(uint16_t)f32_to_bf16_bits(x)};
}

// A run of neighbouring elements.  ONCE: of more than the memory-side cache holds.
template <typename R, bool ONCE> static __device__ __forceinline__ R load_run(const void *p) {
    if constexpr (ONCE && sizeof(R) == 16) return __builtin_bit_cast(R, __builtin_nontemporal_load(reinterpret_cast<const u32x4_nt_t *>(p)));
    else if constexpr (sizeof(R) == 16) return __builtin_bit_cast(R, *reinterpret_cast<const u32x4_nt_t *>(p));
    else return *reinterpret_cast<const R *>(p);
}
template <typename R, bool ONCE> static __device__ __forceinline__ void store_run(void *p, const R &r) {
    if constexpr (ONCE && sizeof(R) == 16) __builtin_nontemporal_store(__builtin_bit_cast(u32x4_nt_t, r), reinterpret_cast<u32x4_nt_t *>(p));
    else if constexpr (sizeof(R) == 16) *reinterpret_cast<u32x4_nt_t *>(p) = __builtin_bit_cast(u32x4_nt_t, r);
    else *reinterpret_cast<R *>(p) = r;
}

// N pairs (p[e], q[e * STEP]) turned by t = (cos, sin), or left to the bit where t is STAY: as a turn by no angle an infinity would give its partner 0 * inf.
static constexpr float STAY = 2.f;
template <int N, int STEP, typename T> static __device__ __forceinline__ void turn_pairs(T *p, T *q, const float2 *turns) {
    float2 t[N];
    float most = 0.f;
#pragma unroll
    for (int e = 0; e < N; ++e) {
        t[e] = turns[e];
        most = fmaxf(most, t[e].x);
    }
    T x[N], y[N];
#pragma unroll
    for (int e = 0; e < N; ++e) {
        const float a = to_f32<T>(p[e * STEP]), b = to_f32<T>(q[e * STEP]);
        x[e] = from_f32<T>(a * t[e].x - b * t[e].y);
        y[e] = from_f32<T>(b * t[e].x + a * t[e].y);
    }
    if (most == STAY) {                                             // rare, so asked once for all (4611 tokens of 32 heads 16.2 us; asked for every pair 17.3)
#pragma unroll
        for (int e = 0; e < N; ++e)
            if (t[e].x == STAY) {
                x[e] = p[e * STEP];
                y[e] = q[e * STEP];
            }
    }
#pragma unroll
    for (int e = 0; e < N; ++e) {
        p[e * STEP] = x[e];
        q[e * STEP] = y[e];
    }
}

// VEC: elements of a lane's run; HALF: pair i is (i, i + pairs), else (2 i, 2 i + 1).
template <typename T, int VEC, bool HALF, bool ONCE> __global__ __launch_bounds__(256) void rope_kernel(RopeArgs a) {
    extern __shared__ __align__(16) float2 turns[];               // [tokens][pairs]
    typedef Wide<T, VEC> run_t;
    const int t0 = (int)blockIdx.x * a.tokens, tokens = a.n - t0 < a.tokens ? a.n - t0 : a.tokens;
    for (int i = threadIdx.x; i < tokens * a.pairs; i += 256) {
        const int t = i / a.pairs, p = i - t * a.pairs;
        const int axis = a.axis ? a.axis[p] : 0;
        turns[i] = axis < a.axes ? turn_of(a.pos[(int64_t)axis * a.n + t0 + t], a.inv_freq[p], a.sign) : make_float2(STAY, 0.f);
    }
    __syncthreads();
    // what a lane takes at a time: runs at i and i + pairs, or 2 VEC neighbouring elements
    const int per_head = HALF ? a.pairs / VEC : 2 * a.pairs / VEC, rest = (a.d - 2 * a.pairs) / VEC, all = per_head + (a.x == a.out ? 0 : rest);
    for (int i = threadIdx.x; i < tokens * a.heads * all; i += 256) {
        const int th = i / all, c = i - th * all, t = th / a.heads, h = th - t * a.heads;
        const T *x = reinterpret_cast<const T *>(a.x + (int64_t)(t0 + t) * a.x_stride) + (int64_t)h * a.d;
        T *out = reinterpret_cast<T *>(a.out + (int64_t)(t0 + t) * a.out_stride) + (int64_t)h * a.d;
        if (c >= per_head) {
            const int at = 2 * a.pairs + (c - per_head) * VEC;
            store_run<run_t, ONCE>(out + at, load_run<run_t, ONCE>(x + at));
            continue;
        }
        if constexpr (HALF) {
            run_t u = load_run<run_t, ONCE>(x + c * VEC), w = load_run<run_t, ONCE>(x + a.pairs + c * VEC);
            turn_pairs<VEC, 1>(u.e, w.e, turns + t * a.pairs + c * VEC);
            store_run<run_t, ONCE>(out + c * VEC, u);
            store_run<run_t, ONCE>(out + a.pairs + c * VEC, w);
        } else {
            run_t u = load_run<run_t, ONCE>(x + c * VEC);
            turn_pairs<VEC / 2, 2>(u.e, u.e + 1, turns + t * a.pairs + c * VEC / 2);
            store_run<run_t, ONCE>(out + c * VEC, u);
        }
    }
}

template <typename T, bool HALF> static void launch_rope(const RopeArgs &a, int vec, hipStream_t s) {
    const dim3 grid((unsigned)((a.n + a.tokens - 1) / a.tokens));
    const unsigned lds = (unsigned)(a.tokens * a.pairs * sizeof(float2));
    // 230 MB: 84 us without the hint, 75 with it; 82 MB: 39.5 and 39.9; 38 MB: 16.2 and 21
    const bool once = (int64_t)a.n * a.heads * a.d * (int64_t)sizeof(T) > 64 << 20;
    const auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(256), lds, s, a); };
    if (vec * sizeof(T) == 16) {
        constexpr int VEC = 16 / sizeof(T);
        return once ? go(rope_kernel<T, VEC, HALF, true>) : go(rope_kernel<T, VEC, HALF, false>);
    }
    if (vec == 4) go(rope_kernel<T, 4, HALF, false>);
    else if (vec == 2 || !HALF) go(rope_kernel<T, 2, HALF, false>);
    else if constexpr (HALF) go(rope_kernel<T, 1, HALF, false>);
}

}  // namespace ssd

using namespace ssd;

extern "C" int ssd_rope_axes(const void *x, void *out, int n_rows, int n_heads, int head_dim, int dtype, int64_t x_stride, int64_t out_stride,
                             const int32_t *pos, int n_axes, const uint8_t *axis, const float *inv_freq, int n_pairs, int rope_layout, int inverse,
                             void *stream) {
    clear_error();
    if (n_rows != 0 && (!x || !out || !pos)) return fail(SSD_ERR_INVALID_ARG, "x, out or pos is NULL");
    if (!inv_freq) return fail(SSD_ERR_INVALID_ARG, "inv_freq is NULL");
    if (dtype != SSD_F32 && dtype != SSD_BF16) return fail(SSD_ERR_INVALID_ARG, "dtype=%d is neither SSD_F32 nor SSD_BF16", dtype);
    if (n_rows < 0 || n_rows >= 1 << 24) return fail(SSD_ERR_INVALID_ARG, "n_rows=%d outside 0..2^24 - 1", n_rows);
    if (n_heads < 1 || n_heads > 4096) return fail(SSD_ERR_INVALID_ARG, "n_heads=%d outside 1..4096", n_heads);
    if (head_dim < 2 || head_dim > 1024 || head_dim % 2 != 0) return fail(SSD_ERR_INVALID_ARG, "head_dim=%d must be even, 2..1024", head_dim);
    if (n_pairs < 1 || n_pairs > head_dim / 2) return fail(SSD_ERR_INVALID_ARG, "n_pairs=%d outside 1..head_dim / 2", n_pairs);
    if (n_axes < 1 || n_axes > 4) return fail(SSD_ERR_INVALID_ARG, "n_axes=%d outside 1..4", n_axes);
    if (!axis && n_axes != 1) return fail(SSD_ERR_INVALID_ARG, "axis is NULL with n_axes=%d", n_axes);
    if (rope_layout != SSD_ROPE_HALF && rope_layout != SSD_ROPE_INTERLEAVED) return fail(SSD_ERR_INVALID_ARG, "rope_layout=%d", rope_layout);
    if (inverse != 0 && inverse != 1) return fail(SSD_ERR_INVALID_ARG, "inverse=%d is neither 0 nor 1", inverse);
    const int64_t e = dtype == SSD_F32 ? 4 : 2, row = (int64_t)n_heads * head_dim;
    if ((x_stride != 0 && (x_stride < row || x_stride > 1ll << 28)) || (out_stride != 0 && (out_stride < row || out_stride > 1ll << 28)))
        return fail(SSD_ERR_INVALID_ARG, "x_stride and out_stride must be 0 or n_heads * head_dim .. 2^28");
    if (!aligned(x, e) || !aligned(out, e) || !aligned(pos, 4) || !aligned(inv_freq, 4))
        return fail(SSD_ERR_INVALID_ARG, "x, out, pos and inv_freq must be aligned to their elements");
    RopeArgs a;
    a.x_stride = (x_stride ? x_stride : row) * e;
    a.out_stride = (out_stride ? out_stride : row) * e;
    // Rows of one array onto themselves, or two arrays that have nothing in common
    const char *x0 = static_cast<const char *>(x), *o0 = static_cast<const char *>(out);
    const int64_t x_size = n_rows > 0 ? (n_rows - 1) * a.x_stride + row * e : 0, o_size = n_rows > 0 ? (n_rows - 1) * a.out_stride + row * e : 0;
    if (x0 == o0 ? n_rows > 1 && a.x_stride != a.out_stride : x0 < o0 + o_size && o0 < x0 + x_size)
        return fail(SSD_ERR_INVALID_ARG, "out must be x with the same stride, or share no memory with it");
    if (n_rows == 0) return SSD_OK;
    a.x = x0;
    a.out = static_cast<char *>(out);
    a.pos = pos;
    a.axis = axis;
    a.inv_freq = inv_freq;
    a.n = n_rows;
    a.heads = n_heads;
    a.d = head_dim;
    a.pairs = n_pairs;
    a.axes = n_axes;
    a.sign = inverse ? -1.f : 1.f;
    // the longest run, up to 16 bytes, that all sizes, strides and addresses are multiples of
    const uint64_t bits = (uint64_t)a.x_stride | (uint64_t)a.out_stride | (uintptr_t)x | (uintptr_t)out | (uint64_t)(head_dim * e) |
                          (uint64_t)((rope_layout == SSD_ROPE_HALF ? n_pairs : 2 * n_pairs) * e) | 16u;
    const int vec = (int)((int64_t)(bits & (0 - bits)) / e);
    // a token to a workgroup, or as many as its threads have pieces for (4611 tokens of 32 heads 16.2 us, of two 16.4, of four 16.4; of 8 heads 9.7, 7.6, 7.7; 22500 of 40 heads
    // 84, 88, 92)
    const int64_t pieces = (int64_t)n_heads * (head_dim / vec);
    a.tokens = 1;
    while (a.tokens < 32 && a.tokens * pieces < 256 && (int64_t)a.tokens * n_pairs < 1024) a.tokens *= 2;
    hipStream_t s = static_cast<hipStream_t>(stream);
    const bool half = rope_layout == SSD_ROPE_HALF;
    if (dtype == SSD_F32) half ? launch_rope<float, true>(a, vec, s) : launch_rope<float, false>(a, vec, s);
    else half ? launch_rope<bf16_t, true>(a, vec, s) : launch_rope<bf16_t, false>(a, vec, s);
    const hipError_t err = hipGetLastError();
    return err == hipSuccess ? SSD_OK : hip_fail(err, "rope launch");
}
