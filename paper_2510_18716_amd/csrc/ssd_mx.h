// The block formats of a quantised pool (OCP microscaling): 32 consecutive elements of a row share 2^E, kept as the byte E + 127 (255: the whole block is
// NaN); an element is E4M3 (MXFP8) or E2M1 (MXFP4, the even element of a byte in its low bits).
//
// E is the smallest exponent with which no element is off by more than half a step: largest |x| <= 464 * 2^E or 7 * 2^E, half a step above the largest
// element there is (448, 6).  Elements are rounded to the nearest, ties to the even code; division by 2^E is exact, so a code follows from the definition
// alone.  E is at least -117 (-125): every element but 0 is then a normal number of fp32 and bf16, and in blocks of
// smaller numbers half of the smallest step stays 2^-127.  The instructions that convert (v_cvt_scalef32_*) take the scale as the fp32 number 2^E, round so, and give NaN for
// the scale byte 255; checked for every scale and code, and for ties, on the device.
#pragma once

#include "ssd_device.h"

namespace ssd {

typedef short s16x2_t __attribute__((ext_vector_type(2)));

template <int BITS> struct Mx;

template <> struct Mx<8> {
    static constexpr int LOWEST = 10, TOP = 8;                     // least byte of a scale; exponent of the largest element
    static constexpr uint32_t HALF = 0x680000u;                    // 464 = 1.8125 * 2^8: its bits behind the point
};
template <> struct Mx<4> {
    static constexpr int LOWEST = 2, TOP = 2;
    static constexpr uint32_t HALF = 0x600000u;                    // 7 = 1.75 * 2^2
};

// The scale byte of a block whose largest |x| has the bits u.
template <int BITS> static __device__ __forceinline__ uint32_t mx_scale_of(uint32_t u) {
    if (u >= 0x7f800000u) return 255;
    const int e = (int)((u + (0x7fffffu - Mx<BITS>::HALF)) >> 23) - Mx<BITS>::TOP;      // one more where the bits behind the point are above HALF
    return (uint32_t)(e < Mx<BITS>::LOWEST ? Mx<BITS>::LOWEST : e);
}

// Largest over the four lanes from a multiple of four on.
static __device__ __forceinline__ uint32_t quad_max(uint32_t v) {
    uint32_t o = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0xB1, 0xF, 0xF, false);
    v = o > v ? o : v;
    o = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x4E, 0xF, 0xF, false);
    return o > v ? o : v;
}

// Eight elements of a row, as they lie in memory.
template <typename T> struct Eight { u32x4_nt_t r[sizeof(T) / 2]; };

template <typename T> static __device__ __forceinline__ Eight<T> load_eight(const char *p) {
    Eight<T> x;
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; ++i) x.r[i] = __builtin_nontemporal_load(reinterpret_cast<const u32x4_nt_t *>(p) + i);
    return x;
}

// Bits of the largest |x| of eight elements.  Compared as whole numbers, so that infinities and NaN are above all others.
template <typename T> static __device__ __forceinline__ uint32_t largest_of(const Eight<T> &x) {
    uint32_t u = 0;
    const auto add = [&](uint32_t bits) {
        bits &= 0x7fffffffu;
        u = bits > u ? bits : u;
    };
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if constexpr (sizeof(T) == 4) {
                add(x.r[i][e]);
            } else {
                add(x.r[i][e] << 16);
                add(x.r[i][e] & 0xffff0000u);
            }
        }
    return u;
}

// A dword as two elements.  By value: the cast of a vector's element would take the first one.
static __device__ __forceinline__ bf16x2_t two(uint32_t v) { return __builtin_bit_cast(bf16x2_t, v); }

// Codes of eight elements: BITS bytes.
template <int BITS> struct Codes { uint32_t c[BITS / 4]; };

template <int BITS, typename T> static __device__ __forceinline__ Codes<BITS> mx_encode(const Eight<T> &x, uint32_t byte) {
    const float scale = __uint_as_float(byte << 23);
    Codes<BITS> o;
    if constexpr (BITS == 4) {
        uint32_t c = 0;
        if constexpr (sizeof(T) == 4) {
            c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, __uint_as_float(x.r[0][0]), __uint_as_float(x.r[0][1]), scale, 0);
            c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, __uint_as_float(x.r[0][2]), __uint_as_float(x.r[0][3]), scale, 1);
            c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, __uint_as_float(x.r[1][0]), __uint_as_float(x.r[1][1]), scale, 2);
            c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, __uint_as_float(x.r[1][2]), __uint_as_float(x.r[1][3]), scale, 3);
        } else {
            c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, two(x.r[0][0]), scale, 0);
            c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, two(x.r[0][1]), scale, 1);
            c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, two(x.r[0][2]), scale, 2);
            c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, two(x.r[0][3]), scale, 3);
        }
        o.c[0] = byte == 255 ? 0u : c;
    } else {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            s16x2_t c = {0, 0};
            if constexpr (sizeof(T) == 4) {
                c = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(c, __uint_as_float(x.r[i][0]), __uint_as_float(x.r[i][1]), scale, false);
                c = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(c, __uint_as_float(x.r[i][2]), __uint_as_float(x.r[i][3]), scale, true);
            } else {
                c = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(c, two(x.r[0][2 * i]), scale, false);
                c = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(c, two(x.r[0][2 * i + 1]), scale, true);
            }
            o.c[i] = byte == 255 ? 0u : __builtin_bit_cast(uint32_t, c);
        }
    }
    return o;
}

// Two neighbouring elements as bf16: pair P of a dword of codes.  Exact: no element has more than four significant bits.
template <int BITS, int P> static __device__ __forceinline__ uint32_t mx_pair(uint32_t codes, float scale) {
    if constexpr (BITS == 4) return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, P));
    else return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, scale, P != 0));
}

// Eight elements from their codes.
template <int BITS, typename T> static __device__ __forceinline__ Eight<T> mx_decode(const Codes<BITS> &c, uint32_t byte) {
    const float scale = __uint_as_float(byte << 23);
    uint32_t p[4];
    if constexpr (BITS == 4) {
        p[0] = mx_pair<4, 0>(c.c[0], scale);
        p[1] = mx_pair<4, 1>(c.c[0], scale);
        p[2] = mx_pair<4, 2>(c.c[0], scale);
        p[3] = mx_pair<4, 3>(c.c[0], scale);
    } else {
        p[0] = mx_pair<8, 0>(c.c[0], scale);
        p[1] = mx_pair<8, 1>(c.c[0], scale);
        p[2] = mx_pair<8, 0>(c.c[1], scale);
        p[3] = mx_pair<8, 1>(c.c[1], scale);
    }
    Eight<T> o;
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int i = 0; i < 2; ++i) o.r[i] = u32x4_nt_t{p[2 * i] << 16, p[2 * i] & 0xffff0000u, p[2 * i + 1] << 16, p[2 * i + 1] & 0xffff0000u};
    } else {
        o.r[0] = u32x4_nt_t{p[0], p[1], p[2], p[3]};
    }
    return o;
}

}  // namespace ssd
