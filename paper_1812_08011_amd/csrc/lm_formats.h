// Values of the storage formats for the language-model operators: one element
// at a time by format tag (FP8T_FMT_*), and the host checks they share.
#pragma once

#include "fp8t_device.h"
#include "fp8t_host.h"
#include "fp8train_lm.h"

namespace fp8t {

template <int FMT>
struct fmt_store;
template <>
struct fmt_store<FP8T_FMT_F32> { using type = float; };
template <>
struct fmt_store<FP8T_FMT_FP16> { using type = uint16_t; };
template <>
struct fmt_store<FP8T_FMT_FP8> { using type = uint8_t; };
template <int FMT>
using fmt_t = typename fmt_store<FMT>::type;

template <int FMT>
__device__ __forceinline__ float fmt_value(fmt_t<FMT> c) {
    if constexpr (FMT == FP8T_FMT_F32) return c;
    else if constexpr (FMT == FP8T_FMT_FP16) return fp16_to_f32(c);
    else return fp8_to_f32<0>(c);
}

template <int FMT>
__device__ __forceinline__ fmt_t<FMT> fmt_code(float x) {
    if constexpr (FMT == FP8T_FMT_F32) return x;
    else if constexpr (FMT == FP8T_FMT_FP16) return f32_to_fp16_rn(x);
    else return (uint8_t)f32_to_fp8(x);
}

// Two FP16 codes of finite values: exponent and significand moved into a
// float's fields, whose bias is 96 higher, restored by an exact product (FP16's
// subnormals are FP32 subnormals there).
__device__ __forceinline__ float2 fp16_finite_pair(uint32_t w) {
    const uint32_t lo = (uint32_t)((int32_t)(w << 16) >> 2) & 0x9FFFC000u;
    const uint32_t hi = (uint32_t)((int32_t)w >> 2) & 0x9FFFC000u;
    return make_float2(__uint_as_float(lo) * 0x1p96f, __uint_as_float(hi) * 0x1p96f);
}
// Bits 15 and 31: whether the codes of a word are Inf or NaN (exponent 63).
__device__ __forceinline__ uint32_t fp16_nonfinite(uint32_t w) {
    return (w & 0x7E007E00u) + 0x02000200u;
}

// Two FP16 codes of values below 2^31 in magnitude, rounded to nearest even once:
// with E the value's power of two, but at least 2^-30 (below, FP16's step stays
// what it is there), the sum |x| + 2^14 E has FP16's step at x, and what it
// passes 2^14 E by is the significand; it carries into the exponent by itself.
__device__ __forceinline__ uint32_t fp16_pair(float a, float b) {
    uint32_t r[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const float x = i ? b : a;
        const uint32_t u = __float_as_uint(x), e0 = 97u << 23, e = max(u & 0x7F800000u, e0);
        const float sum = __builtin_fabsf(x) + __uint_as_float(e + (14u << 23));
        const uint32_t code = __float_as_uint(sum) - e + (e >> 14) - ((14u << 23) + (e0 >> 14));
        r[i] = code | ((u >> 16) & 0x8000u);
    }
    return r[0] | (r[1] << 16);
}

// Eight consecutive elements at any address (rows start where they start), as
// wide as the alignment of one element allows.
template <int FMT>
struct Eight;
template <>
struct Eight<FP8T_FMT_F32> {
    typedef float v4 __attribute__((ext_vector_type(4), aligned(4)));
    v4 a, b;
};
template <>
struct Eight<FP8T_FMT_FP16> {
    typedef uint32_t v4 __attribute__((ext_vector_type(4), aligned(2)));
    v4 a;
};
template <>
struct Eight<FP8T_FMT_FP8> {
    typedef uint32_t v2 __attribute__((ext_vector_type(2), aligned(1)));
    v2 a;
};

// Their values, and whether one is Inf or NaN (FP16).
template <int FMT>
__device__ __forceinline__ void values_of(const Eight<FMT>& e, bool special, float* x) {
    if constexpr (FMT == FP8T_FMT_F32) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[i] = e.a[i];
            x[4 + i] = e.b[i];
        }
    } else if constexpr (FMT == FP8T_FMT_FP8) {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = fp8_to_f32<0>((e.a[i / 4] >> (8 * (i % 4))) & 0xFFu);
    } else if (__builtin_expect(special, 0)) {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = fp16_to_f32((e.a[i / 2] >> (16 * (i % 2))) & 0xFFFFu);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 p = fp16_finite_pair(e.a[i]);
            x[2 * i] = p.x;
            x[2 * i + 1] = p.y;
        }
    }
}
// Whether an element is Inf or NaN.
template <int FMT>
__device__ __forceinline__ bool special_in(const Eight<FMT>& e) {
    if constexpr (FMT != FP8T_FMT_FP16) return false;
    else
        return ((fp16_nonfinite(e.a[0]) | fp16_nonfinite(e.a[1]) | fp16_nonfinite(e.a[2]) |
                 fp16_nonfinite(e.a[3])) & 0x80008000u) != 0;
}
// n <= 8 results to p on, at any address.
template <int FMT>
__device__ __forceinline__ void store_some(fmt_t<FMT>* p, int n, const float* x) {
    if (n == 8) {
        Eight<FMT> e;
        if constexpr (FMT == FP8T_FMT_F32) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                e.a[i] = x[i];
                e.b[i] = x[4 + i];
            }
        } else if constexpr (FMT == FP8T_FMT_FP16) {
            float top = 0.0f;
#pragma unroll
            for (int i = 0; i < 4; ++i) top = maximum3_abs(top, x[2 * i], x[2 * i + 1]);
            if (__builtin_expect(top < 0x1p31f, 1)) {
#pragma unroll
                for (int i = 0; i < 4; ++i) e.a[i] = fp16_pair(x[2 * i], x[2 * i + 1]);
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    e.a[i] = (uint32_t)f32_to_fp16_rn(x[2 * i]) |
                             ((uint32_t)f32_to_fp16_rn(x[2 * i + 1]) << 16);
            }
        } else {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const uint32_t lo = f32x2_to_fp8x2<false>(x[4 * i], x[4 * i + 1], 0u);
                e.a[i] = f32x2_to_fp8x2<true>(x[4 * i + 2], x[4 * i + 3], lo);
            }
        }
        *reinterpret_cast<Eight<FMT>*>(p) = e;
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < n) p[i] = fmt_code<FMT>(x[i]);
    }
}
__device__ __forceinline__ int up_to_8(int n) { return n < 0 ? 0 : n < 8 ? n : 8; }

// Whether the rows of a T x H x D result with strides ts and hs are apart:
// heads inside tokens or tokens inside heads.
inline bool rows_apart(int64_t T, int64_t H, int64_t D, int64_t ts, int64_t hs) {
    if (ts < 0 || hs < 0) return false;
    if (T > 1 && ts < D) return false;
    if (H > 1 && hs < D) return false;
    if (T <= 1 || H <= 1) return true;
    return (ts - D) / (H - 1) >= hs || (hs - D) / (T - 1) >= ts;   // no product: it may pass 64 bits
}

}  // namespace fp8t
