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

// Whether the rows of a T x H x D result with strides ts and hs are apart:
// heads inside tokens or tokens inside heads.
inline bool rows_apart(int64_t T, int64_t H, int64_t D, int64_t ts, int64_t hs) {
    if (ts < 0 || hs < 0) return false;
    if (T > 1 && ts < D) return false;
    if (H > 1 && hs < D) return false;
    if (T <= 1 || H <= 1) return true;
    return ts / H >= hs || ts - D >= (H - 1) * hs || hs / T >= ts || hs - D >= (T - 1) * ts;
}

}  // namespace fp8t
