// Rows of codes or floats at any address, eight elements at a time, and
// reductions over the threads of a row.
#pragma once

#include "fp8train_tokens.h"
#include "lm_formats.h"

namespace fp8t {

// The eight columns of a row that a thread holds: two fours, beside each other
// or (FOURS) apart by the fours of the row's other threads.  Where floats are
// stored they are apart, so that a wave's 16 bytes a lane are whole lines: 16384
// x 2048 floats written in 42 us with eights, in 27 with fours (past the caches;
// 36 through them).  Codes alone move as eights.
template <bool FOURS>
struct Cols {
    int64_t a, b;
    // unit u of thread tid of T
    __device__ __forceinline__ Cols(int64_t u, int tid, int T) {
        a = FOURS ? (u * 2 * T + tid) * 4 : (u * T + tid) * 8;
        b = FOURS ? a + 4 * (int64_t)T : a + 4;
    }
    __device__ __forceinline__ bool any(int64_t W) const { return a < W; }
    __device__ __forceinline__ bool has(int i, int64_t W) const { return (i < 4 ? a + i : b + i - 4) < W; }
};

// Four consecutive elements at any address.
template <int FMT>
struct FourOf;
template <>
struct FourOf<FP8T_FMT_F32> { typedef float type __attribute__((ext_vector_type(4), aligned(4))); };
template <>
struct FourOf<FP8T_FMT_FP16> { typedef uint32_t type __attribute__((ext_vector_type(2), aligned(2))); };
template <>
struct FourOf<FP8T_FMT_FP8> { typedef uint32_t type __attribute__((aligned(1))); };
// Eight codes that are one vector.
template <int FMT>
struct AllOf;
template <>
struct AllOf<FP8T_FMT_FP16> { typedef Eight<FP8T_FMT_FP16>::v4 type; };
template <>
struct AllOf<FP8T_FMT_FP8> { typedef Eight<FP8T_FMT_FP8>::v2 type; };

// Four h (0 or 1) of eight stored elements.
template <int FMT>
__device__ __forceinline__ typename FourOf<FMT>::type four_of(const Eight<FMT>& e, int h) {
    if constexpr (FMT == FP8T_FMT_F32) return h ? e.b : e.a;
    else if constexpr (FMT == FP8T_FMT_FP16) return typename FourOf<FMT>::type{e.a[2 * h], e.a[2 * h + 1]};
    else return e.a[h];
}
template <int FMT>
__device__ __forceinline__ void set_four(Eight<FMT>& e, int h, const typename FourOf<FMT>::type& f) {
    if constexpr (FMT == FP8T_FMT_F32) (h ? e.b : e.a) = f;
    else if constexpr (FMT == FP8T_FMT_FP16) {
        e.a[2 * h] = f[0];
        e.a[2 * h + 1] = f[1];
    } else e.a[h] = f;
}
// Element i of eight stored ones.
template <int FMT>
__device__ __forceinline__ fmt_t<FMT> element_of(const Eight<FMT>& e, int i) {
    if constexpr (FMT == FP8T_FMT_F32) return i < 4 ? e.a[i % 4] : e.b[i % 4];
    else if constexpr (FMT == FP8T_FMT_FP16) return (uint16_t)(e.a[i / 2] >> (16 * (i % 2)));
    else return (uint8_t)(e.a[i / 4] >> (8 * (i % 4)));
}
template <int FMT>
__device__ __forceinline__ void set_element(Eight<FMT>& e, int i, fmt_t<FMT> x) {
    if constexpr (FMT == FP8T_FMT_F32) (i < 4 ? e.a : e.b)[i % 4] = x;
    else if constexpr (FMT == FP8T_FMT_FP16) e.a[i / 2] |= (uint32_t)x << (16 * (i % 2));
    else e.a[i / 4] |= (uint32_t)x << (8 * (i % 4));
}

// A row's elements as they are stored, 0 past its end.
template <int FMT, bool FOURS>
__device__ __forceinline__ Eight<FMT> load8(const fmt_t<FMT>* row, const Cols<FOURS>& c, int64_t W) {
    if (c.b + 4 <= W) {
        if constexpr (!FOURS) return *reinterpret_cast<const Eight<FMT>*>(row + c.a);
        Eight<FMT> e;
        set_four<FMT>(e, 0, *reinterpret_cast<const typename FourOf<FMT>::type*>(row + c.a));
        set_four<FMT>(e, 1, *reinterpret_cast<const typename FourOf<FMT>::type*>(row + c.b));
        return e;
    }
    Eight<FMT> e = {};
    if (FOURS && c.a + 4 <= W) {                            // a row's last fours
        set_four<FMT>(e, 0, *reinterpret_cast<const typename FourOf<FMT>::type*>(row + c.a));
#pragma unroll
        for (int i = 4; i < 8; ++i)
            if (c.b + i - 4 < W) set_element<FMT>(e, i, row[c.b + i - 4]);
        return e;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (c.has(i, W)) set_element<FMT>(e, i, row[i < 4 ? c.a + i : c.b + i - 4]);
    return e;
}

// Results past what the caches hold are stored past them (`stream`): what they
// push out there may be wanted, they will not be found there.
constexpr int64_t kStreamBytes = 32 << 20;
// OF::type: a vector type, whose alignment (a template's own argument would lose it)
// is one element's.
template <typename OF>
__device__ __forceinline__ void put_vector(typename OF::type* p, const typename OF::type& v, bool stream) {
    if (stream) {
        asm volatile("; past the caches");                  // or the two stores become one plain one
        __builtin_nontemporal_store(v, p);
        asm volatile("; past the caches");
    } else {
        *p = v;
    }
}
template <int FMT, bool FOURS>
__device__ __forceinline__ void store8(fmt_t<FMT>* row, const Cols<FOURS>& c, int64_t W, const Eight<FMT>& e,
                                       bool stream) {
    using Four = typename FourOf<FMT>::type;
    if (c.b + 4 <= W) {
        if constexpr (FOURS || FMT == FP8T_FMT_F32) {
            put_vector<FourOf<FMT>>(reinterpret_cast<Four*>(row + c.a), four_of<FMT>(e, 0), stream);
            put_vector<FourOf<FMT>>(reinterpret_cast<Four*>(row + c.b), four_of<FMT>(e, 1), stream);
        } else {
            put_vector<AllOf<FMT>>(reinterpret_cast<typename AllOf<FMT>::type*>(row + c.a), e.a, stream);
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (c.has(i, W)) row[i < 4 ? c.a + i : c.b + i - 4] = element_of<FMT>(e, i);
}

template <int FMT>
__device__ __forceinline__ void values8(const Eight<FMT>& e, float* x) {
    if constexpr (FMT == FP8T_FMT_FP8) {
        // E5M2 to FP32, exact, specials included
        typedef float v2f __attribute__((ext_vector_type(2)));
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const v2f lo = __builtin_amdgcn_cvt_pk_f32_bf8((int)e.a[i], false);
            const v2f hi = __builtin_amdgcn_cvt_pk_f32_bf8((int)e.a[i], true);
            x[4 * i] = lo[0];
            x[4 * i + 1] = lo[1];
            x[4 * i + 2] = hi[0];
            x[4 * i + 3] = hi[1];
        }
    } else {
        values_of<FMT>(e, special_in<FMT>(e), x);
    }
}

// Eight values of a row in a format that is known at run time only (uniform).
template <bool FOURS>
__device__ __forceinline__ void load_values8(const void* row, int fmt, const Cols<FOURS>& c, int64_t W, float* x) {
    if (fmt == FP8T_FMT_F32)
        values8<FP8T_FMT_F32>(load8<FP8T_FMT_F32>(static_cast<const float*>(row), c, W), x);
    else
        values8<FP8T_FMT_FP16>(load8<FP8T_FMT_FP16>(static_cast<const uint16_t*>(row), c, W), x);
}

// Eight floats as a format stores them.
template <int FMT>
__device__ __forceinline__ Eight<FMT> codes8(const float* x) {
    Eight<FMT> e;
    if constexpr (FMT == FP8T_FMT_F32) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            e.a[i] = x[i];
            e.b[i] = x[4 + i];
        }
    } else {
        // results that need no saturation and are no NaN, as nearly always, take
        // four instructions (FP8), or no overflow's (FP16)
        float top = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; i += 2) top = maximum3_abs(top, x[i], x[i + 1]);
        if constexpr (FMT == FP8T_FMT_FP16) {
            if (__builtin_expect(top < 0x1p31f, 1)) {
#pragma unroll
                for (int i = 0; i < 4; ++i) e.a[i] = fp16_pair(x[2 * i], x[2 * i + 1]);
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    e.a[i] = (uint32_t)f32_to_fp16_rn(x[2 * i]) | ((uint32_t)f32_to_fp16_rn(x[2 * i + 1]) << 16);
            }
        } else if (__builtin_expect(top <= 57344.0f, 1)) {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const uint32_t w = __builtin_amdgcn_cvt_pk_bf8_f32(x[4 * i], x[4 * i + 1], 0, false);
                e.a[i] = __builtin_amdgcn_cvt_pk_bf8_f32(x[4 * i + 2], x[4 * i + 3], w, true);
            }
        } else {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const uint32_t lo = f32x2_to_fp8x2<false>(x[4 * i], x[4 * i + 1], 0u);
                e.a[i] = f32x2_to_fp8x2<true>(x[4 * i + 2], x[4 * i + 3], lo);
            }
        }
    }
    return e;
}
template <int FMT, bool FOURS>
__device__ __forceinline__ void put8(fmt_t<FMT>* row, const Cols<FOURS>& c, int64_t W, const float* x, bool stream) {
    store8<FMT>(row, c, W, codes8<FMT>(x), stream);
}
// The same in a format that is known at run time only (uniform).
template <bool FOURS>
__device__ __forceinline__ void put_as8(void* row, int fmt, const Cols<FOURS>& c, int64_t W, const float* x,
                                        bool stream) {
    if (fmt == FP8T_FMT_F32) put8<FP8T_FMT_F32>(static_cast<float*>(row), c, W, x, stream);
    else if (fmt == FP8T_FMT_FP16) put8<FP8T_FMT_FP16>(static_cast<uint16_t*>(row), c, W, x, stream);
    else put8<FP8T_FMT_FP8>(static_cast<uint8_t*>(row), c, W, x, stream);
}
inline int64_t bytes_of(int fmt) { return fmt == FP8T_FMT_F32 ? 4 : fmt == FP8T_FMT_FP16 ? 2 : 1; }

// Eight floats rounded to F32 or FP16: what is stored, and x what that stands for.
template <int FMT>
__device__ __forceinline__ Eight<FMT> rounded8(float* x) {
    const Eight<FMT> e = codes8<FMT>(x);
    if constexpr (FMT != FP8T_FMT_F32) values8<FMT>(e, x);
    return e;
}

// x of another lane of the same 16, without LDS.
template <int CTRL>
__device__ __forceinline__ double dpp(double x) {
    const uint64_t u = __double_as_longlong(x);
    const uint32_t lo = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)u, CTRL, 0xF, 0xF, true);
    const uint32_t hi = __builtin_amdgcn_update_dpp(0, (int)(u >> 32), CTRL, 0xF, 0xF, true);
    return __longlong_as_double((long long)(((uint64_t)hi << 32) | lo));
}

// A reduction over the T threads of a row, T a power of two and rows beside each
// other in the workgroup; every thread gets the same bits.  T up to 64 needs no
// LDS; else red has a number for each wave of the workgroup, free before the
// call, and all its threads call.
template <int T, typename X, typename OP>
__device__ __forceinline__ X row_reduce(X x, X* red, OP op) {
    if constexpr (sizeof(X) == 8) {
        // doubles, half of them at a time: lanes of 16 exchange without LDS, with i ^
        // 15, i ^ 7, i ^ 2 and i ^ 1 (2048 rows of 9000, a workgroup's after each
        // other: 47 us with all steps through it, 45 so)
        static_assert(T >= 8, "a row's threads");
        if constexpr (T >= 64) x = op(x, __shfl_xor(x, 32));
        if constexpr (T >= 32) x = op(x, __shfl_xor(x, 16));
        if constexpr (T >= 16) x = op(x, dpp<0x140>(x));    // row_mirror
        x = op(x, dpp<0x141>(x));                           // row_half_mirror
        x = op(x, dpp<0x4E>(x));                            // quad_perm [2, 3, 0, 1]
        x = op(x, dpp<0xB1>(x));                            // quad_perm [1, 0, 3, 2]
    } else {
#pragma unroll
        for (int d = (T < 64 ? T : 64) / 2; d; d >>= 1) x = op(x, __shfl_xor(x, d));
    }
    if constexpr (T > 64) {
        if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = x;
        __syncthreads();
        const X* mine = red + threadIdx.x / T * (T / 64);
        x = mine[0];
#pragma unroll
        for (int i = 1; i < T / 64; ++i) x = op(x, mine[i]);
    }
    return x;
}
struct RowSum {
    template <typename X>
    __device__ X operator()(X a, X b) const { return a + b; }
};
// NaN wins.
struct RowMax {
    __device__ float operator()(float a, float b) const { return a > b || a != a ? a : b; }
};

inline bool float_or_16(int f) { return f == FP8T_FMT_F32 || f == FP8T_FMT_FP16; }
inline bool storage_format(int f) { return f >= FP8T_FMT_F32 && f <= FP8T_FMT_FP8; }
// The row of W elements with stride ld that a call may read or write.
inline bool matrix_ok(const void* p, int64_t ld, int64_t rows, int64_t W) {
    return rows == 0 || W == 0 || (p && ld >= W);
}

}  // namespace fp8t
