// Rows of codes or floats at any address, eight elements at a time, and
// reductions over the threads of a row.
#pragma once

#include "fp8train_tokens.h"
#include "lm_formats.h"

namespace fp8t {

// Elements c .. c + 7 of a row of W as they are stored, 0 past its end.
template <int FMT>
__device__ __forceinline__ Eight<FMT> load8(const fmt_t<FMT>* row, int64_t c, int64_t W) {
    if (c + 8 <= W) return *reinterpret_cast<const Eight<FMT>*>(row + c);
    Eight<FMT> e;
    if constexpr (FMT == FP8T_FMT_F32) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            e.a[i] = c + i < W ? row[c + i] : 0.0f;
            e.b[i] = c + 4 + i < W ? row[c + 4 + i] : 0.0f;
        }
    } else if constexpr (FMT == FP8T_FMT_FP16) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t lo = c + 2 * i < W ? row[c + 2 * i] : 0;
            const uint32_t hi = c + 2 * i + 1 < W ? row[c + 2 * i + 1] : 0;
            e.a[i] = lo | (hi << 16);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            uint32_t w = 0;
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (c + 4 * i + j < W) w |= (uint32_t)row[c + 4 * i + j] << (8 * j);
            e.a[i] = w;
        }
    }
    return e;
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
__device__ __forceinline__ void load_values8(const void* row, int fmt, int64_t c, int64_t W, float* x) {
    if (fmt == FP8T_FMT_F32)
        values8<FP8T_FMT_F32>(load8<FP8T_FMT_F32>(static_cast<const float*>(row), c, W), x);
    else
        values8<FP8T_FMT_FP16>(load8<FP8T_FMT_FP16>(static_cast<const uint16_t*>(row), c, W), x);
}

// n <= 8 results to p on; eight FP8 results that need no saturation and are no
// NaN, as nearly always, in four instructions.
template <int FMT>
__device__ __forceinline__ void store_eight(fmt_t<FMT>* p, int n, const float* x) {
    if constexpr (FMT == FP8T_FMT_FP8) {
        float top = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; i += 2) top = maximum3_abs(top, x[i], x[i + 1]);
        if (__builtin_expect(n == 8 && top <= 57344.0f, 1)) {
            Eight<FMT> e;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const uint32_t w = __builtin_amdgcn_cvt_pk_bf8_f32(x[4 * i], x[4 * i + 1], 0, false);
                e.a[i] = __builtin_amdgcn_cvt_pk_bf8_f32(x[4 * i + 2], x[4 * i + 3], w, true);
            }
            *reinterpret_cast<Eight<FMT>*>(p) = e;
            return;
        }
    }
    store_some<FMT>(p, n, x);
}

// n <= 8 results (n > 0) to elements c .. of a row.
__device__ __forceinline__ void store_values8(void* row, int fmt, int64_t c, int n, const float* x) {
    if (fmt == FP8T_FMT_F32) store_some<FP8T_FMT_F32>(static_cast<float*>(row) + c, n, x);
    else if (fmt == FP8T_FMT_FP16) store_some<FP8T_FMT_FP16>(static_cast<uint16_t*>(row) + c, n, x);
    else store_eight<FP8T_FMT_FP8>(static_cast<uint8_t*>(row) + c, n, x);
}

// Eight floats rounded to a stream's format: its codes, and x what they stand for.
template <int FMT>
__device__ __forceinline__ Eight<FMT> rounded8(float* x) {
    Eight<FMT> e;
    if constexpr (FMT == FP8T_FMT_F32) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            e.a[i] = x[i];
            e.b[i] = x[4 + i];
        }
    } else {
        float top = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; i += 2) top = maximum3_abs(top, x[i], x[i + 1]);
        if (__builtin_expect(top < 0x1p31f, 1)) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                e.a[i] = fp16_pair(x[2 * i], x[2 * i + 1]);
                const float2 p = fp16_finite_pair(e.a[i]);
                x[2 * i] = p.x;
                x[2 * i + 1] = p.y;
            }
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t lo = f32_to_fp16_rn(x[2 * i]), hi = f32_to_fp16_rn(x[2 * i + 1]);
                e.a[i] = lo | (hi << 16);
                x[2 * i] = fp16_to_f32(lo);
                x[2 * i + 1] = fp16_to_f32(hi);
            }
        }
    }
    return e;
}
// n <= 8 stored elements (F32 or FP16) to p on.
template <int FMT>
__device__ __forceinline__ void store_stored8(fmt_t<FMT>* p, int n, const Eight<FMT>& e) {
    if (n == 8) {
        *reinterpret_cast<Eight<FMT>*>(p) = e;
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        if (i >= n) break;
        if constexpr (FMT == FP8T_FMT_F32) p[i] = i < 4 ? e.a[i % 4] : e.b[i % 4];
        else p[i] = (uint16_t)(e.a[i / 2] >> (16 * (i % 2)));
    }
}

__device__ __forceinline__ int left8(int64_t c, int64_t W) {
    return W - c < 8 ? (int)(W - c) : 8;
}

// A reduction over the T threads of a row, T a power of two and rows beside each
// other in the workgroup; every thread gets the same bits.  T up to 64 needs no
// LDS; else red has a float for each wave of the workgroup, free before the
// call, and all its threads call.
template <int T, typename OP>
__device__ __forceinline__ float row_reduce(float x, float* red, OP op) {
#pragma unroll
    for (int d = (T < 64 ? T : 64) / 2; d; d >>= 1) x = op(x, __shfl_xor(x, d));
    if constexpr (T > 64) {
        if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = x;
        __syncthreads();
        const float* mine = red + threadIdx.x / T * (T / 64);
        x = mine[0];
#pragma unroll
        for (int i = 1; i < T / 64; ++i) x = op(x, mine[i]);
    }
    return x;
}
struct RowSum {
    __device__ float operator()(float a, float b) const { return a + b; }
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
