// Pieces of the matrix-core attention kernels.
//
// Every product is formed transposed, so that a lane owns one column (a query
// in the forward and dq kernels, a key in the dk/dv kernel) and a result's rows
// lie in its registers:
//   * scores: S^T = K Q^T (32x32x16, IEEE half).  The FP8 matrix instructions
//     would take the codes as they are at twice the rate, but they cut the
//     products of eight k to 13 bits below the largest; halves keep every
//     product exact and the sum in FP32.  The order of k is free as long as
//     both operands agree: a lane takes 16 contiguous codes of its row for two
//     instructions.  Result register 4 g + r of lane l is row 8 g + 4 (l / 32)
//     + r, column l % 32.
//   * the second product, e.g. O^T = V^T P^T, takes its
//     right operand from those registers without moving anything between
//     lanes: registers 8 t .. 8 t + 7 are the lane's eight values of
//     instruction t, whose k order is then rows 16 t + {4 h .. 4 h + 3,
//     8 + 4 h .. 8 + 4 h + 3} for lane half h.  The left operand is staged in
//     LDS in that order (HalfTile).
// A 1-5-2 code is the upper byte of the IEEE half of the same value, so codes
// become halves exactly by a byte permutation, which also transposes.
#pragma once

#include "attn.h"

namespace fp8t {

typedef float v16f __attribute__((ext_vector_type(16)));
typedef float v2f __attribute__((ext_vector_type(2)));
typedef _Float16 v2h __attribute__((ext_vector_type(2)));
typedef _Float16 v8h __attribute__((ext_vector_type(8)));

__device__ __forceinline__ v16f mfma_half(v8h a, v8h b, v16f c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
}

// op over the two lanes that hold a column.
template <typename OP>
__device__ __forceinline__ float both_halves(float x, OP op) {
    const uint32_t u = __float_as_uint(x);
    const auto t = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    return op(__uint_as_float(t[0]), __uint_as_float(t[1]));
}

// Eight registers of a result as the half operand of the next product.
__device__ __forceinline__ v8h to_half8(const float* x) {
    v8h r;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const v2f f = {x[2 * i], x[2 * i + 1]};
        const v2h p = __builtin_convertvector(f, v2h);
        r[2 * i] = p[0];
        r[2 * i + 1] = p[1];
    }
    return r;
}

// Bytes d0 .. d0 + 15 of a row of D codes, zero past D or where !live.
template <bool VEC>
__device__ __forceinline__ uint4 load_codes16(const uint8_t* row, int d0, int D, bool live) {
    uint4 v = make_uint4(0, 0, 0, 0);
    if constexpr (VEC) {
        if (live && d0 < D) v = *reinterpret_cast<const uint4*>(row + d0);
    } else if (live) {
        uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
        for (int i = 0; i < 16; ++i)
            if (d0 + i < D) w[i / 4] |= (uint32_t)row[d0 + i] << (8 * (i % 4));
        v = make_uint4(w[0], w[1], w[2], w[3]);
    }
    return v;
}
template <bool VEC>
__device__ __forceinline__ uint2 load_codes8(const uint8_t* row, int d0, int D, bool live) {
    uint2 v = make_uint2(0, 0);
    if constexpr (VEC) {
        if (live && d0 < D) v = *reinterpret_cast<const uint2*>(row + d0);
    } else if (live) {
        uint32_t w[2] = {0, 0};
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (d0 + i < D) w[i / 4] |= (uint32_t)row[d0 + i] << (8 * (i % 4));
        v = make_uint2(w[0], w[1]);
    }
    return v;
}
// Eight codes as halves, in order.  The selectors are in vector registers (an
// instruction that reads a scalar one issues at half rate).
struct Widen {
    uint32_t lo, hi;
    __device__ __forceinline__ Widen() : lo(in_vgpr(0x010C000Cu)), hi(in_vgpr(0x030C020Cu)) {}
    __device__ __forceinline__ v8h operator()(uint32_t a, uint32_t b) const {
        union { uint32_t w[4]; v8h v; } r;
        r.w[0] = __builtin_amdgcn_perm(a, a, lo);
        r.w[1] = __builtin_amdgcn_perm(a, a, hi);
        r.w[2] = __builtin_amdgcn_perm(b, b, lo);
        r.w[3] = __builtin_amdgcn_perm(b, b, hi);
        return r.v;
    }
};

// Bits 7, 15, 23 and 31: whether the code bytes of a word are Inf or NaN.
__device__ __forceinline__ uint32_t nonfinite_in(uint32_t w) {
    return (w & 0x7C7C7C7Cu) + 0x04040404u;
}
// Code bytes that are Inf or NaN (exponent all ones), 0xFF each.
__device__ __forceinline__ uint32_t nonfinite_bytes(uint32_t w) {
    const uint32_t t = (w & 0x7C7C7C7Cu) ^ 0x7C7C7C7Cu;          // 0 where the exponent is all ones
    const uint32_t z = ~(((t & 0x7F7F7F7Fu) + 0x7F7F7F7Fu) | t) & 0x80808080u;
    return (z >> 7) * 0xFFu;
}

// N rows of codes (keys or queries) x DP columns as rows of bytes in LDS, 16
// bytes of padding per row: the eight lanes that one LDS cycle serves read
// distinct banks.
template <int N, int DP>
struct CodeTile {
    static constexpr int kRow = DP + 16, kBytes = N * kRow;
    template <int NT>
    static constexpr int units() { return N * (DP / 16) / NT; }
    // Codes 32 c + 16 h .. + 15 of a row: a lane's operands of two instructions.
    static __device__ __forceinline__ uint4 frag(const uint8_t* lds, int row, int c, int h) {
        return *reinterpret_cast<const uint4*>(lds + row * kRow + 32 * c + 16 * h);
    }
};

// The same rows transposed as halves: row d holds N values in the k order
// above, i.e. of every 16 the blocks of four 0, 2, 1, 3; 16-byte blocks are
// swizzled by the row, so that the readers (32 rows) meet no bank conflicts and
// the writers (eight octets of columns by two blocks of four) none, or with N =
// 32, whose rows have four blocks only, two-way ones.
template <int N, int DP>
struct HalfTile {
    static constexpr int kRow = 2 * N, kBytes = DP * kRow;
    static __device__ __forceinline__ int swizzle(int d) {
        return N == 32 ? ((d >> 1) ^ (d >> 3)) & 3 : (d ^ (d >> 3)) & 7;
    }
    // units of 4 rows x 8 columns, NT threads
    template <int NT>
    static constexpr int units() { return (N / 4) * (DP / 8) / NT; }
    static __device__ __forceinline__ int unit_row(int u) {       // first of four rows
        constexpr int s = DP == 128 ? 5 : 4;
        return ((u >> (s + 1)) << 4) + (((u >> 3) & 1) << 3) + (((u >> s) & 1) << 2);
    }
    static __device__ __forceinline__ int unit_col(int u) {       // first of eight columns
        return ((u & 7) << 3) + (DP == 128 ? ((u >> 4) & 1) << 6 : 0);
    }
    static __device__ __forceinline__ void store(uint8_t* lds, int u, const uint2* w) {
        const int row = unit_row(u), col = unit_col(u);
        const int block = ((row >> 4) << 1) + ((row >> 2) & 1), eight = ((row >> 3) & 1) * 8;
#pragma unroll
        for (int d = 0; d < 8; ++d) {
            const uint32_t k = d & 3, sel = ((4 + k) << 24) | (0x0Cu << 16) | (k << 8) | 0x0Cu;
            const uint32_t w0 = d < 4 ? w[0].x : w[0].y, w1 = d < 4 ? w[1].x : w[1].y;
            const uint32_t w2 = d < 4 ? w[2].x : w[2].y, w3 = d < 4 ? w[3].x : w[3].y;
            uint2 o;
            o.x = __builtin_amdgcn_perm(w1, w0, sel);
            o.y = __builtin_amdgcn_perm(w3, w2, sel);
            const int swz = block ^ swizzle(col + d);
            *reinterpret_cast<uint2*>(lds + (col + d) * kRow + swz * 16 + eight) = o;
        }
    }
    // Left operand of instruction t (16 rows): column d, lane half h.
    static __device__ __forceinline__ v8h frag(const uint8_t* lds, int d, int t, int h) {
        const int swz = (2 * t + h) ^ swizzle(d);
        return *reinterpret_cast<const v8h*>(lds + d * kRow + swz * 16);
    }
};

// Inf or NaN from its code.
__device__ __forceinline__ float fp8_nonfinite(uint32_t c) {
    return __uint_as_float(((c & 0x80u) << 24) | kF32Inf | ((c & 3u) << 21));
}

// How far, in powers of two, sums of one part of the keys are held above those
// of another: a part's exponents are taken from the score `base` and then from
// the reference `ref` (base 2; -Inf before its first key).
__device__ __forceinline__ float part_above(float base, float ref, float base0, float ref0, float c2) {
    return __builtin_fmaf(base - base0, c2, ref - ref0);
}
// A part's weight against the part that is held highest.  It does not underflow
// to 0: an infinity that a seen value has left in the sums stays one, and finite
// sums times 2^-126 are lost in any other rounding.
__device__ __forceinline__ float part_weight(float base, float ref, float base0, float ref0, float c2) {
    return base == base0 && ref == ref0 ? 1.0f
                                        : fmaxf(exp2f(part_above(base, ref, base0, ref0, c2)), 0x1p-126f);
}

// Entries that are not finite, of the rows noted in `bits` (row 0 of them is
// token t0 of `src`), for the columns that see the row: f(d, r, code).
template <int ND, typename SEES, typename F>
__device__ __forceinline__ void add_noted(uint32_t bits, const uint8_t* src, int64_t ts, int t0, int D,
                                          int h, SEES sees, F f) {
    bits = __builtin_amdgcn_readfirstlane(bits);
    while (__builtin_expect(bits != 0, 0)) {
        int hh = h;
        asm volatile("" : "+v"(hh));                        // nothing of this is hoisted
        const int t = t0 + __builtin_ctz(bits);
        bits &= bits - 1;
        if (!sees(t)) continue;
        const uint8_t* p = src + (int64_t)t * ts;
#pragma unroll
        for (int d = 0; d < ND; ++d)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                asm volatile("" : "+v"(hh));                // four loads at a time
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int col = 32 * d + 8 * q + 4 * hh + r;
                    const uint32_t c = col < D ? p[col] : 0u;
                    if ((c & 0x7Cu) == 0x7Cu) f(d, 4 * q + r, c);
                }
            }
    }
}

// A wave's 32 rows (one per lane pair) x DP columns, out of its result registers
// through `xs` (kRowsOut bytes of LDS of its own), 64 columns at a time: store(r,
// col, x) is called with every lane active for row r's eight entries from
// column col on.  Neighbouring lanes get neighbouring entries, and the code
// for the formats is there once per 64 columns, not once per register quartet:
// short calls are bound by fetching their instructions.
constexpr int kRowsOut = 32 * (64 + 4) * 4;
template <int DP, typename STORE>
__device__ __forceinline__ void rows_out(float* xs, const v16f* acc, float scale, int lane, STORE store) {
    const int l31 = lane & 31, h = lane >> 5;
    auto fence = [&]() {
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
    };
#pragma unroll
    for (int part = 0; part < DP / 64; ++part) {
        fence();
#pragma unroll
        for (int d = 0; d < 2; ++d)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const v16f& v = acc[2 * part + d];
                *reinterpret_cast<float4*>(xs + l31 * 68 + 32 * d + 8 * q + 4 * h) =
                    make_float4(v[4 * q] * scale, v[4 * q + 1] * scale, v[4 * q + 2] * scale,
                                v[4 * q + 3] * scale);
            }
        fence();
#pragma unroll 1
        for (int it = 0; it < 4; ++it) {
            const int r = it * 8 + lane / 8, c = lane % 8 * 8;
            const float4 a = *reinterpret_cast<const float4*>(xs + r * 68 + c);
            const float4 b = *reinterpret_cast<const float4*>(xs + r * 68 + c + 4);
            const float x[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
            store(r, 64 * part + c, x);
        }
    }
}

// A value of lane r's, 64 bits.
__device__ __forceinline__ int64_t of_lane(int64_t x, int r) {
    const uint32_t lo = __shfl((int)(uint32_t)x, r), hi = __shfl((int)(uint32_t)((uint64_t)x >> 32), r);
    return (int64_t)(((uint64_t)hi << 32) | lo);
}

}  // namespace fp8t
