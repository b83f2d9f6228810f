// The forward kernels' plan and what they share with their host side.
#pragma once

#include "attn.h"

namespace fp8t {

struct AttnFwdPlan {
    int DP, BM, splits, per;           // padded D, rows per workgroup, key ranges and tiles in each
    int64_t slots;                     // row tiles of all sequences, empty ones included
    bool image, order;                 // keys and values through images; row tiles in an order
    size_t image_bytes, bytes;         // workspace: images and order first, then partial results
};

struct AttnSplit {                     // partial results: rows x DP sums, (reference, sum)
    float* o;
    float2* ml;
    int n, per, BM;
};

AttnFwdPlan attn_fwd_plan(int64_t S, int64_t Tq, int64_t Tk, int64_t max_q, int64_t max_k,
                          int64_t Hq, int64_t Hkv, int64_t D);
void attn_fwd_launch(AttnArgs a, const AttnFwdPlan& p, bool vec, void* workspace,
                     hipStream_t stream);

// One row's results from the two lanes that hold it: value(d, r) is entry 32 d
// + 8 (r / 4) + 4 h + r % 4 of the unnormalized sum, l the sum of p, ref their
// common reference (base 2).
template <int DP, typename F>
__device__ __forceinline__ void attn_write_row(const AttnArgs& a, int64_t t, int hq, int lim, float ref,
                                               float l, int h, F value) {
    const float inv = 1.0f / l;
    uint16_t* o = a.o ? a.o + t * a.o_ts + (int64_t)hq * a.o_hs : nullptr;
    uint8_t* o8 = a.o8 ? a.o8 + t * a.o8_ts + (int64_t)hq * a.o8_hs : nullptr;
#pragma unroll
    for (int d = 0; d < DP / 32; ++d)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int col = 32 * d + 8 * q + 4 * h;
            float x[4];
#pragma unroll
            for (int r = 0; r < 4; ++r) x[r] = lim > 0 ? value(d, 4 * q + r) * inv : 0.0f;
            if (col + 4 <= a.D && o && aligned_to(o + col, 8)) {
                uint2 w;
                w.x = (uint32_t)f32_to_fp16_rn(x[0]) | ((uint32_t)f32_to_fp16_rn(x[1]) << 16);
                w.y = (uint32_t)f32_to_fp16_rn(x[2]) | ((uint32_t)f32_to_fp16_rn(x[3]) << 16);
                *reinterpret_cast<uint2*>(o + col) = w;
            } else if (o) {
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    if (col + r < a.D) o[col + r] = f32_to_fp16_rn(x[r]);
            }
            const float sc = a.o8_scale;
            if (col + 4 <= a.D && o8 && aligned_to(o8 + col, 4)) {
                const uint32_t lo = f32x2_to_fp8x2<false>(x[0] * sc, x[1] * sc, 0u);
                *reinterpret_cast<uint32_t*>(o8 + col) = f32x2_to_fp8x2<true>(x[2] * sc, x[3] * sc, lo);
            } else if (o8) {
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    if (col + r < a.D) o8[col + r] = (uint8_t)f32_to_fp8(x[r] * sc);
            }
        }
    if (a.lse && h == 0)
        a.lse[(int64_t)hq * a.Tq + t] = lim > 0 ? kAttnLn2 * (ref + log2f(l)) : -INFINITY;
}

}  // namespace fp8t
