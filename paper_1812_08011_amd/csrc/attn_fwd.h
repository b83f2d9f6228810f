// The forward kernels' plan and what they share with their host side.
#pragma once

#include "attn.h"

namespace fp8t {

struct AttnFwdPlan {
    int DP, BM, splits, per;           // padded D, rows per workgroup, key ranges and tiles in each
    int64_t slots;                     // row tiles of all sequences, empty ones included
    bool fits;                         // no grid is too large
    bool image, order;                 // keys and values through images; row tiles in an order
    size_t image_bytes, bytes;         // workspace: images and order first, then partial results
};

struct AttnSplit {                     // partial results: rows x DP sums, (base, reference, sum)
    float* o;
    float4* ml;
    int n, per;
};

AttnFwdPlan attn_fwd_plan(int64_t S, int64_t Tq, int64_t Tk, int64_t max_q, int64_t max_k,
                          int64_t Hq, int64_t Hkv, int64_t D);
void attn_fwd_launch(AttnArgs a, const AttnFwdPlan& p, bool vec, void* workspace,
                     hipStream_t stream);

}  // namespace fp8t
