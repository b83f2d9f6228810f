// The backward kernels' plan.
#pragma once

#include "attn.h"

namespace fp8t {

struct AttnBwdPlan {
    int DP, splits;                    // padded D; workgroups that share a key tile's queries
    bool fits;                         // no grid is too large
    int64_t key_tiles, query_tiles;    // of the images
    // byte offsets into the workspace, and its size
    size_t delta, key_image, query_image, order, key_order, parts, bytes;
};

AttnBwdPlan attn_bwd_plan(int64_t S, int64_t Tq, int64_t Tk, int64_t max_q, int64_t max_k, int64_t Hq,
                          int64_t Hkv, int64_t D);
void attn_bwd_launch(AttnArgs a, const AttnBwdPlan& p, int grad_format, bool vec, void* workspace,
                     hipStream_t stream);

}  // namespace fp8t
