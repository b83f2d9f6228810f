// The backward kernels' host side.
#pragma once

#include "attn.h"

namespace fp8t {

// Workgroups of the kernel that takes the norms, each with a place for two.
constexpr int kAttnNorms = 1024;

// Workspace: delta (rounded up to 16 bytes), then the norms.
inline size_t attn_delta_bytes(int64_t Hq, int64_t Tq) { return ((size_t)Hq * Tq * 4 + 15) / 16 * 16; }
inline size_t attn_bwd_bytes(int64_t Hq, int64_t Tq) {
    return attn_delta_bytes(Hq, Tq) + 2 * kAttnNorms * sizeof(float);
}
void attn_bwd_launch(AttnArgs a, int grad_format, bool vec, hipStream_t stream);

}  // namespace fp8t
