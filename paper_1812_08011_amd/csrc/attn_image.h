// Images: tiles of keys or queries laid out in memory as the matrix-core
// kernels keep them in LDS (codes with their row padding, transposed halves
// with their swizzle), so that a kernel brings a tile in by direct loads into
// LDS: no registers, no permutations and no bounds checks in its loop, once
// per call instead of once per workgroup that reads the tile.
//
// Tiles are cut from the packed array (tile t holds tokens N t .. N t + N - 1,
// whatever sequences they belong to; tokens past the end are zero), so there
// are T / N of them for any set of lengths; the kernels mask what is not theirs.
//
// Transposed halves hold 0 where a value is not finite (0 x NaN must not reach
// masked places); the rows that had such values are noted, one bit a row, in
// the padding of code row 0 (8 in a query image), and the kernels add them to
// what sees them.
#pragma once

#include "attn_mfma.h"

namespace fp8t {

// Keys per tile of the forward kernels: 256 threads stage a tile's values as
// one unit of 4 x 8 each.
constexpr int attn_keys(int DP) { return DP == 64 ? 128 : 64; }

template <int DP>
struct FwdImage {                      // keys as codes, values transposed
    static constexpr int N = attn_keys(DP);
    using CT = CodeTile<N, DP>;
    using HT = HalfTile<N, DP>;
    static constexpr int kV = CT::kBytes, kBytes = kV + HT::kBytes, kNoted = DP;
};
template <int DP>
struct KeyImage {                      // keys and values as codes, keys transposed
    static constexpr int N = 64;
    using CT = CodeTile<N, DP>;
    using HT = HalfTile<N, DP>;
    static constexpr int kV = CT::kBytes, kT = 2 * CT::kBytes, kBytes = kT + HT::kBytes, kNoted = DP;
};
template <int DP>
struct QueryImage {                    // queries and errors as codes, both transposed
    static constexpr int N = 32;
    using CT = CodeTile<N, DP>;
    using HT = HalfTile<N, DP>;
    static constexpr int kE = CT::kBytes, kQT = 2 * CT::kBytes, kET = kQT + HT::kBytes,
                         kBytes = kET + HT::kBytes;
    // In the padding of code rows 0 .. 7: the log-sum-exps (base 2, less the
    // power p is held times) and the negated deltas of rows 4 n .. 4 n + 3; in
    // row 8's of the queries: the noted queries and errors.
    static __device__ __forceinline__ int lse(int n) { return n * CT::kRow + DP; }
    static __device__ __forceinline__ int delta(int n) { return kE + n * CT::kRow + DP; }
    static constexpr int kNoted = 8 * CT::kRow + DP;
};
static_assert(FwdImage<64>::kBytes % 1024 == 0 && FwdImage<128>::kBytes % 1024 == 0 &&
                  KeyImage<64>::kBytes % 1024 == 0 && KeyImage<128>::kBytes % 1024 == 0 &&
                  QueryImage<64>::kBytes % 1024 == 0 && QueryImage<128>::kBytes % 1024 == 0,
              "images are read a wave's 1024 bytes at a time");

constexpr int kAttnPUp = 15;           // the backward kernels hold p times 2^15

inline int64_t image_tiles(int64_t T, int N) { return (T + N - 1) / N; }

// An image into LDS, shared out over WAVES waves; the caller waits.
typedef __attribute__((address_space(1))) const void* gptr_t;
typedef __attribute__((address_space(3))) void* lptr_t;
template <int BYTES, int WAVES>
__device__ __forceinline__ void image_to_lds(const uint8_t* src, uint8_t* lds, int wave, int lane) {
    const uint8_t* s = src + lane * 16;
#pragma unroll
    for (int c = 0; c < (BYTES / 1024 + WAVES - 1) / WAVES; ++c) {
        const int n = c * WAVES + wave;
        if (BYTES / 1024 % WAVES == 0 || n < BYTES / 1024)
            __builtin_amdgcn_global_load_lds((gptr_t)(s + n * 1024), (lptr_t)(lds + n * 1024), 16, 0, 0);
    }
}
// Waits for this wave's direct loads (the compiler does not see their LDS
// writes), then for every wave.
__device__ __forceinline__ void image_barrier() {
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
}

void attn_fwd_image_launch(const AttnArgs& a, bool vec, int DP, hipStream_t stream);
void attn_bwd_image_launch(const AttnArgs& a, bool vec, int DP, hipStream_t stream);

}  // namespace fp8t
