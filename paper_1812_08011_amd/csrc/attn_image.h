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

// An image into LDS by direct loads, 1024 bytes a wave and instruction, shared
// out over WAVES waves; the caller waits (image_barrier).  The instruction is
// written out because the compiler, given its builtin, waits for every such
// load in flight before any later LDS read -- also of the other buffer.  It
// has no result register; m0 holds the wave's LDS address.
typedef __attribute__((address_space(3))) const void* lptr_t;
template <int BYTES, int WAVES>
__device__ __forceinline__ void image_to_lds(const uint8_t* src, const uint8_t* lds, int wave, int lane) {
    constexpr int kPieces = BYTES / 1024;
    const uint32_t to = (uint32_t)(uintptr_t)(lptr_t)lds;
#pragma unroll
    for (int c = 0; c < (kPieces + WAVES - 1) / WAVES; ++c) {
        const int n = c * WAVES + wave;
        if ((c + 1) * WAVES <= kPieces || n < kPieces) {
            const uint8_t* s = src + n * 1024;              // uniform
            asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2"
                         :
                         : "s"(to + (uint32_t)n * 1024u), "v"((uint32_t)lane * 16u), "s"(s)
                         : "memory", "m0");
        }
    }
}
// Waits for this wave's direct loads, then for every wave.
__device__ __forceinline__ void image_barrier() {
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
}

// Workgroup 0 or 1 of the kernels that build images writes an order of tiles, if
// any; rows and keys per tile.
constexpr int kAttnRows = 128, kAttnDkvKeys = 128;

void attn_fwd_image_launch(const AttnArgs& a, bool vec, int DP, hipStream_t stream);
void attn_bwd_image_launch(const AttnArgs& a, bool vec, int DP, hipStream_t stream);

}  // namespace fp8t
