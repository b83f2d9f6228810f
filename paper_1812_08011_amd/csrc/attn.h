// Arguments of the attention kernels and what they share.
#pragma once

#include "lm_formats.h"

namespace fp8t {

struct AttnRows {            // T x H x D codes with strides
    const uint8_t* p;
    int64_t ts, hs;
};

struct AttnArgs {
    AttnRows q, k, v, e;     // e: the error of o (backward)
    const int64_t* cu_q;
    const int64_t* cu_k;
    int S, Hq, Hkv, D, causal;
    int G;                   // Hq / Hkv, and floor(2^64 / G) + 1 (0 for G = 1)
    uint64_t g_magic;
    int64_t Tq, Tk;
    float c2;                // sm_scale log2(e): exponents are kept in base 2
    float sm_scale;
    // forward results; o is read by the backward pass
    uint16_t* o;
    int64_t o_ts, o_hs;
    uint8_t* o8;
    int64_t o8_ts, o8_hs;
    float o8_scale;
    float* lse;
    // backward
    void *dq, *dk, *dv;
    int64_t dq_ts, dq_hs, dk_ts, dk_hs, dv_ts, dv_hs;
    float grad_scale;
    float* delta;            // Hq x Tq
    // images (attn_image.h), [head][tile]
    uint8_t* key_image;
    uint8_t* query_image;
    int64_t key_tiles, query_tiles;
    // tiles of rows and of keys, the longest first (attn_image.hip), -1 past the
    // last; null: in the order of their slots
    int* row_order;
    int* key_order;
    float* parts;            // partial dk, dv: [part][token][head][2][padded D]
    int splits;
};

constexpr float kAttnLog2e = 1.44269504088896340736f;
constexpr float kAttnLn2 = 0.69314718055994530942f;

// One sequence's tokens, clamped into the arrays whatever the offsets hold.
struct Seq {
    int64_t q0, k0;
    int nq, nk;
};
__device__ __forceinline__ int64_t clamp_to(int64_t x, int64_t n) {
    return x < 0 ? 0 : x > n ? n : x;
}
__device__ __forceinline__ Seq load_seq(const AttnArgs& a, int s) {
    Seq r;
    r.q0 = clamp_to(a.cu_q[s], a.Tq);
    r.k0 = clamp_to(a.cu_k[s], a.Tk);
    const int64_t q1 = clamp_to(a.cu_q[s + 1], a.Tq), k1 = clamp_to(a.cu_k[s + 1], a.Tk);
    r.nq = q1 > r.q0 ? (int)(q1 - r.q0) : 0;
    r.nk = k1 > r.k0 ? (int)(k1 - r.k0) : 0;
    return r;
}

// n / G, exact while n G < 2^64.
__device__ __forceinline__ int div_g(const AttnArgs& a, int n) {
    return a.g_magic ? (int)__umul64hi((uint64_t)(uint32_t)n, a.g_magic) : n;
}

// Work of sequences of unknown lengths laid out without a scan: with
// `len(s) = (cu[s+1] - cu[s]) * mult` rows in tiles of `tile`, sequence s owns
// the slots from floor(cu[s] mult / tile) + s on -- at least ceil(len / tile)
// of them, since floor(x + y) + 1 >= floor(x) + ceil(y).  Slots beyond a
// sequence's own tiles are empty.  A grid of floor(T mult / tile) + S slots
// holds every sequence; the owner is found by bisection.
__device__ __forceinline__ int slot_owner(const int64_t* cu, int S, int64_t T, int64_t mult,
                                          int64_t tile, int64_t slot, int& local) {
    int lo = 0, hi = S - 1;                 // the last s with start(s) <= slot
    while (lo < hi) {
        const int mid = (lo + hi + 1) / 2;
        if (clamp_to(cu[mid], T) * mult / tile + mid <= slot) lo = mid;
        else hi = mid - 1;
    }
    const int64_t l = slot - (clamp_to(cu[lo], T) * mult / tile + lo);
    local = l < 0 ? INT32_MAX : (int)l;     // before the first sequence: empty
    return lo;
}
// The tile that a workgroup takes: the slot, and its sequence and place there.
__device__ __forceinline__ int ordered_slot(const int* order, int n) { return order ? order[n] : n; }
// Workgroups of 256 threads along a grid's first dimension.
constexpr int64_t kAttnGrid = (1 << 24) - 1;
inline int64_t slots(int64_t S, int64_t T, int64_t mult, int64_t tile) {
    return S > 0 ? T * mult / tile + S : 0;
}
// The size hints as the plans take them: at most what a call may hold, so that
// neither a plan's products nor a kernel's tile numbers (32 bits) overflow
// whatever a caller expects.
inline int64_t hint(int64_t n, int64_t mult) {
    const int64_t most = kMaxGemmDim / (mult > 0 ? mult : 1);
    return n < most ? n : most;
}

}  // namespace fp8t
