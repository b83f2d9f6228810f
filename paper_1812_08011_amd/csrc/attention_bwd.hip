// Attention backward on the matrix cores, in three kernels:
//   prepare: delta = <e, o> of every row, and the largest row norms of e and v;
//   dq:      a wave owns rows (queries) and streams the keys;
//   dk, dv:  a wave owns keys and streams the queries of every head that
//            shares them.
// Scores are computed twice (7 products instead of 5), which needs no atomics
// and no partial sums: the same bits on every run.
#include "attn_bwd.h"
#include "attn_mfma.h"

namespace fp8t {
namespace {

constexpr int kThreads = 256;
constexpr int kN = 64;                // rows per streamed tile
constexpr int kPUp = 15;              // p enters its product times 2^15

// Four entries of a gradient from column col on.
template <int FG>
__device__ __forceinline__ void write4(void* base, int64_t at, int col, int D, const float* x) {
    fmt_t<FG>* p = static_cast<fmt_t<FG>*>(base) + at + col;
    if (col + 4 <= D && aligned_to(p, 4 * sizeof(*p))) {
        if constexpr (FG == FP8T_FMT_FP16) {
            uint2 w;
            w.x = (uint32_t)f32_to_fp16_rn(x[0]) | ((uint32_t)f32_to_fp16_rn(x[1]) << 16);
            w.y = (uint32_t)f32_to_fp16_rn(x[2]) | ((uint32_t)f32_to_fp16_rn(x[3]) << 16);
            *reinterpret_cast<uint2*>(p) = w;
        } else {
            const uint32_t lo = f32x2_to_fp8x2<false>(x[0], x[1], 0u);
            *reinterpret_cast<uint32_t*>(p) = f32x2_to_fp8x2<true>(x[2], x[3], lo);
        }
    } else {
#pragma unroll
        for (int r = 0; r < 4; ++r)
            if (col + r < D) p[r] = fmt_code<FG>(x[r]);
    }
}

// ---- delta and the norms ------------------------------------------------------------

// 16 lanes per row, 8 entries each.  Norms: the largest squared norm among the
// finite rows of e, then of v, per workgroup.
template <bool VEC>
__global__ __launch_bounds__(kThreads) void attn_prepare_kernel(AttnArgs a) {
    __shared__ float red[kThreads / 64];
    const int lane = threadIdx.x & 15, d0 = lane * 8;
    const int64_t rows_e = a.Tq * a.Hq, rows_v = a.Tk * a.Hkv;
    const int64_t step = (int64_t)gridDim.x * (kThreads / 16);
    const int64_t first = (int64_t)blockIdx.x * (kThreads / 16) + threadIdx.x / 16;
    float top[2] = {0.0f, 0.0f};
    for (int64_t r = first; r < rows_e; r += step) {
        const int64_t t = r / a.Hq, hq = r % a.Hq;
        const uint2 w = load_codes8<VEC>(a.e.p + t * a.e.ts + hq * a.e.hs, d0, a.D, true);
        const uint16_t* o = a.o + t * a.o_ts + hq * a.o_hs;
        uint32_t oc[4] = {0, 0, 0, 0};
        if (VEC) {
            if (d0 < a.D) {
                const uint4 q = *reinterpret_cast<const uint4*>(o + d0);
                oc[0] = q.x;
                oc[1] = q.y;
                oc[2] = q.z;
                oc[3] = q.w;
            }
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (d0 + i < a.D) oc[i / 2] |= (uint32_t)o[d0 + i] << (16 * (i % 2));
        }
        float s = 0.0f, n = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float e = fp8_to_f32<0>(((i < 4 ? w.x : w.y) >> (8 * (i % 4))) & 0xFFu);
            s = __builtin_fmaf(e, fp16_to_f32((oc[i / 2] >> (16 * (i % 2))) & 0xFFFFu), s);
            n = __builtin_fmaf(e, e, n);
        }
#pragma unroll
        for (int d = 8; d; d >>= 1) {
            s += __shfl_xor(s, d);
            n += __shfl_xor(n, d);
        }
        if (lane == 0) a.delta[hq * a.Tq + t] = s;
        if (n < INFINITY) top[0] = fmaxf(top[0], n);
    }
    for (int64_t r = first; r < rows_v; r += step) {
        const int64_t t = r / a.Hkv, hk = r % a.Hkv;
        const uint2 w = load_codes8<VEC>(a.v.p + t * a.v.ts + hk * a.v.hs, d0, a.D, true);
        float n = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float v = fp8_to_f32<0>(((i < 4 ? w.x : w.y) >> (8 * (i % 4))) & 0xFFu);
            n = __builtin_fmaf(v, v, n);
        }
#pragma unroll
        for (int d = 8; d; d >>= 1) n += __shfl_xor(n, d);
        if (n < INFINITY) top[1] = fmaxf(top[1], n);
    }
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        float x = top[k];
        for (int d = 32; d >= 16; d >>= 1) x = fmaxf(x, __shfl_xor(x, d));
        __syncthreads();
        if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = x;
        __syncthreads();
        if (threadIdx.x == 0)
            a.norms[k * kAttnNorms + blockIdx.x] = fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]));
    }
}

// The power of two that dS = p (<e, v> - delta) is held times.  Both terms are
// at most |e| |v| (delta is a mean of such products), so with the largest norms
// the scaled dS stays below 2^15, and a dS down to 2^-29 of that bound keeps
// all 11 bits of a half.  Every thread of the workgroup calls this.
__device__ __forceinline__ float ds_scale(const AttnArgs& a, float* red) {
    float x[2];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        x[k] = 0.0f;
        for (int i = threadIdx.x; i < a.norm_count; i += kThreads)
            x[k] = fmaxf(x[k], a.norms[k * kAttnNorms + i]);
        for (int d = 32; d; d >>= 1) x[k] = fmaxf(x[k], __shfl_xor(x[k], d));
        if ((threadIdx.x & 63) == 0) red[k * 4 + (threadIdx.x >> 6)] = x[k];
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 2; ++k)
        x[k] = fmaxf(fmaxf(red[4 * k], red[4 * k + 1]), fmaxf(red[4 * k + 2], red[4 * k + 3]));
    const float bound = __builtin_sqrtf(x[0]) * __builtin_sqrtf(x[1]);
    if (!(bound > 0.0f)) return 1.0f;
    int e;
    (void)__builtin_frexpf(bound, &e);                      // bound < 2^e
    return __builtin_ldexpf(1.0f, 13 - e);
}

// ---- staging ----------------------------------------------------------------------------

template <int DP>
using CT = CodeTile<kN, DP>;
template <int DP>
using HT = HalfTile<kN, DP>;

// Four rows x eight columns of a tile that starts at row t0, rows below n.
template <int DP, bool VEC>
__device__ __forceinline__ void load_unit(uint2* w, const uint8_t* p, int64_t ts, int t0, int n, int D,
                                          int u) {
    const int row = t0 + HT<DP>::unit_row(u), col = HT<DP>::unit_col(u);
#pragma unroll
    for (int r = 0; r < 4; ++r)
        w[r] = load_codes8<VEC>(p + (int64_t)(row + r) * ts, col, D, row + r < n);
}
// A unit as codes and transposed as halves; on partial tiles values that are
// not finite leave the halves (0 x NaN must not reach a masked place) and
// their rows are noted.
template <int DP>
__device__ __forceinline__ void store_unit(uint2* w, uint8_t* codes, uint8_t* halves, int u,
                                           bool partial, uint32_t* bad) {
    const int row = HT<DP>::unit_row(u), col = HT<DP>::unit_col(u);
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        *reinterpret_cast<uint2*>(codes + (row + r) * CT<DP>::kRow + col) = w[r];
        if (partial) {
            const uint32_t nx = nonfinite_bytes(w[r].x), ny = nonfinite_bytes(w[r].y);
            if (nx | ny) {
                atomicOr(bad + (row + r) / 32, 1u << ((row + r) % 32));
                w[r].x &= ~nx;
                w[r].y &= ~ny;
            }
        }
    }
    HT<DP>::store(halves, u, w);
}

// ---- dq ------------------------------------------------------------------------------------

// 128 rows (query, head of the group), 32 per wave; keys and values in LDS,
// double-buffered.  dQ^T = K^T dS^T with dS^T's registers as the operand.
template <int DP, bool VEC, int FG>
__global__ __launch_bounds__(kThreads, 2) void attn_dq_kernel(AttnArgs a) {
    constexpr int BM = 128, NC = DP / 32, ND = DP / 32;
    constexpr int U = (kN / 4) * (DP / 8), KU = (U + kThreads - 1) / kThreads;
    constexpr int VU = kN * (DP / 16) / kThreads;
    constexpr int kBuf = 2 * CT<DP>::kBytes + HT<DP>::kBytes;
    __shared__ __attribute__((aligned(16))) uint8_t lds[2 * kBuf];
    __shared__ uint32_t bad[3][2];
    __shared__ float red[8];
    const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, l31 = lane & 31, h = lane >> 5;
    const int hk = blockIdx.x % a.Hkv, G = a.Hq / a.Hkv;
    int tile;
    const int s = slot_owner(a.cu_q, a.S, a.Tq, G, BM, blockIdx.x / a.Hkv, tile);
    const Seq sq = load_seq(a, s);
    const int64_t nrows = (int64_t)sq.nq * G;
    const int ntiles = (int)((nrows + BM - 1) / BM);
    if (tile >= ntiles) return;
    tile = ntiles - 1 - tile;                               // the longest first
    const int64_t row0 = (int64_t)tile * BM, row = row0 + 32 * wave + l31;
    const bool live = row < nrows;
    const int i = live ? (int)(row / G) : 0, g = live ? (int)(row % G) : 0;
    const int off = sq.nk - sq.nq;
    auto limit = [&](int64_t r) {
        const int64_t n = a.causal ? r / G + 1 + off : sq.nk;
        return (int)(n < 0 ? 0 : n);
    };
    const int lim = live ? limit(row) : 0;
    const int64_t last = row0 + BM < nrows ? row0 + BM - 1 : nrows - 1;
    const int lim_lo = limit(row0), lim_hi = limit(last);
    const int64_t wl = row0 + 32 * wave + 31 < nrows ? row0 + 32 * wave + 31 : nrows - 1;
    const int wave_hi = row0 + 32 * wave < nrows ? limit(wl) : 0;
    const int t1 = (lim_hi + kN - 1) / kN;

    const int64_t tq = sq.q0 + i;
    const int hq = hk * G + g;
    const uint8_t* qp = a.q.p + tq * a.q.ts + (int64_t)hq * a.q.hs;
    const uint8_t* ep = a.e.p + tq * a.e.ts + (int64_t)hq * a.e.hs;
    const uint8_t* kp = a.k.p + sq.k0 * a.k.ts + (int64_t)hk * a.k.hs;
    const uint8_t* vp = a.v.p + sq.k0 * a.v.ts + (int64_t)hk * a.v.hs;
    const Widen widen;
    const float c2 = __uint_as_float(in_vgpr(__float_as_uint(a.c2)));
    v8h qf[NC][2], ef[NC][2];
#pragma unroll
    for (int c = 0; c < NC; ++c) {
        uint4 w = load_codes16<VEC>(qp, 32 * c + 16 * h, a.D, live);
        qf[c][0] = widen(w.x, w.y);
        qf[c][1] = widen(w.z, w.w);
        w = load_codes16<VEC>(ep, 32 * c + 16 * h, a.D, live);
        ef[c][0] = widen(w.x, w.y);
        ef[c][1] = widen(w.z, w.w);
    }
    const float sigma = ds_scale(a, red);
    float lse2 = INFINITY, delta = 0.0f;                    // a row that sees nothing: p = 0
    if (lim > 0) {
        lse2 = a.lse[(int64_t)hq * a.Tq + tq] * kAttnLog2e;
        delta = a.delta[(int64_t)hq * a.Tq + tq] * sigma;
    }
    const float sg = __uint_as_float(in_vgpr(__float_as_uint(sigma)));

    v16f o[ND];
#pragma unroll
    for (int d = 0; d < ND; ++d)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[d][r] = 0.0f;
    const v16f zero = {0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0};

    uint2 ku[KU][4];
    uint4 vu[VU];
    auto load = [&](int t) {
#pragma unroll
        for (int u = 0; u < KU; ++u)
            if (U % kThreads == 0 || tid + u * kThreads < U)
                load_unit<DP, VEC>(ku[u], kp, a.k.ts, t * kN, sq.nk, a.D, tid + u * kThreads);
#pragma unroll
        for (int u = 0; u < VU; ++u) {
            const int id = tid + u * kThreads, r = t * kN + id / (DP / 16), col = id % (DP / 16) * 16;
            vu[u] = load_codes16<VEC>(vp + (int64_t)r * a.v.ts, col, a.D, r < sq.nk);
        }
    };
    auto is_partial = [&](int t) { return (t + 1) * kN > lim_lo || (t + 1) * kN > sq.nk; };
    auto store = [&](int t, uint8_t* buf, uint32_t* badw) {
        const bool partial = is_partial(t);
#pragma unroll
        for (int u = 0; u < KU; ++u)
            if (U % kThreads == 0 || tid + u * kThreads < U)
                store_unit<DP>(ku[u], buf, buf + 2 * CT<DP>::kBytes, tid + u * kThreads, partial, badw);
#pragma unroll
        for (int u = 0; u < VU; ++u) {
            const int id = tid + u * kThreads, r = id / (DP / 16), col = id % (DP / 16) * 16;
            *reinterpret_cast<uint4*>(buf + CT<DP>::kBytes + r * CT<DP>::kRow + col) = vu[u];
        }
    };

    if (tid < 6) bad[tid / 2][tid % 2] = 0u;
    __syncthreads();
    if (t1 > 0) {
        load(0);
        store(0, lds, bad[0]);
    }
    __syncthreads();
    for (int t = 0; t < t1; ++t) {
        const int b = t & 1, q = t % 3, j0 = t * kN;
        if (t + 1 < t1) load(t + 1);
        if (j0 < wave_hi) {
            const uint8_t* kl = lds + b * kBuf;
            const uint8_t* vl = kl + CT<DP>::kBytes;
            const uint8_t* kt_ = vl + CT<DP>::kBytes;
            const bool partial = is_partial(t);
#pragma unroll
            for (int kt = 0; kt < kN / 32; ++kt) {
                v16f st = zero, dp = zero;
#pragma unroll
                for (int c = 0; c < NC; ++c) {
                    uint4 w = CT<DP>::frag(kl, 32 * kt + l31, c, h);
                    st = mfma_half(widen(w.x, w.y), qf[c][0], st);
                    st = mfma_half(widen(w.z, w.w), qf[c][1], st);
                    w = CT<DP>::frag(vl, 32 * kt + l31, c, h);
                    dp = mfma_half(widen(w.x, w.y), ef[c][0], dp);
                    dp = mfma_half(widen(w.z, w.w), ef[c][1], dp);
                }
                float ds[16];
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(st[r], c2, -lse2));
                    ds[r] = p * __builtin_fmaf(dp[r], sg, -delta);
                }
                if (partial) {
                    const int rel = lim - j0 - 32 * kt - 4 * h;
#pragma unroll
                    for (int r = 0; r < 16; ++r)
                        if (8 * (r / 4) + r % 4 >= rel) ds[r] = 0.0f;
                }
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    const v8h f = to_half8(ds + 8 * u);
#pragma unroll
                    for (int d = 0; d < ND; ++d)
                        o[d] = mfma_half(HT<DP>::frag(kt_, 32 * d + l31, 2 * kt + u, h), f, o[d]);
                }
                if (partial) {
                    // keys that are not finite, for the rows that see them
                    uint32_t bw = bad[q][kt];
                    while (bw) {
                        const int key = j0 + 32 * kt + __builtin_ctz(bw);
                        bw &= bw - 1;
                        const uint8_t* kr = kp + (int64_t)key * a.k.ts;
#pragma unroll
                        for (int d = 0; d < ND; ++d)
#pragma unroll
                            for (int r = 0; r < 16; ++r) {
                                const int col = 32 * d + 8 * (r / 4) + 4 * h + r % 4;
                                const uint32_t c = key < lim && col < a.D ? kr[col] : 0u;
                                if ((c & 0x7Cu) == 0x7Cu) o[d][r] = __uint_as_float(kF32NaN);
                            }
                    }
                }
            }
        }
        if (tid < 2) bad[(q + 2) % 3][tid] = 0u;
        if (t + 1 < t1) store(t + 1, lds + (b ^ 1) * kBuf, bad[(q + 1) % 3]);
        __syncthreads();
    }
    if (!live) return;
    const float f = a.sm_scale / sigma * a.grad_scale;
    const int64_t at = tq * a.dq_ts + (int64_t)hq * a.dq_hs;
#pragma unroll
    for (int d = 0; d < ND; ++d)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            float x[4];
#pragma unroll
            for (int r = 0; r < 4; ++r) x[r] = o[d][4 * q + r] * f;
            write4<FG>(a.dq, at, 32 * d + 8 * q + 4 * h, a.D, x);
        }
}

// ---- dk and dv --------------------------------------------------------------------------------

// 32 KT keys per wave; the queries and errors of the group's heads stream
// through LDS.  dV^T = E^T P and dK^T = Q^T dS with P's and dS's registers as
// the operands.
template <int DP, int KT, bool VEC, int FG>
__global__ __launch_bounds__(kThreads, KT == 1 ? 2 : 1) void attn_dkv_kernel(AttnArgs a) {
    constexpr int BN = 128 * KT, NC = DP / 32, ND = DP / 32;
    constexpr int U = (kN / 4) * (DP / 8), NU = 2 * U / kThreads;
    constexpr int kBuf = 2 * CT<DP>::kBytes + 2 * HT<DP>::kBytes;
    __shared__ __attribute__((aligned(16))) uint8_t lds[2 * kBuf];
    __shared__ __attribute__((aligned(16))) float rows[2][2][kN];   // lse and delta of a tile
    __shared__ uint32_t bad[3][2][2];
    __shared__ float red[8];
    const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, l31 = lane & 31, h = lane >> 5;
    const int hk = blockIdx.x % a.Hkv, G = a.Hq / a.Hkv;
    int tile;
    const int s = slot_owner(a.cu_k, a.S, a.Tk, 1, BN, blockIdx.x / a.Hkv, tile);
    const Seq sq = load_seq(a, s);
    if ((int64_t)tile * BN >= sq.nk) return;
    const int off = sq.nk - sq.nq, key0 = tile * BN;
    const int wave0 = key0 + 32 * KT * wave;
    const int key_hi = key0 + BN < sq.nk ? key0 + BN - 1 : sq.nk - 1;
    // query i sees key j iff i >= j - off
    const int first = a.causal && key0 - off > 0 ? key0 - off : 0;
    const int tq0 = first / kN, ntq = (sq.nq + kN - 1) / kN - tq0, steps = ntq > 0 ? ntq * G : 0;
    const int wave_lo = a.causal ? wave0 - off : 0;         // the wave's first key's first query
    const int wg_all = a.causal ? key_hi - off : 0;         // from here on every key is seen

    const uint8_t* kp = a.k.p + sq.k0 * a.k.ts + (int64_t)hk * a.k.hs;
    const uint8_t* vp = a.v.p + sq.k0 * a.v.ts + (int64_t)hk * a.v.hs;
    const Widen widen;
    const float c2 = __uint_as_float(in_vgpr(__float_as_uint(a.c2)));
    v8h kf[KT][NC][2], vf[KT][NC][2];
#pragma unroll
    for (int kt = 0; kt < KT; ++kt) {
        const int j = wave0 + 32 * kt + l31;
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            uint4 w = load_codes16<VEC>(kp + (int64_t)j * a.k.ts, 32 * c + 16 * h, a.D, j < sq.nk);
            kf[kt][c][0] = widen(w.x, w.y);
            kf[kt][c][1] = widen(w.z, w.w);
            w = load_codes16<VEC>(vp + (int64_t)j * a.v.ts, 32 * c + 16 * h, a.D, j < sq.nk);
            vf[kt][c][0] = widen(w.x, w.y);
            vf[kt][c][1] = widen(w.z, w.w);
        }
    }
    const float sigma = ds_scale(a, red);
    // p is held times 2^15, dS times sigma: p (dP - delta) sigma 2^-15
    const float sg = __uint_as_float(in_vgpr(__float_as_uint(__builtin_ldexpf(sigma, -kPUp))));

    v16f dk[KT][ND], dv[KT][ND];
#pragma unroll
    for (int kt = 0; kt < KT; ++kt)
#pragma unroll
        for (int d = 0; d < ND; ++d)
#pragma unroll
            for (int r = 0; r < 16; ++r) dk[kt][d][r] = dv[kt][d][r] = 0.0f;
    const v16f zero = {0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0};

    uint2 st_[NU][4];
    float rowv = 0.0f;
    // step n: head n / ntq of the group, query tile tq0 + n % ntq
    auto head = [&](int n) { return hk * G + n / ntq; };
    auto tile_of = [&](int n) { return tq0 + n % ntq; };
    auto load = [&](int n) {
        const int hq = head(n), t0 = tile_of(n) * kN;
#pragma unroll
        for (int k = 0; k < NU; ++k) {
            const int u = (tid + k * kThreads) % U;
            const bool is_e = tid + k * kThreads >= U;      // uniform in a wave
            const uint8_t* p = is_e ? a.e.p + sq.q0 * a.e.ts + (int64_t)hq * a.e.hs
                                    : a.q.p + sq.q0 * a.q.ts + (int64_t)hq * a.q.hs;
            load_unit<DP, VEC>(st_[k], p, is_e ? a.e.ts : a.q.ts, t0, sq.nq, a.D, u);
        }
        if (tid < 2 * kN) {
            // rows that see no key, or past the last one: p = 0
            const int i = t0 + tid % kN;
            const bool ok = i < sq.nq && (!a.causal || i + off >= 0);
            const float* src = (tid < kN ? a.lse : a.delta) + (int64_t)hq * a.Tq + sq.q0 + i;
            rowv = ok ? *src : tid < kN ? INFINITY : 0.0f;
        }
    };
    auto is_partial = [&](int n) { return tile_of(n) * kN < wg_all; };
    auto store = [&](int n, int b, uint32_t(*badw)[2]) {
        uint8_t* buf = lds + b * kBuf;
        const bool partial = is_partial(n);
#pragma unroll
        for (int k = 0; k < NU; ++k) {
            const int u = (tid + k * kThreads) % U, is_e = tid + k * kThreads >= U;
            store_unit<DP>(st_[k], buf + is_e * CT<DP>::kBytes,
                           buf + 2 * CT<DP>::kBytes + is_e * HT<DP>::kBytes, u, partial, badw[is_e]);
        }
        if (tid < kN) rows[b][0][tid] = rowv * kAttnLog2e - (float)kPUp;
        else if (tid < 2 * kN) rows[b][1][tid - kN] = rowv * sg;
    };

    if (tid < 12) bad[tid / 4][tid / 2 % 2][tid % 2] = 0u;
    __syncthreads();
    if (steps > 0) {
        load(0);
        store(0, 0, bad[0]);
    }
    __syncthreads();
    for (int n = 0; n < steps; ++n) {
        const int b = n & 1, q = n % 3, i0 = tile_of(n) * kN;
        if (n + 1 < steps) load(n + 1);
        const uint8_t* ql = lds + b * kBuf;
        const uint8_t* el = ql + CT<DP>::kBytes;
        const uint8_t* qt = el + CT<DP>::kBytes;
        const uint8_t* et = qt + HT<DP>::kBytes;
        const bool partial = is_partial(n);
#pragma unroll
        for (int u = 0; u < kN / 32; ++u) {
            if (i0 + 32 * u + 31 < wave_lo) continue;       // no row sees a key of the wave
            v16f st[KT], dp[KT];
#pragma unroll
            for (int kt = 0; kt < KT; ++kt) st[kt] = dp[kt] = zero;
#pragma unroll
            for (int c = 0; c < NC; ++c) {
                const uint4 w = CT<DP>::frag(ql, 32 * u + l31, c, h);
                const uint4 x = CT<DP>::frag(el, 32 * u + l31, c, h);
                const v8h w0 = widen(w.x, w.y), w1 = widen(w.z, w.w);
                const v8h x0 = widen(x.x, x.y), x1 = widen(x.z, x.w);
#pragma unroll
                for (int kt = 0; kt < KT; ++kt) {
                    st[kt] = mfma_half(w0, kf[kt][c][0], st[kt]);
                    st[kt] = mfma_half(w1, kf[kt][c][1], st[kt]);
                    dp[kt] = mfma_half(x0, vf[kt][c][0], dp[kt]);
                    dp[kt] = mfma_half(x1, vf[kt][c][1], dp[kt]);
                }
            }
            const float* lr = rows[b][0] + 32 * u + 4 * h;
            const float* dr = rows[b][1] + 32 * u + 4 * h;
            v8h pf[KT][2], sf[KT][2];
#pragma unroll
            for (int kt = 0; kt < KT; ++kt) {
                float p[16], ds[16];
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    p[r] = __builtin_amdgcn_exp2f(
                        __builtin_fmaf(st[kt][r], c2, -lr[8 * (r / 4) + r % 4]));
                    ds[r] = p[r] * __builtin_fmaf(dp[kt][r], sg, -dr[8 * (r / 4) + r % 4]);
                }
                if (partial) {
                    // row i0 + 32 u + 4 h + x is seen iff that >= key - off
                    const int rel = wave0 + 32 * kt + l31 - off - i0 - 32 * u - 4 * h;
#pragma unroll
                    for (int r = 0; r < 16; ++r)
                        if (8 * (r / 4) + r % 4 < rel) p[r] = ds[r] = 0.0f;
                }
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    pf[kt][t] = to_half8(p + 8 * t);
                    sf[kt][t] = to_half8(ds + 8 * t);
                }
            }
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int d = 0; d < ND; ++d) {
                    const v8h ef = HT<DP>::frag(et, 32 * d + l31, 2 * u + t, h);
                    const v8h qf = HT<DP>::frag(qt, 32 * d + l31, 2 * u + t, h);
#pragma unroll
                    for (int kt = 0; kt < KT; ++kt) {
                        dv[kt][d] = mfma_half(ef, pf[kt][t], dv[kt][d]);
                        dk[kt][d] = mfma_half(qf, sf[kt][t], dk[kt][d]);
                    }
                }
            if (partial) {
                // queries (0) and errors (1) that are not finite, for the keys they see
#pragma unroll
                for (int w = 0; w < 2; ++w) {
                    uint32_t bw = bad[q][w][u];
                    while (bw) {
                        const int i = i0 + 32 * u + __builtin_ctz(bw);
                        bw &= bw - 1;
                        const AttnRows& src = w ? a.e : a.q;
                        const uint8_t* r_ = src.p + (sq.q0 + i) * src.ts + (int64_t)head(n) * src.hs;
#pragma unroll
                        for (int kt = 0; kt < KT; ++kt)
#pragma unroll
                            for (int d = 0; d < ND; ++d)
#pragma unroll
                                for (int r = 0; r < 16; ++r) {
                                    const int col = 32 * d + 8 * (r / 4) + 4 * h + r % 4;
                                    const bool sees = wave0 + 32 * kt + l31 <= i + off;
                                    const uint32_t c = sees && col < a.D ? r_[col] : 0u;
                                    if ((c & 0x7Cu) != 0x7Cu) continue;
                                    if (w) dv[kt][d][r] += fp8_to_f32<0>(c);
                                    else dk[kt][d][r] = __uint_as_float(kF32NaN);
                                }
                    }
                }
            }
        }
        if (tid < 4) bad[(q + 2) % 3][tid / 2][tid % 2] = 0u;
        if (n + 1 < steps) store(n + 1, b ^ 1, bad[(q + 1) % 3]);
        __syncthreads();
    }
    const float fk = a.sm_scale / sigma * a.grad_scale;
    const float fv = __builtin_ldexpf(a.grad_scale, -kPUp);
#pragma unroll
    for (int kt = 0; kt < KT; ++kt) {
        const int j = wave0 + 32 * kt + l31;
        if (j >= sq.nk) continue;
        const int64_t t = sq.k0 + j;
#pragma unroll
        for (int d = 0; d < ND; ++d)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                float x[4], y[4];
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    x[r] = dk[kt][d][4 * q + r] * fk;
                    y[r] = dv[kt][d][4 * q + r] * fv;
                }
                const int col = 32 * d + 8 * q + 4 * h;
                write4<FG>(a.dk, t * a.dk_ts + (int64_t)hk * a.dk_hs, col, a.D, x);
                write4<FG>(a.dv, t * a.dv_ts + (int64_t)hk * a.dv_hs, col, a.D, y);
            }
    }
}

template <int DP, bool VEC, int FG>
void launch(const AttnArgs& a, hipStream_t stream) {
    const int G = a.Hq / a.Hkv;
    const dim3 block(kThreads);
    if (a.Tq > 0)
        hipLaunchKernelGGL((attn_dq_kernel<DP, VEC, FG>),
                           dim3((unsigned)(a.Hkv * slots(a.S, a.Tq, G, 128))), block, 0, stream, a);
    if (a.Tk > 0) {
        constexpr int KT = 1;
        hipLaunchKernelGGL((attn_dkv_kernel<DP, KT, VEC, FG>),
                           dim3((unsigned)(a.Hkv * slots(a.S, a.Tk, 1, 128 * KT))), block, 0, stream, a);
    }
}
template <int DP, bool VEC>
void launch_fmt(const AttnArgs& a, int grad_format, hipStream_t stream) {
    if (grad_format == FP8T_FMT_FP16) launch<DP, VEC, FP8T_FMT_FP16>(a, stream);
    else launch<DP, VEC, FP8T_FMT_FP8>(a, stream);
}

}  // namespace

void attn_bwd_launch(AttnArgs a, int grad_format, bool vec, hipStream_t stream) {
    const int64_t rows = a.Tq * a.Hq + a.Tk * a.Hkv, blocks = (rows + 63) / 64;
    a.norm_count = (int)(blocks < kAttnNorms ? blocks : kAttnNorms);
    const dim3 grid((unsigned)a.norm_count), block(kThreads);
    if (vec) hipLaunchKernelGGL(attn_prepare_kernel<true>, grid, block, 0, stream, a);
    else hipLaunchKernelGGL(attn_prepare_kernel<false>, grid, block, 0, stream, a);
    if (a.D <= 64) {
        if (vec) launch_fmt<64, true>(a, grad_format, stream);
        else launch_fmt<64, false>(a, grad_format, stream);
    } else {
        if (vec) launch_fmt<128, true>(a, grad_format, stream);
        else launch_fmt<128, false>(a, grad_format, stream);
    }
}

}  // namespace fp8t
