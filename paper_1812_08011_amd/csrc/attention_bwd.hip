// Attention backward on the matrix cores, from the images that attn_image.hip
// builds first:
//   dq:      a wave owns rows (queries) and streams the keys;
//   dk, dv:  a wave owns keys and streams the queries of every head that
//            shares them.
// Scores are computed twice (7 products instead of 5), which needs no atomics:
// the same bits on every run.  p = exp(s - lse) needs no running statistics;
// delta = <e, o> enters as the start of the product <e, V_j>'s sums.
//
// The operands are IEEE halves, FP8 codes exactly.  p (at most 1) is held times
// 2^15: all 11 bits down to 2^-29, steps of 2^-39 below, so that dv loses at most
// 2^-40 of every error it sums.  dS is held times a power of two that its row or
// its key finds for itself (kDsFirst).  Sums are FP32.
//
// The three products of dq and the four of dk and dv bound them: with 8192
// causal tokens, 16 heads of 128 and 4 key heads 412 GFLOP in 398 us (1035
// TFLOP/s) and 550 GFLOP in 673 us (817 TFLOP/s), of 1138 that a large product
// reaches.  D 64, mixed lengths: 69 GFLOP in 98 us and 92 GFLOP in 148 us; the
// vector ALUs are busy for 58% and 44% of it, the matrix cores for 32% and 28%
// (D 128: 52% and 35%, 48% and 36%).  With D above 64 both keep 2 waves per SIMD
// (246 and 254 registers): the sums take 64 registers of a lane in dq and 128 in
// dk and dv (64 keys a wave spilled: 26 ms for the pass over those 8192 tokens),
// and read their tiles from images, since transposing them in the loop spilled
// too (9 ms).  D up to 64 takes 162 and 168 registers, 3 waves.  Looking for the
// largest dS takes 10 instructions per 32 x 32 scores, 4 to 5% of these times.
#include "attn_bwd.h"
#include "attn_image.h"

namespace fp8t {
namespace {

constexpr int kThreads = 256;

// dS = p (<e, v> - delta) is held times a power of two of the lane's own -- a
// row's in dq, a key's in dk -- so that what one row or key keeps does not
// depend on any other.  It starts so large that any dS that reaches a result
// has all 11 bits of a half, and goes down when one of the sum passes kDsRoom
// (the largest half is 65504), the sums so far with it: the first steps of a
// wave do that, later ones seldom.  The largest then lies in [2^11, 2^12) (one
// power of two higher the sums go down more often, 1 to 2% of the time), so that
// a dS down to 2^-25 of it keeps all 11 bits, with steps of 2^-35 below.
constexpr float kDsFirst = 0x1p64f;    // |<e, v>| and |delta| stay below 2^56: no overflow
constexpr float kDsRoom = 61440.0f;
// A lane's largest, NaN if one is: its row's or its key's result is NaN then.
__device__ __forceinline__ float ds_top(const float* ds) {
    float a = 0.0f, b = 0.0f;                               // two chains
#pragma unroll
    for (int r = 0; r < 16; r += 4) {
        a = maximum3_abs(a, ds[r], ds[r + 1]);
        b = maximum3_abs(b, ds[r + 2], ds[r + 3]);
    }
    return maximum3_abs(0.0f, a, b);
}
// The factor that brings the largest finite one down; ds times it.
__device__ __forceinline__ float ds_down(float* ds, float top) {
    if (__builtin_expect(__any(!(top < INFINITY)), 0)) {
        top = 0.0f;
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            const float x = __builtin_fabsf(ds[r]);
            top = fmaxf(top, x < INFINITY ? x : 0.0f);
        }
    }
    top = both_halves(top, [](float a, float b) { return fmaxf(a, b); });
    const float f = top > kDsRoom ? __builtin_ldexpf(1.0f, 12 - __builtin_amdgcn_frexp_expf(top)) : 1.0f;
#pragma unroll
    for (int r = 0; r < 16; ++r) ds[r] *= f;
    return f;
}

// ---- dq ------------------------------------------------------------------------------------

// 128 rows (query, head of the group), 32 per wave; key tiles one ahead in
// LDS.  dQ^T = K^T dS^T with dS^T's registers as the operand.
template <int DP, bool VEC, int FG>
__global__ __launch_bounds__(kThreads, 2) void attn_dq_kernel(AttnArgs a) {
    using I = KeyImage<DP>;
    constexpr int BM = kAttnRows, N = I::N, NC = DP / 32, ND = DP / 32;
    __shared__ __attribute__((aligned(16))) uint8_t lds[2 * I::kBytes];
    static_assert(sizeof(lds) >= 4 * kRowsOut, "the results' way out fits the buffers");
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int l31 = lane & 31, h = lane >> 5;
    const int hk = blockIdx.x % a.Hkv;
    const int slot = ordered_slot(a.row_order, blockIdx.x / a.Hkv);
    if (slot < 0) return;
    int tile;
    const Seq sq = load_seq(a, slot_owner(a.cu_q, a.S, a.Tq, a.G, BM, slot, tile));
    const int nrows = sq.nq * a.G, ntiles = (nrows + BM - 1) / BM;
    if (tile >= ntiles) return;
    const int row0 = (ntiles - 1 - tile) * BM, row = row0 + 32 * wave + l31;   // the longest first
    const bool live = row < nrows;
    const int i = live ? div_g(a, row) : 0, g = live ? row - i * a.G : 0, off = sq.nk - sq.nq;
    auto limit = [&](int i) {
        const int n = a.causal ? i + 1 + off : sq.nk;
        return n < 0 ? 0 : n;
    };
    const int lim = live ? limit(i) : 0;
    const int lim_lo = limit(div_g(a, row0));
    const int lim_hi = limit(div_g(a, row0 + BM < nrows ? row0 + BM - 1 : nrows - 1));
    const int w0 = row0 + 32 * wave;
    const int wave_hi = w0 < nrows ? limit(div_g(a, w0 + 31 < nrows ? w0 + 31 : nrows - 1)) : 0;
    const int first = (int)(sq.k0 / N), j00 = (int)((int64_t)first * N - sq.k0);
    const int t1 = lim_hi > 0 ? (lim_hi - j00 + N - 1) / N : 0;
    const uint8_t* image = a.key_image + ((int64_t)hk * a.key_tiles + first) * I::kBytes;
    if (t1 > 0) image_to_lds<I::kBytes, 4>(image, lds, wave, lane);

    const int64_t tq = sq.q0 + i;
    const int hq = hk * a.G + g;
    const uint8_t* qp = a.q.p + tq * a.q.ts + (int64_t)hq * a.q.hs;
    const uint8_t* ep = a.e.p + tq * a.e.ts + (int64_t)hq * a.e.hs;
    const uint8_t* kp = a.k.p + sq.k0 * a.k.ts + (int64_t)hk * a.k.hs;
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
    float sigma = kDsFirst, lse2 = INFINITY, delta = 0.0f;  // a row that sees nothing: p = 0
    if (lim > 0) {
        lse2 = a.lse[(int64_t)hq * a.Tq + tq] * kAttnLog2e;
        delta = a.delta[(int64_t)hq * a.Tq + tq] * sigma;
    }

    v16f o[ND];
#pragma unroll
    for (int d = 0; d < ND; ++d)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[d][r] = 0.0f;
    const v16f zero = {0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0};
    uint32_t noted_any = 0;
    for (int t = 0; t < t1; ++t) {
        const uint8_t* buf = lds + (t & 1) * I::kBytes;
        image_barrier();
        if (t + 1 < t1)
            image_to_lds<I::kBytes, 4>(image + (int64_t)(t + 1) * I::kBytes,
                                       lds + ((t + 1) & 1) * I::kBytes, wave, lane);
        const int j0 = j00 + t * N;
        if (j0 >= wave_hi) continue;
        const bool partial = j0 < 0 || j0 + N > lim_lo;
#pragma unroll
        for (int kt = 0; kt < N / 32; ++kt) {
            v16f st = zero, dp = zero;
#pragma unroll
            for (int c = 0; c < NC; ++c) {
                uint4 w = I::CT::frag(buf, 32 * kt + l31, c, h);
                st = mfma_half(widen(w.x, w.y), qf[c][0], st);
                st = mfma_half(widen(w.z, w.w), qf[c][1], st);
                w = I::CT::frag(buf + I::kV, 32 * kt + l31, c, h);
                dp = mfma_half(widen(w.x, w.y), ef[c][0], dp);
                dp = mfma_half(widen(w.z, w.w), ef[c][1], dp);
            }
            float ds[16];
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(st[r], c2, -lse2));
                ds[r] = p * __builtin_fmaf(dp[r], sigma, -delta);
            }
            if (partial) {
                int key = j0 + 32 * kt + 4 * h;
                asm volatile("" : "+v"(key));               // a branch: no selects on whole tiles
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    if ((uint32_t)(key + 8 * (r / 4) + r % 4) >= (uint32_t)lim) ds[r] = 0.0f;
            }
            const float top = ds_top(ds);
            if (__builtin_expect(__any(top > kDsRoom), 0)) {
                const float f = ds_down(ds, top);
                sigma *= f;
                delta *= f;
#pragma unroll
                for (int d = 0; d < ND; ++d)
#pragma unroll
                    for (int r = 0; r < 16; ++r) o[d][r] *= f;
            }
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const v8h f = to_half8(ds + 8 * u);
#pragma unroll
                for (int d = 0; d < ND; ++d)
                    o[d] = mfma_half(I::HT::frag(buf + I::kT, 32 * d + l31, 2 * kt + u, h), f, o[d]);
            }
            noted_any |= reinterpret_cast<const uint32_t*>(buf + I::kNoted)[kt];
        }
    }
    if (__builtin_expect(__any(noted_any != 0), 0)) {
        // keys that are not finite, for the rows that see them
#pragma unroll 1
        for (int i = 0; i < t1 * (N / 32); ++i) {
            const uint8_t* at = image + (int64_t)(i / (N / 32)) * I::kBytes + I::kNoted;
            add_noted<ND>(reinterpret_cast<const uint32_t*>(at)[i % (N / 32)], kp, a.k.ts, j00 + 32 * i, a.D,
                          h, [&](int key) { return (uint32_t)key < (uint32_t)lim; },
                          [&](int d, int r, uint32_t) { o[d][r] = __uint_as_float(kF32NaN); });
        }
    }
    __syncthreads();                                        // the buffers are free
    const int64_t at = tq * a.dq_ts + (int64_t)hq * a.dq_hs;
    rows_out<DP>(reinterpret_cast<float*>(lds + wave * kRowsOut), o, a.sm_scale / sigma * a.grad_scale, lane,
                 [&](int r, int col, const float* x) {
                     const int64_t to = of_lane(at, r);
                     const int n = __shfl((int)live, r) ? up_to_8(a.D - col) : 0;
                     if (n) store_some<FG>(static_cast<fmt_t<FG>*>(a.dq) + to + col, n, x);
                 });
}

// ---- dk and dv --------------------------------------------------------------------------------

// 128 keys of a sequence, 32 per wave; the queries and errors of the group's
// heads stream through LDS in tiles of 32.  dV^T = E^T P and dK^T = Q^T dS with
// P's and dS's registers as the operands.  SPLIT: gridDim.y workgroups share a
// tile's steps (every gridDim.y-th each) and leave FP32 sums in the workspace.
template <int DP, bool VEC, int FG, bool SPLIT>
__global__ __launch_bounds__(kThreads, 2) void attn_dkv_kernel(AttnArgs a) {
    using I = QueryImage<DP>;
    constexpr int BN = kAttnDkvKeys, N = I::N, NC = DP / 32, ND = DP / 32;
    constexpr int kLds = 2 * I::kBytes > 4 * kRowsOut ? 2 * I::kBytes : 4 * kRowsOut;
    __shared__ __attribute__((aligned(16))) uint8_t lds[kLds];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int l31 = lane & 31, h = lane >> 5;
    const int hk = blockIdx.x % a.Hkv, G = a.G;
    const int slot = ordered_slot(a.key_order, blockIdx.x / a.Hkv);
    if (slot < 0) return;
    int tile;
    const Seq sq = load_seq(a, slot_owner(a.cu_k, a.S, a.Tk, 1, BN, slot, tile));
    if ((int64_t)tile * BN >= sq.nk) return;
    const int off = sq.nk - sq.nq, key0 = tile * BN, wave0 = key0 + 32 * wave, j = wave0 + l31;
    const int key_hi = key0 + BN < sq.nk ? key0 + BN - 1 : sq.nk - 1;
    // query i sees key j iff i >= j - off; [lo, nq) see this lane's key
    const int first = a.causal && key0 - off > 0 ? key0 - off : 0;
    const int lo = a.causal && j - off > 0 ? j - off : 0;
    const uint32_t seen_by = sq.nq > lo ? (uint32_t)(sq.nq - lo) : 0u;
    const int wave_lo = a.causal ? wave0 - off : 0;         // the wave's first key's first query
    const int all_lo = a.causal && key_hi - off > 0 ? key_hi - off : 0;   // from here on every key is seen
    // tiles of the packed queries that hold some of [q0 + first, q0 + nq)
    const int ta = (int)((sq.q0 + first) / N), tb = (int)((sq.q0 + sq.nq + N - 1) / N);
    const int ntq = first < sq.nq ? tb - ta : 0, steps = ntq * G;
    const int n0 = SPLIT ? blockIdx.y : 0, dn = SPLIT ? gridDim.y : 1;
    auto issue = [&](int n, int b) {
        const int hq = hk * G + n / ntq, t = ta + n % ntq;
        image_to_lds<I::kBytes, 4>(a.query_image + ((int64_t)hq * a.query_tiles + t) * I::kBytes,
                                   lds + b * I::kBytes, wave, lane);
    };
    if (n0 < steps) issue(n0, 0);

    const uint8_t* kp = a.k.p + (sq.k0 + j) * a.k.ts + (int64_t)hk * a.k.hs;
    const uint8_t* vp = a.v.p + (sq.k0 + j) * a.v.ts + (int64_t)hk * a.v.hs;
    const Widen widen;
    const float c2 = __uint_as_float(in_vgpr(__float_as_uint(a.c2)));
    v8h kf[NC][2];
    uint4 vf[NC];
#pragma unroll
    for (int c = 0; c < NC; ++c) {
        const uint4 w = load_codes16<VEC>(kp, 32 * c + 16 * h, a.D, j < sq.nk);
        kf[c][0] = widen(w.x, w.y);
        kf[c][1] = widen(w.z, w.w);
        vf[c] = load_codes16<VEC>(vp, 32 * c + 16 * h, a.D, j < sq.nk);
    }
    // p is held times 2^15, dS times sigma: p (dP - delta) sigma 2^-15
    float sg = j < sq.nk ? __builtin_ldexpf(kDsFirst, -kAttnPUp) : 0.0f;

    v16f dk[ND], dv[ND];
#pragma unroll
    for (int d = 0; d < ND; ++d)
#pragma unroll
        for (int r = 0; r < 16; ++r) dk[d][r] = dv[d][r] = 0.0f;
    const v16f zero = {0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0};
    int b = 0;
    uint32_t noted_any = 0;
    for (int n = n0; n < steps; n += dn, b ^= 1) {
        image_barrier();
        if (n + dn < steps) issue(n + dn, b ^ 1);
        const int i0 = (int)((int64_t)(ta + n % ntq) * N - sq.q0);
        if (i0 + N - 1 < wave_lo) continue;                 // no row sees a key of the wave
        const bool partial = i0 < all_lo || i0 + N > sq.nq;
        // opaque in every step: the compiler otherwise hoists the widened values
        // out of the loop, past the register budget
#pragma unroll
        for (int c = 0; c < NC; ++c)
            asm volatile("" : "+v"(vf[c].x), "+v"(vf[c].y), "+v"(vf[c].z), "+v"(vf[c].w));
        const uint8_t* buf = lds + b * I::kBytes;
        // dp starts from -delta
        v16f st = zero, dp;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const float4 x = *reinterpret_cast<const float4*>(buf + I::delta(2 * q + h));
            dp[4 * q] = x.x;
            dp[4 * q + 1] = x.y;
            dp[4 * q + 2] = x.z;
            dp[4 * q + 3] = x.w;
        }
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            uint4 w = I::CT::frag(buf, l31, c, h);
            st = mfma_half(widen(w.x, w.y), kf[c][0], st);
            st = mfma_half(widen(w.z, w.w), kf[c][1], st);
            w = I::CT::frag(buf + I::kE, l31, c, h);
            dp = mfma_half(widen(w.x, w.y), widen(vf[c].x, vf[c].y), dp);
            dp = mfma_half(widen(w.z, w.w), widen(vf[c].z, vf[c].w), dp);
        }
        float p[16], ds[16];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const float4 x = *reinterpret_cast<const float4*>(buf + I::lse(2 * q + h));
            const float l[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                p[4 * q + r] = __builtin_amdgcn_exp2f(__builtin_fmaf(st[4 * q + r], c2, -l[r]));
                ds[4 * q + r] = p[4 * q + r] * (dp[4 * q + r] * sg);
            }
        }
        if (partial) {
            int i = i0 + 4 * h - lo;
            asm volatile("" : "+v"(i));                     // a branch: no selects on whole tiles
#pragma unroll
            for (int r = 0; r < 16; ++r)
                if ((uint32_t)(i + 8 * (r / 4) + r % 4) >= seen_by) p[r] = ds[r] = 0.0f;
        }
        const float top = ds_top(ds);
        if (__builtin_expect(__any(top > kDsRoom), 0)) {
            const float f = ds_down(ds, top);
            sg *= f;
#pragma unroll
            for (int d = 0; d < ND; ++d)
#pragma unroll
                for (int r = 0; r < 16; ++r) dk[d][r] *= f;
        }
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const v8h pf = to_half8(p + 8 * t), sf = to_half8(ds + 8 * t);
#pragma unroll
            for (int d = 0; d < ND; ++d) {
                dv[d] = mfma_half(I::HT::frag(buf + I::kET, 32 * d + l31, t, h), pf, dv[d]);
                dk[d] = mfma_half(I::HT::frag(buf + I::kQT, 32 * d + l31, t, h), sf, dk[d]);
            }
        }
        const uint32_t* noted = reinterpret_cast<const uint32_t*>(buf + I::kNoted);
        noted_any |= noted[0] | noted[1];
    }
    if (__builtin_expect(__any(noted_any != 0), 0)) {
        // queries and errors that are not finite, for the keys they see
#pragma unroll 1
        for (int n = n0; n < steps; n += dn) {
            const int hq = hk * G + n / ntq, t = ta + n % ntq, i0 = (int)((int64_t)t * N - sq.q0);
            const uint8_t* at = a.query_image + ((int64_t)hq * a.query_tiles + t) * I::kBytes + I::kNoted;
            const uint32_t* noted = reinterpret_cast<const uint32_t*>(at);
            auto sees = [&](int i) { return (uint32_t)(i - lo) < seen_by; };
            add_noted<ND>(noted[0], a.q.p + sq.q0 * a.q.ts + (int64_t)hq * a.q.hs, a.q.ts, i0, a.D, h, sees,
                          [&](int d, int r, uint32_t) { dk[d][r] = __uint_as_float(kF32NaN); });
            add_noted<ND>(noted[1], a.e.p + sq.q0 * a.e.ts + (int64_t)hq * a.e.hs, a.e.ts, i0, a.D, h, sees,
                          [&](int d, int r, uint32_t c) { dv[d][r] += fp8_nonfinite(c); });
        }
    }
    const float fk = __builtin_ldexpf(a.sm_scale / sg, -kAttnPUp) * a.grad_scale, fv = __builtin_ldexpf(a.grad_scale, -kAttnPUp);
    const int64_t t = sq.k0 + j;
    __syncthreads();                                        // the buffers are free
    float* xs = reinterpret_cast<float*>(lds + wave * kRowsOut);
    auto out = [&](const v16f* acc, float scale, void* base, int64_t ts, int64_t hs) {
        const int64_t at = t * ts + (int64_t)hk * hs;
        rows_out<DP>(xs, acc, scale, lane, [&](int r, int col, const float* x) {
            const int64_t to = of_lane(at, r);
            if (wave0 + r >= sq.nk) return;
            if constexpr (SPLIT) {
                store_some<FP8T_FMT_F32>(static_cast<float*>(base) + to + col, 8, x);
            } else {
                const int n = up_to_8(a.D - col);
                if (n) store_some<FG>(static_cast<fmt_t<FG>*>(base) + to + col, n, x);
            }
        });
    };
    if constexpr (SPLIT) {
        float* part = a.parts + (int64_t)blockIdx.y * a.Tk * a.Hkv * (2 * DP);
        out(dk, fk, part, (int64_t)a.Hkv * (2 * DP), 2 * DP);
        out(dv, fv, part + DP, (int64_t)a.Hkv * (2 * DP), 2 * DP);
    } else {
        out(dk, fk, a.dk, a.dk_ts, a.dk_hs);
        out(dv, fv, a.dv, a.dv_ts, a.dv_hs);
    }
}

// Sums the partial dk and dv in their order: eight entries a thread.  A token
// of no sequence is not written.  HBM-bound: 4 parts of 8192 x 4 x 256 floats in
// 25 us, 6 TB/s (part of it from the caches).
template <int DP, int FG>
__global__ __launch_bounds__(kThreads) void attn_dkv_join_kernel(AttnArgs a) {
    constexpr int kPer = 2 * DP / 8;                        // threads per (token, head)
    const int64_t id = (int64_t)blockIdx.x * kThreads + threadIdx.x, rows = a.Tk * a.Hkv;
    const int64_t row = id / kPer;
    const int c = (int)(id % kPer) * 8, col = c % DP, n = up_to_8(a.D - col);
    if (row >= rows || n == 0) return;
    const int64_t t = row / a.Hkv, hk = row % a.Hkv;
    if (t < clamp_to(a.cu_k[0], a.Tk) || t >= clamp_to(a.cu_k[a.S], a.Tk)) return;
    float x[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    const float* part = a.parts + row * (2 * DP) + c;
    for (int z = 0; z < a.splits; ++z) {
        const float4 p = *reinterpret_cast<const float4*>(part + z * rows * (2 * DP));
        const float4 q = *reinterpret_cast<const float4*>(part + z * rows * (2 * DP) + 4);
        const float y[8] = {p.x, p.y, p.z, p.w, q.x, q.y, q.z, q.w};
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] += y[i];
    }
    const bool is_k = c < DP;
    const int64_t at = is_k ? t * a.dk_ts + hk * a.dk_hs : t * a.dv_ts + hk * a.dv_hs;
    store_some<FG>(static_cast<fmt_t<FG>*>(is_k ? a.dk : a.dv) + at + col, n, x);
}

template <int DP, bool VEC, int FG>
void launch(const AttnArgs& a, hipStream_t stream) {
    const dim3 block(kThreads);
    if (a.Tq > 0)
        hipLaunchKernelGGL((attn_dq_kernel<DP, VEC, FG>),
                           dim3((unsigned)(a.Hkv * slots(a.S, a.Tq, a.G, kAttnRows))), block, 0,
                           stream, a);
    if (a.Tk == 0) return;
    const dim3 grid((unsigned)(a.Hkv * slots(a.S, a.Tk, 1, kAttnDkvKeys)), (unsigned)a.splits);
    if (a.splits > 1) {
        hipLaunchKernelGGL((attn_dkv_kernel<DP, VEC, FG, true>), grid, block, 0, stream, a);
        const int64_t items = a.Tk * a.Hkv * (2 * DP / 8);
        hipLaunchKernelGGL((attn_dkv_join_kernel<DP, FG>), dim3((unsigned)((items + kThreads - 1) / kThreads)),
                           block, 0, stream, a);
    } else {
        hipLaunchKernelGGL((attn_dkv_kernel<DP, VEC, FG, false>), grid, block, 0, stream, a);
    }
}
template <int DP, bool VEC>
void launch_fmt(const AttnArgs& a, int grad_format, hipStream_t stream) {
    if (grad_format == FP8T_FMT_FP16) launch<DP, VEC, FP8T_FMT_FP16>(a, stream);
    else launch<DP, VEC, FP8T_FMT_FP8>(a, stream);
}

}  // namespace

AttnBwdPlan attn_bwd_plan(int64_t S, int64_t Tq, int64_t Tk, int64_t max_q, int64_t max_k, int64_t Hq,
                          int64_t Hkv, int64_t D) {
    AttnBwdPlan p = {};
    const int64_t G = Hkv ? Hq / Hkv : 1;
    max_q = hint(max_q, G);
    max_k = hint(max_k, 1);
    p.DP = D <= 64 ? 64 : 128;
    const auto up = [](int64_t n) { return (size_t)((n + 15) / 16 * 16); };
    p.key_tiles = image_tiles(Tk, 64);
    p.query_tiles = image_tiles(Tq, 32);
    p.delta = 0;
    p.key_image = p.delta + up(Hq * Tq * 4);
    p.query_image = p.key_image + (size_t)(p.key_tiles * Hkv) *
                                      (p.DP == 64 ? KeyImage<64>::kBytes : KeyImage<128>::kBytes);
    p.order = p.query_image + (size_t)(p.query_tiles * Hq) *
                                  (p.DP == 64 ? QueryImage<64>::kBytes : QueryImage<128>::kBytes);
    const int64_t row_slots = slots(S, Tq, G, kAttnRows);
    p.key_order = p.order + (S > 1 ? up(row_slots * 4) : 0);
    p.parts = p.key_order + (S > 1 ? up(slots(S, Tk, 1, kAttnDkvKeys) * 4) : 0);
    // The steps of a key tile are shared out where the tiles leave CUs idle,
    // until there are 4 workgroups per CU, with 16 steps of 32 queries each at
    // least.  8192 causal tokens, 16 heads of 128, 4 key heads, forward and
    // gradients: 1416 us with 4; with 2 1614 (the causal tiles differ in length);
    // with 8 1375, for twice the partial results: 268 MB of workspace more than
    // none in place of 134.
    const int64_t tiles = slots(S, Tk, 1, kAttnDkvKeys);
    const int64_t some = S * ((max_k + kAttnDkvKeys - 1) / kAttnDkvKeys), groups = (tiles < some ? tiles : some) * Hkv;
    const int64_t steps = (max_q + 31) / 32 * G, want = 4 * (int64_t)device_cus();
    int64_t n = groups > 0 && 2 * groups <= want ? want / groups : 1;
    if (n > steps / 16) n = steps / 16;
    if (n > 16) n = 16;
    p.splits = n > 1 ? (int)n : 1;
    p.fits = row_slots * Hkv <= kAttnGrid && tiles * Hkv <= kAttnGrid && p.key_tiles * Hkv < kAttnGrid - 1 &&
             p.query_tiles * Hq <= kAttnGrid &&
             (p.splits == 1 || Tk * Hkv * (2 * p.DP / 8) / kThreads < kAttnGrid);
    p.bytes = p.parts + (p.splits > 1 ? (size_t)p.splits * Tk * Hkv * 2 * p.DP * 4 : 0);
    return p;
}

void attn_bwd_launch(AttnArgs a, const AttnBwdPlan& p, int grad_format, bool vec, void* workspace,
                     hipStream_t stream) {
    uint8_t* w = static_cast<uint8_t*>(workspace);
    a.delta = reinterpret_cast<float*>(w + p.delta);
    a.key_image = w + p.key_image;
    a.query_image = w + p.query_image;
    a.parts = reinterpret_cast<float*>(w + p.parts);
    a.key_tiles = p.key_tiles;
    a.query_tiles = p.query_tiles;
    a.splits = p.splits;
    if (a.S > 1) {
        a.row_order = reinterpret_cast<int*>(w + p.order);
        a.key_order = reinterpret_cast<int*>(w + p.key_order);
    }
    attn_bwd_image_launch(a, vec, p.DP, stream);
    if (p.DP == 64) {
        if (vec) launch_fmt<64, true>(a, grad_format, stream);
        else launch_fmt<64, false>(a, grad_format, stream);
    } else {
        if (vec) launch_fmt<128, true>(a, grad_format, stream);
        else launch_fmt<128, false>(a, grad_format, stream);
    }
}

}  // namespace fp8t
