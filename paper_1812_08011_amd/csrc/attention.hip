// Attention over packed sequences (attn_fwd_fp8, attn_bwd_fp8): host side.
#include "attn_fwd.h"

namespace fp8t {
namespace {

constexpr int kWaves = 4;             // rows per workgroup, one per wave
constexpr int kThreads = 64 * kWaves;

// A wave's dot products of its row (in LDS, as floats) with 64 keys at a time.
__device__ __forceinline__ float dot_row(const float* row, const uint8_t* p, int D) {
    float s = 0.0f;
    for (int d = 0; d < D; ++d) s = __builtin_fmaf(row[d], fp8_to_f32<0>(p[d]), s);
    return s;
}

// delta = <e, o>, a wave per (query, head).
__global__ __launch_bounds__(kThreads) void attn_delta_rows(AttnArgs a) {
    const int lane = threadIdx.x & 63, h = blockIdx.y;
    const int64_t t = (int64_t)blockIdx.x * kWaves + (threadIdx.x >> 6);
    if (t >= a.Tq) return;
    float s = 0.0f;
    for (int d = lane; d < a.D; d += 64)
        s += fp16_to_f32(a.o[t * a.o_ts + h * a.o_hs + d]) *
             fp8_to_f32<0>(a.e.p[t * a.e.ts + h * a.e.hs + d]);
    for (int d = 32; d; d >>= 1) s += __shfl_xor(s, d);
    if (lane == 0) a.delta[(int64_t)h * a.Tq + t] = s;
}

// dq, a wave per (query, head).
template <int FG>
__global__ __launch_bounds__(kThreads) void attn_dq_rows(AttnArgs a) {
    __shared__ float qs[kWaves][FP8T_ATTN_MAX_D], es[kWaves][FP8T_ATTN_MAX_D];
    __shared__ float ps[kWaves][64];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, h = blockIdx.y;
    int local;
    const int s = slot_owner(a.cu_q, a.S, a.Tq, 1, kWaves, blockIdx.x, local);
    const Seq sq = load_seq(a, s);
    if ((int64_t)local * kWaves >= sq.nq) return;
    const int i = local * kWaves + wave;
    const bool live = i < sq.nq;
    const int64_t t = sq.q0 + (live ? i : 0);
    const int hk = h / (a.Hq / a.Hkv);
    for (int d = lane; d < a.D; d += 64) {
        qs[wave][d] = fp8_to_f32<0>(a.q.p[t * a.q.ts + h * a.q.hs + d]);
        es[wave][d] = fp8_to_f32<0>(a.e.p[t * a.e.ts + h * a.e.hs + d]);
    }
    __syncthreads();
    if (!live) return;
    const int64_t lim = a.causal ? (int64_t)i + 1 + sq.nk - sq.nq : sq.nk;
    const int seen = lim < 0 ? 0 : (int)lim;
    const float lse2 = a.lse[(int64_t)h * a.Tq + t] * kAttnLog2e;
    const float delta = a.delta[(int64_t)h * a.Tq + t];
    float o[2] = {0.0f, 0.0f};
    for (int j0 = 0; j0 < seen; j0 += 64) {
        const int j = j0 + lane;
        float ds = 0.0f;
        if (j < seen) {
            const float x = a.c2 * dot_row(qs[wave], a.k.p + (sq.k0 + j) * a.k.ts + hk * a.k.hs, a.D);
            const float dp = dot_row(es[wave], a.v.p + (sq.k0 + j) * a.v.ts + hk * a.v.hs, a.D);
            ds = exp2f(x - lse2) * (dp - delta);
        }
        ps[wave][lane] = ds;
        __builtin_amdgcn_wave_barrier();
        for (int u = 0; u < 2; ++u) {
            const int d = lane + 64 * u;
            if (d < a.D)
                for (int jj = 0; jj < 64 && j0 + jj < seen; ++jj)
                    o[u] += ps[wave][jj] *
                            fp8_to_f32<0>(a.k.p[(sq.k0 + j0 + jj) * a.k.ts + hk * a.k.hs + d]);
        }
        __builtin_amdgcn_wave_barrier();
    }
    for (int u = 0; u < 2; ++u) {
        const int d = lane + 64 * u;
        if (d < a.D)
            static_cast<fmt_t<FG>*>(a.dq)[t * a.dq_ts + h * a.dq_hs + d] =
                fmt_code<FG>(o[u] * a.sm_scale * a.grad_scale);
    }
}

// dk and dv, a wave per (key, key head).
template <int FG>
__global__ __launch_bounds__(kThreads) void attn_dkv_rows(AttnArgs a) {
    __shared__ float ks[kWaves][FP8T_ATTN_MAX_D], vs[kWaves][FP8T_ATTN_MAX_D];
    __shared__ float ps[kWaves][64], ds[kWaves][64];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, hk = blockIdx.y;
    int local;
    const int s = slot_owner(a.cu_k, a.S, a.Tk, 1, kWaves, blockIdx.x, local);
    const Seq sq = load_seq(a, s);
    if ((int64_t)local * kWaves >= sq.nk) return;
    const int j = local * kWaves + wave;
    const bool live = j < sq.nk;
    const int64_t t = sq.k0 + (live ? j : 0);
    for (int d = lane; d < a.D; d += 64) {
        ks[wave][d] = fp8_to_f32<0>(a.k.p[t * a.k.ts + hk * a.k.hs + d]);
        vs[wave][d] = fp8_to_f32<0>(a.v.p[t * a.v.ts + hk * a.v.hs + d]);
    }
    __syncthreads();
    if (!live) return;
    const int64_t lim = a.causal ? (int64_t)j + sq.nq - sq.nk : 0;
    const int first = lim < 0 ? 0 : (int)lim;                 // the first query that sees j
    const int G = a.Hq / a.Hkv;
    float dk[2] = {0.0f, 0.0f}, dv[2] = {0.0f, 0.0f};
    for (int h = hk * G; h < hk * G + G; ++h)
        for (int i0 = first; i0 < sq.nq; i0 += 64) {
            const int i = i0 + lane;
            float p = 0.0f, dsv = 0.0f;
            if (i < sq.nq) {
                const int64_t ti = sq.q0 + i;
                const float x = a.c2 * dot_row(ks[wave], a.q.p + ti * a.q.ts + h * a.q.hs, a.D);
                const float dp = dot_row(vs[wave], a.e.p + ti * a.e.ts + h * a.e.hs, a.D);
                p = exp2f(x - a.lse[(int64_t)h * a.Tq + ti] * kAttnLog2e);
                dsv = p * (dp - a.delta[(int64_t)h * a.Tq + ti]);
            }
            ps[wave][lane] = p;
            ds[wave][lane] = dsv;
            __builtin_amdgcn_wave_barrier();
            for (int u = 0; u < 2; ++u) {
                const int d = lane + 64 * u;
                if (d < a.D)
                    for (int ii = 0; ii < 64 && i0 + ii < sq.nq; ++ii) {
                        const int64_t ti = sq.q0 + i0 + ii;
                        dk[u] += ds[wave][ii] * fp8_to_f32<0>(a.q.p[ti * a.q.ts + h * a.q.hs + d]);
                        dv[u] += ps[wave][ii] * fp8_to_f32<0>(a.e.p[ti * a.e.ts + h * a.e.hs + d]);
                    }
            }
            __builtin_amdgcn_wave_barrier();
        }
    for (int u = 0; u < 2; ++u) {
        const int d = lane + 64 * u;
        if (d >= a.D) continue;
        static_cast<fmt_t<FG>*>(a.dk)[t * a.dk_ts + hk * a.dk_hs + d] =
            fmt_code<FG>(dk[u] * a.sm_scale * a.grad_scale);
        static_cast<fmt_t<FG>*>(a.dv)[t * a.dv_ts + hk * a.dv_hs + d] =
            fmt_code<FG>(dv[u] * a.grad_scale);
    }
}

// Sizes and flags that both directions share.
bool sizes_ok(int64_t S, int64_t Tq, int64_t Tk, int64_t max_q, int64_t max_k, int64_t Hq,
              int64_t Hkv, int64_t D, int causal) {
    return S >= 0 && Tq >= 0 && Tk >= 0 && max_q >= 0 && max_k >= 0 && Hq >= 0 && Hkv >= 0 &&
           D >= 1 && D <= FP8T_ATTN_MAX_D && S <= kMaxGemmDim && Tq <= kMaxGemmDim &&
           Tk <= kMaxGemmDim && Hq <= 65535 && (Hkv > 0 ? Hq % Hkv == 0 : Hq == 0) &&
           (causal | 1) == 1;
}
bool rows_ok(const void* p, int64_t ts, int64_t hs, int64_t T, int64_t H) {
    return ts >= 0 && hs >= 0 && (p || T == 0 || H == 0);
}

bool rows16(const AttnRows& r) {
    return aligned(r.p, 16) && r.ts % 16 == 0 && r.hs % 16 == 0;
}

}  // namespace
}  // namespace fp8t

using namespace fp8t;

extern "C" size_t attn_fwd_fp8_workspace_size(int64_t S, int64_t Tq, int64_t Tk, int64_t max_q,
                                              int64_t max_k, int64_t Hq, int64_t Hkv, int64_t D,
                                              int causal) {
    if (!sizes_ok(S, Tq, Tk, max_q, max_k, Hq, Hkv, D, causal)) return 0;
    if (S == 0 || Tq == 0 || Hq == 0) return 0;
    return attn_fwd_plan(S, Tq, max_q, max_k, Hq, Hkv, D).bytes;
}

extern "C" int attn_fwd_fp8(const uint8_t* q, int64_t q_ts, int64_t q_hs, const uint8_t* k,
                            int64_t k_ts, int64_t k_hs, const uint8_t* v, int64_t v_ts,
                            int64_t v_hs, const int64_t* cu_q, const int64_t* cu_k, int64_t S,
                            int64_t Tq, int64_t Tk, int64_t max_q, int64_t max_k, int64_t Hq,
                            int64_t Hkv, int64_t D, int causal, float sm_scale, uint16_t* o,
                            int64_t o_ts, int64_t o_hs, uint8_t* o8, int64_t o8_ts, int64_t o8_hs,
                            float o8_scale, float* lse, void* workspace, size_t workspace_bytes,
                            hipStream_t stream) {
    if (!sizes_ok(S, Tq, Tk, max_q, max_k, Hq, Hkv, D, causal)) return FP8T_EINVAL;
    if (!(sm_scale > 0.0f) || !(sm_scale <= 3.4e38f)) return FP8T_EINVAL;
    if (!rows_ok(q, q_ts, q_hs, Tq, Hq) || !rows_ok(k, k_ts, k_hs, Tk, Hkv) ||
        !rows_ok(v, v_ts, v_hs, Tk, Hkv) || (!workspace && workspace_bytes))
        return FP8T_EINVAL;
    if (S == 0 || Tq == 0 || Hq == 0) return FP8T_OK;
    if (!cu_q || !cu_k || (!o && !o8 && !lse)) return FP8T_EINVAL;
    if ((o && !rows_apart(Tq, Hq, D, o_ts, o_hs)) || (o8 && !rows_apart(Tq, Hq, D, o8_ts, o8_hs)))
        return FP8T_EINVAL;
    AttnFwdPlan p = attn_fwd_plan(S, Tq, max_q, max_k, Hq, Hkv, D);
    if (workspace_bytes && workspace_bytes < p.bytes) return FP8T_EWORKSPACE;
    if (p.bytes && !workspace_bytes) p.splits = 1;
    if (p.splits > 1 && !aligned(workspace, 16)) return FP8T_EINVAL;
    AttnArgs a = {};
    a.q = {q, q_ts, q_hs};
    a.k = {k, k_ts, k_hs};
    a.v = {v, v_ts, v_hs};
    a.cu_q = cu_q;
    a.cu_k = cu_k;
    a.S = (int)S;
    a.Hq = (int)Hq;
    a.Hkv = (int)Hkv;
    a.D = (int)D;
    a.causal = causal;
    a.Tq = Tq;
    a.Tk = Tk;
    a.c2 = sm_scale * kAttnLog2e;
    a.sm_scale = sm_scale;
    a.o = o;
    a.o_ts = o_ts;
    a.o_hs = o_hs;
    a.o8 = o8;
    a.o8_ts = o8_ts;
    a.o8_hs = o8_hs;
    a.o8_scale = o8_scale;
    a.lse = lse;
    const bool vec = D % 16 == 0 && rows16(a.q) && rows16(a.k) && rows16(a.v);
    attn_fwd_launch(a, p, vec, workspace, stream);
    return launch_status();
}

extern "C" size_t attn_bwd_fp8_workspace_size(int64_t S, int64_t Tq, int64_t Tk, int64_t max_q,
                                              int64_t max_k, int64_t Hq, int64_t Hkv, int64_t D,
                                              int causal) {
    if (!sizes_ok(S, Tq, Tk, max_q, max_k, Hq, Hkv, D, causal)) return 0;
    return (size_t)Hq * Tq * sizeof(float);
}

extern "C" int attn_bwd_fp8(const uint8_t* q, int64_t q_ts, int64_t q_hs, const uint8_t* k,
                            int64_t k_ts, int64_t k_hs, const uint8_t* v, int64_t v_ts,
                            int64_t v_hs, const int64_t* cu_q, const int64_t* cu_k, int64_t S,
                            int64_t Tq, int64_t Tk, int64_t max_q, int64_t max_k, int64_t Hq,
                            int64_t Hkv, int64_t D, int causal, float sm_scale, const uint16_t* o,
                            int64_t o_ts, int64_t o_hs, const uint8_t* d_o, int64_t do_ts,
                            int64_t do_hs, const float* lse, void* dq, int64_t dq_ts,
                            int64_t dq_hs, void* dk, int64_t dk_ts, int64_t dk_hs, void* dv,
                            int64_t dv_ts, int64_t dv_hs, int grad_format, float grad_scale,
                            void* workspace, size_t workspace_bytes, hipStream_t stream) {
    if (!sizes_ok(S, Tq, Tk, max_q, max_k, Hq, Hkv, D, causal)) return FP8T_EINVAL;
    if (!(sm_scale > 0.0f) || !(sm_scale <= 3.4e38f)) return FP8T_EINVAL;
    if (grad_format != FP8T_FMT_FP16 && grad_format != FP8T_FMT_FP8) return FP8T_EINVAL;
    if (!rows_ok(q, q_ts, q_hs, Tq, Hq) || !rows_ok(k, k_ts, k_hs, Tk, Hkv) ||
        !rows_ok(v, v_ts, v_hs, Tk, Hkv) || !rows_ok(o, o_ts, o_hs, Tq, Hq) ||
        !rows_ok(d_o, do_ts, do_hs, Tq, Hq) || !rows_ok(dq, dq_ts, dq_hs, Tq, Hq) ||
        !rows_ok(dk, dk_ts, dk_hs, Tk, Hkv) || !rows_ok(dv, dv_ts, dv_hs, Tk, Hkv) ||
        (!workspace && workspace_bytes))
        return FP8T_EINVAL;
    if (S == 0 || Hq == 0 || (Tq == 0 && Tk == 0)) return FP8T_OK;
    if (!cu_q || !cu_k || (Tq > 0 && !lse)) return FP8T_EINVAL;
    if (!rows_apart(Tq, Hq, D, dq_ts, dq_hs) || !rows_apart(Tk, Hkv, D, dk_ts, dk_hs) ||
        !rows_apart(Tk, Hkv, D, dv_ts, dv_hs) || !aligned(workspace, 16))
        return FP8T_EINVAL;
    if (workspace_bytes <
        attn_bwd_fp8_workspace_size(S, Tq, Tk, max_q, max_k, Hq, Hkv, D, causal))
        return FP8T_EWORKSPACE;
    AttnArgs a = {};
    a.q = {q, q_ts, q_hs};
    a.k = {k, k_ts, k_hs};
    a.v = {v, v_ts, v_hs};
    a.e = {d_o, do_ts, do_hs};
    a.cu_q = cu_q;
    a.cu_k = cu_k;
    a.S = (int)S;
    a.Hq = (int)Hq;
    a.Hkv = (int)Hkv;
    a.D = (int)D;
    a.causal = causal;
    a.Tq = Tq;
    a.Tk = Tk;
    a.c2 = sm_scale * kAttnLog2e;
    a.sm_scale = sm_scale;
    a.o = const_cast<uint16_t*>(o);
    a.o_ts = o_ts;
    a.o_hs = o_hs;
    a.lse = const_cast<float*>(lse);
    a.dq = dq;
    a.dq_ts = dq_ts;
    a.dq_hs = dq_hs;
    a.dk = dk;
    a.dk_ts = dk_ts;
    a.dk_hs = dk_hs;
    a.dv = dv;
    a.dv_ts = dv_ts;
    a.dv_hs = dv_hs;
    a.grad_scale = grad_scale;
    a.delta = static_cast<float*>(workspace);
    const dim3 block(kThreads);
    const dim3 gq((unsigned)slots(S, Tq, 1, kWaves), (unsigned)Hq);
    const dim3 gk((unsigned)slots(S, Tk, 1, kWaves), (unsigned)Hkv);
    if (Tq > 0) {
        hipLaunchKernelGGL(attn_delta_rows, dim3((unsigned)((Tq + kWaves - 1) / kWaves), (unsigned)Hq),
                           block, 0, stream, a);
        if (grad_format == FP8T_FMT_FP16)
            hipLaunchKernelGGL(attn_dq_rows<FP8T_FMT_FP16>, gq, block, 0, stream, a);
        else
            hipLaunchKernelGGL(attn_dq_rows<FP8T_FMT_FP8>, gq, block, 0, stream, a);
    }
    if (Tk > 0) {
        if (grad_format == FP8T_FMT_FP16)
            hipLaunchKernelGGL(attn_dkv_rows<FP8T_FMT_FP16>, gk, block, 0, stream, a);
        else
            hipLaunchKernelGGL(attn_dkv_rows<FP8T_FMT_FP8>, gk, block, 0, stream, a);
    }
    return launch_status();
}
