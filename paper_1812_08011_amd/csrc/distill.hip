// distill_loss: Kullback-Leibler loss against a teacher's top logits and the
// gradient of the student's logits.  One workgroup per row.
#include "lm_formats.h"

namespace fp8t {
namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;
constexpr int kMaxTop = 4096;
constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kLn2 = 0.69314718055994530942f;

struct DistillArgs {
    const void* z;
    const int64_t* idx;
    const void* t;
    const float* w;
    float* loss;
    void* g;
    int64_t z_ld, g_ld;
    int N, V, k;
    float inv_tau, tau, grad_scale;
};

// Exponents are kept in base 2: with to2 = log2(e) / tau and c = RN(m to2), m
// the row's maximum, an entry's is fma(z, to2, -c): one rounding of a small
// number.  The rounding of c itself cancels between an entry and the sum.

template <typename OP>
__device__ __forceinline__ float block_all(float x, float* red, OP op) {
#pragma unroll
    for (int d = 32; d; d >>= 1) x = op(x, __shfl_xor(x, d));
    __syncthreads();
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = x;
    __syncthreads();
    x = red[0];
    for (int i = 1; i < kWaves; ++i) x = op(x, red[i]);
    return x;
}
struct Max { __device__ float operator()(float a, float b) const { return fmaxf(a, b); } };
struct Sum { __device__ float operator()(float a, float b) const { return a + b; } };

template <int FZ, int FT, int FG>
__global__ __launch_bounds__(kThreads) void distill_kernel(DistillArgs a) {
    __shared__ float red[kWaves];
    __shared__ float q[kMaxTop];
    __shared__ float zt[kMaxTop];
    const int n = blockIdx.x, tid = threadIdx.x;
    const fmt_t<FZ>* z = static_cast<const fmt_t<FZ>*>(a.z) + (int64_t)n * a.z_ld;
    const fmt_t<FT>* t = static_cast<const fmt_t<FT>*>(a.t) + (int64_t)n * a.k;
    const int64_t* idx = a.idx + (int64_t)n * a.k;
    fmt_t<FG>* g = a.g ? static_cast<fmt_t<FG>*>(a.g) + (int64_t)n * a.g_ld : nullptr;
    const float w = a.w ? a.w[n] : 1.0f;
    const float to2 = a.inv_tau * kLog2e;
    auto used = [&](int i) { return idx[i] >= 0 && idx[i] < a.V; };

    float mt = -INFINITY;
    for (int i = tid; i < a.k; i += kThreads)
        if (used(i)) mt = fmaxf(mt, fmt_value<FT>(t[i]));
    mt = block_all(mt, red, Max());
    if (w == 0.0f || mt == -INFINITY) {
        if (tid == 0 && a.loss) a.loss[n] = 0.0f;
        if (g)
            for (int v = tid; v < a.V; v += kThreads) g[v] = 0;
        return;
    }
    const float ct = mt * to2;
    float st = 0.0f;
    for (int i = tid; i < a.k; i += kThreads)
        if (used(i)) st += exp2f(__builtin_fmaf(fmt_value<FT>(t[i]), to2, -ct));
    const float log_st = log2f(block_all(st, red, Sum()));

    float m = -INFINITY;
    for (int v = tid; v < a.V; v += kThreads) m = fmaxf(m, fmt_value<FZ>(z[v]));
    const float c = block_all(m, red, Max()) * to2;
    float s = 0.0f;
    for (int v = tid; v < a.V; v += kThreads)
        s += exp2f(__builtin_fmaf(fmt_value<FZ>(z[v]), to2, -c));
    s = block_all(s, red, Sum());
    const float log_s = log2f(s);

    float kl = 0.0f;
    for (int i = tid; i < a.k; i += kThreads) {
        float qi = 0.0f, xi = 0.0f;
        if (used(i)) {
            const float lq = __builtin_fmaf(fmt_value<FT>(t[i]), to2, -ct) - log_st;
            qi = exp2f(lq);
            xi = __builtin_fmaf(fmt_value<FZ>(z[idx[i]]), to2, -c);
            if (qi != 0.0f) kl += qi * (lq - (xi - log_s));
        }
        q[i] = qi;
        zt[i] = xi;
    }
    kl = block_all(kl, red, Sum());
    if (tid == 0 && a.loss) a.loss[n] = w * (a.tau * a.tau) * (kl * kLn2);
    if (!g) return;
    const float f = w * (a.tau * a.grad_scale), inv = 1.0f / s;
    for (int v = tid; v < a.V; v += kThreads)
        g[v] = fmt_code<FG>(f * (exp2f(__builtin_fmaf(fmt_value<FZ>(z[v]), to2, -c)) * inv));
    __syncthreads();
    // the teacher's entries again, each with the sum of its occurrences,
    // written by the first of them
    for (int i = tid; i < a.k; i += kThreads) {
        const int64_t v = idx[i];
        if (v < 0 || v >= a.V) continue;
        float sum = 0.0f;
        bool first = true;
        for (int j = 0; j < a.k; ++j)
            if (idx[j] == v) {
                first &= j >= i;
                sum += q[j];
            }
        if (first) g[v] = fmt_code<FG>(f * (exp2f(zt[i]) * inv - sum));
    }
}

template <int FZ, int FT>
void launch(const DistillArgs& a, int g_format, hipStream_t stream) {
    const dim3 grid((unsigned)a.N), block(kThreads);
    if (g_format == FP8T_FMT_F32)
        hipLaunchKernelGGL((distill_kernel<FZ, FT, FP8T_FMT_F32>), grid, block, 0, stream, a);
    else if (g_format == FP8T_FMT_FP16)
        hipLaunchKernelGGL((distill_kernel<FZ, FT, FP8T_FMT_FP16>), grid, block, 0, stream, a);
    else
        hipLaunchKernelGGL((distill_kernel<FZ, FT, FP8T_FMT_FP8>), grid, block, 0, stream, a);
}

}  // namespace
}  // namespace fp8t

using namespace fp8t;

extern "C" int distill_loss(const void* z, int z_format, int64_t z_ld, const int64_t* idx,
                            const void* t, int t_format, int64_t k, const float* w, int64_t N,
                            int64_t V, float tau, float grad_scale, float* loss, void* g,
                            int g_format, int64_t g_ld, hipStream_t stream) {
    if (N < 0 || V < 0 || k < 0 || k > kMaxTop || N > kMaxGemmDim || V > kMaxGemmDim)
        return FP8T_EINVAL;
    if (z_format != FP8T_FMT_F32 && z_format != FP8T_FMT_FP16) return FP8T_EINVAL;
    if (t_format != FP8T_FMT_F32 && t_format != FP8T_FMT_FP16) return FP8T_EINVAL;
    if (g_format < FP8T_FMT_F32 || g_format > FP8T_FMT_FP8) return FP8T_EINVAL;
    if (!(tau > 0.0f) || !(tau <= 3.4e38f)) return FP8T_EINVAL;
    if (N == 0) return FP8T_OK;
    if (!loss && !g) return FP8T_EINVAL;
    if ((V > 0 && (!z || z_ld < V || (g && g_ld < V))) || (k > 0 && (!idx || !t)))
        return FP8T_EINVAL;
    DistillArgs a;
    a.z = z;
    a.idx = idx;
    a.t = t;
    a.w = w;
    a.loss = loss;
    a.g = g;
    a.z_ld = z_ld;
    a.g_ld = g_ld;
    a.N = (int)N;
    a.V = (int)V;
    a.k = (int)k;
    a.tau = tau;
    a.inv_tau = 1.0f / tau;
    a.grad_scale = grad_scale;
    if (z_format == FP8T_FMT_F32) {
        if (t_format == FP8T_FMT_F32) launch<FP8T_FMT_F32, FP8T_FMT_F32>(a, g_format, stream);
        else launch<FP8T_FMT_F32, FP8T_FMT_FP16>(a, g_format, stream);
    } else {
        if (t_format == FP8T_FMT_F32) launch<FP8T_FMT_FP16, FP8T_FMT_F32>(a, g_format, stream);
        else launch<FP8T_FMT_FP16, FP8T_FMT_FP16>(a, g_format, stream);
    }
    return launch_status();
}
