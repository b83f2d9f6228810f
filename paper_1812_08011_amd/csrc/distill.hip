// distill_loss: Kullback-Leibler loss against a teacher's top logits and the
// gradient of the student's logits.  One workgroup per row.
//
// HBM-bound: every logit is read once from memory and every gradient written
// once.  Between the two, floats stay in registers (rows of 65536 at most)
// where the memory would have to give them again: 4096 x 32768 floats take
// 207 us, read twice 277 us.  FP16 logits are read a second time, from the
// caches: a first pass that takes maximum and sum together decodes a logit once
// more instead of twice more, and a row in flight costs no registers, so a CU
// works on more rows: 4096 x 32768 in 143 us (4 bytes a logit, 3.8 TB/s), from
// registers 159 us; 2048 x 50001, rows at odd addresses, 123 and 189 us.
// exp(z / tau - max) is taken twice, for the sum and for the gradient.
#include "lm_formats.h"

namespace fp8t {
namespace {

constexpr int kMaxTop = 4096;
constexpr int64_t kAcross = 1 << 20;   // rows along a grid's first dimension
constexpr int64_t kMaxV = INT32_MAX - 16384;   // a thread's positions stay in 32 bits
constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kLn2 = 0.69314718055994530942f;

struct DistillArgs {
    const void* z;
    const int64_t* idx;
    const void* t;
    const float* w;
    float* loss;
    void* g;
    int64_t z_ld, g_ld, N;
    int V, k, t_format;
    float to2, tau, grad_scale;        // to2 = log2(e) / tau
};

// An entry's exponent is that of its distance from the row's maximum m, in base
// 2: (x - m) to2.  The distance is exact or off by 2^-24 of itself, whatever m
// is -- x to2 - m to2 would overflow, or lose the distance, where every logit of
// a row is a mask's.
__device__ __forceinline__ float exponent(float x, float m, float to2) { return (x - m) * to2; }

// Two reductions at once over the workgroup's T threads.
template <int T, typename OP>
__device__ __forceinline__ float2 block_both(float2 x, float2* red, OP op) {
#pragma unroll
    for (int d = 32; d; d >>= 1) {
        x.x = op(x.x, __shfl_xor(x.x, d));
        x.y = op(x.y, __shfl_xor(x.y, d));
    }
    __syncthreads();
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = x;
    __syncthreads();
    x = red[0];
#pragma unroll
    for (int i = 1; i < T / 64; ++i) x = make_float2(op(x.x, red[i].x), op(x.y, red[i].y));
    return x;
}
// NaN wins: a row with one is NaN throughout.
struct Max {
    __device__ float operator()(float a, float b) const { return a > b || a != a ? a : b; }
};
struct Sum {
    __device__ float operator()(float a, float b) const { return a + b; }
};

// Elements v .. v + 7 of a row of V as they are stored (-Inf past its end), and
// their values.
template <int FMT>
__device__ __forceinline__ Eight<FMT> load_eight(const fmt_t<FMT>* row, int v, int V) {
    if (v + 8 <= V) return *reinterpret_cast<const Eight<FMT>*>(row + v);
    Eight<FMT> e;
    if constexpr (FMT == FP8T_FMT_F32) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            e.a[i] = v + i < V ? row[v + i] : -INFINITY;
            e.b[i] = v + 4 + i < V ? row[v + 4 + i] : -INFINITY;
        }
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) e.a[i] = 0xFE00FE00u;
        if (v < V) {
#pragma unroll
            for (int i = 0; i < 7; ++i)
                if (v + i < V)
                    e.a[i / 2] = (e.a[i / 2] & ~(0xFFFFu << (16 * (i % 2)))) |
                                 ((uint32_t)row[v + i] << (16 * (i % 2)));
        }
    }
    return e;
}
// The same of a result; `plain`: |x| is finite and no format's overflow.
template <int FMT>
__device__ __forceinline__ void store_eight(fmt_t<FMT>* row, int v, int V, const float* x, bool plain) {
    if (v + 8 <= V && plain) {
        Eight<FMT> e;
        if constexpr (FMT == FP8T_FMT_F32) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                e.a[i] = x[i];
                e.b[i] = x[4 + i];
            }
        } else if constexpr (FMT == FP8T_FMT_FP16) {
#pragma unroll
            for (int i = 0; i < 4; ++i) e.a[i] = fp16_pair(x[2 * i], x[2 * i + 1]);
        } else {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                uint32_t w = __builtin_amdgcn_cvt_pk_bf8_f32(x[4 * i], x[4 * i + 1], 0, false);
                e.a[i] = __builtin_amdgcn_cvt_pk_bf8_f32(x[4 * i + 2], x[4 * i + 3], w, true);
            }
        }
        *reinterpret_cast<Eight<FMT>*>(row + v) = e;
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (v + i < V) row[v + i] = fmt_code<FMT>(x[i]);
    }
}

// T threads, NV times eight elements each kept in registers; NV = 0: the row is
// read a second time.
template <int FZ, int FG, int T, int NV>
__global__ __launch_bounds__(T, T / 256) void distill_kernel(DistillArgs a) {
    extern __shared__ float top[];                          // [k] entries, their q, their exponents
    __shared__ float2 red[T / 64];
    int* at = reinterpret_cast<int*>(top);
    float* q = top + a.k;
    float* xt = q + a.k;
    const int64_t n = (int64_t)blockIdx.y * gridDim.x + blockIdx.x;
    if (n >= a.N) return;
    const int tid = threadIdx.x;
    const fmt_t<FZ>* z = static_cast<const fmt_t<FZ>*>(a.z) + n * a.z_ld;
    fmt_t<FG>* g = a.g ? static_cast<fmt_t<FG>*>(a.g) + n * a.g_ld : nullptr;
    const float w = a.w ? a.w[n] : 1.0f, to2 = a.to2;

    // the row's logits on their way, the teacher's used entries and the
    // student's logits there
    Eight<FZ> raw[NV ? NV : 1];
#pragma unroll
    for (int i = 0; i < NV; ++i) raw[i] = load_eight<FZ>(z, (i * T + tid) * 8, a.V);
    float2 m = make_float2(-INFINITY, -INFINITY);           // of z and of the teacher's
    for (int i = tid; i < a.k; i += T) {
        const int64_t v = a.idx[n * a.k + i];
        const bool used = v >= 0 && v < a.V;
        at[i] = used ? (int)v : -1;
        if (!used) continue;
        const float t = a.t_format == FP8T_FMT_F32
                            ? static_cast<const float*>(a.t)[n * a.k + i]
                            : fp16_to_f32(static_cast<const uint16_t*>(a.t)[n * a.k + i]);
        q[i] = t;
        xt[i] = fmt_value<FZ>(z[v]);
        m.y = Max()(m.y, t);
    }
    float s = 0.0f;                                         // NV = 0: of this thread, relative to m.x
    bool special = false;                                   // an Inf or NaN among this thread's
    if constexpr (NV > 0) {
#pragma unroll
        for (int i = 0; i < NV; ++i)
            if ((i * T + tid) * 8 < a.V) special |= special_in<FZ>(raw[i]);
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            if ((i * T + tid) * 8 >= a.V) continue;
            float x[8];
            values_of<FZ>(raw[i], special, x);
#pragma unroll
            for (int j = 0; j < 8; ++j) m.x = fmaxf(m.x, x[j]);   // a NaN comes with the sum
        }
    } else {
        for (int v = tid * 8; v < a.V; v += T * 8) {
            const Eight<FZ> e = load_eight<FZ>(z, v, a.V);
            float x[8];
            values_of<FZ>(e, special_in<FZ>(e), x);
            float top8 = x[0];
#pragma unroll
            for (int i = 1; i < 8; ++i) top8 = fmaxf(top8, x[i]);
            if (!(top8 <= m.x)) {
                if (m.x != -INFINITY) s *= exp2f(exponent(m.x, top8, to2));
                m.x = top8;
            }
            const float c = m.x == -INFINITY ? 0.0f : m.x;
#pragma unroll
            for (int i = 0; i < 8; ++i) s += __builtin_amdgcn_exp2f(exponent(x[i], c, to2));
        }
    }
    const float own = m.x;
    m = block_both<T>(m, red, Max());
    if (w == 0.0f || m.y == -INFINITY) {
        if (tid == 0 && a.loss) a.loss[n] = 0.0f;
        if (g) {
            const float none[8] = {0, 0, 0, 0, 0, 0, 0, 0};
            for (int v = tid * 8; v < a.V; v += T * 8) store_eight<FG>(g, v, a.V, none, true);
        }
        return;
    }
    float2 sum = make_float2(0.0f, 0.0f);
    if constexpr (NV > 0) {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            if ((i * T + tid) * 8 >= a.V) continue;
            float x[8];
            values_of<FZ>(raw[i], special, x);
#pragma unroll
            for (int j = 0; j < 8; ++j) sum.x += __builtin_amdgcn_exp2f(exponent(x[j], m.x, to2));
        }
    } else {
        if (own == own && own != -INFINITY) s *= exp2f(exponent(own, m.x, to2));
        sum.x = m.x == -INFINITY || m.x != m.x ? NAN : s;
    }
    for (int i = tid; i < a.k; i += T)
        if (at[i] >= 0) sum.y += exp2f(exponent(q[i], m.y, to2));
    sum = block_both<T>(sum, red, Sum());
    const float log_s = log2f(sum.x), log_st = log2f(sum.y), inv = 1.0f / sum.x;

    // the loss's terms in natural logarithms: a target on a logit at the type's
    // lowest value has a finite one
    float2 kl = make_float2(0.0f, 0.0f);
    for (int i = tid; i < a.k; i += T) {
        float qi = 0.0f, pi = 0.0f;
        if (at[i] >= 0) {
            const float lq = exponent(q[i], m.y, to2) - log_st;
            qi = exp2f(lq);
            pi = exp2f(exponent(xt[i], m.x, to2)) * inv;
            if (qi != 0.0f) kl.x += qi * ((lq + log_s) * kLn2 - (xt[i] - m.x) / a.tau);
        }
        q[i] = qi;
        xt[i] = pi;
    }
    kl = block_both<T>(kl, red, Sum());
    if (tid == 0 && a.loss) a.loss[n] = w * (a.tau * a.tau) * kl.x;
    if (!g) return;
    const float f = w * (a.tau * a.grad_scale), fi = f * inv;
    // every |g| is at most |f|
    const bool plain = FG == FP8T_FMT_F32 ||
                       (__builtin_fabsf(fi) < INFINITY &&
                        __builtin_fabsf(f) <= (FG == FP8T_FMT_FP8 ? 57344.0f : 0x1p31f));
    // the teacher's entries, each with the sum of its occurrences, written by
    // the first of them -- after the others, below
    auto corrected = [&](int i, int v, bool& first) {
        float both = 0.0f;
        first = true;
#pragma unroll 8
        for (int j = 0; j < a.k; ++j)
            if (at[j] == v) {
                first &= j >= i;
                both += q[j];
            }
        return f * (xt[i] - both);
    };
    const int v0 = tid < a.k ? at[tid] : -1;
    bool mine = false;
    const float y0 = v0 >= 0 ? corrected(tid, v0, mine) : 0.0f;
    auto gradient = [&](const Eight<FZ>& e, bool odd, int v) {
        float x[8];
        values_of<FZ>(e, odd, x);
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = __builtin_amdgcn_exp2f(exponent(x[j], m.x, to2)) * fi;
        store_eight<FG>(g, v, a.V, x, plain);
    };
    if constexpr (NV > 0) {
#pragma unroll
        for (int i = 0; i < NV; ++i)
            if ((i * T + tid) * 8 < a.V) gradient(raw[i], special, (i * T + tid) * 8);
    } else {
        for (int v = tid * 8; v < a.V; v += T * 8) {
            const Eight<FZ> e = load_eight<FZ>(z, v, a.V);
            gradient(e, special_in<FZ>(e), v);
        }
    }
    __syncthreads();
    if (mine) g[v0] = fmt_code<FG>(y0);
    for (int i = tid + T; i < a.k; i += T) {
        const int v = at[i];
        bool first = false;
        const float y = v >= 0 ? corrected(i, v, first) : 0.0f;
        if (first) g[v] = fmt_code<FG>(y);
    }
}

template <int FZ, int FG, int T, int NV>
void launch_rows(const DistillArgs& a, hipStream_t stream) {
    const size_t lds = 3 * sizeof(float) * (size_t)a.k;
    const int64_t across = a.N < kAcross ? a.N : kAcross;
    const dim3 grid((unsigned)across, (unsigned)((a.N + across - 1) / across));
    hipLaunchKernelGGL((distill_kernel<FZ, FG, T, NV>), grid, dim3(T), lds, stream, a);
}

template <int FZ, int FG>
void launch(const DistillArgs& a, hipStream_t stream) {
    // FP16: threads by the work of a row.  4096 x 10000: 44 us with 256, 51 with
    // 512; 4096 x 32768: 160 and 143; 512 x 300000: 200 with 512, 188 with 1024.
    // Floats: the fewest threads whose registers (64 for the row at most) hold
    // it, as the waits at a row's sums cost more with more waves (4096 x 6000:
    // 39 us with 256, 61 with 1024); then a second reading.
    if constexpr (FZ == FP8T_FMT_FP16) {
        if (a.V <= 12288) launch_rows<FZ, FG, 256, 0>(a, stream);
        else if (a.V <= 65536) launch_rows<FZ, FG, 512, 0>(a, stream);
        else launch_rows<FZ, FG, 1024, 0>(a, stream);
    } else {
        if (a.V <= 256 * 8) launch_rows<FZ, FG, 256, 1>(a, stream);
        else if (a.V <= 256 * 32) launch_rows<FZ, FG, 256, 4>(a, stream);
        else if (a.V <= 256 * 64) launch_rows<FZ, FG, 256, 8>(a, stream);
        else if (a.V <= 512 * 64) launch_rows<FZ, FG, 512, 8>(a, stream);
        else if (a.V <= 1024 * 64) launch_rows<FZ, FG, 1024, 8>(a, stream);
        else launch_rows<FZ, FG, 1024, 0>(a, stream);
    }
}

}  // namespace
}  // namespace fp8t

using namespace fp8t;

extern "C" int distill_loss(const void* z, int z_format, int64_t z_ld, const int64_t* idx,
                            const void* t, int t_format, int64_t k, const float* w, int64_t N,
                            int64_t V, float tau, float grad_scale, float* loss, void* g,
                            int g_format, int64_t g_ld, hipStream_t stream) {
    if (N < 0 || V < 0 || k < 0 || k > kMaxTop || N > kMaxGemmDim || V > kMaxV)
        return FP8T_EINVAL;
    if (z_format != FP8T_FMT_F32 && z_format != FP8T_FMT_FP16) return FP8T_EINVAL;
    if (t_format != FP8T_FMT_F32 && t_format != FP8T_FMT_FP16) return FP8T_EINVAL;
    if (g_format < FP8T_FMT_F32 || g_format > FP8T_FMT_FP8) return FP8T_EINVAL;
    if (!(tau >= 0x1p-30f) || !(tau <= 0x1p30f)) return FP8T_EINVAL;
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
    a.N = N;
    a.V = (int)V;
    a.k = (int)k;
    a.t_format = t_format;
    a.tau = tau;
    a.to2 = kLog2e / tau;
    a.grad_scale = grad_scale;
    if (z_format == FP8T_FMT_F32) {
        if (g_format == FP8T_FMT_F32) launch<FP8T_FMT_F32, FP8T_FMT_F32>(a, stream);
        else if (g_format == FP8T_FMT_FP16) launch<FP8T_FMT_F32, FP8T_FMT_FP16>(a, stream);
        else launch<FP8T_FMT_F32, FP8T_FMT_FP8>(a, stream);
    } else {
        if (g_format == FP8T_FMT_F32) launch<FP8T_FMT_FP16, FP8T_FMT_F32>(a, stream);
        else if (g_format == FP8T_FMT_FP16) launch<FP8T_FMT_FP16, FP8T_FMT_FP16>(a, stream);
        else launch<FP8T_FMT_FP16, FP8T_FMT_FP8>(a, stream);
    }
    return launch_status();
}
