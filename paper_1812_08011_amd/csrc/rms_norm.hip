// rms_norm_fwd: a residual sum and its root-mean-square norm, in one pass.
//
// HBM-bound.  T threads own a row and keep it in registers, NV times eight
// elements each, between the sum of squares and the result: every element is
// read once and written once.  T is the fewest threads that hold a row (8 for 64
// columns: 100000 x 64 FP16 in 11 us, with a wave a row 84).  Rows wider than
// kWidest are read again.
//
// 16384 x 4096, FP16 + floats to floats and FP8, each row scaled: 129 us, 5.7 TB/s
// (a copy of 1 GiB runs at 5.6); 8192 x 2048, all of it FP16, to FP8: 27 us, 4.3
// TB/s, the vector ALUs, between the codes and floats, 72% busy.  Rows of x divided
// by their scale: 4 us of the first, 1 of the second.  2048 x 20000, FP16 + floats to
// floats and FP8: 113 us where a copy's rate is 81, the sum's row read again; 134
// with rows scaled, and again; 2048 x 16384 in registers 70 of 66.  One row: 3.8 us,
// a launch.
// The squares (exact), their sum and 1 / rms are doubles, so that rstd is rounded
// once; n is the floats' two products after it, as a program with rstd in hand
// forms it, Inf and NaN included.
#include "row_ops.h"

namespace fp8t {
namespace {

constexpr int64_t kAcross = 1 << 20;   // workgroups along a grid's first dimension
constexpr int64_t kWidest = 1024 * 16;

struct NormArgs {
    const void* x;
    const float* x_row_scale;
    const void* r;
    const void* w;
    void* h;
    void* y;
    float* y_row_scale;
    float* rstd;
    int64_t x_ld, r_ld, h_ld, y_ld, T, W;
    double inv_W;
    int w_format, y_format;
    bool sum;                          // u is rounded to the stream's format
    bool stream_h, stream_y;           // results past the caches
    float eps, y_scale;
};

// 1 / sqrt(x), x > 0, to 2^-51 of itself: the hardware's estimate and two steps of
// Newton's method (r += r e / 2, e = 1 - x r^2), which square its error each.  An
// Inf gives 0.
__device__ __forceinline__ double inverse_sqrt(double x) {
    double r = __builtin_amdgcn_rsq(x);
    if (r == 0.0) return r;
#pragma unroll
    for (int i = 0; i < 2; ++i) r = __builtin_fma(0.5 * r, __builtin_fma(-x * r, r, 1.0), r);
    return r;
}
__device__ __forceinline__ float row_scale(float top, float y_scale) {
    return top > 0.0f && top < INFINITY ? fminf(y_scale / top, 0x1p126f) : 1.0f;
}

template <int FX, int FS>
struct NormRow {
    static constexpr bool kFours = FX == FP8T_FMT_F32 || FS == FP8T_FMT_F32;
    using C = Cols<kFours>;
    const NormArgs& a;
    const fmt_t<FX>* x;
    const fmt_t<FS>* r;
    fmt_t<FS>* h;
    float div;
    __device__ __forceinline__ NormRow(const NormArgs& a_, int64_t t) : a(a_) {
        x = static_cast<const fmt_t<FX>*>(a.x) + t * a.x_ld;
        r = a.r ? static_cast<const fmt_t<FS>*>(a.r) + t * a.r_ld : nullptr;
        h = a.h ? static_cast<fmt_t<FS>*>(a.h) + t * a.h_ld : nullptr;
        div = a.x_row_scale ? a.x_row_scale[t] : 1.0f;
    }
    // u of elements c .. c + 7 from what was loaded; written to h
    __device__ __forceinline__ void sum(const Eight<FX>& ex, const Eight<FS>& er, const C& c, float* u) const {
        values8<FX>(ex, u);
        if (a.x_row_scale) {
#pragma unroll
            for (int i = 0; i < 8; ++i) u[i] = c.has(i, a.W) ? u[i] / div : 0.0f;
        }
        if (r) {
            float v[8];
            values8<FS>(er, v);
#pragma unroll
            for (int i = 0; i < 8; ++i) u[i] += v[i];
        }
        if (a.sum) {
            const Eight<FS> e = rounded8<FS>(u);
            if (h && c.any(a.W)) store8<FS>(h, c, a.W, e, a.stream_h);
        }
    }
    __device__ __forceinline__ Eight<FS> residual(const C& c) const {
        return r ? load8<FS>(r, c, a.W) : Eight<FS>{};
    }
};

// NV = 0: a row wider than the registers, read again for each of its sums.
template <int FX, int FS, int T, int NV>
__global__ __launch_bounds__(T < 256 ? 256 : T) void rms_norm_kernel(NormArgs a) {
    constexpr int kRows = T < 256 ? 256 / T : 1;            // rows of a workgroup
    __shared__ double sums[T < 256 ? 1 : T / 64];
    __shared__ float red[T < 256 ? 1 : T / 64];
    const int tid = threadIdx.x % T;
    const int64_t t = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * kRows + threadIdx.x / T;
    if (t >= a.T) return;                                   // all threads of a row
    const NormRow<FX, FS> row(a, t);
    using C = typename NormRow<FX, FS>::C;
    const int64_t units = (a.W + 8 * T - 1) / (8 * T);      // of a wide row
    float u[NV ? NV : 1][8], w[NV ? NV : 1][8];
    double ss = 0.0;                                        // squares of floats are exact, and finite
    auto square = [&](const float* v) {
#pragma unroll
        for (int i = 0; i < 8; ++i) ss = __builtin_fma((double)v[i], (double)v[i], ss);
    };
    if constexpr (NV > 0) {
        Eight<FX> ex[NV];
        Eight<FS> er[NV];
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const C c(v, tid, T);
            ex[v] = Eight<FX>{};
            er[v] = Eight<FS>{};
            if (c.any(a.W)) {
                ex[v] = load8<FX>(row.x, c, a.W);
                er[v] = row.residual(c);
            }
        }
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const C c(v, tid, T);
#pragma unroll
            for (int i = 0; i < 8; ++i) w[v][i] = 1.0f;
            if (a.w && c.any(a.W)) load_values8(a.w, a.w_format, c, a.W, w[v]);
        }
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const C c(v, tid, T);
            row.sum(ex[v], er[v], c, u[v]);                 // 0 past the row's end
            square(u[v]);
        }
    } else {
        for (int64_t v = 0; v < units; ++v) {
            const C c(v, tid, T);
            if (!c.any(a.W)) break;
            row.sum(load8<FX>(row.x, c, a.W), row.residual(c), c, u[0]);
            square(u[0]);
        }
    }
    // u of a wide row once more: h may have taken r's or x's place
    auto reload = [&](const C& c, float* v) {
        if (row.h) values8<FS>(load8<FS>(row.h, c, a.W), v);
        else row.sum(load8<FX>(row.x, c, a.W), row.residual(c), c, v);
    };
    const float rstd = (float)inverse_sqrt(row_reduce<T>(ss, sums, RowSum()) * a.inv_W + (double)a.eps);
    if (a.rstd && tid == 0) a.rstd[t] = rstd;
    if (!a.y) return;
    float scale = a.y_scale;
    auto norm = [&](float* v, const float* wv) {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = v[i] * rstd * wv[i];
    };
    auto weights = [&](const C& c, float* wv) {
#pragma unroll
        for (int i = 0; i < 8; ++i) wv[i] = 1.0f;
        if (a.w) load_values8(a.w, a.w_format, c, a.W, wv);
    };
    if constexpr (NV > 0) {
#pragma unroll
        for (int v = 0; v < NV; ++v) norm(u[v], w[v]);
    }
    if (a.y_row_scale) {
        float top = 0.0f;
        auto most = [&](const float* v) {
#pragma unroll
            for (int i = 0; i < 8; i += 2) top = maximum3_abs(top, v[i], v[i + 1]);
        };
        if constexpr (NV > 0) {
#pragma unroll
            for (int v = 0; v < NV; ++v) most(u[v]);
        } else {
            for (int64_t v = 0; v < units; ++v) {
                const C c(v, tid, T);
                if (!c.any(a.W)) break;
                reload(c, u[0]);
                weights(c, w[0]);
                norm(u[0], w[0]);
                most(u[0]);
            }
        }
        scale = row_scale(row_reduce<T>(top, red, RowMax()), a.y_scale);
        if (tid == 0) a.y_row_scale[t] = scale;
    }
    uint8_t* y = static_cast<uint8_t*>(a.y) +
                 t * a.y_ld * (a.y_format == FP8T_FMT_F32 ? 4 : a.y_format == FP8T_FMT_FP16 ? 2 : 1);
    auto out = [&](const C& c, float* v) {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] *= scale;
        put_as8(y, a.y_format, c, a.W, v, a.stream_y);
    };
    if constexpr (NV > 0) {
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const C c(v, tid, T);
            if (c.any(a.W)) out(c, u[v]);
        }
    } else {
        for (int64_t v = 0; v < units; ++v) {
            const C c(v, tid, T);
            if (!c.any(a.W)) break;
            reload(c, u[0]);
            weights(c, w[0]);
            norm(u[0], w[0]);
            out(c, u[0]);
        }
    }
}

template <int FX, int FS, int T, int NV>
void launch_rows(const NormArgs& a, hipStream_t stream) {
    constexpr int kRows = T < 256 ? 256 / T : 1;
    const int64_t n = (a.T + kRows - 1) / kRows, across = n < kAcross ? n : kAcross;
    hipLaunchKernelGGL((rms_norm_kernel<FX, FS, T, NV>),
                       dim3((unsigned)across, (unsigned)((n + across - 1) / across)), dim3(T < 256 ? 256 : T), 0,
                       stream, a);
}

template <int FX, int FS>
void launch(const NormArgs& a, hipStream_t stream) {
    if (a.W <= 8 * 8) launch_rows<FX, FS, 8, 1>(a, stream);
    else if (a.W <= 16 * 8) launch_rows<FX, FS, 16, 1>(a, stream);
    else if (a.W <= 32 * 8) launch_rows<FX, FS, 32, 1>(a, stream);
    else if (a.W <= 64 * 8) launch_rows<FX, FS, 64, 1>(a, stream);
    else if (a.W <= 64 * 16) launch_rows<FX, FS, 64, 2>(a, stream);
    else if (a.W <= 256 * 8) launch_rows<FX, FS, 256, 1>(a, stream);
    else if (a.W <= 256 * 16) launch_rows<FX, FS, 256, 2>(a, stream);
    else if (a.W <= 1024 * 8) launch_rows<FX, FS, 1024, 1>(a, stream);
    else if (a.W <= kWidest) launch_rows<FX, FS, 1024, 2>(a, stream);
    else launch_rows<FX, FS, 1024, 0>(a, stream);
}

}  // namespace
}  // namespace fp8t

using namespace fp8t;

extern "C" int rms_norm_fwd(const void* x, int x_format, int64_t x_ld, const float* x_row_scale,
                            const void* r, int64_t r_ld, const void* w, int w_format, int64_t T,
                            int64_t W, float eps, void* h, int s_format, int64_t h_ld, void* y,
                            int y_format, int64_t y_ld, float y_scale, float* y_row_scale,
                            float* rstd, hipStream_t stream) {
    if (T < 0 || W < 0 || T > kMaxGemmDim || W > FP8T_MAX_NORM_W || !float_or_16(x_format) ||
        !float_or_16(s_format) || !float_or_16(w_format) || !storage_format(y_format) ||
        !(eps >= 0x1p-100f) || !(eps <= 0x1p100f))
        return FP8T_EINVAL;
    if (T == 0 || W == 0) return FP8T_OK;
    if ((!h && !y && !rstd) || !matrix_ok(x, x_ld, T, W) || (r && r_ld < W) || (h && h_ld < W) ||
        (y && y_ld < W))
        return FP8T_EINVAL;
    if (y_row_scale && (!y || !(y_scale > 0.0f) || !(y_scale <= 3.4028234e38f))) return FP8T_EINVAL;
    NormArgs a;
    a.x = x;
    a.x_row_scale = x_row_scale;
    a.r = r;
    a.w = w;
    a.h = h;
    a.y = y;
    a.y_row_scale = y_row_scale;
    a.rstd = rstd;
    a.x_ld = x_ld;
    a.r_ld = r_ld;
    a.h_ld = h_ld;
    a.y_ld = y_ld;
    a.T = T;
    a.W = W;
    a.inv_W = 1.0 / (double)W;
    a.w_format = w_format;
    a.y_format = y_format;
    a.sum = r || h;
    a.stream_h = W <= kWidest && T * W * bytes_of(s_format) > kStreamBytes;   // wide rows are read again
    a.stream_y = T * W * bytes_of(y_format) > kStreamBytes;
    a.eps = eps;
    a.y_scale = y_scale;
    const bool f32 = s_format == FP8T_FMT_F32;
    if (x_format == FP8T_FMT_F32) {
        if (f32) launch<FP8T_FMT_F32, FP8T_FMT_F32>(a, stream);
        else launch<FP8T_FMT_F32, FP8T_FMT_FP16>(a, stream);
    } else {
        if (f32) launch<FP8T_FMT_FP16, FP8T_FMT_F32>(a, stream);
        else launch<FP8T_FMT_FP16, FP8T_FMT_FP16>(a, stream);
    }
    return launch_status();
}
