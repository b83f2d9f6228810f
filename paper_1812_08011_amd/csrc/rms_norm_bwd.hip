// rms_norm_bwd: gradients of the root-mean-square norm.
//
// HBM-bound, one pass.  A workgroup owns a range of rows; the T threads of a
// row keep it in registers, eight elements each, between the mean and the
// gradient, with the next row on its way, and their columns' sums of dw over the
// rows.  Those go to the workspace, one row of sums for each workgroup, and a
// second kernel adds them in order.  The sums and the mean's are doubles of float
// products, a workgroup's dw is stored as floats: the conversions and additions hide
// behind the stream (1 us of the 16 below).
// Rows wider than 8192 are twice eight elements a thread without a row ahead and
// with the sums in LDS (no registers are left), those wider than kWidest are read
// twice, and dw has a kernel of its own.
//
// 8192 x 4096 floats with FP16 errors, to floats and FP8: 98 us and 5 for the
// join, 5.1 TB/s (a copy of 1 GiB runs at 5.6); twice eight elements in 256 threads, 155
// registers, and no row ahead: 109 and 7.  5003 x 1001 in FP16: 16 us and 5, three
// rows for each group of threads one after the other, 2 TB/s.  2048 x 16384: 109 us
// where a copy's rate is 91; 2048 x 20000: 136 and 56 for dw, of 111.
#include "row_ops.h"

namespace fp8t {
namespace {

constexpr int64_t kAcross = 1 << 20;
constexpr int64_t kWidest = 1024 * 16;
constexpr int kDwThreads = 256, kJoinThreads = 1024;

struct NormGradArgs {
    const void* h;
    const void* w;
    const float* rstd;
    const void* dy;
    const void* dr;
    void* dx;
    uint8_t* dx8;
    float* parts;                      // workgroups x W (null: no dw)
    int64_t h_ld, dy_ld, dr_ld, dx_ld, dx8_ld, T, W;
    int64_t share, blocks;             // rows of a group of T threads; workgroups
    double inv_W;
    int w_format;
    float dx8_scale;
    bool stream, stream8;              // dx, dx8 past the caches
};

template <int FD, bool FOURS>
__device__ __forceinline__ void put(const NormGradArgs& a, int64_t t, const Cols<FOURS>& c, float* d) {
    if (a.dx) put8<FD>(static_cast<fmt_t<FD>*>(a.dx) + t * a.dx_ld, c, a.W, d, a.stream);
    if (a.dx8) {
#pragma unroll
        for (int i = 0; i < 8; ++i) d[i] *= a.dx8_scale;
        put8<FP8T_FMT_FP8>(a.dx8 + t * a.dx8_ld, c, a.W, d, a.stream8);
    }
}
// Eight terms, two by two: a chain of additions is three long.
template <typename F>
__device__ __forceinline__ double sum8(F term) {
    return ((term(0) + term(1)) + (term(2) + term(3))) + ((term(4) + term(5)) + (term(6) + term(7)));
}
template <int FH, int FY, int FD>
constexpr bool kFours = FH == FP8T_FMT_F32 || FY == FP8T_FMT_F32 || FD == FP8T_FMT_F32;

// What a thread has loaded of a row.
template <int FH, int FY, int FD, int NV>
struct Loaded {
    Eight<FH> h[NV];
    Eight<FY> y[NV];
    Eight<FD> r[NV];
    float rstd;
};

// Threads of a workgroup: several rows' where they are short, so that there are
// fewer rows of partial sums.
template <int T>
constexpr int kRowThreads = T < 512 ? 512 : T;

// T threads of a row; AHEAD: the next row is on its way while one is worked on.
template <int FH, int FY, int FD, int T, int NV, bool AHEAD>
__global__ __launch_bounds__(kRowThreads<T>) void rms_norm_bwd_kernel(NormGradArgs a) {
    constexpr int kThreads = kRowThreads<T>, kGroups = kThreads / T;
    using C = Cols<kFours<FH, FY, FD>>;
    // doubles of twice eight columns would spill 50 bytes a thread: they lie in LDS,
    // 128 of its 160 KB (a workgroup of 1024 threads has a CU's registers anyway),
    // each thread's beside the next one's.  2048 x 16384 floats with FP16 errors 110
    // us, with float sums in registers 112; 2048 x 9000 of FP16, FP8 and FP16 66 and 64
    constexpr bool kInLds = NV > 1;
    __shared__ double wide[kInLds ? NV * 8 : 1][kInLds ? T : 1];
    __shared__ double red[2][kThreads / 64];
    __shared__ double sums[kGroups > 1 ? kGroups : 1][kGroups > 1 ? T * NV * 8 : 1];
    const int tid = threadIdx.x % T, sub = threadIdx.x / T;
    const int64_t t0 = ((int64_t)blockIdx.x * kGroups + sub) * a.share;
    const bool out = a.dx || a.dx8;
    float w[NV][8];
    double dw[kInLds ? 1 : NV][8];
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        const C c(v, tid, T);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            w[v][i] = 1.0f;
            if constexpr (kInLds) wide[v * 8 + i][tid] = 0.0;
            else dw[v][i] = 0.0;
        }
        if (a.w && c.any(a.W)) load_values8(a.w, a.w_format, c, a.W, w[v]);
    }
    auto load = [&](int64_t t, Loaded<FH, FY, FD, NV>& x) {
        // rows past the end, and columns: 0
        x.rstd = t < a.T ? a.rstd[t] : 0.0f;
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const C c(v, tid, T);
            x.h[v] = Eight<FH>{};
            x.y[v] = Eight<FY>{};
            x.r[v] = Eight<FD>{};
            if (c.any(a.W) && t < a.T) {
                x.h[v] = load8<FH>(static_cast<const fmt_t<FH>*>(a.h) + t * a.h_ld, c, a.W);
                x.y[v] = load8<FY>(static_cast<const fmt_t<FY>*>(a.dy) + t * a.dy_ld, c, a.W);
                if (a.dr && out) x.r[v] = load8<FD>(static_cast<const fmt_t<FD>*>(a.dr) + t * a.dr_ld, c, a.W);
            }
        }
    };
    Loaded<FH, FY, FD, NV> next;
    if (AHEAD) load(t0, next);
    for (int64_t i = 0; i < a.share; ++i) {                 // the same number for all groups
        const int64_t t = t0 + i;
        if (!AHEAD) load(t, next);
        float n[NV][8], g[NV][8];
        double dot = 0.0;
        Eight<FD> r[NV];
        const float rstd = next.rstd;
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            values8<FH>(next.h[v], n[v]);
            values8<FY>(next.y[v], g[v]);
            r[v] = next.r[v];
            if (kInLds && a.parts && C(v, tid, T).any(a.W)) {
#pragma unroll
                for (int j = 0; j < 8; ++j) wide[v * 8 + j][tid] += g[v][j] * (n[v][j] * rstd);
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                n[v][j] *= rstd;
                if constexpr (!kInLds) dw[v][j] += g[v][j] * n[v][j];
                g[v][j] *= w[v][j];
            }
            dot += sum8([&](int j) { return (double)(g[v][j] * n[v][j]); });
        }
        if (AHEAD && i + 1 < a.share) load(t + 1, next);
        if (!out) continue;
        const float m = (float)(row_reduce<T>(dot, red[i & 1], RowSum()) * a.inv_W);
        if (t >= a.T) continue;
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const C c(v, tid, T);
            if (!c.any(a.W)) continue;
            float d[8];
            values8<FD>(r[v], d);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float own = rstd * (g[v][j] - n[v][j] * m);
                d[j] = a.dr ? d[j] + own : own;
            }
            put<FD>(a, t, c, d);
        }
    }
    if (!a.parts) return;
    if constexpr (kGroups > 1) {
#pragma unroll
        for (int v = 0; v < NV; ++v)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const C c(v, tid, T);
                sums[sub][i < 4 ? c.a + i : c.b + i - 4] = dw[v][i];
            }
        __syncthreads();
        for (int c = threadIdx.x; c < a.W; c += kThreads) {
            double s = sums[0][c];
#pragma unroll
            for (int g = 1; g < kGroups; ++g) s += sums[g][c];
            a.parts[(int64_t)blockIdx.x * a.W + c] = (float)s;
        }
    } else {
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const C c(v, tid, T);
            float d[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                if constexpr (kInLds) d[i] = (float)wide[v * 8 + i][tid];
                else d[i] = (float)dw[v][i];
            }
            if (c.any(a.W)) put8<FP8T_FMT_F32>(a.parts + (int64_t)blockIdx.x * a.W, c, a.W, d, false);
        }
    }
}

// Wide rows: one row per workgroup, read twice.
template <int FH, int FY, int FD>
__global__ __launch_bounds__(1024) void rms_norm_bwd_wide_kernel(NormGradArgs a) {
    __shared__ double red[16];
    const int64_t t = (int64_t)blockIdx.y * gridDim.x + blockIdx.x;
    if (t >= a.T) return;
    const fmt_t<FH>* h = static_cast<const fmt_t<FH>*>(a.h) + t * a.h_ld;
    const fmt_t<FY>* dy = static_cast<const fmt_t<FY>*>(a.dy) + t * a.dy_ld;
    const fmt_t<FD>* dr = a.dr ? static_cast<const fmt_t<FD>*>(a.dr) + t * a.dr_ld : nullptr;
    const float rstd = a.rstd[t];
    float n[8], g[8], w[8];
    double dot = 0.0;
    using C = Cols<kFours<FH, FY, FD>>;
    const int64_t units = (a.W + 8191) / 8192;
    auto load = [&](const C& c) {
        values8<FH>(load8<FH>(h, c, a.W), n);
        values8<FY>(load8<FY>(dy, c, a.W), g);
#pragma unroll
        for (int i = 0; i < 8; ++i) w[i] = 1.0f;
        if (a.w) load_values8(a.w, a.w_format, c, a.W, w);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            n[i] *= rstd;
            g[i] *= w[i];
        }
    };
    for (int64_t v = 0; v < units; ++v) {
        const C c(v, threadIdx.x, 1024);
        if (!c.any(a.W)) break;
        load(c);
        dot += sum8([&](int i) { return (double)(g[i] * n[i]); });
    }
    const float m = (float)(row_reduce<1024>(dot, red, RowSum()) / (double)a.W);
    for (int64_t v = 0; v < units; ++v) {
        const C c(v, threadIdx.x, 1024);
        if (!c.any(a.W)) break;
        load(c);
        float d[8];
        if (dr) values8<FD>(load8<FD>(dr, c, a.W), d);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float own = rstd * (g[i] - n[i] * m);
            d[i] = dr ? d[i] + own : own;
        }
        put<FD>(a, t, c, d);
    }
}

// dw of wide rows: a thread owns eight columns and a range of rows.
template <int FH, int FY>
__global__ __launch_bounds__(kDwThreads) void rms_norm_dw_kernel(NormGradArgs a) {
    const Cols<FH == FP8T_FMT_F32 || FY == FP8T_FMT_F32> c(blockIdx.x, threadIdx.x, kDwThreads);
    if (!c.any(a.W)) return;
    const int64_t t0 = blockIdx.y * a.share, t1 = t0 + a.share < a.T ? t0 + a.share : a.T;
    double sum[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    for (int64_t t = t0; t < t1; ++t) {
        float n[8], g[8];
        values8<FH>(load8<FH>(static_cast<const fmt_t<FH>*>(a.h) + t * a.h_ld, c, a.W), n);
        values8<FY>(load8<FY>(static_cast<const fmt_t<FY>*>(a.dy) + t * a.dy_ld, c, a.W), g);
        const float rstd = a.rstd[t];
#pragma unroll
        for (int i = 0; i < 8; ++i) sum[i] += g[i] * (n[i] * rstd);
    }
    float d[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) d[i] = (float)sum[i];
    put8<FP8T_FMT_F32>(a.parts + blockIdx.y * a.W, c, a.W, d, false);
}

// dw = the sum of the workgroups' rows: a lane owns a column, each wave a range
// of the rows, in order; the waves' sums are added in order.
__global__ __launch_bounds__(kJoinThreads) void rms_norm_join_kernel(const float* parts, int64_t blocks,
                                                                     int64_t W, void* dw, int dw_format) {
    constexpr int kWaves = kJoinThreads / 64;
    __shared__ double sums[kWaves][64];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int64_t c = (int64_t)blockIdx.x * 64 + lane;
    const int64_t share = (blocks + kWaves - 1) / kWaves;
    const int64_t g0 = wave * share, g1 = g0 + share < blocks ? g0 + share : blocks;
    double sum = 0.0;
    if (c < W) {
        constexpr int kAhead = 16;
        for (int64_t g = g0; g < g1; g += kAhead) {
            float x[kAhead];                // the last row again past the end: no branches between
#pragma unroll
            for (int u = 0; u < kAhead; ++u) x[u] = parts[(g + u < g1 ? g + u : g1 - 1) * W + c];
#pragma unroll
            for (int u = 0; u < kAhead; ++u) sum += g + u < g1 ? x[u] : 0.0f;
        }
    }
    sums[wave][lane] = sum;
    __syncthreads();
    if (wave > 0 || c >= W) return;
    sum = sums[0][lane];
#pragma unroll
    for (int i = 1; i < kWaves; ++i) sum += sums[i][lane];
    if (dw_format == FP8T_FMT_F32) static_cast<float*>(dw)[c] = (float)sum;
    else static_cast<uint16_t*>(dw)[c] = f32_to_fp16_rn((float)sum);
}

// Rows of a group of T threads, and workgroups (rows of partial sums).
struct NormGradPlan {
    int64_t share, blocks;
};
NormGradPlan norm_grad_plan(int64_t T, int64_t W) {
    int64_t threads = 8;                                    // of a row: eight columns each
    while (threads < 1024 && threads * 8 < W) threads *= 2;
    const int64_t groups = threads < 512 ? 512 / threads : 1;
    int64_t cus = device_cus();
    if (cus <= 0) cus = 256;
    // as many as run at a time, but two rows for each group at least.  Wide rows' dw
    // has a workgroup for 2048 columns besides: ranges of rows 32, 64, 128 and 256, in
    // turn, 2048 x 20000 93, 64, 58 and 58 us, 512 x 100000 79, 77, 78 and 85, 512 x
    // 300000 214, 222, 235 and 287 (more partial sums)
    int64_t most = W > kWidest ? 64 : cus * 1024 / (threads * groups) * groups;
    const int64_t pairs = (T + 1) / 2;
    if (most > pairs) most = pairs;
    if (most < 1) most = 1;
    NormGradPlan p;
    p.share = (T + most - 1) / most;
    if (p.share < 1) p.share = 1;
    const int64_t rows = W > kWidest ? p.share : p.share * groups;
    p.blocks = (T + rows - 1) / rows;
    return p;
}

template <int FH, int FY, int FD, int T, int NV>
void launch_rows(const NormGradArgs& a, hipStream_t stream) {
    hipLaunchKernelGGL((rms_norm_bwd_kernel<FH, FY, FD, T, NV, NV == 1>), dim3((unsigned)a.blocks),
                       dim3(kRowThreads<T>), 0, stream, a);
}

template <int FH, int FY, int FD>
void launch(const NormGradArgs& a, hipStream_t stream) {
    if (a.W <= 8 * 8) launch_rows<FH, FY, FD, 8, 1>(a, stream);
    else if (a.W <= 16 * 8) launch_rows<FH, FY, FD, 16, 1>(a, stream);
    else if (a.W <= 32 * 8) launch_rows<FH, FY, FD, 32, 1>(a, stream);
    else if (a.W <= 64 * 8) launch_rows<FH, FY, FD, 64, 1>(a, stream);
    else if (a.W <= 128 * 8) launch_rows<FH, FY, FD, 128, 1>(a, stream);
    else if (a.W <= 256 * 8) launch_rows<FH, FY, FD, 256, 1>(a, stream);
    else if (a.W <= 512 * 8) launch_rows<FH, FY, FD, 512, 1>(a, stream);
    else if (a.W <= 1024 * 8) launch_rows<FH, FY, FD, 1024, 1>(a, stream);
    else if (a.W <= kWidest) launch_rows<FH, FY, FD, 1024, 2>(a, stream);
    else {
        if (a.dx || a.dx8) {
            const int64_t across = a.T < kAcross ? a.T : kAcross;
            hipLaunchKernelGGL((rms_norm_bwd_wide_kernel<FH, FY, FD>),
                               dim3((unsigned)across, (unsigned)((a.T + across - 1) / across)), dim3(1024), 0,
                               stream, a);
        }
        if (a.parts)
            hipLaunchKernelGGL((rms_norm_dw_kernel<FH, FY>),
                               dim3((unsigned)((a.W + 8 * kDwThreads - 1) / (8 * kDwThreads)),
                                    (unsigned)a.blocks),
                               dim3(kDwThreads), 0, stream, a);
    }
}

template <int FH, int FD>
void launch_dy(const NormGradArgs& a, int dy_format, hipStream_t stream) {
    if (dy_format == FP8T_FMT_F32) launch<FH, FP8T_FMT_F32, FD>(a, stream);
    else if (dy_format == FP8T_FMT_FP16) launch<FH, FP8T_FMT_FP16, FD>(a, stream);
    else launch<FH, FP8T_FMT_FP8, FD>(a, stream);
}

bool norm_sizes_ok(int64_t T, int64_t W) {
    return T >= 0 && W >= 0 && T <= kMaxGemmDim && W <= FP8T_MAX_NORM_W;
}

}  // namespace
}  // namespace fp8t

using namespace fp8t;

extern "C" size_t rms_norm_bwd_workspace_size(int64_t T, int64_t W) {
    if (!norm_sizes_ok(T, W) || T == 0 || W == 0) return 0;
    return sizeof(float) * (size_t)norm_grad_plan(T, W).blocks * (size_t)W;
}

extern "C" int rms_norm_bwd(const void* h, int h_format, int64_t h_ld, const void* w, int w_format,
                            const float* rstd, const void* dy, int dy_format, int64_t dy_ld,
                            const void* dr, int64_t dr_ld, int64_t T, int64_t W, void* dx,
                            int d_format, int64_t dx_ld, uint8_t* dx8, int64_t dx8_ld,
                            float dx8_scale, void* dw, int dw_format, void* workspace,
                            size_t workspace_bytes, hipStream_t stream) {
    if (!norm_sizes_ok(T, W) || !float_or_16(h_format) || !float_or_16(w_format) ||
        !storage_format(dy_format) || !float_or_16(d_format) || !float_or_16(dw_format) ||
        (!workspace && workspace_bytes))
        return FP8T_EINVAL;
    if (W == 0) return FP8T_OK;
    if (!dx && !dx8 && !dw) return FP8T_EINVAL;
    if (!matrix_ok(h, h_ld, T, W) || !matrix_ok(dy, dy_ld, T, W) || (T > 0 && !rstd) ||
        (dr && dr_ld < W) || (dx && dx_ld < W) || (dx8 && dx8_ld < W) || !aligned(workspace, 16))
        return FP8T_EINVAL;
    const NormGradPlan p = norm_grad_plan(T, W);
    if (dw && T > 0 && workspace_bytes < rms_norm_bwd_workspace_size(T, W)) return FP8T_EWORKSPACE;
    NormGradArgs a;
    a.h = h;
    a.w = w;
    a.rstd = rstd;
    a.dy = dy;
    a.dr = dr;
    a.dx = dx;
    a.dx8 = dx8;
    a.parts = dw ? static_cast<float*>(workspace) : nullptr;
    a.h_ld = h_ld;
    a.dy_ld = dy_ld;
    a.dr_ld = dr_ld;
    a.dx_ld = dx_ld;
    a.dx8_ld = dx8_ld;
    a.T = T;
    a.W = W;
    a.inv_W = 1.0 / (double)W;
    a.share = p.share;
    a.blocks = p.blocks;
    a.w_format = w_format;
    a.dx8_scale = dx8_scale;
    a.stream = T * W * bytes_of(d_format) > kStreamBytes;
    a.stream8 = T * W > kStreamBytes;
    if (T > 0) {
        const bool f32 = d_format == FP8T_FMT_F32;
        if (h_format == FP8T_FMT_F32) {
            if (f32) launch_dy<FP8T_FMT_F32, FP8T_FMT_F32>(a, dy_format, stream);
            else launch_dy<FP8T_FMT_F32, FP8T_FMT_FP16>(a, dy_format, stream);
        } else {
            if (f32) launch_dy<FP8T_FMT_FP16, FP8T_FMT_F32>(a, dy_format, stream);
            else launch_dy<FP8T_FMT_FP16, FP8T_FMT_FP16>(a, dy_format, stream);
        }
    }
    if (dw) {
        const int64_t n = T > 0 ? p.blocks : 0;
        hipLaunchKernelGGL(rms_norm_join_kernel, dim3((unsigned)((W + 63) / 64)), dim3(kJoinThreads), 0, stream,
                           a.parts, n, W, dw, dw_format);
    }
    return launch_status();
}
