// rotary_embed: pairs of a head's entries turned by position-dependent angles.
//
// HBM-bound.  A thread owns eight pairs of one token and walks heads with
// their cosines and sines in registers, so that the angles cost little next to
// the codes; eight consecutive elements move with one load or store at any
// address.  A head's entries past R are units of sixteen that are only
// converted.
//
// 16384 tokens of 40 heads of 128, FP16 to FP8: 64 us, 3.9 TB/s (a copy of 1 GiB
// runs at 5.2), and 49 us where the caches still hold part of the operands;
// four heads a thread, or one or four of them in flight in place of two, change
// that by 3% either way.  5003 tokens of 12 heads of 80, FP16 to FP16: 9 us (2.2 TB/s; 11 us from
// cold caches, most of it the reduction of the angles and one round of loads).
// One token: 3.5 us, a launch.
#include "lm_formats.h"

namespace fp8t {
namespace {

constexpr int kThreads = 256;
constexpr int64_t kAcross = 1 << 20;   // workgroups along a grid's first dimension

struct RotaryArgs {
    const void* x;
    void* y;
    const int64_t* positions;
    const double* freqs;
    int64_t x_ts, x_hs, y_ts, y_hs, T;
    int H, D, R, inverse;
    float mscale, scale;
    int pair_units, units, groups;     // units per head; threads that share a unit's heads
    int tokens;                        // per workgroup (gridDim.y > 1: one)
};

// The fraction of a turn, in [-1/2, 1/2], of position * freq where the product in
// double precision has lost it: freq / (2 pi) in two doubles, the position in
// two parts of 32 bits, each product with its rounding error.  Off by 2^-44 of a
// turn and of freq.
__device__ __forceinline__ float far_fraction(int64_t position, double freq) {
    constexpr double kHi = 0x1.45f306dc9c883p-3, kLo = -0x1.6b01ec5417056p-57;   // 1 / (2 pi)
    const double g = freq * kHi, g2 = __builtin_fma(freq, kHi, -g) + freq * kLo;
    const int64_t low = (int64_t)((uint64_t)position & 0xFFFFFFFFu);
    const double part[2] = {(double)(position - low), (double)low};              // both exact
    double sum = 0.0;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const double t = part[i] * g, e = __builtin_fma(part[i], g, -t) + part[i] * g2;
        sum += (t - __builtin_rint(t)) + (e - __builtin_rint(e));
    }
    return (float)(sum - __builtin_rint(sum));
}

// cos and sin of position * freq: the angle in turns is reduced in double
// precision (a float angle of 10^5 radians is off by 0.004), its fraction in
// [-1/2, 1/2] holds float accuracy.  Up to 2^20 turns one product is off by
// 2^-31 of a turn at most.
// The nearest quarter turn is taken off; on the eighth of a turn that is left,
// either way, the Taylor series to the 9th and 8th power are off by less than
// 3e-8, half a step of FP32 at 1.
__device__ __forceinline__ float2 turn(int64_t position, double freq, float m, int inverse) {
    const double turns = (double)position * (freq * 0.15915494309189533577);
    float f = (float)(turns - __builtin_rint(turns));
    if (__builtin_expect(!(__builtin_fabs(turns) <= 0x1p20), 0)) f = far_fraction(position, freq);
    const float k = __builtin_rintf(4.0f * f), r = __builtin_fmaf(k, -0.25f, f), r2 = r * r;
    float s = __builtin_fmaf(r2, 42.0586939f, -76.7058598f);
    s = __builtin_fmaf(r2, s, 81.6052493f);
    s = __builtin_fmaf(r2, s, -41.3417022f);
    s = __builtin_fmaf(r2, s, 6.28318531f) * r;
    float c = __builtin_fmaf(r2, 60.2446414f, -85.4568172f);
    c = __builtin_fmaf(r2, c, 64.939394f);
    c = __builtin_fmaf(r2, c, -19.7392088f);
    c = __builtin_fmaf(r2, c, 1.0f);
    // quarter turns: (c, s) -> (-s, c)
    const int q = (int)k;
    const float cq = q & 1 ? -s : c, sq = q & 1 ? c : s, sign = q & 2 ? -m : m;
    return make_float2(sign * cq, (inverse ? -sign : sign) * sq);
}

// n <= 8 elements from p on.
template <int FMT>
__device__ __forceinline__ void load_some(const fmt_t<FMT>* p, int n, float* x) {
    if (n == 8) {
        const Eight<FMT> e = *reinterpret_cast<const Eight<FMT>*>(p);
        values_of<FMT>(e, special_in<FMT>(e), x);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = i < n ? fmt_value<FMT>(p[i]) : 0.0f;
    }
}
template <int FX, int FY, bool INTERLEAVED>
__global__ __launch_bounds__(kThreads) void rotary_kernel(RotaryArgs a) {
    const int items = a.units * a.groups;                   // threads of a token
    int64_t t;
    int id;
    const int64_t block = (int64_t)blockIdx.z * gridDim.x + blockIdx.x;
    if (gridDim.y > 1) {
        t = block;
        id = blockIdx.y * kThreads + threadIdx.x;
        if (id >= items || t >= a.T) return;
    } else {
        t = block * a.tokens + threadIdx.x / items;
        id = threadIdx.x % items;
        if ((int)threadIdx.x >= a.tokens * items || t >= a.T) return;
    }
    const int u = id % a.units, group = id / a.units, half = a.R / 2;
    // the unit's two runs of up to eight entries
    const bool turned = u < a.pair_units;
    const int j0 = 8 * u, c0 = a.R + 16 * (u - a.pair_units), pairs = up_to_8(half - j0);
    int i0, i1, n0, n1;
    if (!turned) {
        i0 = c0;
        i1 = c0 + 8;
        n0 = up_to_8(a.D - i0);
        n1 = up_to_8(a.D - i1);
    } else if (INTERLEAVED) {
        i0 = 2 * j0;
        i1 = i0 + 8;
        n0 = up_to_8(2 * pairs);
        n1 = up_to_8(2 * pairs - 8);
    } else {
        i0 = j0;
        i1 = j0 + half;
        n0 = n1 = pairs;
    }
    float2 cs[8];
    if (turned) {
        const int64_t position = a.positions[t];
#pragma unroll
        for (int i = 0; i < 8; ++i)
            cs[i] = i < pairs ? turn(position, a.freqs[j0 + i], a.mscale, a.inverse) : make_float2(1.0f, 0.0f);
    }
    const fmt_t<FX>* x = static_cast<const fmt_t<FX>*>(a.x) + t * a.x_ts;
    fmt_t<FY>* y = static_cast<fmt_t<FY>*>(a.y) + t * a.y_ts;
#pragma unroll 2
    for (uint32_t h = group; h < (uint32_t)a.H; h += a.groups) {   // the last step may pass 2^31
        float p[8], q[8];
        load_some<FX>(x + h * a.x_hs + i0, n0, p);
        load_some<FX>(x + h * a.x_hs + i1, n1, q);
        if (turned) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                // pair i: entries i of both runs, or neighbours in one of them
                float& x0 = INTERLEAVED ? (i < 4 ? p[2 * (i % 4)] : q[2 * (i % 4)]) : p[i];
                float& x1 = INTERLEAVED ? (i < 4 ? p[2 * (i % 4) + 1] : q[2 * (i % 4) + 1]) : q[i];
                const float r0 = __builtin_fmaf(x0, cs[i].x, -(x1 * cs[i].y));
                const float r1 = __builtin_fmaf(x1, cs[i].x, x0 * cs[i].y);
                x0 = r0;
                x1 = r1;
            }
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            p[i] *= a.scale;
            q[i] *= a.scale;
        }
        store_some<FY>(y + h * a.y_hs + i0, n0, p);
        store_some<FY>(y + h * a.y_hs + i1, n1, q);
    }
}

template <int FX, int FY>
void launch(RotaryArgs a, int interleaved, hipStream_t stream) {
    a.pair_units = (a.R / 2 + 7) / 8;
    a.units = a.pair_units + (a.D - a.R + 15) / 16;
    // Eight heads a thread (16384 x 40 x 128 in part cached: 50 us, with one head
    // 81, since its angles are used once); fewer where that leaves the card empty, below 2048
    // threads a CU (1024 x 40 x 128: 8.4 us, with eight heads 13; 256 x 8 x 128:
    // 5 and 12).
    const int64_t want = (int64_t)device_cus() * 2048;
    int64_t groups = (a.H + 7) / 8;
    while (groups < a.H && a.T * a.units * groups < want) groups = 2 * groups < a.H ? 2 * groups : a.H;
    const int64_t cap = (1 << 23) / a.units;
    a.groups = (int)(groups < cap ? groups : cap);
    const int64_t items = (int64_t)a.units * a.groups;
    a.tokens = items < kThreads ? (int)(kThreads / items) : 1;
    const int64_t blocks = (a.T + a.tokens - 1) / a.tokens, across = blocks < kAcross ? blocks : kAcross;
    const dim3 grid((unsigned)across, (unsigned)((items + kThreads - 1) / kThreads),
                    (unsigned)((blocks + across - 1) / across));
    if (interleaved)
        hipLaunchKernelGGL((rotary_kernel<FX, FY, true>), grid, dim3(kThreads), 0, stream, a);
    else
        hipLaunchKernelGGL((rotary_kernel<FX, FY, false>), grid, dim3(kThreads), 0, stream, a);
}

template <int FX>
void launch_y(const RotaryArgs& a, int fy, int interleaved, hipStream_t stream) {
    if (fy == FP8T_FMT_F32) launch<FX, FP8T_FMT_F32>(a, interleaved, stream);
    else if (fy == FP8T_FMT_FP16) launch<FX, FP8T_FMT_FP16>(a, interleaved, stream);
    else launch<FX, FP8T_FMT_FP8>(a, interleaved, stream);
}

}  // namespace
}  // namespace fp8t

using namespace fp8t;

extern "C" int rotary_embed(const void* x, int x_format, int64_t x_ts, int64_t x_hs,
                            const int64_t* positions, const double* freqs, int64_t T, int64_t H,
                            int64_t D, int64_t R, int interleaved, int inverse, float mscale,
                            float scale, void* y, int y_format, int64_t y_ts, int64_t y_hs,
                            hipStream_t stream) {
    if (T < 0 || H < 0 || D < 0 || D > 65536 || R < 0 || R > D || R % 2) return FP8T_EINVAL;
    if (T > kMaxGemmDim || H > kMaxGemmDim) return FP8T_EINVAL;
    if (x_format < FP8T_FMT_F32 || x_format > FP8T_FMT_FP8) return FP8T_EINVAL;
    if (y_format < FP8T_FMT_F32 || y_format > FP8T_FMT_FP8) return FP8T_EINVAL;
    if ((interleaved | 1) != 1 || (inverse | 1) != 1) return FP8T_EINVAL;
    if (T == 0 || H == 0 || D == 0) return FP8T_OK;
    if (x_ts < 0 || x_hs < 0 || !rows_apart(T, H, D, y_ts, y_hs)) return FP8T_EINVAL;
    if (!x || !y || (R && (!positions || !freqs))) return FP8T_EINVAL;
    RotaryArgs a;
    a.x = x;
    a.y = y;
    a.positions = positions;
    a.freqs = freqs;
    a.x_ts = x_ts;
    a.x_hs = x_hs;
    a.y_ts = y_ts;
    a.y_hs = y_hs;
    a.T = T;
    a.H = (int)H;
    a.D = (int)D;
    a.R = (int)R;
    a.inverse = inverse;
    a.mscale = mscale;
    a.scale = scale;
    if (x_format == FP8T_FMT_F32) launch_y<FP8T_FMT_F32>(a, y_format, interleaved, stream);
    else if (x_format == FP8T_FMT_FP16) launch_y<FP8T_FMT_FP16>(a, y_format, interleaved, stream);
    else launch_y<FP8T_FMT_FP8>(a, y_format, interleaved, stream);
    return launch_status();
}
