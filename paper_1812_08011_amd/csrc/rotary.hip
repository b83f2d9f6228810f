// rotary_embed: pairs of a head's entries turned by position-dependent angles.
//
// A workgroup takes a few tokens at a time: their cosines and sines go to LDS
// once and serve every head, then the threads walk the tokens' pairs.
#include "lm_formats.h"

namespace fp8t {
namespace {

constexpr int kThreads = 256;

struct RotaryArgs {
    const void* x;
    void* y;
    const int64_t* positions;
    const double* freqs;
    int64_t x_ts, x_hs, y_ts, y_hs, T;
    int H, D, R, inverse;
    float mscale, scale;
};

// cos and sin of position * freq: the angle in turns is reduced in double
// precision (a float angle of 10^5 radians is off by 0.004), its fraction in
// [-1/2, 1/2] holds float accuracy whatever the position.
__device__ __forceinline__ float2 turn(int64_t position, double freq, float m, int inverse) {
    const double turns = (double)position * (freq * 0.15915494309189533577);
    const float f = (float)(turns - __builtin_rint(turns));
    float s, c;
    sincospif(2.0f * f, &s, &c);
    return make_float2(m * c, inverse ? -m * s : m * s);
}

template <int FX, int FY, bool INTERLEAVED>
__global__ __launch_bounds__(kThreads) void rotary_kernel(RotaryArgs a) {
    using TX = fmt_t<FX>;
    using TY = fmt_t<FY>;
    const int half = a.R / 2, rest = a.D - a.R;
    const int items = half + rest;                 // a head's pairs and its copied entries
    for (int64_t t = blockIdx.x; t < a.T; t += gridDim.x) {
        const int64_t pos = half ? a.positions[t] : 0;
        for (int j = threadIdx.x; j < items; j += kThreads) {
            float2 cs = make_float2(1.0f, 0.0f);
            if (j < half) cs = turn(pos, a.freqs[j], a.mscale, a.inverse);
            for (int h = 0; h < a.H; ++h) {
                const TX* x = static_cast<const TX*>(a.x) + t * a.x_ts + h * a.x_hs;
                TY* y = static_cast<TY*>(a.y) + t * a.y_ts + h * a.y_hs;
                if (j < half) {
                    const int i0 = INTERLEAVED ? 2 * j : j, i1 = INTERLEAVED ? 2 * j + 1 : j + half;
                    const float x0 = fmt_value<FX>(x[i0]), x1 = fmt_value<FX>(x[i1]);
                    const float r0 = __builtin_fmaf(x0, cs.x, -(x1 * cs.y));
                    const float r1 = __builtin_fmaf(x1, cs.x, x0 * cs.y);
                    y[i0] = fmt_code<FY>(r0 * a.scale);
                    y[i1] = fmt_code<FY>(r1 * a.scale);
                } else {
                    const int i = a.R + j - half;
                    y[i] = fmt_code<FY>(fmt_value<FX>(x[i]) * a.scale);
                }
            }
        }
    }
}

template <int FX, int FY>
void launch(const RotaryArgs& a, int interleaved, hipStream_t stream) {
    const dim3 grid((unsigned)(a.T < 65536 ? a.T : 65536));
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
