// fp16_dequantize: FP16 (1,6,9) codes to floats or IEEE halves.  HBM-bound:
// eight codes per thread and iteration, one 16-byte load, 16-byte stores.  4.8 M
// codes to halves: 5.6 us, 3.4 TB/s; below a million codes a launch, 2 to 4 us.
#include <hip/hip_fp16.h>

#include "lm_formats.h"

namespace fp8t {
namespace {

constexpr int kThreads = 256;

// The half nearest to a float.  The float is the product already rounded: the
// compiler would otherwise join product and conversion into one mixed FMA,
// which rounds once and turns -0 into +0.
__device__ __forceinline__ uint32_t half_bits(float x) {
    asm("" : "+v"(x));
    return (uint32_t)__half_as_ushort(__float2half_rn(x));
}

template <bool HALF>
__global__ __launch_bounds__(kThreads) void dequantize_kernel(const uint16_t* __restrict__ src,
                                                              float scale, void* __restrict__ dst,
                                                              int64_t n, int vec_ok) {
    const int64_t tid = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    const int64_t stride = (int64_t)gridDim.x * kThreads;
    const int64_t nvec = vec_ok ? n / 8 : 0;
    const uint4* s8 = reinterpret_cast<const uint4*>(src);
    for (int64_t i = tid; i < nvec; i += stride) {
        const uint4 w = s8[i];
        const uint32_t ws[4] = {w.x, w.y, w.z, w.w};
        float f[8];
#pragma unroll
        for (int v = 0; v < 8; ++v)
            f[v] = fp16_to_f32((ws[v / 2] >> (16 * (v % 2))) & 0xFFFFu) * scale;
        if constexpr (HALF) {
            uint32_t h[4];
#pragma unroll
            for (int v = 0; v < 4; ++v) h[v] = half_bits(f[2 * v]) | (half_bits(f[2 * v + 1]) << 16);
            reinterpret_cast<uint4*>(dst)[i] = make_uint4(h[0], h[1], h[2], h[3]);
        } else {
            float4* d = reinterpret_cast<float4*>(dst) + 2 * i;
            d[0] = make_float4(f[0], f[1], f[2], f[3]);
            d[1] = make_float4(f[4], f[5], f[6], f[7]);
        }
    }
    for (int64_t i = nvec * 8 + tid; i < n; i += stride) {
        const float f = fp16_to_f32(src[i]) * scale;
        if constexpr (HALF) static_cast<uint16_t*>(dst)[i] = (uint16_t)half_bits(f);
        else static_cast<float*>(dst)[i] = f;
    }
}

}  // namespace
}  // namespace fp8t

using namespace fp8t;

extern "C" int fp16_dequantize(const uint16_t* src, float scale, void* dst, int dst_format,
                               int64_t n, hipStream_t stream) {
    if (n < 0) return FP8T_EINVAL;
    if (dst_format != FP8T_FMT_F32 && dst_format != FP8T_FMT_HALF) return FP8T_EINVAL;
    if (n == 0) return FP8T_OK;
    if (!src || !dst) return FP8T_EINVAL;
    const int vec_ok = aligned(src, 16) && aligned(dst, 16);
    const dim3 grid(stride_blocks((n + 7) / 8, kThreads) < 8192 ? stride_blocks((n + 7) / 8, kThreads)
                                                                : 8192);
    if (dst_format == FP8T_FMT_HALF)
        hipLaunchKernelGGL(dequantize_kernel<true>, grid, dim3(kThreads), 0, stream, src, scale,
                           dst, n, vec_ok);
    else
        hipLaunchKernelGGL(dequantize_kernel<false>, grid, dim3(kThreads), 0, stream, src, scale,
                           dst, n, vec_ok);
    return launch_status();
}
