// The linear layer on 8-bit floating-point operands (include/slim.h, slim_linear_fwd_fp8):
//     Y[m][n] = sum_g xs[m][g] ws[n / 128][g] * (sum over the 128 columns k of group g of xq[m][k] wq[n][k])
#include <cuda_fp16.h>
#include "fp8.cuh"

namespace slim {

// Four codes' values: either format's values are exact in half precision.
template <int FMT>
__device__ __forceinline__ float4 values4(uint32_t w) {
    uint32_t lo, hi;
    if (FMT == SLIM_FP8_E4M3) {
        asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(lo) : "h"((uint16_t)w));
        asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(hi) : "h"((uint16_t)(w >> 16)));
    } else {
        asm("cvt.rn.f16x2.e5m2x2 %0, %1;" : "=r"(lo) : "h"((uint16_t)w));
        asm("cvt.rn.f16x2.e5m2x2 %0, %1;" : "=r"(hi) : "h"((uint16_t)(w >> 16)));
    }
    const float2 a = __half22float2(*reinterpret_cast<__half2*>(&lo)), b = __half22float2(*reinterpret_cast<__half2*>(&hi));
    return make_float4(a.x, a.y, b.x, b.y);
}

// A warp per output, four columns a lane: one group at a time.
template <int FX, int FW>
__global__ void __launch_bounds__(256)
fp8_simple_kernel(const uint8_t* Xq, const float* Xs, const uint8_t* Wq, const float* Ws, size_t outputs, int d_out, int d_in, int groups, __nv_bfloat16* Y)
{
    after_previous_grid();
    const int lane = threadIdx.x & 31;
    for (size_t o = (size_t)blockIdx.x * 8 + (threadIdx.x >> 5); o < outputs; o += (size_t)gridDim.x * 8) {
        const size_t m = o / d_out, n = o - m * d_out;
        float acc = 0.f;
        for (int g = 0; g < groups; ++g) {
            const int k = g * kF8Group + lane * 4;
            float part = 0.f;
            if (k < d_in) {
                const float4 x = values4<FX>(*reinterpret_cast<const uint32_t*>(Xq + m * d_in + k)), w = values4<FW>(*reinterpret_cast<const uint32_t*>(Wq + n * d_in + k));
                part = x.x * w.x + x.y * w.y + x.z * w.z + x.w * w.w;
            }
#pragma unroll
            for (int s = 16; s; s >>= 1) part += __shfl_xor_sync(0xffffffffu, part, s);
            acc = fmaf(part, Xs[m * groups + g] * Ws[n / kF8Group * groups + g], acc);
        }
        if (lane == 0) Y[o] = __float2bfloat16_rn(acc);
    }
}

slim_status_t launch_fp8(const uint8_t* Xq, const float* Xs, int x_format, int b, const uint8_t* Wq, const float* Ws, int w_format, int d_out, int d_in,
                         __nv_bfloat16* Y, uint32_t* status_dev, cudaStream_t st)
{
    (void)status_dev;
    const size_t outputs = (size_t)b * d_out;
    const unsigned grid = (unsigned)(outputs / 8 + 1 < 65536 ? outputs / 8 + 1 : 65536);
    auto* kernel = x_format == SLIM_FP8_E4M3 ? (w_format == SLIM_FP8_E4M3 ? fp8_simple_kernel<0, 0> : fp8_simple_kernel<0, 1>)
                                             : (w_format == SLIM_FP8_E4M3 ? fp8_simple_kernel<1, 0> : fp8_simple_kernel<1, 1>);
    launch_dependent(kernel, dim3(grid), dim3(256), 0, st, Xq, Xs, Wq, Ws, outputs, d_out, d_in, ceil_div(d_in, kF8Group), Y);
    count_launch(1);
    return cudaGetLastError() == cudaSuccess ? SLIM_OK : SLIM_ERR_CUDA;
}

}  // namespace slim
