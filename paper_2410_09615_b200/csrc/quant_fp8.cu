// What feeds a linear layer: the residual's addition and the root-mean-square norm, with a bf16 or an 8-bit output, and the
// quantisers that make 8-bit operands of activations (groups of 128 columns of a row) and of weights (blocks of 128 x 128).
// Definitions: include/slim.h.  All of them read every input once and write every output once.  The HBM bounds most of them (share of a copy's
// 6456 GB/s, inputs in rotation: norm of 4096 x 8192 with residual into 8 bits 37.4 us, 97 %; 2048 x 13824 into 8 bits 14.0 us, 94 %;
// a bf16 weight of 11008 x 4096 20.9 us, 100 %), or, for few rows, a launch and a trip to it (1.3 to 2.1 us).  Two forms do not reach it, since few
// CTAs fit on an SM and each loads all it has before it stores: a weight from binary32 (96 registers, two CTAs: 4096 x 4096 17.6 us, 74 %; 11008 x 4096
// 44.4 us, 79 %; 8192 x 28672 209 us, 87 %) and norms of more than 16384 columns (1024 threads of 50 registers, one CTA: 300 x 28672 with residual into
// 8 bits 18.0 us, 52 %; 2000 x 28672 82.5 us, 75 %).
#include "fp8.cuh"

namespace slim {

// ---------------------------------------------------------------- norm
struct NormParams {
    const uint4* X; const uint4* residual; const uint4* gamma;     // eight bf16 each
    uint4* H; uint4* Y;
    uint2* codes; float* scales;
    float eps;
    int d;
    int vecs;                                                      // of eight columns, a row
};

__device__ __forceinline__ uint32_t bf16x2(float lo, float hi) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&v);
}

// A CTA has a row, a thread V vectors of eight columns of it, in registers from the first load to the last store: h = x + residual is
// added in binary32 and normalised as it is; only the copy that goes back to the residual stream is rounded.  Sixteen neighbouring
// threads hold a group of 128 columns.  FMT: the 8-bit format, or -1 for a bf16 output.  TINY_EPS: eps is below 2^-64; a sum below 2^-64 and eps
// are then taken 2^64-fold, which is exact, so that division, sum and root see no subnormal number.  (A larger eps makes the mean square of such a sum
// what it is; as a question that every call asks, 16 x 8192 into bf16 took 1.96 us instead of 1.91.)
template <int V, int FMT, bool TINY_EPS>
__global__ void __launch_bounds__(1024)
rmsnorm_kernel(const NormParams p)
{
    after_previous_grid();
    __shared__ float parts[32];
    const int tid = threadIdx.x, lane = tid & 31;
    const size_t row = (size_t)blockIdx.x * p.vecs;
    float h[V][8];
    float sum = 0.f;
    {
        uint4 x[V], r[V];
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int at = i * blockDim.x + tid;
            x[i] = r[i] = make_uint4(0u, 0u, 0u, 0u);
            if (at < p.vecs) {
                x[i] = p.X[row + at];
                if (p.residual) r[i] = p.residual[row + at];
            }
        }
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const uint32_t xw[4] = {x[i].x, x[i].y, x[i].z, x[i].w}, rw[4] = {r[i].x, r[i].y, r[i].z, r[i].w};
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                h[i][2 * k] = bf16_lo(xw[k]); h[i][2 * k + 1] = bf16_hi(xw[k]);
                if (p.residual) { h[i][2 * k] = add_rn(h[i][2 * k], bf16_lo(rw[k])); h[i][2 * k + 1] = add_rn(h[i][2 * k + 1], bf16_hi(rw[k])); }
            }
#pragma unroll
            for (int k = 0; k < 8; ++k) sum = fma_rn(h[i][k], h[i][k], sum);
        }
    }
#pragma unroll
    for (int o = 16; o; o >>= 1) sum = add_rn(sum, __shfl_xor_sync(0xffffffffu, sum, o));
    if (lane == 0) parts[tid >> 5] = sum;
    if (p.H) {
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int at = i * blockDim.x + tid;
            if (at < p.vecs) p.H[row + at] = make_uint4(bf16x2(h[i][0], h[i][1]), bf16x2(h[i][2], h[i][3]), bf16x2(h[i][4], h[i][5]), bf16x2(h[i][6], h[i][7]));
        }
    }
    __syncthreads();
    // every warp adds the parts up itself, in the same order
    sum = lane < ((int)blockDim.x >> 5) ? parts[lane] : 0.f;
#pragma unroll
    for (int o = 16; o; o >>= 1) sum = add_rn(sum, __shfl_xor_sync(0xffffffffu, sum, o));
    float inv_rms;
    if (TINY_EPS && sum < 0x1p-64f) inv_rms = __frsqrt_rn(__fdiv_rn(mul_rn(sum, 0x1p64f), (float)p.d) + mul_rn(p.eps, 0x1p64f)) * 0x1p32f;
    else inv_rms = __frsqrt_rn(__fdiv_rn(sum, (float)p.d) + p.eps);
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const int at = i * blockDim.x + tid;
        const bool in = at < p.vecs;
        const uint4 g = in ? p.gamma[at] : make_uint4(0u, 0u, 0u, 0u);
        const uint32_t gw[4] = {g.x, g.y, g.z, g.w};
        float y[8];
        uint32_t largest = 0;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            y[2 * k] = mul_rn(mul_rn(h[i][2 * k], inv_rms), bf16_lo(gw[k]));
            y[2 * k + 1] = mul_rn(mul_rn(h[i][2 * k + 1], inv_rms), bf16_hi(gw[k]));
            largest = max(largest, max(magnitude(y[2 * k]), magnitude(y[2 * k + 1])));
        }
        if (FMT < 0) {
            if (in) p.Y[row + at] = make_uint4(bf16x2(y[0], y[1]), bf16x2(y[2], y[3]), bf16x2(y[4], y[5]), bf16x2(y[6], y[7]));
            continue;
        }
        // (vectors past the row's end are zeros: a NaN would come from an infinite factor alone, and then the row is NaN)
        if (!in) largest = 0;
#pragma unroll
        for (int o = 8; o; o >>= 1) largest = max(largest, __shfl_xor_sync(0xffffffffu, largest, o));
        const Scale s(largest, f8_largest(FMT));
        if (in) {
            p.codes[row + at] = make_uint2(codes4<FMT < 0 ? 0 : FMT>(y, s.inv), codes4<FMT < 0 ? 0 : FMT>(y + 4, s.inv));
            if ((tid & 15) == 0) p.scales[(size_t)blockIdx.x * ((p.vecs + 15) >> 4) + (at >> 4)] = s.scale;
        }
    }
}

template <int FMT>
static void run_norm(const NormParams& p, int b, int sms, cudaStream_t st)
{
    // Two vectors a thread where the row fits so, else four (32768 columns at most); one where rows are short, or so few that each has an SM
    // (one row of 4096 1.8 us, with two 2.15; 4096 rows of 8192 37.4 us, with one 47).
    const int v = p.vecs <= 256 || (p.vecs <= 1024 && b <= sms) ? 1 : p.vecs <= 2048 ? 2 : 4;
    const int threads = ceil_div(ceil_div(p.vecs, v), 32) * 32;
    auto* kernel = p.eps < 0x1p-64f ? (v == 1 ? rmsnorm_kernel<1, FMT, true> : v == 2 ? rmsnorm_kernel<2, FMT, true> : rmsnorm_kernel<4, FMT, true>)
                                    : (v == 1 ? rmsnorm_kernel<1, FMT, false> : v == 2 ? rmsnorm_kernel<2, FMT, false> : rmsnorm_kernel<4, FMT, false>);
    launch_dependent(kernel, dim3((unsigned)b), dim3((unsigned)threads), 0, st, p);
}

slim_status_t launch_rmsnorm(const void* X, const void* residual, const void* gamma, float eps, int b, int d, void* H, void* Y,
                             int format, void* codes, float* scales, cudaStream_t st)
{
    NormParams p = {};
    p.X = static_cast<const uint4*>(X); p.residual = static_cast<const uint4*>(residual); p.gamma = static_cast<const uint4*>(gamma);
    p.H = static_cast<uint4*>(H); p.Y = static_cast<uint4*>(Y); p.codes = static_cast<uint2*>(codes); p.scales = scales;
    p.eps = eps; p.d = d; p.vecs = d / 8;
    slim_status_t err;
    const DeviceInfo* di = device_info(&err);
    if (!di) return err;
    if (Y) run_norm<-1>(p, b, di->sm_count, st);
    else if (format == SLIM_FP8_E4M3) run_norm<SLIM_FP8_E4M3>(p, b, di->sm_count, st);
    else run_norm<SLIM_FP8_E5M2>(p, b, di->sm_count, st);
    count_launch(1);
    return cudaGetLastError() == cudaSuccess ? SLIM_OK : SLIM_ERR_CUDA;
}

// ---------------------------------------------------------------- activations: groups of 128 columns of a row
// Sixteen lanes a group, a vector of eight columns a lane, K groups' loads in flight.  Scales are [rows][groups], so a group's number is
// its scale's place.
template <int FMT, int K>
__global__ void __launch_bounds__(256)
quant_rows_kernel(const uint4* X, uint32_t items, uint32_t groups, uint32_t vecs, uint2* codes, float* scales)
{
    after_previous_grid();
    const uint32_t lane = threadIdx.x & 15;
    const uint32_t first = (blockIdx.x * 16 + (threadIdx.x >> 4)) * K;
    uint4 u[K];
    size_t at[K];
    bool in[K];
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const uint32_t item = first + k, row = item / groups, v = (item - row * groups) * 16 + lane;
        in[k] = item < items && v < vecs;
        at[k] = (size_t)row * vecs + v;
        u[k] = in[k] ? X[at[k]] : make_uint4(0u, 0u, 0u, 0u);
    }
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const uint32_t m2 = __vmaxu2(__vmaxu2(magnitude2(u[k].x), magnitude2(u[k].y)), __vmaxu2(magnitude2(u[k].z), magnitude2(u[k].w)));
        uint32_t largest = max(m2 >> 16, m2 & 0xFFFFu);
#pragma unroll
        for (int o = 8; o; o >>= 1) largest = max(largest, __shfl_xor_sync(0xffffffffu, largest, o));
        const Scale s(largest << 16, f8_largest(FMT));
        const uint32_t w[4] = {u[k].x, u[k].y, u[k].z, u[k].w};
        float v[8];
#pragma unroll
        for (int i = 0; i < 4; ++i) { v[2 * i] = bf16_lo(w[i]); v[2 * i + 1] = bf16_hi(w[i]); }
        if (in[k]) codes[at[k]] = make_uint2(codes4<FMT>(v, s.inv), codes4<FMT>(v + 4, s.inv));
        if (lane == 0 && first + k < items) scales[first + k] = s.scale;
    }
}

slim_status_t launch_quant_fp8(const void* X, int b, int d, int format, void* codes, float* scales, cudaStream_t st)
{
    const uint32_t groups = (uint32_t)ceil_div(d, kF8Group);
    const unsigned long long items = (unsigned long long)b * groups;
    if (items > 0x7FFFFFC0ull) return SLIM_ERR_INVALID_ARG;
    // Four groups' loads in flight, two where there are few: 2048 x 13824 14.0 us, with two 14.4; 300 x 28672 5.4 us, with four 5.9; 1 x 4096 1.25, 1.84.
    const bool many = items >= 131072;
    auto* kernel = format == SLIM_FP8_E4M3 ? (many ? quant_rows_kernel<SLIM_FP8_E4M3, 4> : quant_rows_kernel<SLIM_FP8_E4M3, 2>)
                                           : (many ? quant_rows_kernel<SLIM_FP8_E5M2, 4> : quant_rows_kernel<SLIM_FP8_E5M2, 2>);
    const unsigned per_block = many ? 64 : 32;
    launch_dependent(kernel, dim3((unsigned)((items + per_block - 1) / per_block)), dim3(256), 0, st, static_cast<const uint4*>(X), (uint32_t)items, groups,
                     (uint32_t)(d / 8), static_cast<uint2*>(codes), scales);
    count_launch(1);
    return cudaGetLastError() == cudaSuccess ? SLIM_OK : SLIM_ERR_CUDA;
}

// ---------------------------------------------------------------- weights: blocks of 128 x 128
// A CTA has a block, in registers from its loads to its stores.  T: uint16_t (bf16) or float.
template <typename T, int FMT>
__global__ void __launch_bounds__(256)
pack_fp8_kernel(const T* W, int d_out, int d_in, int blocks_in, uint8_t* codes, float* scales)
{
    after_previous_grid();
    constexpr bool kBf16 = sizeof(T) == 2;
    constexpr int kVec = 16 / sizeof(T);                 // columns of a 16-byte load
    constexpr int kPerRow = kF8Group / kVec, kRowsAtOnce = 256 / kPerRow, kLoads = kF8Group / kRowsAtOnce;
    __shared__ uint32_t parts[8];
    const int block = blockIdx.x, bo = block / blocks_in, bi = block - bo * blocks_in;
    const int row0 = bo * kF8Group + (int)threadIdx.x / kPerRow, col = bi * kF8Group + ((int)threadIdx.x % kPerRow) * kVec;
    uint4 u[kLoads];
    uint32_t largest = 0;
#pragma unroll
    for (int k = 0; k < kLoads; ++k) {
        const int row = row0 + k * kRowsAtOnce;
        u[k] = row < d_out && col < d_in ? *reinterpret_cast<const uint4*>(W + (size_t)row * d_in + col) : make_uint4(0u, 0u, 0u, 0u);
    }
#pragma unroll
    for (int k = 0; k < kLoads; ++k) {
        if (kBf16) {
            const uint32_t m2 = __vmaxu2(__vmaxu2(magnitude2(u[k].x), magnitude2(u[k].y)), __vmaxu2(magnitude2(u[k].z), magnitude2(u[k].w)));
            largest = max(largest, max(m2 & 0xFFFF0000u, m2 << 16));
        } else {
            const uint32_t m = 0x7FFFFFFFu;
            largest = max(largest, max(max(u[k].x & m, u[k].y & m), max(u[k].z & m, u[k].w & m)));
        }
    }
#pragma unroll
    for (int o = 16; o; o >>= 1) largest = max(largest, __shfl_xor_sync(0xffffffffu, largest, o));
    if ((threadIdx.x & 31) == 0) parts[threadIdx.x >> 5] = largest;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 8; ++i) largest = max(largest, parts[i]);
    const Scale s(largest, f8_largest(FMT));
    if (threadIdx.x == 0) scales[block] = s.scale;
#pragma unroll
    for (int k = 0; k < kLoads; ++k) {
        const int row = row0 + k * kRowsAtOnce;
        if (row >= d_out || col >= d_in) continue;
        uint8_t* to = codes + (size_t)row * d_in + col;
        const uint32_t w[4] = {u[k].x, u[k].y, u[k].z, u[k].w};
        if (kBf16) {
            float v[8];
#pragma unroll
            for (int i = 0; i < 4; ++i) { v[2 * i] = bf16_lo(w[i]); v[2 * i + 1] = bf16_hi(w[i]); }
            *reinterpret_cast<uint2*>(to) = make_uint2(codes4<FMT>(v, s.inv), codes4<FMT>(v + 4, s.inv));
        } else {
            const float v[4] = {__uint_as_float(w[0]), __uint_as_float(w[1]), __uint_as_float(w[2]), __uint_as_float(w[3])};
            *reinterpret_cast<uint32_t*>(to) = codes4<FMT>(v, s.inv);
        }
    }
}

slim_status_t launch_pack_fp8(const void* W, int type, int d_out, int d_in, int format, void* codes, float* scales, cudaStream_t st)
{
    const int blocks_in = ceil_div(d_in, kF8Group);
    const unsigned long long blocks = (unsigned long long)ceil_div(d_out, kF8Group) * blocks_in;
    if (blocks > 0x7FFFFFFFull) return SLIM_ERR_INVALID_ARG;
    auto run = [&](auto* kernel, auto* w) {
        launch_dependent(kernel, dim3((unsigned)blocks), dim3(256), 0, st, w, d_out, d_in, blocks_in, static_cast<uint8_t*>(codes), scales);
    };
    if (type == SLIM_TYPE_BF16) {
        const uint16_t* w = static_cast<const uint16_t*>(W);
        if (format == SLIM_FP8_E4M3) run(pack_fp8_kernel<uint16_t, SLIM_FP8_E4M3>, w); else run(pack_fp8_kernel<uint16_t, SLIM_FP8_E5M2>, w);
    } else {
        const float* w = static_cast<const float*>(W);
        if (format == SLIM_FP8_E4M3) run(pack_fp8_kernel<float, SLIM_FP8_E4M3>, w); else run(pack_fp8_kernel<float, SLIM_FP8_E5M2>, w);
    }
    count_launch(1);
    return cudaGetLastError() == cudaSuccess ? SLIM_OK : SLIM_ERR_CUDA;
}

}  // namespace slim
