// e4m3 codes of activations (a scale for 128 channels of a token) and of weights (a scale for 128 x 128).
#include "fp8.h"

namespace haq {

namespace {

constexpr int AQ_WAVES = 4;

// A wave takes RW rows, 64 / RW chunks of 16 channels of each, a chunk to a lane: eight neighbouring lanes hold the 128 channels
// of a block, whose maximum takes three lane exchanges, and with RW = 8 the codes of 8 rows fill the 128-byte lines of the
// packed layout.  Bound: memory, two bytes read and one written an element: 4096 x 14336 in 33.9 us (5.2 TB/s, a copy's rate).
template <int DT, int RW>
__global__ __launch_bounds__(AQ_WAVES * 64) void act_quant_kernel(ActQuantArgs a, int groups, int rows_x) {
    constexpr int LPR = 64 / RW;
    const int lane = threadIdx.x & 63;
    // work-group: AQ_WAVES pieces of a row group; `groups` of them to a row group, one behind the other, so that rows are read on
    const int row = ((int)(blockIdx.x / groups) + (int)blockIdx.y * rows_x) * RW + lane / LPR;
    const int c = ((int)(blockIdx.x % groups) * AQ_WAVES + (threadIdx.x >> 6)) * LPR + lane % LPR;
    const bool here = row < a.T && c < a.K / 16;
    float v[16] = {};
    if (here) {
        const uint4* px = reinterpret_cast<const uint4*>((const uint16_t*)a.x + (size_t)row * a.ldx + c * 16);
        const uint4 r0 = px[0], r1 = px[1];
        unpack8<DT>(r0, v);
        unpack8<DT>(r1, v + 8);
    }
    const BlockScale s = block_scale(max_of_8_lanes(absmax16(v)));
    if (here) {
        *reinterpret_cast<uint4*>(a.q + ((size_t)c * a.R + row) * 16) = e4m3x16(v, s.r);
        if (c % 8 == 0) a.scale[(size_t)(c / 8) * a.R + row] = s.scale;
    }
}

template <int DT, int RW>
int launch_act(const ActQuantArgs& a, hipStream_t st) {
    const int groups = cdiv(cdiv(a.K / 16, 64 / RW), AQ_WAVES), row_groups = cdiv(a.T, RW);
    const int most = (1 << 22) / groups, rows_x = row_groups < most ? row_groups : most;  // a grid has fewer than 2^32 threads in a direction
    hipLaunchKernelGGL((act_quant_kernel<DT, RW>), dim3(rows_x * groups, cdiv(row_groups, rows_x)), dim3(AQ_WAVES * 64), 0, st, a, groups, rows_x);
    HAQ_CHECK_HIP(hipGetLastError());
    return HAQ_OK;
}

// A work-group takes one block of 128 x 128: 32 lanes read a row of it, four values each, eight rows at a time; the values stay
// in registers between the maximum and the rounding.  Bound: memory, four bytes read and one written an element: 4096 x 14336 in
// 53.8 us (5.5 TB/s, a copy's rate).
__global__ __launch_bounds__(256) void weight_quant_kernel(const float* w, int K, int N, uint8_t* wq, float* scale) {
    __shared__ float red[4];
    const int n = blockIdx.x * FP8_BLOCK + (threadIdx.x & 31) * 4, k0 = blockIdx.y * FP8_BLOCK + (threadIdx.x >> 5);
    float4 v[16];
    float m = 0.0f;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const int k = k0 + 8 * i;
        v[i] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        if (k < K && n < N) v[i] = *reinterpret_cast<const float4*>(w + (size_t)k * N + n);
    }
#pragma unroll
    for (int i = 0; i < 16; ++i)
        m = fmaxf(fmaxf(fmaxf(m, fabsf(v[i].x)), fmaxf(fabsf(v[i].y), fabsf(v[i].z))), fabsf(v[i].w));
    m = wave_max(m);
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = m;
    __syncthreads();
    const BlockScale s = block_scale(fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3])));
    if (threadIdx.x == 0) scale[(size_t)blockIdx.y * gridDim.x + blockIdx.x] = s.scale;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const int k = k0 + 8 * i;
        if (k < K && n < N) *reinterpret_cast<uint32_t*>(wq + (size_t)k * N + n) = e4m3x4(v[i].x * s.r, v[i].y * s.r, v[i].z * s.r, v[i].w * s.r);
    }
}

}  // namespace

// One row or eight to a wave, us at K = 4096:  1 row 1.9 / 2.2,  4 2.07 / 2.05,  7 2.2 / 2.05,  33 2.4 / 2.1,  256 3.4 / 2.6,  4096 27 / 10.9.
int launch_act_quant_fp8(const ActQuantArgs& a, int dtype, hipStream_t st) {
    if (a.T >= 4) return dtype == HAQ_F16 ? launch_act<HAQ_F16, 8>(a, st) : launch_act<HAQ_BF16, 8>(a, st);
    return dtype == HAQ_F16 ? launch_act<HAQ_F16, 1>(a, st) : launch_act<HAQ_BF16, 1>(a, st);
}

int launch_weight_quant_fp8(const float* w, int K, int N, uint8_t* wq, float* scale, hipStream_t st) {
    hipLaunchKernelGGL(weight_quant_kernel, dim3(cdiv(N, FP8_BLOCK), cdiv(K, FP8_BLOCK)), dim3(256), 0, st, w, K, N, wq, scale);
    HAQ_CHECK_HIP(hipGetLastError());
    return HAQ_OK;
}

}  // namespace haq
