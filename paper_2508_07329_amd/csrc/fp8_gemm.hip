// Linear on e4m3 codes with a scale for 128 channels of a token and for 128 x 128 of the weights:
//   y[t][n] = round16(act(sum_b (sa[b][t] sb[b][n / 128]) p_b)),  p_b = sum over the 128 channels k of block b of a[t][k] w[k][n].
// One v_mfma_f32_16x16x128_f8f6f4 forms p_b for 16 tokens x 16 channels; the scaled sum over the blocks is kept in binary32.
#include "fp8.h"

namespace haq {

namespace {

typedef int v8i __attribute__((ext_vector_type(8)));
typedef float v4f __attribute__((ext_vector_type(4)));

__device__ __forceinline__ v4f mfma_e4m3(v8i w, v8i x, v4f c) { return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(w, x, c, 0, 0, 0, 0, 0, 0); }

// A wave for each 16 tokens x 16 channels.  Lane l holds 32 of the 128 channels of a block for weight channel and token l % 16 (the
// order of the 128 does not matter as long as both operands agree) and ends up with channels 4 (l / 16) .. + 3 of token l % 16.
template <int DT>
__global__ __launch_bounds__(256) void fp8_simple_kernel(Fp8GemmArgs a) {
    const int lane = threadIdx.x & 63, l16 = lane & 15, q = lane >> 4;
    const int m0 = blockIdx.x * 16, n0 = (blockIdx.y * 4 + (threadIdx.x >> 6)) * 16;
    if (n0 >= a.N) return;
    const int nb = (a.K + FP8_BLOCK - 1) / FP8_BLOCK, nn = (a.N + FP8_BLOCK - 1) / FP8_BLOCK, row = min(m0 + l16, a.M - 1);
    v4f acc = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int b = 0; b < nb; ++b) {
        v8i w, x;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int c = 8 * b + 2 * q + h;
            uint4 wv = make_uint4(0, 0, 0, 0), xv = wv;
            if (c * 16 < a.K) {
                wv = *reinterpret_cast<const uint4*>(a.B + ((size_t)c * a.Npad + n0 + l16) * 16);
                xv = *reinterpret_cast<const uint4*>(a.A + ((size_t)c * a.R + row) * 16);
            }
            w[4 * h] = wv.x, w[4 * h + 1] = wv.y, w[4 * h + 2] = wv.z, w[4 * h + 3] = wv.w;
            x[4 * h] = xv.x, x[4 * h + 1] = xv.y, x[4 * h + 2] = xv.z, x[4 * h + 3] = xv.w;
        }
        const v4f p = mfma_e4m3(w, x, v4f{0.0f, 0.0f, 0.0f, 0.0f});
        const float s = a.sa[(size_t)b * a.R + row] * a.sb[(size_t)b * nn + n0 / FP8_BLOCK];
#pragma unroll
        for (int r = 0; r < 4; ++r) acc[r] = __builtin_fmaf(s, p[r], acc[r]);
    }
    if (m0 + l16 >= a.M) return;
    float v[4];
#pragma unroll
    for (int r = 0; r < 4; ++r) v[r] = a.act == HAQ_ACT_RELU && acc[r] < 0.0f ? 0.0f : acc[r];
    *reinterpret_cast<uint2*>((uint16_t*)a.Y + (size_t)(m0 + l16) * a.ldy + n0 + 4 * q) = make_uint2(pack2<DT>(v[0], v[1]), pack2<DT>(v[2], v[3]));
}

}  // namespace

int launch_fp8_gemm(const Fp8GemmArgs& a, int dtype, hipStream_t st) {
    const dim3 grid(cdiv(a.M, 16), cdiv(a.N, 64));
    if (dtype == HAQ_F16)
        hipLaunchKernelGGL(fp8_simple_kernel<HAQ_F16>, grid, dim3(256), 0, st, a);
    else
        hipLaunchKernelGGL(fp8_simple_kernel<HAQ_BF16>, grid, dim3(256), 0, st, a);
    HAQ_CHECK_HIP(hipGetLastError());
    return HAQ_OK;
}

}  // namespace haq
