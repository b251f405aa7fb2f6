// Shared by the kernels of the 8-bit floating-point linear (e4m3 codes, a scale for 128 channels of a token and for
// 128 x 128 of the weights) and of the root-mean-square norm in front of it.
#pragma once
#include "haq_common.h"
#include "quant_math.h"

namespace haq {

constexpr int FP8_BLOCK = 128;          // channels that share a scale
constexpr float E4M3_MAX = 448.0f;      // largest finite magnitude
constexpr float TINY_MAX = 0x1p-100f;   // a block or row whose largest magnitude is below counts as zero

struct NormArgs {
    const void* x;
    const void* residual;  // null: none
    const float* weight;   // [K]
    int64_t ldx, ldr, lds, ldy;
    void* sum;             // optional, 16 bits
    void* y;               // optional, 16 bits
    double eps;
    int T, K;
    int codes;             // HAQ_CODES_*
    uint8_t* q;            // packed [K/16][R][16]
    int64_t R;
    float* scale;          // int8: [T]; e4m3: [K blocks][R]
};
int launch_rmsnorm(const NormArgs& a, int dtype, hipStream_t st);

struct ActQuantArgs {
    const void* x;
    int64_t ldx;
    int T, K;
    uint8_t* q;      // packed [K/16][R][16]
    int64_t R;
    float* scale;    // [K blocks][R]
};
int launch_act_quant_fp8(const ActQuantArgs& a, int dtype, hipStream_t st);
int launch_weight_quant_fp8(const float* w, int K, int N, uint8_t* wq, float* scale, hipStream_t st);

struct Fp8GemmArgs {
    const uint8_t* A;   // packed token codes [K/16][R][16]
    int64_t R;
    const float* sa;    // [K blocks][R]
    const uint8_t* B;   // packed weight codes [Kpad/16][Npad][16]
    int64_t Npad;
    const float* sb;    // [K blocks][N blocks]
    int M, K, N;
    int act;
    void* Y;            // 16 bits
    int64_t ldy;
};
int launch_fp8_gemm(const Fp8GemmArgs& a, int dtype, hipStream_t st);
bool fp8_stream_rows16_fits(int M, int K);  // a few rows in 16 bits: codes and linear in one launch (A, sa and R of `a` not used)
int launch_fp8_stream_rows16(const Fp8GemmArgs& a, const void* x, int64_t ldx, int dtype, hipStream_t st);
// The streaming kernel in tiles of 16 row_blocks rows x 16 channel_blocks channels: 1 x 1, 1 x 2, 1 x 4, 2 x 2, 2 x 4, 4 x 2 or 4 x 4.
int launch_fp8_stream(const Fp8GemmArgs& a, int row_blocks, int channel_blocks, int dtype, hipStream_t st);

// ---- device ----------------------------------------------------------------------------------------------------
#ifdef __HIPCC__
// 16-bit rows, eight values to a 16-byte load.
template <int DT>
__device__ __forceinline__ void unpack8(const uint4& r, float* v) {
    const uint32_t u[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (DT == HAQ_F16) {
            const __half2 h = *reinterpret_cast<const __half2*>(&u[i]);
            v[2 * i] = __low2float(h);
            v[2 * i + 1] = __high2float(h);
        } else {
            v[2 * i] = __uint_as_float(u[i] << 16);
            v[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
        }
    }
}
template <int DT>
__device__ __forceinline__ uint32_t pack2(float a, float b) {  // each rounded once, to nearest even
    if constexpr (DT == HAQ_F16) {
        const __half h[2] = {f2h(a), f2h(b)};
        return *reinterpret_cast<const uint32_t*>(h);
    } else {
        asm("" : "+v"(a), "+v"(b));
        typedef __bf16 bf2 __attribute__((ext_vector_type(2)));
        const bf2 h = {(__bf16)a, (__bf16)b};
        return *reinterpret_cast<const uint32_t*>(&h);
    }
}
template <int DT>
__device__ __forceinline__ uint4 pack8(const float* v) {
    return make_uint4(pack2<DT>(v[0], v[1]), pack2<DT>(v[2], v[3]), pack2<DT>(v[4], v[5]), pack2<DT>(v[6], v[7]));
}

// Lane exchanges of the vector unit: neighbours, pairs, halves of 8, rows of 16.
#define HAQ_LANES_XOR1 0xB1
#define HAQ_LANES_XOR2 0x4E
#define HAQ_LANES_MIRROR8 0x141
#define HAQ_LANES_MIRROR16 0x140
template <int CTRL>
__device__ __forceinline__ float lanes(float v) {
    return __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v), CTRL, 0xf, 0xf, true));
}
// Maximum over each 8 neighbouring lanes (the 128 channels of a block at 16 channels a lane).  All lanes must be active.
__device__ __forceinline__ float max_of_8_lanes(float v) {
    v = fmaxf(v, lanes<HAQ_LANES_XOR1>(v));
    v = fmaxf(v, lanes<HAQ_LANES_XOR2>(v));
    return fmaxf(v, lanes<HAQ_LANES_MIRROR8>(v));
}

// Codes of a block: scale = a / 448, codes e4m3(v (448 / a)) with a the largest magnitude.  |v (448 / a)| <= 448 (1 + 2^-23)
// rounds to 448 at most, so the conversion never overflows.  A NaN is ignored by the maximum and stays a NaN code; an
// infinity makes the scale infinite, 448 / a zero and its own code NaN.
struct BlockScale {
    float scale, r;
};
__device__ __forceinline__ BlockScale block_scale(float a) {
    BlockScale s{a / E4M3_MAX, E4M3_MAX / a};
    if (a < TINY_MAX) s.scale = s.r = 0.0f;
    return s;
}
__device__ __forceinline__ float absmax16(const float (&v)[16]) {
    float m = 0.0f;
#pragma unroll
    for (int i = 0; i < 16; i += 2) m = fmaxf(fmaxf(m, fabsf(v[i])), fabsf(v[i + 1]));
    return m;
}
__device__ __forceinline__ uint32_t e4m3x4(float a, float b, float c, float d) {
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
}
__device__ __forceinline__ uint4 e4m3x16(const float (&v)[16], float r) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = e4m3x4(v[4 * i] * r, v[4 * i + 1] * r, v[4 * i + 2] * r, v[4 * i + 3] * r);
    return make_uint4(w[0], w[1], w[2], w[3]);
}
#endif

}  // namespace haq
