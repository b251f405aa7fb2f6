// Root-mean-square norm with the residual's addition, and codes as output: the step between two layers that feeds a linear on
// 8-bit codes (int8 with a scale for each token, or e4m3 with a scale for 128 channels of a token).
//
//   h = round16(x + residual);  inv = binary32(1 / sqrt(sum h^2 / K + eps)), in binary64 up to that rounding;
//   v = (h inv) weight;  y = round16(v);  codes of v (not of y: one rounding fewer).
//
// Bound: memory, 2 to 4 reads and writes of 16 bits and one of 8 an element.  A row is read once: it stays in registers as
// 16-bit values between the sum of squares, the row maximum (int8) and the rounding.  The squares of 16-bit values are exact
// in binary64 and so are summed there; the binary64 units of this chip are as wide as the binary32 ones.  The order of the sum goes by
// K alone, so that a row gives the same bits whatever rows are with it: 16 channels one behind the other; 16 such chunks (256 channels)
// as a tree over their lanes; then the sums of 256, 16 apart one behind the other and the 16 of those as a tree.
#include "fp8.h"

namespace haq {

namespace {

constexpr int NORM_WAVES = 16;             // most waves of a work-group
constexpr int NORM_SUMS = 256;             // sums of 256 channels: K <= 65536 in one row, K <= 16384 in each of four
constexpr int MAX_GROUPS_X = 1 << 20;      // a grid has fewer than 2^32 threads in a direction

template <int CTRL>
__device__ __forceinline__ double lanes_f64(double v) {
    const uint64_t u = __double_as_longlong(v);
    const uint32_t lo = __builtin_amdgcn_mov_dpp((int)(uint32_t)u, CTRL, 0xf, 0xf, true);
    const uint32_t hi = __builtin_amdgcn_mov_dpp((int)(uint32_t)(u >> 32), CTRL, 0xf, 0xf, true);
    return __longlong_as_double((long long)(((uint64_t)hi << 32) | lo));
}

// Sum over each 16 neighbouring lanes, as a tree.  All lanes must be active.
__device__ __forceinline__ double sum_of_16_lanes(double v) {
    v += lanes_f64<HAQ_LANES_XOR1>(v);
    v += lanes_f64<HAQ_LANES_XOR2>(v);
    v += lanes_f64<HAQ_LANES_MIRROR8>(v);
    return v + lanes_f64<HAQ_LANES_MIRROR16>(v);
}

// h = round16(x + residual), eight values.  In binary16 the sum of two values rounds the same at once or by way of binary32
// (24 bits >= 2 * 11 + 2).
template <int DT>
__device__ __forceinline__ uint4 add16(const uint4& x, const uint4& r) {
    if constexpr (DT == HAQ_F16) {
        typedef _Float16 h8 __attribute__((ext_vector_type(8)));
        const h8 s = *reinterpret_cast<const h8*>(&x) + *reinterpret_cast<const h8*>(&r);
        return *reinterpret_cast<const uint4*>(&s);
    } else {
        float a[8], b[8];
        unpack8<DT>(x, a);
        unpack8<DT>(r, b);
#pragma unroll
        for (int i = 0; i < 8; ++i) a[i] = a[i] + b[i];
        return pack8<DT>(a);
    }
}

// A work-group holds RW rows; each of its waves 64 / RW chunks of 16 channels of all of them, a chunk to a lane, NB times; MAXW: its
// most waves, which sets the register budget.  int8 keeps the normalised values across the reduction of the row maximum: normalising
// twice reads the weight twice, which through a CU's load path costs as much as a row (8192 x 8192 bfloat16 without residual and sum 64.5 -> 59.0 us).
template <int DT, int RW, int NB, int MAXW, bool I8>
__global__ __launch_bounds__(MAXW * 64) void rmsnorm_kernel(NormArgs a) {
    constexpr int LPR = 64 / RW;  // lanes of a wave that share a row
    constexpr int MOST = NORM_SUMS / RW;
    __shared__ double sums[RW][MOST];
    __shared__ float maxima[NORM_WAVES][RW];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, nw = blockDim.x >> 6;
    int group = (int)(blockIdx.y * gridDim.x + blockIdx.x);
    if (a.codes) {  // ids go round-robin to the 8 XCDs: the work-groups whose codes share lines go to one of them, whose L2 fills the lines
        constexpr int LINE = 8 / RW;
        const int in = group % (8 * LINE);
        group += (in % 8) * LINE + in / 8 - in;
        if (group * RW >= a.T) return;  // the grid is in whole lines
    }
    const int rl = lane / LPR, row = group * RW + rl;
    const int nchunk = a.K / 16;
    const bool live = row < a.T;
    const size_t r = live ? row : 0;
    auto chunk = [&](int b) { return (b * nw + wave) * LPR + lane % LPR; };

    uint4 h[NB][2];
#pragma unroll
    for (int b = 0; b < NB; ++b) {
        const int c = chunk(b);
        h[b][0] = h[b][1] = make_uint4(0, 0, 0, 0);
        if (live && c < nchunk) {
            const uint4* px = reinterpret_cast<const uint4*>((const uint16_t*)a.x + r * a.ldx + c * 16);
            h[b][0] = px[0];
            h[b][1] = px[1];
        }
    }
    if (a.residual) {
        uint4 s[NB][2];
#pragma unroll
        for (int b = 0; b < NB; ++b) {
            const int c = chunk(b);
            s[b][0] = s[b][1] = make_uint4(0, 0, 0, 0);
            if (live && c < nchunk) {
                const uint4* pr = reinterpret_cast<const uint4*>((const uint16_t*)a.residual + r * a.ldr + c * 16);
                s[b][0] = pr[0];
                s[b][1] = pr[1];
            }
        }
#pragma unroll
        for (int b = 0; b < NB; ++b) {
            h[b][0] = add16<DT>(h[b][0], s[b][0]);
            h[b][1] = add16<DT>(h[b][1], s[b][1]);
        }
    }
    const int nsum = (nchunk + 15) / 16;
#pragma unroll
    for (int b = 0; b < NB; ++b) {
        float v[16];
        unpack8<DT>(h[b][0], v);
        unpack8<DT>(h[b][1], v + 8);
        double ss = 0.0;
#pragma unroll
        for (int i = 0; i < 16; ++i) ss = __builtin_fma((double)v[i], (double)v[i], ss);
        ss = sum_of_16_lanes(ss);
        const int at = chunk(b) / 16;
        if (lane % 16 == 0 && at < nsum) sums[rl][at] = ss;
    }
    __syncthreads();
    // every input has been read: outputs may take the place of x and residual
    if (a.sum && live) {
#pragma unroll
        for (int b = 0; b < NB; ++b) {
            const int c = chunk(b);
            if (c < nchunk) {
                uint4* p = reinterpret_cast<uint4*>((uint16_t*)a.sum + r * a.lds + c * 16);
                p[0] = h[b][0];
                p[1] = h[b][1];
            }
        }
    }
    double ss = lane % 16 < nsum ? sums[rl][lane % 16] : 0.0;
    for (int at = 16; at < nsum; at += 16) ss += at + lane % 16 < nsum ? sums[rl][at + lane % 16] : 0.0;
    ss = sum_of_16_lanes(ss);
    const float inv = (float)(1.0 / sqrt(ss / (double)a.K + a.eps));

    uint32_t top = 0;  // int8: largest magnitude, as bits, so that infinities and NaN (larger yet) show in it
    float keep[I8 ? NB : 1][16];
#pragma unroll
    for (int b = 0; b < NB; ++b) {
        const int c = chunk(b);
        const bool here = live && c < nchunk;
        float(&v)[16] = keep[I8 ? b : 0];
        unpack8<DT>(h[b][0], v);
        unpack8<DT>(h[b][1], v + 8);
        const float4* pg = reinterpret_cast<const float4*>(a.weight + (c < nchunk ? c : 0) * 16);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float4 g = pg[i];
            v[4 * i] = (v[4 * i] * inv) * g.x;
            v[4 * i + 1] = (v[4 * i + 1] * inv) * g.y;
            v[4 * i + 2] = (v[4 * i + 2] * inv) * g.z;
            v[4 * i + 3] = (v[4 * i + 3] * inv) * g.w;
        }
        if (a.y && here) {
            uint4* p = reinterpret_cast<uint4*>((uint16_t*)a.y + r * a.ldy + c * 16);
            p[0] = pack8<DT>(v);
            p[1] = pack8<DT>(v + 8);
        }
        if (I8) {
            if (here) {
#pragma unroll
                for (int i = 0; i < 16; ++i) top = max(top, __float_as_uint(v[i]) & 0x7fffffffu);
            }
        } else if (a.codes == HAQ_CODES_E4M3) {
            const BlockScale s = block_scale(max_of_8_lanes(here ? absmax16(v) : 0.0f));
            if (here) {
                *reinterpret_cast<uint4*>(a.q + ((size_t)c * a.R + row) * 16) = e4m3x16(v, s.r);
                if (c % 8 == 0) a.scale[(size_t)(c / 8) * a.R + row] = s.scale;
            }
        }
    }
    if (!I8) return;
#pragma unroll
    for (int o = 1; o < LPR; o <<= 1) top = max(top, (uint32_t)__shfl_xor((int)top, o));
    if (lane % LPR == 0) maxima[wave][rl] = __uint_as_float(top);
    __syncthreads();
    for (int w = 0; w < nw; ++w) top = max(top, __float_as_uint(maxima[w][rl]));
    const float amax = __uint_as_float(top);
    const bool zero = !(amax >= TINY_MAX && amax < __builtin_inff());
    const float scale = amax < TINY_MAX ? 0.0f : amax / 127.0f, rscale = 1.0f / scale;
    const bool fast = scale >= 0x1p-100f && scale <= 0x1p100f;
    if (live && wave == 0 && lane % LPR == 0) a.scale[row] = scale;
#pragma unroll
    for (int b = 0; b < NB; ++b) {
        const int c = chunk(b);
        float(&v)[16] = keep[I8 ? b : 0];
        uint32_t w[4] = {0, 0, 0, 0};
        if (!zero) {
#pragma unroll
            for (int i = 0; i < 16; ++i) v[i] = fast ? div_by(v[i], scale, rscale, true) : fminf(fmaxf(v[i] / scale, -127.0f), 127.0f);
#pragma unroll
            for (int i = 0; i < 4; ++i) w[i] = round_pack4(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]);
        }
        if (live && c < nchunk) *reinterpret_cast<uint4*>(a.q + ((size_t)c * a.R + row) * 16) = make_uint4(w[0], w[1], w[2], w[3]);
    }
}

template <int DT, int RW, int NB, int MAXW>
int launch_one(const NormArgs& a, int waves, hipStream_t st) {
    const int groups = a.codes ? (int)round_up(cdiv(a.T, RW), 64 / RW) : cdiv(a.T, RW), x = groups < MAX_GROUPS_X ? groups : MAX_GROUPS_X;
    const dim3 grid(x, cdiv(groups, x)), block(waves * 64);
    if (a.codes == HAQ_CODES_I8)
        hipLaunchKernelGGL((rmsnorm_kernel<DT, RW, NB, MAXW, true>), grid, block, 0, st, a);
    else
        hipLaunchKernelGGL((rmsnorm_kernel<DT, RW, NB, MAXW, false>), grid, block, 0, st, a);
    HAQ_CHECK_HIP(hipGetLastError());
    return HAQ_OK;
}

template <int DT, int RW>
int launch_rows(const NormArgs& a, hipStream_t st) {
    const int need = cdiv(a.K / 16, 64 / RW);  // wave-wide pieces of RW rows
    if (need <= 8) return launch_one<DT, RW, 1, 8>(a, need, st);
    if (need <= 16) return launch_one<DT, RW, 2, 8>(a, cdiv(need, 2), st);
    if constexpr (RW == 4) {  // two rows of K <= 16384 never need more
        if (need > 32) return launch_one<DT, RW, 4, 16>(a, cdiv(need, 4), st);
    }
    return launch_one<DT, RW, 4, 8>(a, cdiv(need, 4), st);
}

// One row to a work-group; where there are codes to write, two from 512 rows (two for each CU) on and four from 2048, up to K = 16384.
// us with one row / two / four:
//   rows and the sum, no codes:  777 x 2064 5.3 / 5.5 / 6.0,  8192 x 8192 100 / 105 / 105
//   with e4m3 codes and the sum:  1 x 4096 2.8 / 3.1 / 4.2,  64: 3.1 / 3.5 / 4.5;  700 x 2048 4.7 / 4.8 / 5.0,  1024 x 8192 18.5 / 17.0 / 18.6,
//                     1500 x 6144 20.4 / 18.9 / 20.2,  2048 x 4096 19.0 / 16.9 / 17.2,  8000 x 1040 19.6 / 17.6 / 17.4,  8192 x 8192 129 / 117 / 105
//   with int8 codes and the sum:  512 x 8192 10.9 / 11.8 / 14.5,  1024 x 4096 10.7 / 10.5 / 12.1,  4096 x 8192 58.9 / 55.7 / 59.0;  with rows too:
//                     6000 x 2048 31.4 / 29.0 / 28.9;  without residual and sum:  8192 x 8192 61.4 / 56.0 / 58.5
// (The line from two to four is that of e4m3; int8 gives some 5 % away to it at K = 8192.)
// Eight rows, whole lines without the help of the L2, gain up to 5 % at 4096 x 4096 and lose as much at 8192 x 8192, where they fill
// the registers.  (The work-groups of a line's rows on different XCDs: 256 x 4096 4.9 against 4.3, 8192 x 8192 109 against 104.)
template <int DT>
int launch_type(const NormArgs& a, hipStream_t st) {
    if (a.codes != HAQ_CODES_NONE && a.K <= 16384) {
        if (a.T >= 8 * cu_count()) return launch_rows<DT, 4>(a, st);
        if (a.T >= 2 * cu_count()) return launch_rows<DT, 2>(a, st);
    }
    const int need = cdiv(a.K / 16, 64);
    if (need <= 16) return launch_one<DT, 1, 1, 16>(a, need, st);
    return launch_one<DT, 1, 4, 16>(a, cdiv(need, 4), st);
}

}  // namespace

int launch_rmsnorm(const NormArgs& a, int dtype, hipStream_t st) {
    return dtype == HAQ_F16 ? launch_type<HAQ_F16>(a, st) : launch_type<HAQ_BF16>(a, st);
}

}  // namespace haq
