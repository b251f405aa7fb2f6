// Linear on e4m3 codes with a scale for 128 channels of a token and for 128 x 128 of the weights:
//   y[t][n] = round16(act(sum_b (sa[b][t] sb[b][n / 128]) p_b)),  p_b = sum over the 128 channels k of block b of a[t][k] w[k][n].
// Launcher: the streaming kernel for few rows, else a tile shape.
#include <mutex>

#include "fp8_gemm_kernel.h"

namespace haq {

namespace {

template <int DT, int BM, int BN, int WAVES_M, int WAVES_N, int STAGES, int KG, int MINB>
int launch_tiles(const Fp8GemmArgs& a, hipStream_t st) {
    using S = Fp8Shape<BM, BN, WAVES_M, WAVES_N, STAGES, KG>;
    static_assert(MINB * S::LDS_BYTES <= 160 * 1024, "the LDS of a CU");
    auto kern = fp8_gemm_kernel<DT, BM, BN, WAVES_M, WAVES_N, STAGES, KG, (MINB * KG * S::NW + 3) / 4>;
    static std::once_flag once;
    static hipError_t attr_err = hipSuccess;
    std::call_once(once, [&] { attr_err = hipFuncSetAttribute((const void*)kern, hipFuncAttributeMaxDynamicSharedMemorySize, S::LDS_BYTES); });
    HAQ_CHECK_HIP(attr_err);
    const int tiles = cdiv(a.M, BM) * cdiv(a.N, BN);
    hipLaunchKernelGGL(kern, dim3((unsigned)round_up(tiles, 8)), dim3(S::THREADS), S::LDS_BYTES, st, a, tiles);
    HAQ_CHECK_HIP(hipGetLastError());
    return HAQ_OK;
}

template <int DT>
int launch_halves(const Fp8GemmArgs& a, hipStream_t st) {
    using S = Fp8Shape<256, 256, 4, 2, 2, 1>;
    using Half = Fp8Shape<256, 128, 4, 2, 2, 1>;
    static_assert(Half::LDS_BYTES <= S::LDS_BYTES && Half::THREADS == S::THREADS && S::THREADS == 512, "one launch for both");
    auto kern = fp8_gemm_halves_kernel<DT>;
    static std::once_flag once;
    static hipError_t attr_err = hipSuccess;
    std::call_once(once, [&] { attr_err = hipFuncSetAttribute((const void*)kern, hipFuncAttributeMaxDynamicSharedMemorySize, S::LDS_BYTES); });
    HAQ_CHECK_HIP(attr_err);
    const int tiles = cdiv(a.M, 256) * cdiv(a.N, 256), whole = tiles - tiles % cu_count();
    const int64_t groups = round_up(whole, 8) + round_up(2 * (tiles - whole), 8);
    hipLaunchKernelGGL(kern, dim3((unsigned)groups), dim3(S::THREADS), S::LDS_BYTES, st, a, whole, tiles);
    HAQ_CHECK_HIP(hipGetLastError());
    return HAQ_OK;
}

// Estimated us of a launch of T tiles on C compute units.  A round is per_cu C tiles; one of n tiles, k = ceil(n / C) to a CU, takes
// fix + K-steps step: fix between fix[0] and fix[1] in proportion to n / (per_cu C), step between step[k-1][0] (a CU alone) and
// step[k-1][1] (every CU busy) in proportion to n / (k C).  Full rounds before the last one overlap (`round` of that each); the
// last one costs its share of a full round and, as far as `tail` goes, what it takes alone.
struct Fp8TileShape {
    int bm, bn, per_cu;
    float fix[2], step[2][2], round, tail;
};
// S_..: the streaming kernel (rows x channels; K split over eight waves; operands straight into registers: a third of the others'
// time for a K-step, of far smaller tiles).  T_..: the tiled kernel.
enum { S16x16, S16x32, S16x64, S32x32, S32x64, S64x32, S64x64, T64x128, T64x128K2, T128x128, T256x128, T256x256, N_FP8_TILES, H256x256 = N_FP8_TILES };
// Fitted to 1600 problems (9 to 4096 rows, layers of 256 to 16384 input and output channels, both spread over their logarithm; weights cold;
// 1113 to 1445 launches of each shape, mean deviation 1 to 8 %).  The shape with the lowest estimate is on average 0.8 % slower than the
// fastest of these and five more (128 x 128 of four waves, with two groups or twice to a CU, 64 x 64 of four in two groups, streaming
// 32 x 16); over 10 % at 43 problems.  Without T128x128 0.9 % more, without T64x128K2 1.8, without S64x32 1.5.
// us, the best streaming / the best tiled shape:  16 rows of 4096 x 14336 12.5 / 20.4,  48: 15.4 / 20.1,  64 of 14336 x 4096 20.7 / 46.7,  128 of
// 4096 x 14336 25.5 / 20.5,  256: 44 / 24.6,  333 of 2064 x 8208 22.9 / 13.5,  328 of 10048 x 8640 79 / 45,  1866 of 10784 x 272 24.2 / 27.3
// and among the tiled shapes (64 x 128, two groups / 128 x 128 / 256 x 128 / 256 x 256):  1295 rows of 10432 x 944 28.5 / 39.6 / 60 / 92,
// 443 of 16000 x 5456 87 / 67 / 90 / 155,  4096 of 4096 x 4096 118 / 86 / 72 / 57,  8192 of 8192 x 8192 819 / 607 / 504 / 404.
constexpr Fp8TileShape FP8_TILES[N_FP8_TILES] = {
    {16, 16, 2, {2.230f, 2.056f}, {{0.0661f, 0.0780f}, {0.0875f, 0.1461f}}, 0.600f, 0.776f},
    {16, 32, 2, {2.269f, 2.080f}, {{0.0784f, 0.1053f}, {0.0968f, 0.2261f}}, 0.600f, 0.751f},
    {16, 64, 1, {2.396f, 2.245f}, {{0.1140f, 0.2036f}}, 0.622f, 0.921f},
    {32, 32, 1, {2.456f, 2.344f}, {{0.1055f, 0.1554f}}, 0.665f, 0.973f},
    {32, 64, 1, {2.614f, 2.739f}, {{0.1483f, 0.2536f}}, 0.650f, 0.916f},
    {64, 32, 1, {2.821f, 2.406f}, {{0.1265f, 0.2120f}}, 0.740f, 0.937f},
    {64, 64, 1, {3.209f, 3.111f}, {{0.1781f, 0.3091f}}, 0.728f, 1.000f},
    {64, 128, 2, {3.212f, 4.309f}, {{0.3372f, 0.4454f}, {0.3535f, 0.7963f}}, 0.707f, 0.883f},
    {64, 128, 1, {4.006f, 4.271f}, {{0.2827f, 0.4028f}}, 0.792f, 0.972f},
    {128, 128, 1, {3.795f, 4.360f}, {{0.4113f, 0.5658f}}, 0.826f, 0.977f},
    {256, 128, 1, {5.120f, 5.893f}, {{0.5883f, 0.8930f}}, 0.909f, 0.966f},
    {256, 256, 1, {6.432f, 8.591f}, {{1.0096f, 1.4343f}}, 0.940f, 0.899f},
};
float tile_us(const Fp8TileShape& t, int64_t tiles, int nk, int n_cu) {
    const int64_t round = (int64_t)t.per_cu * n_cu;
    auto one_round = [&](int n) {
        const int k = cdiv(n, n_cu);
        const float* step = t.step[k - 1];
        return t.fix[0] + (t.fix[1] - t.fix[0]) * (float)n / (float)round + (float)nk * (step[0] + (step[1] - step[0]) * (float)n / (float)(k * n_cu));
    };
    if (tiles <= round) return one_round((int)tiles);
    const float full_us = one_round((int)round);
    const int rem = (int)(tiles % round);
    const float share = full_us * (float)rem / (float)round;
    return (float)(tiles / round) * full_us * t.round + share + (rem ? t.tail * (one_round(rem) - share) : 0.0f);
}
// H256x256: whole rounds of 256 x 256 and the tiles behind them in halves, where those are one round at most.  They wait for the
// whole ones to end and have 2 stages in place of 3: 1.2 times what 256 x 128 takes alone.  Of 150 sizes near the line the estimate is 0.1 %
// off the best; without the halves 5.3 %.
int fastest_shape(const Fp8GemmArgs& a) {
    const int n_cu = cu_count(), nk = cdiv(a.K, FP8_BLOCK);
    int best = T256x256;
    float best_us = 0.0f;
    for (int i = N_FP8_TILES - 1; i >= 0; --i) {
        const Fp8TileShape& t = FP8_TILES[i];
        const int64_t tiles = (int64_t)cdiv(a.M, t.bm) * cdiv(a.N, t.bn), rest = tiles % n_cu;
        if (i <= S64x64 && tiles > 4 * t.per_cu * n_cu) continue;  // streaming tiles in many rounds were hardly measured, and never the fastest
        const float us = tile_us(t, tiles, nk, n_cu);
        if (i == T256x256 || us < best_us) best = i, best_us = us;
        if (i == T256x256 && tiles > n_cu && rest && 2 * rest <= n_cu) {
            const float h = tile_us(t, tiles - rest, nk, n_cu) + 1.2f * tile_us(FP8_TILES[T256x128], 2 * rest, nk, n_cu);
            if (h < best_us) best = H256x256, best_us = h;
        }
    }
    return best;
}

template <int DT>
int launch_type(const Fp8GemmArgs& a, hipStream_t st) {
    const int shape = fastest_shape(a);
    if (shape <= S64x64) return launch_fp8_stream(a, FP8_TILES[shape].bm / 16, FP8_TILES[shape].bn / 16, DT, st);
    switch (shape) {
        case T64x128: return launch_tiles<DT, 64, 128, 2, 2, 3, 1, 2>(a, st);    // wave tile 32 x 64
        case T64x128K2: return launch_tiles<DT, 64, 128, 2, 2, 3, 2, 1>(a, st);  // 32 x 64, two groups of waves
        case T128x128: return launch_tiles<DT, 128, 128, 4, 2, 4, 1, 1>(a, st);  // 32 x 64
        case T256x128: return launch_tiles<DT, 256, 128, 4, 2, 3, 1, 1>(a, st);  // 64 x 64
        case T256x256: return launch_tiles<DT, 256, 256, 4, 2, 2, 1, 1>(a, st);  // 64 x 128
        default: return launch_halves<DT>(a, st);
    }
}

}  // namespace

int launch_fp8_gemm(const Fp8GemmArgs& a, int dtype, hipStream_t st) {
    return dtype == HAQ_F16 ? launch_type<HAQ_F16>(a, st) : launch_type<HAQ_BF16>(a, st);
}

}  // namespace haq
