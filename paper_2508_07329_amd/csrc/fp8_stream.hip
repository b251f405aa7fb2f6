// 8-bit floating-point linear for few token rows: the weights are streamed from HBM once, straight into the operand registers of
// the matrix instructions.
//
// Bound: the weight stream (K N bytes) and, with few of them, the start and the end of a work-group: 1 row of 4096 x 6144 in 6.8 us
// (3.7 TB/s), of 4096 x 65536 in 49 (5.5);  48 rows of 4096 x 14336 in 15 (3.9).  A work-group owns 16 C channels and deals the blocks of 128 input channels to its
// waves in turn; each of them has room for the fragments of DEPTH blocks on their way, and the partial sums are added in LDS, in the
// order of the waves, so that a call repeated gives the same bits.
// Where the rows come as codes the ring is not kept full: the compiler mixes the loads of the first DEPTH blocks, and the wait at the head
// of the loop, which serves its entry and every later trip, holds for the mixed order.  Loads still on their way at a trip's first
// product, and what the order of the blocks would allow: 16 x 16 6 of 20 (15), 16 x 32 4 of 21 (14), 16 x 64 6 of 44 (33), 32 x 32 12 of 40
// (30), 64 x 32 16 of 48 (32), 64 x 64 8 of 40 (20); 32 x 64 and the rows in 16 bits, whose fetch stands between barriers, keep theirs.
#include <mutex>

#include "fp8_gemm_kernel.h"

namespace haq {

namespace {

typedef int v4i __attribute__((ext_vector_type(4)));

__device__ __forceinline__ v4i load16(const void* p) { return *(const __attribute__((address_space(1))) v4i*)(uintptr_t)p; }
__device__ __forceinline__ v4i load16_once(const void* p) { return __builtin_nontemporal_load((const __attribute__((address_space(1))) v4i*)(uintptr_t)p); }

struct Fp8StreamArgs {
    Fp8GemmArgs g;     // A and sa not used where the rows come in 16 bits
    const void* x;
    int64_t ldx;
};

// The codes of a wave's own blocks from rows in 16 bits, into LDS: [block][chunk of 16 channels][row][16] and [block][row] scales.  A
// step covers RW rows of 8 / RW blocks, a chunk to a lane; chunks past K get zeros.
template <int DT, int NW, int RW>
struct BlockQuantiser {
    static constexpr int G = 8 / RW, BATCH = 4;  // blocks of a step; steps whose rows are on their way together
    const Fp8StreamArgs& args;
    int wave, n, steps;
    uint4* codes;
    float* scales;
    uint4 x[BATCH][2];
    __device__ __forceinline__ BlockQuantiser(const Fp8StreamArgs& a, int wave_, int n_, uint4* codes_, float* scales_)
        : args(a), wave(wave_), n(n_), steps((n_ + G - 1) / G), codes(codes_), scales(scales_) {}
    __device__ __forceinline__ void place(int s, int& r, int& k, int& chunk) const {
        const int lane = threadIdx.x & 63;
        r = (lane >> 3) % RW;
        k = s * G + (lane >> 3) / RW;
        chunk = 8 * (wave + k * NW) + (lane & 7);
    }
    __device__ __forceinline__ void fetch(int s0) {
#pragma unroll
        for (int i = 0; i < BATCH; ++i) {
            int r, k, chunk;
            place(min(s0 + i, steps - 1), r, k, chunk);
            const uint16_t* px = (const uint16_t*)args.x + (size_t)min(r, args.g.M - 1) * args.ldx + min(chunk, args.g.K / 16 - 1) * 16;
            x[i][0] = *reinterpret_cast<const uint4*>(px);
            x[i][1] = *reinterpret_cast<const uint4*>(px + 8);
        }
    }
    __device__ __forceinline__ void store(int s0) {
#pragma unroll
        for (int i = 0; i < BATCH; ++i) {
            if (s0 + i >= steps) break;
            int r, k, chunk;
            place(s0 + i, r, k, chunk);
            float v[16];
            unpack8<DT>(x[i][0], v);
            unpack8<DT>(x[i][1], v + 8);
            const bool in = chunk < args.g.K / 16;
            const BlockScale t = block_scale(max_of_8_lanes(in ? absmax16(v) : 0.0f));
            if (k < n) {
                codes[(k * 8 + chunk % 8) * RW + r] = in ? e4m3x16(v, t.r) : make_uint4(0, 0, 0, 0);
                if (chunk % 8 == 0) scales[k * RW + r] = t.scale;
            }
        }
    }
};

// C: blocks of 16 channels; RB: blocks of 16 token rows; NW: waves.  RW > 0: at most RW rows in 16 bits, whose codes every work-group
// forms itself while its first weights are on their way, so that the linear is one launch.  TILES: several row tiles of 16 RB
// rows; work-group ids go round-robin to the 8 XCDs, each of which (one L2) takes a contiguous range of tiles, rows fastest, and
// keeps the weights in its cache.  Weights that one work-group alone reads pass the caches by (non-temporal; 1 row of 4096 x 6144 6.8
// against 7.3 us, 48 of 4096 x 14336 17.7 with the codes' launch against 18.5).
template <int DT, int C, int RB, int NW, int DEPTH, int WPS, int RW, bool TILES>
__global__ __launch_bounds__(NW * 64, WPS) void fp8_stream_kernel(Fp8StreamArgs args, int mt) {
    const Fp8GemmArgs& a = args.g;
    static_assert(RW == 0 || (RB == 1 && !TILES), "a few rows");
    extern __shared__ __attribute__((aligned(16))) int8_t lds[];
    float(*sum)[C * RB][4][64] = reinterpret_cast<float(*)[C * RB][4][64]>(lds);  // [NW]
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), l16 = lane & 15, q = lane >> 4;
    int unit = blockIdx.x, row0 = 0;
    if (TILES) {
        const int total = mt * ((a.N + 16 * C - 1) / (16 * C)), per = (total + 7) / 8, slot = blockIdx.x / 8, id = (int)(blockIdx.x % 8) * per + slot;
        if (slot >= per || id >= total) return;
        unit = id / mt;
        row0 = id % mt * 16 * RB;
    }
    const int n0 = unit * 16 * C;
    const int nb = (a.K + FP8_BLOCK - 1) / FP8_BLOCK, nn = (a.N + FP8_BLOCK - 1) / FP8_BLOCK, nchunk = a.K / 16;
    const int n = nb > wave ? (nb - wave + NW - 1) / NW : 0, most = (nb + NW - 1) / NW;  // this wave's blocks: wave, wave + NW, ...
    uint4* codes = reinterpret_cast<uint4*>(lds + NW * C * RB * 1024) + (size_t)wave * most * 8 * RW;
    float* scales = reinterpret_cast<float*>(reinterpret_cast<uint4*>(lds + NW * C * RB * 1024) + (size_t)NW * most * 8 * RW) + wave * most * RW;

    struct Frag {
        v4i w[C][2], x[RW ? 1 : RB][2];
        float sa[RW ? 1 : RB], sw;
    } fr[DEPTH];
    int row[RB];  // rows past the last one re-read it (their results are dropped)
#pragma unroll
    for (int r = 0; r < RB; ++r) row[r] = min(row0 + 16 * r + l16, a.M - 1);
    int fetched = 0;  // loads stay unconditional: past this wave's last block they re-read it; chunks past K re-read the last one
    auto next = [&](Frag& f) {
        const int b = wave + min(fetched, n - 1) * NW;
        ++fetched;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int c = min(8 * b + 2 * q + h, nchunk - 1);
            const uint8_t* pw = a.B + ((size_t)c * a.Npad + n0 + l16) * 16;
#pragma unroll
            for (int j = 0; j < C; ++j) f.w[j][h] = TILES ? load16(pw + j * 256) : load16_once(pw + j * 256);
            if constexpr (RW == 0) {
#pragma unroll
                for (int r = 0; r < RB; ++r) f.x[r][h] = load16(a.A + ((size_t)c * a.R + row[r]) * 16);
            }
        }
        if constexpr (RW == 0) {
#pragma unroll
            for (int r = 0; r < RB; ++r) f.sa[r] = a.sa[(size_t)b * a.R + row[r]];
        }
        f.sw = a.sb[(size_t)b * nn + n0 / FP8_BLOCK];
    };
    v4f acc[C][RB];
#pragma unroll
    for (int j = 0; j < C; ++j)
#pragma unroll
        for (int r = 0; r < RB; ++r) acc[j][r] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
    auto mac = [&](const Frag& f, int k) {
#pragma unroll
        for (int r = 0; r < RB; ++r) {
            v4i x[2];
            float s;
            if constexpr (RW > 0) {
#pragma unroll
                for (int h = 0; h < 2; ++h) x[h] = *reinterpret_cast<const v4i*>(codes + (k * 8 + 2 * q + h) * RW + row[r]);
                s = scales[k * RW + row[r]] * f.sw;
            } else {  // tokens' chunks past K count as zeros, whatever was re-read for the weights'
                const v4i zero = {0, 0, 0, 0};
                const int c = 8 * (wave + k * NW) + 2 * q;
                x[0] = c < nchunk ? f.x[r][0] : zero;
                x[1] = c + 1 < nchunk ? f.x[r][1] : zero;
                s = f.sa[r] * f.sw;
            }
            const v8i xf = __builtin_shufflevector(x[0], x[1], 0, 1, 2, 3, 4, 5, 6, 7);
#pragma unroll
            for (int j = 0; j < C; ++j) {
                const v4f p = mfma_e4m3(__builtin_shufflevector(f.w[j][0], f.w[j][1], 0, 1, 2, 3, 4, 5, 6, 7), xf, v4f{0.0f, 0.0f, 0.0f, 0.0f});
#pragma unroll
                for (int i = 0; i < 4; ++i) acc[j][r][i] = __builtin_fmaf(s, p[i], acc[j][r][i]);
            }
        }
    };
    if (n > 0) {
        auto first = [&](auto&& fetch_weights) {  // the rows' loads in front of the weights' (loads return in order), their use behind
            if constexpr (RW > 0) {
                BlockQuantiser<DT, NW, RW> quant(args, wave, n, codes, scales);
                quant.fetch(0);
                __builtin_amdgcn_sched_barrier(0);
                fetch_weights();
                __builtin_amdgcn_sched_barrier(0);
                quant.store(0);
                for (int s = quant.BATCH; s < quant.steps; s += quant.BATCH) {
                    quant.fetch(s);
                    quant.store(s);
                }
                HAQ_FP8_FENCE();  // the wave reads what its own lanes have written: LDS serves its requests in order
                __builtin_amdgcn_wave_barrier();
            } else {
                fetch_weights();
            }
        };
        if (n < DEPTH) {
            first([&] {
#pragma unroll
                for (int i = 0; i < DEPTH - 1; ++i)
                    if (i < n) next(fr[i]);
            });
#pragma unroll
            for (int i = 0; i < DEPTH - 1; ++i)
                if (i < n) mac(fr[i], i);
        } else {
            first([&] {
#pragma unroll
                for (int i = 0; i < DEPTH; ++i) next(fr[i]);
            });
            int k = 0;
            for (; k + DEPTH < n; k += DEPTH) {
#pragma unroll
                for (int i = 0; i < DEPTH; ++i) {
                    mac(fr[i], k + i);
                    next(fr[i]);
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
#pragma unroll
            for (int i = 0; i < DEPTH; ++i)
                if (k + i < n) mac(fr[i], k + i);
        }
    }
#pragma unroll
    for (int j = 0; j < C; ++j)
#pragma unroll
        for (int r = 0; r < RB; ++r)
#pragma unroll
            for (int i = 0; i < 4; ++i) sum[wave][j * RB + r][i][lane] = acc[j][r][i];
    __syncthreads();
    for (int i = tid; i < C * RB * 64; i += NW * 64) {
        const int jr = i >> 6, ln = i & 63, t = row0 + 16 * (jr % RB) + (ln & 15), ch = n0 + 16 * (jr / RB) + 4 * (ln >> 4);
        if (t >= a.M || ch >= a.N) continue;
        float v[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            v[e] = sum[0][jr][e][ln];
#pragma unroll
            for (int w = 1; w < NW; ++w) v[e] += sum[w][jr][e][ln];
            if (a.act == HAQ_ACT_RELU && v[e] < 0.0f) v[e] = 0.0f;
        }
        *reinterpret_cast<uint2*>((uint16_t*)a.Y + (size_t)t * a.ldy + ch) = make_uint2(pack2<DT>(v[0], v[1]), pack2<DT>(v[2], v[3]));
    }
}

template <int DT, int C, int RB, int NW, int DEPTH, int WPS, int RW, bool TILES = false>
int launch_one(const Fp8StreamArgs& a, hipStream_t st) {
    auto kern = fp8_stream_kernel<DT, C, RB, NW, DEPTH, WPS, RW, TILES>;
    const int bytes = NW * C * RB * 1024 + RW * (int)round_up(a.g.K, NW * FP8_BLOCK) * (FP8_BLOCK + 4) / FP8_BLOCK;
    const int mt = TILES ? cdiv(a.g.M, 16 * RB) : 1, units = cdiv(a.g.N, 16 * C);
    static std::once_flag once;
    static hipError_t attr_err = hipSuccess;
    std::call_once(once, [&] { attr_err = hipFuncSetAttribute((const void*)kern, hipFuncAttributeMaxDynamicSharedMemorySize, 160 * 1024); });
    HAQ_CHECK_HIP(attr_err);
    const unsigned grid = TILES ? (unsigned)round_up((int64_t)mt * units, 8) : (unsigned)units;
    hipLaunchKernelGGL(kern, dim3(grid), dim3(NW * 64), bytes, st, a, mt);
    HAQ_CHECK_HIP(hipGetLastError());
    return HAQ_OK;
}

// Blocks of 16 channels to a work-group where it forms the rows' codes itself.  One: two work-groups share a CU and overlap start and
// end; four: the codes are formed once for four times the channels, in fewer rounds.  us with one / two / four, weights cold:
//   1 row:   1024 x 2048 2.9 / 3.1 / 3.8,  4096 x 4096 5.3 / 5.9 / 9.5,  4096 x 6144 7.4 / 6.8 / 10.5,  4096 x 8208 8.6 / 11.2 / 11.4,
//            4096 x 14336 13.0 / 13.4 / 14.1,  4096 x 65536 49 / 56 / 68,  8192 x 28672 44 / 43 / 42,  1024 x 16384 6.4 / 6.1 / 5.3
//   4 rows:  4096 x 8208 9.2 / 11.8 / 11.3,  4096 x 14336 14.0 / 14.1 / 14.0,  4096 x 65536 52 / 59 / 66,  1024 x 131072 40 / 39 / 34
//   8 rows:  4096 x 8208 10.2 / 12.0 / 11.7,  4096 x 14336 15.2 / 14.0 / 14.2,  8192 x 28672 51 / 48 / 43,  1024 x 131072 46 / 37 / 35
// (One row of long K on wide layers lies close: at 8192 x 28672 the line gives 2 us of 44 away, at 4096 x 65536 it gains 19 of 68.)
int channel_blocks(int M, int K, int N) {
    const int n_cu = cu_count();
    if (N <= 32 * n_cu) return N > 16 * n_cu ? 2 : 1;
    return K >= 2048 && (M <= 4 || N <= 40 * n_cu) ? 1 : 4;
}

template <int DT, int RW>
int launch_rows16(const Fp8StreamArgs& a, hipStream_t st) {
    switch (channel_blocks(a.g.M, a.g.K, a.g.N)) {
        case 4: return launch_one<DT, 4, 1, 8, 3, 2, RW>(a, st);
        case 2: return launch_one<DT, 2, 1, 8, 4, 2, RW>(a, st);
        default: return launch_one<DT, 1, 1, 8, 4, 4, RW>(a, st);
    }
}
// Room for 1, 2, 4 or 8 rows: fewer rows of 8 in vain (4096 x 6144, room for 8 instead: 1 row 6.8 -> 7.1 us, 2 7.0 -> 7.2, 4 7.0 -> 7.2)
// and longer ones in the same LDS.
template <int DT>
int launch_rows16(const Fp8StreamArgs& a, hipStream_t st) {
    if (a.g.M <= 1) return launch_rows16<DT, 1>(a, st);
    if (a.g.M <= 2) return launch_rows16<DT, 2>(a, st);
    if (a.g.M <= 4) return launch_rows16<DT, 4>(a, st);
    return launch_rows16<DT, 8>(a, st);
}

template <int DT, int RB, int C, int DEPTH, int WPS>
int launch_codes(const Fp8StreamArgs& a, hipStream_t st) {
    return a.g.M <= 16 * RB ? launch_one<DT, C, RB, 8, DEPTH, WPS, 0, false>(a, st) : launch_one<DT, C, RB, 8, DEPTH, WPS, 0, true>(a, st);
}
template <int DT>
int launch_codes(const Fp8StreamArgs& a, int RB, int C, hipStream_t st) {
    switch (RB * 8 + C) {
        case 1 * 8 + 1: return launch_codes<DT, 1, 1, 4, 4>(a, st);
        case 1 * 8 + 2: return launch_codes<DT, 1, 2, 3, 4>(a, st);
        case 1 * 8 + 4: return launch_codes<DT, 1, 4, 4, 2>(a, st);
        case 2 * 8 + 2: return launch_codes<DT, 2, 2, 4, 2>(a, st);
        case 2 * 8 + 4: return launch_codes<DT, 2, 4, 4, 2>(a, st);
        case 4 * 8 + 2: return launch_codes<DT, 4, 2, 3, 2>(a, st);
        case 4 * 8 + 4: return launch_codes<DT, 4, 4, 2, 2>(a, st);
        default: return HAQ_ERR_UNSUPPORTED;
    }
}

}  // namespace

// At most 8 rows in 16 bits whose codes fit 64 KB of LDS: codes and linear in one launch.  us in one / in two, weights cold:  1 row of
// 4096 x 4096 5.3 / 7.5, of 4096 x 6144 6.8 / 9.7;  8 rows of 1024 x 2048 3.1 / 4.9, of 4096 x 4096 6.1 / 7.7, of 4096 x 14336 14.2 / 14.2;
// 4 of 14336 x 4096 13.8 / 15.3.  (16 rows of 4096 x 6144 9.1 / 9.0: the vector units of every work-group round all of the rows.)
bool fp8_stream_rows16_fits(int M, int K) { return M >= 1 && M <= 8 && (M <= 2 ? M : M <= 4 ? 4 : 8) * round_up(K, 1024) <= 65536; }
int launch_fp8_stream_rows16(const Fp8GemmArgs& a, const void* x, int64_t ldx, int dtype, hipStream_t st) {
    const Fp8StreamArgs s{a, x, ldx};
    return dtype == HAQ_F16 ? launch_rows16<HAQ_F16>(s, st) : launch_rows16<HAQ_BF16>(s, st);
}

int launch_fp8_stream(const Fp8GemmArgs& a, int row_blocks, int channel_blocks, int dtype, hipStream_t st) {
    const Fp8StreamArgs s{a, nullptr, 0};
    return dtype == HAQ_F16 ? launch_codes<HAQ_F16>(s, row_blocks, channel_blocks, st) : launch_codes<HAQ_BF16>(s, row_blocks, channel_blocks, st);
}

}  // namespace haq
