// C ABI entry points of the 8-bit floating-point linear and of the root-mean-square norm with codes as output: argument
// validation on the host, workspace carving and launches.
#include <cmath>

#include "fp8.h"

namespace haq {
namespace {

constexpr int MAX_K = 65536, MAX_ROWS = 1 << 24;  // a K-step of 128 channels of all rows or channels keeps its offsets in 32 bits
constexpr int64_t MAX_OUT = (int64_t)1 << 38;     // a launch has fewer than 2^32 threads

int64_t act_rows(int T) { return round_up(T, 16) + 256; }
size_t codes_bytes(int T, int K) { return (size_t)round_up(K, 64) * act_rows(T); }
size_t scales_bytes(int T, int K) { return (size_t)cdiv(K, FP8_BLOCK) * act_rows(T) * sizeof(float); }
size_t scales_at(int T, int K) { return (size_t)round_up((int64_t)codes_bytes(T, K), 256); }  // in the linear's workspace

int check_rows(const char* name, int T, int K, int dtype) {
    if (T < 0 || K <= 0) HAQ_FAIL(HAQ_ERR_INVALID_ARG, "%s: T=%d K=%d", name, T, K);
    if (K % 16 != 0 || K > MAX_K || T > MAX_ROWS)
        HAQ_FAIL(HAQ_ERR_UNSUPPORTED, "%s: K=%d must be a multiple of 16 (<= %d), T=%d at most %d", name, K, MAX_K, T, MAX_ROWS);
    if (dtype != HAQ_F16 && dtype != HAQ_BF16) HAQ_FAIL(HAQ_ERR_UNSUPPORTED, "%s: dtype=%d", name, dtype);
    return HAQ_OK;
}
int check_linear(const char* name, int T, int K, int N, int act, int dtype) {
    if (const int rc = check_rows(name, T, K, dtype)) return rc;
    if (N <= 0) HAQ_FAIL(HAQ_ERR_INVALID_ARG, "%s: N=%d", name, N);
    if (N % 16 != 0 || N > MAX_ROWS) HAQ_FAIL(HAQ_ERR_UNSUPPORTED, "%s: N=%d must be a multiple of 16, at most %d", name, N, MAX_ROWS);
    if ((int64_t)T * N > MAX_OUT) HAQ_FAIL(HAQ_ERR_UNSUPPORTED, "%s: T=%d N=%d: more than 2^38 outputs", name, T, N);
    if (act != HAQ_ACT_NONE && act != HAQ_ACT_RELU) HAQ_FAIL(HAQ_ERR_UNSUPPORTED, "%s: act=%d", name, act);
    return HAQ_OK;
}

Fp8GemmArgs gemm_args(const uint8_t* q, const float* sa, const uint8_t* w, const float* sb, int T, int K, int N, int act, void* y, int64_t ldy) {
    Fp8GemmArgs a{};
    a.A = q;
    a.R = act_rows(T);
    a.sa = sa;
    a.B = w;
    a.Npad = round_up(N, NPAD);
    a.sb = sb;
    a.M = T;
    a.K = K;
    a.N = N;
    a.act = act;
    a.Y = y;
    a.ldy = ldy;
    return a;
}

}  // namespace
}  // namespace haq

using namespace haq;

extern "C" {

int32_t haq_quant_weight_fp8(const float* w, int32_t K, int32_t N, uint8_t* wq, float* w_scale, void* stream) {
    if (K <= 0 || N <= 0) HAQ_FAIL(HAQ_ERR_INVALID_ARG, "haq_quant_weight_fp8: K=%d N=%d", K, N);
    if (K % 16 != 0 || K > MAX_K || N % 16 != 0 || N > MAX_ROWS)
        HAQ_FAIL(HAQ_ERR_UNSUPPORTED, "haq_quant_weight_fp8: K=%d (<= %d) and N=%d must be multiples of 16", K, MAX_K, N);
    if (!w || !wq || !w_scale) HAQ_FAIL(HAQ_ERR_INVALID_ARG, "haq_quant_weight_fp8: null buffer");
    if (!aligned16(w) || !aligned16(wq) || !aligned16(w_scale)) HAQ_FAIL(HAQ_ERR_INVALID_ARG, "haq_quant_weight_fp8: pointers must be 16-byte aligned");
    return launch_weight_quant_fp8(w, K, N, wq, w_scale, (hipStream_t)stream);
}

size_t haq_act_scales_fp8_bytes(int32_t T, int32_t K) { return T < 0 || K <= 0 ? 0 : scales_bytes(T, K); }

int32_t haq_quant_act_fp8_packed(const void* x, int64_t ldx, int32_t dtype, int32_t T, int32_t K, uint8_t* q_packed, float* block_scale,
                                 void* stream) {
    if (const int rc = check_rows("haq_quant_act_fp8_packed", T, K, dtype)) return rc;
    if (T == 0) return HAQ_OK;
    if (!x || !q_packed || !block_scale) HAQ_FAIL(HAQ_ERR_INVALID_ARG, "haq_quant_act_fp8_packed: null buffer");
    if (ldx < K || ldx % 8 != 0) HAQ_FAIL(HAQ_ERR_INVALID_ARG, "haq_quant_act_fp8_packed: ldx=%lld (multiple of 8)", (long long)ldx);
    if (!aligned16(x) || !aligned16(q_packed) || !aligned16(block_scale))
        HAQ_FAIL(HAQ_ERR_INVALID_ARG, "haq_quant_act_fp8_packed: pointers must be 16-byte aligned");
    return launch_act_quant_fp8({x, ldx, T, K, q_packed, act_rows(T), block_scale}, dtype, (hipStream_t)stream);
}

int32_t haq_gemm_fp8_packed(const uint8_t* q_packed, const float* block_scale, const uint8_t* w_packed, const float* w_scale, int32_t T,
                            int32_t K, int32_t N, int32_t act, int32_t dtype, void* y, int64_t ldy, void* stream) {
    if (const int rc = check_linear("haq_gemm_fp8_packed", T, K, N, act, dtype)) return rc;
    if (T == 0) return HAQ_OK;
    if (!q_packed || !block_scale || !w_packed || !w_scale || !y) HAQ_FAIL(HAQ_ERR_INVALID_ARG, "haq_gemm_fp8_packed: null buffer");
    if (ldy < N || ldy % 8 != 0) HAQ_FAIL(HAQ_ERR_INVALID_ARG, "haq_gemm_fp8_packed: ldy=%lld (multiple of 8)", (long long)ldy);
    if (!aligned16(q_packed) || !aligned16(block_scale) || !aligned16(w_packed) || !aligned16(w_scale) || !aligned16(y))
        HAQ_FAIL(HAQ_ERR_INVALID_ARG, "haq_gemm_fp8_packed: pointers must be 16-byte aligned");
    return launch_fp8_gemm(gemm_args(q_packed, block_scale, w_packed, w_scale, T, K, N, act, y, ldy), dtype, (hipStream_t)stream);
}

size_t haq_fp8_linear_workspace_bytes(int32_t T, int32_t K, int32_t N) {
    (void)N;
    return T < 0 || K <= 0 ? 0 : scales_at(T, K) + scales_bytes(T, K);
}

int32_t haq_fp8_linear(const void* x, int64_t ldx, int32_t dtype, const uint8_t* w_packed, const float* w_scale, int32_t T, int32_t K,
                       int32_t N, int32_t act, void* y, int64_t ldy, void* workspace, size_t workspace_bytes, void* stream) {
    if (const int rc = check_linear("haq_fp8_linear", T, K, N, act, dtype)) return rc;
    if (T == 0) return HAQ_OK;
    if (!x || !w_packed || !w_scale || !y) HAQ_FAIL(HAQ_ERR_INVALID_ARG, "haq_fp8_linear: null buffer");
    if (ldx < K || ldx % 8 != 0 || ldy < N || ldy % 8 != 0)
        HAQ_FAIL(HAQ_ERR_INVALID_ARG, "haq_fp8_linear: ldx=%lld ldy=%lld (multiples of 8)", (long long)ldx, (long long)ldy);
    if (!aligned16(x) || !aligned16(w_packed) || !aligned16(w_scale) || !aligned16(y))
        HAQ_FAIL(HAQ_ERR_INVALID_ARG, "haq_fp8_linear: pointers must be 16-byte aligned");
    const size_t need = scales_at(T, K) + scales_bytes(T, K);
    if (!workspace || workspace_bytes < need || ((uintptr_t)workspace & 255u))
        HAQ_FAIL(HAQ_ERR_WORKSPACE, "haq_fp8_linear: workspace of %zu bytes (256-byte aligned) needed, got %zu", need, workspace_bytes);
    uint8_t* q = (uint8_t*)workspace;
    float* sa = (float*)(q + scales_at(T, K));
    const Fp8GemmArgs a = gemm_args(q, sa, w_packed, w_scale, T, K, N, act, y, ldy);
    // In the one launch some work-groups read x while others store y: not where the two overlap (their rows may lie side by side).
    const uintptr_t xb = (uintptr_t)x, xe = xb + ((size_t)(T - 1) * ldx + K) * 2, yb = (uintptr_t)y, ye = yb + ((size_t)(T - 1) * ldy + N) * 2;
    if (fp8_stream_rows16_fits(T, K) && (xe <= yb || ye <= xb)) return launch_fp8_stream_rows16(a, x, ldx, dtype, (hipStream_t)stream);
    if (const int rc = launch_act_quant_fp8({x, ldx, T, K, q, act_rows(T), sa}, dtype, (hipStream_t)stream)) return rc;
    return launch_fp8_gemm(a, dtype, (hipStream_t)stream);
}

int32_t haq_rmsnorm_quant(const void* x, int64_t ldx, const void* residual, int64_t ldr, const float* weight, double eps, int32_t dtype,
                          int32_t T, int32_t K, void* sum, int64_t lds, void* y, int64_t ldy, int32_t codes, void* q_packed, float* scale,
                          void* stream) {
    if (const int rc = check_rows("haq_rmsnorm_quant", T, K, dtype)) return rc;
    if (codes != HAQ_CODES_NONE && codes != HAQ_CODES_I8 && codes != HAQ_CODES_E4M3) HAQ_FAIL(HAQ_ERR_UNSUPPORTED, "haq_rmsnorm_quant: codes=%d", codes);
    if (!(eps >= 1e-30 && eps <= 1e30)) HAQ_FAIL(HAQ_ERR_INVALID_ARG, "haq_rmsnorm_quant: eps=%g outside [1e-30, 1e30]", eps);
    if (T == 0) return HAQ_OK;
    const bool coded = codes != HAQ_CODES_NONE;
    if (!x || !weight) HAQ_FAIL(HAQ_ERR_INVALID_ARG, "haq_rmsnorm_quant: null buffer");
    if (coded != (q_packed != nullptr) || coded != (scale != nullptr))
        HAQ_FAIL(HAQ_ERR_INVALID_ARG, "haq_rmsnorm_quant: codes=%d with q_packed=%p scale=%p", codes, q_packed, (void*)scale);
    if (!coded && !y) HAQ_FAIL(HAQ_ERR_INVALID_ARG, "haq_rmsnorm_quant: neither y nor codes asked for");
    if (sum && !residual) HAQ_FAIL(HAQ_ERR_INVALID_ARG, "haq_rmsnorm_quant: sum without a residual");
    auto bad_ld = [&](const void* p, int64_t ld) { return p && (ld < K || ld % 8 != 0); };
    if (bad_ld(x, ldx) || bad_ld(residual, ldr) || bad_ld(sum, lds) || bad_ld(y, ldy))
        HAQ_FAIL(HAQ_ERR_INVALID_ARG, "haq_rmsnorm_quant: row strides %lld %lld %lld %lld (multiples of 8, at least K)", (long long)ldx, (long long)ldr,
                 (long long)lds, (long long)ldy);
    if (!aligned16(x) || !aligned16(residual) || !aligned16(weight) || !aligned16(sum) || !aligned16(y) || !aligned16(q_packed) || !aligned16(scale))
        HAQ_FAIL(HAQ_ERR_INVALID_ARG, "haq_rmsnorm_quant: pointers must be 16-byte aligned");
    NormArgs a{};
    a.x = x;
    a.residual = residual;
    a.weight = weight;
    a.ldx = ldx;
    a.ldr = ldr;
    a.lds = lds;
    a.ldy = ldy;
    a.sum = sum;
    a.y = y;
    a.eps = eps;
    a.T = T;
    a.K = K;
    a.codes = codes;
    a.q = (uint8_t*)q_packed;
    a.R = act_rows(T);
    a.scale = scale;
    return launch_rmsnorm(a, dtype, (hipStream_t)stream);
}

}  // extern "C"
