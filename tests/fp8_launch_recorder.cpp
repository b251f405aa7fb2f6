// Stands in for the HIP runtime under the host code of the 8-bit floating-point calls and the norm: kernels are not run, the name,
// work-groups, threads and LDS of each launch are printed, and a line "=" and the status behind each call.  Reads one call per line:
// g T K N (haq_gemm_fp8_packed), l T K N (haq_fp8_linear), q T K dtype (haq_quant_act_fp8_packed), n T K codes (haq_rmsnorm_quant),
// w K N 0 (haq_quant_weight_fp8), c n 0 0 (compute units from here on).
#include <cstdarg>
#include <cstdio>
#include <map>
#include <string>

#include "haq_common.h"

static std::map<const void*, std::string>& kernels() {  // filled before this file's own constructors have run
    static std::map<const void*, std::string> m;
    return m;
}
static dim3 grid_, block_;
static size_t lds_;
static int n_cu = 256;

extern "C" {
void** __hipRegisterFatBinary(const void*) {
    static void* handle;
    return &handle;
}
void __hipUnregisterFatBinary(void**) {}
void __hipRegisterFunction(void**, const void* host, char*, const char* name, unsigned, void*, void*, void*, void*, int*) { kernels()[host] = name; }
hipError_t __hipPushCallConfiguration(dim3 grid, dim3 block, size_t lds, hipStream_t) {
    grid_ = grid;
    block_ = block;
    lds_ = lds;
    return hipSuccess;
}
hipError_t __hipPopCallConfiguration(dim3* grid, dim3* block, size_t* lds, hipStream_t* st) {
    *grid = grid_;
    *block = block_;
    *lds = lds_;
    *st = nullptr;
    return hipSuccess;
}
hipError_t hipLaunchKernel(const void* f, dim3 grid, dim3 block, void**, size_t lds, hipStream_t) {
    printf("%s %u %u %u %zu\n", kernels()[f].c_str(), grid.x, grid.y * grid.z, block.x, lds);
    return hipSuccess;
}
hipError_t hipFuncSetAttribute(const void*, hipFuncAttribute, int) { return hipSuccess; }
hipError_t hipGetLastError() { return hipSuccess; }
const char* hipGetErrorString(hipError_t) { return ""; }
}

namespace haq {
void set_error(const char* fmt, ...) {
    va_list ap;
    va_start(ap, fmt);
    vfprintf(stderr, fmt, ap);
    va_end(ap);
}
int cu_count() { return n_cu; }
}  // namespace haq

int main() {
    char what;
    int a, b, c;
    uint8_t* u = (uint8_t*)256;  // addresses that nothing follows
    uint8_t* far = (uint8_t*)((uintptr_t)1 << 46);
    float* f = (float*)256;
    while (scanf(" %c %d %d %d", &what, &a, &b, &c) == 4) {
        int rc = HAQ_OK;
        switch (what) {
            case 'g': rc = haq_gemm_fp8_packed(u, f, u, f, a, b, c, HAQ_ACT_NONE, HAQ_F16, u, c, nullptr); break;
            case 'l': rc = haq_fp8_linear(u, b, HAQ_F16, u, f, a, b, c, HAQ_ACT_NONE, far, c, u, (size_t)1 << 46, nullptr); break;
            case 'q': rc = haq_quant_act_fp8_packed(u, b, c, a, b, u, f, nullptr); break;
            case 'n': rc = haq_rmsnorm_quant(u, b, u, b, f, 1e-5, HAQ_BF16, a, b, u, b, u, b, c, c ? u : nullptr, c ? f : nullptr, nullptr); break;
            case 'w': rc = haq_quant_weight_fp8(f, a, b, u, f, nullptr); break;
            case 'c': n_cu = a; break;
        }
        printf("= %d\n", rc);
    }
    return 0;
}
