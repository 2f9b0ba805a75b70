// What libmoe.so enqueues, without a GPU: this program stands in for the HIP runtime (its symbols come before the runtime's), hands
// out addresses that nobody reads and notes every launch. A launch of 2^32 threads or more fails, as the runtime's does.
// Compiled and run by test_mx4_launches.py; one call a line on stdin, for each: status, number of launches, and one line for each
// launch with its kernel, grid and threads of a workgroup. "kernels" prints the names of all kernels that the library holds.
#define __HIP_PLATFORM_AMD__
#include <cxxabi.h>
#include <hip/hip_runtime_api.h>

#include <cstdio>
#include <cstdlib>
#include <iostream>
#include <map>
#include <sstream>
#include <string>
#include <vector>

#include "moe.h"

namespace {

constexpr int kComputeUnits = 256;

struct Launch {
    std::string kernel;
    unsigned grid, threads;
};
std::map<const void*, std::string>& kernels() {      // the library registers them before main
    static std::map<const void*, std::string> all;
    return all;
}
std::vector<Launch> launches;
hipError_t last_error = hipSuccess;
uintptr_t next_address = uintptr_t{1} << 44;

void* address(size_t bytes) {
    void* p = reinterpret_cast<void*>(next_address);
    next_address += (bytes + 4095) / 4096 * 4096;
    return p;
}
dim3 pushed_grid, pushed_block;
size_t pushed_smem;
hipStream_t pushed_stream;

}  // namespace

extern "C" {
void** __hipRegisterFatBinary(const void*) { static void* handle; return &handle; }
void __hipUnregisterFatBinary(void**) {}
void __hipRegisterVar(void**, void*, char*, char*, int, size_t, int, int) {}
void __hipRegisterFunction(void**, const void* host, char*, const char* name, unsigned, void*, void*, void*, void*, int*) {
    int status = 0;
    char* text = abi::__cxa_demangle(name, nullptr, nullptr, &status);
    kernels()[host] = status == 0 ? text : name;
    std::free(text);
}
hipError_t __hipPushCallConfiguration(dim3 grid, dim3 block, size_t smem, hipStream_t stream) {
    pushed_grid = grid, pushed_block = block, pushed_smem = smem, pushed_stream = stream;
    return hipSuccess;
}
hipError_t __hipPopCallConfiguration(dim3* grid, dim3* block, size_t* smem, hipStream_t* stream) {
    *grid = pushed_grid, *block = pushed_block, *smem = pushed_smem, *stream = pushed_stream;
    return hipSuccess;
}
hipError_t hipLaunchKernel(const void* host, dim3 grid, dim3 block, void**, size_t, hipStream_t) {
    if (static_cast<unsigned long long>(grid.x) * block.x >= 1ull << 32) return last_error = hipErrorInvalidConfiguration;
    launches.push_back({kernels()[host], grid.x, block.x});
    return hipSuccess;
}
hipError_t hipGetLastError() {
    const hipError_t e = last_error;
    last_error = hipSuccess;
    return e;
}
hipError_t hipGetDeviceCount(int* n) { *n = 1; return hipSuccess; }
hipError_t hipGetDevice(int* device) { *device = 0; return hipSuccess; }
hipError_t hipSetDevice(int) { return hipSuccess; }
hipError_t hipDeviceGetAttribute(int* value, hipDeviceAttribute_t, int) { *value = kComputeUnits; return hipSuccess; }
hipError_t hipFuncSetAttribute(const void*, hipFuncAttribute, int) { return hipSuccess; }
hipError_t hipMalloc(void** p, size_t bytes) { *p = address(bytes); return hipSuccess; }
hipError_t hipFree(void*) { return hipSuccess; }
hipError_t hipMemcpy(void*, const void*, size_t, hipMemcpyKind) { return hipSuccess; }
hipError_t hipGetSymbolAddress(void** p, const void*) { *p = address(1 << 20); return hipSuccess; }
}

int main() {
    moe_ctx* ctx = nullptr;
    moe_shape shape{};
    std::string line, what;
    while (std::getline(std::cin, line)) {
        std::istringstream in(line);
        in >> what;
        if (what == "kernels") {
            for (const auto& k : kernels()) std::printf("%s\n", k.second.c_str());
            continue;
        }
        launches.clear();
        int rc = -100;
        auto p = [] { return address(4096); };
        auto f = [&] { return static_cast<float*>(p()); };
        auto b = [&] { return static_cast<uint8_t*>(p()); };
        auto i = [&] { return static_cast<int32_t*>(p()); };
        auto h = [&] { return static_cast<moe_bf16*>(p()); };
        moe_scoring sc{};
        auto scoring = [&] { in >> sc.score >> sc.groups >> sc.top_groups; sc.group_best = 2, sc.renormalise = 1, sc.scale = 1.f; };
        int T = 0, R = 0;
        if (what == "context") {                     // T_max d_model d_ff E k
            in >> shape.T_max >> shape.d_model >> shape.d_ff >> shape.E >> shape.k;
            if (ctx != nullptr) moe_destroy(ctx);
            ctx = nullptr;
            rc = moe_create(&ctx, &shape, 0);
        } else if (what == "route") {                // T score groups top_groups
            in >> T;
            scoring();
            rc = moe_route_scored(ctx, h(), f(), f(), f(), &sc, T, i(), f(), nullptr, nullptr);
        } else if (what == "logits") {
            in >> T;
            scoring();
            rc = moe_route_scored_from_logits(ctx, f(), f(), &sc, T, i(), f(), nullptr);
        } else if (what == "layer") {                // T, and score groups top_groups or score -1
            in >> T;
            scoring();
            const bool scored = sc.score >= 0;
            rc = moe_layer_forward_mx4(ctx, h(), f(), f(), scored ? f() : nullptr, scored ? &sc : nullptr, b(), b(), b(), b(), b(),
                                       b(), T, h(), nullptr);
        } else if (what == "experts") {              // R
            in >> R;
            rc = moe_expert_ffn_mx4(ctx, b(), b(), i(), R, b(), b(), b(), b(), b(), b(), h(), nullptr);
        } else if (what == "product") {              // R E N K fp32 grouped
            int E, N, K, fp32, grouped;
            in >> R >> E >> N >> K >> fp32 >> grouped;
            rc = moe_gemm_mx4(ctx, b(), b(), grouped ? i() : nullptr, R, E, N, K, b(), b(), p(), fp32 ? MOE_OUT_FP32 : MOE_OUT_BF16,
                              nullptr);
        } else if (what == "rows") {                 // T d
            int d;
            in >> T >> d;
            rc = moe_quantize_mx4(h(), d, T, d, b(), b(), nullptr);
        } else if (what == "back") {                 // T d
            int d;
            in >> T >> d;
            rc = moe_dequantize_mx4(b(), b(), T, d, h(), nullptr);
        }
        if (!in) rc = -101;
        std::printf("%d %zu\n", rc, launches.size());
        for (const Launch& l : launches) std::printf("%s|%u|%u\n", l.kernel.c_str(), l.grid, l.threads);
    }
    if (ctx != nullptr) moe_destroy(ctx);
    return 0;
}
