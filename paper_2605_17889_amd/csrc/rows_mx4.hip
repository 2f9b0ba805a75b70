// Rows of bf16 in microscaled 4-bit floating point (mx4.h) and back.
#include "mx4.h"
#include "rows_i8.h"

namespace moe {
namespace {

// Four lanes hold a block, 8 elements each: a wavefront reads 1 KB and writes 256 bytes of codes, both in one piece. The largest
// |element| of a block is found in the lanes' bits (integers order like the magnitudes, a NaN above all), across the four lanes by
// two moves inside quads.
__device__ __forceinline__ uint32_t quad_max(uint32_t v) {
    v = max(v, static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(v), 0xb1, 0xf, 0xf, false)));
    return max(v, static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(v), 0x4e, 0xf, 0xf, false)));
}

// One run of a row (256 elements, 32 lanes) per half wavefront; a workgroup takes 16 rows of one run, so that the scales of a run's
// rows are written next to each other, and a thread two of them, loaded together. Bound by memory: 8192 x 6144 to 4 bits and back, 2 x
// 127 MB, 39.7 us with the launches (6.4 TB/s); one row per thread 43.3, four 40.4, eight 42.5.
constexpr int kRowThreads = 256, kRowsPerThread = 2, kRowsPerGroup = kRowThreads / 32 * kRowsPerThread;

// GROUPED: row t goes to the k rows places[t * k] .. of the T * k that are grouped by expert.
template <bool GROUPED>
__global__ __launch_bounds__(kRowThreads) void quantize_mx4_kernel(const uint16_t* __restrict__ x, long long x_stride, int T,
                                                                   int d, const int32_t* __restrict__ places, int k,
                                                                   uint8_t* __restrict__ q, uint8_t* __restrict__ scale) {
    const int lane = threadIdx.x & 31;
    const int run = blockIdx.x % mx_runs(d);
    const int t0 = blockIdx.x / mx_runs(d) * kRowsPerGroup + threadIdx.x / 32;
    const int at = run * kMxRun + lane * kVec;
    const bool in = at < d;                          // whole quads: d is a multiple of 32
    Raw16 raw[kRowsPerThread] = {};
#pragma unroll
    for (int r = 0; r < kRowsPerThread; ++r) {
        const int t = t0 + r * (kRowThreads / 32);
        if (in && t < T) raw[r] = load_any<Raw16>(x + static_cast<long long>(t) * x_stride + at);
    }
#pragma unroll
    for (int r = 0; r < kRowsPerThread; ++r) {
        const int t = t0 + r * (kRowThreads / 32);
        if (t >= T) return;
        float v[kVec];
        uint32_t peak = 0;
#pragma unroll
        for (int i = 0; i < kVec; ++i) {
            v[i] = unpack(raw[r], i);
            peak = max(peak, __float_as_uint(v[i]) & 0x7fffffffu);
        }
        const uint32_t s = mx_scale(quad_max(peak)), codes = mx_codes(v, s);
        for (int n = 0; n < k; ++n) {
            const size_t row = GROUPED ? places[static_cast<size_t>(t) * k + n] : t;
            if (in) store_any(q + row * (d / 2) + at / 2, codes);
            if ((lane & 3) == 0)                     // behind the last block: 0
                scale[(static_cast<size_t>(run) * T * k + row) * kMxRunBytes + mx_byte(lane >> 2)] = static_cast<uint8_t>(in ? s : 0u);
        }
    }
}

__global__ __launch_bounds__(kRowThreads) void dequantize_mx4_kernel(const uint8_t* __restrict__ q,
                                                                     const uint8_t* __restrict__ scale, int T, int d,
                                                                     uint16_t* __restrict__ y) {
    const int lane = threadIdx.x & 31;
    const int run = blockIdx.x % mx_runs(d);
    const int t0 = blockIdx.x / mx_runs(d) * kRowsPerGroup + threadIdx.x / 32;
    const int at = run * kMxRun + lane * kVec;
    if (at >= d) return;
    uint32_t w[kRowsPerThread], s[kRowsPerThread];
#pragma unroll
    for (int r = 0; r < kRowsPerThread; ++r) {
        const int t = min(t0 + r * (kRowThreads / 32), T - 1);
        w[r] = load_any<uint32_t>(q + static_cast<size_t>(t) * (d / 2) + at / 2);
        s[r] = scale[(static_cast<size_t>(run) * T + t) * kMxRunBytes + mx_byte(lane >> 2)];
    }
#pragma unroll
    for (int r = 0; r < kRowsPerThread; ++r) {
        const int t = t0 + r * (kRowThreads / 32);
        if (t >= T) return;
        uint16_t o[kVec];
#pragma unroll
        for (int i = 0; i < kVec; ++i) {
            // Twice the value of the three low bits, 0 1 2 3 4 6 8 12, in a nibble each; the product with a power of two is exact
            // in bf16 down to 2^-133, its smallest step, and 6 * 2^127 is infinite as it is when rounded.
            const uint32_t code = w[r] >> (4 * i);
            const int twice = static_cast<int>((0xc8643210u >> (4 * (code & 7u))) & 15u);
            const float v = ldexpf(static_cast<float>(twice), static_cast<int>(s[r]) - 128);
            const uint32_t bits = s[r] == 255u ? 0x7fc00000u : __float_as_uint(v) | (code & 8u) << 28;
            o[i] = static_cast<uint16_t>(bits >> 16);
        }
        store_any(y + static_cast<size_t>(t) * d + at, o);
    }
}

int enqueue_error() { return hipGetLastError() == hipSuccess ? MOE_OK : MOE_ERR_HIP; }
long long row_groups(int T, int d) {
    return (static_cast<long long>(T) + kRowsPerGroup - 1) / kRowsPerGroup * mx_runs(d);
}

}  // namespace

bool rows_mx4_fit(int T, int d) { return row_groups(T, d) * kRowThreads <= kMaxThreads; }

template <bool GROUPED>
static int quantize(const moe_bf16* x, long long x_stride, int T, int d, const int32_t* places, int k, moe_mx4* q, moe_e8m0* scale,
                    hipStream_t s) {
    if (T == 0) return MOE_OK;
    if (!rows_mx4_fit(T, d)) return MOE_ERR_UNSUPPORTED_SHAPE;
    hipLaunchKernelGGL((quantize_mx4_kernel<GROUPED>), dim3(static_cast<unsigned>(row_groups(T, d))), dim3(kRowThreads), 0, s, x,
                       x_stride, T, d, places, k, q, scale);
    return enqueue_error();
}
int launch_quantize_mx4(const moe_bf16* x, long long x_stride, int T, int d, moe_mx4* q, moe_e8m0* scale, hipStream_t s) {
    return quantize<false>(x, x_stride, T, d, nullptr, 1, q, scale, s);
}
int launch_quantize_grouped_mx4(const moe_bf16* x, const int32_t* inv_perm, int T, int d, int k, moe_mx4* q, moe_e8m0* scale,
                                hipStream_t s) {
    return quantize<true>(x, d, T, d, inv_perm, k, q, scale, s);
}

int launch_dequantize_mx4(const moe_mx4* q, const moe_e8m0* scale, int T, int d, moe_bf16* y, hipStream_t s) {
    if (T == 0) return MOE_OK;
    if (!rows_mx4_fit(T, d)) return MOE_ERR_UNSUPPORTED_SHAPE;
    hipLaunchKernelGGL(dequantize_mx4_kernel, dim3(static_cast<unsigned>(row_groups(T, d))), dim3(kRowThreads), 0, s, q, scale, T, d, y);
    return enqueue_error();
}

}  // namespace moe
