// Rows in 8-bit integers with a scale each: the root-mean-square norm with the residual's addition in front of an 8-bit
// product, and the plain conversion of bf16 rows (the experts' intermediate, a matrix's output channels).
//
//   h = x + residual,  r = 1 / sqrt(mean(h^2) + eps),  y = h * w * r,  scale = max|y| / 127,  q = rint(y / scale)
//
// One pass over the data: a row stays in registers between its loads and its stores. With u = h * w the largest |y| is
// the largest |u| times r and y / scale is u * 127 / max|u|, so the sum of squares and the maximum are reduced
// together, once per row, and q does not wait for r. All of it is fp32; the sum's order is fixed by d and T.
#include "rows_i8.h"

namespace moe {
namespace {

__device__ __forceinline__ void load_row(const uint16_t* row, int at, int n, float (&v)[kVec]) {
    const Raw16 r = load_packed(row, at, n);
#pragma unroll
    for (int i = 0; i < kVec; ++i) v[i] = unpack(r, i);
}
__device__ __forceinline__ void load_row(const float* row, int at, int n, float (&v)[kVec]) {
    if (n == kVec) {
        const Raw16 a = load_any<Raw16>(row + at), b = load_any<Raw16>(row + at + 4);
#pragma unroll
        for (int i = 0; i < kVec; ++i) v[i] = __uint_as_float(i < 4 ? a.w[i & 3] : b.w[i & 3]);
    } else {
#pragma unroll
        for (int i = 0; i < kVec; ++i) v[i] = i < n ? row[at + i] : 0.f;
    }
}
__device__ __forceinline__ uint32_t bf16_pair(float a, float b) {      // round to nearest even
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, bf16x2{static_cast<__bf16>(a), static_cast<__bf16>(b)});
}
__device__ __forceinline__ void store_row(uint16_t* row, int at, int n, const float (&v)[kVec]) {
    if (n == kVec) {
        Raw16 r;
#pragma unroll
        for (int i = 0; i < kVec; i += 2) r.w[i >> 1] = bf16_pair(v[i], v[i + 1]);
        store_any(row + at, r);
    } else {
#pragma unroll
        for (int i = 0; i < kVec; ++i)
            if (i < n) row[at + i] = f32_to_bf16(v[i]);
    }
}
__device__ __forceinline__ void store_row(float* row, int at, int n, const float (&v)[kVec]) {
    if (n == kVec) {
        Raw16 a, b;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            a.w[i] = __float_as_uint(v[i]);
            b.w[i] = __float_as_uint(v[i + 4]);
        }
        store_any(row + at, a);
        store_any(row + at + 4, b);
    } else {
#pragma unroll
        for (int i = 0; i < kVec; ++i)
            if (i < n) row[at + i] = v[i];
    }
}

__device__ __forceinline__ void store_q(int8_t* row, int at, int n, const float (&u)[kVec], float k, bool fine) {
    const Raw8 r = to_8_bits(u, k, fine);
    if (n == kVec) {
        store_any(row + at, r);
    } else {
#pragma unroll
        for (int i = 0; i < kVec; ++i)
            if (i < n) row[at + i] = static_cast<int8_t>(r.w[i >> 2] >> (8 * (i & 3)));
    }
}

// Sum and maximum over the threads of a row, the same bits in all of them: butterflies inside a wavefront, then the
// wavefronts' results in their order. |values| as integers: a NaN counts as more than infinity and stays.
template <int TPR>
__device__ __forceinline__ void reduce_row(float& sum, uint32_t& peak, float* sums, uint32_t* peaks) {
    constexpr int WAVES = TPR / kWave;
#pragma unroll
    for (int s = (TPR < kWave ? TPR : kWave) / 2; s > 0; s >>= 1) {
        sum += __shfl_xor(sum, s);
        peak = max(peak, static_cast<uint32_t>(__shfl_xor(static_cast<int>(peak), s)));
    }
    if constexpr (WAVES > 1) {
        const int wave = threadIdx.x >> 6;
        if ((threadIdx.x & 63) == 0) {
            sums[wave] = sum;
            peaks[wave] = peak;
        }
        __syncthreads();
        sum = sums[0];
        peak = peaks[0];
#pragma unroll
        for (int w = 1; w < WAVES; ++w) {
            sum += sums[w];
            peak = max(peak, peaks[w]);
        }
    }
}

struct RowArgs {
    const uint16_t* x;               // [T, d], rows x_stride elements apart
    long long x_stride;
    const void* residual;            // [T, d] of Residual, or null
    const uint16_t* weight;          // [d], with NORM
    float eps;
    int T, d;
    void* residual_out;              // [T, d] of Residual, or null; may be `residual` itself
    uint16_t* y;                     // [T, d], or null
    moe_i8* q;                       // [T, d], or null
    float* scale;                    // [T]
};

constexpr int threads_of(int tpr) { return tpr <= kWave ? 256 : tpr; }

// TPR threads per row, each with CHUNKS chunks of 8 elements: chunk c of thread t is elements 8 * (c * TPR + t) to + 7. The last
// chunk of a width that is no multiple of 8 starts at d - 8: it holds some elements of the one before a second time, leaves
// them out of the sum and stores the same bits to them. Element by element, in one lane of a row, it cost more than all others.
// A workgroup holds one row, or with up to 64 threads per row as many as its 256 threads have room for.
template <int TPR, int CHUNKS, bool NORM, class Residual>
__global__ __launch_bounds__(threads_of(TPR)) void rows_i8_kernel(RowArgs a) {
    constexpr int WAVES = TPR > kWave ? TPR / kWave : 1, ROWS = threads_of(TPR) / TPR;
    __shared__ float sums[2][WAVES];
    __shared__ uint32_t peaks[2][WAVES];
    const int t = blockIdx.x * ROWS + threadIdx.x / TPR;
    if (ROWS > 1 && t >= a.T) return;                // all threads of the row; no barrier follows where there are several
    const int lane = threadIdx.x % TPR;
    const size_t row = static_cast<size_t>(t) * a.d;
    const uint16_t* x = a.x + static_cast<long long>(t) * a.x_stride;
    const Residual* res = a.residual ? static_cast<const Residual*>(a.residual) + row : nullptr;
    auto nominal = [&](int c) { return (c * TPR + lane) * kVec; };
    auto at = [&](int c) { return min(nominal(c), max(a.d - kVec, 0)); };
    auto count = [&](int c) { return nominal(c) < a.d ? min(kVec, a.d) : 0; };       // 0: nothing of this chunk is in the row

    float h[CHUNKS][kVec];
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
        for (int i = 0; i < kVec; ++i) h[c][i] = 0.f;
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c)
        if (count(c) > 0) load_row(x, at(c), count(c), h[c]);
    if (NORM && res) {
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c)
            if (count(c) > 0) {
                float v[kVec];
                load_row(res, at(c), count(c), v);
#pragma unroll
                for (int i = 0; i < kVec; ++i) h[c][i] += v[i];
            }
    }
    Raw16 w[NORM ? CHUNKS : 1] = {};
    if constexpr (NORM) {
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c)
            if (count(c) > 0) w[c] = load_packed(a.weight, at(c), count(c));
    }
    auto weighted = [&](int c, int i) { return NORM ? h[c][i] * unpack(w[NORM ? c : 0], i) : h[c][i]; };
    auto reduce = [&](float& sum, uint32_t& peak, int which) {
        sum = 0.f;
        peak = 0;
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
            for (int i = 0; i < kVec; ++i) {
                if constexpr (NORM) {
                    const float once = nominal(c) <= at(c) + i ? h[c][i] : 0.f;
                    sum = fmaf(once, once, sum);
                }
                peak = max(peak, __float_as_uint(weighted(c, i)) & 0x7fffffffu);
            }
        reduce_row<TPR>(sum, peak, sums[which], peaks[which]);
    };
    float sum;
    uint32_t peak;
    reduce(sum, peak, 0);
    if (NORM && a.residual_out) {
        Residual* out = static_cast<Residual*>(a.residual_out) + row;
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c)
            if (count(c) > 0) store_row(out, at(c), count(c), h[c]);
    }
    float r = 1.f;
    if constexpr (NORM) {
        float down = 1.f;
        // A sum of squares that leaves the range of fp32: again with the row scaled by 2^-96 (the same decision in all threads of
        // the row; a row that holds an infinity or a NaN stays one that does). Of at most 2^16 values one is then 2^56 or more, its
        // square 2^-80, and the sum stays below 2^(64 + 16). An eps that falls below the range on that scale is nothing beside it.
        if (!(sum < __builtin_inff())) {
            down = 0x1p-96f;
#pragma unroll
            for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
                for (int i = 0; i < kVec; ++i) h[c][i] *= down;
            reduce(sum, peak, 1);
        }
        r = 1.f / sqrtf(sum / static_cast<float>(a.d) + a.eps * down * down);
    }
    const float top = __uint_as_float(peak) * r;     // the largest |y|
    if (NORM && a.y) {
        uint16_t* out = a.y + row;
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c)
            if (count(c) > 0) {
                float v[kVec];
#pragma unroll
                for (int i = 0; i < kVec; ++i) v[i] = weighted(c, i) * r;
                store_row(out, at(c), count(c), v);
            }
    }
    if (a.q) {
        const bool fine = peak < 0x7f800000u && top < __builtin_inff();
        const Factors8 by = factors_8_bits(top > 0.f ? peak : 0u);     // a row of zeros, also by the product with r
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c)
            if (count(c) > 0) {
                float u[kVec];
#pragma unroll
                for (int i = 0; i < kVec; ++i) u[i] = weighted(c, i) * by.up;
                store_q(a.q + row, at(c), count(c), u, by.k, fine);
            }
        if (lane == 0) a.scale[t] = fine ? top / 127.f : __builtin_nanf("");
    }
}

template <int TPR, int CHUNKS, bool NORM, class Residual>
int launch_rows(const RowArgs& all, hipStream_t s) {
    constexpr int threads = threads_of(TPR), rows = threads / TPR;
    constexpr int most = (1 << 30) / threads * rows;     // of a launch, whose threads have to be fewer than 2^32
    for (int t0 = 0; t0 < all.T; t0 += most) {
        RowArgs a = all;
        a.T = all.T - t0 < most ? all.T - t0 : most;
        const size_t at = static_cast<size_t>(t0) * all.d;
        a.x += t0 * all.x_stride;
        if (a.residual) a.residual = static_cast<const Residual*>(a.residual) + at;
        if (a.residual_out) a.residual_out = static_cast<Residual*>(a.residual_out) + at;
        if (a.y) a.y += at;
        if (a.q) {
            a.q += at;
            a.scale += t0;
        }
        hipLaunchKernelGGL((rows_i8_kernel<TPR, CHUNKS, NORM, Residual>), dim3((a.T + rows - 1) / rows), dim3(threads), 0, s, a);
        if (hipGetLastError() != hipSuccess) return MOE_ERR_HIP;
        if (all.T - t0 <= most) break;                   // t0 + most may pass the range
    }
    return MOE_OK;
}

// Threads and chunks by the row's length: the norm, which holds three tensors' chunks, runs with one chunk per thread up to
// 1024 threads, the conversion with a wavefront per row (no barrier) or a few chunks per thread. us, 256 threads -> so: norm of
// 8192 rows of 4096 57.1 -> 51.4 (5.9 TB/s), of 6144 89.6 -> 84.9 (5.3), with an fp32 residual 128 -> 116 (5.6), 16384 of 768
// 31.4 -> 22.9, one of 6144 4.5 -> 3.5; rows in 8 bits, 40024 of 768 33.6 -> 19.7 (4.7), of 1408 39.0 -> 29.9 (5.7), 16384 of 16384
// 146 -> 133 (6.1), 32 of 14336 4.7 -> 3.2; 4000 of 4096 10.7 with two chunks, 11.6 with 512 threads. Narrow rows (one head) share a
// wavefront, a wavefront per row -> so: norm of 390625 rows of 128 190 -> 83 us, rows in 8 bits 89 -> 29, of 64 166 -> 29 (781250).
template <bool NORM, class Residual>
int launch_rows_of(const RowArgs& a, hipStream_t s) {
    if (a.T == 0) return MOE_OK;
    const int chunks = (a.d + kVec - 1) / kVec;
    if (chunks <= 8) return launch_rows<8, 1, NORM, Residual>(a, s);
    if (chunks <= 16) return launch_rows<16, 1, NORM, Residual>(a, s);
    if (chunks <= 32) return launch_rows<32, 1, NORM, Residual>(a, s);
    if (chunks <= 64) return launch_rows<64, 1, NORM, Residual>(a, s);
    if constexpr (NORM) {
        if (chunks <= 128) return launch_rows<128, 1, NORM, Residual>(a, s);
        if (chunks <= 256) return launch_rows<256, 1, NORM, Residual>(a, s);
        if (chunks <= 512) return launch_rows<512, 1, NORM, Residual>(a, s);
        if (chunks <= 1024) return launch_rows<1024, 1, NORM, Residual>(a, s);
    } else {
        if (chunks <= 128) return launch_rows<64, 2, NORM, Residual>(a, s);
        if (chunks <= 192) return launch_rows<64, 3, NORM, Residual>(a, s);
        if (chunks <= 256) return launch_rows<256, 1, NORM, Residual>(a, s);
        if (chunks <= 512) return launch_rows<256, 2, NORM, Residual>(a, s);
        if (chunks <= 768) return launch_rows<256, 3, NORM, Residual>(a, s);
        if (chunks <= 1024) return launch_rows<256, 4, NORM, Residual>(a, s);
    }
    if (chunks <= 2048) return launch_rows<1024, 2, NORM, Residual>(a, s);
    if (chunks <= 4096) return launch_rows<1024, 4, NORM, Residual>(a, s);
    return launch_rows<1024, 8, NORM, Residual>(a, s);
}

}  // namespace

int launch_rmsnorm_i8(const moe_bf16* x, long long x_stride, const void* residual, bool residual_f32,
                      const moe_bf16* weight, float eps, int T, int d, void* residual_out, moe_bf16* y, moe_i8* q,
                      float* q_scale, hipStream_t s) {
    const RowArgs a{x, x_stride, residual, weight, eps, T, d, residual_out, y, q, q_scale};
    return residual_f32 ? launch_rows_of<true, float>(a, s) : launch_rows_of<true, uint16_t>(a, s);
}

int launch_quantize_i8(const moe_bf16* x, long long x_stride, int T, int d, moe_i8* q, float* q_scale, hipStream_t s) {
    const RowArgs a{x, x_stride, nullptr, nullptr, 0.f, T, d, nullptr, nullptr, q, q_scale};
    return launch_rows_of<false, uint16_t>(a, s);
}

// Token rows in 8 bits and their scales in the order of the grouped rows: row p is token perm[p] / k. A wavefront per row.
__global__ __launch_bounds__(256) void gather_i8_kernel(const uint4* __restrict__ q, const float* __restrict__ scale,
                                                        const int32_t* __restrict__ perm, int R, int pieces, int k,
                                                        uint4* __restrict__ q_perm, float* __restrict__ scale_perm) {
    const int p = blockIdx.x * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
    if (p >= R) return;
    const int t = perm[p] / k;
    const uint4* from = q + static_cast<size_t>(t) * pieces;
    uint4* to = q_perm + static_cast<size_t>(p) * pieces;
    for (int i = lane; i < pieces; i += kWave) to[i] = from[i];
    if (lane == 0) scale_perm[p] = scale[t];
}

int launch_gather_i8(const moe_i8* q, const float* scale, const int32_t* perm, int R, int d, int k, moe_i8* q_perm,
                     float* scale_perm, hipStream_t s) {
    if (R == 0) return MOE_OK;
    hipLaunchKernelGGL(gather_i8_kernel, dim3((R + 3) / 4), dim3(256), 0, s, reinterpret_cast<const uint4*>(q), scale, perm, R,
                       d / 16, k, reinterpret_cast<uint4*>(q_perm), scale_perm);
    return hipGetLastError() == hipSuccess ? MOE_OK : MOE_ERR_HIP;
}

}  // namespace moe
