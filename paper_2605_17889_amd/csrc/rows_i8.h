// Pieces of the conversion of rows to 8-bit integers (device code; norm.hip, expert_gemm_i8.hip).
#pragma once
#include "common.h"

namespace moe {
namespace {

constexpr int kVec = 8;             // consecutive elements that a thread holds per chunk

// Addresses need not be multiples of anything: rows of odd lengths and rows cut out of wider tensors start anywhere.
// The compiler makes one wide load or store of these (the hardware takes any address).
struct Raw16 { uint32_t w[4]; };
struct Raw8 { uint32_t w[2]; };
template <class T> __device__ __forceinline__ T load_any(const void* p) {
    T v;
    __builtin_memcpy(&v, p, sizeof(T));
    return v;
}
template <class T> __device__ __forceinline__ void store_any(void* p, const T& v) { __builtin_memcpy(p, &v, sizeof(T)); }

// Elements [at, at + n) of a row, n <= 8; those past n are zero. bf16 ones stay packed, two to a register.
__device__ __forceinline__ Raw16 load_packed(const uint16_t* row, int at, int n) {
    if (n == kVec) return load_any<Raw16>(row + at);
    Raw16 r{};
#pragma unroll
    for (int i = 0; i < kVec; ++i)
        if (i < n) r.w[i >> 1] |= static_cast<uint32_t>(row[at + i]) << (16 * (i & 1));
    return r;
}
__device__ __forceinline__ float unpack(const Raw16& r, int i) {
    return __uint_as_float((i & 1) ? (r.w[i >> 1] & 0xffff0000u) : (r.w[i >> 1] << 16));
}

// q = rint(u * k), |u * k| <= 127 up to rounding: in fma(u, k, 1.5 * 2^23) the sum's unit is 1, so that the one rounding
// of the fused operation is the one to the nearest integer (ties to even), whose two's complement is the low byte.
__device__ __forceinline__ Raw8 to_8_bits(const float (&u)[kVec], float k, bool fine) {
    uint32_t b[kVec];
#pragma unroll
    for (int i = 0; i < kVec; ++i) b[i] = __float_as_uint(fmaf(u[i], k, 12582912.f));
    Raw8 r;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const uint32_t lo = __builtin_amdgcn_perm(b[4 * i + 1], b[4 * i], 0x0c0c0400u);
        const uint32_t hi = __builtin_amdgcn_perm(b[4 * i + 3], b[4 * i + 2], 0x04000c0cu);
        r.w[i] = fine ? lo | hi : 0u;
    }
    return r;
}

// How a row whose largest |u| has the bits `peak` is brought to 8 bits: elements times `up`, then times k. 127 / max|u| leaves the
// range of fp32 for the smallest maxima, both factors are then moved by 2^100.
// k is 127 / max|u| rounded up, which decides the ties of bf16 rows as they are to be: 127 is prime, so that of a largest element
// of 8 bits only its halves are ties, 63.5, which then go to 64 (unless it is 127 times a power of two; k is exact then, and
// to_8_bits takes all ties to even). Rounded to nearest, k gave 63 for 66 of the 128 mantissas. Quotients of 8-bit mantissas that are no
// ties lie 2^-16 of themselves and more from one, k is off by less than 2^-23 of itself.
struct Factors8 { float up, k; };
__device__ __forceinline__ Factors8 factors_8_bits(uint32_t peak) {
    const float up = peak < 0x0d800000u ? 0x1p100f : 1.f;        // below 2^-100
    const float largest = __uint_as_float(peak) * up;
    float k = peak == 0 ? 0.f : 127.f / largest;
    if (fmaf(k, largest, -127.f) < 0.f && peak != 0) k = __uint_as_float(__float_as_uint(k) + 1);
    return {up, k};
}

}  // namespace
}  // namespace moe
