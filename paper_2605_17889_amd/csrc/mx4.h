// Microscaled 4-bit floating point (device code; rows_mx4.hip and the products of expert_gemm_mx4.hip).
//
// A row is cut into blocks of 32 elements. Element i of a block stands for 2^(scale - 127) * v(code), where the 4-bit code is
// a sign, two bits of exponent (bias 1) and one of fraction: 0, 0.5, 1, 1.5, 2, 3, 4, 6; scale is a byte, 255 stands for NaN.
// Codes lie two to a byte, the even element in the low half. Scales lie in runs of 256 elements (8 blocks): those of a run
// side by side for each row, the rows of one run after the other, block 4 t + g of the run at byte 2 g + t. That is what the
// matrix instruction wants: of a k-step of 256 elements, two instructions of 128, lane group g multiplies blocks g and 4 + g
// and finds both scales in the 16 bits at byte 2 g; and a tile's rows are one piece of memory.
#pragma once
#include "common.h"

namespace moe {
namespace {

constexpr int kMxBlock = 32, kMxRun = 256, kMxRunBytes = kMxRun / kMxBlock;

__host__ __device__ constexpr int mx_runs(int K) { return (K + kMxRun - 1) / kMxRun; }
// Byte of block b inside the 8 of its row and run.
__host__ __device__ constexpr int mx_byte(int b) { return 2 * (b & 3) + ((b >> 2) & 1); }

// The scale of a block whose largest |element| has the fp32 bits `peak`: the power of two that brings it to 4 .. 8, where 4 to
// 6 are the largest codes and what is above 6 becomes 6. Smaller than 2^-125: the smallest scale, 2^-127. NaN and infinities
// (their bits are the largest): 255.
__device__ __forceinline__ uint32_t mx_scale(uint32_t peak) {
    const int exponent = static_cast<int>(peak >> 23);
    return exponent == 255 ? 255u : static_cast<uint32_t>(max(exponent - 2, 0));
}

// Eight elements as codes of blocks of that scale: divided by it, to the nearest code, ties to the even one. The instruction takes
// the power of two from a float's exponent field, where 0 is 2^-127 too. A block of scale 255 has codes 0.
__device__ __forceinline__ uint32_t mx_codes(const float (&v)[8], uint32_t scale) {
    const float by = __uint_as_float(scale << 23);
    uint32_t w = 0;
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[0], v[1], by, 0);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[2], v[3], by, 1);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[4], v[5], by, 2);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[6], v[7], by, 3);
    return scale == 255u ? 0u : w;
}

}  // namespace
}  // namespace moe
