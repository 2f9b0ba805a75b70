// Products of rows and weights in microscaled 4-bit floating point, dense or grouped by expert:
//
//   gate/up : H[p, j] = SiLU(g) * u in 4 bits, blocks of 32 columns;  g = x[p] . W1_e[j], u likewise with W3
//   product : C[p, n] = x[p] . W_e[n],  bf16 or fp32
//
// H's blocks lie inside a tile, so the gate/up product writes it in 4 bits straight from its fp32 sums: a quarter of the bytes of
// bf16, one rounding, and no launch in between.
#include <algorithm>
#include <atomic>
#include <cmath>

#include "expert_gemm_mx4_kernel.h"
#include "mx4_tile_rules.h"

namespace moe {
namespace {

using mx4::Operands;
using mx4::Outputs;
using mx4::Tile;

//                       BM   BN  WM WN NSTAGE DUAL STREAM_B
using GateUpFew    = Tile<32, 64, 2, 1, 6, true, true>;
using GateUp32     = Tile<32, 128, 2, 2, 3, true, true>;
using GateUp64     = Tile<64, 128, 2, 2, 3, true, true>;
using GateUp128    = Tile<128, 256, 2, 4, 3, true>;
template <bool F32> using Plain16x64 = Tile<16, 64, 1, 4, 6, false, true, F32>;
template <bool F32> using Plain32x64Deep = Tile<32, 64, 2, 2, 6, false, true, F32>;
template <bool F32> using Plain32x64 = Tile<32, 64, 2, 2, 3, false, true, F32>;
template <bool F32> using Plain64x64 = Tile<64, 64, 2, 2, 4, false, true, F32>;
template <bool F32> using Plain64x128 = Tile<64, 128, 2, 2, 3, false, true, F32>;
template <bool F32> using Plain128x128 = Tile<128, 128, 2, 2, 4, false, false, F32>;
template <bool F32> using Plain128x128Pair = Tile<128, 128, 2, 2, 2, false, false, F32>;

// ---- a few rows and few tiles: weights straight to registers, the reduction shared by the wavefronts of a workgroup ---------
// A tile is 16 rows and 16 * CF output columns, so that a projection of a few thousand columns has a workgroup for every compute
// unit. Its eight wavefronts take contiguous parts of the reduction, DEPTH k-steps in flight each; the fp32 parts are added in LDS
// in their order, which K alone decides. Bound by latency: one row, 14336 x 4096, weights from memory 9.0 us (31 MB, of which 4.8 at
// 6.5 TB/s), with two k-steps in flight 9.3, with 16 x 64 tiles 17.6. 32 columns read the rows half as often: 16 rows, 8192 x 8192 11.7
// -> 10.9 us, 16384 x 6144 20.4 -> 17.4; one row, 14336 x 4096 (128 workgroups) 9.0 -> 13.8.
constexpr int kFewWaves = 8, kFewRows = 16;

template <bool F32, int CF>
__global__ __launch_bounds__(kFewWaves * kWave) void few_rows_kernel(Operands op, Outputs out) {
    using namespace mx4;
    constexpr int COLS = 16 * CF, DEPTH = CF == 1 ? 4 : 3;
    __shared__ f32x4 part[kFewWaves][CF][kWave];
    const int NT = op.N / COLS;
    const TileCoord tc =
        op.offsets ? gemm::locate_tile<kFewRows>(op.offsets, op.E, NT) : gemm::locate_tile_of_one<kFewRows>(op.R, NT);
    if (tc.expert < 0) return;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int frag_row = lane & 15, g = lane >> 4;
    const uint32_t pitch = static_cast<uint32_t>(op.K) / 2;
    const int runs = mx_runs(op.K), col0 = tc.nt * COLS;
    const int first = wave * runs / kFewWaves, last = (wave + 1) * runs / kFewWaves;

    const __amdgpu_buffer_rsrc_t a = resource(op.a + static_cast<size_t>(tc.row0) * pitch, tc.rows * pitch);
    const __amdgpu_buffer_rsrc_t b = resource(op.b[0] + (static_cast<size_t>(tc.expert) * op.N + col0) * pitch, COLS * pitch);
    const uint8_t* a_scale = op.a_scale + static_cast<size_t>(tc.row0) * kMxRunBytes;
    const uint8_t* b_scale = op.b_scale[0] + (static_cast<size_t>(tc.expert) * runs * op.N + col0) * kMxRunBytes;
    const uint32_t voff = frag_row * pitch + g * 16, soff = frag_row * kMxRunBytes + 2 * g;
    const bool row_in = frag_row < tc.rows;

    f32x4 acc[CF];
#pragma unroll
    for (int c = 0; c < CF; ++c) acc[c] = f32x4{0.f, 0.f, 0.f, 0.f};
    struct Run { i32x4 a[2], b[CF][2]; int as, bs[CF]; } held[DEPTH];
    auto load = [&](Run& r, int run) {
#pragma unroll
        for (int c = 0; c < CF; ++c) {
#pragma unroll
            for (int h = 0; h < 2; ++h)
                r.b[c][h] = __builtin_amdgcn_raw_buffer_load_b128(b, voff + c * 16 * pitch + h * 64, run * 128, 2);
            r.bs[c] = *reinterpret_cast<const uint16_t*>(b_scale + static_cast<size_t>(run) * op.N * kMxRunBytes + soff +
                                                         c * 16 * kMxRunBytes);
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) r.a[h] = __builtin_amdgcn_raw_buffer_load_b128(a, voff + h * 64, run * 128, 0);
        r.as = row_in ? *reinterpret_cast<const uint16_t*>(a_scale + static_cast<size_t>(run) * op.R * kMxRunBytes + soff) : 0;
    };
    auto multiply = [&](const Run& r) {
#pragma unroll
        for (int c = 0; c < CF; ++c) {
            acc[c] = mma<0>(r.b[c][0], r.a[0], acc[c], r.bs[c], r.as);
            acc[c] = mma<1>(r.b[c][1], r.a[1], acc[c], r.bs[c], r.as);
        }
    };
#pragma unroll
    for (int q = 0; q < DEPTH - 1; ++q)
        if (first + q < last) load(held[q], first + q);
    for (int p = first; p < last; p += DEPTH) {
#pragma unroll
        for (int q = 0; q < DEPTH; ++q) {
            if (p + q >= last) break;
            if (p + q + DEPTH - 1 < last) load(held[(q + DEPTH - 1) % DEPTH], p + q + DEPTH - 1);
            multiply(held[q]);
        }
    }
#pragma unroll
    for (int c = 0; c < CF; ++c) part[wave][c][lane] = acc[c];
    __syncthreads();
    if (wave >= CF || !row_in) return;               // a wavefront for each 16 columns
    f32x4 sum = part[0][wave][lane];
#pragma unroll
    for (int w = 1; w < kFewWaves; ++w) sum += part[w][wave][lane];
    const size_t at = (static_cast<size_t>(tc.row0) + frag_row) * op.N + col0 + wave * 16 + 4 * g;
    if constexpr (F32) {
        *reinterpret_cast<f32x4*>(static_cast<float*>(out.c) + at) = sum;
    } else {
        gemm::bf16x4 o;
#pragma unroll
        for (int q = 0; q < 4; ++q) o[q] = static_cast<__bf16>(sum[q]);
        *reinterpret_cast<gemm::bf16x4*>(static_cast<uint16_t*>(out.c) + at) = o;
    }
}

// ---- launches -------------------------------------------------------------------------------------------------------------
template <class Kernel, class... Args>
int launch(const GemmEnv& env, std::atomic<uint64_t>& attr_set, Kernel kern, int smem, int threads, long long grid,
           hipStream_t s, Args... args) {
    if (env.device < 0 || env.device >= 64) return MOE_ERR_INVALID_ARG;
    const uint64_t bit = 1ull << env.device;         // the attribute belongs to the kernel on one device
    if (smem > 0 && !(attr_set.load(std::memory_order_acquire) & bit)) {
        if (hipFuncSetAttribute(reinterpret_cast<const void*>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, smem) != hipSuccess)
            return MOE_ERR_HIP;
        attr_set.fetch_or(bit, std::memory_order_release);
    }
    grid = (grid + kXcds - 1) / kXcds * kXcds;       // every XCD's range of tiles is as long
    if (grid * threads >= 1ll << 32) return MOE_ERR_UNSUPPORTED_SHAPE;
    hipLaunchKernelGGL(kern, dim3(static_cast<unsigned>(grid)), dim3(threads), smem, s, args...);
    return hipGetLastError() == hipSuccess ? MOE_OK : MOE_ERR_HIP;
}

template <class Cfg>
int ring(const GemmEnv& env, const Operands& op, const Outputs& out, hipStream_t s) {
    static std::atomic<uint64_t> attr_set{0};
    return launch(env, attr_set, mx4::ring_kernel<Cfg>, Cfg::SMEM, Cfg::NTHREADS,
                  mx_most_row_tiles(op.R, op.E, Cfg::BM) * ((op.N + Cfg::BN_OUT - 1) / Cfg::BN_OUT), s, op, out);
}

using GateUpLarge = mx4::Mx4<gemm::Config<256, 256, 64, 2, 2, 2, true>>;
template <bool F32>
using PlainLarge = mx4::Mx4<std::conditional_t<F32, gemm::F32Out<gemm::Config<256, 256, 64, 2, 2, 2, false>>,
                                               gemm::Config<256, 256, 64, 2, 2, 2, false>>>;
// Workgroups that run one tile after the other where there are tiles for more than a round. A workgroup per tile -> so: 8192 rows
// of 2048 x 16384 columns 175 -> 170 us, 6144 x 16384 379 -> 375, 16384 x 16384 867 -> 857, experts of 8 x 6144 x 16384 with 8192
// tokens 2213 -> 2180, 5003 skewed tokens through 64 of 2048 x 1408 229 -> 223. What they gain is bounded by the board's power: the
// clock falls from 1.9 to 1.6 GHz as the matrix units get busier (8192 x 16384 x 16384: busy 70 % of the time, 5.1 PFLOP/s; the
// same without a load or an LDS read, 8.0).
template <class Cfg, bool ODD>
int large_of(const GemmEnv& env, const Operands& op, const Outputs& out, hipStream_t s) {
    static std::atomic<uint64_t> attr_set[2];
    const int cus = compute_units(env.device), nt = gemm::n_tiles<Cfg>(op.N);
    // tiles, and the halves that the last round's are cut into
    const long long slots = mx_most_row_tiles(op.R, op.E, 256) * nt + kXcds * ((cus / 2 + kXcds - 1) / kXcds + 1);
    const double tiles = static_cast<double>(op.R) / 256 * nt;
    if (tiles > 1.5 * cus)
        return launch(env, attr_set[0], mx4::large_kernel<Cfg, true, ODD>, mx4::Large<Cfg>::SMEM, 256, std::min<long long>(slots, cus), s,
                      op, out, cus, env.tile_counters);
    return launch(env, attr_set[1], mx4::large_kernel<Cfg, false, ODD>, mx4::Large<Cfg>::SMEM, 256, slots, s, op, out, cus,
                  env.tile_counters);
}
template <class Cfg>
int large(const GemmEnv& env, const Operands& op, const Outputs& out, hipStream_t s) {
    const bool odd = mx_runs(op.K) & 1;
    if (op.K <= kMxRun || op.N < Cfg::BN_OUT || (Cfg::DUAL && odd)) return MOE_ERR_UNSUPPORTED_SHAPE;
    if constexpr (!Cfg::DUAL) {                      // gate/up: K is d_model, a multiple of 512
        if (odd) return large_of<Cfg, true>(env, op, out, s);
    }
    return large_of<Cfg, false>(env, op, out, s);
}

template <bool F32, int CF>
int few_rows(const GemmEnv& env, const Operands& op, const Outputs& out, hipStream_t s) {
    if (op.N % (16 * CF) != 0) return MOE_ERR_UNSUPPORTED_SHAPE;
    static std::atomic<uint64_t> attr_set{0};
    return launch(env, attr_set, few_rows_kernel<F32, CF>, 0, kFewWaves * kWave,
                  mx_most_row_tiles(op.R, op.E, kFewRows) * (op.N / (16 * CF)), s, op, out);
}

template <bool F32>
int product(const GemmEnv& env, const Operands& op, const Outputs& out, hipStream_t s) {
    switch (mx_plain_tile(op.R, op.E, op.N, op.K, compute_units(env.device))) {
        case kMxFew: return few_rows<F32, 1>(env, op, out, s);
        case kMxFewWide: return few_rows<F32, 2>(env, op, out, s);
        case kMx16x64: return ring<Plain16x64<F32>>(env, op, out, s);
        case kMx32x64Deep: return ring<Plain32x64Deep<F32>>(env, op, out, s);
        case kMx32x64: return ring<Plain32x64<F32>>(env, op, out, s);
        case kMx64x64: return ring<Plain64x64<F32>>(env, op, out, s);
        case kMx64x128: return ring<Plain64x128<F32>>(env, op, out, s);
        case kMx128x128: return ring<Plain128x128<F32>>(env, op, out, s);
        case kMx128x128Pair: return ring<Plain128x128Pair<F32>>(env, op, out, s);
        default: return large<PlainLarge<F32>>(env, op, out, s);
    }
}

}  // namespace

int launch_gateup_mx4(const GemmEnv& env, const moe_mx4* x, const moe_e8m0* x_scale, const int32_t* offsets, int R, int d, int f,
                      int E, const moe_mx4* W1, const moe_e8m0* w1_scale, const moe_mx4* W3, const moe_e8m0* w3_scale,
                      moe_mx4* H, moe_e8m0* h_scale, hipStream_t s) {
    const Operands op{x, x_scale, {W1, W3}, {w1_scale, w3_scale}, offsets, R, E, f, d};
    const Outputs out{H, h_scale};
    switch (mx_gateup_tile(R, E, f, d, compute_units(env.device))) {
        case kMxGateFew: return ring<GateUpFew>(env, op, out, s);
        case kMxGate32: return ring<GateUp32>(env, op, out, s);
        case kMxGate64: return ring<GateUp64>(env, op, out, s);
        case kMxGate128: return ring<GateUp128>(env, op, out, s);
        default: return large<GateUpLarge>(env, op, out, s);
    }
}

int launch_product_mx4(const GemmEnv& env, const moe_mx4* x, const moe_e8m0* x_scale, const int32_t* offsets, int R, int N,
                       int K, int E, const moe_mx4* W, const moe_e8m0* w_scale, void* out, bool out_f32, hipStream_t s) {
    const Operands op{x, x_scale, {W, nullptr}, {w_scale, nullptr}, offsets, R, E, N, K};
    return out_f32 ? product<true>(env, op, Outputs{out, nullptr}, s) : product<false>(env, op, Outputs{out, nullptr}, s);
}

}  // namespace moe
