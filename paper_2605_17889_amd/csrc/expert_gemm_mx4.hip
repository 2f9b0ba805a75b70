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

namespace moe {
namespace {

using mx4::Operands;
using mx4::Outputs;
using mx4::Tile;

//                     BM   BN  WM WN NSTAGE DUAL
using GateUp128 = Tile<128, 128, 2, 2, 4, true>;
using GateUp32  = Tile<32, 128, 2, 2, 5, true>;
template <bool F32> using Plain128 = Tile<128, 128, 2, 2, 4, false, false, F32>;
template <bool F32> using Plain32 = Tile<32, 64, 2, 2, 6, false, false, F32>;

// ---- a few rows: weights straight to registers, the reduction shared by the wavefronts of a workgroup -----------------------
// A tile is 16 rows and 16 output columns (with DUAL a block of 32, of both matrices). Its eight wavefronts take contiguous parts
// of the reduction; the fp32 parts are added in LDS in their order, which K alone decides.
constexpr int kFewWaves = 8, kFewRows = 16;

template <bool DUAL, bool F32>
__global__ __launch_bounds__(kFewWaves * kWave) void few_rows_kernel(Operands op, Outputs out) {
    using namespace mx4;
    constexpr int NB = DUAL ? 4 : 1, COLS = DUAL ? 32 : 16;      // weight fragments: 32 columns of W1, the same of W3
    __shared__ f32x4 part[kFewWaves][NB][kWave];
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
    __amdgpu_buffer_rsrc_t b[NB];
    const uint8_t* b_scale[NB];
#pragma unroll
    for (int j = 0; j < NB; ++j) {
        const int m = DUAL ? j >> 1 : 0, col = col0 + (DUAL ? (j & 1) * 16 : 0);
        b[j] = resource(op.b[m] + (static_cast<size_t>(tc.expert) * op.N + col) * pitch, 16 * pitch);
        b_scale[j] = op.b_scale[m] + (static_cast<size_t>(tc.expert) * runs * op.N + col) * kMxRunBytes;
    }
    const uint32_t voff = frag_row * pitch + g * 16, soff = frag_row * kMxRunBytes + 2 * g;
    const bool row_in = frag_row < tc.rows;

    f32x4 acc[NB];
#pragma unroll
    for (int j = 0; j < NB; ++j) acc[j] = f32x4{0.f, 0.f, 0.f, 0.f};
    struct Run { i32x4 a[2], b[NB][2]; int as, bs[NB]; } held[2];
    auto load = [&](Run& r, int run) {
#pragma unroll
        for (int j = 0; j < NB; ++j) {
#pragma unroll
            for (int h = 0; h < 2; ++h)
                r.b[j][h] = __builtin_amdgcn_raw_buffer_load_b128(b[j], voff + h * 64, run * 128, 2);
            r.bs[j] = *reinterpret_cast<const uint16_t*>(b_scale[j] + static_cast<size_t>(run) * op.N * kMxRunBytes + soff);
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) r.a[h] = __builtin_amdgcn_raw_buffer_load_b128(a, voff + h * 64, run * 128, 0);
        r.as = row_in ? *reinterpret_cast<const uint16_t*>(
                            op.a_scale + (static_cast<size_t>(run) * op.R + tc.row0) * kMxRunBytes + soff) : 0;
    };
    auto multiply = [&](const Run& r) {
#pragma unroll
        for (int j = 0; j < NB; ++j) {
            acc[j] = mma<0>(r.b[j][0], r.a[0], acc[j], r.bs[j], r.as);
            acc[j] = mma<1>(r.b[j][1], r.a[1], acc[j], r.bs[j], r.as);
        }
    };
    if (first < last) load(held[0], first);
    for (int p = first; p < last; p += 2) {
        if (p + 1 < last) load(held[1], p + 1);
        multiply(held[0]);
        if (p + 1 >= last) break;
        if (p + 2 < last) load(held[0], p + 2);
        multiply(held[1]);
    }
#pragma unroll
    for (int j = 0; j < NB; ++j) part[wave][j][lane] = acc[j];
    __syncthreads();
    if (wave != 0) return;
    f32x4 sum[NB];
#pragma unroll
    for (int j = 0; j < NB; ++j) {
        sum[j] = part[0][j][lane];
#pragma unroll
        for (int w = 1; w < kFewWaves; ++w) sum[j] += part[w][j][lane];
    }
    const size_t row = static_cast<size_t>(tc.row0) + frag_row;
    if constexpr (DUAL) {
        float v[8];
#pragma unroll
        for (int q = 0; q < 8; ++q) v[q] = gemm::silu(sum[q / 4][q & 3]) * sum[2 + q / 4][q & 3];
        uint32_t scale;
        int at;
        const uint32_t codes = block_codes(v, g, scale, at);
        if (!row_in) return;
        *reinterpret_cast<uint32_t*>(static_cast<uint8_t*>(out.c) + row * (op.N / 2) + col0 / 2 + at * 4) = codes;
        if (g == 0) store_scale(out.scale, op.R, row, col0 / 32, op.N / 32, scale);
    } else {
        if (!row_in) return;
        const size_t at = row * op.N + col0 + 4 * g;
        if constexpr (F32) {
            *reinterpret_cast<f32x4*>(static_cast<float*>(out.c) + at) = sum[0];
        } else {
            gemm::bf16x4 o;
#pragma unroll
            for (int q = 0; q < 4; ++q) o[q] = static_cast<__bf16>(sum[0][q]);
            *reinterpret_cast<gemm::bf16x4*>(static_cast<uint16_t*>(out.c) + at) = o;
        }
    }
}

// ---- launches -------------------------------------------------------------------------------------------------------------
// Upper bound on the number of row tiles of E groups with R rows in all.
long long most_row_tiles(int R, int E, int BM) { return R / BM + std::min(E, R); }

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
    if (grid > 0x7fffffffLL) return MOE_ERR_UNSUPPORTED_SHAPE;
    hipLaunchKernelGGL(kern, dim3(static_cast<unsigned>(grid)), dim3(threads), smem, s, args...);
    return hipGetLastError() == hipSuccess ? MOE_OK : MOE_ERR_HIP;
}

template <class Cfg>
int ring(const GemmEnv& env, const Operands& op, const Outputs& out, hipStream_t s) {
    static std::atomic<uint64_t> attr_set{0};
    return launch(env, attr_set, mx4::ring_kernel<Cfg>, Cfg::SMEM, Cfg::NTHREADS,
                  most_row_tiles(op.R, op.E, Cfg::BM) * ((op.N + Cfg::BN_OUT - 1) / Cfg::BN_OUT), s, op, out);
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
    const long long slots = most_row_tiles(op.R, op.E, 256) * nt + kXcds * ((cus / 2 + kXcds - 1) / kXcds + 1);
    const double tiles = static_cast<double>(op.R) / 256 * nt;
    if (tiles > 1.5 * cus)
        return launch(env, attr_set[0], mx4::large_kernel<Cfg, true, ODD>, mx4::Large<Cfg>::SMEM, 256, std::min<long long>(slots, cus), s,
                      op, out, cus, env.tile_counters);
    return launch(env, attr_set[1], mx4::large_kernel<Cfg, false, ODD>, mx4::Large<Cfg>::SMEM, 256, slots, s, op, out, cus,
                  env.tile_counters);
}
template <class Cfg>
bool large_fits(const Operands& op) { return op.K > 512 && op.N >= Cfg::BN_OUT; }
template <class Cfg>
int large(const GemmEnv& env, const Operands& op, const Outputs& out, hipStream_t s) {
    if (!large_fits<Cfg>(op)) return MOE_ERR_UNSUPPORTED_SHAPE;
    return mx_runs(op.K) & 1 ? large_of<Cfg, true>(env, op, out, s) : large_of<Cfg, false>(env, op, out, s);
}

template <bool DUAL, bool F32>
int few_rows(const GemmEnv& env, const Operands& op, const Outputs& out, hipStream_t s) {
    static std::atomic<uint64_t> attr_set{0};
    return launch(env, attr_set, few_rows_kernel<DUAL, F32>, 0, kFewWaves * kWave,
                  most_row_tiles(op.R, op.E, kFewRows) * (op.N / (DUAL ? 32 : 16)), s, op, out);
}

// Rows of a group: the average and two standard deviations of a uniform routing.
double upper_rows(int R, int E) {
    const double avg = static_cast<double>(R) / E;
    return E == 1 ? avg : avg + 2.0 * std::sqrt(avg);
}

template <bool F32>
int product(const GemmEnv& env, const Operands& op, const Outputs& out, hipStream_t s) {
    const double rows = upper_rows(op.R, op.E);
    if (rows <= 16.0) return few_rows<false, F32>(env, op, out, s);
    if (rows <= 64.0) return ring<Plain32<F32>>(env, op, out, s);
    if (rows <= 128.0 || !large_fits<PlainLarge<F32>>(op)) return ring<Plain128<F32>>(env, op, out, s);
    return large<PlainLarge<F32>>(env, op, out, s);
}

}  // namespace

int launch_gateup_mx4(const GemmEnv& env, const moe_mx4* x, const moe_e8m0* x_scale, const int32_t* offsets, int R, int d, int f,
                      int E, const moe_mx4* W1, const moe_e8m0* w1_scale, const moe_mx4* W3, const moe_e8m0* w3_scale,
                      moe_mx4* H, moe_e8m0* h_scale, hipStream_t s) {
    const Operands op{x, x_scale, {W1, W3}, {w1_scale, w3_scale}, offsets, R, E, f, d};
    const Outputs out{H, h_scale};
    const double rows = upper_rows(R, E);
    if (rows <= 16.0) return few_rows<true, false>(env, op, out, s);
    if (rows <= 64.0) return ring<GateUp32>(env, op, out, s);
    if (rows <= 128.0 || !large_fits<GateUpLarge>(op)) return ring<GateUp128>(env, op, out, s);
    return large<GateUpLarge>(env, op, out, s);
}

int launch_product_mx4(const GemmEnv& env, const moe_mx4* x, const moe_e8m0* x_scale, const int32_t* offsets, int R, int N,
                       int K, int E, const moe_mx4* W, const moe_e8m0* w_scale, void* out, bool out_f32, hipStream_t s) {
    const Operands op{x, x_scale, {W, nullptr}, {w_scale, nullptr}, offsets, R, E, N, K};
    return out_f32 ? product<true>(env, op, Outputs{out, nullptr}, s) : product<false>(env, op, Outputs{out, nullptr}, s);
}

}  // namespace moe
