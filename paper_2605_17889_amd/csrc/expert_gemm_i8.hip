// Products of 8-bit integers with a scale for each row and each output channel, dense or grouped by expert:
//
//   gate/up : H[p, j] = bf16( SiLU(g) * u ),  g = s_p s1_e[j] sum_i q_p[i] W1_e[j,i],  u likewise with W3
//   product : C[p, n] = s_p s_e[n] sum_k q_p[k] W_e[n,k],  bf16 or fp32
//
// The kernels and the rules by which tiles are chosen are those of the bf16 products, with rows of half as many 16-bit
// units (expert_gemm_kernel.h). The sums are whole numbers: every tile and order of them gives the same bits.
#include "expert_gemm_launch.h"
#include "i8_tile_rules.h"
#include "rows_i8.h"

namespace moe {
namespace {

//                      BM   BN  BK WM WN NSTAGE DUAL [STREAM_B]
template <class Cfg> using I8 = gemm::OperandsI8<Cfg>;
using GateUp1W         = I8<Config<256, 256, 64, 2, 2, 2, true>>;
using GateUpMid        = I8<Config<128, 256, 64, 2, 4, 3, true>>;
using GateUpMidS       = I8<Config<128, 256, 64, 2, 4, 3, true, true>>;
using GateUpMid96      = I8<Config<96, 256, 64, 1, 4, 3, true>>;
using GateUpMid96S     = I8<Config<96, 256, 64, 1, 4, 3, true, true>>;
using GateUpSmall      = I8<Config<64, 128, 64, 2, 2, 3, true>>;
using GateUpSmallS     = I8<Config<64, 128, 64, 2, 2, 3, true, true>>;
using GateUpTiny       = I8<Config<32, 128, 64, 2, 2, 4, true>>;
using GateUpTinyS      = I8<Config<32, 128, 64, 2, 2, 4, true, true>>;
using GateUpTinyDeepS  = I8<Config<32, 128, 64, 2, 2, 7, true, true>>;
using GateUpFewS       = I8<Config<32, 64, 64, 2, 2, 4, true, true>>;
using GateUpFewDeepS   = I8<Config<32, 64, 64, 2, 2, 6, true, true>>;
using Plain1W          = I8<Config<256, 256, 64, 2, 2, 2, false>>;
using PlainMid         = I8<Config<128, 128, 64, 2, 2, 4, false>>;
using PlainMidS        = I8<Config<128, 128, 64, 2, 2, 4, false, true>>;
using PlainMidWide     = I8<Config<128, 256, 64, 2, 4, 3, false>>;
using PlainMidWideS    = I8<Config<128, 256, 64, 2, 4, 3, false, true>>;
using PlainMid96       = I8<Config<96, 128, 64, 1, 4, 5, false>>;
using PlainMid96S      = I8<Config<96, 128, 64, 1, 4, 5, false, true>>;
using PlainMid96Wide   = I8<Config<96, 256, 64, 1, 4, 3, false>>;
using PlainMid96WideS  = I8<Config<96, 256, 64, 1, 4, 3, false, true>>;
using PlainSmallWide   = I8<Config<64, 128, 64, 2, 2, 3, false>>;
using PlainSmallWideS  = I8<Config<64, 128, 64, 2, 2, 3, false, true>>;
using PlainSmall       = I8<Config<64, 64, 64, 2, 2, 5, false>>;
using PlainSmallS      = I8<Config<64, 64, 64, 2, 2, 5, false, true>>;
using PlainTiny        = I8<Config<32, 64, 64, 2, 2, 4, false>>;
using PlainTinyS       = I8<Config<32, 64, 64, 2, 2, 4, false, true>>;
using PlainFew         = I8<Config<16, 32, 64, 1, 2, 6, false>>;
using PlainFewS        = I8<Config<16, 32, 64, 1, 2, 6, false, true>>;

// ---- a few rows and few tiles: weights straight to registers, the reduction shared by wavefronts and workgroups ------
// A tile is 16 rows and 16 output columns (with DUAL of both matrices). Its eight wavefronts take contiguous parts of the
// reduction, so that a projection of a few thousand columns has a workgroup for every compute unit, which streams from eight
// places of its weight rows; the int32 parts are added in LDS. Where even so there are few tiles and the reduction is long, it
// is split over `splits` workgroups as well, whose parts are added in memory. Weights and rows go from memory to the lanes that
// multiply them, the next 128 bytes of a row while those before are multiplied. The sums are whole numbers: how they are split
// changes no bit.
//
// Bound by the latency of its loads and launch, not by bandwidth: one token, weights from memory, tiles of
// 32 columns with the reduction in one workgroup (16 x 32) -> so: 14336 x 4096 19.1 -> 13.7 us (58.7 MB, of which 8.6 at
// 6.8 TB/s), 4096 x 4096 7.5 -> 5.5, 2048 x 2048 4.8 -> 3.8; 16 tokens 20.1 -> 18.4, 7.9 -> 6.8, 4.7 -> 4.5. Past one tile per compute
// unit the 32-column tiles win: 6144 x 6144 10.1 against 12.0, 4096 x 14336 columns 12.6 against 14.2. Four wavefronts, 32 columns
// and two or four pieces in flight per wavefront are all within 5 % or slower.
constexpr int kFewWaves = 8, kFewRows = 16;

template <bool STREAM>
__device__ __forceinline__ gemm::i32x4 load_frag(const int8_t* p) {
    if constexpr (STREAM) return __builtin_nontemporal_load(reinterpret_cast<const gemm::i32x4*>(p));
    else return *reinterpret_cast<const gemm::i32x4*>(p);
}

template <bool DUAL, bool F32>
__global__ __launch_bounds__(kFewWaves * kWave) void few_rows_i8_kernel(
    const int8_t* __restrict__ A, const int8_t* __restrict__ B0, const int8_t* __restrict__ B1, void* __restrict__ C,
    const int32_t* __restrict__ offsets, int E, int N, int K, gemm::ScalesI8 sc, int splits, int32_t* __restrict__ sums) {
    using gemm::i32x4;
    constexpr int NB = DUAL ? 2 : 1;                 // weight fragments
    __shared__ i32x4 part[kFewWaves][NB][kWave];
    // the parts of a split reduction are mapped as the n-tiles of a matrix `splits` times as wide
    const int NT = N / 16 * splits;
    const gemm::TileCoord tc =
        offsets ? gemm::locate_tile<kFewRows>(offsets, E, NT) : gemm::locate_tile_of_one<kFewRows>(sc.rows, NT);
    if (tc.expert < 0) return;
    int split;
    const int nt = gemm::div_small(tc.nt, splits, split);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int frag_row = lane & 15, kg = lane >> 4;
    const size_t wrow = static_cast<size_t>(tc.expert) * N + nt * 16;
    const int row = tc.row0 + min(frag_row, tc.rows - 1);

    float xs = 0.f;                                  // the scales of the outputs that the first wavefront will write
    gemm::f32x4 ws[NB] = {};
    if (wave == 0) {
        xs = sc.x[row];
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            ws[0][r] = sc.w0[wrow + 4 * kg + r];
            if constexpr (DUAL) ws[1][r] = sc.w1[wrow + 4 * kg + r];
        }
    }
    const int pieces = K / 128;                      // of 128 bytes, two k-steps of the instruction
    const int part_of = split * kFewWaves + wave, parts = splits * kFewWaves;
    const int first = part_of * pieces / parts, last = (part_of + 1) * pieces / parts;
    const int8_t* a = A + static_cast<size_t>(row) * K + kg * 16;
    const int8_t* b[NB];
#pragma unroll
    for (int j = 0; j < NB; ++j) b[j] = (j == 0 ? B0 : B1) + (wrow + frag_row) * K + kg * 16;

    i32x4 acc[NB];
#pragma unroll
    for (int j = 0; j < NB; ++j) acc[j] = i32x4{0, 0, 0, 0};
    if (first < last) {
        i32x4 fa[2][2], fb[2][2][NB];
        auto load = [&](auto tag, int p) {
            constexpr int S = decltype(tag)::value;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const size_t k = static_cast<size_t>(p) * 128 + h * 64;
#pragma unroll
                for (int j = 0; j < NB; ++j) fb[S][h][j] = load_frag<true>(b[j] + k);
                fa[S][h] = load_frag<false>(a + k);
            }
        };
        auto multiply = [&](auto tag) {
            constexpr int S = decltype(tag)::value;
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int j = 0; j < NB; ++j)
                    acc[j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(fb[S][h][j], fa[S][h], acc[j], 0, 0, 0);
        };
        using Even = std::integral_constant<int, 0>;
        using Odd = std::integral_constant<int, 1>;
        load(Even{}, first);
        for (int p = first; p < last; p += 2) {
            if (p + 1 < last) load(Odd{}, p + 1);
            multiply(Even{});
            if (p + 1 >= last) break;
            if (p + 2 < last) load(Even{}, p + 2);
            multiply(Odd{});
        }
    }
#pragma unroll
    for (int j = 0; j < NB; ++j) part[wave][j][lane] = acc[j];
    __syncthreads();
    if (wave != 0) return;
    i32x4 sum[NB];
#pragma unroll
    for (int j = 0; j < NB; ++j) {
        sum[j] = part[0][j][lane];
#pragma unroll
        for (int w = 1; w < kFewWaves; ++w) sum[j] += part[w][j][lane];
    }
    if constexpr (!DUAL) {
        if (splits > 1) {
            // Memory that is zero between launches: 256 sums of each tile, then a counter each. Every access is an atomic
            // operation, performed in one place for all compute units, and its returned value says that it has been: the
            // counter moves on behind this part's sums. Who moves it last takes the sums and leaves zeros.
            int32_t *mine = sums + nt * 256 + lane, *arrived = sums + N / 16 * 256 + nt;
            int old[4];
#pragma unroll
            for (int r = 0; r < 4; ++r)
                old[r] = __hip_atomic_fetch_add(mine + r * kWave, sum[0][r], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            asm volatile("" :: "v"(old[0]), "v"(old[1]), "v"(old[2]), "v"(old[3]) : "memory");
            int before = 0;
            if (lane == 0) before = __hip_atomic_fetch_add(arrived, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            if (__builtin_amdgcn_readfirstlane(before) != splits - 1) return;
            asm volatile("" ::: "memory");
#pragma unroll
            for (int r = 0; r < 4; ++r)
                sum[0][r] = __hip_atomic_exchange(mine + r * kWave, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            if (lane == 0) __hip_atomic_store(arrived, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        }
    }
    if (frag_row >= tc.rows) return;
    const size_t at = static_cast<size_t>(row) * N + nt * 16 + 4 * kg;
    gemm::f32x4 v;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        v[r] = static_cast<float>(sum[0][r]) * xs * ws[0][r];
        if constexpr (DUAL) v[r] = gemm::silu(v[r]) * (static_cast<float>(sum[1][r]) * xs * ws[1][r]);
    }
    if constexpr (F32) {
        *reinterpret_cast<gemm::f32x4*>(static_cast<float*>(C) + at) = v;
    } else {
        gemm::bf16x4 o;
#pragma unroll
        for (int r = 0; r < 4; ++r) o[r] = static_cast<__bf16>(v[r]);
        *reinterpret_cast<gemm::bf16x4*>(static_cast<uint16_t*>(C) + at) = o;
    }
}

using Piped32x64       = I8<Config<32, 64, 64, 2, 2, 4, false>>;
using Converted16      = I8<Config<16, 64, 64, 1, 2, 4, false, true>>;
using PipedShort       = I8<Config<64, 128, 64, 2, 2, 3, false>>;
using Piped64x64       = I8<Config<64, 64, 64, 2, 2, 5, false>>;
using Piped64x128      = I8<Config<64, 128, 64, 2, 2, 6, false>>;
using Piped128x128     = I8<Config<128, 128, 64, 2, 2, 5, false>>;

// ---- down projection of a few rows straight from bf16 H -------------------------------------------------------------------
// C = H W^T with H's rows brought to 8 bits by every workgroup for itself: the rows of its tile (K <= 2048) go through registers
// (largest element, scale, 8-bit values: the formulas of moe_quantize_i8, bit for bit) into LDS, where they stay for the whole
// reduction while the weights stream through a ring of stages. It saves the launch in between and costs every tile the conversion
// of its rows. Expert FFN with the launch -> without: one token through 8 of 128 experts of 2048 x 768 13.5 -> 10.9 us, 2 17.5 ->
// 14.9, 8 40.1 -> 38.1; one through 2 of 8 of 512 x 1024 9.5 -> 8.3, 16 (four rows an expert) 11.2 -> 10.3, 64 (16 rows) 11.9 -> 12.2.
constexpr int kConvertedK = 2048;
template <class Cfg>
constexpr int converted_smem(int K) { return K / 128 * Cfg::A_BYTES + Cfg::NSTAGE * Cfg::B_BYTES + Cfg::BM * 4; }

template <class Cfg, int ITS>        // ITS: 512 elements of a row each
__global__ __launch_bounds__(Cfg::NTHREADS) void converted_rows_kernel(const uint16_t* __restrict__ H,
                                                                       const uint16_t* __restrict__ B0, uint16_t* __restrict__ C,
                                                                       const int32_t* __restrict__ offsets, int E, int N, int K,
                                                                       gemm::ScalesI8 scales) {
    using namespace gemm;
    using Plan = LoadPlan<Cfg>;
    constexpr int TM = Cfg::TM, TN = Cfg::TN, S = Cfg::NSTAGE, LB = Plan::LB, RPW = Cfg::BM / Cfg::NW;
    extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];
    const TileCoord tc = locate_tile<Cfg::BM>(offsets, E, n_tiles<Cfg>(N));
    if (tc.expert < 0) return;
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave / Cfg::WN, wn = wave % Cfg::WN;
    const int KT = K / Cfg::BK, f = 2 * K;           // K counts pairs of elements
    const uint32_t ring = KT * Cfg::A_BYTES;
    float* row_scale = reinterpret_cast<float*>(smem + ring + S * Cfg::B_BYTES);
    TileScales<Cfg> sc;
    sc.load_columns(scales, tc, wn, lane, N);
    Raw16 raw[RPW][ITS] = {};
#pragma unroll
    for (int q = 0; q < RPW; ++q) {
        const int r = q * Cfg::NW + wave;            // rows in turn: a few rows keep all wavefronts busy
        if (r >= tc.rows) continue;
        const uint16_t* row = H + static_cast<size_t>(tc.row0 + r) * f;
#pragma unroll
        for (int i = 0; i < ITS; ++i)
            if ((i * kWave + lane) * kVec < f) raw[q][i] = load_any<Raw16>(row + (i * kWave + lane) * kVec);
    }
    Plan lp;
    lp.init_fixed(wave, lane, K);
    lp.init_b(tc, wave, B0, nullptr, N, K);
    auto issue = [&](int stage, int kt) {
#pragma unroll
        for (int i = 0; i < LB; ++i)
            dma16<Cfg::STREAM_B>(lp.b_src(i) + static_cast<size_t>(kt) * Cfg::BK, lp.b_voff[i],
                                 ring + stage * Cfg::B_BYTES + (lp.b_lds - Cfg::A_BYTES) + i * 1024);
    };
#pragma unroll
    for (int s = 0; s < S - 1; ++s)
        if (s < KT) issue(s, s);
    auto convert = [&](int q) {
        const int r = q * Cfg::NW + wave;
        if (r >= tc.rows) return;
        uint32_t peak = 0;
#pragma unroll
        for (int i = 0; i < ITS; ++i)
#pragma unroll
            for (int v = 0; v < kVec; ++v) peak = max(peak, __float_as_uint(unpack(raw[q][i], v)) & 0x7fffffffu);
        auto with = [&](int other) { peak = max(peak, static_cast<uint32_t>(other)); };
        with(row_move<0x111, 0xf>(peak));            // the largest of all lanes ends up in lane 63
        with(row_move<0x112, 0xf>(peak));
        with(row_move<0x114, 0xf>(peak));
        with(row_move<0x118, 0xf>(peak));
        with(row_move<0x142, 0xa>(peak));
        with(row_move<0x143, 0xc>(peak));
        peak = __builtin_amdgcn_readlane(static_cast<int>(peak), 63);
        const bool fine = peak < 0x7f800000u;
        const Factors8 by = factors_8_bits(peak);
#pragma unroll
        for (int i = 0; i < ITS; ++i) {
            const int piece = i * kWave + lane;      // of 8 elements; 16 to a k-step
            if (piece * kVec >= f) continue;
            float u[kVec];
#pragma unroll
            for (int v = 0; v < kVec; ++v) u[v] = unpack(raw[q][i], v) * by.up;
            const int chunk = (piece & 15) >> 1;
            store_any(smem + (piece >> 4) * Cfg::A_BYTES + r * Cfg::ROW_BYTES + ((chunk ^ swz<Cfg::BK>(r)) << 4) + (piece & 1) * 8,
                      to_8_bits(u, by.k, fine));
        }
        if (lane == 0) row_scale[r] = fine ? __uint_as_float(peak) / 127.f : __builtin_nanf("");
    };
#pragma unroll
    for (int q = 0; q < RPW; ++q) convert(q);
    __syncthreads();
#pragma unroll
    for (int i = 0; i < TileScales<Cfg>::NX; ++i) sc.x[i] = row_scale[min(wm * Cfg::WTM + i * 64 + lane, tc.rows - 1)];

    FragPlan<Cfg> fp;
    fp.init(lane, wm, wn);
    f32x4 acc[TM][TN];
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    int stage = 0;
    for (int kt = 0; kt < KT; ++kt) {
        if (kt + S - 2 < KT) wait_vmcnt<(S - 2) * LB>(); else wait_vmcnt<0>();
        __builtin_amdgcn_s_barrier();                // stage `stage` is there, the one before is no longer read
        const unsigned char *a = smem + kt * Cfg::A_BYTES, *b = smem + ring + stage * Cfg::B_BYTES - Cfg::A_BYTES;
        bf16x8 af[2][TM], bfr[2][TN];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
#pragma unroll
            for (int i = 0; i < TM; ++i) af[h][i] = lds16(a + fp.a_off[h] + i * Cfg::TILE_STEP);
#pragma unroll
            for (int j = 0; j < TN; ++j) bfr[h][j] = lds16(b + fp.b_off[h] + j * Cfg::TILE_STEP);
        }
        if (kt + S - 1 < KT) issue(stage == 0 ? S - 1 : stage - 1, kt + S - 1);
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int i = 0; i < TM; ++i)
#pragma unroll
                for (int j = 0; j < TN; ++j) acc[i][j] = mma16<true>(bfr[h][j], af[h][i], acc[i][j]);
        stage = stage + 1 == S ? 0 : stage + 1;
    }
    store_tile<Cfg>(acc, tc, fp, wm, wn, C, N, sc);
}

// A product's operands: matrices as 16-bit units, K of them per row.
struct Call {
    const GemmEnv& env;
    const uint16_t *A, *B0, *B1;
    void* C;
    const int32_t* offsets;          // null: one group of R rows
    gemm::ScalesI8 scales;
    int R, E, N, K;
    hipStream_t s;
};
const uint16_t* units(const moe_i8* p) { return reinterpret_cast<const uint16_t*>(p); }

template <class Cfg>
int grouped(const Call& c) {
    return launch_grouped<Cfg>(c.env, c.A, c.B0, c.B1, static_cast<uint16_t*>(c.C), c.offsets, nullptr, 1, c.R, c.E, c.N,
                               c.K, c.s, c.scales);
}
template <class Cfg>
int piped(const Call& c) {
    return launch_pipelined<Cfg>(c.env, c.A, c.B0, c.B1, static_cast<uint16_t*>(c.C), c.offsets, c.R, c.E, c.N, c.K, c.s,
                                 c.scales);
}
// Sums of `splits` parts of a reduction, part by part [R, N], as outputs.
template <bool F32>
__global__ __launch_bounds__(256) void join_parts_kernel(const gemm::i32x4* __restrict__ parts, int splits, long long quads, int N,
                                                         gemm::ScalesI8 sc, void* __restrict__ C) {
    const long long q = static_cast<long long>(blockIdx.x) * 256 + threadIdx.x;
    if (q >= quads) return;
    gemm::i32x4 sum = parts[q];
    for (int p = 1; p < splits; ++p) sum += parts[p * quads + q];
    const int row = static_cast<int>(q * 4 / N), col = static_cast<int>(q * 4 - static_cast<long long>(row) * N);
    const float xs = sc.x[row];
    gemm::f32x4 v;
#pragma unroll
    for (int r = 0; r < 4; ++r) v[r] = static_cast<float>(sum[r]) * xs * sc.w0[col + r];
    if constexpr (F32) {
        static_cast<gemm::f32x4*>(C)[q] = v;
    } else {
        gemm::bf16x4 o;
#pragma unroll
        for (int r = 0; r < 4; ++r) o[r] = static_cast<__bf16>(v[r]);
        static_cast<gemm::bf16x4*>(C)[q] = o;
    }
}
template <bool F32, class Cfg>
int split(const Call& c, int splits) {
    int32_t* parts = c.env.part_sums;
    Call d = c;
    d.scales.splits = splits;
    d.C = parts;
    const int rc = piped<gemm::RawSums<Cfg>>(d);
    if (rc != MOE_OK) return rc;
    const long long quads = static_cast<long long>(c.R) * c.N / 4;
    hipLaunchKernelGGL((join_parts_kernel<F32>), dim3(static_cast<unsigned>((quads + 255) / 256)), dim3(256), 0, c.s,
                       reinterpret_cast<const gemm::i32x4*>(parts), splits, quads, c.N, c.scales, c.C);
    return hipGetLastError() == hipSuccess ? MOE_OK : MOE_ERR_HIP;
}
// Weights that a single row tile reads are loaded as non-temporal.
template <class Cached, class Streamed>
int grouped(const Call& c) {
    return single_m_tile(c.env, c.R, c.E, Cached::BM) ? grouped<Streamed>(c) : grouped<Cached>(c);
}
template <class Cfg>
int large(const Call& c) {
    uint16_t* out = static_cast<uint16_t*>(c.C);
    if constexpr (!Cfg::DUAL)                        // gate/up reduces over d_model, a multiple of 512
        if (c.K % 128 != 0)
            return launch_1w<Cfg, true>(c.env, c.A, c.B0, c.B1, out, c.offsets, nullptr, 1, c.R, c.E, c.N, c.K, c.s, c.scales);
    return launch_1w<Cfg, false>(c.env, c.A, c.B0, c.B1, out, c.offsets, nullptr, 1, c.R, c.E, c.N, c.K, c.s, c.scales);
}
// Experts that the call is expected to touch.
double touched(const Call& c) { return c.E == 1 ? 1.0 : touched_experts(c.R, c.E); }

// Whether the tiles of 16 rows and columns find a compute unit each.
bool few_rows_fits(const Call& c) {
    if (c.env.forced_config >= 0) return false;
    const bool few = c.E == 1 ? c.R <= kFewRows : single_m_tile(c.env, c.R, c.E, kFewRows);
    return few && touched(c) * (c.N / 16) <= compute_units(c.env.device);
}
// Workgroups that share the reduction of a tile, 2048 elements of it each, up to one workgroup per compute unit. One token, split
// by 1 -> as here: 16384 x 256 12.3 -> 6.1 us (8), 8192 x 1024 7.7 -> 5.9 (4), 8192 x 2048 7.9 -> 6.9 (2); joining costs about 1 us,
// 4096 x 512 4.9 -> 5.1 (2), 2048 x 1024 3.8 -> 4.6, and more with more parts (16384 x 256 in 16 7.0).
int few_rows_splits(const Call& c) {
    if (c.E != 1 || c.K < 3 * 1024 || c.env.whole_reductions) return 1;      // K counts pairs of elements
    const int tiles = c.N / 16;
    if (tiles > kSplitTiles) return 1;
    return std::max(1, std::min(compute_units(c.env.device) / tiles, c.K / 1024));
}
template <bool DUAL, bool F32>
int few_rows(const Call& c) {
    const int splits = DUAL ? 1 : few_rows_splits(c);
    if (splits > 1 && c.env.split_sums == nullptr) return kNeedsSums;
    const long long grid = (most_row_tiles(c.R, c.E, kFewRows) * (c.N / 16) * splits + kXcds - 1) / kXcds * kXcds;
    if (grid > 0x7fffffffLL) return MOE_ERR_UNSUPPORTED_SHAPE;
    hipLaunchKernelGGL((few_rows_i8_kernel<DUAL, F32>), dim3(static_cast<unsigned>(grid)), dim3(kFewWaves * kWave), 0, c.s,
                       reinterpret_cast<const int8_t*>(c.A), reinterpret_cast<const int8_t*>(c.B0),
                       reinterpret_cast<const int8_t*>(c.B1), c.C, c.offsets, c.E, c.N, 2 * c.K, c.scales, splits,
                       c.env.split_sums);
    return hipGetLastError() == hipSuccess ? MOE_OK : MOE_ERR_HIP;
}
bool large_takes(int N, int K) { return gemm::offsets_fit_1w(N, K) && K >= 256; }

// Few rows for each of many experts with a short reduction: three rounds and more of 128-column tiles are mostly what a tile
// costs outside its reduction, and tiles of 256 weight rows are half as many. 32- or 64-row tiles -> 96-row ones, through 8 of
// 128 experts of 2048 x 768: 120 tokens 113 -> 104 us, 300 122 -> 111, 600 132 -> 123; 37 tokens (2.7 rounds) 92 -> 94, 300
// through 6 of 64 of 2048 x 1408 (2.7) 101 -> 103.
bool many_short_tiles(const Call& c) {
    return c.env.forced_config < 0 && c.K <= 1024 && touched(c) * (c.N / 128) >= 2.9 * compute_units(c.env.device);
}

template <class Cfg>
int converted(const Call& c) {
    static std::atomic<uint64_t> attr_set[2];
    const int which = c.K <= 512 ? 0 : 1;
    const auto kern = which == 0 ? converted_rows_kernel<Cfg, 2> : converted_rows_kernel<Cfg, 4>;
    return launch_tiles_sized(c.env, attr_set[which], kern, converted_smem<Cfg>(which == 0 ? 1024 : kConvertedK),
                              converted_smem<Cfg>(2 * c.K), Cfg::NTHREADS, most_row_tiles(c.R, c.E, Cfg::BM) * gemm::n_tiles<Cfg>(c.N),
                              c.s, c.A, c.B0, static_cast<uint16_t*>(c.C), c.offsets, c.E, c.N, c.K, c.scales);
}

int gateup(const Call& c) {
    if (few_rows_fits(c)) return few_rows<true, false>(c);
    int config = pick_config(c.env, c.R, c.E, gateup_tiles(c.E, c.K, c.N));
    if (config == 0 && !large_takes(c.N, c.K)) config = 1;
    if (c.env.forced_config < 0) config = i8_gateup_config(config, c.R, c.E, c.N, c.K, compute_units(c.env.device));
    switch (config) {
        case 0: return large<GateUp1W>(c);
        case 1: return grouped<GateUpMid, GateUpMidS>(c);
        case 4: return grouped<GateUpMid96, GateUpMid96S>(c);
        case 3: {
            if (!single_m_tile(c.env, c.R, c.E, 32)) return grouped<GateUpTiny>(c);
            if (many_short_tiles(c)) return grouped<GateUpMid96S>(c);
            const double nt = touched(c) * (c.N / 64);
            const int cus = compute_units(c.env.device);
            if (narrow_gateup_tiles(c.R, c.E, c.N, cus) || narrow_short_gateup_tiles(c.R, c.E, c.K, c.N, cus))
                return one_tile_per_cu(c.R, c.E, c.N, cus) ? grouped<GateUpFewDeepS>(c) : grouped<GateUpFewS>(c);
            // Long reductions, every expert with a few rows: 64-row tiles leave more loads in flight. 32- -> 64-row ones, layers
            // of experts of 4096 x 14336: 16 tokens through 2 of 8 213 -> 207 us, 64 223 -> 216; 4 tokens (one row each) 139 -> 145
            if (c.K > 1024 && c.R >= 4 * c.E) return grouped<GateUpSmallS>(c);
            return last_round_use(nt, 2.0 * cus) < 0.93 * last_round_use(nt, cus) ? grouped<GateUpTinyDeepS>(c)
                                                                                 : grouped<GateUpTinyS>(c);
        }
        default:
            if (many_short_tiles(c)) return grouped<GateUpMid96, GateUpMid96S>(c);
            return grouped<GateUpSmall, GateUpSmallS>(c);
    }
}

// ---- one matrix, or a few not so large ones: the tile and the split of the reduction are priced ---------------------------
// A compute unit takes in 50 GB/s of rows and weights that come from memory (85 from L2), whatever the tile, so that a k-step
// costs by the bytes of its stage; small tiles load each byte more often, large ones leave compute units without any. Where
// both hurt (few rows, narrow outputs, long reductions) the reduction is split over workgroups, whose int32 sums go to memory
// and are joined by a second launch. us of a k-step of 128 elements, weights from memory; `pair`: of two workgroups on a
// compute unit. Priced -> the tile that the grouped rules take, in us: 64 rows, 14336 x 4096 columns 30.8 -> 17.7; 128 rows there
// 36.0 -> 22.9; 512 rows 93 -> 51; 1003 92 -> 68; 256 rows, 8192 x 1024 17.8 -> 11.9; 2048 rows there 50.7 -> 28.8; 128 rows,
// 16384 x 256 24.6 -> 9.2; 1003 rows, 2048 x 2048 13.6 -> 9.2; 512 rows, 8192 x 8192 53 -> 41. Groups of 128 rows and more, up to
// 128 MB of weights: 750 rows for each of 2 of 2048 x 2048 18.3 -> 14.1, 188 of 8 there 19.1 -> 16.9, 150 of 2 of 8192 x 4096 33.6
// -> 28.0; with more weights or fewer rows their stream decides, for which the grouped rules are drawn (112 rows of 64 of 1408 x
// 2048, 184 MB, gate/up included: 149, priced 162).
enum class Tile { t32x64, t64x64, t64x128, short64x128, t128x128, large };
struct TilePrice {
    Tile tile;
    int rows, cols, stages;
    double step, pair, fixed;        // us; without a pair one workgroup fills a compute unit
};
constexpr TilePrice kTiles[] = {
    {Tile::t32x64, 32, 64, 4, 0.28, 0.46, 1.5},    {Tile::t64x64, 64, 64, 5, 0.32, 0.57, 1.5},
    {Tile::t64x128, 64, 128, 6, 0.47, 0.0, 1.5},   {Tile::short64x128, 64, 128, 3, 0.50, 0.85, 1.5},
    {Tile::t128x128, 128, 128, 5, 0.62, 0.0, 1.5}, {Tile::large, 256, 256, 4, 1.45, 0.0, 4.0},
};
struct Plan {
    Tile tile;
    int splits;
    double us;
};
Plan price(const Call& c) {
    const int cus = compute_units(c.env.device);
    const double bytes = 2.0 * c.E * c.N * c.K, ksteps = c.K / 64.0;
    Plan best{Tile::t32x64, 1, 1e30};
    for (const TilePrice& t : kTiles) {
        if (c.N < t.cols || c.K / 64 < t.stages || (t.tile == Tile::large && !large_takes(c.N, c.K))) continue;
        const double row_tiles_of = c.E == 1 ? std::ceil(c.R / static_cast<double>(t.rows)) : row_tiles(c.R, c.E, t.rows);
        const double tiles = row_tiles_of * ((c.N + t.cols - 1) / t.cols);
        const bool can_split = c.offsets == nullptr && t.tile <= Tile::t64x128 && !c.env.whole_reductions;
        for (int s = 1; s <= (can_split ? 16 : 1); ++s) {
            if (c.K / 64 / s < t.stages || (s > 1 && static_cast<double>(s) * c.R * c.N > kPartSums)) break;
            const double n = tiles * s, each = std::ceil(n / cus);           // workgroups of a compute unit
            double step = each * t.step, rounds = each;
            if (t.pair > 0.0) {
                rounds = std::ceil(each / 2);
                step = std::floor(each / 2) * t.pair + (each - 2 * std::floor(each / 2)) * t.step;
            }
            if (t.tile == Tile::large) {          // the tiles of a last round that is less than half full are run as two halves
                const double rem = n - std::floor(n / cus) * cus;
                if (rem > 0 && 2 * rem <= cus) step += 0.88 - t.step;
            }
            // joining: a launch, every sum written and read, and a tenth as the margin that a split has to win by
            const double us = std::max(ksteps / s * step, bytes / 6e6) + rounds * t.fixed +
                              (s > 1 ? 3.0 + 8e-6 / 4 * s * c.R * c.N : 0.0);
            const double price = s > 1 ? us / 0.9 : us;
            if (price < best.us) best = Plan{t.tile, s, price};
        }
    }
    return best;
}
template <bool F32, class Cfg>
int one_tile(const Call& c, int splits) {
    if constexpr (Cfg::BN <= 128 && Cfg::BM <= 64)
        if (splits > 1) return split<F32, Cfg>(c, splits);
    return piped<Out<F32, Cfg>>(c);
}
bool is_priced(const Call& c) {
    if (c.env.forced_config >= 0 || c.R <= kFewRows) return false;
    return c.E == 1 || (c.R >= 128.0 * c.E && 2.0 * c.E * c.N * c.K <= 128e6);
}
template <bool F32>
int priced(const Call& c) {
    const Plan plan = price(c);
    if (plan.splits > 1 && c.env.part_sums == nullptr) return kNeedsSums;
    switch (plan.tile) {
        case Tile::t64x64: return one_tile<F32, Piped64x64>(c, plan.splits);
        case Tile::t64x128: return one_tile<F32, Piped64x128>(c, plan.splits);
        case Tile::short64x128: return one_tile<F32, PipedShort>(c, 1);
        case Tile::t128x128: return one_tile<F32, Piped128x128>(c, 1);
        case Tile::large: return large<Out<F32, Plain1W>>(c);
        default: break;
    }
    if (c.N < 64) return grouped<Out<F32, PlainFew>>(c);
    if (c.K / 64 >= Piped32x64::NSTAGE) return one_tile<F32, Piped32x64>(c, plan.splits);
    // Shorter than the rings of the table's tiles: the grouped form of two workgroups per compute unit where they fill those (6649
    // rows, 256 x 11776 110 -> 72 us, 1000 rows, 256 x 4096 9.0 -> 6.4), else smaller tiles (300 rows, 256 x 2048 4.2, 3.5)
    if (c.N >= 128 && std::ceil(c.R / 64.0) * (c.N / 128) >= compute_units(c.env.device)) return grouped<Out<F32, PlainSmallWide>>(c);
    return grouped<Out<F32, PlainSmall>>(c);
}

template <bool F32>
int product(const Call& c) {
    if (few_rows_fits(c)) return few_rows<false, F32>(c);
    if (is_priced(c)) return priced<F32>(c);
    const int d = c.N;
    const bool wide_mid = static_cast<long long>(c.E) * (d / 256) >= 160;
    const int cus = compute_units(c.env.device);
    int config = pick_config(c.env, c.R, c.E, NTiles{(d + 255) / 256, wide_mid ? (d + 255) / 256 : (d + 127) / 128, (d + 63) / 64,
                                                     wide_mid ? 0.82 : 0.6, 0.27, 0.38, 2e-6 * c.E * d * c.K, c.K / 64});
    if (config == 0 && (!large_takes(d, c.K) || d < 256)) config = 1;
    if ((config == 1 || config == 4) && d < 128) config = 2;
    if (config == 2 && d < 64) config = 3;
    if (c.env.forced_config < 0) config = i8_product_config(config, c.R, c.E, d, c.K, wide_mid ? d / 256 : d / 128, cus);
    // Reductions of up to 1024 elements over many tiles: the pipelined 64 x 128 tile, two on a compute unit. Grouped forms -> so,
    // through 8 of 128 experts of 2048 x 768: 120 tokens 113 -> 111 us, 300 122 -> 115, 600 132 -> 122, 1000 140 -> 131 (all with
    // gate/up); 1408 elements, 600 tokens through 6 of 64 119 -> 122.
    if (c.env.forced_config < 0 && (config == 2 || config == 3 || config == 4) && c.K <= 512 && c.K / 64 >= PipedShort::NSTAGE &&
        d >= 128 && touched(c) * (d / 128) >= 3.5 * cus)
        return piped<Out<F32, PipedShort>>(c);
    switch (config) {
        case 0: return large<Out<F32, Plain1W>>(c);
        case 1:
            if (wide_mid) return grouped<Out<F32, PlainMidWide>, Out<F32, PlainMidWideS>>(c);
            return grouped<Out<F32, PlainMid>, Out<F32, PlainMidS>>(c);
        case 4:
            if (wide_mid) return grouped<Out<F32, PlainMid96Wide>, Out<F32, PlainMid96WideS>>(c);
            return grouped<Out<F32, PlainMid96>, Out<F32, PlainMid96S>>(c);
        case 3:
            if (touched(c) * (d / 64) < cus) {
                if (single_m_tile(c.env, c.R, c.E, 16)) return grouped<Out<F32, PlainFewS>>(c);
                if (d < 64 || row_tiles(c.R, c.E, 16) * (d / 32) <= cus) return grouped<Out<F32, PlainFew>>(c);
            }
            return grouped<Out<F32, PlainTiny>, Out<F32, PlainTinyS>>(c);
        default:
            if (row_tiles(c.R, c.E, 64) * (d / 64) <= 0.5 * cus) return grouped<Out<F32, PlainTiny>>(c);
            if (touched(c) * (d / 128) >= 3.5 * cus)
                return grouped<Out<F32, PlainSmallWide>, Out<F32, PlainSmallWideS>>(c);
            return grouped<Out<F32, PlainSmall>, Out<F32, PlainSmallS>>(c);
    }
}

}  // namespace

int launch_gateup_i8(const GemmEnv& env, const moe_i8* x, const float* x_scale, const int32_t* offsets, int R, int d, int f,
                     int E, const moe_i8* W1, const float* w1_scale, const moe_i8* W3, const float* w3_scale, moe_bf16* H,
                     hipStream_t s) {
    if (R == 0) return MOE_OK;
    return gateup(Call{env, units(x), units(W1), units(W3), H, offsets, {x_scale, w1_scale, w3_scale, R, 1}, R, E, f, d / 2, s});
}

// A few rows for each expert that has any, and not so many tiles that the conversions add up.
bool down_converts(const GemmEnv& env, int R, int d, int f, int E) {
    const double touched = E == 1 ? 1.0 : touched_experts(R, E);
    return env.forced_config < 0 && f <= kConvertedK && R <= 5.0 * touched && touched * (d / 64) <= 6.0 * compute_units(env.device);
}

int launch_down_converting_i8(const GemmEnv& env, const moe_bf16* H, const int32_t* offsets, int R, int d, int f, int E,
                              const moe_i8* W2, const float* w2_scale, void* y, bool y_f32, hipStream_t s) {
    if (R == 0) return MOE_OK;
    const Call c{env, H, units(W2), nullptr, y, offsets, {nullptr, w2_scale, nullptr, R, 1}, R, E, d, f / 2, s};
    // Where the tiles are more than a few: 16 rows and weights past the caches (8 tokens through 8 of 128 of 2048 x 768 40.8 ->
    // 38.1 us, 2 through 6 of 64 of 2048 x 1408 27.5 -> 24.0); with fewer tiles the 32-row form, whose four wavefronts share the
    // conversion (16 tokens of 512 x 1024 11.3 -> 10.3, one through 8 of 128 11.2 -> 10.6)
    if (touched(c) * (d / 64) > (f <= 1024 ? 2.0 : 1.0) * compute_units(env.device))
        return y_f32 ? converted<gemm::F32Out<Converted16>>(c) : converted<Converted16>(c);
    return y_f32 ? converted<gemm::F32Out<PlainTiny>>(c) : converted<PlainTiny>(c);
}

int launch_product_i8(const GemmEnv& env, const moe_i8* x, const float* x_scale, const int32_t* offsets, int R, int N, int K,
                      int E, const moe_i8* W, const float* w_scale, void* out, bool out_f32, hipStream_t s) {
    if (R == 0) return MOE_OK;
    const Call c{env, units(x), units(W), nullptr, out, offsets, {x_scale, w_scale, nullptr, R, 1}, R, E, N, K / 2, s};
    return out_f32 ? product<true>(c) : product<false>(c);
}

}  // namespace moe
