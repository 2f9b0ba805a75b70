// Grouped expert GEMMs on the gfx950 matrix cores (paper Table 1 row 3: per expert three
// d_h x d_e bf16 matrices, 6*rows*d_h*d_e FLOPs; Section 4.1: each expert is a gated FFN).
//
//   gate/up : H[p, j]  = bf16( SiLU(sum_i Xp[p,i] W1_e[j,i]) * (sum_i Xp[p,i] W3_e[j,i]) )
//   down    : Yp[p, c] = bf16( sum_j H[p,j] W2_e[c,j] )
// for every row p of expert e's group, offsets[e] <= p < offsets[e+1].
//
// A workgroup owns a BM x BN output tile of ONE expert; tiles are enumerated on the device
// from `offsets` (no host synchronisation, variable rows per expert, empty experts produce no
// tile). Every output element is one accumulator chain over k = 0,16,32,... with the same
// MFMA instruction in every tile configuration, so results do not depend on how many rows an
// expert has, on its place among the experts of a call or on which configuration is picked
// (coalesced == micro-batched, some experts == all of them, bit for bit).
#include <atomic>

#include "expert_gemm_launch.h"

namespace moe {

constexpr int kCounterSets = 64;
static __device__ __align__(256) int32_t tile_counter_sets[kCounterSets][kTileCounterBytes / sizeof(int32_t)];
static std::atomic<uint64_t> counter_sets_taken[64];         // one bit per set and device
static std::atomic<int32_t*> counter_sets_at[64];

int32_t* take_tile_counters(int device, int* set) {
    *set = -1;
    int32_t* base = counter_sets_at[device].load(std::memory_order_acquire);
    if (base == nullptr) {
        void* p = nullptr;
        if (hipGetSymbolAddress(&p, HIP_SYMBOL(tile_counter_sets)) != hipSuccess) {
            (void)hipGetLastError();
            return nullptr;
        }
        base = static_cast<int32_t*>(p);
        counter_sets_at[device].store(base, std::memory_order_release);
    }
    uint64_t taken = counter_sets_taken[device].load(std::memory_order_relaxed);
    while (~taken != 0) {
        const int n = __builtin_ctzll(~taken);
        if (counter_sets_taken[device].compare_exchange_weak(taken, taken | (1ull << n), std::memory_order_acq_rel)) {
            *set = n;
            return base + n * (kTileCounterBytes / sizeof(int32_t));
        }
    }
    return nullptr;
}

void give_tile_counters(int device, int set) {
    if (set >= 0) counter_sets_taken[device].fetch_and(~(1ull << set), std::memory_order_acq_rel);
}

int compute_units(int device) {
    static std::atomic<int> cached[64];
    int n = cached[device].load(std::memory_order_relaxed);
    if (n == 0) {
        if (hipDeviceGetAttribute(&n, hipDeviceAttributeMultiprocessorCount, device) != hipSuccess || n <= 0) {
            (void)hipGetLastError();
            n = 256;
        }
        cached[device].store(n, std::memory_order_relaxed);
    }
    return n;
}

namespace {

// Large tiles: four wavefronts of 128 x 128 outputs (one per SIMD) or eight of 128 x 64.
bool use_one_wave_per_simd(const GemmEnv& env, int N, int K) {
    if (!gemm::offsets_fit_1w(N, K)) return false;
    if (K % 128 != 0) return false;       // its k-loop takes two 64-wide steps per trip
    if (env.large_tile_waves != 0) return env.large_tile_waves == 4;
    return true;     // faster at every shape measured (reductions of 768 to 16384)
}

//                      BM   BN  BK WM WN NSTAGE DUAL [STREAM_B]
using GateUpLarge = Config<256, 256, 64, 2, 4, 2, true>;
// one wavefront per SIMD: 2 x 2 wavefronts of 128 x 128 outputs, fewer rows in lower tiles
using GateUpLarge1W = Config<256, 256, 64, 2, 2, 2, true>;
using DownLarge1W   = Config<256, 256, 64, 2, 2, 2, false>;
using GateUpMid   = Config<128, 256, 64, 2, 4, 3, true>;   // also the half-height tile of GateUpLarge
// 64 rows: four wavefronts of 32 rows share a workgroup, and its ring leaves room for a second
// workgroup on the compute unit, so that one streams weights while the other looks its tile up,
// waits for its first loads or stores; the two-wavefront tile with a four-stage ring of its own
// (one workgroup per compute unit) took 134 us at 500 tokens through 128 experts of 2048 x 768, gate/up,
// this one 126.5 us, and the down projection 86 -> 74 us
using GateUpSmall  = Config<64, 128, 64, 2, 2, 3, true>;
using GateUpSmallS = Config<64, 128, 64, 2, 2, 3, true, true>;
using DownSmallWide  = Config<64, 128, 64, 2, 2, 3, false>;
using DownSmallWideS = Config<64, 128, 64, 2, 2, 3, false, true>;
using DownSmall  = Config<64, 64, 64, 2, 2, 5, false>;    // more tiles
using DownSmallS = Config<64, 64, 64, 2, 2, 5, false, true>;
using DownLarge   = Config<256, 256, 64, 2, 4, 2, false>;
using DownMid     = Config<128, 128, 64, 2, 2, 4, false>;
using DownMidWide = Config<128, 256, 64, 2, 4, 3, false>;
using GateUpMidS   = Config<128, 256, 64, 2, 4, 3, true, true>;
using DownMidS     = Config<128, 128, 64, 2, 2, 4, false, true>;
using DownMidWideS = Config<128, 256, 64, 2, 4, 3, false, true>;
using GateUpMid96  = Config<96, 256, 64, 1, 4, 3, true>;
using GateUpMid96S = Config<96, 256, 64, 1, 4, 3, true, true>;
using DownMid96      = Config<96, 128, 64, 1, 4, 5, false>;
using DownMid96S     = Config<96, 128, 64, 1, 4, 5, false, true>;
using DownMid96Wide  = Config<96, 256, 64, 1, 4, 3, false>;
using DownMid96WideS = Config<96, 256, 64, 1, 4, 3, false, true>;
// A handful of rows per expert (decode). Four stages let two gate/up workgroups (three of the narrow
// down tiles) share a compute unit: at 2048 x 768 and 128 experts a tile has 32 or 12 k-steps, and with
// one workgroup per compute unit its lookup and first loads were a fifth of its time (37 tokens:
// gate/up 122 -> 114 us, down 72 -> 54 us). Seven stages where one workgroup per compute unit divides
// into whole rounds and two do not.
using GateUpTiny      = Config<32, 128, 64, 2, 2, 4, true>;
using GateUpTinyS     = Config<32, 128, 64, 2, 2, 4, true, true>;
using GateUpTinyDeepS = Config<32, 128, 64, 2, 2, 7, true, true>;
// A few tokens: more, narrower tiles. Four wavefronts (two, down) share their loads, which leave a wavefront
// one by one, some 100 cycles apart: one wavefront per tile took 15.8 us for gate/up of one token through 8 of
// 128 experts of 2048 x 768, four take 14.9, and 14.2 with the deep ring where no second tile has to fit; down
// of one token through 2 of 8 of 4096 x 14336 51.4 -> 45.5 us, of 6144 x 16384 73.1 -> 72.3.
using GateUpFewS     = Config<32, 64, 64, 2, 2, 4, true, true>;
using GateUpFewDeepS = Config<32, 64, 64, 2, 2, 6, true, true>;
using DownTiny     = Config<32, 64, 64, 2, 2, 4, false>;
using DownTinyS    = Config<32, 64, 64, 2, 2, 4, false, true>;
using DownFew      = Config<16, 32, 64, 1, 2, 6, false>;
using DownFewS     = Config<16, 32, 64, 1, 2, 6, false, true>;

// Tile of a gate/up launch that derives the groups from the selected experts (grouped_gemm_routed_kernel): those of
// launch_gateup's choice that leave every workgroup one tile or two. Beyond that each tile would pay for the
// derivation again.
enum class RoutedTile { none, few_deep, few, small_stream, small };
RoutedTile routed_tile(const GemmEnv& env, int R, int E, int d, int f) {
    if (R > gemm::kRoutedIds || env.forced_config >= 0 || env.stream_mode >= 0) return RoutedTile::none;
    const int cus = compute_units(env.device);
    switch (pick_config(env, R, E, gateup_tiles(E, d, f))) {
        case 3:
            if (!single_m_tile(env, R, E, 32) || !narrow_gateup_tiles(R, E, f, cus)) return RoutedTile::none;
            return one_tile_per_cu(R, E, f, cus) ? RoutedTile::few_deep : RoutedTile::few;
        case 2:
            if (most_row_tiles(R, E, 64) * (f / 64) > 2 * cus) return RoutedTile::none;
            return single_m_tile(env, R, E, 64) ? RoutedTile::small_stream : RoutedTile::small;
        default: return RoutedTile::none;
    }
}

template <class Cfg, int EW>
int launch_routed(const GemmEnv& env, const moe_bf16* x, const gemm::Routing& rt, int d, int f, int E,
                  const moe_bf16* W1, const moe_bf16* W3, moe_bf16* H, hipStream_t s) {
    static std::atomic<uint64_t> attr_set{0};
    const long long tiles = most_row_tiles(rt.T * rt.k, E, Cfg::BM) * (f / Cfg::BN_OUT);
    return launch_tiles(env, attr_set, gemm::grouped_gemm_routed_kernel<Cfg, EW>, Cfg::SMEM, Cfg::NTHREADS,
                        tiles + kXcds, s, x, W1, W3, H, rt, gemm::RowDiv(rt.k), E, f, d);
}

}  // namespace

bool gateup_routes(const GemmEnv& env, int T, int d, int f, int E, int k) {
    const RoutedTile t = routed_tile(env, T * k, E, d, f);
    if (t == RoutedTile::none) return false;
    // Ids at hand (device time of a layer call, separate launch -> without): 8 experts of 512 x 1024, 1 token 19.3 -> 17.4 us,
    // 16 20.1 -> 18.9, 256 24.8 -> 23.0, 500 27.9 -> 26.5. With the selection on the way, about one tile per compute unit: one
    // token through 8 of 128 experts of 2048 x 768 33.8 -> 32.2, 6 of 64 of 2048 x 1408 (1.03) 37.4 -> 36.7; two through 8 of 128
    // (1.5) 41.8 -> 43.1. Up to a token per wavefront.
    return E <= 16 || (T <= GateUpFewS::NW && (t == RoutedTile::few || t == RoutedTile::few_deep) &&
                       4 * most_row_tiles(T * k, E, 32) * (f / 32) <= 5 * compute_units(env.device));
}

int launch_gateup_routed(const GemmEnv& env, const moe_bf16* x, const float* logits, int32_t* topk_idx, float* topk_w,
                         int32_t* counts, int32_t* offsets, int32_t* perm, int32_t* inv_perm, int T, int d, int f,
                         int E, int k, const moe_bf16* W1, const moe_bf16* W3, moe_bf16* H, hipStream_t s) {
    const gemm::Routing rt{logits, topk_idx, topk_w, counts, offsets, perm, inv_perm, T, k};
    const RoutedTile tile = routed_tile(env, T * k, E, d, f);
    auto with = [&](auto cfg) {
        using Cfg = decltype(cfg);
        if (E <= 16) return launch_routed<Cfg, 0>(env, x, rt, d, f, E, W1, W3, H, s);
        if (E <= 64) return launch_routed<Cfg, 1>(env, x, rt, d, f, E, W1, W3, H, s);
        if (E <= 128) return launch_routed<Cfg, 2>(env, x, rt, d, f, E, W1, W3, H, s);
        return launch_routed<Cfg, 4>(env, x, rt, d, f, E, W1, W3, H, s);
    };
    switch (tile) {
        case RoutedTile::few_deep: return with(GateUpFewDeepS{});
        case RoutedTile::few: return with(GateUpFewS{});
        case RoutedTile::small_stream: return launch_routed<GateUpSmallS, 0>(env, x, rt, d, f, E, W1, W3, H, s);
        case RoutedTile::small: return launch_routed<GateUpSmall, 0>(env, x, rt, d, f, E, W1, W3, H, s);
        default: return MOE_ERR_UNSUPPORTED_SHAPE;
    }
}

// `a` is the grouped activation matrix [R, d] when row_index is NULL; otherwise it is the
// token matrix [T, d] and grouped row p reads token row_index[p] / index_div (the caller makes
// sure that T * d * 2 bytes fit a 32-bit offset). R bounds the rows of the E launched experts
// (it sizes the grid); R_hint is how many rows they are expected to hold together (it picks the
// tile configuration): the two differ when a call covers a subset of a layer's experts.
int launch_gateup(const GemmEnv& env, const moe_bf16* a, const int32_t* row_index, int index_div,
                  const int32_t* offsets, int R, int R_hint, int d, int f, int E,
                  const moe_bf16* W1, const moe_bf16* W3, moe_bf16* H, hipStream_t s) {
    if (R == 0) return MOE_OK;
    const moe_bf16* x_perm = a;
    int config = pick_config(env, R_hint, E, gateup_tiles(E, d, f));
    if (config == 0 && d / 64 < 3) config = 1;     // the pipelined kernel needs three k-steps
    // Row counts that lead to 96- or 128-row tiles let every group fit one, so their weights are streamed; the cached forms
    // (GateUpMid96, DownMid96 and DownMid96Wide) run under the tuning knob, those of 128 rows also where groups of about
    // 256 rows take two tiles and where a reduction is too short for the pipelined kernel.
    switch (config) {
        case 0:
            if (use_one_wave_per_simd(env, f, d))
                return launch_1w<GateUpLarge1W>(env, x_perm, W1, W3, H, offsets, row_index, index_div, R, E, f, d, s);
            return launch_ring<GateUpLarge, GateUpMid, 2, 3>(env, x_perm, W1, W3, H, offsets, row_index, index_div, R, E, f, d, s);
        case 1:
            if (single_m_tile(env, R_hint, E, 128))
                return launch_grouped<GateUpMidS>(env, x_perm, W1, W3, H, offsets, row_index, index_div, R, E, f, d, s);
            return launch_grouped<GateUpMid>(env, x_perm, W1, W3, H, offsets, row_index, index_div, R, E, f, d, s);
        case 4:
            if (single_m_tile(env, R_hint, E, 96))
                return launch_grouped<GateUpMid96S>(env, x_perm, W1, W3, H, offsets, row_index, index_div, R, E, f, d, s);
            return launch_grouped<GateUpMid96>(env, x_perm, W1, W3, H, offsets, row_index, index_div, R, E, f, d, s);
        case 3:
            if (single_m_tile(env, R_hint, E, 32)) {
                const double nt = touched_experts(R_hint, E) * (f / 64);
                const int cus = compute_units(env.device);
                if (narrow_gateup_tiles(R_hint, E, f, cus) || narrow_short_gateup_tiles(R_hint, E, d, f, cus)) {
                    if (one_tile_per_cu(R_hint, E, f, cus))
                        return launch_grouped<GateUpFewDeepS>(env, x_perm, W1, W3, H, offsets, row_index, index_div, R, E, f, d, s);
                    return launch_grouped<GateUpFewS>(env, x_perm, W1, W3, H, offsets, row_index, index_div, R, E, f, d, s);
                }
                // 16 tokens through 8 experts of 4096 x 14336, 7 rounds of one workgroup per compute unit or
                // 3.5 of two: 280 against 284 us; 4 tokens at 6144 x 16384, 6 or 3 rounds: 397 against 367
                if (last_round_use(nt, 2.0 * cus) < 0.93 * last_round_use(nt, cus))
                    return launch_grouped<GateUpTinyDeepS>(env, x_perm, W1, W3, H, offsets, row_index, index_div, R, E, f, d, s);
                return launch_grouped<GateUpTinyS>(env, x_perm, W1, W3, H, offsets, row_index, index_div, R, E, f, d, s);
            }
            return launch_grouped<GateUpTiny>(env, x_perm, W1, W3, H, offsets, row_index, index_div, R, E, f, d, s);
        default:
            if (single_m_tile(env, R_hint, E, 64))
                return launch_grouped<GateUpSmallS>(env, x_perm, W1, W3, H, offsets, row_index, index_div, R, E, f, d, s);
            return launch_grouped<GateUpSmall>(env, x_perm, W1, W3, H, offsets, row_index, index_div, R, E, f, d, s);
    }
}

namespace {

// F32: the same tilings with a float output matrix (gemm::F32Out).
template <bool F32>
int launch_down_as(const GemmEnv& env, const moe_bf16* H, const int32_t* offsets, int R, int R_hint,
                   int d, int f, int E, const moe_bf16* W2, moe_bf16* y_perm, hipStream_t s) {
    if (R == 0) return MOE_OK;
    const bool wide_mid = static_cast<long long>(E) * (d / 256) >= 160 && d % 256 == 0;
    const int cus = compute_units(env.device);
    int config = pick_config(env, R_hint, E, NTiles{d / 256, wide_mid ? d / 256 : d / 128, d / 64,
                                                    wide_mid ? 0.82 : 0.6, 0.27, 0.38, 2e-6 * E * d * f, f / 64});
    if (config == 0 && f / 64 < 3) config = 1;     // the pipelined kernel needs three k-steps
    switch (config) {
        case 0:
            if (use_one_wave_per_simd(env, d, f))
                return launch_1w<Out<F32, DownLarge1W>>(env, H, W2, nullptr, y_perm, offsets, nullptr, 1, R, E, d, f, s);
            return launch_ring<Out<F32, DownLarge>, Out<F32, DownMidWide>, 2, 3>(env, H, W2, nullptr, y_perm, offsets, nullptr, 1, R, E, d, f, s);
        case 1:
            // HBM-bound: wide tiles stream more bytes per workgroup, but only if there are
            // enough of them to occupy the 256 compute units (about one m-tile per expert).
            if (wide_mid) {
                if (single_m_tile(env, R_hint, E, 128))
                    return launch_grouped<Out<F32, DownMidWideS>>(env, H, W2, nullptr, y_perm, offsets, nullptr, 1, R, E, d, f, s);
                return launch_grouped<Out<F32, DownMidWide>>(env, H, W2, nullptr, y_perm, offsets, nullptr, 1, R, E, d, f, s);
            }
            if (single_m_tile(env, R_hint, E, 128))
                return launch_grouped<Out<F32, DownMidS>>(env, H, W2, nullptr, y_perm, offsets, nullptr, 1, R, E, d, f, s);
            return launch_grouped<Out<F32, DownMid>>(env, H, W2, nullptr, y_perm, offsets, nullptr, 1, R, E, d, f, s);
        case 4:
            // wide tiles where there are enough of them for the 256 compute units, as for case 1
            if (wide_mid) {
                if (single_m_tile(env, R_hint, E, 96))
                    return launch_grouped<Out<F32, DownMid96WideS>>(env, H, W2, nullptr, y_perm, offsets, nullptr, 1, R, E, d, f, s);
                return launch_grouped<Out<F32, DownMid96Wide>>(env, H, W2, nullptr, y_perm, offsets, nullptr, 1, R, E, d, f, s);
            }
            if (single_m_tile(env, R_hint, E, 96))
                return launch_grouped<Out<F32, DownMid96S>>(env, H, W2, nullptr, y_perm, offsets, nullptr, 1, R, E, d, f, s);
            return launch_grouped<Out<F32, DownMid96>>(env, H, W2, nullptr, y_perm, offsets, nullptr, 1, R, E, d, f, s);
        case 3:
            // 32-column tiles where 64-column ones would leave compute units without any: one token through 2 of
            // 8 experts of 4096 x 14336 45.5 against 61.7 us; and while all of their row tiles find one: 64 tokens
            // through 2 of 8 of 512 x 1024 7.9 against 9.1 us
            if (touched_experts(R_hint, E) * (d / 64) < cus) {
                if (single_m_tile(env, R_hint, E, 16))
                    return launch_grouped<Out<F32, DownFewS>>(env, H, W2, nullptr, y_perm, offsets, nullptr, 1, R, E, d, f, s);
                if (row_tiles(R_hint, E, 16) * (d / 32) <= cus)
                    return launch_grouped<Out<F32, DownFew>>(env, H, W2, nullptr, y_perm, offsets, nullptr, 1, R, E, d, f, s);
            }
            if (single_m_tile(env, R_hint, E, 32))
                return launch_grouped<Out<F32, DownTinyS>>(env, H, W2, nullptr, y_perm, offsets, nullptr, 1, R, E, d, f, s);
            return launch_grouped<Out<F32, DownTiny>>(env, H, W2, nullptr, y_perm, offsets, nullptr, 1, R, E, d, f, s);
        default:
            // 32-row tiles where the 64-row ones would leave half of the compute units without any: 256 tokens through
            // 2 of 8 experts of 512 x 1024 (96 tiles) 9.2 against 9.9 us, 600 (192 tiles) 10.9 against 10.2
            if (row_tiles(R_hint, E, 64) * (d / 64) <= 0.5 * cus)
                return launch_grouped<Out<F32, DownTiny>>(env, H, W2, nullptr, y_perm, offsets, nullptr, 1, R, E, d, f, s);
            // 128 columns where that makes about two rounds of two workgroups per compute unit, else 64. Layer calls
            // with cold weights, 128 against 64 columns: 500 tokens through 128 experts of 2048 x 768 (8 tiles of 128
            // columns per compute unit) 239 and 243 us, 448 through 56 of 2048 x 1024, 4 per token (3.5) 149.2 and
            // 150.5; 110 tokens through 8 of 6144 x 16384 (1.5) 806 and 783. In between the sides are mixed (3.0: 384
            // tokens through 48 of 2048 x 1024 128.7 and 134.6, 192 through 24 of 4096 x 2048 242 and 238)
            if (touched_experts(R_hint, E) * (d / 128) >= 3.5 * cus) {
                if (single_m_tile(env, R_hint, E, 64))
                    return launch_grouped<Out<F32, DownSmallWideS>>(env, H, W2, nullptr, y_perm, offsets, nullptr, 1, R, E, d, f, s);
                return launch_grouped<Out<F32, DownSmallWide>>(env, H, W2, nullptr, y_perm, offsets, nullptr, 1, R, E, d, f, s);
            }
            if (single_m_tile(env, R_hint, E, 64))
                return launch_grouped<Out<F32, DownSmallS>>(env, H, W2, nullptr, y_perm, offsets, nullptr, 1, R, E, d, f, s);
            return launch_grouped<Out<F32, DownSmall>>(env, H, W2, nullptr, y_perm, offsets, nullptr, 1, R, E, d, f, s);
    }
}

}  // namespace

// y_perm is [R, d] bf16, or [R, d] fp32 when y_f32 is set.
int launch_down(const GemmEnv& env, const moe_bf16* H, const int32_t* offsets, int R, int R_hint,
                int d, int f, int E, const moe_bf16* W2, void* y_perm, bool y_f32, hipStream_t s) {
    moe_bf16* out = static_cast<moe_bf16*>(y_perm);
    return y_f32 ? launch_down_as<true>(env, H, offsets, R, R_hint, d, f, E, W2, out, s)
                 : launch_down_as<false>(env, H, offsets, R, R_hint, d, f, E, W2, out, s);
}

}  // namespace moe
