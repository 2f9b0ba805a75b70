// Launch wrappers of the expert GEMM kernels and the rules by which a call picks its tiles, shared by the translation units
// that instantiate them for bf16 and for 8-bit operands.
#pragma once
#include <algorithm>
#include <atomic>
#include <cmath>

#include "expert_gemm_kernel.h"

namespace moe {
namespace {

using gemm::Config;
template <bool F32, class Cfg>
using Out = std::conditional_t<F32, gemm::F32Out<Cfg>, Cfg>;

// `most_smem`: the LDS of the largest launch of this kernel, `smem` that of this one.
template <class Kernel, class... Args>
int launch_tiles_sized(const GemmEnv& env, std::atomic<uint64_t>& attr_set, Kernel kern, int most_smem, int smem,
                       int threads, long long grid, hipStream_t s, Args... args) {
    // The attribute belongs to the kernel's code object on ONE device: one bit per device, set
    // by whichever thread launches this kernel there first (setting it twice is harmless).
    if (env.device < 0 || env.device >= 64) return MOE_ERR_INVALID_ARG;
    const uint64_t bit = 1ull << env.device;
    if (!(attr_set.load(std::memory_order_acquire) & bit)) {
        if (hipFuncSetAttribute(reinterpret_cast<const void*>(kern),
                                hipFuncAttributeMaxDynamicSharedMemorySize, most_smem) != hipSuccess)
            return MOE_ERR_HIP;
        attr_set.fetch_or(bit, std::memory_order_release);
    }
    grid = (grid + kXcds - 1) / kXcds * kXcds;
    if (grid > 0x7fffffffLL) return MOE_ERR_UNSUPPORTED_SHAPE;
    hipLaunchKernelGGL(kern, dim3(static_cast<unsigned>(grid)), dim3(threads), smem, s, args...);
    return hipGetLastError() == hipSuccess ? MOE_OK : MOE_ERR_HIP;
}
template <class Kernel, class... Args>
int launch_tiles(const GemmEnv& env, std::atomic<uint64_t>& attr_set, Kernel kern, int smem,
                 int threads, long long grid, hipStream_t s, Args... args) {
    return launch_tiles_sized(env, attr_set, kern, smem, smem, threads, grid, s, args...);
}

// Most row tiles that R rows in E groups can make: a group of m > 0 rows has ceil(m / BM) of them, so
// all groups together have at most R / BM + min(E, R). The bound sizes the grid, and a workgroup
// without a tile still occupies a compute unit's LDS while it finds that out (about 1 us, one at
// a time per compute unit with the deep rings): one token through 8 of 128 experts used to launch
// 4096 workgroups for the 256 tiles of the down projection, 25.0 us for 25 MB of weights; with
// min(E, R) in place of E it takes 9.0 us (gate/up 18.5 -> 16.5 us).
long long most_row_tiles(int R, int E, int BM) { return R / BM + std::min(E, R); }

// Experts that R rows are expected to touch.
double touched_experts(int R, int E) { return E * (1.0 - std::exp(-static_cast<double>(R) / E)); }

// Step of the staggered first starts of the weight-bound tiles (gemm::spread_start), 0: together. Together -> steps of
// 1 -> of 2, in us: pitch of 32 KB (down, 8 experts of 6144 x 16384) 16 tokens 257, 251, 246; 64 261, 256, 252; 256 291, 279,
// 271; 420 314, 306, 297. Pitch of 12 KB (gate/up there) 489, 485, 480; 501, 501, 501; 549, 547, 543; 594, 594, 590; 200 tokens
// 582, 536, 531. Pitch of 28 KB (down, 4096 x 14336) 64 tokens 154, 152, 150; 128 160, 160, 159; 200 188, 187, 186; but 256, a tile
// per compute unit, 168, 169, 176, so steps of 2 only at the worst pitch. A reduction of 4096 ends too soon for it: gate/up,
// 16 tokens at 4096 x 14336 279 together, 290 with eight starts over the same span; nor does a launch of few weights pay for
// the last starts, 11 us late with steps of 1 (one token through 2 of 8 experts of 4096 x 14336, 235 MB of W2: layer call
// 126.8 us together, 137.5; of 6144 x 16384, 403 MB, 202.7 and 211). Other reductions, both projections of 8 experts with
// the same rows each, together -> as here: 8192 x 8192 4 rows 514 -> 506, 60 531 -> 519; 10240 x 10240 4 775 -> 738, 32
// 803 -> 790; 12288 x 8192 32 754 -> 747; 7168 x 18432 60 1101 -> 1072; within 1 % of each other where the pitch is no multiple
// of 4 KB (11008, 6656, 7680, 17920). A gate/up reduction of 5120 gains nothing: 4 rows 485 -> 487 with steps of 1, 60 593 -> 595.
int spread_steps(int R, int E, int N, int K, bool dual) {
    const double bytes = touched_experts(R, E) * (dual ? 4.0 : 2.0) * N * K;
    return K < 6144 || bytes < 0.8e9 ? 0 : K % 16384 == 0 ? 2 : 1;
}

// Whether weight rows that far apart in bytes, streamed at the same k by workgroups that started together, fall on few memory
// channels: a multiple of 4 KB, or a divisor of it, with which every few rows come round to the same place.
bool rows_on_few_channels(int pitch) { return pitch % 4096 == 0 || 4096 % pitch == 0; }

// Whether the n-tiles of a product of whole numbers start at k-steps of their own (gemm::first_kstep) instead of together or late:
//   - rows 4 KB or a multiple apart;
//   - gate/up of 32 n-tiles and more, rows a divisor of 4 KB apart;
//   - 96- and 128-row tiles, rows more than 4 KB apart.
// Never 16-row tiles (8192 x 2048, one row 19.6 -> 22 us). Together -> so, us, other weights for every call. Multiples: expert FFN
// of 8 experts of 8192 x 8192, 12 rows each 271 -> 257, 64 317 -> 260. Divisors, gate/up: 6 rows for each of 8 of 2048 x 8192 53.5 ->
// 44.3, 32 of 2048 x 2048 55 -> 46, 8 of 1024 x 16384 53.8 -> 52.6, of 512 x 16384 32.5 -> 31.8 (at worst 24 for each of 32 of 1024 x 2048
// 27.5 -> 28.3); fewer n-tiles, 24 for each of 64 of 2048 x 1408 65 -> 67; down, 7168 x 2048 22 -> 23. Others: gate/up at 1536 and
// 10240 within 1 %, 2560 57 -> 58, 3584 76 -> 77, 14336 563 -> 568, but all longer ones of 96- and 128-row tiles, whose workgroups are
// the fewest, gain: 90 rows, 8 of 4096 x 14336, down turned too 290 -> 275.
template <class Cfg>
bool turned_ksteps(int N, int K) {
    if (!gemm::operands_i8<Cfg>::value || Cfg::BM == 16) return false;
    const int pitch = 2 * K;
    return pitch % 4096 == 0 || (Cfg::BM >= 96 && pitch > 4096) ||
           (Cfg::DUAL && N >= 32 * Cfg::BN_OUT && rows_on_few_channels(pitch));
}
// The same of the pipelined tiles: for one matrix and one row tile (several share an n-tile's weights, but each n-tile then asks
// for rows of its own: 14336 x 4096, 1003 rows 68 -> 75) at both kinds of distance. us, 37 rows, 32000 columns, other weights for
// every call: of 1024 10.4 -> 10.0, 2048 18.2 -> 16.1, 4096 31.2 -> 27.7, 8192 57 -> 51; between them 1536 13.7 -> 13.5, 2560 21.6 ->
// 21.5, 3584 25.8 -> 26.2, 5120 37.4 -> 36.7, 7168 46.4 -> 47.3; 16384 columns of 14336 45 -> 47. 4096 columns: within 1 %.
template <class Cfg>
bool turned_ksteps_of_one(int R, int E, int K) {
    return E == 1 && R <= Cfg::BM && rows_on_few_channels(2 * K);
}

// Whether tiles of Cfg::BN_OUT columns cover N of them (gemm::n_tiles).
template <class Cfg>
bool columns_fit(int N) {
    return gemm::operands_i8<Cfg>::value ? N >= Cfg::BN_OUT : N % Cfg::BN_OUT == 0;
}

// The generic kernel with Cfg::NSTAGE stages.
template <class Cfg>
int launch_grouped(const GemmEnv& env, const moe_bf16* A, const moe_bf16* B0, const moe_bf16* B1, moe_bf16* C,
                   const int32_t* offsets, const int32_t* row_index, int index_div,
                   int R, int E, int N, int K, hipStream_t s, const gemm::ScalesOf<Cfg>& scales = {}) {
    if (!columns_fit<Cfg>(N) || K % Cfg::BK != 0) return MOE_ERR_UNSUPPORTED_SHAPE;
    static std::atomic<uint64_t> attr_set{0};
    const long long max_mt = most_row_tiles(R, E, Cfg::BM);
    return launch_tiles(env, attr_set, gemm::grouped_gemm_kernel<Cfg>, Cfg::SMEM, Cfg::NTHREADS,
                        max_mt * gemm::n_tiles<Cfg>(N), s, A, B0, B1, C, offsets, row_index,
                        gemm::RowDiv(index_div), E, N, K,
                        turned_ksteps<Cfg>(N, K) ? -1 : spread_steps(R, E, N, K, Cfg::DUAL), scales);
}

// The pipelined form of the generic kernel.
template <class Cfg>
int launch_pipelined(const GemmEnv& env, const moe_bf16* A, const moe_bf16* B0, const moe_bf16* B1, moe_bf16* C,
                     const int32_t* offsets, int R, int E, int N, int K, hipStream_t s,
                     const gemm::ScalesOf<Cfg>& scales = {}) {
    int splits = 1;
    if constexpr (gemm::raw_sums<Cfg>::value) splits = scales.splits;
    if (!columns_fit<Cfg>(N) || K % Cfg::BK != 0 || K / Cfg::BK / splits < Cfg::NSTAGE) return MOE_ERR_UNSUPPORTED_SHAPE;
    static std::atomic<uint64_t> attr_set{0};
    return launch_tiles(env, attr_set, gemm::grouped_gemm_pipelined_kernel<Cfg>, Cfg::SMEM, Cfg::NTHREADS,
                        most_row_tiles(R, E, Cfg::BM) * gemm::n_tiles<Cfg>(N) * splits, s, A, B0, B1, C, offsets, gemm::RowDiv(1), E, N, K,
                        turned_ksteps_of_one<Cfg>(R, E, K), scales);
}

// Slots of all tiles that R rows in E groups can make: the tiles, and where the last round is split two slots
// per tile there, at most ceil(cus / 2 / 8) more in every XCD's range.
long long most_slots(int R, int E, int BM, int NT, int split_cus) {
    return most_row_tiles(R, E, BM) * NT + kXcds * ((split_cus / 2 + kXcds - 1) / kXcds + 1);
}

// The pipelined kernel of eight wavefronts with operand rings of NA and NB stages; tiles of at most HalfCfg::BM
// rows and the tiles of a last round that is less than half full run at half the height.
template <class Cfg, class HalfCfg, int NA, int NB>
int launch_ring(const GemmEnv& env, const moe_bf16* A, const moe_bf16* B0, const moe_bf16* B1, moe_bf16* C,
                const int32_t* offsets, const int32_t* row_index, int index_div,
                int R, int E, int N, int K, hipStream_t s) {
    if (N % Cfg::BN_OUT != 0 || K % Cfg::BK != 0) return MOE_ERR_UNSUPPORTED_SHAPE;
    if (K / Cfg::BK < (NA > NB ? NA : NB)) return MOE_ERR_UNSUPPORTED_SHAPE;
    static std::atomic<uint64_t> attr_set{0};
    const int cus = env.split_last_round ? compute_units(env.device) : 0;
    return launch_tiles(env, attr_set, gemm::grouped_gemm_ring_kernel<Cfg, HalfCfg, NA, NB>,
                        gemm::RingCfg<Cfg, NA, NB>::SMEM, Cfg::NTHREADS,
                        most_slots(R, E, Cfg::BM, N / Cfg::BN_OUT, cus), s, A, B0, B1, C,
                        offsets, row_index, gemm::RowDiv(index_div), E, N, K, cus);
}

// Expected row tiles of height h: groups one standard deviation below and above the mean.
double mean_row_tiles(double avg, double sigma, int h) {
    return 0.5 * (std::ceil(std::max(1.0, avg - sigma) / h) + std::ceil((avg + sigma) / h));
}

// Expected row tiles of height h of a launch.
double row_tiles(int R, int E, int h) {
    const double avg = static_cast<double>(R) / (E > 0 ? E : 1);
    return E * mean_row_tiles(avg, std::sqrt(avg), h);
}

// The pipelined kernel of one wavefront per SIMD: a persistent workgroup per compute unit where the reduction is
// short and most of them get two tiles and more, else a workgroup per tile (4000 tokens through 8 experts of 512 x 1024,
// one tile per compute unit, 62.4 us a layer with persistent ones, 60.9 without).
template <class Cfg, bool ODD = false>
int launch_1w(const GemmEnv& env, const moe_bf16* A, const moe_bf16* B0, const moe_bf16* B1, moe_bf16* C,
              const int32_t* offsets, const int32_t* row_index, int index_div,
              int R, int E, int N, int K, hipStream_t s, const gemm::ScalesOf<Cfg>& scales = {}) {
    if (!columns_fit<Cfg>(N) || K % (ODD ? Cfg::BK : 2 * Cfg::BK) != 0 || K < 4 * Cfg::BK) return MOE_ERR_UNSUPPORTED_SHAPE;
    static std::atomic<uint64_t> attr_set[2];
    const int cus = compute_units(env.device), split = env.split_last_round ? cus : 0, nt = gemm::n_tiles<Cfg>(N);
    const long long slots = most_slots(R, E, Cfg::BM, nt, split);
    if (K < gemm::kLongK && row_tiles(R, E, Cfg::BM) * nt > 1.5 * cus)
        return launch_tiles(env, attr_set[0], gemm::grouped_gemm_1w_kernel<Cfg, true, ODD>, gemm::Ring1W<Cfg>::SMEM,
                            Cfg::NTHREADS, std::min<long long>(slots, cus), s, A, B0, B1, C, offsets, row_index,
                            gemm::RowDiv(index_div), E, N, K, split, env.tile_counters, scales);
    return launch_tiles(env, attr_set[1], gemm::grouped_gemm_1w_kernel<Cfg, false, ODD>, gemm::Ring1W<Cfg>::SMEM,
                        Cfg::NTHREADS, slots, s, A, B0, B1, C, offsets, row_index, gemm::RowDiv(index_div), E, N, K,
                        split, env.tile_counters, scales);
}

// The n-tiles of one projection in each kind of tile, and what the small tiles of config 2 cost.
struct NTiles {
    int large, mid, small;
    double mid_step;             // k-step of the 96- and 128-row tiles, of a 256-row tile's
    double small_alone, small_pair;   // k-step of a 64-row tile alone on a compute unit / of two on one
    double weight_mb;            // of the launched experts
    int ksteps;                  // of the reduction
};

// Tile configuration by average rows per expert. All configurations give identical bits.
//
// The measured constants of this rule and of the variants in launch_gateup and launch_down, and what each stands
// on ("cold": a graph of calls with other weights every time, 1.2 GB and more of them; else the same ones):
//   0.82, 0.6   k-step of a 96- or 128-row tile (256 or 128 columns), 0.41 / 0.58 and 0.27 / 0.38 of one 64-row
//               tile alone on a compute unit / of two: one expert of 4096 x 14336, 512 rows (below)
//   0.56, 0.8   k-step of a 256-row tile where at most half the compute units have one, weights from cache / from
//   (64 MB)     memory. The line only has to keep large weights from the lower price: 512 rows through one
//               expert of 4096 x 14336 234 us a layer cold with 0.8, 293 with 0.56. Layers of up to 64 MB differ
//               by -4 to +5 % either way, cold or not (1024 rows through 4 of 2048 x 1408 cold 82.7 us with 0.56,
//               80.8 with 0.8; 1600 through 8 of 2048 x 768 61.6 and 64.5), and of three such layers, 256 to 6000
//               rows, none is over 1 % slower cold than with the 128- or the 256-row tiles throughout
//   + 3, + 6    a tile's cost outside its reduction, in k-steps, and 0.9 the margin that small tiles have to win by:
//               512 and 900 tokens through 8 experts of 512 x 1024 (below)
//   0.93        seven stages against four, 2.5 narrow gate/up tiles, 3.5 128 columns down: where they are used
int pick_config(const GemmEnv& env, int R, int E, const NTiles& nt) {
    if (env.forced_config >= 0) return env.forced_config;
    // 0: pipelined 256-row tiles (lower ones at the end). 1: 128-row tiles (generic kernel).
    // 2: up to 64 rows per expert (64-row tiles, two workgroups per compute unit). 3: up to 32
    // (32-row tiles). 4: 96-row tiles of four wavefronts side by side (groups of 65 to 96 rows: a
    // quarter fewer matrix instructions and fragment reads per k-step than the 128-row tile, and
    // room for a deeper weight ring in the down projection). Per-expert counts are not known on
    // the host, so the choice prices a uniform routing: the average group and its standard deviation.
    const double avg = static_cast<double>(R) / (E > 0 ? E : 1);
    const double sigma = std::sqrt(avg);
    const double upper = avg + 2.0 * sigma;
    if (upper <= 32.0) return 3;
    // The 64-row tiles against the 96-row ones, gate/up + down: 500 tokens through 128 experts of
    // 2048 x 768 205 us against 218; with a few experts past 64 rows (560 tokens through 64 experts of
    // 2048 x 1408) 226 against 211. Layers on the same weights: 195 tokens through 8 of 4096 x 14336 502 against 524, of
    // 6144 x 16384 830 against 817; past the line, 205 there 905 against 849, 810 through 128 of 2048 x 768 281 against 268.
    if (upper <= 64.0) return 2;
    const int cus = compute_units(env.device);
    // The 96- and 128-row tiles only where the largest group is expected to fit one: a second tile costs more than
    // they gain. The largest of E groups lies about sqrt(2 ln E) standard deviations above the mean (two for the
    // 8 experts that the lines were drawn at). Gate/up and down, 96- / 128- / 256-row tiles: 800 tokens through 64 experts
    // of 2048 x 1408 (75 rows each) 154 and 79, 154 and 79, 154 and 77 us; 280 through 8 of 6144 x 16384 (70) 517 and 277,
    // 520 and 276, 543 and 336. 128- / 256-row: 1700 through 128 of 2048 x 768 (106) 174 and 111, 158 and 103;
    // 420 through 8 of 4096 x 14336 (105) 354 and 185, 358 and 232; 460 (115) 370 and 306, 362 and 234. With more rows the
    // 256-row tiles and their lower tails are the faster ones (4096 x 14336, 600 tokens 479 and 313, 393 and 240, 2048 1000
    // and 725, 761 and 498; two experts of 4096 x 14336 with 300 rows each, gate/up 179 and 147).
    const double largest = avg + std::max(2.0, std::sqrt(2.0 * std::log(static_cast<double>(E)))) * sigma;
    int config = largest <= 96.0 ? 4 : largest <= 128.0 ? 1 : 0;
    // Groups around 256 rows, where one 256-row tile per expert leaves compute units idle and the few groups of more
    // than 256 rows start a second round: two or three 128-row tiles per expert are two rounds too, of half the
    // height. Down, 8 experts of 6144 x 16384, 256- against 128-row tiles: 1000 tokens 656 and 544 us, 1024 671 and 547;
    // below the lines, one large round, 975 472 and 528; above, three of the others, 1050 633 and 742. With reductions of
    // 12288, 8192, 6144 438 and 407, 290 and 261, 229 and 217 (1024 tokens); below that a wrong guess of the groups costs as
    // much as a right one gains (12 experts, K = 4096 102 and 134 or 143 and 132, as the routing falls).
    const double past256 = 0.5 * E * std::erfc((256.0 - avg) / (std::sqrt(2.0) * sigma));   // groups, expected
    if (config == 0 && nt.ksteps >= 96 && E * nt.large <= cus && (E + past256) * nt.large > cus &&
        (2.0 * E + past256) * nt.mid <= 0.95 * 2.0 * cus)
        config = 1;
    // A launch of at most one such tile per compute unit takes one tile's time however many compute
    // units idle: small tiles are worth their extra loads if they use the idle ones. Units of a
    // k-step of a full 256-row tile (about 1 us), measured on one expert of 4096 x 14336 (512 rows,
    // down projection: 125 us with large tiles, 94 and 87 us with 64-row ones of 128 and 64 columns;
    // 181 against 124 us when the weights come from memory, which a compute unit reads at 60 GB/s). What a
    // tile costs outside its reduction is added in k-steps, and decides where that is short (layer call of
    // 512 tokens through 8 experts of 512 x 1024 27.9 us with large gate/up tiles, 26.6 with 64-row ones; 900
    // tokens 29.1 and 28.1).
    const int rows = config == 0 ? 256 : config == 1 ? 128 : 96;
    const double tiles = E * mean_row_tiles(avg, sigma, rows) * (config == 0 ? nt.large : nt.mid);
    if (tiles <= cus) {
        const double step = config != 0 ? nt.mid_step : tiles <= 0.5 * cus ? (nt.weight_mb > 64.0 ? 0.8 : 0.56) : 1.0;
        const double small = E * mean_row_tiles(avg, sigma, 64) * nt.small;
        const double rounds = std::floor(small / (2.0 * cus)), rem = small - rounds * 2.0 * cus;
        const double fill = rounds * nt.small_pair + (rem <= 0.0 ? 0.0 : rem <= cus ? nt.small_alone : nt.small_pair);
        if ((nt.ksteps + 3.0) * fill < 0.9 * (nt.ksteps + 6.0) * step) return 2;
    }
    return config;
}

NTiles gateup_tiles(int E, int d, int f) {
    return NTiles{f / 128, f / 128, f / 64, 0.82, 0.41, 0.58, 4e-6 * E * d * f, d / 64};
}

// Tiles of half the width while up to two and a half of them go to a compute unit, gate/up against
// the 128-column ones: one token through 8 of 128 experts of 2048 x 768 (0.75 per compute unit) 14.2
// and 18.2 us, 2 (1.4) 21.6 and 22.3, 2 through 6 of 64 of 2048 x 1408 (2.1) 23.9 and 25.0, 64 through
// 2 of 8 of 512 x 1024 (1.0) 7.7 and 8.7. Longer reductions than those below lose past the line: layers of 4096 x 14336,
// one token through 2 of 8 (3.3) 142 and 129, of 6144 x 16384 (3.7) 229 and 220
bool narrow_gateup_tiles(int R, int E, int f, int cus) { return 2.0 * touched_experts(R, E) * (f / 64) <= 2.5 * cus; }

// Workgroups of `tiles` tiles that find a free slot per round, over the slots of those rounds.
double last_round_use(double tiles, double slots) { return tiles / (slots * std::ceil(tiles / slots)); }

// Short reductions, more than that: a tile of half the width leaves half as much of the last round empty, except
// where both widths take two rounds (three to four narrow tiles per compute unit) or the wide ones fill theirs. Layers
// through 8 of 128 experts of 2048 x 768, wide -> narrow: 4 tokens (2.6) 66.6 -> 62.8 us, 5 (3.3) 69.8 -> 72.7, 7 (4.4)
// 99.4 -> 88.6, 20 (8.7) 155 -> 150, 37 (10.8) 184 -> 180, 120 (12, all full) 209 -> 213; 6 of 64 of 2048 x 1408, 4 tokens
// (3.6) 70.0 -> 70.8, 16 (8.7) 151 -> 145, 80 (11) 182 -> 178; 4 of 60 of 1536 x 1536, 30 tokens 133 -> 127.
bool narrow_short_gateup_tiles(int R, int E, int d, int f, int cus) {
    const double wide = touched_experts(R, E) * (f / 64);
    return d <= 2048 && (2.0 * wide <= 3.0 * cus || wide > 2.0 * cus) && last_round_use(wide, cus) <= 0.97;
}

// The deep ring where no compute unit gets a second tile, whichever experts are touched: one
// token through 8 of 128 of 2048 x 768 (192 tiles) 14.3 against 14.9 us, through 4 of 32 of 2048 x 2048
// (256) 16.7 against 17.5; through 6 of 64 of 2048 x 1408 (264) 20.2 against 18.2
bool one_tile_per_cu(int R, int E, int f, int cus) { return std::min(E, R) * (f / 32) <= cus; }

// Weights may be loaded as non-temporal when (almost) every expert has a single m-tile: then no
// other tile asks for the same weight bytes and keeping them cached only displaces the rows.
bool single_m_tile(const GemmEnv& env, int R, int E, int BM) {
    if (env.stream_mode >= 0) return env.stream_mode != 0;
    const double avg = static_cast<double>(R) / (E > 0 ? E : 1);
    return avg + 2.0 * std::sqrt(avg) <= BM;
}

}  // namespace
}  // namespace moe
