// By which rules 8-bit products of many groups depart from the tiles that bf16 products of the same sizes take (pick_config): plain
// arithmetic on sizes. K counts pairs of elements. Configurations: 0 256-row tiles, 1 128, 4 96, 2 64, 3 32 rows.
#pragma once
#include "expert_gemm_launch.h"

namespace moe {
namespace {

// Whether that many tiles, one on each compute unit at a time, leave at most a twentieth of their rounds' compute units idle.
bool full_rounds(double tiles, int cus) { return last_round_use(tiles, cus) >= 0.95; }

// Groups that pick_config expects to outgrow 128 rows now and then, and that mostly fit them (1.5 standard deviations above the
// mean): 128-row tiles instead of 256-row ones, with tiles for all compute units, where
//   - weight rows are a multiple of 4 KB apart: 256-row tiles stream them at the same k, 128-row ones in turn (turned_ksteps);
//   - the reduction has 4096 elements or more, but no more than `longest`, since a group that does outgrow its tile costs the stream
//     of a second one: 8192 for gate/up, 4096 down.
// us at 110 rows, 256- -> 128-row tiles, groups alike | drawn evenly, one or two past 128 rows | as skewed as rank^-0.5 (means of four
// places of the weights in memory). Gate/up: 16 experts of 4096 x 4096 140 -> 109 | 134 -> 127 | 151 -> 118, 8 of 4096 x 14336 219 ->
// 195 | 218 -> 193 | 219 -> 204, of 8192 x 8192 221 -> 199 | 214 -> 235 | 232 -> 224; longer, of 12288 x 8192 328 -> 298 | 315 -> 361 |
// 331 -> 354; other distances, of 7168 x 8192 186 -> 185 | 178 -> 214 | 197 -> 207. Down: 16 of 4096 x 4096 73 -> 57 | 72 -> 83 | 90 -> 75,
// 32 144 -> 115 | 139 -> 134 | 164 -> 124; longer, 8 of 4096 x 8192 78 -> 56 | 75 -> 87 | 70 -> 85, 16 of 8192 x 8192 205 -> 218 | 196 ->
// 254 | 244 -> 233; other distances, 8 of 4096 x 14336 131 -> 102 | 121 -> 157 | 119 -> 153.
bool mostly_fit_128_rows(int R, int E, int K, int longest, double tiles, int cus) {
    const double avg = static_cast<double>(R) / E;
    return K >= 2048 && 2 * K <= longest && 2 * K % 4096 == 0 && tiles >= cus && avg + 1.5 * std::sqrt(avg) <= 128.0;
}

// Gate/up. Reductions from 4096 elements on whose 128-row tiles make full rounds: those instead of 64- and 96-row ones from 46 rows
// a group on, because a group that outgrows the smaller tile costs more than the rows to spare. us, smaller -> 128-row tiles,
// groups alike | drawn evenly | as skewed as rank^-0.5: 46 rows, 8 experts of 8192 x 8192 180 -> 176 | 179 -> 176 | 200 -> 173, of 6144 x
// 16384 282 -> 277 | 276 -> 276 | 304 -> 278, 16 of 4096 x 4096 93 -> 95 | 92 -> 93 | 100 -> 94; 58 and 66 within 1 % even, skewed
// 205 -> 174 (8 of 8192 x 8192) to 234 -> 242 (16 of 6144 x 6144). With part of a round more: 46 rows, 8 of 4096 x 14336 157 -> 178 |
// 154 -> 168 | 174 -> 169, of 5120 x 10240 154 -> 166 | 154 -> 165 | 172 -> 166, 66 rows there 169 -> 173 | 164 -> 167 | 168 -> 178.
int i8_gateup_config(int config, int R, int E, int N, int K, int cus) {
    const double tiles = static_cast<double>(E) * (N / 128);
    if (config == 0) return mostly_fit_128_rows(R, E, K, 8192, tiles, cus) ? 1 : 0;
    const bool rows_to_spare = (config == 2 || config == 4) && K >= 2048 && R >= 46.0 * E && tiles >= cus && full_rounds(tiles, cus);
    return rows_to_spare ? 1 : config;
}

// A product whose tiles of 96 and 128 rows number `mid_n_tiles` across its N columns. Long reductions whose weights stream past
// groups of few rows: a tile with rows to spare takes the time of one that just holds the mean, and a group that outgrows its tile
// costs a second tile's stream, often a second round. So, of reductions from 4096 elements on:
//   - 96- and 128-row tiles where one round of them, or two full ones, leave few compute units idle;
//   - elsewhere 64- instead of 32-row tiles where those find all compute units, and 128- instead of 96-row ones.
// us, smaller tiles -> so, groups alike | as skewed as rank^-0.5: 8 experts of 4096 x 14336, 20 rows 72 -> 76 | 99 -> 73, 52 114 -> 78 |
// 108 -> 84; of 8192 x 8192, 20 88 -> 85 | 98 -> 82, 72 84 -> 85 | 130 -> 88; 32 -> 64 rows, 8 of 2048 x 8192, 18 27 -> 27 | 33 -> 27. Half
// the compute units idle: 8 of 2048 x 8192, 28 rows 22, 96-row tiles 34; a round and a half: 16 of 6144 x 6144, 20 rows 96, 114 |
// 101, 106; below 4096 elements: 64 of 2048 x 1408, 72 rows 43, 45 | 51, 55.
int i8_product_config(int config, int R, int E, int N, int K, int mid_n_tiles, int cus) {
    const double avg = static_cast<double>(R) / E, mid = static_cast<double>(E) * mid_n_tiles;
    if (config == 0) return mostly_fit_128_rows(R, E, K, 4096, mid, cus) ? 1 : 0;
    if (config == 1 || avg < 16.0 || K < 2048) return config;
    if (mid >= 0.6 * cus && mid <= 2.0 * cus && (mid <= cus || full_rounds(mid, cus))) return avg <= 32.0 ? 4 : 1;
    if (config == 3 && static_cast<double>(E) * (N / 64) >= cus) return 2;
    return config == 4 ? 1 : config;
}

}  // namespace
}  // namespace moe
