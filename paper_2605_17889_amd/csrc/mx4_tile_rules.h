// By what price 4-bit products pick their tiles: plain arithmetic on sizes.
//
// A launch runs in rounds of `resident` tiles per compute unit. A round takes `fixed` us and, for each k-step of 256 elements,
// `alone` us with a tile on a compute unit or `full` with all it holds; a launch takes its rounds, or the time that its weights
// take from memory if that is longer, and a fifth of the shorter of the two. The figures are fits to single products of 4096 and
// 14336 elements through 4096 columns (one and two tiles per compute unit) and, for gate/up, to the experts of the presets;
// at 111 launches (the two of each of 36 expert FFNs, 39 products), those among them, the tile of the lowest price is the fastest
// one or within 6 % of it but for six (7 to 14 %); 1 % on average.
#pragma once
#include <algorithm>
#include <cmath>

namespace moe {
namespace {

struct MxTile {
    int id, rows, columns;           // of outputs
    int resident;
    double alone, full, fixed;
};
enum MxPlain { kMxFew, kMxFewWide, kMx16x64, kMx32x64Deep, kMx32x64, kMx64x64, kMx64x128, kMx128x128, kMx128x128Pair,
               kMxLarge };
enum MxGateUp { kMxGateFew, kMxGate32, kMxGate64, kMxGate128, kMxGateLarge };

//                                    id              rows cols res. alone   full    fixed
constexpr MxTile kMxPlainTiles[] = {{kMxFew,          16,  16,  2,   0.12,   0.25,   2.5},
                                    {kMxFewWide,      16,  32,  2,   0.20,   0.35,   4.2},
                                    {kMx16x64,        16,  64,  2,   0.265,  0.3775, 3.0},
                                    {kMx32x64Deep,    32,  64,  2,   0.2575, 0.4425, 3.3},
                                    {kMx32x64,        32,  64,  4,   0.3625, 0.75,   3.0},
                                    {kMx64x64,        64,  64,  2,   0.3325, 0.5825, 3.1},
                                    {kMx64x128,       64,  128, 2,   0.5175, 1.0075, 4.0},
                                    {kMx128x128,      128, 128, 1,   0.7175, 0.7175, 6.0},
                                    {kMx128x128Pair,  128, 128, 2,   1.0,    1.2,    6.5},
                                    {kMxLarge,        256, 256, 1,   1.0,    1.5,    8.0}};
constexpr MxTile kMxGateUpTiles[] = {{kMxGateFew,     32,  32,  2,   0.34,   0.60,   3.8},
                                     {kMxGate32,      32,  64,  2,   0.44,   0.80,   4.0},
                                     {kMxGate64,      64,  64,  2,   0.52,   1.0,    5.0},
                                     {kMxGate128,     128, 128, 1,   1.25,   1.4,    7.0},
                                     {kMxGateLarge,   256, 128, 1,   1.0,    1.5,    8.0}};
constexpr double kMxWeightBytesPerUs = 6.4e6;
constexpr int kMxRunElements = 256;  // of a k-step
// The large tiles draw on the board's power: up to this part of the compute units they run at the pace of one alone.
constexpr double kMxLargeAlone = 0.6;

// Experts that hold a row, and row tiles of `h` rows, under uniform routing: half of the groups a standard deviation below the mean
// and half above it.
double mx_touched(int R, int E) { return E == 1 ? 1.0 : std::ceil(E * (1.0 - std::exp(-static_cast<double>(R) / E))); }
double mx_row_tiles(int R, int E, int h) {
    if (E == 1) return std::ceil(static_cast<double>(R) / h);
    const double touched = mx_touched(R, E), avg = R / touched, sigma = touched > 1.5 ? std::sqrt(avg) : 0.0;
    return touched * 0.5 * (std::ceil(std::max(1.0, avg - sigma) / h) + std::ceil((avg + sigma) / h));
}

double mx_price(const MxTile& t, bool large, bool dual, int R, int E, int N, int K, int cus) {
    const double ksteps = (K + 255) / 256, tiles = mx_row_tiles(R, E, t.rows) * ((N + t.columns - 1) / t.columns);
    const double slots = static_cast<double>(t.resident) * cus, rounds = std::floor(tiles / slots), rest = tiles - rounds * slots;
    double us = rounds * (ksteps * t.full + t.fixed);
    if (rest > 0.0) us += ksteps * (rest <= (large ? kMxLargeAlone : 1.0) * cus ? t.alone : t.full) + t.fixed;
    const double memory = mx_touched(R, E) * N * K * (17.0 / 32) * (dual ? 2 : 1) / kMxWeightBytesPerUs;
    return std::max(us, memory) + 0.2 * std::min(us, memory);
}

// Upper bound on the row tiles of E groups with R rows in all.
long long mx_most_row_tiles(int R, int E, int rows) { return R / rows + std::min(E, R); }
// A launch counts its threads in 32 bits: 512 for each tile of up to 32 columns, 256 for each of the others. Many groups and columns
// (256 rows in 256 groups through 2^22 columns) take larger tiles for that; a large kernel's workgroup takes many.
bool mx_launchable(const MxTile& t, int R, int E, int N) {
    const long long tiles = mx_most_row_tiles(R, E, t.rows) * ((N + t.columns - 1) / t.columns);
    return (tiles + 8) * (t.columns <= 32 ? 512 : 256) < 1ll << 32;
}

// The large tiles need two k-steps and as many columns as they have, the wider ones of a few rows whole tiles.
int mx_plain_tile(int R, int E, int N, int K, int cus) {
    int best = kMxFew;
    double least = 1e30;
    for (const MxTile& t : kMxPlainTiles) {
        if (t.id == kMxLarge && (K <= kMxRunElements || N < t.columns)) continue;
        if (t.id == kMxFewWide && N % t.columns != 0) continue;
        if (t.id != kMxLarge && !mx_launchable(t, R, E, N)) continue;
        const double p = mx_price(t, t.id == kMxLarge, false, R, E, N, K, cus);
        if (p < least) { least = p; best = t.id; }
    }
    return best;
}
int mx_gateup_tile(int R, int E, int f, int d, int cus) {
    int best = kMxGate32;
    double least = 1e30;
    for (const MxTile& t : kMxGateUpTiles) {
        if (t.id == kMxGateLarge && (d <= kMxRunElements || f < t.columns)) continue;
        const double p = mx_price(t, t.id == kMxGateLarge, true, R, E, f, d, cus);
        if (p < least) { least = p; best = t.id; }
    }
    return best;
}

}  // namespace
}  // namespace moe
