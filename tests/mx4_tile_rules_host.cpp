// Host build of the rules by which 4-bit products pick their tiles: prints the tile of every product given on the command line.
// Compiled and run by test_mx4_tile_rules.py.
#include <cstdio>
#include <cstdlib>
#include <cstring>

#include "mx4_tile_rules.h"

// (plain|gateup) R E N K ...
int main(int argc, char** argv) {
    for (int i = 1; i + 4 < argc; i += 5) {
        const int R = std::atoi(argv[i + 1]), E = std::atoi(argv[i + 2]), N = std::atoi(argv[i + 3]), K = std::atoi(argv[i + 4]);
        std::printf("%d\n", std::strcmp(argv[i], "gateup") ? moe::mx_plain_tile(R, E, N, K, 256) : moe::mx_gateup_tile(R, E, N, K, 256));
    }
    return 0;
}
