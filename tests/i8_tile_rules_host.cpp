// Host build of the rules by which 8-bit products pick their tiles: prints what they say of sizes given on the command line.
// Compiled and run by test_i8_tile_rules.py.
#include <cstdio>
#include <cstdlib>
#include <cstring>

#include "i8_tile_rules.h"

int moe::compute_units(int) { return 256; }

using Gateup = moe::gemm::OperandsI8<moe::gemm::Config<64, 128, 64, 2, 2, 3, true>>;
using Down = moe::gemm::OperandsI8<moe::gemm::Config<64, 64, 64, 2, 2, 5, false>>;
using Mid = moe::gemm::OperandsI8<moe::gemm::Config<128, 128, 64, 2, 2, 4, false>>;
using Few = moe::gemm::OperandsI8<moe::gemm::Config<16, 32, 64, 1, 2, 6, false>>;
using Bf16 = moe::gemm::Config<64, 128, 64, 2, 2, 3, true>;

// gateup|product config R E N elements [n-tiles of the 128-row tile]; turned 0 N elements; one R E elements
int main(int argc, char** argv) {
    int v[8] = {};
    for (int i = 2; i < argc && i < 10; ++i) v[i - 2] = std::atoi(argv[i]);
    if (argc == 7 && !std::strcmp(argv[1], "gateup"))
        std::printf("%d\n", moe::i8_gateup_config(v[0], v[1], v[2], v[3], v[4] / 2, 256));
    else if (argc == 8 && !std::strcmp(argv[1], "product"))
        std::printf("%d\n", moe::i8_product_config(v[0], v[1], v[2], v[3], v[4] / 2, v[5], 256));
    else if (argc == 5 && !std::strcmp(argv[1], "turned"))
        std::printf("%d%d%d%d%d\n", moe::turned_ksteps<Gateup>(v[1], v[2] / 2), moe::turned_ksteps<Down>(v[1], v[2] / 2),
                    moe::turned_ksteps<Mid>(v[1], v[2] / 2), moe::turned_ksteps<Few>(v[1], v[2] / 2), moe::turned_ksteps<Bf16>(v[1], v[2] / 2));
    else if (argc == 5 && !std::strcmp(argv[1], "one"))
        std::printf("%d\n", moe::turned_ksteps_of_one<Down>(v[0], v[1], v[2] / 2));
    else
        return 2;
    return 0;
}
