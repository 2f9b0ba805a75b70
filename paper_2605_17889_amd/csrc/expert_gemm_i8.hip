// Products of 8-bit integers with a scale for each row and each output channel, dense or grouped by expert:
//
//   gate/up : H[p, j] = bf16( SiLU(g) * u ),  g = s_p s1_e[j] sum_i q_p[i] W1_e[j,i],  u likewise with W3
//   product : C[p, n] = s_p s_e[n] sum_k q_p[k] W_e[n,k],  bf16 or fp32
//
// The kernels and the rules by which tiles are chosen are those of the bf16 products, with rows of half as many 16-bit
// units (expert_gemm_kernel.h). The sums are whole numbers: every tile and order of them gives the same bits.
#include "expert_gemm_launch.h"

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
// Weights that a single row tile reads are loaded as non-temporal.
template <class Cached, class Streamed>
int grouped(const Call& c) {
    return single_m_tile(c.env, c.R, c.E, Cached::BM) ? grouped<Streamed>(c) : grouped<Cached>(c);
}
template <class Cfg>
int large(const Call& c) {
    uint16_t* out = static_cast<uint16_t*>(c.C);
    if (c.K % 128 == 0)
        return launch_1w<Cfg, false>(c.env, c.A, c.B0, c.B1, out, c.offsets, nullptr, 1, c.R, c.E, c.N, c.K, c.s, c.scales);
    return launch_1w<Cfg, true>(c.env, c.A, c.B0, c.B1, out, c.offsets, nullptr, 1, c.R, c.E, c.N, c.K, c.s, c.scales);
}
bool large_takes(int N, int K) { return gemm::offsets_fit_1w(N, K) && K >= 256; }

int gateup(const Call& c) {
    int config = pick_config(c.env, c.R, c.E, gateup_tiles(c.E, c.K, c.N));
    if (config == 0 && !large_takes(c.N, c.K)) config = 1;
    switch (config) {
        case 0: return large<GateUp1W>(c);
        case 1: return grouped<GateUpMid, GateUpMidS>(c);
        case 4: return grouped<GateUpMid96, GateUpMid96S>(c);
        case 3: {
            if (!single_m_tile(c.env, c.R, c.E, 32)) return grouped<GateUpTiny>(c);
            const double nt = touched_experts(c.R, c.E) * (c.N / 64);
            const int cus = compute_units(c.env.device);
            if (narrow_gateup_tiles(c.R, c.E, c.N, cus) || narrow_short_gateup_tiles(c.R, c.E, c.K, c.N, cus))
                return one_tile_per_cu(c.R, c.E, c.N, cus) ? grouped<GateUpFewDeepS>(c) : grouped<GateUpFewS>(c);
            return last_round_use(nt, 2.0 * cus) < 0.93 * last_round_use(nt, cus) ? grouped<GateUpTinyDeepS>(c)
                                                                                 : grouped<GateUpTinyS>(c);
        }
        default: return grouped<GateUpSmall, GateUpSmallS>(c);
    }
}

template <bool F32>
int product(const Call& c) {
    const int d = c.N;
    const bool wide_mid = static_cast<long long>(c.E) * (d / 256) >= 160;
    const int cus = compute_units(c.env.device);
    int config = pick_config(c.env, c.R, c.E, NTiles{(d + 255) / 256, wide_mid ? (d + 255) / 256 : (d + 127) / 128, (d + 63) / 64,
                                                     wide_mid ? 0.82 : 0.6, 0.27, 0.38, 2e-6 * c.E * d * c.K, c.K / 64});
    if (config == 0 && (!large_takes(d, c.K) || d < 256)) config = 1;
    if ((config == 1 || config == 4) && d < 128) config = 2;
    if (config == 2 && d < 64) config = 3;
    switch (config) {
        case 0: return large<Out<F32, Plain1W>>(c);
        case 1:
            if (wide_mid) return grouped<Out<F32, PlainMidWide>, Out<F32, PlainMidWideS>>(c);
            return grouped<Out<F32, PlainMid>, Out<F32, PlainMidS>>(c);
        case 4:
            if (wide_mid) return grouped<Out<F32, PlainMid96Wide>, Out<F32, PlainMid96WideS>>(c);
            return grouped<Out<F32, PlainMid96>, Out<F32, PlainMid96S>>(c);
        case 3:
            if (touched_experts(c.R, c.E) * (d / 64) < cus) {
                if (single_m_tile(c.env, c.R, c.E, 16)) return grouped<Out<F32, PlainFewS>>(c);
                if (d < 64 || row_tiles(c.R, c.E, 16) * (d / 32) <= cus) return grouped<Out<F32, PlainFew>>(c);
            }
            return grouped<Out<F32, PlainTiny>, Out<F32, PlainTinyS>>(c);
        default:
            if (row_tiles(c.R, c.E, 64) * (d / 64) <= 0.5 * cus) return grouped<Out<F32, PlainTiny>>(c);
            if (touched_experts(c.R, c.E) * (d / 128) >= 3.5 * cus)
                return grouped<Out<F32, PlainSmallWide>, Out<F32, PlainSmallWideS>>(c);
            return grouped<Out<F32, PlainSmall>, Out<F32, PlainSmallS>>(c);
    }
}

}  // namespace

int launch_gateup_i8(const GemmEnv& env, const moe_i8* x, const float* x_scale, const int32_t* offsets, int R, int d, int f,
                     int E, const moe_i8* W1, const float* w1_scale, const moe_i8* W3, const float* w3_scale, moe_bf16* H,
                     hipStream_t s) {
    if (R == 0) return MOE_OK;
    return gateup(Call{env, units(x), units(W1), units(W3), H, offsets, {x_scale, w1_scale, w3_scale, R}, R, E, f, d / 2, s});
}

int launch_product_i8(const GemmEnv& env, const moe_i8* x, const float* x_scale, const int32_t* offsets, int R, int N, int K,
                      int E, const moe_i8* W, const float* w_scale, void* out, bool out_f32, hipStream_t s) {
    if (R == 0) return MOE_OK;
    const Call c{env, units(x), units(W), nullptr, out, offsets, {x_scale, w_scale, nullptr, R}, R, E, N, K / 2, s};
    return out_f32 ? product<true>(c) : product<false>(c);
}

}  // namespace moe
