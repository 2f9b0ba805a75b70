// Internal helpers shared by the HIP translation units of libmoe (not part of the C ABI).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "moe.h"

namespace moe {

constexpr int kWave = 64;        // CDNA wavefront width
constexpr int kMaxExperts = 256; // four experts per lane in the permutation and routing kernels
constexpr int kMaxRowI8 = 65536; // a row in the registers of a workgroup (norm.hip)
constexpr int kMaxSumI8 = 130944; // products of -128 .. 127 whose sum stays below 2^31, a multiple of 128
constexpr int kMaxDimI8 = 1 << 23; // widths of outputs, for 32-bit offsets inside a tile
constexpr int kMaxDimMx4 = 1 << 22; // lengths of rows in 4 bits and of fp32 outputs: 128 rows of a tile stay below 2^32 bytes
constexpr int kMaxGroups = 64;   // of experts: a lane each
constexpr int kXcds = 8;         // workgroups are dealt round-robin to the 8 XCDs (own L2 each)
constexpr long long kMaxThreads = (1ll << 32) - 1; // of a launch, which counts them in 32 bits

__device__ __forceinline__ float bf16_to_f32(uint16_t b) {
    return __uint_as_float(static_cast<uint32_t>(b) << 16);
}

// fp32 -> bf16, round to nearest even; NaN stays a quiet NaN.
__device__ __forceinline__ uint16_t f32_to_bf16(float f) {
    uint32_t u = __float_as_uint(f);
    if ((u & 0x7fffffffu) > 0x7f800000u) return static_cast<uint16_t>((u >> 16) | 0x0040u);
    u += 0x7fffu + ((u >> 16) & 1u);
    return static_cast<uint16_t>(u >> 16);
}

#define MOE_HIP_TRY(expr)                         \
    do {                                          \
        hipError_t e__ = (expr);                  \
        if (e__ != hipSuccess) return MOE_ERR_HIP; \
    } while (0)

// Compute units of a device (0..63), asked once. Large tiles and the router's workgroups run in rounds of
// that many.
int compute_units(int device);

// Launch wrappers (defined in the .hip files). Each returns a moe_status and only enqueues.
int launch_route(const moe_bf16* x, const float* w_router, const float* bias, int T, int d, int E,
                 int k, int32_t* topk_idx, float* topk_w, float* logits_out,
                 float* logits_scratch, hipStream_t s);
int route_launches(int E);       // kernels that launch_route enqueues for a call of at least one token
int launch_route_logits(const moe_bf16* x, const float* w_router, const float* bias, int T, int d, int E,
                        float* logits, hipStream_t s);
int launch_route_from_logits(const float* logits, int T, int E, int k, int32_t* topk_idx,
                             float* topk_w, hipStream_t s);
size_t permute_scratch_ints(int R_max, int E);
int permute_launches(int R);     // kernels that launch_permute enqueues for R ids
int launch_permute(const int32_t* topk_idx, int R, int E, int32_t* counts, int32_t* offsets,
                   int32_t* perm, int32_t* inv_perm, int32_t* scratch, hipStream_t s);
// Selection, gates and permutation of a few tokens (E > 16) in one workgroup, and up to how many tokens
// that is shorter than the two launches.
bool select_permute_fits(int T, int E, int k);
int launch_select_permute(const float* logits, int T, int E, int k, int32_t* topk_idx, float* topk_w,
                          int32_t* counts, int32_t* offsets, int32_t* perm, int32_t* inv_perm, hipStream_t s);
// The same for larger batches in two launches: selection with the histograms of its ids, then the scatter.
bool select_hist_fits(int T, int E, int k);
int launch_select_hist_permute(const float* logits, int T, int E, int k, int32_t* topk_idx, float* topk_w,
                               int32_t* counts, int32_t* offsets, int32_t* perm, int32_t* inv_perm,
                               int32_t* seg_tables, hipStream_t s);
int launch_gather(const moe_bf16* x, const int32_t* perm, const int32_t* offsets, int R, int d,
                  int k, int E, moe_bf16* x_perm, hipStream_t s);
// Counters from which persistent workgroups draw their tiles, kTileCounterBytes that are zero between launches.
// A context takes a set of its device's 64 and gives it back; set -1: there is none left (the caller then zeroes
// memory of its own). The calling thread's current device must be `device`.
constexpr size_t kTileCounterBytes = kXcds * 128;
int32_t* take_tile_counters(int device, int* set);
void give_tile_counters(int device, int set);
// Sums of split reductions, in memory that a context allocates for its first call that splits one.
constexpr int kPartSums = 6 << 18;        // 6 MB of them
constexpr int kSplitTiles = 128;
constexpr size_t kSplitSumBytes = kSplitTiles * (256 + 1) * sizeof(int32_t);   // of 256 sums and a counter each
// Where and how a context launches its expert GEMMs: its device, its tile counters and the tuning knobs of
// moe_set_gemm_config (all settings give identical bits).
struct GemmEnv {
    int device = 0;
    int forced_config = -1;           // -1: automatic; 0..4: force a tile configuration
    int stream_mode = -1;             // -1: automatic; 0: weights never non-temporal; 1: always
    bool materialise_gather = false;  // layer calls write x_perm instead of fusing the gather
    bool split_last_round = true;     // large tiles: halve the tiles of a last round under half full
    int large_tile_waves = 0;         // 0: automatic; 4 / 8: wavefronts of the 256 x 256 tile
    int32_t* tile_counters = nullptr; // kTileCounterBytes, zero between launches
    int32_t* split_sums = nullptr;    // kSplitSumBytes, zero between launches: 8-bit products of few rows through one matrix
    int32_t* part_sums = nullptr;     // kPartSums: of more rows without offsets, parts that a second launch joins
    bool whole_reductions = false;    // split none (there is no such memory, and none can be had)
};
int launch_gateup(const GemmEnv& env, const moe_bf16* a, const int32_t* row_index, int index_div,
                  const int32_t* offsets, int R, int R_hint, int d, int f, int E,
                  const moe_bf16* W1, const moe_bf16* W3, moe_bf16* H, hipStream_t s);
// Gate/up of a few tokens without a permutation launch: it derives the groups from the selected experts, for more than
// 16 experts from the logits, and writes the routing tables. gateup_routes: whether it takes such a call.
bool gateup_routes(const GemmEnv& env, int T, int d, int f, int E, int k);
int launch_gateup_routed(const GemmEnv& env, const moe_bf16* x, const float* logits, int32_t* topk_idx, float* topk_w,
                         int32_t* counts, int32_t* offsets, int32_t* perm, int32_t* inv_perm, int T, int d, int f,
                         int E, int k, const moe_bf16* W1, const moe_bf16* W3, moe_bf16* H, hipStream_t s);
int launch_down(const GemmEnv& env, const moe_bf16* H, const int32_t* offsets, int R, int R_hint,
                int d, int f, int E, const moe_bf16* W2, void* y_perm, bool y_f32, hipStream_t s);
bool combine_fits(int T);        // whether a launch holds the tokens
int launch_combine(const void* y_perm, bool y_f32, const int32_t* inv_perm, const float* topk_w, int T,
                   int d, int k, moe_bf16* y, hipStream_t s);
// Rows in 8 bits, of up to kMaxRowI8 elements: the norm in front of an 8-bit product, and bf16 rows as they are.
int launch_rmsnorm_i8(const moe_bf16* x, long long x_stride, const void* residual, bool residual_f32,
                      const moe_bf16* weight, float eps, int T, int d, void* residual_out, moe_bf16* y, moe_i8* q,
                      float* q_scale, hipStream_t s);
int launch_quantize_i8(const moe_bf16* x, long long x_stride, int T, int d, moe_i8* q, float* q_scale, hipStream_t s);
// Token rows in 8 bits with their scales, grouped by expert (d a multiple of 16, every row of perm filled).
int launch_gather_i8(const moe_i8* q, const float* scale, const int32_t* perm, int R, int d, int k, moe_i8* q_perm,
                     float* scale_perm, hipStream_t s);
// Products of 8-bit integers with scales (expert_gemm_i8.hip). R rows in E groups; without offsets they are one group.
int launch_gateup_i8(const GemmEnv& env, const moe_i8* x, const float* x_scale, const int32_t* offsets, int R, int d, int f,
                     int E, const moe_i8* W1, const float* w1_scale, const moe_i8* W3, const float* w3_scale, moe_bf16* H,
                     hipStream_t s);
// The down projection straight from H in bf16, whose rows it brings to 8 bits by itself; whether it takes such a call.
bool down_converts(const GemmEnv& env, int R, int d, int f, int E);
int launch_down_converting_i8(const GemmEnv& env, const moe_bf16* H, const int32_t* offsets, int R, int d, int f, int E,
                              const moe_i8* W2, const float* w2_scale, void* y, bool y_f32, hipStream_t s);
// kNeedsSums: nothing was enqueued; the reduction would be split, and env has no memory for its sums.
constexpr int kNeedsSums = 1;
int launch_product_i8(const GemmEnv& env, const moe_i8* x, const float* x_scale, const int32_t* offsets, int R, int N, int K,
                      int E, const moe_i8* W, const float* w_scale, void* out, bool out_f32, hipStream_t s);
// Scores, groups and weights from logits; sc is checked. route_scored_fits: whether a launch holds the tokens.
bool route_scored_fits(int T, int groups);
int launch_route_scored(const float* logits, const float* correction, const moe_scoring& sc, int T, int E, int k,
                        int32_t* topk_idx, float* topk_w, hipStream_t s);
// Rows in microscaled 4-bit floating point (mx4.h), d a multiple of 32. rows_mx4_fit: whether a launch holds them.
bool rows_mx4_fit(int T, int d);
int launch_quantize_mx4(const moe_bf16* x, long long x_stride, int T, int d, moe_mx4* q, moe_e8m0* scale, hipStream_t s);
// Token rows to their k places in the rows grouped by expert.
int launch_quantize_grouped_mx4(const moe_bf16* x, const int32_t* inv_perm, int T, int d, int k, moe_mx4* q, moe_e8m0* scale,
                                hipStream_t s);
int launch_dequantize_mx4(const moe_mx4* q, const moe_e8m0* scale, int T, int d, moe_bf16* y, hipStream_t s);
// Products of such rows (expert_gemm_mx4.hip). Without offsets they are one group. H's scales have a pitch of R rows.
int launch_gateup_mx4(const GemmEnv& env, const moe_mx4* x, const moe_e8m0* x_scale, const int32_t* offsets, int R, int d, int f,
                      int E, const moe_mx4* W1, const moe_e8m0* w1_scale, const moe_mx4* W3, const moe_e8m0* w3_scale,
                      moe_mx4* H, moe_e8m0* h_scale, hipStream_t s);
int launch_product_mx4(const GemmEnv& env, const moe_mx4* x, const moe_e8m0* x_scale, const int32_t* offsets, int R, int N,
                       int K, int E, const moe_mx4* W, const moe_e8m0* w_scale, void* out, bool out_f32, hipStream_t s);

}  // namespace moe
