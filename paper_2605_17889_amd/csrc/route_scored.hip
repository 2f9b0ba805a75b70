// Router of layers with many experts: selection by scores, with a correction for balance and limits on groups.
//
//   s[e] = 1 / (1 + exp(-l[e]))  or  exp(l[e] - max l) / sum exp(l - max l),      c[e] = s[e] + correction[e]
//   value of a group = its largest c, or the sum of its two largest;  the top_groups best groups are kept
//   idx = the k largest c of the kept groups;  w = s[idx] (/ sum of them) * scale
//
// A token belongs to LPT lanes of a wavefront (16, or 64 where there are few tokens), and inside them every group of experts
// to L lanes of its own, so that a group's best two are found by moves among those lanes and a group is kept or dropped by its
// own lanes. Selection is k rounds of a maximum over the token's lanes, on integers of the scores' order (route_select.h).
// The weights are formed from the selected experts' logits once more: a slot's lane reads its own.
#include <algorithm>

#include "route_select.h"

namespace moe {
namespace {

struct ScoredArgs {
    const float* logits;             // [T, E]
    const float* correction;         // [E] or null
    int T, E, k;
    int groups, size;                // groups of `size` experts
    int lane_shift;                  // log2 of the lanes of a group
    int top_groups;
    bool two_best, sigmoid, renormalise;
    float scale;
    int32_t* idx;                    // [T, k]
    float* weight;                   // [T, k]
};

// Over the LPT lanes of a token, in all of them: butterflies by row moves (distances inside 16 lanes) and shuffles.
template <int LPT, class Op>
__device__ __forceinline__ uint32_t over_token(uint32_t v, Op&& op) {
    v = over_16_lanes(v, op);
    if constexpr (LPT == 64) {
        v = op(v, static_cast<uint32_t>(__shfl_xor(static_cast<int>(v), 16)));
        v = op(v, static_cast<uint32_t>(__shfl_xor(static_cast<int>(v), 32)));
    }
    return v;
}
template <int LPT, class T>
__device__ __forceinline__ T sum_over_token(T v) {
#pragma unroll
    for (int s = LPT / 2; s > 0; s >>= 1) v += __shfl_xor(v, s);
    return v;
}

__device__ __forceinline__ float sigmoid(float l) { return 1.f / (1.f + expf(-l)); }
// exp(l - top), 1 for every logit that is the largest, also where that is infinite
__device__ __forceinline__ float exp_below(float l, float top) { return l == top ? 1.f : expf(l - top); }
__device__ __forceinline__ float number(float l) { return l != l ? -INFINITY : l; }      // a NaN counts as -infinity

template <int LPT, int EW>
__global__ __launch_bounds__(256) void route_scored_kernel(ScoredArgs a) {
    constexpr int PER = kWave / LPT, SLOTS = kWave / LPT;      // tokens of a wavefront; slots of a lane (k <= 64)
    const int lane = threadIdx.x & (LPT - 1), base = threadIdx.x & (kWave - 1) & ~(LPT - 1);
    const int t_of = (blockIdx.x * 4 + threadIdx.x / kWave) * PER + (threadIdx.x & (kWave - 1)) / LPT;
    const int t = min(t_of, a.T - 1);                          // all lanes stay for the moves between them
    const float* row = a.logits + static_cast<size_t>(t) * a.E;
    const int L = 1 << a.lane_shift, g = lane >> a.lane_shift, j = lane & (L - 1);

    float c[EW];
    bool has[EW];
#pragma unroll
    for (int i = 0; i < EW; ++i) {
        const int at = i * L + j;
        has[i] = g < a.groups && at < a.size;
        c[i] = has[i] ? number(row[g * a.size + at]) : -INFINITY;
    }
    float top = 0.f, total = 1.f;
    if (!a.sigmoid) {
        uint32_t key = 0;
#pragma unroll
        for (int i = 0; i < EW; ++i) key = max(key, logit_key(c[i]));
        top = key_logit(over_token<LPT>(key, [](uint32_t x, uint32_t y) { return max(x, y); }));
        // In multiples of 2^-44, to which a double near 256 rounds: the sum of up to 256 of them, each at most 1, is exact,
        // so its one rounding to fp32 is the same however the experts lie on the lanes.
        double sum = 0.0;
#pragma unroll
        for (int i = 0; i < EW; ++i) {
            c[i] = exp_below(c[i], top);
            sum += has[i] ? (static_cast<double>(c[i]) + 256.0) - 256.0 : 0.0;
        }
        total = static_cast<float>(sum_over_token<LPT>(sum));
    }
    uint32_t key[EW];
#pragma unroll
    for (int i = 0; i < EW; ++i) {
        float s = a.sigmoid ? sigmoid(c[i]) : c[i] / total;
        if (a.correction != nullptr && has[i]) s += a.correction[g * a.size + i * L + j];
        key[i] = has[i] ? logit_key(s) : 0u;
    }

    if (a.top_groups < a.groups) {
        uint32_t first = 0, second = 0;                        // the group's two largest
#pragma unroll
        for (int i = 0; i < EW; ++i) {
            second = max(second, min(first, key[i]));
            first = max(first, key[i]);
        }
        for (int s = 1; s < L; s <<= 1) {
            const uint32_t f = static_cast<uint32_t>(__shfl_xor(static_cast<int>(first), s));
            const uint32_t h = static_cast<uint32_t>(__shfl_xor(static_cast<int>(second), s));
            second = max(min(first, f), max(second, h));
            first = max(first, f);
        }
        uint32_t value = first;
        if (a.two_best && a.size > 1) value = logit_key(key_logit(first) + key_logit(second));
        int better = 0;                                        // groups ahead of this one
        for (int o = 0; o < a.groups; ++o) {
            const uint32_t v = static_cast<uint32_t>(__shfl(static_cast<int>(value), base + (o << a.lane_shift)));
            better += v > value || (v == value && o < g) ? 1 : 0;
        }
#pragma unroll
        for (int i = 0; i < EW; ++i) key[i] = better < a.top_groups ? key[i] : 0u;
    }

    int slot_of[SLOTS] = {};                                   // lane l keeps slots l, l + LPT, ...
    for (int s = 0; s < a.k; ++s) {
        uint32_t best = key[0];
#pragma unroll
        for (int i = 1; i < EW; ++i) best = max(best, key[i]);
        best = over_token<LPT>(best, [](uint32_t x, uint32_t y) { return max(x, y); });
        uint32_t e = 0xffffffffu;                              // the lowest index that has it
#pragma unroll
        for (int i = 0; i < EW; ++i)
            e = min(e, key[i] == best ? static_cast<uint32_t>(g * a.size + i * L + j) : 0xffffffffu);
        const uint32_t mine = e;
        e = over_token<LPT>(e, [](uint32_t x, uint32_t y) { return min(x, y); });
#pragma unroll
        for (int i = 0; i < EW; ++i)
            key[i] = mine == e && e == static_cast<uint32_t>(g * a.size + i * L + j) ? 0u : key[i];
#pragma unroll
        for (int q = 0; q < SLOTS; ++q) slot_of[q] = s == q * LPT + lane ? static_cast<int>(e) : slot_of[q];
    }

    float w[SLOTS];
#pragma unroll
    for (int q = 0; q < SLOTS; ++q) {
        w[q] = 0.f;
        if (q * LPT + lane < a.k) {
            const float l = number(row[slot_of[q]]);
            w[q] = a.sigmoid ? sigmoid(l) : exp_below(l, top) / total;
        }
    }
    if (a.renormalise) {                                       // slots 32 apart first, then 16, 8, 4, 2, 1
        float sum = w[0];
        if constexpr (SLOTS == 4) sum = (w[0] + w[2]) + (w[1] + w[3]);
        sum = sum_over_token<LPT>(sum);
#pragma unroll
        for (int q = 0; q < SLOTS; ++q) w[q] = sum > 0.f ? w[q] / sum : 0.f;
    }
    if (t_of >= a.T) return;
#pragma unroll
    for (int q = 0; q < SLOTS; ++q) {
        const int s = q * LPT + lane;
        if (s < a.k) {
            a.idx[static_cast<size_t>(t) * a.k + s] = slot_of[q];
            a.weight[static_cast<size_t>(t) * a.k + s] = w[q] * a.scale;
        }
    }
}

template <int LPT, int EW>
int launch(const ScoredArgs& a, hipStream_t s) {
    constexpr int PER = 4 * kWave / LPT;
    hipLaunchKernelGGL((route_scored_kernel<LPT, EW>), dim3(static_cast<unsigned>((a.T + PER - 1) / PER)), dim3(256), 0, s, a);
    return hipGetLastError() == hipSuccess ? MOE_OK : MOE_ERR_HIP;
}

// Lanes of a group where a token has `lpt` of them, or 0 if there are more groups than lanes.
int group_lanes(int groups, int lpt) {
    int L = lpt;
    while (L > 0 && lpt / L < groups) L >>= 1;
    return L;
}

}  // namespace

int launch_route_scored(const float* logits, const float* correction, const moe_scoring& sc, int T, int E, int k,
                        int32_t* topk_idx, float* topk_w, hipStream_t s) {
    if (T == 0) return MOE_OK;
    ScoredArgs a{logits, correction, T, E, k, sc.groups, E / sc.groups, 0, sc.top_groups, sc.group_best == 2,
                 sc.score == MOE_SCORE_SIGMOID, sc.renormalise != 0, sc.scale, topk_idx, topk_w};
    const int lpt = T <= 2048 || group_lanes(a.groups, 16) == 0 ? 64 : 16;
    const int L = group_lanes(a.groups, lpt);
    while ((2 << a.lane_shift) <= L) ++a.lane_shift;
    const int held = (a.size + L - 1) / L;           // of a lane
    if (lpt == 64) return held <= 1 ? launch<64, 1>(a, s) : held <= 4 ? launch<64, 4>(a, s) : launch<64, 8>(a, s);
    return held <= 4 ? launch<16, 4>(a, s) : held <= 8 ? launch<16, 8>(a, s) : held <= 16 ? launch<16, 16>(a, s)
                                                                                        : launch<16, 32>(a, s);
}

}  // namespace moe
