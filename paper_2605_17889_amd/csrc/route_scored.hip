// Router of layers with many experts: selection by scores, with a correction for balance and limits on groups.
//
//   s[e] = 1 / (1 + exp(-l[e]))  or  exp(l[e] - max l) / sum exp(l - max l),      c[e] = s[e] + correction[e]
//   value of a group = its largest c, or the sum of its two largest;  the top_groups best groups are kept
//   idx = the k largest c of the kept groups;  w = s[idx] (/ sum of them) * scale
//
// A token belongs to LPT lanes of a wavefront (16, or 64 where there are few tokens), and inside them every group of experts
// to L lanes of its own, so that a group's best two are found by moves among those lanes and a group is kept or dropped by its
// own lanes. Selection is k rounds of a maximum over the token's lanes, on integers of the scores' order (route_select.h).
// The weights are formed from the selected experts' logits once more: a slot's lane reads its own. No result depends on the
// number of lanes. Bound by the chain of the rounds (0.2 us each for one token) and, with many tokens, by their instructions:
// 8192 tokens of 256 experts read 8.4 MB, 1.3 us of the 8.9.
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

// f(a, b) of a value and the one S lanes away for S = 1, 2, 4 .. 32, for symmetric f and values that the lanes of every S share
// already (the partner at 4 and 8 is then any lane of the other half: the mirrored one).
template <int S, class F>
__device__ __forceinline__ auto with_partner(uint32_t v, F&& f) {
    constexpr int CTRL = S == 1 ? 0xb1 : S == 2 ? 0x4e : S == 4 ? 0x141 : 0x140;      // quad_perm, row_half_mirror, row_mirror
    if constexpr (S < 16) {
        return f(v, static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(v), CTRL, 0xf, 0xf, false)));
    } else if constexpr (S == 16) {
        const auto p = __builtin_amdgcn_permlane16_swap(v, v, false, false);
        return f(p[0], p[1]);
    } else {
        const auto p = __builtin_amdgcn_permlane32_swap(v, v, false, false);
        return f(p[0], p[1]);
    }
}
struct Pair { uint32_t lo, hi; };
template <int S>
__device__ __forceinline__ Pair partners(uint32_t v) {
    return with_partner<S>(v, [](uint32_t x, uint32_t y) { return Pair{x, y}; });
}
template <int LPT, int S = 1>
__device__ __forceinline__ uint32_t max_over_token(uint32_t v) {
    if constexpr (S < LPT) return max_over_token<LPT, 2 * S>(with_partner<S>(v, [](uint32_t x, uint32_t y) { return max(x, y); }));
    else return v;
}
// Of numbers, without the quieting of signalling NaNs that a language's maximum has to do.
__device__ __forceinline__ double larger(double x, double y) {
    double r;
    asm("v_max_f64 %0, %1, %2" : "=v"(r) : "v"(x), "v"(y));
    return r;
}
template <int LPT, int S = 1>
__device__ __forceinline__ double max_over_token(double v) {
    if constexpr (S < LPT) {
        const Pair lo = partners<S>(__double2loint(v)), hi = partners<S>(__double2hiint(v));
        return max_over_token<LPT, 2 * S>(larger(__hiloint2double(hi.lo, lo.lo), __hiloint2double(hi.hi, lo.hi)));
    } else {
        return v;
    }
}
// The sum in the order of the distances 1, 2, 4, ..
template <int LPT, int S = 1>
__device__ __forceinline__ float sum_over_token(float v) {
    if constexpr (S < LPT) {
        const Pair p = partners<S>(__float_as_uint(v));
        return sum_over_token<LPT, 2 * S>(__uint_as_float(p.lo) + __uint_as_float(p.hi));
    } else {
        return v;
    }
}
template <int LPT, int S = 1>
__device__ __forceinline__ double sum_over_token(double v) {
    if constexpr (S < LPT) {
        const Pair lo = partners<S>(__double2loint(v)), hi = partners<S>(__double2hiint(v));
        return sum_over_token<LPT, 2 * S>(__hiloint2double(hi.lo, lo.lo) + __hiloint2double(hi.hi, lo.hi));
    } else {
        return v;
    }
}
// A group's two largest over its L lanes.
template <int LPT, int S = 1>
__device__ __forceinline__ void two_largest(uint32_t& first, uint32_t& second, int L) {
    if constexpr (S < LPT) {
        if (S >= L) return;
        const Pair f = partners<S>(first), g = partners<S>(second);
        second = max(min(f.lo, f.hi), max(g.lo, g.hi));
        first = max(f.lo, f.hi);
        two_largest<LPT, 2 * S>(first, second, L);
    }
}

__device__ __forceinline__ float sigmoid(float l) { return 1.f / (1.f + expf(-l)); }
// exp(l - top), 1 for every logit that is the largest, also where that is infinite
__device__ __forceinline__ float exp_below(float l, float top) { return l == top ? 1.f : expf(l - top); }
__device__ __forceinline__ float number(float l) { return l != l ? -INFINITY : l; }      // a NaN counts as -infinity

// A lane's EW experts of its group: every L-th one, or (QUADS) runs of four, every L-th of those, which it loads 16 bytes at a time.
template <bool QUADS>
__device__ __forceinline__ int in_group(int i, int j, int L) {
    return QUADS ? ((i >> 2) * L + j) * 4 + (i & 3) : i * L + j;
}
template <int EW, bool QUADS>
__device__ __forceinline__ void load_experts(float (&v)[EW], const bool (&has)[EW], const float* from, int j, int L, float none) {
    if constexpr (QUADS) {
#pragma unroll
        for (int i = 0; i < EW; i += 4) {
            float4 q = {none, none, none, none};
            if (has[i]) q = *reinterpret_cast<const float4*>(from + in_group<true>(i, j, L));
            v[i] = q.x;
            v[i + 1] = q.y;
            v[i + 2] = q.z;
            v[i + 3] = q.w;
        }
    } else {
#pragma unroll
        for (int i = 0; i < EW; ++i) v[i] = has[i] ? from[in_group<false>(i, j, L)] : none;
    }
}

constexpr int kThreads = 256;

template <int LPT, int EW, bool QUADS>
__global__ __launch_bounds__(kThreads) void route_scored_kernel(ScoredArgs a) {
    constexpr int PER = kWave / LPT, SLOTS = kWave / LPT;      // tokens of a wavefront; slots of a lane (k <= 64)
    const int lane = threadIdx.x & (LPT - 1);
    const int t_of = (blockIdx.x * 4 + threadIdx.x / kWave) * PER + (threadIdx.x & (kWave - 1)) / LPT;
    if (LPT == kWave && t_of >= a.T) return;                   // a whole wavefront
    const int t = min(t_of, a.T - 1);                          // all lanes stay for the moves between them
    const float* row = a.logits + static_cast<size_t>(t) * a.E;
    const int L = 1 << a.lane_shift, g = lane >> a.lane_shift, j = lane & (L - 1);

    float c[EW], add[EW];
    bool has[EW];
#pragma unroll
    for (int i = 0; i < EW; ++i) has[i] = g < a.groups && in_group<QUADS>(i, j, L) < a.size;
    load_experts<EW, QUADS>(c, has, row + g * a.size, j, L, -INFINITY);
    if (a.correction != nullptr) load_experts<EW, QUADS>(add, has, a.correction + g * a.size, j, L, 0.f);
#pragma unroll
    for (int i = 0; i < EW; ++i) c[i] = number(c[i]);
    float top = 0.f, total = 1.f;
    if (!a.sigmoid) {
        uint32_t key = 0;
#pragma unroll
        for (int i = 0; i < EW; ++i) key = max(key, logit_key(c[i]));
        top = key_logit(max_over_token<LPT>(key));
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
        if (a.correction != nullptr) s += add[i];
        key[i] = has[i] ? logit_key(s) : 0u;
    }

    if (a.top_groups < a.groups) {
        uint32_t first = 0, second = 0;                        // the group's two largest
#pragma unroll
        for (int i = 0; i < EW; ++i) {
            second = max(second, min(first, key[i]));
            first = max(first, key[i]);
        }
        two_largest<LPT>(first, second, L);
        uint32_t value = first;
        if (a.two_best && a.size > 1) value = logit_key(key_logit(first) + key_logit(second));
        const int base = threadIdx.x & (kWave - 1) & ~(LPT - 1);
        int better = 0;                                        // groups ahead of this one
        for (int o = 0; o < a.groups; ++o) {
            const uint32_t v = LPT == kWave ? __builtin_amdgcn_readlane(value, o << a.lane_shift)
                                            : static_cast<uint32_t>(__shfl(static_cast<int>(value), base + (o << a.lane_shift)));
            better += v > value || (v == value && o < g) ? 1 : 0;
        }
#pragma unroll
        for (int i = 0; i < EW; ++i) key[i] = better < a.top_groups ? key[i] : 0u;
    }

    int slot_of[SLOTS] = {};                                   // lane l keeps slots l, l + LPT, ...
    // 16 lanes: c's order and the index (the lower one above) in the fraction of a double, so that a round is a maximum of numbers
    // of which no two are equal, and needs no search for who has it. Maximum, then the lowest index that has it -> so: 8192 tokens
    // of 256 experts, k = 8 9.8 -> 8.9 us, 16384, k = 16 18.2 -> 15.5, 128 experts 6.5 -> 6.0; of 64 and fewer 0 to 3 % slower.
    // Its 8 bits of index are enough for all experts, and different in two low words.
    double both[LPT == kWave ? 1 : EW];
    if constexpr (LPT != kWave) {
#pragma unroll
        for (int i = 0; i < EW; ++i) {
            const uint32_t e = static_cast<uint32_t>(g * a.size + in_group<QUADS>(i, j, L));
            both[i] = __hiloint2double(static_cast<int>(0x3ff00000u | key[i] >> 24), static_cast<int>(key[i] << 8 | ((255u - e) & 255u)));
        }
    }
    for (int s = 0; s < a.k; ++s) {
        if constexpr (LPT == kWave) {
            uint32_t own = key[0];
#pragma unroll
            for (int i = 1; i < EW; ++i) own = max(own, key[i]);
            const uint32_t best = max_over_token<LPT>(own);
            // The lowest index that has it, on the scalar unit: of the first group that has it the first i (with QUADS four of
            // them), of those the first lane.
            uint64_t in[EW], any = 0;
#pragma unroll
            for (int i = 0; i < EW; ++i) any |= in[i] = __ballot(key[i] == best);
            const int found = __builtin_ctzll(any) >> a.lane_shift, first = found << a.lane_shift;
            const uint64_t group = (L == kWave ? ~0ull : ((1ull << L) - 1)) << first;
            constexpr int STEP = QUADS ? 4 : 1;
            int which = 0, from = 0;
#pragma unroll
            for (int i = EW - STEP; i >= 0; i -= STEP) {
                uint64_t of = in[i];
#pragma unroll
                for (int n = 1; n < STEP; ++n) of |= in[i + n];
                of &= group;
                if (of != 0) {
                    from = __builtin_ctzll(of);
                    which = i;
#pragma unroll
                    for (int n = STEP - 1; n >= 0; --n) which = (in[i + n] >> from) & 1 ? i + n : which;
                }
            }
            const int e = found * a.size + in_group<QUADS>(which, from - first, L);
#pragma unroll
            for (int i = 0; i < EW; ++i) key[i] = i == which && lane == from ? 0u : key[i];
            slot_of[0] = s == lane ? e : slot_of[0];
        } else {
            double of[EW];
#pragma unroll
            for (int i = 0; i < EW; ++i) of[i] = both[i];
#pragma unroll
            for (int n = EW; n > 1; n = (n + 1) / 2)
#pragma unroll
                for (int i = 0; i < n / 2; ++i) of[i] = larger(of[i], of[n - 1 - i]);
            const double best = max_over_token<LPT>(of[0]);
#pragma unroll
            for (int i = 0; i < EW; ++i)
                both[i] = __hiloint2double(__double2loint(both[i]) == __double2loint(best) ? 0 : __double2hiint(both[i]), __double2loint(both[i]));
            const int e = 255 - (__double2loint(best) & 255);
#pragma unroll
            for (int q = 0; q < SLOTS; ++q) slot_of[q] = s == q * LPT + lane ? e : slot_of[q];
        }
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
    if (a.renormalise) {                                       // slots 1, 2, 4, 8 apart, then 16, then 32
        float part[4] = {};
#pragma unroll
        for (int q = 0; q < SLOTS; ++q) part[q] = a.k > q * LPT ? sum_over_token<LPT>(w[q]) : 0.f;
        const float sum = (part[0] + part[1]) + (part[2] + part[3]);
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

long long workgroups(int T, int lpt) { return (static_cast<long long>(T) * lpt + kThreads - 1) / kThreads; }

template <int LPT, int EW, bool QUADS>
int launch(const ScoredArgs& a, hipStream_t s) {
    hipLaunchKernelGGL((route_scored_kernel<LPT, EW, QUADS>), dim3(static_cast<unsigned>(workgroups(a.T, LPT))), dim3(kThreads), 0, s, a);
    return hipGetLastError() == hipSuccess ? MOE_OK : MOE_ERR_HIP;
}

// Lanes of a group where a token has `lpt` of them, or 0 if there are more groups than lanes.
int group_lanes(int groups, int lpt) {
    int L = lpt;
    while (L > 0 && lpt / L < groups) L >>= 1;
    return L;
}
// Lanes of a token. us, 16 | 64 lanes: 256 experts in 8 groups, one token 6.7 | 4.2, 2000 7.1 | 5.3, 4000 7.3 | 7.0, 5000 8.7 | 7.9,
// 8192 8.9 | 10.4, 16384 13.3 | 17.7; 128 experts, 4000 tokens 4.9 | 4.9; 64, softmax, 2000 3.8 | 3.6, 4000 3.9 | 4.3, 16384 6.0 | 9.2.
int token_lanes(int T, int groups) { return T <= 4096 || group_lanes(groups, 16) == 0 ? 64 : 16; }

}  // namespace

bool route_scored_fits(int T, int groups) { return workgroups(T, token_lanes(T, groups)) * kThreads <= kMaxThreads; }

int launch_route_scored(const float* logits, const float* correction, const moe_scoring& sc, int T, int E, int k,
                        int32_t* topk_idx, float* topk_w, hipStream_t s) {
    if (T == 0) return MOE_OK;
    if (!route_scored_fits(T, sc.groups)) return MOE_ERR_UNSUPPORTED_SHAPE;
    ScoredArgs a{logits, correction, T, E, k, sc.groups, E / sc.groups, 0, sc.top_groups, sc.group_best == 2,
                 sc.score == MOE_SCORE_SIGMOID, sc.renormalise != 0, sc.scale, topk_idx, topk_w};
    const int lpt = token_lanes(T, a.groups);
    const int L = group_lanes(a.groups, lpt);
    while ((2 << a.lane_shift) <= L) ++a.lane_shift;
    const int held = (a.size + L - 1) / L;           // of a lane, where it takes every L-th expert
    const bool quads = a.size % 4 == 0 && held > 2 && ((reinterpret_cast<uintptr_t>(logits) | reinterpret_cast<uintptr_t>(correction)) & 15) == 0;
    if (quads) {
        const int runs = (a.size / 4 + L - 1) / L;   // of four
        if (lpt == 64) return runs <= 1 ? launch<64, 4, true>(a, s) : launch<64, 8, true>(a, s);
        return runs <= 1   ? launch<16, 4, true>(a, s)
               : runs <= 2 ? launch<16, 8, true>(a, s)
               : runs <= 4 ? launch<16, 16, true>(a, s)
                           : launch<16, 32, true>(a, s);
    }
    if (lpt == 64)
        return held <= 1   ? launch<64, 1, false>(a, s)
               : held <= 2 ? launch<64, 2, false>(a, s)
               : held <= 4 ? launch<64, 4, false>(a, s)
                           : launch<64, 8, false>(a, s);
    return held <= 1   ? launch<16, 1, false>(a, s)
           : held <= 4 ? launch<16, 4, false>(a, s)
           : held <= 8 ? launch<16, 8, false>(a, s)
           : held <= 16 ? launch<16, 16, false>(a, s)
                        : launch<16, 32, false>(a, s);
}

}  // namespace moe
