// Products of rows and weights in microscaled 4-bit floating point (mx4.h), dense or grouped by expert (device code; included
// by expert_gemm_mx4.hip):
//
//   C[p, n] = sum_b 2^(sx[p,b] - 127) 2^(sw[n,b] - 127) sum_{k in block b} x[p,k] w[n,k]      for the rows p of expert e
//
// on v_mfma_scale_f32_16x16x128_f8f6f4: a lane holds the 32 elements of one block of one row (16 bytes) and the block's scale,
// the instruction multiplies 16 rows with 16 columns over four blocks and adds to fp32. Bytes, cycles and layout are those of the
// 8-bit instruction (16 bytes of a row per lane, 16 cycles), so that the tiles are those of expert_gemm_kernel.h, whose tile
// map, LDS swizzle and fragments are used here; what is added is the scales, a sixteenth of the operands' bytes.
//
// A k-step is 256 elements: 128 bytes of a row, eight blocks, and 8 bytes of scales per row in one piece per tile. Operands come
// through buffer resources that end behind the tile's last row: rows that are not there read as zeros without memory traffic,
// and no address needs a comparison. A reduction whose length is no multiple of 256 reads on into the next row; the scales
// of the blocks that are not there are 0 (2^-127) in both operands, so their products, below 2^-248, add nothing.
#pragma once
#include "expert_gemm_kernel.h"
#include "mx4.h"

namespace moe {
namespace mx4 {

using gemm::f32x4;
using gemm::i32x4;
using gemm::TileCoord;
typedef int i32x8 __attribute__((ext_vector_type(8)));

// acc (16x16, rows = weight rows, columns = activation rows) += blocks of k-substep KK of a k-step; the scales of both of a
// lane's blocks lie in the low 16 bits.
template <int KK>
__device__ __forceinline__ f32x4 mma(const i32x4& w, const i32x4& x, const f32x4& acc, int ws, int xs) {
    const i32x8 w8 = {w[0], w[1], w[2], w[3], 0, 0, 0, 0}, x8 = {x[0], x[1], x[2], x[3], 0, 0, 0, 0};
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(w8, x8, acc, 4, 4, KK, ws, KK, xs);
}

// Operands of a product. A [R, K / 2] with scales [runs, R, 8]; matrices [E, N, K / 2] with scales [E, runs, N, 8].
struct Operands {
    const uint8_t *a, *a_scale;
    const uint8_t *b[2], *b_scale[2];
    const int32_t* offsets;          // null: one group of R rows
    int R, E, N, K;
};
// Outputs: bf16 or fp32 rows of N, or (gate/up) rows of N in 4 bits with scales [runs of N, R, 8].
struct Outputs {
    void* c;
    uint8_t* scale;
};

// The same in all lanes: into scalar registers, where a resource has to be.
__device__ __forceinline__ __amdgpu_buffer_rsrc_t resource(const void* base, uint32_t bytes) {
    const uint64_t at = reinterpret_cast<uint64_t>(base);
    const uint64_t uniform = static_cast<uint32_t>(__builtin_amdgcn_readfirstlane(static_cast<uint32_t>(at))) |
                             static_cast<uint64_t>(__builtin_amdgcn_readfirstlane(static_cast<uint32_t>(at >> 32))) << 32;
    return __builtin_amdgcn_make_buffer_rsrc(reinterpret_cast<void*>(uniform), 0,
                                             static_cast<int>(__builtin_amdgcn_readfirstlane(bytes)), 0x00027000);
}

// Direct-to-LDS loads through a resource: 64 lanes x 16 (or 4) bytes land contiguously at LDS byte offset lds_off. The
// kernels place their own waits (see dma16 in expert_gemm_kernel.h). A scalar register that the vector unit has written may be
// read by a vector memory instruction five instructions later; the compiler does not see that this is one.
template <bool STREAM = false>
__device__ __forceinline__ void dma16(__amdgpu_buffer_rsrc_t from, uint32_t voff, uint32_t soff, uint32_t lds_off) {
    if constexpr (STREAM)
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tbuffer_load_dwordx4 %1, %2, %3 offen nt lds"
                     :: "s"(lds_off), "v"(voff), "s"(from), "s"(soff) : "memory", "m0");
    else
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds"
                     :: "s"(lds_off), "v"(voff), "s"(from), "s"(soff) : "memory", "m0");
}
__device__ __forceinline__ void dma4(__amdgpu_buffer_rsrc_t from, uint32_t voff, uint32_t lds_off) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tbuffer_load_dword %1, %2, 0 offen lds"
                 :: "s"(lds_off), "v"(voff), "s"(from) : "memory", "m0");
}

// ---- epilogues -----------------------------------------------------------------------------------------------------------
// Largest value over the four lane groups that hold a row's columns, in all of them.
__device__ __forceinline__ uint32_t max_over_groups(uint32_t v) {
    const auto a = __builtin_amdgcn_permlane16_swap(v, v, false, false);
    v = max(a[0], a[1]);
    const auto b = __builtin_amdgcn_permlane32_swap(v, v, false, false);
    return max(b[0], b[1]);
}

// 32 columns of a row as a block: v[4 jj + r] is column 16 jj + 4 g + r. Codes as the row's 16 bytes, 4 to a lane: `part` says
// which 4 (lane groups 0 to 3 hold parts 0, 2, 1, 3).
__device__ __forceinline__ uint32_t block_codes(const float (&v)[8], int g, uint32_t& scale, int& part) {
    uint32_t peak = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) peak = max(peak, __float_as_uint(v[i]) & 0x7fffffffu);
    scale = mx_scale(max_over_groups(peak));
    const uint32_t w = mx_codes(v, scale);           // columns 4 g .. + 3 in the low half, 16 + 4 g .. + 3 in the high one
    // lane groups 2 i and 2 i + 1 see each other's: the even one ends up with columns 8 i .. + 7, the odd one with 16 + 8 i .. + 7
    const auto of = __builtin_amdgcn_permlane16_swap(w, w, false, false);
    part = (g & 1) * 2 + (g >> 1);
    return (g & 1) ? __builtin_amdgcn_perm(of[1], of[0], 0x07060302u) : __builtin_amdgcn_perm(of[1], of[0], 0x05040100u);
}

// A block's scale, by one lane of the row's: and where the row ends in the middle of a run of 8 blocks, a 0 for the block behind
// it in the same 16 bits (rows of a multiple of 128: half a run).
__device__ __forceinline__ void store_scale(uint8_t* scales, int R, long long row, int block, int blocks, uint32_t scale) {
    uint8_t* at = scales + (static_cast<size_t>(block >> 3) * R + row) * kMxRunBytes + mx_byte(block & 7);
    if (block + 4 >= blocks && (block & 4) == 0) *reinterpret_cast<uint16_t*>(at) = static_cast<uint16_t>(scale);
    else *at = static_cast<uint8_t>(scale);
}

// ---- tiles of a ring of LDS stages, every wavefront loads and computes ----------------------------------------------------
template <int BM_, int BN_, int WM_, int WN_, int NSTAGE_, bool DUAL_, bool STREAM_B_ = false, bool F32_ = false>
struct Tile {
    static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_, NSTAGE = NSTAGE_;
    static constexpr bool DUAL = DUAL_, STREAM_B = STREAM_B_, F32 = F32_;
    static constexpr int NW = WM * WN, NTHREADS = NW * kWave;
    static constexpr int WTM = BM / WM, WTN = BN / WN, TM = WTM / 16, TN = WTN / 16;
    static constexpr int BN_OUT = DUAL ? BN / 2 : BN;
    static constexpr int A_BYTES = BM * 128, B_BYTES = BN * 128;
    static constexpr int SA_BYTES = (BM * 8 + 255) / 256 * 256, SB_BYTES = (BN * 8 + 255) / 256 * 256;
    static constexpr int B_AT = A_BYTES, SA_AT = B_AT + B_BYTES, SB_AT = SA_AT + SA_BYTES, STAGE = SB_AT + SB_BYTES;
    static constexpr int SMEM = NSTAGE * STAGE;
    static constexpr int NIA = BM / 8, NIB = BN / 8, NSA = SA_BYTES / 256, NS = NSA + SB_BYTES / 256;
    // loads of a wavefront per stage; where they do not divide evenly the last ones are made twice
    static constexpr int LA = (NIA + NW - 1) / NW, LB = (NIB + NW - 1) / NW, LS = (NS + NW - 1) / NW, LPW = LA + LB + LS;
    static_assert(BM % (WM * 16) == 0 && BN % (WN * 16) == 0 && (!DUAL || WTN % 64 == 0), "wave tile");
    static_assert(NSTAGE >= 2 && SMEM <= 160 * 1024 && NSTAGE * LPW < 64, "LDS, loads in flight");
};

template <class Cfg>
__device__ __forceinline__ TileCoord tile_of_workgroup(const Operands& op) {
    const int nt = (op.N + Cfg::BN_OUT - 1) / Cfg::BN_OUT;
    return op.offsets == nullptr ? gemm::locate_tile_of_one<Cfg::BM>(op.R, nt) : gemm::locate_tile<Cfg::BM>(op.offsets, op.E, nt);
}

// Loads of a wavefront: DUAL tiles hold 32 rows of W1, then the same 32 of W3, in turn.
template <class Cfg>
struct Loads {
    // four loads are 32 rows of one matrix: of DUAL tiles a wavefront's loads are of both in turn, or of one
    static constexpr int BLOCKS = Cfg::DUAL && Cfg::LB > 4 ? 2 : 1;
    static_assert(!Cfg::DUAL || Cfg::LB % 8 == 0 || 4 % Cfg::LB == 0, "whole blocks");
    __amdgpu_buffer_rsrc_t a, b[BLOCKS];
    const uint8_t *a_scale, *b_scale[2];             // of the first k-step
    uint32_t a_scale_bytes, b_scale_bytes;
    uint32_t a_voff[Cfg::LA], b_voff[Cfg::LB];
    int wave, lane;
    __device__ __forceinline__ void init(const Operands& op, const TileCoord& tc, int wave_, int lane_) {
        wave = wave_;
        lane = lane_;
        const uint32_t pitch = static_cast<uint32_t>(op.K) / 2;
        const int col0 = tc.nt * Cfg::BN_OUT, cols = min(Cfg::BN_OUT, op.N - col0), runs = mx_runs(op.K);
        a = resource(op.a + static_cast<size_t>(tc.row0) * pitch, tc.rows * pitch);
        a_scale = op.a_scale + static_cast<size_t>(tc.row0) * kMxRunBytes;
        a_scale_bytes = tc.rows * kMxRunBytes;
        b_scale_bytes = cols * kMxRunBytes;
#pragma unroll
        for (int n = 0; n < BLOCKS; ++n) {
            const uint8_t* from = Cfg::DUAL && (BLOCKS == 2 ? n : (wave * Cfg::LB >> 2) & 1) ? op.b[1] : op.b[0];
            b[n] = resource(from + (static_cast<size_t>(tc.expert) * op.N + col0) * pitch, cols * pitch);
        }
#pragma unroll
        for (int m = 0; m < (Cfg::DUAL ? 2 : 1); ++m) {
            b_scale[m] = op.b_scale[m] + (static_cast<size_t>(tc.expert) * runs * op.N + col0) * kMxRunBytes;
        }
        const int lrow = lane >> 3;
        auto at = [&](int row, int column) {
            return static_cast<uint32_t>(column) * pitch + (((lane & 7) ^ gemm::swz<64>(row)) * 16);
        };
#pragma unroll
        for (int i = 0; i < Cfg::LA; ++i) a_voff[i] = at(load_a(i) * 8 + lrow, load_a(i) * 8 + lrow);
#pragma unroll
        for (int i = 0; i < Cfg::LB; ++i) {
            const int row = load_b(i) * 8 + lrow;
            b_voff[i] = at(row, Cfg::DUAL ? row / 64 * 32 + row % 32 : row);
        }
    }
    __device__ __forceinline__ int load_a(int i) const { return min(wave * Cfg::LA + i, Cfg::NIA - 1); }
    __device__ __forceinline__ int load_b(int i) const { return min(wave * Cfg::LB + i, Cfg::NIB - 1); }
    // all loads of k-step kt into the stage at LDS byte offset `stage`
    __device__ __forceinline__ void issue(const Operands& op, uint32_t stage, int kt) {
        const uint32_t koff = kt * 128;
#pragma unroll
        for (int i = 0; i < Cfg::LB; ++i) {
            dma16<Cfg::STREAM_B>(b[BLOCKS == 2 ? (i >> 2) & 1 : 0], b_voff[i], koff, stage + Cfg::B_AT + load_b(i) * 1024);
        }
#pragma unroll
        for (int i = 0; i < Cfg::LA; ++i) dma16(a, a_voff[i], koff, stage + load_a(i) * 1024);
#pragma unroll
        for (int i = 0; i < Cfg::LS; ++i) {
            const int q = min(wave * Cfg::LS + i, Cfg::NS - 1);
            if (q < Cfg::NSA) {
                const uint8_t* from = a_scale + static_cast<size_t>(kt) * op.R * kMxRunBytes;
                dma4(resource(from, a_scale_bytes), q * 256 + lane * 4, stage + Cfg::SA_AT + q * 256);
            } else {
                const int p = q - Cfg::NSA;          // 32 rows of the tile
                const int m = Cfg::DUAL ? p & 1 : 0;
                const uint8_t* from = (m ? b_scale[1] : b_scale[0]) + static_cast<size_t>(kt) * op.N * kMxRunBytes;
                dma4(resource(from, b_scale_bytes), (Cfg::DUAL ? p >> 1 : p) * 256 + lane * 4, stage + Cfg::SB_AT + p * 256);
            }
        }
    }
};

template <class Cfg>
__device__ __forceinline__ void store_tile(const f32x4 (&acc)[Cfg::TM][Cfg::TN], const Operands& op, const TileCoord& tc,
                                           const Outputs& out, int wm, int wn, int frag_row, int g) {
#pragma unroll
    for (int i = 0; i < Cfg::TM; ++i) {
        const int r = wm * Cfg::WTM + i * 16 + frag_row;
        const bool in = r < tc.rows;                 // lanes of a row together
        const size_t row = static_cast<size_t>(tc.row0) + r;
        if constexpr (Cfg::DUAL) {
#pragma unroll
            for (int b = 0; b < Cfg::TN / 4; ++b) {
                const int col = tc.nt * Cfg::BN_OUT + wn * (Cfg::WTN / 2) + b * 32;
                float v[8];
#pragma unroll
                for (int q = 0; q < 8; ++q)
                    v[q] = gemm::silu(acc[i][4 * b + q / 4][q & 3]) * acc[i][4 * b + 2 + q / 4][q & 3];
                uint32_t scale;
                int part;
                const uint32_t codes = block_codes(v, g, scale, part);
                if (!in || col >= op.N) continue;
                *reinterpret_cast<uint32_t*>(static_cast<uint8_t*>(out.c) + row * (op.N / 2) + col / 2 + part * 4) = codes;
                if (g == 0) store_scale(out.scale, op.R, row, col / 32, op.N / 32, scale);
            }
        } else {
#pragma unroll
            for (int j = 0; j < Cfg::TN; ++j) {
                const int col = tc.nt * Cfg::BN + wn * Cfg::WTN + j * 16;
                if (!in || col >= op.N) continue;
                const size_t at = row * op.N + col + 4 * g;
                if constexpr (Cfg::F32) {
                    *reinterpret_cast<f32x4*>(static_cast<float*>(out.c) + at) = acc[i][j];
                } else {
                    gemm::bf16x4 o;
#pragma unroll
                    for (int q = 0; q < 4; ++q) o[q] = static_cast<__bf16>(acc[i][j][q]);
                    *reinterpret_cast<gemm::bf16x4*>(static_cast<uint16_t*>(out.c) + at) = o;
                }
            }
        }
    }
}

// The k-step that a tile begins with; the others follow in turn. Workgroups that start together stay at the same k, where weight rows
// a multiple of 4 KB apart fall on few memory channels: n-tiles then begin at k-steps that their numbers draw (those that share
// weights share the order). Expert FFN, 8 experts of 8192 x 8192, all from the first k-step -> so: 8 tokens 144 -> 121 us, 64 160 ->
// 142, 256 179 -> 168, 400 182 -> 174; one matrix of 8192 x 32000, 37 rows 35.4 -> 29.6; rows of 2 KB, or no multiple: no difference.
template <class Cfg>
__device__ __forceinline__ int first_kstep(const Operands& op, const TileCoord& tc, int KT) {
    if (op.K % 8192 != 0) return 0;
    const uint32_t tile = static_cast<uint32_t>(tc.expert) * ((op.N + Cfg::BN_OUT - 1) / Cfg::BN_OUT) + tc.nt;
    return static_cast<int>(__umulhi(tile * 0x9e3779b9u, static_cast<uint32_t>(KT)));
}

template <class Cfg>
__global__ __launch_bounds__(Cfg::NTHREADS) void ring_kernel(Operands op, Outputs out) {
    constexpr int TM = Cfg::TM, TN = Cfg::TN, S = Cfg::NSTAGE;
    extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];
    const TileCoord tc = tile_of_workgroup<Cfg>(op);
    if (tc.expert < 0) return;                       // the same for the whole workgroup
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave / Cfg::WN, wn = wave % Cfg::WN, frag_row = lane & 15, g = lane >> 4;
    Loads<Cfg> loads;
    loads.init(op, tc, wave, lane);
    const int KT = mx_runs(op.K), first = first_kstep<Cfg>(op, tc, KT);
    auto issue = [&](int stage, int s) {             // k-step number s here
        const int t = first + s;
        loads.issue(op, stage * Cfg::STAGE, t >= KT ? t - KT : t);
    };
#pragma unroll
    for (int s = 0; s < S - 1; ++s)
        if (s < KT) issue(s, s);
    f32x4 acc[TM][TN];
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    uint32_t at[2];                                  // of a lane's two chunks inside 16 rows
#pragma unroll
    for (int h = 0; h < 2; ++h) at[h] = frag_row * 128 + (((h * 4 + g) ^ gemm::swz<64>(frag_row)) << 4);
    int stage = 0;
    for (int kt = 0; kt < KT; ++kt) {
        if (kt + S - 2 < KT) gemm::wait_vmcnt<(S - 2) * Cfg::LPW>(); else gemm::wait_vmcnt<0>();
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");       // own reads of the stage before, wherever their MFMAs are
        __builtin_amdgcn_s_barrier();                // stage `stage` is there, the one before is no longer read
        asm volatile("" ::: "memory");               // and is not read ahead of the barrier
        const unsigned char* base = smem + stage * Cfg::STAGE;
        i32x4 fa[2][TM], fb[2][TN];
        int sa[TM], sb[TN];
#pragma unroll
        for (int i = 0; i < TM; ++i)
            sa[i] = *reinterpret_cast<const uint16_t*>(base + Cfg::SA_AT + (wm * Cfg::WTM + i * 16 + frag_row) * 8 + 2 * g);
#pragma unroll
        for (int j = 0; j < TN; ++j)
            sb[j] = *reinterpret_cast<const uint16_t*>(base + Cfg::SB_AT + (wn * Cfg::WTN + j * 16 + frag_row) * 8 + 2 * g);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
#pragma unroll
            for (int i = 0; i < TM; ++i)
                fa[h][i] = *reinterpret_cast<const i32x4*>(base + (wm * Cfg::WTM + i * 16) * 128 + at[h]);
#pragma unroll
            for (int j = 0; j < TN; ++j)
                fb[h][j] = *reinterpret_cast<const i32x4*>(base + Cfg::B_AT + (wn * Cfg::WTN + j * 16) * 128 + at[h]);
        }
        if (kt + S - 1 < KT) issue(stage == 0 ? S - 1 : stage - 1, kt + S - 1);
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
            for (int j = 0; j < TN; ++j) acc[i][j] = mma<0>(fb[0][j], fa[0][i], acc[i][j], sb[j], sa[i]);
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
            for (int j = 0; j < TN; ++j) acc[i][j] = mma<1>(fb[1][j], fa[1][i], acc[i][j], sb[j], sa[i]);
        stage = stage + 1 == S ? 0 : stage + 1;
    }
    store_tile<Cfg>(acc, op, tc, out, wm, wn, frag_row, g);
}

// ---- large tiles: one wavefront per SIMD, hand-placed pipeline -------------------------------------------------------------
// 256 x 256 outputs, 128 x 128 to a wavefront, as grouped_gemm_1w_kernel has them (expert_gemm_kernel.h): two half-steps of one
// instruction of 128 elements each, every LDS read, direct-to-LDS load and scalar update behind an MFMA of its own, the barrier
// of a k-step between its halves. LDS does not hold that kernel's five stages of 32 KB and the scales, so the B ring holds two and a
// half: five halves of 128 rows, of which k-step kt has numbers 2 kt and 2 kt + 1 modulo 5. In the first half of k-step kt go out
// the loads of the first B half of kt + 2, into the place that has been idle since the barrier of kt - 1, and its scales (a
// ring of four k-steps), in the second half the loads of its A rows and second B half, into the places that the barrier of kt
// has freed: at that barrier only the first half's loads may still be on their way. The scales of k-step kt + 1 are read from
// LDS in the second half of kt, 16 bits for each fragment's row and lane group: one byte for each half-step.
// Loads go through resources that advance by a k-step at a time and end where the tile's rows do. In the last two k-steps of a
// tile they stand on the next one, or are empty where there is none: they then bring zeros and read nothing, and every k-step
// runs the same code.
template <class Cfg>
struct Mx4 : Cfg {
    static constexpr bool ANY_WIDTH = true;
};
template <class Cfg>
struct Large {
    static constexpr uint32_t AB = 256 * 128, HB = 128 * 128, A_RING = 2 * AB, B_RING = 5 * HB, SCALES = A_RING + B_RING;
    static constexpr uint32_t SA = 256 * 8, SS = 2 * SA, SMEM = SCALES + 4 * SS;      // a k-step's scales: of A, then of B
    static_assert(SMEM <= 160 * 1024 && Cfg::BM == 256 && Cfg::BN == 256 && Cfg::NW == 4, "256 x 256");
};

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
// A resource in four scalar registers: address, bytes, format.
__device__ __forceinline__ u32x4 resource_words(const void* base, uint32_t bytes) {
    const uint64_t at = reinterpret_cast<uint64_t>(base);
    return u32x4{static_cast<uint32_t>(__builtin_amdgcn_readfirstlane(static_cast<uint32_t>(at))),
                 static_cast<uint32_t>(__builtin_amdgcn_readfirstlane(static_cast<uint32_t>(at >> 32))),
                 static_cast<uint32_t>(__builtin_amdgcn_readfirstlane(bytes)), 0x00027000u};
}
__device__ __forceinline__ void advance(u32x4& r, uint64_t by) {
    const uint64_t at = (r[0] | static_cast<uint64_t>(r[1]) << 32) + by;
    r[0] = static_cast<uint32_t>(at);
    r[1] = static_cast<uint32_t>(at >> 32);
}
template <int BYTES>
__device__ __forceinline__ void dma(const u32x4& from, uint32_t voff, uint32_t lds_off) {
    if constexpr (BYTES == 16)
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds"
                     :: "s"(lds_off), "v"(voff), "s"(from) : "memory", "m0");
    else
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tbuffer_load_dword %1, %2, 0 offen lds"
                     :: "s"(lds_off), "v"(voff), "s"(from) : "memory", "m0");
}

// acc += W_frag * X_frag with the accumulator pinned to AGPRs (see mma16_agpr), and the same with one direct-to-LDS load behind
// it, whose LDS address goes to M0 in front.
template <int H>
__device__ __forceinline__ void mma_agpr(const i32x4& w, const i32x4& x, f32x4& acc, int ws, int xs) {
    if constexpr (H == 0)
        asm volatile("v_mfma_scale_f32_16x16x128_f8f6f4 %0, %1, %2, %0, %3, %4 op_sel:[0,0,0] op_sel_hi:[0,0,0] cbsz:4 blgp:4"
                     : "+a"(acc) : "v"(w), "v"(x), "v"(ws), "v"(xs));
    else
        asm volatile("v_mfma_scale_f32_16x16x128_f8f6f4 %0, %1, %2, %0, %3, %4 op_sel:[1,1,0] op_sel_hi:[0,0,0] cbsz:4 blgp:4"
                     : "+a"(acc) : "v"(w), "v"(x), "v"(ws), "v"(xs));
}
template <int H, int BYTES, int LDS_OFF>
__device__ __forceinline__ void mma_then_dma(const i32x4& w, const i32x4& x, f32x4& acc, int ws, int xs, uint32_t lds_base,
                                             uint32_t voff, const u32x4& from) {
#define MOE_MX4_STEP(SEL, LOAD)                                                                                        \
    asm volatile("s_add_u32 m0, %5, %6\n\t"                                                                            \
                 "v_mfma_scale_f32_16x16x128_f8f6f4 %0, %1, %2, %0, %3, %4 op_sel:" SEL " op_sel_hi:[0,0,0] cbsz:4 blgp:4\n\t" \
                 LOAD " %7, %8, 0 offen lds"                                                                           \
                 : "+a"(acc)                                                                                           \
                 : "v"(w), "v"(x), "v"(ws), "v"(xs), "s"(lds_base), "n"(LDS_OFF), "v"(voff), "s"(from)                 \
                 : "memory", "m0", "scc")
    if constexpr (H == 0 && BYTES == 16) MOE_MX4_STEP("[0,0,0]", "buffer_load_dwordx4");
    else if constexpr (H == 0) MOE_MX4_STEP("[0,0,0]", "buffer_load_dword");
    else if constexpr (BYTES == 16) MOE_MX4_STEP("[1,1,0]", "buffer_load_dwordx4");
    else MOE_MX4_STEP("[1,1,0]", "buffer_load_dword");
#undef MOE_MX4_STEP
}

// Loads of a tile: A load i of wavefront w is tile rows 8 (4 i + w) .. + 7, so that the first TM loads of all wavefronts are the
// rows of a tile of TM * 32 rows; B load i of half b is B-tile rows 128 b + 32 w + 8 i .. + 7 (with DUAL 32 rows of one matrix).
template <class Cfg>
struct LargeLoads {
    u32x4 a, b, sa, sb[Cfg::DUAL ? 2 : 1];           // at the k-step whose loads are next
    uint32_t a_voff[8], b_voff[8], sa_voff, sb_voff; // of the first scale loads; the second ones are 256 bytes on
    uint64_t sa_step, sb_step;
    uint32_t shorter;                                // what a and b lose with a k-step: nothing where they are empty
    // what is the same for every tile
    __device__ __forceinline__ void init(const Operands& op, int wave, int lane) {
        const uint32_t pitch = static_cast<uint32_t>(op.K) / 2;
        sa_step = static_cast<uint64_t>(op.R) * kMxRunBytes;
        sb_step = static_cast<uint64_t>(op.N) * kMxRunBytes;
        const int lrow = lane >> 3;
        const uint32_t achunk = ((lane & 7) ^ gemm::swz<64>(8 * wave + lrow)) * 16;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            a_voff[i] = (8 * (4 * i + wave) + lrow) * pitch + achunk;
            const int row = 128 * (i >> 2) + 32 * wave + 8 * (i & 3) + lrow;
            b_voff[i] = (Cfg::DUAL ? row / 64 * 32 + row % 32 : row) * pitch + ((lane & 7) ^ gemm::swz<64>(row)) * 16;
        }
        sa_voff = wave * 512 + lane * 4;
        sb_voff = (Cfg::DUAL ? wave * 256 : wave * 512) + lane * 4;
    }
    // to the first k-step of a tile; one without rows loads nothing
    __device__ __forceinline__ void start(const Operands& op, const TileCoord& tc, int wave) {
        const uint32_t pitch = static_cast<uint32_t>(op.K) / 2;
        const int col0 = gemm::first_column<Cfg>(tc, op.N), cols = tc.rows > 0 ? Cfg::BN_OUT : 0;
        const size_t first = static_cast<size_t>(tc.expert) * op.N + col0;
        const size_t first_scale = (static_cast<size_t>(tc.expert) * mx_runs(op.K) * op.N + col0) * kMxRunBytes;
        shorter = tc.rows > 0 ? 128u : 0u;
        a = resource_words(op.a + static_cast<size_t>(tc.row0) * pitch, tc.rows * pitch);
        b = resource_words((Cfg::DUAL && (wave & 1) ? op.b[1] : op.b[0]) + first * pitch, cols * pitch);
        sa = resource_words(op.a_scale + static_cast<size_t>(tc.row0) * kMxRunBytes, tc.rows * kMxRunBytes);
#pragma unroll
        for (int m = 0; m < (Cfg::DUAL ? 2 : 1); ++m) sb[m] = resource_words(op.b_scale[m] + first_scale, cols * kMxRunBytes);
    }
    // from here on nothing is loaded: zeros go to LDS
    __device__ __forceinline__ void stop() {
        a[2] = b[2] = sa[2] = shorter = 0;
#pragma unroll
        for (int m = 0; m < (Cfg::DUAL ? 2 : 1); ++m) sb[m][2] = 0;
    }
    // to the next k-step
    __device__ __forceinline__ void next_scales() {
        advance(sa, sa_step);
#pragma unroll
        for (int m = 0; m < (Cfg::DUAL ? 2 : 1); ++m) advance(sb[m], sb_step);
    }
    __device__ __forceinline__ void next_rows() {
        advance(a, 128);
        a[2] -= shorter;
        advance(b, 128);
        b[2] -= shorter;
    }
    __device__ __forceinline__ u32x4 scale_source(int m) const { return sb[Cfg::DUAL ? m : 0]; }
    static constexpr uint32_t sb_second = Cfg::DUAL ? 0 : 256;
};

struct LargeState {
    uint32_t sa, s0, ss;             // LDS offsets of k-step kt: A stage, first B half's place, scales (of its ring)
};

// One k-step. On entry f[0] holds its first-half fragments and sc its scales; on return those of k-step kt + 1 are in f[0] and
// nsc. pa, pb, psa, psb: the wavefront's fragment and scale addresses in a first stage.
template <class Cfg, class Full>
__device__ __forceinline__ void large_kstep(f32x4 (&acc)[Cfg::TM][8], i32x4 (&fa)[2][Cfg::TM], i32x4 (&fb)[2][8],
                                            const int (&sca)[Cfg::TM], const int (&scb)[8], int (&nsa)[Cfg::TM], int (&nsb)[8],
                                            LargeState& st, LargeLoads<Full>& lp, int wave, int wn, const unsigned char* pa0,
                                            const unsigned char* pa1, const unsigned char* pb0, const unsigned char* pb1,
                                            const unsigned char* psa, const unsigned char* psb) {
    using L = Large<Full>;
    constexpr int TM = Cfg::TM, NM = TM * 8, NR = TM + 8;
    constexpr int STRIDE1 = NM / 8, NL2 = TM + 4, STRIDE2 = NM / NL2;
    constexpr int SPAN1 = (3 * NR <= NM - 4) ? 3 * NR : 2 * NR;
    static_assert(TM >= 4 && TM <= 8, "64 to 128 rows of a wavefront");
    auto wrap = [](uint32_t v) { return v >= L::B_RING ? v - L::B_RING : v; };
    const uint32_t own = wrap(st.s0 + wn * L::HB);                       // the wavefront's columns
    const uint32_t s0n = wrap(st.s0 + 2 * L::HB), own_n = wrap(s0n + wn * L::HB);
    const uint32_t idle = wrap(st.s0 + 4 * L::HB);                       // place of the first B half of kt + 2
    const uint32_t ssn = (st.ss + L::SS) & (4 * L::SS - 1);
    const uint32_t scales_to = L::SCALES + ((st.ss + 2 * L::SS) & (4 * L::SS - 1)) + wave * 512;
    const uint32_t b0_to = L::A_RING + idle + wave * 4096, b1_to = L::A_RING + st.s0 + wave * 4096, a_to = st.sa + wave * 1024;
    const unsigned char *pa_h1 = pa1 + st.sa, *pb_h1 = pb1 + own, *pa_n0 = pa0 + (st.sa ^ L::AB), *pb_n0 = pb0 + own_n;
    const unsigned char *psa_n = psa + ssn, *psb_n = psb + ssn;
    // ---- first half: MFMAs on f[0]; read f[1]; four B loads, four scale loads
    auto first = [&](auto mtag) {
        constexpr int m = decltype(mtag)::value, i = m >> 3, j = m & 7, n = m / STRIDE1;
        if constexpr (m % STRIDE1 == STRIDE1 - 1 && n < 4)
            mma_then_dma<0, 16, n * 1024>(fb[0][j], fa[0][i], acc[i][j], scb[j], sca[i], b0_to, lp.b_voff[n], lp.b);
        else if constexpr (m % STRIDE1 == STRIDE1 - 1 && n < 6)
            mma_then_dma<0, 4, (n - 4) * 256>(fb[0][j], fa[0][i], acc[i][j], scb[j], sca[i], scales_to, lp.sa_voff + (n - 4) * 256, lp.sa);
        else if constexpr (m % STRIDE1 == STRIDE1 - 1)
            mma_then_dma<0, 4, L::SA + (n - 6) * 256>(fb[0][j], fa[0][i], acc[i][j], scb[j], sca[i], scales_to,
                                                      lp.sb_voff + (n - 6) * LargeLoads<Full>::sb_second, lp.scale_source(n - 6));
        else
            mma_agpr<0>(fb[0][j], fa[0][i], acc[i][j], scb[j], sca[i]);
        MOE_FENCE();
        constexpr int r = (m * NR + SPAN1 - 1) / SPAN1;
        if constexpr (r < NR && (r * SPAN1) / NR == m) {
            if constexpr (r < 8) fb[1][r] = *reinterpret_cast<const i32x4*>(pb_h1 + r * 2048);
            else fa[1][r - 8] = *reinterpret_cast<const i32x4*>(pa_h1 + (r - 8) * 2048);
            MOE_FENCE();
        }
    };
    // ---- second half: MFMAs on f[1]; read f[0] and the scales of kt + 1; the A loads and four B loads
    auto second = [&](auto mtag) {
        constexpr int m = decltype(mtag)::value, i = m >> 3, j = m & 7, n = m / STRIDE2;
        if constexpr (m % STRIDE2 == STRIDE2 - 1 && n < 4)
            mma_then_dma<1, 16, n * 1024>(fb[1][j], fa[1][i], acc[i][j], scb[j], sca[i], b1_to, lp.b_voff[4 + n], lp.b);
        else if constexpr (m % STRIDE2 == STRIDE2 - 1 && n < NL2)
            mma_then_dma<1, 16, (n - 4) * 4096>(fb[1][j], fa[1][i], acc[i][j], scb[j], sca[i], a_to, lp.a_voff[n - 4], lp.a);
        else
            mma_agpr<1>(fb[1][j], fa[1][i], acc[i][j], scb[j], sca[i]);
        MOE_FENCE();
        constexpr int r = (m * 2 * NR + NM - 1) / NM;                    // read r behind MFMA r * NM / (2 NR)
        if constexpr (r < 2 * NR && (r * NM) / (2 * NR) == m) {
            if constexpr (r % 2 == 0) {
                if constexpr (r / 2 < 8) fb[0][r / 2] = *reinterpret_cast<const i32x4*>(pb_n0 + r / 2 * 2048);
                else fa[0][r / 2 - 8] = *reinterpret_cast<const i32x4*>(pa_n0 + (r / 2 - 8) * 2048);
            } else {
                if constexpr (r / 2 < 8) nsb[r / 2] = *reinterpret_cast<const uint16_t*>(psb_n + r / 2 * 128);
                else nsa[r / 2 - 8] = *reinterpret_cast<const uint16_t*>(psa_n + (r / 2 - 8) * 128);
            }
            MOE_FENCE();
        }
    };
    gemm::static_for<NM>(first);
    lp.next_scales();
    asm volatile("s_waitcnt vmcnt(8) lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();      // k-step kt + 1 complete in LDS; this k-step's stages are free
    MOE_FENCE();
    gemm::static_for<NM>(second);
    lp.next_rows();
    st.sa ^= L::AB;
    st.s0 = s0n;
    st.ss = ssn;
}

// H's columns of a wavefront, two blocks of 32, straight from the accumulators. `before_stores` runs once, ahead of the first.
// A lane holds 4 columns of each of the blocks' halves. One swap of neighbouring lane groups turns (mine of both blocks) into (mine
// and the neighbour's of one block), groups 0 and 2 of the first, 1 and 3 of the second, one of the upper and lower half
// wavefronts brings 8 bytes of codes together; the maxima go the same way, and a third swap back. Stores go through resources
// that end behind the wavefront's last row. What is left is bound by the exponentials and reciprocals of SiLU (16 cycles each,
// by count 3.2 us of a tile's 4.6 at 1.9 GHz).
template <class Cfg, class Before>
__device__ __forceinline__ void store_blocks(const f32x4 (&acc)[Cfg::TM][8], const Operands& op, const TileCoord& tc,
                                             const Outputs& out, int wm, int wn, int lane, Before&& before_stores) {
    const int frag_row = lane & 15, g = lane >> 4;
    const int col0 = tc.nt * Cfg::BN_OUT + wn * 64, block0 = col0 / 32;
    const uint32_t pitch = static_cast<uint32_t>(op.N) / 2;
    const int rows = max(0, min(Cfg::WTM, tc.rows - wm * Cfg::WTM));
    const size_t row0 = static_cast<size_t>(tc.row0) + wm * Cfg::WTM;
    const __amdgpu_buffer_rsrc_t codes_to = resource(static_cast<uint8_t*>(out.c) + row0 * pitch, rows * pitch);
    const __amdgpu_buffer_rsrc_t scales_to =
        resource(out.scale + (static_cast<size_t>(block0 >> 3) * op.R + row0) * kMxRunBytes, rows * kMxRunBytes);
    // the scales of a row that ends in the middle of a run of 8 blocks: with a 0 each for the blocks behind
    const bool ends = (block0 & 4) == 0 && block0 + 4 >= op.N / 32;
    uint32_t codes_at = frag_row * pitch + col0 / 2 + (g & 1) * 16 + (g >> 1) * 8;
    uint32_t scale_at = g < 2 ? frag_row * kMxRunBytes + mx_byte((block0 & 7) + (g & 1)) : 0x40000000u;      // groups 0 and 1
#pragma unroll
    for (int i = 0; i < Cfg::TM; ++i) {
        float v[2][8], u[2][8];
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int q = 0; q < 8; ++q) {
                v[b][q] = gemm::read_acc(acc[i][4 * b + q / 4], q & 3);
                u[b][q] = gemm::read_acc(acc[i][4 * b + 2 + q / 4], q & 3);
            }
        uint32_t peak[2] = {0, 0};
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int q = 0; q < 8; ++q) {
                v[b][q] = gemm::silu(v[b][q]) * u[b][q];
                peak[b] = max(peak[b], __float_as_uint(v[b][q]) & 0x7fffffffu);
            }
        const auto p = __builtin_amdgcn_permlane16_swap(peak[0], peak[1], false, false);
        const uint32_t m = max(p[0], p[1]);
        const auto h = __builtin_amdgcn_permlane32_swap(m, m, false, false);
        const uint32_t mine = max(h[0], h[1]);
        const auto both = __builtin_amdgcn_permlane16_swap(mine, mine, false, false);
        const uint32_t w0 = mx_codes(v[0], mx_scale(both[0])), w1 = mx_codes(v[1], mx_scale(both[1]));
        const auto w = __builtin_amdgcn_permlane16_swap(w0, w1, false, false);
        const uint32_t low = __builtin_amdgcn_perm(w[1], w[0], 0x05040100u), high = __builtin_amdgcn_perm(w[1], w[0], 0x07060302u);
        const auto c = __builtin_amdgcn_permlane32_swap(low, high, false, false);
        if (i == 0) before_stores();
        typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
        __builtin_amdgcn_raw_buffer_store_b64(u32x2{c[0], c[1]}, codes_to, codes_at, 0, 0);
        const uint32_t scale = mx_scale(mine);
        if (ends) __builtin_amdgcn_raw_buffer_store_b16(static_cast<uint16_t>(scale), scales_to, scale_at, 0, 0);
        else __builtin_amdgcn_raw_buffer_store_b8(static_cast<uint8_t>(scale), scales_to, scale_at, 0, 0);
        codes_at += 16 * pitch;
        scale_at += 16 * kMxRunBytes;
        MOE_FENCE();
    }
}

// One tile of at least two k-steps, three if ODD. On entry its first two are in the rings, at the places of `st`, and every
// wavefront knows it; on return those of the next tile are, and the stores of this one are on their way.
//   lp     loads of this tile at k-step 2, then of the next one; last: there is none
//   draw   called once in each wavefront two k-steps before the end; drawn() before the first store, when all loads of the
//          wavefront have landed
template <class Cfg, class Full, bool ODD, class Draw, class Drawn>
__device__ __forceinline__ void large_tile(const Operands& op, const Outputs& out, const TileCoord& tc, const TileCoord& nxt,
                                           bool last, LargeLoads<Full>& lp, LargeState& st, unsigned char* smem, int wave, int lane,
                                           Draw&& draw, Drawn&& drawn) {
    using L = Large<Full>;
    constexpr int TM = Cfg::TM;
    const int wm = wave / Cfg::WN, wn = wave % Cfg::WN, frag_row = lane & 15, g = lane >> 4;
    gemm::FragPlan<Cfg> fp;
    fp.init(lane, wm, wn);
    const unsigned char* pa[2] = {smem + fp.a_off[0], smem + fp.a_off[1]};
    // B-tile rows of a wavefront from the start of its half
    const unsigned char* pb[2] = {smem + L::A_RING + (fp.b_off[0] - Cfg::A_BYTES - wn * L::HB),
                                  smem + L::A_RING + (fp.b_off[1] - Cfg::A_BYTES - wn * L::HB)};
    const unsigned char* psa = smem + L::SCALES + (wm * Cfg::WTM + frag_row) * 8 + 2 * g;
    const unsigned char* psb = smem + L::SCALES + L::SA + (wn * 128 + frag_row) * 8 + 2 * g;
    i32x4 fa[2][TM], fb[2][8];
    int sa[2][TM], sb[2][8];
    const uint32_t own = st.s0 + wn * L::HB >= L::B_RING ? st.s0 + wn * L::HB - L::B_RING : st.s0 + wn * L::HB;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        fb[0][j] = *reinterpret_cast<const i32x4*>(pb[0] + own + j * 2048);
        sb[0][j] = *reinterpret_cast<const uint16_t*>(psb + st.ss + j * 128);
    }
#pragma unroll
    for (int i = 0; i < TM; ++i) {
        fa[0][i] = *reinterpret_cast<const i32x4*>(pa[0] + st.sa + i * 2048);
        sa[0][i] = *reinterpret_cast<const uint16_t*>(psa + st.ss + i * 128);
    }
    MOE_FENCE();
    f32x4 acc[TM][8];
    gemm::zero_accumulators(acc);
    auto step = [&](auto from) {
        constexpr int S = decltype(from)::value;
        large_kstep<Cfg, Full>(acc, fa, fb, sa[S], sb[S], sa[S ^ 1], sb[S ^ 1], st, lp, wave, wn, pa[0], pa[1], pb[0], pb[1], psa, psb);
    };
    if constexpr (ODD) step(std::integral_constant<int, 0>{});
    for (int left = mx_runs(op.K) - 2 - ODD;; left -= 2) {         // k-steps whose loads are this tile's
        if (left == 0) {
            if (last) {
                lp.stop();
            } else {
                lp.start(op, nxt, wave);
                draw();
            }
        }
        step(std::integral_constant<int, ODD ? 1 : 0>{});
        step(std::integral_constant<int, ODD ? 0 : 1>{});
        if (left == 0) break;
    }
    gemm::mfma_drain(acc[TM - 1]);
    // rows of a higher next tile that this one's loads did not reach, of both its k-steps: lp is two k-steps on
    if constexpr (TM < 8) {
        if (!last && nxt.height > Cfg::BM) {
            u32x4 first = lp.a, second = lp.a;
            const uint32_t bytes = nxt.rows * (static_cast<uint32_t>(op.K) / 2);
            advance(first, -256ll);
            advance(second, -128ll);
            first[2] = bytes;
            second[2] = bytes - 128u;
#pragma unroll
            for (int i = TM; i < 8; ++i) {
                dma<16>(first, lp.a_voff[i], st.sa + wave * 1024 + i * 4096);
                dma<16>(second, lp.a_voff[i], (st.sa ^ L::AB) + wave * 1024 + i * 4096);
            }
        }
    }
    auto before = [&] {
        __builtin_amdgcn_s_waitcnt(0x0f70);          // vmcnt(0): the next tile's first loads, and what draw() asked for
        drawn();
    };
    if constexpr (Cfg::DUAL) {
        store_blocks<Cfg>(acc, op, tc, out, wm, wn, lane, before);
    } else {
        // through the B half that is idle: every wavefront had read it at the last barrier, and the next load into it is the next
        // tile's first
        const uint32_t idle = st.s0 + 4 * L::HB >= L::B_RING ? st.s0 + 4 * L::HB - L::B_RING : st.s0 + 4 * L::HB;
        static_assert(4 * gemm::kEpilogueBytes <= L::HB, "room for the outputs");
        gemm::store_tile_via_lds<Cfg>(acc, tc, fp, wave, lane, smem + L::A_RING + idle + wave * gemm::kEpilogueBytes,
                                      static_cast<uint16_t*>(out.c), op.N, gemm::KeptScales<Cfg>{}, before);
    }
}

// PERSISTENT: a workgroup runs one tile after the other, as grouped_gemm_1w_kernel's do (slots, draws and their counter are
// described there): the next tile's first two k-steps are loaded in the last two of this one and arrive under its stores.
template <class Cfg, bool PERSISTENT, bool ODD>
__global__ __launch_bounds__(256) void large_kernel(Operands op, Outputs out, int split_cus, int32_t* __restrict__ counters) {
    using L = Large<Cfg>;
    extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];
    int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int xcd = blockIdx.x % kXcds, workgroups = gridDim.x / kXcds;
    int32_t* counter = counters + xcd * gemm::kCounterInts;
    const int NT = gemm::n_tiles<Cfg>(op.N);
    const gemm::Cut cut = op.K < 4 * gemm::kLongK ? gemm::Cut::kAlways : gemm::Cut::kLong;
    gemm::TileTable<256> table;                      // kept over the tiles: a lookup then reads no memory
    const uint32_t magic = gemm::division_magic(lane);
    TileCoord tc;
    if constexpr (PERSISTENT) {
        if (op.offsets == nullptr) table.init_one(op.R, NT, split_cus, xcd, lane);
        else table.init(op.offsets, op.E, NT, split_cus, xcd, lane);
        tc = gemm::uniform_tile(table.find(NT, cut, blockIdx.x / kXcds, magic));
        if (tc.expert == gemm::kNoTile) return;      // the same for the whole workgroup
    } else {
        tc = op.offsets == nullptr ? gemm::locate_tile_of_one<256>(op.R, NT, split_cus, cut)
                                   : gemm::locate_tile<256>(op.offsets, op.E, NT, split_cus, cut);
        if (tc.expert < 0) return;
    }
    // an empty slot is a tile without rows: it loads and stores nothing
    const TileCoord none{0, 0, 0, 0, 128};
    if (tc.expert == gemm::kEmptySlot) tc = none;
    bool last = !PERSISTENT, drew = false;
    int ahead = 0;                                   // lane 0 of wavefront 0: the latest draw
    LargeState st{0, 0, 0};
    // the scales of the tile's last k-step are no longer read when it is drawn, and overwritten in the next one's second k-step
    auto draw_at = [&] { return reinterpret_cast<int*>(smem + L::SCALES + ((st.ss + 3 * L::SS) & (4 * L::SS - 1))); };
    auto draw = [&] {
        if (PERSISTENT && threadIdx.x == 0) {
            int at = 0;                              // an address that the compiler does not know to be uniform
            asm volatile("" : "+v"(at));
            ahead = __hip_atomic_fetch_add(counter + at, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        }
    };
    auto drawn = [&] {
        if (PERSISTENT && wave == 0) {
            const int v = __builtin_amdgcn_readfirstlane(ahead);
            if (lane == 0) *draw_at() = v;
        }
    };
    LargeLoads<Cfg> lp;
    lp.init(op, wave, lane);
    lp.start(op, tc, wave);
#pragma unroll
    for (int s = 0; s < 2; ++s) {
#pragma unroll
        for (int i = 0; i < 8; ++i) dma<16>(lp.b, lp.b_voff[i], L::A_RING + (2 * s + (i >> 2)) * L::HB + wave * 4096 + (i & 3) * 1024);
#pragma unroll
        for (int i = 0; i < 8; ++i) dma<16>(lp.a, lp.a_voff[i], s * L::AB + wave * 1024 + i * 4096);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            dma<4>(lp.sa, lp.sa_voff + i * 256, L::SCALES + s * L::SS + wave * 512 + i * 256);
            dma<4>(lp.scale_source(i), lp.sb_voff + i * LargeLoads<Cfg>::sb_second, L::SCALES + s * L::SS + L::SA + wave * 512 + i * 256);
        }
        lp.next_scales();
        lp.next_rows();
    }
    gemm::wait_vmcnt<20>();                          // k-step 0 landed
    int slot = blockIdx.x / kXcds + workgroups;      // of the next tile
    while (true) {
        // lane-dependent addresses are formed anew for every tile: kept over the loop they would take the registers of fragments
        asm volatile("s_waitcnt lgkmcnt(0)" : "+v"(lane) :: "memory");
        __builtin_amdgcn_s_barrier();                // the tile's first k-step has landed for every wavefront
        asm volatile("" ::: "memory");
        TileCoord nxt = tc;
        if constexpr (PERSISTENT) {
            if (drew) slot = 2 * workgroups + __builtin_amdgcn_readfirstlane(*draw_at());
            const TileCoord found = gemm::uniform_tile(table.find(NT, cut, slot, magic));
            last = found.expert == gemm::kNoTile;
            if (found.expert == gemm::kEmptySlot)
                nxt = none;
            else if (!last)
                nxt = found;
            else if (drew && slot == table.range.slots + workgroups - 1 && threadIdx.x == 0)
                __hip_atomic_store(counter, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        }
        auto run = [&](auto tag) {
            using TileCfg = typename decltype(tag)::type;
            large_tile<TileCfg, Cfg, ODD>(op, out, tc, nxt, last, lp, st, smem, wave, lane, draw, drawn);
        };
        switch (tc.height) {
            case 128: run(gemm::type_tag<gemm::AtHeight<Cfg, 128>>{}); break;
            case 160: run(gemm::type_tag<gemm::AtHeight<Cfg, 160>>{}); break;
            case 192: run(gemm::type_tag<gemm::AtHeight<Cfg, 192>>{}); break;
            case 224: run(gemm::type_tag<gemm::AtHeight<Cfg, 224>>{}); break;
            default: run(gemm::type_tag<Cfg>{}); break;
        }
        if (last) break;
        tc = nxt;
        drew = true;
    }
}

}  // namespace mx4
namespace gemm {
template <class Cfg, int H>
struct WithHeight<mx4::Mx4<Cfg>, H> { using type = mx4::Mx4<typename WithHeight<Cfg, H>::type>; };
}  // namespace gemm
}  // namespace moe
