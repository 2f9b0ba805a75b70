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
// kernels place their own waits (see dma16 in expert_gemm_kernel.h).
template <bool STREAM = false>
__device__ __forceinline__ void dma16(__amdgpu_buffer_rsrc_t from, uint32_t voff, uint32_t soff, uint32_t lds_off) {
    if constexpr (STREAM)
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, %3 offen nt lds"
                     :: "s"(lds_off), "v"(voff), "s"(from), "s"(soff) : "memory", "m0");
    else
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds"
                     :: "s"(lds_off), "v"(voff), "s"(from), "s"(soff) : "memory", "m0");
}
__device__ __forceinline__ void dma4(__amdgpu_buffer_rsrc_t from, uint32_t voff, uint32_t lds_off) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dword %1, %2, 0 offen lds"
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
    // lane groups 2 i and 2 i + 1 exchange halves: the even one ends up with columns 8 i .. + 7, the odd one with 16 + 8 i .. + 7
    const uint32_t other = static_cast<uint32_t>(__shfl_xor(static_cast<int>(w), 16));
    part = (g & 1) * 2 + (g >> 1);
    return (g & 1) ? __builtin_amdgcn_perm(w, other, 0x07060302u) : __builtin_amdgcn_perm(other, w, 0x05040100u);
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
    const uint8_t *a_scale, *b_scale[2];             // of the k-step whose loads are next
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
    // all loads of k-step kt into the stage at LDS byte offset `stage`; k-steps are asked for one after the other
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
                dma4(resource(a_scale, a_scale_bytes), q * 256 + lane * 4, stage + Cfg::SA_AT + q * 256);
            } else {
                const int p = q - Cfg::NSA;          // 32 rows of the tile
                const int m = Cfg::DUAL ? p & 1 : 0;
                const uint8_t* from = m ? b_scale[1] : b_scale[0];
                dma4(resource(from, b_scale_bytes), (Cfg::DUAL ? p >> 1 : p) * 256 + lane * 4, stage + Cfg::SB_AT + p * 256);
            }
        }
        a_scale += static_cast<size_t>(op.R) * kMxRunBytes;
#pragma unroll
        for (int m = 0; m < (Cfg::DUAL ? 2 : 1); ++m) b_scale[m] += static_cast<size_t>(op.N) * kMxRunBytes;
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
    const int KT = mx_runs(op.K);
#pragma unroll
    for (int s = 0; s < S - 1; ++s)
        if (s < KT) loads.issue(op, s * Cfg::STAGE, s);
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
        if (kt + S - 1 < KT) loads.issue(op, (stage == 0 ? S - 1 : stage - 1) * Cfg::STAGE, kt + S - 1);
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

}  // namespace mx4
}  // namespace moe
