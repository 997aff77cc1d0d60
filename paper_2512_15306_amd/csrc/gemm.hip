// FP8 contraction with both operands contraction-contiguous ("TN"), its BF16 baseline, and the kernels for
// shapes no tuned tile divides.  The tile kernel itself is in gemm_tile.h, those of small problems in gemm_small.h.
#include "gemm_small.h"

namespace llmq {

void launch_gemm_generic(const uint8_t* A, int fmtA, int layout_a, const uint8_t* B, int fmtB, int layout_b, int64_t R, int64_t C,
                         int64_t T, const float* sA, const float* sB, void* c, int accumulate, unsigned* amax,
                         hipStream_t stream);

// BF16 operands, any shape: one output element per lane and trip, binary32 accumulation along t.
__global__ __launch_bounds__(256) void gemm_bf16_generic_kernel(
    const uint16_t* __restrict__ A, const uint16_t* __restrict__ B, uint16_t* __restrict__ C,
    int64_t R, int64_t Cn, int64_t T, int accumulate) {
    const int64_t n = R * Cn;
    for (int64_t idx = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; idx < n; idx += (int64_t)gridDim.x * blockDim.x) {
        const int64_t r = idx / Cn, c = idx - r * Cn;
        float acc = 0.0f;
        for (int64_t t = 0; t < T; ++t)
            acc = __builtin_fmaf(__uint_as_float((unsigned)A[r * T + t] << 16), __uint_as_float((unsigned)B[c * T + t] << 16), acc);
        if (accumulate) acc += __uint_as_float((unsigned)C[idx] << 16);
        C[idx] = __builtin_bit_cast(uint16_t, (__bf16)acc);
    }
}

__global__ void gemm_amax_reset_kernel(unsigned* amax_bits) {
    if (threadIdx.x == 0 && blockIdx.x == 0) *amax_bits = 0u;
}

// ---- host side: tile choice and launch

// Picks the wave tile NI x NJ (workgroup tile 64 NI x 64 NJ) that finishes soonest under a simple
// model: every CU works through its share of the tiles, a tile costs NI * NJ MFMA blocks per K step
// divided by the measured efficiency of that shape relative to 4 x 4 (smaller tiles read more LDS
// and L2 bytes per MFMA; 2 x 2 tiles fit two workgroups per CU, which hide each other's stalls).
TileChoice choose_tile(int64_t R, int64_t C, int64_t T, int num_cus, size_t scratch_bytes, bool bf16) {
    static const float eff[5][5] = {{0, 0, 0, 0, 0}, {0, 0, 0, 0, 0}, {0, 0, 0.90f, 0.74f, 0.77f},
                                    {0, 0, 0.74f, 0.70f, 0.83f}, {0, 0, 0.77f, 0.83f, 1.00f}};
    TileChoice best{0, 0};
    if (T % BK != 0 || T >= (1ll << 23)) return best;
    // Override for tests and tuning: LLMQ_GEMM_TILE=IxJ forces that wave tile where it divides the problem.
    if (const char* force = tuning_env("LLMQ_GEMM_TILE")) {
        const int ni = force[0] - '0', nj = force[0] && force[1] ? force[2] - '0' : 0;
        if (ni >= 2 && ni <= 4 && nj >= 2 && nj <= 4 && R % (64 * ni) == 0 && C % (64 * nj) == 0) return TileChoice{ni, nj};
    }
    // At most one 128 x 128 tile per CU: that tile, with four LDS stages, whatever the model says about larger ones (1024 x
    // 3072 x 3072: 14.6 us against 18.0 with 192 x 128 tiles; 128 x 9984 x 13184: 68 against 98).  Contractions long enough
    // for sharing out tiles keep the model's choice when there is scratch for it.
    if (R % 128 == 0 && C % 128 == 0 && (scratch_bytes == 0 || T / BK < 64) &&
        (R / 128) * (C / 128) <= resident_slots(num_cus, 2, 2) / 2)
        return TileChoice{2, 2};
    double best_cost = 0;
    for (int ni = 4; ni >= 2; --ni)
        for (int nj = 4; nj >= 2; --nj) {
            if (R % (64 * ni) != 0 || C % (64 * nj) != 0) continue;
            const int64_t tiles = (R / (64 * ni)) * (C / (64 * nj));
            if (tiles >= (1ll << 30)) continue;
            const int per_cu = (ni == 2 && nj == 2) ? 2 : 1;          // workgroups resident per CU
            const int64_t slots = resident_slots(num_cus, ni, nj);
            const int64_t rounds = (tiles + slots - 1) / slots;
            // two resident 2 x 2 workgroups overlap each other's prologue and epilogue, which pays most
            // when the contraction is short
            // (BF16 moves twice the bytes per product, which costs 128 x 128 tiles more and the 2 : 1 ones less.  Over 32 shapes
            // from 2560^3 to 16384 x 5120 these numbers' choice is 1.6 % behind the best tile on average and FP8's 4.2 %; they differ on
            // eleven.  The 128 x 128 tiles were slower then; 256 x 128 / 128 x 128 now, microseconds: 4096 x 5120 x 3072 118 / 120, x 4096 152 / 150, 8192 x 1024 x 4096
            // 55 / 60, 16384 x 1280 x 5120 185 / 193; and where they lose, 4096 x 5120 x 2048 84 / 82, 2560^3 40 / 38.  Where a larger tile is far ahead, 4096 x 5120 x 3072 90
            // and 16384 x 1280 x 5120 138 with 256 x 320, better_tile takes it.)
            const double e = per_cu == 2 ? (bf16 ? 0.66 : T <= 3072 ? 0.90 : 0.80) : bf16 && ni * nj == 8 ? 0.80 : eff[ni][nj];
            // a ragged last round may be shared out among all CUs (choose_split): the model's gain scales the cost
            const SplitChoice sc = choose_split((int)tiles, (int)(T / BK), (int)slots, ni, nj, scratch_bytes);
            const double cost = (double)rounds * per_cu * ni * nj / e * (sc.cost_us / sc.whole_cost_us);
            if (best.ni == 0 || cost < best_cost * 0.97) { best = {ni, nj}; best_cost = cost; }   // larger tile on near ties
        }
    return best;
}

// The choice of choose_tile as a plan, and what sharing out its last round of tiles saves.
struct WholePlan {
    TilePlan tile;
    SplitChoice split;
};
static WholePlan plan_whole(int64_t R, int64_t C, int64_t T, int num_cus, bool bf16, size_t scratch_bytes) {
    WholePlan p{{0, 0, kNoEdge}, {}};
    const TileChoice tc = choose_tile(R, C, T, num_cus, scratch_bytes, bf16);
    if (tc.ni == 0) return p;
    p.tile = {tc.ni, tc.nj, kNoEdge};
    p.split = choose_split((int)((R / (64 * tc.ni)) * (C / (64 * tc.nj))), (int)(T / BK), resident_slots(num_cus, tc.ni, tc.nj), tc.ni, tc.nj, scratch_bytes);
    return p;
}

TilePlan plan_tile(int64_t R, int64_t C, int64_t T, int num_cus, bool ta, bool tb, bool slabs_a, bool slabs_b, bool accumulate, bool with_amax, bool bf16,
                   size_t scratch_bytes) {
    WholePlan p = plan_whole(R, C, T, num_cus, bf16, ta || tb || bf16 ? 0 : scratch_bytes);
    if (p.tile.ni) {
        // better_tile prices whole tiles, so a tile of its choice is computed whole, scratch or not: gemm_scratch_bytes has nothing for it (1024 x 24320 x 8192,
        // where 256 x 256 tiles replace smaller ones).
        TilePlan tile = better_tile(R, C, T, num_cus, ta, tb, slabs_a, slabs_b, accumulate, p.tile, p.split.cost_us / p.split.whole_cost_us, p.split.n_groups > 0);
        tile.shares = p.split.n_groups > 0 && tile.ni == p.tile.ni && tile.nj == p.tile.nj && tile.edge == kNoEdge;
        return tile;
    }
    if (!ta || tb) {
        const EdgeChoice ec = choose_edge_tile(R, C, T, num_cus, ta, tb, slabs_a, slabs_b, accumulate, with_amax, bf16);
        p.tile = {ec.ni, ec.nj, ec.edge};
    }
    return better_tile(R, C, T, num_cus, ta, tb, slabs_a, slabs_b, accumulate, p.tile, 1.0);
}

// What a contraction of operands in rows or slabs takes: small tiles of `side`, or (0) the tile; the generic kernel if that has no size either.
struct RowsPlan {
    int side;
    TilePlan tile;
};
static RowsPlan plan_rows(int64_t R, int64_t C, int64_t T, int num_cus, bool slabs_a, bool slabs_b, bool accumulate, bool with_amax, bool bf16, size_t scratch_bytes) {
    // (an operand in slabs is addressed with 32-bit offsets from its first tile row, 0x7FFFFF00 being out of range)
    const int64_t lim = 0x7FFFFF00ll - ((int64_t)1 << 24);
    RowsPlan plan{0, {0, 0, kNoEdge}};
    if ((slabs_a && (T + 256) * R >= lim) || (slabs_b && (T + 256) * C >= lim)) return plan;
    double shared_us = 0.0;
    if (!bf16 && scratch_bytes && T >= 64 * BK && ((R + 127) / 128) * ((C + 127) / 128) <= num_cus) {       // (what the planner shares is that long)
        const WholePlan p = plan_whole(R, C, T, num_cus, false, scratch_bytes);
        if (p.tile.ni) shared_us = shared_tiles_us(p.split);
    }
    plan.side = takes_mini(R, C, T, slabs_a, slabs_b, accumulate, with_amax, bf16, num_cus, shared_us);
    if (plan.side == 0) plan.tile = plan_tile(R, C, T, num_cus, false, false, slabs_a, slabs_b, accumulate, with_amax, bf16, scratch_bytes);
    return plan;
}

template <int FA, int FB>
static void launch_mini(int side, const uint8_t* A, const uint8_t* B, int64_t R, int64_t C, int64_t T, const float* sA, const float* sB,
                        void* c, int accumulate, unsigned* amax, hipStream_t stream, bool slabs_a, bool slabs_b) {
    const int tiles_r = (int)((R + side - 1) / side), tiles = tiles_r * (int)((C + side - 1) / side), grid = (tiles + kXcds - 1) / kXcds * kXcds;
    auto launch = [&](auto kernel) {
        hipLaunchKernelGGL(kernel, dim3(grid), dim3(kGemmThreads), 0, stream, A, B, reinterpret_cast<uint16_t*>(c), (int)R, (int)C, (int)T, sA, sB, accumulate, amax,
                           slabs_a ? BK : (int)T, slabs_b ? BK : (int)T, slabs_a ? (int)(R * BK) : BK, slabs_b ? (int)(C * BK) : BK, tiles_r, tiles);
    };
    if (side == 32) launch(gemm_mini_kernel<FA, FB, 32>);
    else launch(gemm_mini_kernel<FA, FB, 64>);
}

template <int FA, int FB>
static void launch_one(const uint8_t* A, const uint8_t* B, int64_t R, int64_t C, int64_t T,
                       const float* sA, const float* sB, void* c, int accumulate, unsigned* amax,
                       hipStream_t stream, int num_cus, GemmScratch scratch, bool slabs_a = false, bool slabs_b = false) {
    const RowsPlan plan = plan_rows(R, C, T, num_cus, slabs_a, slabs_b, accumulate != 0, amax != nullptr, FA == kFmtBf16, scratch.ptr ? scratch.bytes : 0);
    const TilePlan tile = plan.tile;
    if (plan.side) { launch_mini<FA, FB>(plan.side, A, B, R, C, T, sA, sB, c, accumulate, amax, stream, slabs_a, slabs_b); return; }
    if (tile.ni && tile.edge == kNoEdge && launch_chosen_tile<FA, FB, false, false>(A, B, R, C, T, sA, sB, c, accumulate, amax, stream, num_cus, tile.shares ? scratch : GemmScratch{}, slabs_a, slabs_b, tile)) return;
    if (tile.ni && launch_edge_tile<FA, FB, false, false>(A, B, R, C, T, sA, sB, c, accumulate, amax, stream, num_cus, slabs_a, slabs_b, tile)) return;
    if constexpr (FA == kFmtBf16) {
        const int64_t n = R * C;
        int64_t blocks = (n + 255) / 256;
        if (blocks > 65536) blocks = 65536;
        hipLaunchKernelGGL(gemm_bf16_generic_kernel, dim3((unsigned)blocks), dim3(256), 0, stream,
                           reinterpret_cast<const uint16_t*>(A), reinterpret_cast<const uint16_t*>(B),
                           reinterpret_cast<uint16_t*>(c), R, C, T / 2, accumulate);
    } else {
        launch_gemm_generic(A, FA, slabs_a ? kLayoutSlabs : kLayoutRows, B, FB, slabs_b ? kLayoutSlabs : kLayoutRows, R, C, T, sA, sB, c,
                            accumulate, amax, stream);
    }
}

void launch_gemm_generic(const uint8_t* A, int fmtA, int ta, const uint8_t* B, int fmtB, int tb, int64_t R, int64_t C,
                         int64_t T, const float* sA, const float* sB, void* c, int accumulate, unsigned* amax,
                         hipStream_t stream) {
    dim3 grid((unsigned)((C + 31) / 32), (unsigned)((R + 31) / 32));
    uint16_t* out = reinterpret_cast<uint16_t*>(c);
    if (fmtA == 0 && fmtB == 0) hipLaunchKernelGGL((gemm_generic_kernel<0, 0>), grid, dim3(256), 0, stream, A, B, out, R, C, T, sA, sB, accumulate, amax, (int)ta, (int)tb);
    else if (fmtA == 1 && fmtB == 0) hipLaunchKernelGGL((gemm_generic_kernel<1, 0>), grid, dim3(256), 0, stream, A, B, out, R, C, T, sA, sB, accumulate, amax, (int)ta, (int)tb);
    else if (fmtA == 0 && fmtB == 1) hipLaunchKernelGGL((gemm_generic_kernel<0, 1>), grid, dim3(256), 0, stream, A, B, out, R, C, T, sA, sB, accumulate, amax, (int)ta, (int)tb);
    else hipLaunchKernelGGL((gemm_generic_kernel<1, 1>), grid, dim3(256), 0, stream, A, B, out, R, C, T, sA, sB, accumulate, amax, (int)ta, (int)tb);
}

void launch_gemm_amax_reset(unsigned* amax, hipStream_t stream) {
    hipLaunchKernelGGL(gemm_amax_reset_kernel, dim3(1), dim3(64), 0, stream, amax);
}

int launch_gemm_tn(const uint8_t* A, int fmtA, const uint8_t* B, int fmtB, int64_t R, int64_t C,
                   int64_t T, const float* d_scaleA, const float* d_scaleB, void* c_bf16,
                   int accumulate, float* d_amax_c, bool amax_is_zeroed, hipStream_t stream, int num_cus, GemmScratch scratch,
                   bool slabs_a, bool slabs_b) {
    unsigned* amax = reinterpret_cast<unsigned*>(d_amax_c);
    if (amax && !amax_is_zeroed) hipLaunchKernelGGL(gemm_amax_reset_kernel, dim3(1), dim3(64), 0, stream, amax);
    if (fmtA == 0 && fmtB == 0) launch_one<0, 0>(A, B, R, C, T, d_scaleA, d_scaleB, c_bf16, accumulate, amax, stream, num_cus, scratch, slabs_a, slabs_b);
    else if (fmtA == 1 && fmtB == 0) launch_one<1, 0>(A, B, R, C, T, d_scaleA, d_scaleB, c_bf16, accumulate, amax, stream, num_cus, scratch, slabs_a, slabs_b);
    else if (fmtA == 0 && fmtB == 1) launch_one<0, 1>(A, B, R, C, T, d_scaleA, d_scaleB, c_bf16, accumulate, amax, stream, num_cus, scratch, slabs_a, slabs_b);
    else launch_one<1, 1>(A, B, R, C, T, d_scaleA, d_scaleB, c_bf16, accumulate, amax, stream, num_cus, scratch, slabs_a, slabs_b);
    return hipGetLastError() == hipSuccess ? 0 : -6;
}

// Scratch a launch of this shape would use when given as much as it likes, with or without addition to the output and its absmax (0: every tile is
// computed whole).
size_t gemm_scratch_bytes(int64_t R, int64_t C, int64_t T, int num_cus) {
    const size_t unlimited = ~(size_t)0;
    const WholePlan p = plan_whole(R, C, T, num_cus, false, unlimited);
    if (p.tile.ni == 0 || p.split.n_groups == 0) return 0;
    const size_t bytes = p.split.slots * (size_t)(4 * 4096 * p.tile.ni * p.tile.nj);
    // shared out unless another kernel takes the shape: small tiles, whole larger ones (plan_tile: the same with addition and without)
    for (int with = 0; with < 4; ++with) {
        const RowsPlan plan = plan_rows(R, C, T, num_cus, false, false, (with & 1) != 0, (with & 2) != 0, false, unlimited);
        if (plan.side == 0) return plan.tile.shares ? bytes : 0;
    }
    return 0;
}

// Phase stamps of the 256 x 256 tile kernel (E4M3 x E4M3, contraction-contiguous operands): the same kernel with
// kProfile, which makes wave 0 of every workgroup record cycle and 100 MHz stamps of its phases, 16 words of 64 bits
// per workgroup id (see GemmTuning::kProfile).
template <bool IEEE>
struct GemmPhaseTuning : GemmTuning {
    static constexpr bool kProfile = true;
    static constexpr bool kIeeeMaximum = IEEE;
    static __device__ void record(float* buf, int block, int slot, long long value) {
        reinterpret_cast<long long*>(buf)[(size_t)block * 16 + slot] = value;
    }
};

int gemm_phase_stamp_blocks(int64_t R, int64_t C) { return (int)((((R / 256) * (C / 256) + kXcds - 1) / kXcds) * kXcds); }

int launch_gemm_phase_stamps(const uint8_t* A, const uint8_t* B, int64_t R, int64_t C, int64_t T, const float* sA,
                             const float* sB, void* c_bf16, float* d_amax_c, long long* stamps, int ieee_maximum,
                             hipStream_t stream, int num_cus) {
    const int tiles_r = (int)(R / 256), tiles_c = (int)(C / 256), nt = tiles_r * tiles_c;
    const int grid = gemm_phase_stamp_blocks(R, C);
    const int slots = resident_slots(num_cus, 4, 4);
    const int band = band_rows();
    const int share_b = band < tiles_r ? band : tiles_r, share_a = 4 < tiles_c ? 4 : tiles_c;
    const int next_stride = successor_stride(4, 4, nt, slots);
    SplitPlan plan{};
    plan.n_whole = nt;
    plan.partials = reinterpret_cast<float*>(stamps);
    unsigned* amax = reinterpret_cast<unsigned*>(d_amax_c);
    hipLaunchKernelGGL(gemm_amax_reset_kernel, dim3(1), dim3(64), 0, stream, amax);
    auto launch = [&](auto kernel) {
        hipLaunchKernelGGL(kernel, dim3(grid), dim3(kGemmThreads), 0, stream, A, B, reinterpret_cast<uint16_t*>(c_bf16),
                           (int)C, (int)T, sA, sB, amax, tiles_r, tiles_c, touch_ahead(), band, next_stride, (int)T, (int)T,
                           BK, BK, share_a, share_b, plan, (int)R, 0);
    };
    if (ieee_maximum) launch(gemm_tile_kernel<0, 0, 4, 4, false, GemmPhaseTuning<true>>);
    else launch(gemm_tile_kernel<0, 0, 4, 4, false, GemmPhaseTuning<false>>);
    return hipGetLastError() == hipSuccess ? 0 : -6;
}

// BF16 baseline: same tile kernels with the BF16 MFMA; T counts elements here, rows are 2 T bytes long.
int launch_gemm_bf16_tn(const void* A, const void* B, int64_t R, int64_t C, int64_t T, void* c_bf16,
                        int accumulate, hipStream_t stream, int num_cus) {
    launch_one<kFmtBf16, kFmtBf16>(reinterpret_cast<const uint8_t*>(A), reinterpret_cast<const uint8_t*>(B), R, C, 2 * T,
                                   nullptr, nullptr, c_bf16, accumulate, nullptr, stream, num_cus, GemmScratch{nullptr, 0});
    return hipGetLastError() == hipSuccess ? 0 : -6;
}

}  // namespace llmq
