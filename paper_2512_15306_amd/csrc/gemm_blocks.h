// The contraction of FP8 operands with a scale for each block of 128 contraction bytes (llmq_fp8_gemm_blocks).
//
//   C[r,c] = bf16( sum_t A[r,t] 2^(a[r, t/128] - 127) B[c,t] 2^(b[c, t/128] - 127) )
//
// The scales are powers of two because the matrix cores take those: v_mfma_scale_f32_16x16x128_f8f6f4 has an 8-bit exponent
// for every row and 32 contraction bytes of both operands, adds them to the exponents of the products and accumulates on in binary32, at the rate of
// the instruction without them.  Scales that are ordinary numbers would need a second set of accumulators, and a multiply-add of every output in every K step:
// 4 vector instructions behind each MFMA.  A product of a code and a power of two is exact, so nothing is rounded but the sums.
//
// The kernels are those of the tensor-wise contraction (gemm_tile.h, gemm_small.h) with the scales of a K step in two to four registers.  Where a row's
// block was 128 rows high, every row has a copy of its code: 1/128 of a byte per operand byte, and one form of operand instead of three.
#pragma once
#include "gemm_small.h"

namespace llmq {

struct GemmBlocksTuning : GemmTuning { static constexpr bool kBlockScales = true; };
struct GemmBlocksDeepTuning : GemmDeepTuning { static constexpr bool kBlockScales = true; };
struct GemmBlocksDeepWideTuning : GemmDeepWideTuning { static constexpr bool kBlockScales = true; };

struct BlocksOperands {
    const uint8_t *A, *sA, *B, *sB;
    int64_t R, C, T;
    void* c;
    int accumulate;
    unsigned* amax;
};

template <int FA, int FB, int NI, int NJ, int EDGE>
static void launch_blocks_tile(const BlocksOperands& p, hipStream_t stream, int num_cus) {
    const int tiles_r = (int)((p.R + 64 * NI - 1) / (64 * NI)), tiles_c = (int)((p.C + 64 * NJ - 1) / (64 * NJ));
    SplitPlan plan{};
    plan.n_whole = tiles_r * tiles_c;
    const int grid = ((plan.n_whole + kXcds - 1) / kXcds) * kXcds, slots = resident_slots(num_cus, NI, NJ);
    const int touch = (NI == 2 && NJ == 2) ? touch_ahead_pair() : touch_ahead();
    const int band = band_rows(), share_b = band < tiles_r ? band : tiles_r, share_a = 4 < tiles_c ? 4 : tiles_c;
    const int next_stride = EDGE == kNoEdge ? successor_stride(NI, NJ, plan.n_whole, slots) : 0;
    auto launch = [&](auto kernel, int threads = kGemmThreads) {
        hipLaunchKernelGGL(kernel, dim3(grid), dim3(threads), 0, stream, p.A, p.B, reinterpret_cast<uint16_t*>(p.c), (int)p.C, (int)p.T,
                           reinterpret_cast<const float*>(p.sA), reinterpret_cast<const float*>(p.sB), p.amax, tiles_r, tiles_c, touch, band, next_stride,
                           (int)p.T, (int)p.T, BK, BK, share_a, share_b, plan, (int)p.R, p.accumulate);
    };
    // (guarded tiles add to the output by a run-time flag)
    auto launch_form = [&](auto tuning, int threads = kGemmThreads) {
        typedef decltype(tuning) V;
        if constexpr (EDGE == kNoEdge) {
            if (!p.accumulate) { launch(gemm_tile_kernel<FA, FB, NI, NJ, false, V>, threads); return; }
        }
        launch(gemm_tile_kernel<FA, FB, NI, NJ, true, V, false, false, kWholeTiles, EDGE>, threads);
    };
    if constexpr (NI == 2 && NJ == 2 && EDGE != kEdgeUnaligned) {
        if (deep_stages(plan.n_whole, slots)) {
            if (deep_takes_eight_waves((p.T + BK - 1) / BK, false)) launch_form(GemmBlocksDeepWideTuning{}, 2 * kGemmThreads);
            else launch_form(GemmBlocksDeepTuning{});
            return;
        }
    }
    launch_form(GemmBlocksTuning{});
}

// What a contraction takes: small tiles of `side`, else the tile, else the generic kernel (tile.ni == 0).
struct BlocksPlan {
    int side;
    TilePlan tile;
};

// Launches the kernel of the plan; gemm_blocks_*.hip instantiate it for a pair of formats each.
template <int FA, int FB>
void launch_blocks(const BlocksOperands& p, const BlocksPlan& plan, hipStream_t stream, int num_cus) {
    if (plan.side) {
        const int side = plan.side, tiles_r = (int)((p.R + side - 1) / side), tiles = tiles_r * (int)((p.C + side - 1) / side), grid = (tiles + kXcds - 1) / kXcds * kXcds;
        auto launch = [&](auto kernel) {
            hipLaunchKernelGGL(kernel, dim3(grid), dim3(kGemmThreads), 0, stream, p.A, p.B, reinterpret_cast<uint16_t*>(p.c), (int)p.R, (int)p.C, (int)p.T,
                               reinterpret_cast<const float*>(p.sA), reinterpret_cast<const float*>(p.sB), p.accumulate, p.amax, (int)p.T, (int)p.T, BK, BK, tiles_r, tiles);
        };
        if (side == 32) launch(gemm_mini_kernel<FA, FB, 32, true>);
        else launch(gemm_mini_kernel<FA, FB, 64, true>);
        return;
    }
#define LLMQ_BLOCKS_CASE(I, J, KIND)                                      \
    case KIND * 64 + I * 8 + J:                                           \
        launch_blocks_tile<FA, FB, I, J, KIND>(p, stream, num_cus);       \
        return;
    switch (plan.tile.edge * 64 + plan.tile.ni * 8 + plan.tile.nj) {
        LLMQ_BLOCKS_CASE(4, 4, kNoEdge) LLMQ_BLOCKS_CASE(4, 3, kNoEdge) LLMQ_BLOCKS_CASE(4, 2, kNoEdge)
        LLMQ_BLOCKS_CASE(3, 4, kNoEdge) LLMQ_BLOCKS_CASE(3, 3, kNoEdge) LLMQ_BLOCKS_CASE(3, 2, kNoEdge)
        LLMQ_BLOCKS_CASE(2, 4, kNoEdge) LLMQ_BLOCKS_CASE(2, 3, kNoEdge) LLMQ_BLOCKS_CASE(2, 2, kNoEdge)
        LLMQ_BLOCKS_CASE(4, 4, kEdge) LLMQ_BLOCKS_CASE(4, 2, kEdge) LLMQ_BLOCKS_CASE(3, 4, kEdge) LLMQ_BLOCKS_CASE(2, 4, kEdge) LLMQ_BLOCKS_CASE(2, 2, kEdge)
        LLMQ_BLOCKS_CASE(4, 2, kEdgeUnaligned) LLMQ_BLOCKS_CASE(2, 4, kEdgeUnaligned) LLMQ_BLOCKS_CASE(2, 2, kEdgeUnaligned)
        default: break;
    }
#undef LLMQ_BLOCKS_CASE
    // one wave for each 16 x 16 outputs, columns along the grid's first dimension; a launch has fewer than 2^24 workgroups, and 65535 of the second
    const int64_t grid_c = (p.C + 31) / 32, grid_r = (p.R + 31) / 32;
    hipLaunchKernelGGL((gemm_generic_kernel<FA, FB, true>), dim3((unsigned)grid_c, (unsigned)grid_r), dim3(256), 0, stream, p.A, p.B,
                       reinterpret_cast<uint16_t*>(p.c), p.R, p.C, p.T, reinterpret_cast<const float*>(p.sA), reinterpret_cast<const float*>(p.sB), p.accumulate, p.amax, kLayoutRows, kLayoutRows);
}
extern template void launch_blocks<0, 0>(const BlocksOperands&, const BlocksPlan&, hipStream_t, int);
extern template void launch_blocks<1, 0>(const BlocksOperands&, const BlocksPlan&, hipStream_t, int);
extern template void launch_blocks<0, 1>(const BlocksOperands&, const BlocksPlan&, hipStream_t, int);
extern template void launch_blocks<1, 1>(const BlocksOperands&, const BlocksPlan&, hipStream_t, int);

}  // namespace llmq
