// The contraction of FP8 operands with a scale for each block of 128 contraction bytes (llmq_fp8_gemm_blocks).
//
//   C[r,c] = bf16( sum_t A[r,t] 2^(a[r, t/128] - 127) B[c,t] 2^(b[c, t/128] - 127) )
//
// The scales are powers of two because the matrix cores take those: v_mfma_scale_f32_16x16x128_f8f6f4 has an 8-bit exponent
// for every row and 32 contraction bytes of both operands, adds them to the exponents of the products and accumulates on in binary32, at the rate of
// the instruction without them.  Scales that are ordinary numbers would need a second set of accumulators, and a multiply-add of every output in every K step:
// 4 vector instructions behind each MFMA.  A product of a code and a power of two is exact, so what is lost is lost in the sums: inside a K step, whose 128 products the instruction aligns to the largest (up to 2^-12.3 of the
// sum of their magnitudes was seen), and by binary32 from step to step.
//
// 8192 x 4608 x 3584 in E4M3: 118 us, 2.3 PFLOP/s (107 to 115 with one scale an operand); 3584 x 18944 x 8192, E5M2 by E4M3, added to the output: 430 us, 2.6 PFLOP/s; bound by the power
// that the matrix instructions and the operands' way to them take.
//
// The kernels are those of the tensor-wise contraction (gemm_tile.h, gemm_small.h) with the scales of a K step in two to four registers.  Where a row's
// block was 128 rows high, every row has a copy of its code: 1/128 of a byte per operand byte, and one form of operand instead of three.
#pragma once
#include "gemm_small.h"

namespace llmq {

struct GemmBlocksTuning : GemmTuning { static constexpr bool kBlockScales = true; };
struct GemmBlocksDeepTuning : GemmDeepTuning { static constexpr bool kBlockScales = true; };
struct GemmBlocksDeepWideTuning : GemmDeepWideTuning { static constexpr bool kBlockScales = true; };

// R x C: the whole contraction, whose scales and output rows are laid out by them; rows x cols: the part of it that the pointers begin (all of it, except for strips)
struct BlocksOperands {
    const uint8_t *A, *sA, *B, *sB;
    int64_t R, C, T, rows, cols;
    void* c;
    int accumulate;
    unsigned* amax;
};

template <int FA, int FB, int NI, int NJ, int EDGE>
static void launch_blocks_tile(const BlocksOperands& p, hipStream_t stream, int num_cus) {
    const int tiles_r = (int)((p.rows + 64 * NI - 1) / (64 * NI)), tiles_c = (int)((p.cols + 64 * NJ - 1) / (64 * NJ));
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

// ---- Few rows: 16 RB of them (decoding, one row a sequence), or groups of so many along the grid's second dimension.
//
// What there is to do is to read B once (for every group).  The small tiles have a workgroup for every 32 columns, whose waves meet at two barriers every four K steps; here a workgroup has
// 16 CB columns, its four waves take every fourth K step each, with LDS of their own, and meet once, to add their sums in the order of the waves.  A wave keeps
// the operands of four of its steps on their way (four slots of LDS): slabs of 16 rows x 128 bytes with eight lanes to a row, as in the tile kernel, and for the same reason
// through LDS: loads straight into the layout of the matrix instruction have 16 rows side by side, which the memory pipeline takes 16 bytes at a time (80 cycles for a load of
// 1 KB; 16 x 4608 x 3584 10 us with two such loads to an operand and step).
// ALIGNED: rows are whole 16-byte chunks and go straight to LDS; otherwise through registers, from any address.
constexpr int kFewWaves = 4, kFewSlots = 4;
template <int FA, int FB, int RB, int CB, bool ALIGNED>
__global__ __launch_bounds__(kFewWaves * kWave) void gemm_blocks_few_kernel(const uint8_t* __restrict__ A, const uint8_t* __restrict__ sA, const uint8_t* __restrict__ B,
                                                                          const uint8_t* __restrict__ sB, uint16_t* __restrict__ C, int R, int Cn, int T, int accumulate,
                                                                          unsigned* __restrict__ amax_bits) {
    constexpr int kRows = 16 * (RB + CB), kSlot = kRows * BK, kLoads = kRows / 8, kOutOfRange = 0x7FFFFF00;
    // one LDS object per slot, which the compiler tells apart (see the tile kernel)
    __shared__ __attribute__((aligned(1024))) uint8_t s_0[kFewWaves * kSlot];
    __shared__ __attribute__((aligned(1024))) uint8_t s_1[kFewWaves * kSlot];
    __shared__ __attribute__((aligned(1024))) uint8_t s_2[kFewWaves * kSlot];
    __shared__ __attribute__((aligned(1024))) uint8_t s_3[kFewWaves * kSlot];
    const int lane = threadIdx.x & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int r0 = (int)blockIdx.y * (16 * RB), c0 = (int)blockIdx.x * (16 * CB), steps = (T + BK - 1) / BK, mine = (steps - wave + kFewWaves - 1) / kFewWaves;      // steps wave, wave + 4, ...
    const int rows_a = R - r0 < 16 * RB ? R - r0 : 16 * RB, rows_b = Cn - c0 < 16 * CB ? Cn - c0 : 16 * CB;
    const uint8_t *const a0 = A + (int64_t)r0 * T, *const b0 = B + (int64_t)c0 * T;
    const __amdgpu_buffer_rsrc_t rsA = make_rsrc(a0, (unsigned)((int64_t)rows_a * T)), rsB = make_rsrc(b0, (unsigned)((int64_t)rows_b * T));
    const int pitchA = (R + 127) & ~127, pitchB = (Cn + 127) & ~127;
    const __amdgpu_buffer_rsrc_t rsSA = make_rsrc(sA, (unsigned)(steps * pitchA)), rsSB = make_rsrc(sB, (unsigned)(steps * pitchB));
    int code_a[RB], code_b[CB];
#pragma unroll
    for (int i = 0; i < RB; ++i) code_a[i] = (int)block_scale_offset(r0 + 16 * i + (lane & 15), 0, R);
#pragma unroll
    for (int j = 0; j < CB; ++j) code_b[j] = (int)block_scale_offset(c0 + 16 * j + (lane & 15), 0, Cn);
    // a wave's n-th step in a slot: slabs of A, then of B, load p rows 8 p .. of them
    struct Codes { int a[RB], b[CB]; };
    struct Chunks { v4u c[ALIGNED ? 1 : kLoads]; };
    Codes codes[kFewSlots];
    Chunks chunks[kFewSlots];
    const int ld_row = lane >> 3;
    auto request = [&](uint8_t* slot, int n, Codes& e, Chunks& held) __attribute__((always_inline)) {
        const int step = wave + n * kFewWaves;
        const bool there = n < mine;
#pragma unroll
        for (int i = 0; i < RB; ++i) e.a[i] = (int)(unsigned char)__builtin_amdgcn_raw_buffer_load_b8(rsSA, code_a[i], there ? step * pitchA : kOutOfRange, 0);
#pragma unroll
        for (int j = 0; j < CB; ++j) e.b[j] = (int)(unsigned char)__builtin_amdgcn_raw_buffer_load_b8(rsSB, code_b[j], there ? step * pitchB : kOutOfRange, 0);
        __builtin_amdgcn_sched_barrier(0);
        static_for<kLoads>([&](auto piece) {
            constexpr int p = decltype(piece)::value;
            constexpr bool of_a = p < 2 * RB;
            constexpr int row0 = 8 * (of_a ? p : p - 2 * RB);
            const int row = row0 + ld_row, k = step * BK + (((lane & 7) ^ row_swizzle(row & 15)) << 4);
            if constexpr (ALIGNED) {
                // (T % 16 == 0: a chunk exists or not; rows behind the operand lie outside the buffer)
                __builtin_amdgcn_raw_ptr_buffer_load_lds(of_a ? rsA : rsB, (lds_void*)(slot + wave * kSlot + p * 8 * BK), 16, there && k < T ? row * T + k : kOutOfRange, 0, 0, 0);
            } else {
                const int rows = of_a ? rows_a : rows_b;
                held.c[p] = v4u{0, 0, 0, 0};
                if (there && row < rows) {
                    const uint8_t* src = (of_a ? a0 : b0) + (int64_t)row * T + k;
                    if (k + 16 <= T) held.c[p] = *reinterpret_cast<const v4u_any*>(src);
                    else held.c[p] = load16_upto(src, T - k);
                }
            }
        });
        __builtin_amdgcn_sched_barrier(0);
    };
    const int fr_row = lane & 15, fr_q = lane >> 4, swz = row_swizzle(fr_row);
    const int ch0 = ((fr_q * 2) ^ swz) << 4, ch1 = ((fr_q * 2 + 1) ^ swz) << 4;
    v4f acc[RB][CB];
#pragma unroll
    for (int i = 0; i < RB; ++i)
#pragma unroll
        for (int j = 0; j < CB; ++j) acc[i][j] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
    // LDS runs a wave's accesses in order, and the direct loads that follow are requested behind the wait for the reads
    // behind: steps requested after this one.  The last steps request none, whose codes would be no use to anybody and dropped by the compiler, but counted here.
    auto multiply = [&](uint8_t* slot, int n, Codes& e, Chunks& held, auto behind, auto more) __attribute__((always_inline)) {
        uint8_t* const slab = slot + wave * kSlot;
        if constexpr (ALIGNED) {
            wait_vmcnt<decltype(behind)::value * (kLoads + RB + CB)>();
        } else {
            static_for<kLoads>([&](auto piece) { *reinterpret_cast<v4u*>(slab + decltype(piece)::value * 8 * BK + lane * 16) = held.c[decltype(piece)::value]; });
        }
        auto fragment = [&](int first_row) -> v8i {
            const uint8_t* p = slab + (first_row + fr_row) * BK;
            const v4i lo = *reinterpret_cast<const v4i*>(p + ch0), hi = *reinterpret_cast<const v4i*>(p + ch1);
            return v8i{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
        };
        v8i a[RB], b[CB];
#pragma unroll
        for (int i = 0; i < RB; ++i) a[i] = fragment(16 * i);
#pragma unroll
        for (int j = 0; j < CB; ++j) b[j] = fragment(16 * (RB + j));
        const Codes now = e;
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < RB; ++i)
#pragma unroll
            for (int j = 0; j < CB; ++j) acc[i][j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(b[j], a[i], acc[i][j], FB, FA, 0, now.b[j], 0, now.a[i]);
        __builtin_amdgcn_sched_barrier(0);
        if constexpr (decltype(more)::value) request(slot, n + kFewSlots, e, held);
    };
    request(s_0, 0, codes[0], chunks[0]);
    request(s_1, 1, codes[1], chunks[1]);
    request(s_2, 2, codes[2], chunks[2]);
    request(s_3, 3, codes[3], chunks[3]);
    int n = 0;
    for (; n + 3 < mine; n += 4) {
        multiply(s_0, n, codes[0], chunks[0], IntTag<3>{}, BoolTag<true>{});
        multiply(s_1, n + 1, codes[1], chunks[1], IntTag<3>{}, BoolTag<true>{});
        multiply(s_2, n + 2, codes[2], chunks[2], IntTag<3>{}, BoolTag<true>{});
        multiply(s_3, n + 3, codes[3], chunks[3], IntTag<3>{}, BoolTag<true>{});
    }
    if (n < mine) multiply(s_0, n, codes[0], chunks[0], IntTag<3>{}, BoolTag<false>{});
    if (n + 1 < mine) multiply(s_1, n + 1, codes[1], chunks[1], IntTag<2>{}, BoolTag<false>{});
    if (n + 2 < mine) multiply(s_2, n + 2, codes[2], chunks[2], IntTag<1>{}, BoolTag<false>{});
    wait_vmcnt<0>();                             // nothing lands in LDS any more
    __syncthreads();
    v4f* const s_sum = reinterpret_cast<v4f*>(s_0);                          // [wave][block][lane]
    static_assert(RB * CB * kWave * sizeof(v4f) <= (size_t)kSlot, "the sums of a wave fit its slot");
#pragma unroll
    for (int i = 0; i < RB; ++i)
#pragma unroll
        for (int j = 0; j < CB; ++j) s_sum[(wave * (RB * CB) + i * CB + j) * kWave + lane] = acc[i][j];
    __syncthreads();
    unsigned mag = 0;
    // a wave finishes every fourth block
    for (int block = wave; block < RB * CB; block += kFewWaves) {
        v4f y = s_sum[block * kWave + lane];
#pragma unroll
        for (int w = 1; w < kFewWaves; ++w) y += s_sum[(w * (RB * CB) + block) * kWave + lane];
        const int r = r0 + 16 * (block / CB) + (lane & 15), c = c0 + 16 * (block % CB) + (lane >> 4) * 4, left = Cn - c;
        if (r >= R || left <= 0) continue;
        uint16_t* dst = C + (int64_t)r * Cn + c;
        if (Cn % 4 == 0) {
            if (accumulate) {
                const v2u o = *reinterpret_cast<const v2u*>(dst);
                y[0] += __uint_as_float(o[0] << 16), y[1] += __uint_as_float(o[0] & 0xFFFF0000u), y[2] += __uint_as_float(o[1] << 16), y[3] += __uint_as_float(o[1] & 0xFFFF0000u);
            }
            const v2u out = __builtin_bit_cast(v2u, __builtin_convertvector(y, bf16x4));
            mag = pk_max_mag(pk_max_mag(mag, out[0]), out[1]);
            *reinterpret_cast<v2u*>(dst) = out;
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (e < left) {
                    const float v = accumulate ? y[e] + __uint_as_float((unsigned)dst[e] << 16) : y[e];
                    const unsigned bits = __builtin_bit_cast(uint16_t, (__bf16)v);
                    dst[e] = (uint16_t)bits;
                    mag = pk_max_mag(mag, bits);
                }
        }
    }
    if (amax_bits) {
        mag = wave_max_u32((mag & 0xFFFFu) > (mag >> 16) ? mag & 0xFFFFu : mag >> 16);
        const unsigned bits = amax_bits_from_bf16_mag(mag);
        if (lane == 0 && bits > __hip_atomic_load(amax_bits, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT)) atomicMax(amax_bits, bits);
    }
}

template <int FA, int FB, int RB, int CB>
static void launch_blocks_few(const BlocksOperands& p, hipStream_t stream) {
    auto launch = [&](auto kernel) {
        hipLaunchKernelGGL(kernel, dim3((unsigned)((p.C + 16 * CB - 1) / (16 * CB)), (unsigned)((p.R + 16 * RB - 1) / (16 * RB))), dim3(kFewWaves * kWave), 0, stream, p.A, p.sA, p.B, p.sB, reinterpret_cast<uint16_t*>(p.c), (int)p.R, (int)p.C,
                           (int)p.T, p.accumulate, p.amax);
    };
    if (p.T % 16 == 0) launch(gemm_blocks_few_kernel<FA, FB, RB, CB, true>);
    else if constexpr (CB == 1) launch(gemm_blocks_few_kernel<FA, FB, RB, CB, false>);
}

// What a contraction takes: the kernel for few rows, else small tiles of `side`, else the tile, else the generic kernel (tile.ni == 0).
// strip_rows / strip_cols: so many of the last rows or columns are a launch of their own, of whole `strip` tiles.
struct BlocksPlan {
    bool few;
    int side;
    TilePlan tile;
    int64_t strip_rows, strip_cols;
    TilePlan strip;
};

// The tiles, the small tiles and the generic kernel add in one order and give the same bytes; the kernel for few rows adds in another.
// Launches the kernel of the plan; gemm_blocks_*.hip instantiate it for a pair of formats each.
template <int FA, int FB>
void launch_blocks(const BlocksOperands& p, const BlocksPlan& plan, hipStream_t stream, int num_cus) {
    if (plan.strip_rows || plan.strip_cols) {
        // (whole tiles from rows and columns that are multiples of 128 on, so the strip's scales are the rest of each K step's)
        const int64_t r = plan.strip_rows ? p.R - plan.strip_rows : 0, c = plan.strip_cols ? p.C - plan.strip_cols : 0;
        BlocksOperands first = p, strip = p;
        if (r) first.rows = r, strip.rows = plan.strip_rows;
        if (c) first.cols = c, strip.cols = plan.strip_cols;
        strip.A += r * p.T, strip.sA += r, strip.B += c * p.T, strip.sB += c, strip.c = static_cast<uint16_t*>(p.c) + r * p.C + c;
        launch_blocks<FA, FB>(first, BlocksPlan{false, 0, plan.tile, 0, 0, {}}, stream, num_cus);
        launch_blocks<FA, FB>(strip, BlocksPlan{false, 0, plan.strip, 0, 0, {}}, stream, num_cus);
        return;
    }
    if (plan.few) {
        // Two blocks of columns to a workgroup read A half as often; where that leaves half of the CUs without one, or chunks go through registers (twice as many of them), one.
        // R x C x T, one / two, microseconds: 16 x 4608 x 3584 6.9 / 5.8, 26 x 5227 x 11488 22.2 / 16.3;  20 x 3492 x 16864 17.9 / 22.5, 5 x 2589 x 4720 6.6 / 7.9;
        // 9 x 5305 x 4643 17.0 / 24.0
        const bool two = p.T % 16 == 0 && (p.C + 31) / 32 >= num_cus / 2;
        if (p.R <= 16) two ? launch_blocks_few<FA, FB, 1, 2>(p, stream) : launch_blocks_few<FA, FB, 1, 1>(p, stream);
        else two ? launch_blocks_few<FA, FB, 2, 2>(p, stream) : launch_blocks_few<FA, FB, 2, 1>(p, stream);
        return;
    }
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
        LLMQ_BLOCKS_CASE(4, 4, kEdge) LLMQ_BLOCKS_CASE(4, 2, kEdge) LLMQ_BLOCKS_CASE(3, 4, kEdge) LLMQ_BLOCKS_CASE(3, 2, kEdge) LLMQ_BLOCKS_CASE(2, 4, kEdge) LLMQ_BLOCKS_CASE(2, 2, kEdge)
        LLMQ_BLOCKS_CASE(4, 2, kEdgeUnaligned) LLMQ_BLOCKS_CASE(2, 4, kEdgeUnaligned) LLMQ_BLOCKS_CASE(2, 2, kEdgeUnaligned)
        default: break;
    }
#undef LLMQ_BLOCKS_CASE
    // one wave for each 16 x 16 outputs, columns along the grid's first dimension; a launch has fewer than 2^24 workgroups, and 65536 along the second (R < 2^21)
    const int64_t grid_c = (p.C + 31) / 32, grid_r = (p.R + 31) / 32;
    hipLaunchKernelGGL((gemm_generic_kernel<FA, FB, true>), dim3((unsigned)grid_c, (unsigned)grid_r), dim3(256), 0, stream, p.A, p.B,
                       reinterpret_cast<uint16_t*>(p.c), p.R, p.C, p.T, reinterpret_cast<const float*>(p.sA), reinterpret_cast<const float*>(p.sB), p.accumulate, p.amax, kLayoutRows, kLayoutRows);
}
extern template void launch_blocks<0, 0>(const BlocksOperands&, const BlocksPlan&, hipStream_t, int);
extern template void launch_blocks<1, 0>(const BlocksOperands&, const BlocksPlan&, hipStream_t, int);
extern template void launch_blocks<0, 1>(const BlocksOperands&, const BlocksPlan&, hipStream_t, int);
extern template void launch_blocks<1, 1>(const BlocksOperands&, const BlocksPlan&, hipStream_t, int);

}  // namespace llmq
