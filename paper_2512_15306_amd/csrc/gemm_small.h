// Kernels of the contraction for small problems: the generic one (any shape) and tiles of 64 x 64 or 32 x 32 outputs.
#pragma once
#include "gemm_tile.h"

namespace llmq {

// Codes of block scales of an operand [rows, T]: K step by K step, 128 rows at a time, row r of them at 8 (r % 16) + r / 16.
__host__ __device__ inline int64_t block_scale_offset(int64_t row, int64_t step, int64_t rows) {
    return step * ((rows + 127) & ~(int64_t)127) + (row & ~(int64_t)127) + 8 * (row & 15) + ((row >> 4) & 7);
}

// ---- generic kernel: one wavefront per 16x16 outputs, v_mfma_f32_16x16x128_f8f6f4, guarded loads.
// ta / tb: the operand's OperandLayout; the bytes of a T-major operand ([T, R] or [T, Cn]) are gathered one by one.
// BLOCKS: d_sA / d_sB are the codes of scales for each block of 128 contraction bytes (block_scale_offset).
template <int FA, int FB, bool BLOCKS = false>
__global__ __launch_bounds__(256) void gemm_generic_kernel(
    const uint8_t* __restrict__ A, const uint8_t* __restrict__ B, uint16_t* __restrict__ C,
    int64_t R, int64_t Cn, int64_t T, const float* __restrict__ d_sA, const float* __restrict__ d_sB,
    int accumulate, unsigned* __restrict__ amax_bits, int ta, int tb) {
    const int lane = threadIdx.x & (kWave - 1);
    const int wave = threadIdx.x / kWave;
    const int64_t r0 = ((int64_t)blockIdx.y * 2 + (wave >> 1)) * 16;
    const int64_t c0 = ((int64_t)blockIdx.x * 2 + (wave & 1)) * 16;
    const int64_t ar = r0 + (lane & 15), bc = c0 + (lane & 15);
    const bool a_ok = ar < R, b_ok = bc < Cn;
    const bool vec_ok = (T % 16) == 0;
    auto load32 = [&](const uint8_t* base, bool ok, int64_t row, int64_t k, int tmajor, int64_t ld) -> v8i {
        v8i v = {0, 0, 0, 0, 0, 0, 0, 0};
        if (!ok || k >= T) return v;
        if (tmajor == kLayoutSlabs) {                 // 32 contiguous bytes of the row's K step (T % 128 == 0)
            const uint8_t* p = base + (k >> 7) * (ld * 128) + row * 128 + (k & 127);
            v4i lo = *reinterpret_cast<const v4i*>(p), hi = *reinterpret_cast<const v4i*>(p + 16);
            return v8i{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
        }
        if (tmajor) {
            for (int w = 0; w < 8; ++w) {
                unsigned word = 0;
                for (int e = 0; e < 4; ++e) {
                    int64_t kk = k + w * 4 + e;
                    if (kk < T) word |= (unsigned)base[kk * ld + row] << (8 * e);
                }
                v[w] = (int)word;
            }
            return v;
        }
        const uint8_t* p = base + row * T + k;
        if (vec_ok && k + 32 <= T) {
            v4i lo = *reinterpret_cast<const v4i*>(p), hi = *reinterpret_cast<const v4i*>(p + 16);
            return v8i{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
        }
        for (int w = 0; w < 8; ++w) {
            unsigned word = 0;
            for (int e = 0; e < 4; ++e) {
                int64_t kk = k + w * 4 + e;
                if (kk < T) word |= (unsigned)p[w * 4 + e] << (8 * e);   // beyond T: code 0x00 = +0
            }
            v[w] = (int)word;
        }
        return v;
    };
    v4f acc = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int64_t k0 = 0; k0 < T; k0 += 128) {
        const int64_t k = k0 + (lane >> 4) * 32;
        v8i a = load32(A, a_ok, ar, k, ta, R);
        v8i b = load32(B, b_ok, bc, k, tb, Cn);
        if constexpr (BLOCKS) {
            const int sa = a_ok ? reinterpret_cast<const uint8_t*>(d_sA)[block_scale_offset(ar, k0 >> 7, R)] : 0, sb = b_ok ? reinterpret_cast<const uint8_t*>(d_sB)[block_scale_offset(bc, k0 >> 7, Cn)] : 0;
            acc = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(b, a, acc, FB, FA, 0, sb, 0, sa);
        } else {
            acc = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(b, a, acc, FB, FA, 0, 0, 0, 0);
        }
    }
    // lane holds row r0 + lane % 16, columns c0 + 4 * (lane / 16) + 0..3
    // de-scaled as the tile kernels do it, so that the same sums give the same bytes whichever kernel ran
    const float inv_a = BLOCKS ? 1.0f : 1.0f / *d_sA, inv_b = BLOCKS ? 1.0f : 1.0f / *d_sB, inv_ab = inv_a * inv_b;
    const bool one_mul = inv_ab >= 1.17549435e-38f && inv_ab <= 3.402823466e+38f;
    const float m1 = one_mul ? inv_ab : inv_a, m2 = one_mul ? 1.0f : inv_b;
    unsigned mag = 0;
    const int64_t r = r0 + (lane & 15);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const int64_t c = c0 + (lane >> 4) * 4 + e;
        if (r < R && c < Cn) {
            float y = acc[e] * m1 * m2;
            uint16_t* dst = C + r * Cn + c;
            if (accumulate) y += __uint_as_float((unsigned)*dst << 16);
            __bf16 o = (__bf16)y;
            unsigned bits = __builtin_bit_cast(uint16_t, o);
            *dst = (uint16_t)bits;
            bits &= 0x7FFFu;
            mag = mag > bits ? mag : bits;
        }
    }
    if (amax_bits) {
        mag = wave_max_u32(mag);
        if (lane == 0) atomicMax(amax_bits, amax_bits_from_bf16_mag(mag));
    }
}

// ---- Few outputs: tiles of 64 x 64 or 32 x 32.
//
// What a CU reads per K step sets the pace of a problem that has fewer tiles than the chip has CUs: a 128 x 128 tile takes 32 KB and
// 0.29 us, and the rest of the chip looks on.  Here a workgroup of four waves (2 x 2) has a tile of SIDE x SIDE, 16 or 8 KB a
// step.  Four K steps make a stage: one wait and two barriers for all four, and 64 (SIDE 64: two stages) or 96 KB (SIDE 32: four) on
// their way while one is multiplied.  Slabs, swizzle and fragments are those of the tile kernel; the sums have its order, so the bytes are
// the same.  Operands in rows of whole 16-byte chunks, or in slabs; what lies behind an operand or the end of a row arrives
// as zeros (offsets beyond the buffer's range).
constexpr int kMiniSteps = 4;                                            // K steps of a stage
// BLOCKS: d_sA / d_sB are the codes of scales for each block of 128 contraction bytes.  A stage's codes are requested with its slabs, a register for
// each K step and operand: the four bytes of it are the lane's row of four neighbouring blocks of 16 rows, the wave's among them.
template <int FA, int FB, int SIDE, bool BLOCKS = false>
__global__ __launch_bounds__(kGemmThreads, 1) void gemm_mini_kernel(
    const uint8_t* __restrict__ A, const uint8_t* __restrict__ B, uint16_t* __restrict__ C, int R, int Cn, int T,
    const float* __restrict__ d_sA, const float* __restrict__ d_sB, int accumulate, unsigned* __restrict__ amax_bits, int ldA, int ldB, int ksA, int ksB,
    int tiles_r, int n_tiles) {
    constexpr int kOutOfRange = 0x7FFFFF00;
    constexpr int kSlab = SIDE * BK, kOperand = kMiniSteps * kSlab;      // bytes of one operand in a K step, in a stage
    constexpr int ST = SIDE == 64 ? 2 : 4, NB = SIDE / 32;               // stages; blocks of 16 x 16 per wave and side
    // one LDS object per stage and operand or per stage, which the compiler tells apart (see the tile kernel)
    __shared__ __attribute__((aligned(1024))) uint8_t s_0[32768];
    __shared__ __attribute__((aligned(1024))) uint8_t s_1[32768];
    __shared__ __attribute__((aligned(1024))) uint8_t s_2[32768];
    __shared__ __attribute__((aligned(1024))) uint8_t s_3[32768];
    static_assert(ST * 2 * kOperand == 4 * 32768, "");
    const int pos = walk_position(blockIdx.x, n_tiles);
    if (pos < 0) return;
    const int tc = pos / tiles_r, tr = pos - tc * tiles_r;               // down the rows: neighbours share the columns' operand
    const int lane = threadIdx.x & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int r0 = tr * SIDE, c0 = tc * SIDE;
    const float scale_a = FA == kFmtBf16 || BLOCKS ? 1.0f : *d_sA, scale_b = FB == kFmtBf16 || BLOCKS ? 1.0f : *d_sB;
    const int nk = (T + BK - 1) / BK, ns = (nk + kMiniSteps - 1) / kMiniSteps;
    auto range = [&](int rows_left, int ld, int ks) -> unsigned {
        const int n = rows_left < SIDE ? rows_left : SIDE;
        return ks == BK ? (unsigned)((size_t)(n - 1) * ld + T) : (unsigned)((size_t)(T / BK - 1) * ks + (size_t)(n - 1) * ld + BK);
    };
    const __amdgpu_buffer_rsrc_t rsA = make_rsrc(A + (size_t)r0 * ldA, range(R - r0, ldA, ksA));
    const __amdgpu_buffer_rsrc_t rsB = make_rsrc(B + (size_t)c0 * ldB, range(Cn - c0, ldB, ksB));
    // Loads: an instruction moves 8 rows x 128 bytes; the wave's rows are [SIDE / 4 wave, SIDE / 4 (wave + 1))
    constexpr int kPerSlab = SIDE / 32, kLoads = 2 * kMiniSteps * kPerSlab;
    const int ld_row = lane >> 3;
    // wave tile: block rows 16 wr NB .., of which the codes' register of a step holds four: the first of them is a multiple of 4
    const int wr = wave >> 1, wc = wave & 1;
    const int blockA = (r0 >> 4) + wr * NB, blockB = (c0 >> 4) + wc * NB;
    const int shiftA = 8 * (blockA & 3), shiftB = 8 * (blockB & 3);
    struct StageScales { int a[BLOCKS ? kMiniSteps : 1], b[BLOCKS ? kMiniSteps : 1]; };
    StageScales scales[ST];
    const int pitchA = (R + 127) & ~127, pitchB = (Cn + 127) & ~127;
    const __amdgpu_buffer_rsrc_t rsSA = BLOCKS ? make_rsrc(d_sA, (unsigned)(nk * pitchA)) : rsA, rsSB = BLOCKS ? make_rsrc(d_sB, (unsigned)(nk * pitchB)) : rsB;
    const int sc_voffA = (blockA >> 3) * 128 + 8 * (lane & 15) + (blockA & 4), sc_voffB = (blockB >> 3) * 128 + 8 * (lane & 15) + (blockB & 4);
    constexpr int kScaleLoads = BLOCKS ? 2 * kMiniSteps : 0;
    auto issue_stage = [&](uint8_t* bufA, uint8_t* bufB, int stage, StageScales& sc) {
        if constexpr (BLOCKS) {
#pragma unroll
            for (int j = 0; j < kMiniSteps; ++j) {
                const int step = stage * kMiniSteps + j;
                sc.a[j] = (int)__builtin_amdgcn_raw_buffer_load_b32(rsSA, sc_voffA, step < nk ? step * pitchA : kOutOfRange, 0);
                sc.b[j] = (int)__builtin_amdgcn_raw_buffer_load_b32(rsSB, sc_voffB, step < nk ? step * pitchB : kOutOfRange, 0);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
#pragma unroll
        for (int j = 0; j < kMiniSteps; ++j) {
            const int step = stage * kMiniSteps + j;
#pragma unroll
            for (int m = 0; m < kPerSlab; ++m) {
                const int row = wave * (SIDE / 4) + 8 * m + ld_row;      // its index modulo 16 sets the swizzle
                const int chunk = ((lane & 7) ^ row_swizzle(row & 15)) << 4;
                const bool there = step < nk && step * BK + chunk < T;   // (T % 16 == 0: a chunk exists or not)
                const int offA = there ? row * ldA + chunk + (int)((unsigned)step * (unsigned)ksA) : kOutOfRange;
                const int offB = there ? row * ldB + chunk + (int)((unsigned)step * (unsigned)ksB) : kOutOfRange;
                const int dst = j * kSlab + (wave * (SIDE / 4) + 8 * m) * BK;
                __builtin_amdgcn_raw_ptr_buffer_load_lds(rsA, (lds_void*)(bufA + dst), 16, offA, 0, 0, 0);
                __builtin_amdgcn_raw_ptr_buffer_load_lds(rsB, (lds_void*)(bufB + dst), 16, offB, 0, 0, 0);
            }
        }
    };
    const int fr_row = lane & 15, fr_q = lane >> 4, swz = row_swizzle(fr_row);
    const int ch0 = ((fr_q * 2) ^ swz) << 4, ch1 = ((fr_q * 2 + 1) ^ swz) << 4;
    auto fragment = [&](const uint8_t* slab, int first_row) -> v8i {
        const uint8_t* p = slab + (first_row + fr_row) * BK;
        const v4i lo = *reinterpret_cast<const v4i*>(p + ch0), hi = *reinterpret_cast<const v4i*>(p + ch1);
        return v8i{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
    };
    v4f acc[NB][NB];
#pragma unroll
    for (int i = 0; i < NB; ++i)
#pragma unroll
        for (int j = 0; j < NB; ++j) acc[i][j] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
    // behind: stages requested after this one.  The last stages (fewer than ST - 1 behind, or the first of them) request none: their codes would be no use to anybody and dropped by the compiler, but counted here.
    auto stage_step = [&](uint8_t* bufA, uint8_t* bufB, int stage, StageScales& sc, auto behind, auto more) __attribute__((always_inline)) {
        wait_vmcnt<decltype(behind)::value * (kLoads + kScaleLoads)>();                  // this stage has landed, the later ones are on their way
        lds_barrier_in_flight();
        v8i a[kMiniSteps][NB], b[kMiniSteps][NB];
#pragma unroll
        for (int j = 0; j < kMiniSteps; ++j)
#pragma unroll
            for (int i = 0; i < NB; ++i) {
                a[j][i] = fragment(bufA + j * kSlab, wr * 16 * NB + 16 * i);
                b[j][i] = fragment(bufB + j * kSlab, wc * 16 * NB + 16 * i);
            }
#pragma unroll
        for (int j = 0; j < kMiniSteps; ++j)
#pragma unroll
            for (int i = 0; i < NB; ++i)
#pragma unroll
                for (int k = 0; k < NB; ++k) {
                    if constexpr (FA == kFmtBf16) {
                        const v8i &x = b[j][k], &y = a[j][i];
                        const v4i x0 = {x[0], x[1], x[2], x[3]}, x1 = {x[4], x[5], x[6], x[7]}, y0 = {y[0], y[1], y[2], y[3]}, y1 = {y[4], y[5], y[6], y[7]};
                        acc[i][k] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, x0), __builtin_bit_cast(bf16x8, y0), acc[i][k], 0, 0, 0);
                        acc[i][k] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, x1), __builtin_bit_cast(bf16x8, y1), acc[i][k], 0, 0, 0);
                    } else if constexpr (BLOCKS) {
                        acc[i][k] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(b[j][k], a[j][i], acc[i][k], FB, FA, 0, sc.b[j] >> (shiftB + 8 * k), 0, sc.a[j] >> (shiftA + 8 * i));
                    } else {
                        acc[i][k] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(b[j][k], a[j][i], acc[i][k], FB, FA, 0, 0, 0, 0);
                    }
                }
        if constexpr (decltype(more)::value) {
            lds_barrier_in_flight();                                     // everybody has read the stage: it may be overwritten
            issue_stage(bufA, bufB, stage + ST, sc);                         // (beyond the last stage: nothing is fetched, zeros are written)
        }
    };
    typedef IntTag<ST - 1> All;
    typedef BoolTag<true> More;
    typedef BoolTag<false> Last;
    auto half = [&](uint8_t* buf) { return SIDE == 64 ? buf : buf + kOperand; };
    if constexpr (SIDE == 64) {
        issue_stage(s_0, s_1, 0, scales[0]);
        issue_stage(s_2, s_3, 1, scales[1]);
        int st = 0;
        for (; st + 1 < ns; st += 2) {                                   // (the same order of loads on every way round: the compiler counts them)
            stage_step(s_0, s_1, st, scales[0], All{}, More{});
            stage_step(s_2, s_3, st + 1, scales[1], All{}, More{});
        }
        if (st < ns) stage_step(s_0, s_1, st, scales[0], All{}, Last{});
    } else {
        issue_stage(s_0, half(s_0), 0, scales[0]);
        issue_stage(s_1, half(s_1), 1, scales[1]);
        issue_stage(s_2, half(s_2), 2, scales[ST == 4 ? 2 : 0]);
        issue_stage(s_3, half(s_3), 3, scales[ST == 4 ? 3 : 0]);
        int st = 0;
        for (; st + 3 < ns; st += 4) {
            stage_step(s_0, half(s_0), st, scales[0], All{}, More{});
            stage_step(s_1, half(s_1), st + 1, scales[1], All{}, More{});
            stage_step(s_2, half(s_2), st + 2, scales[ST == 4 ? 2 : 0], All{}, More{});
            stage_step(s_3, half(s_3), st + 3, scales[ST == 4 ? 3 : 0], All{}, More{});
        }
        if (st < ns) stage_step(s_0, half(s_0), st, scales[0], IntTag<3>{}, Last{});
        if (st + 1 < ns) stage_step(s_1, half(s_1), st + 1, scales[1], IntTag<2>{}, Last{});
        if (st + 2 < ns) stage_step(s_2, half(s_2), st + 2, scales[ST == 4 ? 2 : 0], IntTag<1>{}, Last{});
    }
    wait_vmcnt<0>();                                                     // nothing lands in LDS behind the workgroup's end
    const float inv_a = 1.0f / scale_a, inv_b = 1.0f / scale_b, inv_ab = inv_a * inv_b;
    const bool one_mul = inv_ab >= 1.17549435e-38f && inv_ab <= 3.402823466e+38f;
    const float m1 = one_mul ? inv_ab : inv_a, m2 = one_mul ? 1.0f : inv_b;
    const bool vector = Cn % 4 == 0;
    unsigned mag = 0;
#pragma unroll
    for (int i = 0; i < NB; ++i) {
        const int r = r0 + wr * 16 * NB + 16 * i + (lane & 15);
#pragma unroll
        for (int k = 0; k < NB; ++k) {
            const int c = c0 + wc * 16 * NB + 16 * k + (lane >> 4) * 4;
            if (r >= R || c >= Cn) continue;
            uint16_t* dst = C + (size_t)r * Cn + c;
            const int valid = Cn - c;
            uint16_t old[4] = {0, 0, 0, 0}, out[4];
            if (accumulate) {
                if (vector) {
                    const v2u o = *reinterpret_cast<const v2u*>(dst);
                    old[0] = (uint16_t)o[0]; old[1] = (uint16_t)(o[0] >> 16); old[2] = (uint16_t)o[1]; old[3] = (uint16_t)(o[1] >> 16);
                } else {
#pragma unroll
                    for (int e = 0; e < 4; ++e) if (e < valid) old[e] = dst[e];
                }
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                float y = acc[i][k][e] * m1 * m2;
                if (accumulate) y += __uint_as_float((unsigned)old[e] << 16);
                out[e] = __builtin_bit_cast(uint16_t, (__bf16)y);
                const unsigned m = out[e] & 0x7FFFu;
                if (e < valid) mag = mag > m ? mag : m;
            }
            if (vector) *reinterpret_cast<v2u*>(dst) = v2u{out[0] | (unsigned)out[1] << 16, out[2] | (unsigned)out[3] << 16};
            else {
#pragma unroll
                for (int e = 0; e < 4; ++e) if (e < valid) dst[e] = out[e];
            }
        }
    }
    if (amax_bits) {
        __syncthreads();
        mag = block_max_u32<kGemmThreads>(mag, reinterpret_cast<unsigned*>(s_0));
        if (threadIdx.x == 0) {
            const unsigned bits = amax_bits_from_bf16_mag(mag);
            if (bits > __hip_atomic_load(amax_bits, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT)) atomicMax(amax_bits, bits);
        }
    }
}

}  // namespace llmq
