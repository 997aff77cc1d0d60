// BF16 -> FP8 with a power-of-two scale for every block of 128 values along the contraction, row-wise and transposed copy in one pass.
//
// HBM-bound: 2 bytes read, 1 + 1 written per element.  Per-tensor scaling needs a pass over the tensor for its absmax first; here a 128 x 128 tile holds every
// block that crosses it whole, along its rows and along its columns, so a workgroup reads its tile once, finds the magnitudes in registers
// and converts from there.  The two copies have different scales (1 x 128 blocks) and are converted each by itself: the row-wise one
// pair by pair along the row, the transposed one from pairs of rows, which byte permutes have put side by side, and which leaves its bytes in the order of
// the transposed tensor.
//
// Both copies of 8192 x 3584 (118 MB): 22.5 us, 5.2 TB/s, nine tenths of a large copy's rate; of 1777 x 4608 in E5M2 (33 MB): 9.6 us, one round of 504 tiles that load, convert and
// store one after the other.
#include "api_checks.h"
#include "blocks.h"
#include "rmsnorm.h"

namespace llmq {

struct QuantBlocks {
    const uint16_t* x;
    int64_t rows, cols;
    uint8_t *q, *s, *qt, *st;
    SmallGrid grid;                             // of 128 x 128 tiles
    const uint16_t* w;                          // NORM: the norm's weight and statistics, and y or NULL
    const float* rstd;
    uint16_t* y;
};

// Packed maxima over the lanes side by side (wave_patch: bits 0, 1, 4 and 5 of the lane), and over those stacked (bits 2 and 3)
__device__ inline unsigned max_beside(unsigned v) {
    v = pk_max_u16(v, (unsigned)__builtin_amdgcn_update_dpp(0, (int)v, 0xB1, 0xF, 0xF, false));      // quad_perm [1,0,3,2]
    v = pk_max_u16(v, (unsigned)__builtin_amdgcn_update_dpp(0, (int)v, 0x4E, 0xF, 0xF, false));      // quad_perm [2,3,0,1]
    const auto a = __builtin_amdgcn_permlane16_swap(v, v, false, false);
    v = pk_max_u16(a[0], a[1]);
    const auto b = __builtin_amdgcn_permlane32_swap(v, v, false, false);
    return pk_max_u16(b[0], b[1]);
}
__device__ inline unsigned max_stacked(unsigned v) {
    v = pk_max_u16(v, (unsigned)__builtin_amdgcn_update_dpp(0, (int)v, 0x128, 0xF, 0xF, false));     // row_ror:8
    return pk_max_u16(v, (unsigned)__builtin_amdgcn_update_dpp(0, (int)v, 0x124, 0xF, 0xF, false));  // row_ror:4 of what repeats every 8
}

__device__ inline void tile_write_transposed_upto(const uint8_t* s_t, uint8_t* dt, int64_t row_stride, int64_t rows_left, int64_t cols_left) {
#pragma unroll
    for (int m = 0; m < kTileCols * (kTileRows / 16) / kTileThreads; ++m) {
        const int p = threadIdx.x + m * kTileThreads;
        const int c = p >> 3, ch = p & 7;
        const int64_t valid = rows_left - ch * 16;
        if (c >= cols_left || valid <= 0) continue;
        const v2u lo = *reinterpret_cast<const v2u*>(s_t + c * kTilePitch + ch * 16), hi = *reinterpret_cast<const v2u*>(s_t + c * kTilePitch + ch * 16 + 8);
        const v4u v = {lo[0], lo[1], hi[0], hi[1]};
        uint8_t* dst = dt + (int64_t)c * row_stride + ch * 16;
        if (valid >= 16) *reinterpret_cast<v4u_at1*>(dst) = v;
        else store16_codes_upto(dst, v, (int)valid);
    }
}

// SQUARE: blocks of 128 x 128 (both copies have the same codes), else 1 x 128 of each copy's rows.  ROWS / COLS: which copies are wanted.
// STREAM: the row-wise copy is stored with the streaming hint.
// NORM: the codes are those of y = bf16((x rstd) w) (llmq_rmsnorm_fwd_fp8_blocks).
template <int FMT, bool SQUARE, bool ROWS, bool COLS, bool GUARD, bool STREAM, bool NORM = false>
__global__ __launch_bounds__(kTileThreads) void quantize_blocks_kernel(const QuantBlocks t) {
    __shared__ __attribute__((aligned(16))) uint8_t s_t[COLS ? kTileLdsBytes : 16];
    __shared__ __attribute__((aligned(16))) unsigned s_mag[4][64];           // column pairs of each wave
    __shared__ __attribute__((aligned(16))) uint8_t s_code[2][kBlock];       // codes of the tile's rows and columns, in the order they are kept in
    unsigned brow, bcol;
    if (!small_tile(t.grid, blockIdx.x + t.grid.first, brow, bcol)) return;
    const int wave = threadIdx.x / kWave;
    int stacked, beside;
    wave_patch(stacked, beside);
    const int tr = wave * (4 * kPatchRows) + stacked * kPatchRows, tc = beside * 8;
    const int64_t cols = t.cols, R0 = (int64_t)brow * kTileRows, C0 = (int64_t)bcol * kTileCols, r0 = R0 + tr, c0 = C0 + tc;
    v4u in[kPatchRows];
    const uint16_t* src = t.x + r0 * cols + c0;
    if constexpr (GUARD) {
        load_patch_upto(in, src, cols, c0, t.rows - r0, cols - c0);
    } else {
#pragma unroll
        for (int i = 0; i < kPatchRows; ++i) in[i] = __builtin_nontemporal_load(reinterpret_cast<const v4u*>(src + (int64_t)i * cols));
    }
    if constexpr (NORM) {
        v4u wv;
        float rs[kPatchRows];
        if constexpr (GUARD) {
            // (what does not exist is zero times zero, also in a row whose statistic, or a column whose weight, is no number or infinite)
            wv = load8_upto(t.w + c0, c0, r0 < t.rows ? cols - c0 : 0);
#pragma unroll
            for (int i = 0; i < kPatchRows; ++i) rs[i] = r0 + i < t.rows && c0 < cols ? t.rstd[r0 + i] : 0.0f;
        } else {
            wv = *reinterpret_cast<const v4u*>(t.w + c0);
#pragma unroll
            for (int i = 0; i < kPatchRows; i += 4) {
                const v4f four = *reinterpret_cast<const v4f*>(t.rstd + r0 + i);
#pragma unroll
                for (int k = 0; k < 4; ++k) rs[i + k] = four[k];
            }
        }
#pragma unroll
        for (int i = 0; i < kPatchRows; ++i) in[i] = normalize8(in[i], rs[i], wv);
        if constexpr (GUARD) {
            // (in patches that the tensor ends in; the same answer for the whole launch)
            if (cols % 8 != 0) {
#pragma unroll
                for (int i = 0; i < kPatchRows; ++i) in[i] = keep_upto(in[i], cols - c0 < 8 ? (int)(cols - c0) : 8);
            }
            if (t.rows % kPatchRows != 0) {
#pragma unroll
                for (int i = 0; i < kPatchRows; ++i)
                    if (r0 + i >= t.rows) in[i] = v4u{0, 0, 0, 0};
            }
        }
        if (t.y) {
            uint16_t* dst = t.y + r0 * cols + c0;
            if constexpr (GUARD) {
                store_patch_upto(in, dst, cols, t.rows - r0, cols - c0);
            } else {
#pragma unroll
                for (int i = 0; i < kPatchRows; ++i) *reinterpret_cast<v4u*>(dst + (int64_t)i * cols) = in[i];
            }
        }
    }
    // magnitudes: of rows i and i + 1 in one register each, of columns 2 k and 2 k + 1
    unsigned row_mag[kPatchRows / 2], col_mag[4] = {0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < kPatchRows; i += 2) {
        unsigned m[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            unsigned mag[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                mag[k] = in[i + h][k] & 0x7FFF7FFFu;
                col_mag[k] = pk_max_u16(col_mag[k], mag[k]);
            }
            m[h] = pk_max_u16(pk_max_u16(mag[0], mag[1]), pk_max_u16(mag[2], mag[3]));
        }
        row_mag[i / 2] = pk_max_u16(__builtin_amdgcn_perm(m[1], m[0], 0x05040100u), __builtin_amdgcn_perm(m[1], m[0], 0x07060302u));
    }
    unsigned row_code[kPatchRows], col_code[8];
    if constexpr (SQUARE) {
        unsigned m = pk_max_u16(pk_max_u16(col_mag[0], col_mag[1]), pk_max_u16(col_mag[2], col_mag[3]));
        m = (m & 0xFFFFu) > (m >> 16) ? m & 0xFFFFu : m >> 16;
        const unsigned code = scale_code<FMT>(block_max_u32<kTileThreads>(m, &s_mag[0][0]) << 16);
#pragma unroll
        for (int i = 0; i < 8; ++i) row_code[i] = col_code[i] = code;
        if (threadIdx.x < kBlock / 4) {
            const unsigned four = code * 0x01010101u;
            const int64_t pr = (t.rows + kBlock - 1) / kBlock * kBlock, pc = (cols + kBlock - 1) / kBlock * kBlock;
            if constexpr (ROWS) *reinterpret_cast<unsigned*>(t.s + bcol * pr + R0 + 4 * threadIdx.x) = four;
            if constexpr (COLS) *reinterpret_cast<unsigned*>(t.st + brow * pc + C0 + 4 * threadIdx.x) = four;
        }
    } else {
        if constexpr (ROWS) {
#pragma unroll
            for (int i = 0; i < kPatchRows; i += 2) {
                const unsigned m = max_beside(row_mag[i / 2]);
                row_code[i] = scale_code<FMT>(m << 16);
                row_code[i + 1] = scale_code<FMT>(m & 0xFFFF0000u);
            }
            if (beside == 0) {
#pragma unroll
                for (int i = 0; i < kPatchRows; ++i) s_code[0][8 * ((tr + i) & 15) + (tr >> 4)] = (uint8_t)row_code[i];
            }
        }
        if constexpr (COLS) {
            v4u m;
#pragma unroll
            for (int k = 0; k < 4; ++k) m[k] = max_stacked(col_mag[k]);
            if (stacked == 0) *reinterpret_cast<v4u*>(&s_mag[wave][tc / 2]) = m;
        }
        __syncthreads();
        if constexpr (COLS) {
            v4u m = *reinterpret_cast<const v4u*>(&s_mag[0][tc / 2]);
#pragma unroll
            for (int w = 1; w < 4; ++w) {
                const v4u o = *reinterpret_cast<const v4u*>(&s_mag[w][tc / 2]);
#pragma unroll
                for (int k = 0; k < 4; ++k) m[k] = pk_max_u16(m[k], o[k]);
            }
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                col_code[2 * k] = scale_code<FMT>(m[k] << 16);
                col_code[2 * k + 1] = scale_code<FMT>(m[k] & 0xFFFF0000u);
            }
            if (stacked == 0 && wave == 0) {
#pragma unroll
                for (int j = 0; j < 8; ++j) s_code[1][8 * ((tc + j) & 15) + (tc >> 4)] = (uint8_t)col_code[j];
            }
        }
    }
    if constexpr (ROWS) {
        unsigned w[kPatchRows][2];
#pragma unroll
        for (int i = 0; i < kPatchRows; ++i) {
            w[i][0] = cvt_four<FMT>(in[i][0], in[i][1], row_code[i]);
            w[i][1] = cvt_four<FMT>(in[i][2], in[i][3], row_code[i]);
        }
        uint8_t* dst = t.q + r0 * cols + c0;
        if constexpr (GUARD) {
            store_codes_upto(w, dst, cols, t.rows - r0, cols - c0);
        } else {
#pragma unroll
            for (int i = 0; i < kPatchRows; ++i) store_hinted<STREAM>(v2u{w[i][0], w[i][1]}, reinterpret_cast<v2u*>(dst + (int64_t)i * cols));
        }
    }
    if constexpr (COLS) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            // column tc + j, rows in pairs
            unsigned pair[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) pair[i] = __builtin_amdgcn_perm(in[2 * i + 1][j / 2], in[2 * i][j / 2], j & 1 ? 0x07060302u : 0x05040100u);
            *reinterpret_cast<v2u*>(s_t + (tc + j) * kTilePitch + tr) = v2u{cvt_four<FMT>(pair[0], pair[1], col_code[j]), cvt_four<FMT>(pair[2], pair[3], col_code[j])};
        }
    }
    if constexpr (COLS || !SQUARE) __syncthreads();
    if constexpr (!SQUARE) {
        if (threadIdx.x < kBlock / 4) {
            const int64_t pr = (t.rows + kBlock - 1) / kBlock * kBlock, pc = (cols + kBlock - 1) / kBlock * kBlock;
            if constexpr (ROWS) *reinterpret_cast<unsigned*>(t.s + bcol * pr + R0 + 4 * threadIdx.x) = *reinterpret_cast<const unsigned*>(&s_code[0][4 * threadIdx.x]);
            if constexpr (COLS) *reinterpret_cast<unsigned*>(t.st + brow * pc + C0 + 4 * threadIdx.x) = *reinterpret_cast<const unsigned*>(&s_code[1][4 * threadIdx.x]);
        }
    }
    if constexpr (COLS) {
        uint8_t* dt = t.qt + C0 * t.rows + R0;
        if constexpr (GUARD) tile_write_transposed_upto(s_t, dt, t.rows, t.rows - R0, cols - C0);
        else tile_write_transposed(s_t, dt, t.rows);
    }
}

template <int FMT, bool SQUARE, bool ROWS, bool COLS, bool NORM = false>
static int launch_quantize_blocks(QuantBlocks t, hipStream_t stream) {
    const bool whole = t.rows % kTileRows == 0 && t.cols % kTileCols == 0;
    SmallGrid g{};
    g.rows = (unsigned)((t.rows + kTileRows - 1) / kTileRows);
    g.cols = (unsigned)((t.cols + kTileCols - 1) / kTileCols);
    g.blocks = (g.rows * g.cols + kSmallXcds - 1) / kSmallXcds * kSmallXcds;
    // Rows of either copy that do not start at cache lines share lines with the tiles beside them, which then belong on one XCD (launch order / XCD ranges: 1777 x 4601 13.6 / 11.2 us,
    // 1777 x 4608 10.8 / 10.5, 8191 x 3583 38.2 / 38.1;  rows of lines 8192 x 3584 21.5 / 22.6).
    g.xcd_ranges = t.rows % 64 != 0 || t.cols % 64 != 0;
    // (plain / streamed: 8192 x 18944 130.2 / 124.6 us, 8192 x 3584 23.7 / 24.5)
    const bool stream_q = whole && ROWS && streams_out((ROWS + COLS) * t.rows * t.cols, t.cols, 128, 96);
    small_launches(g, [&](const SmallGrid& part, unsigned blocks) {
        t.grid = part;
        auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(blocks), dim3(kTileThreads), 0, stream, t); };
        if (!whole) launch(quantize_blocks_kernel<FMT, SQUARE, ROWS, COLS, true, false, NORM>);
        else if (stream_q) launch(quantize_blocks_kernel<FMT, SQUARE, ROWS, COLS, false, ROWS, NORM>);
        else launch(quantize_blocks_kernel<FMT, SQUARE, ROWS, COLS, false, false, NORM>);
    });
    return hipGetLastError() == hipSuccess ? LLMQ_OK : LLMQ_ERR_DEVICE;
}

template <int FMT, bool SQUARE>
static int launch_copies(const QuantBlocks& t, hipStream_t stream) {
    if (t.q && t.qt) return launch_quantize_blocks<FMT, SQUARE, true, true>(t, stream);
    if (t.q) return launch_quantize_blocks<FMT, SQUARE, true, false>(t, stream);
    return launch_quantize_blocks<FMT, SQUARE, false, true>(t, stream);
}

int launch_norm_quantize_blocks(const void* res, const void* w, const float* rstd, int64_t M, int64_t C, int fmt, uint8_t* q, uint8_t* s, uint8_t* q_t, uint8_t* s_t, void* y, hipStream_t stream) {
    const QuantBlocks t{static_cast<const uint16_t*>(res), M, C, q, s, q_t, s_t, {}, static_cast<const uint16_t*>(w), rstd, static_cast<uint16_t*>(y)};
    if (fmt == LLMQ_E4M3) return q ? launch_quantize_blocks<0, false, true, true, true>(t, stream) : launch_quantize_blocks<0, false, false, true, true>(t, stream);
    return q ? launch_quantize_blocks<1, false, true, true, true>(t, stream) : launch_quantize_blocks<1, false, false, true, true>(t, stream);
}

}  // namespace llmq

extern "C" {

size_t llmq_block_scales_bytes(int64_t rows, int64_t cols) {
    if (!dim_ok(rows) || !dim_ok(cols)) return 0;
    return (size_t)((rows + 127) / 128 * 128) * (size_t)((cols + 127) / 128);
}

int llmq_quantize_fp8_blocks(const void* x_bf16, int64_t rows, int64_t cols, int fmt, int block_rows, uint8_t* q, uint8_t* s,
                             uint8_t* q_t, uint8_t* s_t, void* stream) {
    if (!x_bf16 || (!q && !q_t) || !q != !s || !q_t != !s_t) return LLMQ_ERR_NULL;
    if (!dim_ok(rows) || !dim_ok(cols) || rows * cols >= kMaxElems) return LLMQ_ERR_SHAPE;
    if (!fmt_ok(fmt)) return LLMQ_ERR_FORMAT;
    if (block_rows != 1 && block_rows != 128) return LLMQ_ERR_FLAGS;
    if (!aligned(x_bf16, 16) || !aligned(q, 16) || !aligned(s, 16) || !aligned(q_t, 16) || !aligned(s_t, 16)) return LLMQ_ERR_ALIGN;
    const llmq::QuantBlocks t{static_cast<const uint16_t*>(x_bf16), rows, cols, q, s, q_t, s_t, {}, nullptr, nullptr, nullptr};
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (fmt == LLMQ_E4M3) return block_rows == 128 ? llmq::launch_copies<0, true>(t, st) : llmq::launch_copies<0, false>(t, st);
    return block_rows == 128 ? llmq::launch_copies<1, true>(t, st) : llmq::launch_copies<1, false>(t, st);
}

}  // extern "C"
