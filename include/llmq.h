/*
 * llmq.h -- C ABI of the MI355X (gfx950) FP8 linear-layer path of LLMQ's 8-bit training pipeline.
 *
 * What the path computes (paper, Section 3 "Overview" and the kernel-fusion paragraph of Section 3):
 *   1. just-in-time tensor-level absmax scaling: find the largest |x| of a BF16 tensor and choose the
 *      scale that maps it onto the largest finite FP8 value, so that nothing is clipped;
 *   2. convert BF16 -> FP8 (E4M3 or E5M2, Section 2) with that scale, fused with the transposed copy,
 *      because the FP8 GEMM takes both operands with the contraction index contiguous ("TN");
 *   3. the transformer-block matmuls in FP8 with BF16 results: forward Y = X W^T, and in the backward
 *      pass dX = dY W and dW = dY^T X.
 *
 * Conventions for every entry point
 *   - Tensors are row-major with the last index contiguous.  X is [M,K], W is [N,K], Y and dY are
 *     [M,N], dX is [M,K], dW is [N,K].  BF16 tensors are arrays of 16-bit patterns, FP8 tensors are
 *     arrays of 8-bit OCP codes.
 *   - Every pointer is DEVICE memory owned by the caller, except `stream`, which is a hipStream_t
 *     passed as void* (NULL = the default stream).  The library allocates nothing, frees nothing and
 *     keeps no pointer after a call returns (Section 3 "Overview": all allocation happens at start-up).
 *   - Calls only enqueue work on `stream` and return; nothing synchronises with the host.  Scales and
 *     absmax values are read from and written to device memory.  The calls enqueue kernels only (no memory
 *     set or copy commands), so a stream that is being captured into a HIP graph can take them, and replays
 *     compute from what the buffers hold then.  Several host threads may call at the same time on streams
 *     and buffers of their own; the one piece of state the library keeps on a GPU is the scratch array of
 *     llmq_amax_static (see there).
 *   - BF16 and FP8 tensor pointers must be 16-byte aligned, float pointers 4-byte aligned.
 *   - Return value: LLMQ_OK or a negative llmq_status.  Argument errors are found on the host before
 *     anything is launched and leave all outputs untouched.  LLMQ_ERR_DEVICE reports a launch failure.
 *   - Results are bitwise deterministic: same inputs, same bytes (Section 3 "Reproducibility").  The
 *     only atomic used is an integer max (fused output absmax), whose result does not depend on order.
 *   - Dimensions may be any positive value.  Contractions run fastest when their dimensions are multiples of 128 and
 *     the quantizers on multiples of 128 rows x 256 columns; contractions of other shapes take the same tile kernels
 *     with guarded edges (fastest with a contraction length, or T-major row pitch, that is a multiple of 16).
 */
#ifndef LLMQ_H
#define LLMQ_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
    LLMQ_OK = 0,
    LLMQ_ERR_NULL = -1,       /* a required pointer is NULL */
    LLMQ_ERR_SHAPE = -2,      /* a dimension is < 1 or too large */
    LLMQ_ERR_ALIGN = -3,      /* a pointer is not aligned as required */
    LLMQ_ERR_FORMAT = -4,     /* not an llmq_fp8_format */
    LLMQ_ERR_WORKSPACE = -5,  /* workspace missing or smaller than llmq_fp8_linear_workspace_bytes() */
    LLMQ_ERR_DEVICE = -6,     /* the HIP runtime reported an error at launch */
    LLMQ_ERR_FLAGS = -7,      /* unknown bits in `flags` */
    LLMQ_ERR_VALUE = -8       /* a number is out of range, or arrays overlap that must not */
} llmq_status;

/* OCP 8-bit floating point formats (Section 2): E4M3 has bias 7 and max 448 (no Inf, NaN = S.1111.111),
 * E5M2 has bias 15 and max 57344 (IEEE-like Inf/NaN). */
typedef enum { LLMQ_E4M3 = 0, LLMQ_E5M2 = 1 } llmq_fp8_format;

const char* llmq_status_string(int status);
int llmq_version(void);

/*
 * Absmax and scale of a BF16 tensor (Section 3 "Overview": tensor-level absmax scaling, the scale maps the
 * tensor's largest magnitude onto the largest finite value of the FP8 format).
 *   x_bf16   [n] BF16, device, 16-byte aligned; n >= 1.
 *   fmt      target FP8 format, selects FMAX (448 or 57344) for the scale.
 *   d_amax   [1] float, device, written: max_i |x_i| exactly; the canonical quiet NaN 0x7FC00000 if the
 *            tensor holds a NaN; +Inf if it holds an Inf and no NaN.
 *   d_scale  [1] float, device, written if not NULL: min(FMAX / amax, FLT_MAX) with one IEEE binary32
 *            division (FLT_MAX for an absmax so small that the quotient overflows); 1 for an all-zero
 *            tensor, where the rule defines no scale and every code is +-0 whatever the scale; 0 when amax
 *            is +Inf; NaN when amax is NaN.
 *   ws       device scratch of at least llmq_amax_workspace_bytes() bytes, 4-byte aligned; contents on
 *            entry do not matter, it holds per-block partial results between the two launches (a
 *            streaming reduction, then a one-block kernel that reduces the partial results and writes
 *            both outputs; no atomics: Section 3 "Reproducibility").  Calls that may overlap on the
 *            device (different streams) need different workspaces.
 */
size_t llmq_amax_workspace_bytes(void);
int llmq_amax(const void* x_bf16, size_t n, int fmt, float* d_amax, float* d_scale,
              void* ws, size_t ws_bytes, void* stream);

/*
 * llmq_amax for callers that cannot allocate device memory and have no workspace to hand over: code under
 * HIP graph capture, tight serving loops, harnesses that forbid hipMalloc.  Same arguments, same kernels and
 * bit-identical outputs, but the per-block partial results go to a 4 KB array inside the library's device
 * image (one copy per GPU, held until the process ends) instead of `ws`.  The call allocates and frees
 * nothing.  n: 1 <= n < 2^40 elements as for llmq_amax, LLMQ_ERR_SHAPE beyond; the array's size does not
 * depend on n.  It uses the copy of the device that is current when the call is made, which must be the
 * stream's device; LLMQ_ERR_DEVICE if the runtime cannot resolve the array.  Every call on a GPU shares that
 * GPU's array: calls that may overlap on one device (different streams, or graphs replayed side by side) race
 * on it and need llmq_amax with separate workspaces instead.  Nothing in the array has to be cleared between
 * calls: every word the second stage reads has been written by the first stage of the same call.
 */
int llmq_amax_static(const void* x_bf16, size_t n, int fmt, float* d_amax, float* d_scale, void* stream);

/*
 * Fused scale + FP8 cast + transposed copy (Section 3, kernel-fusion paragraph: quantization and the
 * transposition the backward GEMMs need are one kernel).
 *   q[i,j]   = cast( fl32( fl32(x[i,j]) * d_scale[0] ) ),  q_t[j,i] = q[i,j]
 * cast = round-to-nearest-even onto the FP8 grid, saturating at +-FMAX (a finite product never yields
 * an Inf or NaN code).  The result for NaN inputs is unspecified.
 *   x_bf16   [rows, cols] BF16;  d_scale [1] float (device);  q [rows, cols] FP8;
 *   q_t      [cols, rows] FP8, or NULL when no transposed copy is wanted.
 */
int llmq_quantize_fp8(const void* x_bf16, int64_t rows, int64_t cols, const float* d_scale, int fmt,
                      uint8_t* q, uint8_t* q_t, void* stream);
/*
 * The same with the transposed copy stored in slabs of 128 contraction bytes, the form the backward contractions
 * read fastest (LLMQ_LAYOUT_SLABS of llmq_fp8_gemm, there with rows = cols of x and T = rows of x):
 *   q_t byte of element (j, i) of the transposed tensor at (i / 128) * cols * 128 + j * 128 + i % 128.
 * A 128 x 128 tile of x is then one contiguous 16 KB piece of q_t instead of 128 pieces of 128 bytes.  rows must
 * be a multiple of 128 and cols a multiple of 256 (LLMQ_ERR_SHAPE otherwise); q_t must not be NULL.
 */
int llmq_quantize_fp8_slabs(const void* x_bf16, int64_t rows, int64_t cols, const float* d_scale, int fmt,
                            uint8_t* q, uint8_t* q_t, void* stream);

/*
 * The FP8 contraction that forward, dgrad and wgrad share (Section 3: FP8 GEMM is TN-only):
 *   c[r,cc] = bf16( ( sum_t A[r,t] * B[cc,t] ) / (sA * sB) )        accumulate == 0
 *   c[r,cc] = bf16( c[r,cc] + (sum ...) / (sA * sB) )                accumulate != 0 (BF16 gradient
 *                                                                    accumulation, Section 3 "Overview")
 *   A [R,T] FP8 in format fmtA, B [C,T] FP8 in format fmtB (any mix of E4M3 / E5M2), products exact,
 *   accumulation in binary32 on the matrix cores, de-scaling in binary32, one rounding to BF16 (RNE).
 *   d_scaleA, d_scaleB  [1] float each (device): the scales the operands were quantized with.
 *   c_bf16   [R,C] BF16, written (read first when accumulate != 0).
 *   d_amax_c [1] float (device) or NULL: if given, receives max |c| of the BF16 result, bit-identical to
 *            llmq_amax of c (the next layer's quantization then needs no separate reduction; Section 3,
 *            kernel-fusion paragraph).
 * Error of each element is bounded by 2^-7 * sum_t |A[r,t] B[cc,t]| / (sA sB).
 */
int llmq_fp8_gemm_tn(const uint8_t* A, int fmtA, const uint8_t* B, int fmtB,
                     int64_t R, int64_t C, int64_t T,
                     const float* d_scaleA, const float* d_scaleB,
                     void* c_bf16, int accumulate, float* d_amax_c, void* stream);

/*
 * The same contraction with either operand in another layout than [rows, T] (LLMQ_LAYOUT_ROWS = 0):
 *   LLMQ_LAYOUT_T_MAJOR = 1: stored [T, rows] (the contraction index runs down the rows, the rows index is
 *     contiguous);
 *   LLMQ_LAYOUT_SLABS = 2: stored K step by K step, byte (r, t) at (t / 128) * rows * 128 + r * 128 + t % 128
 *     (T a multiple of 128, else LLMQ_ERR_SHAPE): the 128 contraction bytes of all rows for one K step are one
 *     contiguous piece.  The arithmetic and its order are those of LLMQ_LAYOUT_ROWS: same result bytes.
 *   a_t_major: layout of A ([T,R] when T-major);   b_t_major: layout of B;   both 0: identical to
 *   llmq_fp8_gemm_tn.  Other values: LLMQ_ERR_FLAGS.
 * The paper keeps transposed FP8 copies of every quantized tensor because the FP8 GEMM it builds on only
 * takes contraction-contiguous operands, and names the extra transposes and buffers as the cost of FP8
 * (Section 3, kernel-fusion paragraph; Section 4 "Impact of FP8").  Here the tile kernel transposes a
 * T-major operand on its way from LDS to the matrix cores, so the backward GEMMs can read the row-major
 * copies the forward pass made:
 *   dX[m,k] = sum_n dYq[m,n] Wq[n,k]   : A = dYq [M,N],            B = Wq [N,K] T-major, T = N
 *   dW[n,k] = sum_m dYq[m,n] Xq[m,k]   : A = dYq [M,N] T-major,    B = Xq [M,K] T-major, T = M
 * Tuned for B in E4M3 and T-major operands below 2 GiB (dimensions that are no multiples of 128 with guarded edges);
 * T-major B in E5M2, ragged shapes with only A T-major, contractions (and T-major widths) below 16 and dimensions of
 * millions take a slow generic kernel, ragged problems so small that it is the faster one too.  In the tuned kernel (and likewise in the generic one) every product lands in the same accumulator
 * position as with transposed copies, so the result is bit-identical to llmq_fp8_gemm_tn on those copies
 * whenever both calls run the same kind of kernel, which is the case for what the linear calls below launch
 * on operands below 2 GiB.  Arguments otherwise as above.
 */
#define LLMQ_LAYOUT_ROWS    0
#define LLMQ_LAYOUT_T_MAJOR 1
#define LLMQ_LAYOUT_SLABS   2
int llmq_fp8_gemm(const uint8_t* A, int fmtA, int a_t_major, const uint8_t* B, int fmtB, int b_t_major,
                  int64_t R, int64_t C, int64_t T,
                  const float* d_scaleA, const float* d_scaleB,
                  void* c_bf16, int accumulate, float* d_amax_c, void* stream);

/*
 * The same contraction with caller-owned scratch, which lets the library share out a ragged last round of
 * output tiles: the chip computes one tile per CU at a time, and when the number of tiles is not a multiple of
 * the number of CUs the last round leaves CUs idle (560 tiles on 256 CUs take three rounds, the third with 48
 * tiles).  With scratch, the left-over tiles are cut along the contraction index and dealt to all CUs; every
 * piece is written to the scratch as binary32 accumulators, and a second launch adds the pieces of a tile in
 * the fixed order of their contraction ranges and finishes the tile (de-scale, BF16, absmax).  No atomic
 * additions, no dependence on timing: same inputs, same bytes (Section 3 "Reproducibility": an intermediate
 * buffer and a second step instead of atomics).  The sums are grouped differently from a call without scratch,
 * so the two may differ in the last bit of an output; both are within the error bound above.
 *   scratch        device memory, 256-byte aligned, at least llmq_fp8_gemm_scratch_bytes(R, C, T) bytes for the
 *                  sharing to happen; NULL or a smaller buffer: every tile is computed whole (as llmq_fp8_gemm).
 *                  Contents on entry do not matter; calls that may overlap on the device need separate scratch.
 * llmq_fp8_gemm_scratch_bytes returns 0 for shapes the library computes whole anyway: whole rounds, small
 * problems, shapes that larger tiles compute faster whole, and every shape for which sharing was not measured to
 * win (and T-major operands take no scratch).  The chip is
 * power-limited on real data, so CUs left idle by a ragged round let the busy ones clock higher and the round
 * costs less than a full one; sharing pays (3-7 % of one isolated GEMM) only for long contractions
 * (T >= 16384) whose left-over tiles all fit one group of pieces.  The linear calls below do not use it.
 */
size_t llmq_fp8_gemm_scratch_bytes(int64_t R, int64_t C, int64_t T);
int llmq_fp8_gemm_with_scratch(const uint8_t* A, int fmtA, int a_t_major, const uint8_t* B, int fmtB, int b_t_major,
                               int64_t R, int64_t C, int64_t T,
                               const float* d_scaleA, const float* d_scaleB,
                               void* c_bf16, int accumulate, float* d_amax_c,
                               void* scratch, size_t scratch_bytes, void* stream);

/*
 * BF16 baseline of the same contraction, for the FP8-versus-BF16 comparison the paper reports (Section 4,
 * "Impact of FP8", speed-up column of Table 1): no quantization, no scales,
 *   c[r,cc] = bf16( sum_t A[r,t] * B[cc,t] )   (+ c[r,cc] first when accumulate != 0)
 * A [R,T], B [C,T] BF16 with the contraction index contiguous, binary32 accumulation on the matrix cores
 * (v_mfma_f32_16x16x32_bf16 in the same tile kernel), one RNE rounding.  Error per element is bounded by
 * 2^-8 |c| + T 2^-24 sum_t |A[r,t] B[cc,t]|.  Shapes with R, C multiples of 128 and T a multiple of 64
 * are fastest, others take the same kernel with guarded edges (a generic one below T = 8 and for small problems, with its
 * sums in another order).
 */
int llmq_bf16_gemm_tn(const void* A_bf16, const void* B_bf16, int64_t R, int64_t C, int64_t T,
                      void* c_bf16, int accumulate, void* stream);

/*
 * FP8 with a scale for each block of 128 values along the contraction, for tensors whose rows or columns differ so much in size that one scale a
 * tensor (llmq_amax) leaves the small ones few bits.
 *
 *   A scale is a power of two, kept as one byte: the byte b stands for d = 2^(b-127), the smallest power of two with amax / d <= FMAX of
 *   the format (448 or 57344), amax the largest magnitude of the block; not below 2^-127 (b = 0), and b = 127 for a block of zeros.
 *     q = cast( x / d ),  round to nearest even; nothing is clipped and x / d is exact, so q d is x rounded to the format's bits.
 *   A block that holds an Inf or NaN has b = 255: the contractions that read it give NaN, its codes are unspecified.
 *
 *   The bytes of an operand [rows, T] (T the contraction) are kept K step by K step of 128, the rows of a step in groups of 128:
 *     byte of (row r, step k) at  k * rows128 + 128 (r / 128) + 8 (r % 16) + (r / 16) % 8,   rows128 = rows rounded up to a multiple of 128,
 *   which is the order the matrix cores' registers take them in.  llmq_block_scales_bytes(rows, T) = rows128 * ceil(T / 128).  Bytes of rows that do
 *   not exist are written (127, or their block's) and never matter.
 *
 * llmq_quantize_fp8_blocks: x [rows, cols] BF16 in one pass, without an absmax pass before it.
 *   block_rows 1:    q [rows, cols] with a scale for each row and 128 columns, and q_t [cols, rows] (the transposed tensor, for contractions over the rows of
 *                    x) with a scale for each column and 128 rows; the codes of the two are different ones.
 *   block_rows 128:  blocks of 128 x 128, whose codes and scales q and q_t share: weights, which are read along both dimensions.
 *   s and s_t: scale bytes of q as an operand [rows, T = cols] and of q_t as an operand [cols, T = rows].  Every row of a block of 128 x 128 has a copy of its
 *   byte, so operands of either kind are read alike.  q and s may be NULL together, or q_t and s_t; one pair must be there.
 *   Other values of block_rows: LLMQ_ERR_FLAGS.  All pointers 16-byte aligned.  Multiples of 128 rows and columns are fastest.
 *
 * llmq_fp8_gemm_blocks: c[r,cc] = bf16( sum_t A[r,t] dA[r,t/128] B[cc,t] dB[cc,t/128] )   (+ c[r,cc] first when accumulate != 0, one rounding)
 *   A [R,T] and B [C,T], rows of T contiguous bytes, any mix of formats; sA, sB their scale bytes.  Products are exact; the matrix cores
 *   align the 128 products of a K step to the largest before they add them (up to 2^-12.3 of the sum of their magnitudes was seen to be lost, as in llmq_fp8_gemm_tn) and add the steps in binary32.  Up to 32 rows, and some
 *   small outputs whose T is no multiple of 16, take a kernel that adds every fourth step by itself and joins the four sums: the last bits of a row may differ from those the same row has in a larger call (the same call
 *   gives the same bytes).  d_amax_c as in llmq_fp8_gemm_tn.  Error of each element bounded as there, by 2^-7 of the sum of the products' magnitudes.  Fastest with R and C
 *   multiples of 256 and T a multiple of 128 (16 at least).  T < 16, T or C >= 2^22 and scales of 2 GB take a slow generic kernel, which has R < 2^21 and
 *   C < 2^28 (LLMQ_ERR_SHAPE otherwise).
 *   forward         Y = X W^T     A = q of X,      B = q of W
 *   input gradient  dX = dY W     A = q of dY,     B = q_t of W
 *   weight gradient dW = dY^T X   A = q_t of dY,   B = q_t of X
 */
size_t llmq_block_scales_bytes(int64_t rows, int64_t cols);
int llmq_quantize_fp8_blocks(const void* x_bf16, int64_t rows, int64_t cols, int fmt, int block_rows,
                             uint8_t* q, uint8_t* s, uint8_t* q_t, uint8_t* s_t, void* stream);
int llmq_fp8_gemm_blocks(const uint8_t* A, const uint8_t* sA, int fmtA, const uint8_t* B, const uint8_t* sB, int fmtB,
                         int64_t R, int64_t C, int64_t T, void* c_bf16, int accumulate, float* d_amax_c, void* stream);

/*
 * The two products of a gated feed-forward block that meet its SwiGLU, from operands with block scales, each with the non-linearity in the same kernel.
 *
 * llmq_fp8_gemm_blocks_swiglu_fwd: both projections of a block and its non-linearity.  A [M, T] codes of the input and sA; W [2 I, T] codes of the gate and up weights and sW, as one operand: rows [0, I) are the
 *   gate's, rows [I, 2 I) the up branch's (the layout of GU that llmq_swiglu_fwd reads):
 *     g[m,i] = sum_t A[m,t] dA W[i,t] dW,   u[m,i] = sum_t A[m,t] dA W[I+i,t] dW,   h[m,i] = bf16( silu(g) u ),  silu(g) = g sg,  sg = 1 / (1 + e^-g)
 *   h [M, I] BF16; gu [M, 2 I] BF16 receives bf16(g) and bf16(u) for the backward pass if it is not NULL.  h is made from the sums in binary32, not from their rounded values, and does not depend on whether gu is wanted.
 * llmq_fp8_gemm_blocks_swiglu_bwd: the gradient through the down projection and the non-linearity.  A [M, T] codes of dY (T the model's width) and sA; B [I, T] codes of the transposed copy of the down projection's weight
 *   [T, I] and sB; gu [M, 2 I] what the forward pass kept:
 *     dh[m,i] = sum_t A[m,t] dA B[i,t] dB  (binary32, not rounded);   dgu[m, i] = bf16( dh u sg (1 + g (1 - sg)) ),   dgu[m, I+i] = bf16( dh g sg )
 *   dgu [M, 2 I] BF16, the dY of the gate and up projections; h [M, I] BF16 receives bf16( g sg u ) of the kept gu for the down projection's weight gradient if it is not NULL.  dgu may be gu itself.
 *   d_amax_h, d_amax_dgu [1] float or NULL: absmax of h or dgu, as llmq_amax of them has it.
 * Sums as in llmq_fp8_gemm_blocks: products exact, their error bounded by 2^-7 of the sum of the products' magnitudes; few rows (up to 32) and small problems take a kernel that adds in another order.  The exponential and the reciprocal are the
 *   hardware's: sg is off by at most 2^-20 + 2^-24 |g| of it; for g < -87, where |silu(g)| < 2^-118, silu(g) and its derivative may be +-0.  A sum that is no number makes its own output NaN, no other.
 * fmtA: E4M3 or E5M2, the weights E4M3 (LLMQ_ERR_FORMAT otherwise).  16 <= T < 2^22, I < 2^21, (rows of an operand rounded up to 128) ceil(T / 128) < 2^31 - 4096, 128 x 64 tiles of [M, I] below 2^24 (LLMQ_ERR_SHAPE).
 * Fastest with M a multiple of 256, I of 128 and T of 128; I a multiple of 32 (forward; any multiple of 8 backward) and T of 16, or at least 4, otherwise.  All pointers 16-byte aligned (d_amax: 4).
 */
int llmq_fp8_gemm_blocks_swiglu_fwd(const uint8_t* A, const uint8_t* sA, int fmtA, const uint8_t* W, const uint8_t* sW,
                                    int fmtW, int64_t M, int64_t I, int64_t T, void* h_bf16, void* gu_bf16,
                                    float* d_amax_h, void* stream);
int llmq_fp8_gemm_blocks_swiglu_bwd(const uint8_t* A, const uint8_t* sA, int fmtA, const uint8_t* B, const uint8_t* sB,
                                    int fmtB, const void* gu_bf16, int64_t M, int64_t I, int64_t T, void* dgu_bf16,
                                    void* h_bf16, float* d_amax_dgu, void* stream);

/*
 * Workspace of the three linear-layer calls below, for one (M, N, K).  It holds the FP8 copies
 *   Xq [M,K], Wq [N,K], dYq [M,N], then 12 KB of scratch for the LLMQ_JIT_* flags, then
 *   Xq_t [K,M], Wq_t [K,N], dYq_t [N,M],
 * each starting at a multiple of 256 bytes.  llmq_fp8_linear_workspace_offsets() returns the byte offsets of
 * the copies in the order Xq, Xq_t, Wq, Wq_t, dYq, dYq_t.  Calls that carry LLMQ_NO_TRANSPOSE touch nothing
 * behind the scratch and accept a workspace of llmq_fp8_linear_workspace_bytes_no_transpose() bytes (half the
 * FP8 copies); calls that carry LLMQ_SHARE_TILES need llmq_fp8_linear_workspace_bytes_shared() bytes: the same
 * layout with a section for the binary32 pieces of shared tiles behind it (0-100 MB more, by the shapes).
 * The caller owns the workspace and may read the copies between calls.
 */
size_t llmq_fp8_linear_workspace_bytes(int64_t M, int64_t N, int64_t K);
size_t llmq_fp8_linear_workspace_bytes_no_transpose(int64_t M, int64_t N, int64_t K);
size_t llmq_fp8_linear_workspace_bytes_shared(int64_t M, int64_t N, int64_t K);
int llmq_fp8_linear_workspace_offsets(int64_t M, int64_t N, int64_t K, size_t offsets[6]);

/* `flags` of the linear calls: the named operand's FP8 copies are already in the workspace (written by
 * an earlier call with the same M, N, K and the same scale) and are not produced again.  The library takes the
 * caller's word for it: nothing in the workspace records what it holds, and a call that claims copies that are
 * not there computes on stale bytes and still returns LLMQ_OK.  The copies are both of the operand's: the row-major
 * one and, unless the call carries LLMQ_NO_TRANSPOSE, the transposed one.  A workspace filled by hand needs both, with
 * the same codes: the weight gradient reads one or the other of X and dY, whichever is faster at its sizes.  Weights are
 * quantized once per optimizer step and reused across micro-steps and in the backward pass (Section 3,
 * weight caching), and the backward pass reuses the forward's copies of X. */
#define LLMQ_REUSE_X  1
#define LLMQ_REUSE_W  2
#define LLMQ_REUSE_DY 4
/* Just-in-time scaling inside the call (Section 3 "Overview": the scale is found right before the conversion,
 * at the price of one extra kernel for the global reduction): the named operand's d_scale_* is then an OUTPUT.
 * The call runs the first stage of the absmax reduction over the operand and the quantize kernel finishes it,
 * so the scale, the FP8 bytes and everything downstream are bit-identical to llmq_amax followed by the call
 * with the scale given, with one launch less.  Not together with the operand's REUSE flag. */
#define LLMQ_JIT_X   8
#define LLMQ_JIT_W  16
#define LLMQ_JIT_DY 32
/* No transposed copies: the call writes only the row-major FP8 copies (Xq, Wq, dYq) and the backward GEMMs
 * read those T-major (see llmq_fp8_gemm), which saves one byte written per quantized element and half the
 * workspace: the sections Xq_t, Wq_t, dYq_t are neither written nor read and need not exist.  Copies made
 * under this flag can only be reused (LLMQ_REUSE_*) by calls that carry it too, copies made without it by
 * any call; results are bit-identical either way. */
#define LLMQ_NO_TRANSPOSE 64
/* The call's contraction may share the output tiles of a ragged last round among all compute units, as
 * llmq_fp8_gemm_with_scratch does (pieces along the contraction index, added in a fixed order by a second
 * launch: Section 3 "Reproducibility"; run to run the same bytes).  The planner shares only where it was
 * measured to win (long contractions with few left-over tiles), so most shapes are not affected at all; where it
 * shares, the binary32 sums are taken in another order than with whole tiles, so the BF16 results may differ in
 * the last bit from those of a call without the flag (both within the error bound of llmq_fp8_gemm_tn).  In a
 * block's sequence of contractions it measured +1 % (32B- and 14B-class shapes).  Not together with LLMQ_NO_TRANSPOSE
 * (LLMQ_ERR_FLAGS); the workspace must hold llmq_fp8_linear_workspace_bytes_shared() bytes. */
#define LLMQ_SHARE_TILES 128
/* The transposed copies Xq_t, Wq_t, dYq_t are stored in slabs of 128 contraction bytes (LLMQ_LAYOUT_SLABS of the
 * contraction that reads them) instead of as plain transposed tensors, wherever the quantizer can write them so
 * (the untransposed tensor has a multiple of 128 rows and of 256 columns, less than 0x70000000 elements; other
 * tensors keep the plain form): a 128 x 128 tile of a tensor then lands as one contiguous 16 KB piece of its
 * transposed copy instead of 128 pieces of 128 bytes, and every K step of a backward contraction reads one
 * contiguous piece per operand.  Results are the same bytes as without the flag.  Copies made under this flag can
 * only be reused (LLMQ_REUSE_*) by calls that carry it too (the producers that write FP8 directly make such
 * copies with llmq_swiglu_fwd_fp8_slabs and llmq_rmsnorm_apply_fp8_slabs), and copies made without it (or by
 * llmq_swiglu_fwd_fp8 and llmq_rmsnorm_apply_fp8) only by calls without it.  Not together with
 * LLMQ_NO_TRANSPOSE (LLMQ_ERR_FLAGS). */
#define LLMQ_SLAB_COPIES 256

/*
 * Forward: Y[M,N] = X[M,K] W[N,K]^T in FP8 (E4M3 x E4M3), BF16 out.
 * Quantizes X and W (both layouts each, unless LLMQ_REUSE_X / LLMQ_REUSE_W; row-major only under
 * LLMQ_NO_TRANSPOSE) with the given scales, then
 * runs the contraction on Xq and Wq.  d_amax_y may be NULL.
 */
int llmq_fp8_linear_fwd(const void* X, const void* W, int64_t M, int64_t N, int64_t K,
                        float* d_scale_x, float* d_scale_w,
                        void* Y, float* d_amax_y, void* ws, size_t ws_bytes, int flags, void* stream);

/*
 * Input gradient: dX[M,K] = dY[M,N] W[N,K].  dY is quantized to fmt_dy (E5M2 or E4M3; the paper tried
 * both, Section 5 Scenario 1) unless LLMQ_REUSE_DY; W unless LLMQ_REUSE_W.  Contraction over N on dYq and
 * Wq_t (on Wq read T-major under LLMQ_NO_TRANSPOSE).  W and dY pointers are not read for operands whose REUSE flag is set (and may then be NULL).
 */
int llmq_fp8_linear_dgrad(const void* dY, const void* W, int64_t M, int64_t N, int64_t K,
                          float* d_scale_dy, float* d_scale_w, int fmt_dy,
                          void* dX, float* d_amax_dx, void* ws, size_t ws_bytes, int flags, void* stream);

/*
 * Weight gradient: dW[N,K] = dY[M,N]^T X[M,K] (accumulate != 0: dW += ..., in BF16).  Contraction over M on
 * dYq_t and Xq_t, or on dYq and Xq read T-major (under LLMQ_NO_TRANSPOSE, and for values of M that are no multiples of 64
 * wherever that is faster): an operand whose REUSE flag is set has both of its copies in the workspace.
 */
int llmq_fp8_linear_wgrad(const void* dY, const void* X, int64_t M, int64_t N, int64_t K,
                          float* d_scale_dy, float* d_scale_x, int fmt_dy,
                          void* dW, int accumulate, void* ws, size_t ws_bytes, int flags, void* stream);

/*
 * Scale from an absmax that a fused producer left on the device (the d_amax_* outputs of the calls above):
 *   d_scale[0] = min(FMAX(fmt) / d_amax[0], FLT_MAX), 1 if d_amax[0] == 0: the same rule and rounding as llmq_amax.
 */
int llmq_scale_from_amax(const float* d_amax, int fmt, float* d_scale, void* stream);

/*
 * SwiGLU with the extra outputs of the FP8 pipeline (Section 3, kernel-fusion paragraph: every
 * non-linearity also returns the absmax of its result; Section 3 "Activation checkpointing": with the
 * absmax known, as in recomputation during backward, the FP8 conversion is fused into the non-linearity).
 *
 *   GU [M, 2I] BF16, the output of the gate+up projection: columns [0, I) are the gate g, columns
 *   [I, 2I) the up branch u.   h[m,i] = bf16( silu(g) * u ),  silu(g) = g * sg,  sg = 1 / (1 + e^-g).
 *   The value is evaluated in IEEE binary32, operation by operation (so that the BF16 bits, and with them
 *   the absmax and the FP8 codes, are reproducible anywhere):
 *     a = -min(max(g, -100), 86);  n = rint(a * LOG2E);  r = fma(n, -LN2_HI, a);  r = fma(n, -LN2_LO, r);
 *     p = 1 + r(1 + r(1/2 + r(1/6 + r(1/24 + r(1/120 + r/720)))))  (Horner, one fma per level);
 *     e = p * 2^n;  sg = 1 / (1 + e);  h = bf16( (g * sg) * u ),  one RNE rounding to BF16.
 *   LOG2E, LN2_HI, LN2_LO, 1/k! are the binary32 numbers nearest to log2 e, ln 2, ln 2 - LN2_HI, 1/k!.
 *   Against the exact function the result is within half a BF16 ulp (+ 2^-20 relative); for g <= -89,
 *   where |silu(g)| < 2^-121, it is +-0.  Non-finite inputs are outside the contract.
 *
 * llmq_swiglu_fwd: writes h [M, I] (BF16), d_amax_h[0] = max |h| and, if d_scale_h is not NULL, the scale of
 *   h for format fmt (as llmq_amax would for h, bit for bit).  ws: device scratch of at least
 *   llmq_swiglu_workspace_bytes(M, I) bytes, 16-byte aligned, contents irrelevant on entry (per-workgroup
 *   partial results, reduced by a second kernel: no atomics).
 * llmq_swiglu_fwd_fp8: the scale is known (kept from the forward pass): writes q [M, I] = the FP8 codes
 *   llmq_quantize_fp8 would produce from h with *d_scale_h, q_t [I, M] their transposed copy if not NULL,
 *   and h itself only if h_bf16 is not NULL.  With q and q_t pointing at the Xq / Xq_t sections of a linear
 *   workspace, the down projection then runs with LLMQ_REUSE_X.
 * llmq_swiglu_fwd_fp8_slabs: the same with q_t (required) in slabs of 128 contraction bytes, exactly what
 *   llmq_quantize_fp8_slabs writes from h (byte (i, m) of the transposed tensor at (m / 128) I 128 + i 128 + m % 128),
 *   for a down projection that runs with LLMQ_REUSE_X | LLMQ_SLAB_COPIES.  M % 128 == 0, I % 256 == 0 and
 *   M I < 0x70000000 (the tensors such a linear call keeps in slabs), else LLMQ_ERR_SHAPE.
 * llmq_swiglu_bwd: dh [M, I], GU [M, 2I] -> dGU [M, 2I] (same column layout):
 *     dGU[m, I+i] = bf16( dh * (g * sg) ),   dGU[m, i] = bf16( ((dh * u) * sg) * fma(g, 1 - sg, 1) ),
 *   plus absmax and, if wanted, scale (format fmt) of dGU, which is the dY of the gate+up projection.
 * M, I >= 1, I < 2^24; GU, h, dh, dGU 16-byte aligned.  I % 8 == 0 (every row aligned) and M % 4 == 0 are fastest, with
 * q_t M % 128 == 0 and I % 256 == 0; other shapes take the same arithmetic with guarded edges.
 */
size_t llmq_swiglu_workspace_bytes(int64_t M, int64_t I);
int llmq_swiglu_fwd(const void* gu_bf16, int64_t M, int64_t I, void* h_bf16, int fmt,
                    float* d_amax_h, float* d_scale_h, void* ws, size_t ws_bytes, void* stream);
int llmq_swiglu_fwd_fp8(const void* gu_bf16, int64_t M, int64_t I, const float* d_scale_h, int fmt,
                        uint8_t* q, uint8_t* q_t, void* h_bf16, void* stream);
int llmq_swiglu_fwd_fp8_slabs(const void* gu_bf16, int64_t M, int64_t I, const float* d_scale_h, int fmt,
                              uint8_t* q, uint8_t* q_t, void* h_bf16, void* stream);
int llmq_swiglu_bwd(const void* dh_bf16, const void* gu_bf16, int64_t M, int64_t I, void* dgu_bf16, int fmt,
                    float* d_amax_dgu, float* d_scale_dgu, void* ws, size_t ws_bytes, void* stream);

/*
 * RMSNorm joined with the residual addition, with the extra outputs of the FP8 pipeline (Section 3,
 * kernel-fusion paragraph: one kernel for both, which also returns the absmax of the normalised output;
 * Section 3 "Activation checkpointing": statistics kept from the forward pass let the recomputation emit
 * FP8 directly).
 *
 *   res'[m,c] = bf16( res[m,c] + x[m,c] )       one binary32 addition, one RNE rounding; the stored stream
 *   rstd[m]   = 1 / sqrt( (1/C) sum_c res'[m,c]^2 + eps )     of the BF16-rounded res'; binary32
 *   y[m,c]    = bf16( (res'[m,c] * rstd[m]) * w[c] )          two binary32 multiplications, one rounding
 *   res, x, res', y [M, C] BF16; w [C] BF16; rstd [M] float.
 *
 * llmq_rmsnorm_fwd: x may be NULL (no addition: res is normalised as it is and res_out is ignored);
 *   otherwise res_out receives res' and may be the same buffer as res (in place).  Writes y, rstd (kept for
 *   the backward pass / recomputation), d_amax_y = max |y| and, if not NULL, d_scale_y for format fmt, both
 *   bit-identical to llmq_amax of y.  The row sum runs in binary32 in an order that depends on C alone, so
 *   rstd is reproducible from run to run and batch to batch but only equal to the exact value within 2^-20 relative; y then is the
 *   formula above evaluated with that rstd.  ws: at least llmq_rmsnorm_workspace_bytes(M) bytes, 16-byte
 *   aligned, contents irrelevant (per-workgroup partial absmax; no atomics).
 * llmq_rmsnorm_apply_fp8: the recompute path.  res (the stored stream), w, rstd and the scale of y are
 *   given; writes q [M, C] = the FP8 codes llmq_quantize_fp8 would produce from y with *d_scale_y, their
 *   transposed copy q_t [C, M] if not NULL, and y itself only if y_bf16 is not NULL.  Element-wise, hence
 *   reproducible bit for bit from its inputs.  rstd must be 16-byte aligned.
 * llmq_rmsnorm_apply_fp8_slabs: the same with q_t (required) in slabs of 128 contraction bytes, as
 *   llmq_quantize_fp8_slabs writes it from y, for a linear call with LLMQ_REUSE_X | LLMQ_SLAB_COPIES.
 *   M % 128 == 0, C % 256 == 0 and M C < 0x70000000, else LLMQ_ERR_SHAPE.
 * M, C >= 1, C < 2^24.  C % 8 == 0 is fastest; rows of C <= 16384 are read once, wider and narrow ragged ones twice.
 * The recompute calls are fastest with M % 128 == 0 and C % 256 == 0 (M % 4 == 0 and C % 8 == 0 without q_t).
 */
size_t llmq_rmsnorm_workspace_bytes(int64_t M);
int llmq_rmsnorm_fwd(const void* res_bf16, const void* x_bf16, const void* w_bf16, int64_t M, int64_t C,
                     float eps, void* res_out_bf16, void* y_bf16, float* rstd, int fmt, float* d_amax_y,
                     float* d_scale_y, void* ws, size_t ws_bytes, void* stream);
int llmq_rmsnorm_apply_fp8(const void* res_bf16, const void* w_bf16, const float* rstd, int64_t M, int64_t C,
                           const float* d_scale_y, int fmt, uint8_t* q, uint8_t* q_t, void* y_bf16,
                           void* stream);
int llmq_rmsnorm_apply_fp8_slabs(const void* res_bf16, const void* w_bf16, const float* rstd, int64_t M,
                                 int64_t C, const float* d_scale_y, int fmt, uint8_t* q, uint8_t* q_t,
                                 void* y_bf16, void* stream);

/*
 * The same norm in front of a contraction with block scales, and its gradient.
 *
 * llmq_rmsnorm_fwd_fp8_blocks: res' as llmq_rmsnorm_fwd leaves it, rstd = 1 / sqrt(mean of the squares + eps) with sums in binary64 and one rounding (llmq_rmsnorm_fwd has sums in binary32), and
 *   y = bf16( (res' rstd) w ) as llmq_quantize_fp8_blocks with block_rows 1 would write it, bit for bit:
 *   q [M, C] and s: codes of y with a scale for each row and 128 columns;   q_t [C, M] and s_t: of the transposed tensor, a scale for each column and 128 rows.
 *   q and s may be NULL together, or q_t and s_t; one pair must be there.  Without q_t (serving) it is one pass.  y is rounded to BF16 before its codes are made, so that both copies
 *   are made from the same values; y_bf16 receives them if it is not NULL.  x, res_out as in llmq_rmsnorm_fwd (x may be NULL, res_out may be res).  No workspace, no absmax.
 *   0 <= eps, finite (LLMQ_ERR_VALUE).  M < 2^25, C < 2^24.  All pointers 16-byte aligned, rstd too.
 * llmq_rmsnorm_bwd: dy [M, C], the gradient of y; dres [M, C] or NULL, the gradient of the stored stream res' from where else it is read; res [M, C] = res' (the stored stream); w, rstd:
 *     n = res' rstd,  g = dy w:    dx[m,c] = bf16( dres + rstd (g - n mean_c(g n)) ),    dw[c] = sum_m dy[m,c] n[m,c]
 *   dx [M, C] BF16 is the gradient of both terms of the addition; it may be dy or dres itself.  dw [C] float, added to if accumulate != 0; NULL: not wanted.  d_amax, d_scale [1] float or NULL: absmax of dx
 *   and its scale for fmt, bit for bit as llmq_amax of dx has them.  Sums in binary32, in an order that the sizes alone decide.
 *   ws: llmq_rmsnorm_bwd_workspace_bytes(M, C) bytes, 16-byte aligned, contents irrelevant (calls that may overlap on the device, graphs among them, need different ones); NULL if
 *   neither dw nor d_amax is wanted.  C < 2^24; rows of C <= 16384 are read once, wider ones take a slow kernel.  C % 8 == 0 is fastest.
 */
int llmq_rmsnorm_fwd_fp8_blocks(const void* res_bf16, const void* x_bf16, const void* w_bf16, int64_t M, int64_t C,
                                float eps, void* res_out_bf16, float* rstd, int fmt, uint8_t* q, uint8_t* s,
                                uint8_t* q_t, uint8_t* s_t, void* y_bf16, void* stream);
size_t llmq_rmsnorm_bwd_workspace_bytes(int64_t M, int64_t C);
int llmq_rmsnorm_bwd(const void* dy_bf16, const void* dres_bf16, const void* res_bf16, const void* w_bf16,
                     const float* rstd, int64_t M, int64_t C, void* dx_bf16, float* dw, int accumulate, int fmt,
                     float* d_amax, float* d_scale, void* ws, size_t ws_bytes, void* stream);

/*
 * RMSNorm of every query and key head joined with the rotation by position, between the QKV projection and attention, and the gradient of both, which
 * is the dY of the QKV projection.
 *
 *   qkv [M, (Hq + 2 Hkv) D] BF16: a row is Hq query heads, Hkv key heads and Hkv value heads of D values each.
 *   n[i] = (x[i] rstd) w[i],   rstd = 1 / sqrt(mean of x^2 over the head + eps),   w = wq or wk, [D] BF16; both NULL: no norm, n = x.  0 <= eps, finite (LLMQ_ERR_VALUE)
 *   the first `rot` values of a head (even, 0 .. D) are turned in pairs, the others stay:  interleaved == 0: i with i + rot/2;  1: 2 i with 2 i + 1
 *     y_a = n_a cos t - n_b sin t,   y_b = n_b cos t + n_a sin t,   t = d_positions[m] d_inv_freq[pair]
 *   d_positions [M] int64 (any value; those of a cache go on where it ends), d_inv_freq [rot/2] double, radians per position, finite.  The angle is found in 64-bit
 *   fractions of a turn: off by at most |position| (2^-52 of the frequency + 2^-64 of a turn; 2^-54 of a turn for negative frequencies) + 2^-32 of a turn, for any position; its sine and cosine by 2^-22.
 *   Sums and everything else in binary32, one rounding to BF16.
 *
 * llmq_qk_norm_rope_fwd: q [M, Hq D] and k [M, Hkv D] BF16; rstd [M, Hq + Hkv] float, kept for the backward pass, or NULL (not with NULL weights: ignored).
 *   The values V stay where they are.  q and k may be the query and key columns of qkv themselves (in place).
 * llmq_qk_norm_rope_bwd: dq, dk of q and k, dv of V (or NULL: V's columns of dqkv already hold it, or dv points at them) -> dqkv, laid out as qkv, and
 *     g = dy turned back;   dw[i] = sum over rows and heads of g[i] x[i] rstd;   dx[i] = rstd (g[i] w[i] - x[i] rstd mean(g w x rstd))
 *   dwq, dwk [D] float, added to if accumulate != 0; NULL: not wanted (and there are none without a norm: LLMQ_ERR_NULL).  They share no memory (LLMQ_ERR_VALUE): the gradient of one weight for both is the
 *   sum of the two.  The sums are taken in an order that depends on the sizes alone.  d_amax, d_scale [1] float or
 *   NULL: absmax of all of dqkv and its scale for fmt, bit for bit as llmq_amax of dqkv has them.  qkv and rstd are not read without a norm (and may be NULL).
 *   dq and dk may be the query and key columns of dqkv.  ws: llmq_qk_norm_rope_workspace_bytes bytes, 16-byte aligned, contents irrelevant (calls that may overlap on
 *   the device, graphs among them, need different ones); NULL if neither dw nor d_amax is wanted.
 * *_stride: elements from row to row, at least a row's width.  Rows may start at any element (2-byte aligned); D and rot multiples of 8 (D up to 512) with rows that
 * start at multiples of 8 bytes are fast, others take a slow kernel.  M, Hq, Hkv >= 1, heads up to 65536, 1 <= D <= 1024.
 */
int llmq_qk_norm_rope_fwd(const void* qkv_bf16, int64_t qkv_stride, int64_t M, int Hq, int Hkv, int D,
                          const void* wq_bf16, const void* wk_bf16, float eps, const int64_t* d_positions,
                          const double* d_inv_freq, int rot, int interleaved, void* q_bf16, int64_t q_stride,
                          void* k_bf16, int64_t k_stride, float* rstd, void* stream);
size_t llmq_qk_norm_rope_workspace_bytes(int64_t M, int Hq, int Hkv, int D);
int llmq_qk_norm_rope_bwd(const void* dq_bf16, int64_t dq_stride, const void* dk_bf16, int64_t dk_stride,
                          const void* dv_bf16, int64_t dv_stride, const void* qkv_bf16, int64_t qkv_stride,
                          int64_t M, int Hq, int Hkv, int D, const void* wq_bf16, const void* wk_bf16,
                          const float* rstd, const int64_t* d_positions, const double* d_inv_freq, int rot,
                          int interleaved, void* dqkv_bf16, int64_t dqkv_stride, float* dwq, float* dwk,
                          int accumulate, int fmt, float* d_amax, float* d_scale, void* ws, size_t ws_bytes,
                          void* stream);

/*
 * One AdamW step over any number of tensors in one launch, from the gradients the calls above leave (BF16 weight gradients, binary32 gradients of norm weights) to the
 * weights they read.
 *
 *   g' = g s                        s = *d_grad_scale (a clipping factor, say), 1 if it is NULL; where it is not finite the whole step is skipped and nothing is written
 *   m' = m b1 + g' (1 - b1)         v' = v b2 + g'^2 (1 - b2)
 *   w' = (w - w lr weight_decay) - (m' / (sqrt(v') / sqrt(1 - b2^step) + eps)) (lr / (1 - b1^step))        LLMQ_ADAMW_NO_DECAY: without the decay
 *   in binary32, each operation rounded by itself; the factors made of b1, b2, lr and step in binary64 and rounded once.
 *
 * llmq_adamw_tensor, all pointers device memory, each array of n >= 1 elements, 16-byte aligned (the scales: any).  No array that is written shares memory with
 * another of the call (LLMQ_ERR_VALUE from llmq_adamw_plan: a tensor that is named twice, say):
 *   w_bf16, w_f32   the weights: BF16 alone;  binary32 alone;  or both: w_f32 is the master copy, which is stepped, and w_bf16 receives it rounded to nearest
 *                   even.  BF16 alone is rounded to nearest even, or with LLMQ_ADAMW_STOCHASTIC up or down with the probability that keeps the mean.
 *   grad            BF16, or binary32 with LLMQ_ADAMW_GRAD_F32.
 *   m, v            binary32, zeros before the first step.  LLMQ_ADAMW_STATES_8BIT: one byte each, E4M3 codes of m and of sqrt(v) with m_scale and v_scale [ceil(n / 128)], a
 *                   power-of-two scale for each 128 elements as llmq_quantize_fp8_blocks has them; codes 0 and scales 127 before the first step.  Codes are rounded up or
 *                   down with the probability that keeps the mean, to 2^-16 of their distance (but a root above 0 stays above 0: at least the smallest code, 2^-18 to 2^-17 of the block's largest
 *                   root, so weights whose gradients are below that move less than they would); of a root below 2^-6, and of all for beta2 > 31/32, the mean of its
 *                   square, without which v would grow by its rounding; up to 31/32 the others' growth is 4 % of v at most.  A gradient that is not finite makes
 *                   its whole block NaN.
 *   d_amax          [1] float or NULL: absmax of the new w_bf16 (canonical NaN as llmq_amax), of all tensors that name the same word: the next quantization of these
 *                   weights then needs no pass of its own (llmq_scale_from_amax).  The word lies in no array of the call, read or written (llmq_adamw_plan does not look at that; llmq.py refuses it).
 *   first_counter   number of the tensor's first element among all that are rounded at random (>= 0): element i takes its bits from first_counter + i, the seed and the step.
 *                   Tensors should not share numbers.  Same inputs, same bytes.
 *
 * llmq_adamw_plan (host code): checks `count` tensors and writes the table that a step reads into `plan`, llmq_adamw_plan_bytes bytes of HOST memory, which the caller copies to
 *   device memory (16-byte aligned) once; info [4]: host words that llmq_adamw_step takes back.  The plan holds as long as the pointers do.  Making one sorts the arrays and writes
 *   8 bytes for every 1024 elements: 0.2 to 1 ms with the copy for 8 tensors of 233 million elements together, 0.6 ms for 96 small ones through llmq.py, so gradients keep their place from step to step.
 * llmq_adamw_hyper (host code): the numbers of a step (1, 2, ...) as LLMQ_ADAMW_HYPER_WORDS 32-bit words.  0 <= beta < 1, lr and weight_decay >= 0, eps > 0 in binary32, and eps and
 *   the factors of a step finite there, else LLMQ_ERR_VALUE.
 * llmq_adamw_step: exactly one of hyper (HOST words, read during the call) and d_hyper (the same words in device memory, read when the step runs: a captured step takes new ones with
 *   every replay) is given.
 */
#define LLMQ_ADAMW_GRAD_F32    1
#define LLMQ_ADAMW_STATES_8BIT 2
#define LLMQ_ADAMW_NO_DECAY    4
#define LLMQ_ADAMW_STOCHASTIC  8
#define LLMQ_ADAMW_HYPER_WORDS 10
typedef struct llmq_adamw_tensor {
    void* w_bf16;
    float* w_f32;
    const void* grad;
    void *m, *v;
    uint8_t *m_scale, *v_scale;
    float* d_amax;
    int64_t n, first_counter;
    int flags;
} llmq_adamw_tensor;
size_t llmq_adamw_plan_bytes(const llmq_adamw_tensor* tensors, int64_t count);
int llmq_adamw_plan(const llmq_adamw_tensor* tensors, int64_t count, void* plan, size_t plan_bytes, int64_t info[4]);
int llmq_adamw_hyper(int64_t step, double lr, double beta1, double beta2, double eps, double weight_decay,
                     uint64_t seed, uint32_t hyper[LLMQ_ADAMW_HYPER_WORDS]);
int llmq_adamw_step(const void* d_plan, const int64_t info[4], const uint32_t* hyper, const void* d_hyper,
                    const float* d_grad_scale, void* stream);

/*
 * Peak calibration (the paper's appendix "A note on MFU" measures the attainable peak with a large-matmul
 * micro-benchmark instead of trusting the spec sheet).  Both calls only enqueue; the caller times them.
 *
 * llmq_calibrate_mfma: a register-only loop of the GEMM's FP8 MFMA instruction (v_mfma_f32_16x16x128_f8f6f4 in
 *   the 8 x 8 block pattern of a wave tile, one workgroup of 4 waves per CU, `iters` passes of 64 MFMAs per wave;
 *   the 32x32x64 form of the instruction sustains about a tenth less on random bits) with operand registers holding
 *   constants (random_bits == 0) or random FP8 bits (random_bits != 0; the matrix cores are power-limited and
 *   sustain a lower clock on random bits, as on real quantized data).  d_sink: [1] float, device, practically
 *   never written.  *flops (host pointer, may be NULL) receives the FLOP count of the launch.
 * llmq_calibrate_copy: plain device copy of `bytes` (multiple of 16, 16-byte aligned pointers): 2 * bytes of
 *   HBM traffic.
 */
/*
 * llmq_calibrate_gemm_phases: one E4M3 x E4M3 contraction (arguments as llmq_fp8_gemm_tn; R, C multiples of 256,
 *   T a multiple of 128) by the 256 x 256 tile kernel built with phase stamps: wave 0 of every workgroup writes
 *   the cycle counter into d_stamps[16 * workgroup + s] and the 100 MHz clock into d_stamps[16 * workgroup + 8 + s]
 *   (64-bit words) for s = 0 start, 1 first operand fragments in registers (end of the prologue), 2 end of the
 *   contraction loop, 4 last output store issued, 5 absmax done, 3 all stores completed.  Workgroup ids beyond the
 *   number of tiles leave their words untouched.  d_stamps: device, 8-byte aligned, at least
 *   llmq_calibrate_gemm_phases_bytes(R, C) bytes.  ieee_maximum != 0: the fused absmax as the library computes
 *   it (IEEE 754-2019 maximum); 0: the maxNum form it replaced, for comparison.  The results c and d_amax_c are
 *   those of llmq_fp8_gemm_tn.
 */
size_t llmq_calibrate_gemm_phases_bytes(int64_t R, int64_t C);
int llmq_calibrate_gemm_phases(const uint8_t* A, const uint8_t* B, int64_t R, int64_t C, int64_t T,
                               const float* d_scaleA, const float* d_scaleB, void* c_bf16, float* d_amax_c,
                               void* d_stamps, size_t stamps_bytes, int ieee_maximum, void* stream);
int llmq_calibrate_mfma(int fmtA, int fmtB, int random_bits, int iters, float* d_sink, double* flops,
                        void* stream);
int llmq_calibrate_copy(const void* src, void* dst, size_t bytes, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* LLMQ_H */
