// Residual addition and RMSNorm whose result is FP8 with a power-of-two scale for every block of 128 (llmq_rmsnorm_fwd_fp8_blocks).
//
// HBM-bound.  A scale of the row-wise copy belongs to 128 values of a row, which the forward kernels have in registers: one pass (rmsnorm.hip), 4 bytes read and 2 + 1 written an
// element.  A scale of the transposed copy belongs to 128 rows, and a row's statistic to all of its columns: no workgroup holds both, so with a transposed copy there are two passes, one
// for the sum and its statistics, and the block quantizer's over tiles of 128 x 128 (quantize_blocks.hip), which norms what it loads: 4 + 2 bytes read, 2 + 1 + 1 written, of
// which the 2 read again come from the memory-side cache up to about 100 MB.  8192 x 3584 with both copies 48.5 us (6.0 TB/s in either pass), 1777 x 2880 16.2; 32 x 3584 along the
// rows alone 3.7 us.  (The norm and the quantizer one after the other write and read y besides, 118 MB at 8192 x 3584.)
#include "api_checks.h"
#include "llmq_kernels.h"

extern "C" int llmq_rmsnorm_fwd_fp8_blocks(const void* res_bf16, const void* x_bf16, const void* w_bf16, int64_t M, int64_t C, float eps, void* res_out_bf16, float* rstd, int fmt, uint8_t* q, uint8_t* s,
                                           uint8_t* q_t, uint8_t* s_t, void* y_bf16, void* stream) {
    if (!res_bf16 || !w_bf16 || !rstd || (x_bf16 && !res_out_bf16) || (!q && !q_t) || !q != !s || !q_t != !s_t) return LLMQ_ERR_NULL;
    if (!dim_ok(M) || !dim_ok(C) || C >= ((int64_t)1 << 24) || M >= ((int64_t)1 << 25) || M * C >= kMaxElems) return LLMQ_ERR_SHAPE;
    if (!(eps >= 0.0f && eps <= 3.402823466e+38f)) return LLMQ_ERR_VALUE;
    if (!fmt_ok(fmt)) return LLMQ_ERR_FORMAT;
    if (!aligned(res_bf16, 16) || !aligned(x_bf16, 16) || !aligned(w_bf16, 16) || (x_bf16 && !aligned(res_out_bf16, 16)) || !aligned(rstd, 16) || !aligned(q, 16) || !aligned(s, 16) ||
        !aligned(q_t, 16) || !aligned(s_t, 16) || !aligned(y_bf16, 16))
        return LLMQ_ERR_ALIGN;
    hipStream_t st = static_cast<hipStream_t>(stream);
    const bool rows_only = !q_t;
    const int status = llmq::launch_rmsnorm_rows(res_bf16, x_bf16, w_bf16, M, C, eps, x_bf16 ? res_out_bf16 : nullptr, rows_only ? y_bf16 : nullptr, rstd, fmt, rows_only ? q : nullptr,
                                                 rows_only ? s : nullptr, st, num_cus());
    if (status != 0 || rows_only) return status;
    return llmq::launch_norm_quantize_blocks(x_bf16 ? res_out_bf16 : res_bf16, w_bf16, rstd, M, C, fmt, q, s, q_t, s_t, y_bf16, st);
}
