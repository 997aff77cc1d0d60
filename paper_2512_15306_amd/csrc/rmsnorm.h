// Elements and rows of RMSNorm, shared by its forward kernels, the codes made from its result and its backward pass.
#pragma once
#include "llmq_device.h"
#include "llmq_kernels.h"

#pragma clang fp contract(off)

namespace llmq {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float v2f __attribute__((ext_vector_type(2)));

__device__ inline unsigned rn_pack(float lo, float hi) {
    v2f v = {lo, hi};
    return __builtin_bit_cast(unsigned, __builtin_convertvector(v, bf16x2));
}
__device__ inline float rn_lo(unsigned w) { return __uint_as_float(w << 16); }
__device__ inline float rn_hi(unsigned w) { return __uint_as_float(w & 0xFFFF0000u); }

__device__ inline float wave_sum_f32(float v) {
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) v += __shfl_xor(v, off, kWave);
    return v;
}

// y = bf16((r * rstd) * w) for the eight elements of one 16-byte vector
__device__ inline v4u normalize8(const v4u& r, float rstd, const v4u& w) {
    v4u o;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const float a = rn_lo(r[j]) * rstd, b = rn_hi(r[j]) * rstd;
        o[j] = rn_pack(a * rn_lo(w[j]), b * rn_hi(w[j]));
    }
    return o;
}

// The first `valid` of eight elements, zeros for the others: what lies behind the end of a row counts for nothing, also where
// 0 * rstd * w is NaN (a row whose squares underflow, eps = 0: rstd is infinite and the row's own results are too).
__device__ inline v4u keep_upto(v4u v, int valid) {
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] &= (2 * j < valid ? 0xFFFFu : 0u) | (2 * j + 1 < valid ? 0xFFFF0000u : 0u);
    return v;
}

}  // namespace llmq
