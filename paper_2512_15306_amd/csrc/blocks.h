// Blocks of 128 values in 8 bits with a power-of-two scale each (llmq_quantize_fp8_blocks, the 8-bit moments of llmq_adamw_step).
#pragma once
#include "llmq_device.h"

namespace llmq {

constexpr int kBlock = 128;

// Code of a block's scale: 2^(code - 127) is the smallest power of two that brings the block's largest magnitude to at most the format's largest
// value, 1.75 2^8 (E4M3) or 1.75 2^15 (E5M2), so nothing is clipped; not below 2^-127.  The magnitude as binary32 bits.  127 (no scale) for a block of zeros,
// 255 (which the matrix cores take for NaN) if an Inf or NaN is among the values.
template <int FMT>
__device__ inline unsigned scale_code(unsigned mag) {
    const int b = (int)(mag >> 23) - (FMT == 0 ? 8 : 15) + ((mag & 0x7FFFFFu) > 0x600000u ? 1 : 0);
    return mag >= 0x7F800000u ? 255u : mag == 0 ? 127u : (unsigned)(b < 0 ? 0 : b);
}

typedef __bf16 v2bf __attribute__((ext_vector_type(2)));
typedef short v2s __attribute__((ext_vector_type(2)));

// Two BF16 values divided by 2^(code - 127) as two codes in the low or high half of old.  The instruction reads the exponent of its scale, rounds to
// nearest even, and nothing it is given here is beyond the format's largest value.
template <int FMT, bool HIGH>
__device__ inline unsigned cvt_scaled(unsigned pair, unsigned code, unsigned old) {
    const float d = __uint_as_float(code << 23);
    if constexpr (FMT == 0) return __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(__builtin_bit_cast(v2s, old), __builtin_bit_cast(v2bf, pair), d, HIGH));
    else return __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf8_bf16(__builtin_bit_cast(v2s, old), __builtin_bit_cast(v2bf, pair), d, HIGH));
}
template <int FMT>
__device__ inline unsigned cvt_four(unsigned p0, unsigned p1, unsigned code) {
    return cvt_scaled<FMT, true>(p1, code, cvt_scaled<FMT, false>(p0, code, 0u));
}

// Where the code of a row's scale is kept in a K step of an operand: 128 rows at a time, row r of them at 8 (r % 16) + r / 16.
__device__ inline int64_t code_place(int64_t row) { return (row & ~(int64_t)127) + 8 * (row & 15) + ((row >> 4) & 7); }

// Maximum over each 16 lanes side by side, in all of them.  All lanes of the wave take part.
__device__ inline unsigned max_of_16_lanes(unsigned v) {
    unsigned t = (unsigned)__builtin_amdgcn_update_dpp(0, (int)v, 0xB1, 0xF, 0xF, false);      // quad_perm [1,0,3,2]
    v = v > t ? v : t;
    t = (unsigned)__builtin_amdgcn_update_dpp(0, (int)v, 0x4E, 0xF, 0xF, false);               // quad_perm [2,3,0,1]
    v = v > t ? v : t;
    t = (unsigned)__builtin_amdgcn_update_dpp(0, (int)v, 0x141, 0xF, 0xF, false);              // row_half_mirror
    v = v > t ? v : t;
    t = (unsigned)__builtin_amdgcn_update_dpp(0, (int)v, 0x140, 0xF, 0xF, false);              // row_mirror
    return v > t ? v : t;
}

}  // namespace llmq
