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

}  // namespace llmq
