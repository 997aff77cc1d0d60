// Argument checks that the C entry points share.
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "../../include/llmq.h"

namespace {

constexpr int64_t kMaxDim = (int64_t)1 << 31;        // per dimension
constexpr int64_t kMaxElems = (int64_t)1 << 40;      // per tensor

inline bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }
inline bool fmt_ok(int f) { return f == LLMQ_E4M3 || f == LLMQ_E5M2; }
inline bool dim_ok(int64_t d) { return d >= 1 && d < kMaxDim; }
inline size_t round256(size_t v) { return (v + 255) & ~(size_t)255; }

inline int num_cus() {
    static int cached = 0;                              // benign race: every thread computes the same value
    if (cached == 0) {
        int dev = 0, n = 0;
        if (hipGetDevice(&dev) != hipSuccess ||
            hipDeviceGetAttribute(&n, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || n <= 0)
            n = 256;
        cached = n;
    }
    return cached;
}

}  // namespace
