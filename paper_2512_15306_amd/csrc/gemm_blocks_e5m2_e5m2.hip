// The kernels of E5M2 x E5M2 operands with block scales.
#include "gemm_blocks.h"

namespace llmq {
template void launch_blocks<1, 1>(const BlocksOperands&, const BlocksPlan&, hipStream_t, int);
}
