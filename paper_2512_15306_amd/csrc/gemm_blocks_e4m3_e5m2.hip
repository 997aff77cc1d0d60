// The kernels of E4M3 x E5M2 operands with block scales.
#include "gemm_blocks.h"

namespace llmq {
template void launch_blocks<0, 1>(const BlocksOperands&, const BlocksPlan&, hipStream_t, int);
}
