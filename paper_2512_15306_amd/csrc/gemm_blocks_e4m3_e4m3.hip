// The kernels of E4M3 x E4M3 operands with block scales.
#include "gemm_blocks.h"

namespace llmq {
template void launch_blocks<0, 0>(const BlocksOperands&, const BlocksPlan&, hipStream_t, int);
}
