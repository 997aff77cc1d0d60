// The kernels of contractions of E5M2 x E4M3 operands with block scales joined with a SwiGLU, backward.
#include "gemm_glu.h"

namespace llmq {
template void launch_glu<1, 0, kGluBackward>(const GluOperands&, const GluChoice&, hipStream_t, int);
}
