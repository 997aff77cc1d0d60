// The kernels of contractions of E4M3 x E4M3 operands with block scales joined with a SwiGLU, backward.
#include "gemm_glu.h"

namespace llmq {
template void launch_glu<0, 0, kGluBackward>(const GluOperands&, const GluChoice&, hipStream_t, int);
}
