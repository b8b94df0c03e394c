// Residual addition between two norms, backward: the kernel for rows of bf16, from the inputs.
#include "norm_bwd.cuh"

namespace mx {

template cudaError_t launch_norm_bwd<__nv_bfloat16, false>(const NormBwd &, const RowPlan &, bool, bool, bool, bool, bool, cudaStream_t);

}  // namespace mx
