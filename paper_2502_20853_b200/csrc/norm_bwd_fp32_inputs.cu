// Residual addition between two norms, backward: the kernel for rows of fp32, from the inputs.
#include "norm_bwd.cuh"

namespace mx {

template cudaError_t launch_norm_bwd<float, false>(const NormBwd &, const RowPlan &, bool, bool, bool, bool, bool, cudaStream_t);

}  // namespace mx
