// Residual addition between two norms, forward: the kernel for rows of fp32.
#include "norm_fwd.cuh"

namespace mx {

template cudaError_t launch_norm_fwd<float>(NormFwd &, const RowPlan &, bool, bool, bool, cudaStream_t);

}  // namespace mx
