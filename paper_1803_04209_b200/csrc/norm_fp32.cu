// The norm kernels of fp32 values.
#include "norm_launch.cuh"

namespace cutoff {
namespace layers {
template bool run_norm<float>(const NormArgs&, bool, int, cudaStream_t);
template bool run_norm_grad<float>(NormFinishArgs&, const GradPlan&, bool, bool, bool, int64_t, cudaStream_t);
}  // namespace layers
}  // namespace cutoff
