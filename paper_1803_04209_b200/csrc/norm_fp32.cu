// The norm kernels of fp32 values.
#include "norm_launch.cuh"

namespace cutoff {
namespace layers {
template void run_norm<float>(const NormArgs&, bool, cudaStream_t);
template void run_norm_grad<float>(const NormFinishArgs&, const GradPlan&, bool, bool, bool, int, cudaStream_t);
}  // namespace layers
}  // namespace cutoff
