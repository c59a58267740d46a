// The norm kernels of fp16 values.
#include "norm_launch.cuh"

namespace cutoff {
namespace layers {
template bool run_norm<__half>(const NormArgs&, bool, int, cudaStream_t);
template bool run_norm_grad<__half>(NormFinishArgs&, const GradPlan&, bool, bool, bool, int64_t, cudaStream_t);
}  // namespace layers
}  // namespace cutoff
