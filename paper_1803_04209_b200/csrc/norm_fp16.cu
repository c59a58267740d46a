// The norm kernels of fp16 values.
#include "norm_launch.cuh"

namespace cutoff {
namespace layers {
template void run_norm<__half>(const NormArgs&, bool, cudaStream_t);
template void run_norm_grad<__half>(const NormFinishArgs&, const GradPlan&, bool, bool, bool, int, cudaStream_t);
}  // namespace layers
}  // namespace cutoff
