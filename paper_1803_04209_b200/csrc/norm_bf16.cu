// The norm kernels of bf16 values.
#include "norm_launch.cuh"

namespace cutoff {
namespace layers {
template bool run_norm<__nv_bfloat16>(const NormArgs&, bool, int, cudaStream_t);
template bool run_norm_grad<__nv_bfloat16>(NormFinishArgs&, const GradPlan&, bool, bool, bool, int64_t, cudaStream_t);
}  // namespace layers
}  // namespace cutoff
