// The linear layer's kernels for bfloat16 tensors.
#include "linear_launch.cuh"

namespace e3j {
namespace layer {
template int linear_fwd<bf16>(LinArgs&, int, cudaStream_t);
template int linear_bwd<bf16>(LinArgs&, int, const BwdLayout&, void*, void*, void*, void*, cudaStream_t);
}  // namespace layer
}  // namespace e3j
