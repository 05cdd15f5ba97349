// The linear layer's kernels for float32 tensors.
#include "linear_launch.cuh"

namespace e3j {
namespace layer {
template int linear_fwd<float>(LinArgs&, int, cudaStream_t);
template int linear_bwd<float>(LinArgs&, int, const BwdLayout&, void*, void*, void*, void*, cudaStream_t);
}  // namespace layer
}  // namespace e3j
