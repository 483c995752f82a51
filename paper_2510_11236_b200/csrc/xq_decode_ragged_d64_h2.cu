// Tensor-core decode kernels for head_dim 64 and sequences of their own lengths, two query heads per kv head.
#include "xq_decode_mma64.cuh"

namespace xq {
template cudaError_t launch_decode_ragged64_t<2, 1>(const DecodeParams&, cudaStream_t);
}  // namespace xq
