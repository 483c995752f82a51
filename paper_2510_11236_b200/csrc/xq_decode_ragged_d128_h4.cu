// Tensor-core decode kernels for head_dim 128 and sequences of their own lengths, three or four query heads per kv head.
#include "xq_decode_mma.cuh"

namespace xq {
template cudaError_t launch_decode_ragged_t<4>(const DecodeParams&, cudaStream_t);
}  // namespace xq
