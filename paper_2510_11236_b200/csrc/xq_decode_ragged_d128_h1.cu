// Tensor-core decode kernels for head_dim 128 and sequences of their own lengths, one query head per kv head.
#include "xq_decode_mma.cuh"

namespace xq {
template cudaError_t launch_decode_ragged_t<1>(const DecodeParams&, cudaStream_t);
}  // namespace xq
