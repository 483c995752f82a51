// Tensor-core decode kernels for head_dim 128 and many rows that read one cache, one row per kv head.
#include "xq_decode_mma.cuh"

namespace xq {
template cudaError_t launch_decode_shared_t<1>(const DecodeParams&, cudaStream_t);
template int decode_shared_warps_t<1>(int, int, int);
}  // namespace xq
