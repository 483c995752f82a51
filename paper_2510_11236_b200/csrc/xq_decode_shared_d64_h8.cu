// Tensor-core decode kernels for head_dim 64 and many rows that read one cache, five to eight rows per kv head.
#include "xq_decode_mma64.cuh"

namespace xq {
template cudaError_t launch_decode_shared64_t<4, 2>(const DecodeParams&, cudaStream_t);
template int decode_shared64_warps_t<4, 2>(int, int, int);
}  // namespace xq
