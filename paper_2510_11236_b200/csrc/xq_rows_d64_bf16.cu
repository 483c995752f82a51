// Kernels of prefix and cross attention for head_dim 64, bfloat16.
#include "xq_rows.cuh"

namespace xq {
template cudaError_t launch_rows_t<64, false>(const RowsParams&, cudaStream_t);
}  // namespace xq
