// Kernels of prefix and cross attention for head_dim 128, bfloat16.
#include "xq_rows.cuh"

namespace xq {
template cudaError_t launch_rows_t<128, false>(const RowsParams&, cudaStream_t);
}  // namespace xq
