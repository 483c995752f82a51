// Kernels of prefix and cross attention for head_dim 64, half precision.
#include "xq_rows.cuh"

namespace xq {
template cudaError_t launch_rows_t<64, true>(const RowsParams&, cudaStream_t);
}  // namespace xq
