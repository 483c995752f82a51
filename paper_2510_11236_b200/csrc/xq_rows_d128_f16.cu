// Kernels of prefix and cross attention for head_dim 128, half precision.
#include "xq_rows.cuh"

namespace xq {
template cudaError_t launch_rows_t<128, true>(const RowsParams&, cudaStream_t);
}  // namespace xq
