// The counters of a handle that start at zero (merge tickets, status word, code differences), and the mark that says so.
#include <algorithm>

#include "xq_internal.h"

namespace xq {
namespace {

constexpr int CLEAR_THREADS = 256;

// The mark is this one or a later one of the same handle.  (Marks of a handle are consecutive, of two handles far apart; what a
// buffer held before is neither but for one chance in 2^32.)
__device__ __forceinline__ bool marked(const HandleState* state, unsigned long long mark) {
  return state->mark - mark <= 0xffffffffull;
}

__global__ void __launch_bounds__(CLEAR_THREADS) clear_kernel(const HandleState* state, unsigned long long mark, unsigned int* tickets, size_t n,
                                                              unsigned long long* delta, size_t n_delta) {
  if (marked(state, mark)) return;
  const size_t first = (size_t)blockIdx.x * CLEAR_THREADS + threadIdx.x, step = (size_t)gridDim.x * CLEAR_THREADS;
  for (size_t i = first; i < n; i += step) tickets[i] = 0u;
  for (size_t i = first; i < n_delta; i += step) delta[i] = 0ull;
}

__global__ void mark_kernel(HandleState* state, unsigned long long mark) {
  if (marked(state, mark)) return;
  state->status = 0;
  state->mark = mark;
}

}  // namespace

cudaError_t launch_clear(HandleState* state, unsigned long long mark, unsigned int* tickets, size_t n, unsigned long long* delta, size_t n_delta,
                         cudaStream_t st) {
  const unsigned ctas = (unsigned)std::min<size_t>((n + CLEAR_THREADS - 1) / CLEAR_THREADS, 592);
  clear_kernel<<<std::max(1u, ctas), CLEAR_THREADS, 0, st>>>(state, mark, tickets, n, delta, n_delta);
  const cudaError_t e = cudaGetLastError();
  if (e != cudaSuccess) return e;
  mark_kernel<<<1, 1, 0, st>>>(state, mark);  // (a kernel of its own: a block of the other one may begin after all others)
  return cudaGetLastError();
}

}  // namespace xq
