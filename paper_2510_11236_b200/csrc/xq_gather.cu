// Copies of sequences between two caches, or within one: sequence b of the destination becomes sequence index[b] of the
// source, in all layers and regions (codes, scales and zero-points, windows).  Nothing is computed; bound: HBM.  A prompt of 8192
// tokens to 32 sequences, 8 layers (1.06 GB written): 175 us, 6.2 TB/s; 17 of 24 sequences of 4100 tokens to another cache (1.15 GB
// moved): 179 us, 6.4 TB/s.  In place, 16 beams of 1000 tokens, 32 layers: 45 to 58 us, by the share of them that changes.
//
// A region of a stream is one contiguous run of bytes, and the layouts of two caches differ in the streams' spacing alone,
// so a work item is a piece of (layer, region, kv head) with the sequences it goes to.
#include <algorithm>

#include "xq_internal.h"
#include "xq_layout.cuh"
#include "xq_mma.cuh"

namespace xq {
namespace {

constexpr int REGIONS = 6;         // as xq_region counts them
constexpr int COPY_THREADS = 256;
constexpr int COPY_VECS = 2;       // 16-byte vectors of a thread in a piece
constexpr int COPY_PIECE = COPY_THREADS * COPY_VECS * 16;
constexpr int PLACE_SMEM = 200 * 1024;

// bytes of a stream in use / from one stream to the next, region by region
__host__ __device__ inline size_t used_bytes(const GatherParams& p, const GatherLayer& L, int which) {
  switch (which) {
    case 0: return (size_t)L.n_q * p.D * L.bk / 8;
    case 1: return (size_t)((L.n_q + XQ_BATCH - 1) / XQ_BATCH) * (XQ_BATCH / 8) * p.D * L.bv;
    case 2: return (size_t)(L.n_q / p.g) * 4 * p.D;
    case 3: return (size_t)L.n_q * 4 * p.NG;
    default: return (size_t)L.r * p.D * 2;
  }
}
__host__ __device__ inline size_t stream_bytes(const GatherParams& p, const GatherLayer& L, int which, int cap) {
  switch (which) {
    case 0: return (size_t)cap * p.D * L.bk / 8;
    case 1: return (size_t)cap * p.D * L.bv / 8;
    case 2: return (size_t)(cap / p.g) * 4 * p.D;
    case 3: return (size_t)cap * 4 * p.NG;
    default: return (size_t)p.R * p.D * 2;
  }
}

// The pieces of a launch, counted through (layer, region): first[i] is the first item of (layer i / 6, region i % 6).
struct Items {
  uint32_t first[GATHER_MAX_LAYERS * REGIONS + 1];
  int parts;   // the sequences of a piece are dealt to this many items
  int lanes;   // in place: 16-byte lanes of an item
};
struct Launch {
  GatherParams g;
  Items it;
};

struct Place {
  const uint8_t* src;  // of kv head hk of sequence 0, at the piece
  uint8_t* dst;
  size_t src_stride, dst_stride;  // from one sequence to the next
  uint32_t bytes;                 // of the piece
  int part;
};
template <int PIECE_OF_LANES>
__device__ __forceinline__ Place place_of(const Launch& p, uint32_t item) {
  const int n = p.g.n_layers * REGIONS;
  int lo = 0, hi = n - 1;  // the last entry whose first item is at or before `item`
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (p.it.first[mid] <= item) lo = mid; else hi = mid - 1;
  }
  const GatherLayer& L = p.g.layer[lo / REGIONS];
  const int which = lo % REGIONS;
  const uint32_t piece = PIECE_OF_LANES ? (uint32_t)p.it.lanes * 16u : (uint32_t)COPY_PIECE;
  const size_t used = used_bytes(p.g, L, which), ss = stream_bytes(p.g, L, which, p.g.src_cap), ds = stream_bytes(p.g, L, which, p.g.dst_cap);
  const uint32_t pieces = (uint32_t)((used + piece - 1) / piece);
  uint32_t i = item - p.it.first[lo];
  Place r;
  r.part = (int)(i % (uint32_t)p.it.parts);
  i /= (uint32_t)p.it.parts;
  const uint32_t hk = i / pieces, at = i - hk * pieces;
  const size_t off = (size_t)at * piece;
  r.src = p.g.src + (size_t)L.src[which] * 256 + hk * ss + off;
  r.dst = p.g.dst + (size_t)L.dst[which] * 256 + hk * ds + off;
  r.src_stride = ss * p.g.Hkv;
  r.dst_stride = ds * p.g.Hkv;
  r.bytes = (uint32_t)(used - off < piece ? used - off : piece);
  return r;
}

// From one cache to another: a thread holds its vectors of a source while the sequences that follow have the same one.  A prompt
// that is forked into neighbouring sequences is read once by each item (of `parts` that share a piece's sequences); indices in
// turn, 0, 1, 0, 1, fetch it each time, from L2 where it still is there.
__global__ void __launch_bounds__(COPY_THREADS) gather_kernel(const __grid_constant__ Launch p) {
  const Place r = place_of<0>(p, blockIdx.x);
  int b0, b1;
  share_of(p.g.B_dst, p.it.parts, r.part, b0, b1);
  grid_dependency_wait();
  grid_dependents_go();
  uint4 v[COPY_VECS];
  int have = -1;
  for (int b = b0; b < b1; ++b) {
    const int s = p.g.index[b];
    if (s < 0 || s >= p.g.B_src) {
      if (threadIdx.x == 0 && blockIdx.x < (unsigned)p.it.parts) atomicExch(p.g.status, 1);
      continue;
    }
#pragma unroll
    for (int k = 0; k < COPY_VECS; ++k) {
      const uint32_t at = (k * COPY_THREADS + threadIdx.x) * 16;
      if (at < r.bytes && s != have) v[k] = *reinterpret_cast<const uint4*>(r.src + s * r.src_stride + at);
    }
    have = s;
#pragma unroll
    for (int k = 0; k < COPY_VECS; ++k) {
      const uint32_t at = (k * COPY_THREADS + threadIdx.x) * 16;
      if (at < r.bytes) *reinterpret_cast<uint4*>(r.dst + b * r.dst_stride + at) = v[k];
    }
  }
}

// Within one cache: a thread owns a 16-byte lane of all sequences.  It reads the sources of every sequence that changes
// before it writes any, so whatever the indices are no sequence is overwritten before it has been read.
__global__ void gather_place_kernel(const __grid_constant__ Launch p) {
  extern __shared__ __align__(16) uint8_t held[];  // [sequences that change][lanes] vectors, then their lists
  __shared__ int n_moved;
  const Place r = place_of<1>(p, blockIdx.x);
  const int lanes = p.it.lanes, B = p.g.B_dst;
  int* const moved = reinterpret_cast<int*>(held + (size_t)B * lanes * 16);  // sequences that change, any order; their sources
  if (threadIdx.x == 0) n_moved = 0;
  __syncthreads();
  grid_dependency_wait();
  grid_dependents_go();
  for (int b = threadIdx.x; b < B; b += blockDim.x) {
    const int s = p.g.index[b];
    if (s < 0 || s >= p.g.B_src) {
      if (blockIdx.x == 0) atomicExch(p.g.status, 1);
    } else if (s != b) {
      const int k = atomicAdd(&n_moved, 1);
      moved[k] = b;
      moved[B + k] = s;
    }
  }
  __syncthreads();
  const int n = n_moved, lane = threadIdx.x;
  const uint32_t at = lane * 16;
  if (lane >= lanes || at >= r.bytes) return;
  const uint32_t mine = (uint32_t)__cvta_generic_to_shared(held) + at, row = lanes * 16;
  for (int k = 0; k < n; ++k) cp_async16(mine + k * row, r.src + moved[B + k] * r.src_stride + at);
  cp_async_commit();
  cp_async_wait_all();
  for (int k = 0; k < n; ++k) *reinterpret_cast<uint4*>(r.dst + moved[k] * r.dst_stride + at) = lds128(mine + k * row);
}

}  // namespace

// 16-byte lanes of an item in place, 0: the sequences are too many
static int place_lanes(int B) {
  for (int lanes : {128, 32, 8})
    if ((size_t)B * (lanes * 16 + 8) <= (size_t)PLACE_SMEM) return lanes;
  return 0;
}
int gather_place_limit() { return PLACE_SMEM / (8 * 16 + 8); }

cudaError_t launch_gather(const GatherParams& g, cudaStream_t st, long long* launches) {
  const bool place = g.src == g.dst;
  Launch p;
  p.g = g;
  p.it.lanes = place ? place_lanes(g.B_dst) : 0;
  if (place && p.it.lanes == 0) return cudaErrorInvalidValue;
  const size_t piece = place ? (size_t)p.it.lanes * 16 : (size_t)COPY_PIECE;
  auto pieces = [&](int i) {
    const GatherLayer& L = g.layer[i / REGIONS];
    return (used_bytes(g, L, i % REGIONS) + piece - 1) / piece * g.Hkv;
  };
  const int n = g.n_layers * REGIONS;
  size_t total = 0;
  for (int i = 0; i < n; ++i) total += pieces(i);
  if (total == 0) return cudaSuccess;
  ++*launches;
  // enough items for several CTAs on every SM
  constexpr size_t ENOUGH = 148 * 8 * 2;
  p.it.parts = place ? 1 : (int)std::min<size_t>(g.B_dst, std::max<size_t>(1, (ENOUGH + total - 1) / total));
  if (total * p.it.parts > 0x7fffffffull) return cudaErrorInvalidValue;
  uint32_t at = 0;
  for (int i = 0; i < n; ++i) {
    p.it.first[i] = at;
    at += (uint32_t)(pieces(i) * p.it.parts);
  }
  p.it.first[n] = at;
  if (!place) return launch_dependent(gather_kernel, dim3(at), dim3(COPY_THREADS), 0, st, p);
  const size_t smem = (size_t)g.B_dst * (p.it.lanes * 16 + 8);
  const cudaError_t e = cudaFuncSetAttribute(gather_place_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, PLACE_SMEM);
  if (e != cudaSuccess) return e;
  return launch_dependent(gather_place_kernel, dim3(at), dim3((unsigned)std::max(32, p.it.lanes)), smem, st, p);
}

}  // namespace xq
