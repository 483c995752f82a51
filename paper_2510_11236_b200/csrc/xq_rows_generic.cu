// Scalar kernel of attention over a whole cache for many query rows (prefix and cross attention): every supported shape,
// slow, the on-device cross-check of the tensor-core kernel; and the kernel that joins partial results.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <math_constants.h>

#include "xq_internal.h"
#include "xq_layout.cuh"

namespace xq {
namespace {

__device__ __forceinline__ float f16_f(uint16_t u) { return __half2float(__ushort_as_half(u)); }
__device__ __forceinline__ float io_f(uint16_t u, int f16) { return f16 ? f16_f(u) : __uint_as_float(((uint32_t)u) << 16); }

constexpr int ROW_WARPS = 4;

// A warp takes one row and one split of the tokens; lanes cover channels (d = lane + 32 j), and keep an online softmax.
template <int DPL>
__global__ void __launch_bounds__(ROW_WARPS * 32) rows_generic_kernel(const __grid_constant__ RowsParams p) {
  constexpr int D = DPL * 32;
  const Dims& dm = p.dm;
  const int lane = threadIdx.x & 31, split = blockIdx.y;
  const int Bq = dm.B * p.each;
  const long long row = (long long)blockIdx.x * ROW_WARPS + (threadIdx.x >> 5);
  if (row >= (long long)p.T * Bq * dm.Hq) return;
  const int hq = (int)(row % dm.Hq), u = (int)(row / dm.Hq % Bq) / p.each;
  const int bh = u * dm.Hkv + hq / dm.G, g = dm.g, NG = dm.NG;
  int S = p.n_q + p.r;
  if (p.lengths != nullptr) S = max(0, min(S, p.lengths[u]));
  int t0, t1;
  share_of(S, p.ns, split, t0, t1);
  const int bk = p.L.bk, bv = p.L.bv;
  const uint32_t* kc = p.L.k_codes + (size_t)bh * ((size_t)dm.nq_cap * D * bk / 32);
  const uint32_t* vc = p.L.v_codes + (size_t)bh * ((size_t)dm.nq_cap * D * bv / 32);
  const uint16_t* km = p.L.k_meta + (size_t)bh * (dm.nq_cap / g) * 2 * D;
  const uint16_t* vm = p.L.v_meta + (size_t)bh * dm.nq_cap * 2 * NG;
  const uint16_t* wk = p.L.win_k + (size_t)bh * dm.R * D;
  const uint16_t* wv = p.L.win_v + (size_t)bh * dm.R * D;
  const float scale2 = p.scale * 1.4426950408889634f;
  float q[DPL], acc[DPL], m = -CUDART_INF_F, l = 0.f;
#pragma unroll
  for (int j = 0; j < DPL; ++j) {
    acc[j] = 0.f;
    q[j] = io_f(p.q[row * D + lane + 32 * j], p.f16);
  }
  for (int t = t0; t < t1; ++t) {
    float kx[DPL], vx[DPL];
#pragma unroll
    for (int j = 0; j < DPL; ++j) {
      const int d = lane + 32 * j;
      if (t < p.n_q) {
        const CodePos pk = k_code_position(t, d, bk, D), pv = v_code_position(t, d, bv, D);
        const uint16_t* mk = km + (size_t)(t / g) * 2 * D;
        const int pos = k_meta_position(d, D);
        kx[j] = fmaf((float)((kc[pk.word] >> pk.bit) & ((1u << bk) - 1)), f16_f(mk[pos]), f16_f(mk[D + pos]));
        vx[j] = fmaf((float)((vc[pv.word] >> pv.bit) & ((1u << bv) - 1)), f16_f(vm[v_scale_index(t, d / g, NG)]),
                     f16_f(vm[v_zero_index(t, d / g, NG)]));
      } else {
        kx[j] = io_f(wk[(size_t)(t - p.n_q) * D + d], p.f16);
        vx[j] = io_f(wv[(size_t)(t - p.n_q) * D + d], p.f16);
      }
    }
    float x = 0.f;
#pragma unroll
    for (int j = 0; j < DPL; ++j) x = fmaf(q[j], kx[j], x);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
    x *= scale2;
    const float mn = fmaxf(m, x), corr = exp2f(m - mn), pe = exp2f(x - mn);
    l = l * corr + pe;
#pragma unroll
    for (int j = 0; j < DPL; ++j) acc[j] = acc[j] * corr + pe * vx[j];
    m = mn;
  }
#pragma unroll
  for (int j = 0; j < DPL; ++j) p.part_acc[(row * p.ns + split) * D + lane + 32 * j] = acc[j];
  if (lane == 0) {
    p.part_ml[(row * p.ns + split) * 2] = t1 > t0 && m == -CUDART_INF_F ? CUDART_NAN_F : m;  // (no logit is a number, nor is the result)
    p.part_ml[(row * p.ns + split) * 2 + 1] = l;
  }
}

// out = (sum_s acc_s 2^(m_s - M) + own 2^(lse - M)) / (sum_s l_s 2^(m_s - M) + 2^(lse - M)): a part without tokens has
// m = -infinity and counts nothing.  A warp takes a row, a lane D / 32 neighbouring channels.  Bound: trips to L2; the sums of the
// first JOIN_SPLITS splits are asked for together with the references, so that most calls make one.
constexpr int JOIN_SPLITS = 16;
template <int DPL>
__global__ void __launch_bounds__(256) join_kernel(const __grid_constant__ JoinParams p) {
  constexpr int D = DPL * 32;
  grid_dependents_go();
  const long long row = (long long)blockIdx.x * 8 + (threadIdx.x >> 5);
  const int lane = threadIdx.x & 31;
  const float2* ml = reinterpret_cast<const float2*>(p.part_ml) + row * p.ns;
  const float* acc = p.part_acc + row * p.ns * D + lane * DPL;
  grid_dependency_wait();
  if (row >= p.rows) return;
  const float lse = p.own != nullptr ? p.own_lse[row] : -CUDART_INF_F;
  float2 x[JOIN_SPLITS];
  float v[JOIN_SPLITS][DPL];
  auto fetch = [&](int s0) {
#pragma unroll
    for (int k = 0; k < JOIN_SPLITS; ++k) {
      const bool there = s0 + k < p.ns;
      x[k] = there ? ml[s0 + k] : make_float2(-CUDART_INF_F, 0.f);
#pragma unroll
      for (int j = 0; j < DPL; j += 2)
        *reinterpret_cast<float2*>(&v[k][j]) = there ? *reinterpret_cast<const float2*>(acc + (size_t)(s0 + k) * D + j) : make_float2(0.f, 0.f);
    }
  };
  fetch(0);
  float M = lse;
#pragma unroll
  for (int k = 0; k < JOIN_SPLITS; ++k) M = fmaxf(M, x[k].x);
  if (p.ns > JOIN_SPLITS) {
    for (int s = JOIN_SPLITS + lane; s < p.ns; s += 32) M = fmaxf(M, ml[s].x);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) M = fmaxf(M, __shfl_xor_sync(0xffffffffu, M, o));
  }
  float a[DPL], L = 0.f;
#pragma unroll
  for (int j = 0; j < DPL; ++j) a[j] = 0.f;
  auto add = [&](float m, float l, const float* y) {
    const bool none = m == -CUDART_INF_F;  // the sums are then not defined
    const float f = exp2f(m - M);
    L = none ? L : fmaf(l, f, L);
#pragma unroll
    for (int j = 0; j < DPL; ++j) a[j] = none ? a[j] : fmaf(y[j], f, a[j]);
  };
  for (int s0 = 0;;) {
#pragma unroll
    for (int k = 0; k < JOIN_SPLITS; ++k) add(x[k].x, x[k].y, v[k]);
    s0 += JOIN_SPLITS;
    if (s0 >= p.ns) break;
    fetch(s0);
  }
  if (p.own != nullptr) {
    float v[DPL];
#pragma unroll
    for (int j = 0; j < DPL; j += 2) *reinterpret_cast<float2*>(v + j) = *reinterpret_cast<const float2*>(p.own + row * D + lane * DPL + j);
    add(lse, 1.f, v);
  }
  const float inv = M == -CUDART_INF_F ? 0.f : 1.f / L;
#pragma unroll
  for (int j = 0; j < DPL; j += 2) {
    const float x = a[j] * inv, y = a[j + 1] * inv;
    const size_t at = row * D + lane * DPL + j;
    if (p.out_f32) {
      *reinterpret_cast<float2*>(reinterpret_cast<float*>(p.out) + at) = make_float2(x, y);
    } else if (p.f16) {
      *reinterpret_cast<__half2*>(reinterpret_cast<__half*>(p.out) + at) = __floats2half2_rn(x, y);
    } else {
      *reinterpret_cast<__nv_bfloat162*>(reinterpret_cast<__nv_bfloat16*>(p.out) + at) = __floats2bfloat162_rn(x, y);
    }
  }
}

}  // namespace

cudaError_t launch_rows_generic(const RowsParams& p, cudaStream_t st) {
  const long long rows = (long long)p.T * p.dm.B * p.each * p.dm.Hq;
  const dim3 grid((unsigned)((rows + ROW_WARPS - 1) / ROW_WARPS), p.ns);
  if (p.dm.D == 128) rows_generic_kernel<4><<<grid, ROW_WARPS * 32, 0, st>>>(p);
  else rows_generic_kernel<2><<<grid, ROW_WARPS * 32, 0, st>>>(p);
  return cudaGetLastError();
}

cudaError_t launch_join(const JoinParams& p, cudaStream_t st) {
  const dim3 grid((unsigned)((p.rows + 7) / 8));
  return p.D == 128 ? launch_dependent(join_kernel<4>, grid, dim3(256), 0, st, p) : launch_dependent(join_kernel<2>, grid, dim3(256), 0, st, p);
}

}  // namespace xq
