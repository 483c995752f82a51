// Results of the decode kernels' variants for many rows that read one cache (DecodeParams::shared): a row may have no token,
// and its result may have to be joined with the row's result over other tokens.
#pragma once
#include "xq_internal.h"
#include "xq_mma.cuh"

namespace xq {
namespace {

// no token of sequence b exists (the cache itself has some)
__device__ __forceinline__ bool no_tokens(const DecodeParams& p, int b) { return p.lengths != nullptr && p.lengths[b] <= 0; }

// (factor of the sums, factor of the row's own result): 1 / l and 0, or the shares that both have of one softmax.  M, l: the
// sums' reference and denominator.  (Where no logit is a number M is -infinity and l zero: the result is not a number.)
__device__ __forceinline__ float2 with_own(const DecodeParams& p, size_t row, bool none, float M, float l) {
  if (none) return make_float2(0.f, 0.f);
  const float inv = 1.f / l;
  if (p.own == nullptr) return make_float2(inv, 0.f);
  const float lse = M + log2f(l), own = p.own_lse[row], X = fmaxf(lse, own);
  const float a = exp2f(lse - X), c = exp2f(own - X), n = 1.f / (a + c);
  return make_float2(inv * (a * n), c * n);
}
// y and f times four channels, element `at`, of the own results
__device__ __forceinline__ float4 add_own(const DecodeParams& p, size_t at, float4 y, float f) {
  if (p.own == nullptr) return y;
  const float4 o = *reinterpret_cast<const float4*>(p.own + at);
  return make_float4(fmaf(o.x, f, y.x), fmaf(o.y, f, y.y), fmaf(o.z, f, y.z), fmaf(o.w, f, y.w));
}

}  // namespace
}  // namespace xq
