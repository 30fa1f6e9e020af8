// Merging partial results of attention: sums of weighted values relative to a reference (log2), and the sum of the weights.
#pragma once
#include "common.cuh"

namespace dkv {

// One 4-value piece x (query qi = x / (D/4)) of the warps' parked results, merged in warp order: value sums, and the
// query's (max, sum); max = -inf: no rows.
template <int D, int QB, int NW>
__device__ __forceinline__ float2 merge_warps(const float* part, const float2* ml, int x, float4& v) {
  const int qi = x / (D / 4), d = x % (D / 4) * 4;
  float mm = -INFINITY, l = 0.f;
  float2 p[NW];
#pragma unroll
  for (int w = 0; w < NW; ++w) { p[w] = ml[w * QB + qi]; mm = fmaxf(mm, p[w].x); }
  v = make_float4(0.f, 0.f, 0.f, 0.f);
  if (mm > -INFINITY) {
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      const float s = fast_exp2(p[w].x - mm);
      const float4 y = *reinterpret_cast<const float4*>(part + (w * QB + qi) * (D + 4) + d);
      v.x = fmaf(y.x, s, v.x); v.y = fmaf(y.y, s, v.y); v.z = fmaf(y.z, s, v.z); v.w = fmaf(y.w, s, v.w);
      l = fmaf(p[w].y, s, l);
    }
  }
  return make_float2(mm, l);
}

// Running merge of partial results (value sums relative to their max, max, sum).
struct DecodeMerge {
  float m = -INFINITY, l = 0.f;
  float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
  __device__ __forceinline__ void add(float2 ml, float4 y) {
    const float mn = fmaxf(m, ml.x);
    if (mn == -INFINITY) return;
    const float s0 = fast_exp2(m - mn), s1 = fast_exp2(ml.x - mn);
    v.x = v.x * s0 + y.x * s1; v.y = v.y * s0 + y.y * s1; v.z = v.z * s0 + y.z * s1; v.w = v.w * s0 + y.w * s1;
    l = l * s0 + ml.y * s1;
    m = mn;
  }
  __device__ __forceinline__ void store(float* out) const {
    *reinterpret_cast<float4*>(out) = make_float4(v.x / l, v.y / l, v.z / l, v.w / l);
  }
};

}  // namespace dkv
