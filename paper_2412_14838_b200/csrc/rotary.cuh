// Rotary positions: of a head's first rot_dim dims, every pair (a, b) is turned by the angle pos * f_i,
//   (a, b) -> A (a cos - b sin, a sin + b cos),
// pairs being dims (i, i + rot_dim/2) or (2i, 2i+1); the gradient is the same with sin negated (A times the inverse turn).
//
// Angles are computed in turns (f_i / 2 pi, in 64 bits on the host): position times turns is exact to 2^-53 of its size, its
// whole part is dropped, and what is left goes to sincospif in 32 bits, with a correction.  A 32-bit angle would be off by 2^-24 of itself, 0.06
// radians at position 10^6.  The pair itself is turned in 32 bits and rounded once.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <type_traits>
#include "common.cuh"
#include "../../include/dkv.h"

namespace dkv {

// cos and sin of `turns` turns a position.  What the argument loses when it is rounded to 32 bits, up to 2^-25 of a half turn or two
// steps of the result, is added back to first order.
__device__ __forceinline__ void turn_of(int pos, double turns, float& c, float& s) {
  const double x = (double)pos * turns, y = 2.0 * (x - rint(x));
  const float hi = (float)y, lo = 3.14159265f * (float)(y - (double)hi);
  float c0, s0;
  sincospif(hi, &s0, &c0);
  c = fmaf(-lo, s0, c0);
  s = fmaf(lo, c0, s0);
}

template <typename T> __device__ __forceinline__ float to_float(T x);
template <> __device__ __forceinline__ float to_float<float>(float x) { return x; }
template <> __device__ __forceinline__ float to_float<__half>(__half x) { return __half2float(x); }
template <> __device__ __forceinline__ float to_float<__nv_bfloat16>(__nv_bfloat16 x) { return __bfloat162float(x); }
template <typename T> __device__ __forceinline__ T from_float(float x);
template <> __device__ __forceinline__ float from_float<float>(float x) { return x; }
template <> __device__ __forceinline__ __half from_float<__half>(float x) { return __float2half_rn(x); }
template <> __device__ __forceinline__ __nv_bfloat16 from_float<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }

// V values of type T that move together: 16 bytes, or one value.
template <typename T, int V>
struct alignas(sizeof(T) * V) Pack { T x[V]; };

struct RotateTensor { const void* in; void* out; long long in_b, in_h, in_t, out_b, out_h, out_t; int heads; };

struct RotateArgs {
  RotateTensor x[2];           // two tensors as one sequence of heads
  const int* pos;              // [batch][tokens]
  long long all;               // batch * tokens
  int tokens, pieces, rot_pieces, heads;
  int block_tokens, groups;    // tokens of a block, and ways its threads deal out the heads
  int rot, in_place;
  float amplitude, sign;
  double turns[128];
};

// (a, b) * (x, y) + (p, q) as one packed instruction each.
__device__ __forceinline__ float2 mul2(float2 a, float2 x) {
  float2 r;
  asm("{.reg .b64 p, q; mov.b64 p, {%2, %3}; mov.b64 q, {%4, %5}; mul.rn.f32x2 p, p, q; mov.b64 {%0, %1}, p;}" : "=f"(r.x), "=f"(r.y) : "f"(a.x), "f"(a.y), "f"(x.x), "f"(x.y));
  return r;
}
__device__ __forceinline__ float2 fma2(float2 a, float2 x, float2 c) {
  float2 r;
  asm("{.reg .b64 p, q, r; mov.b64 p, {%2, %3}; mov.b64 q, {%4, %5}; mov.b64 r, {%6, %7}; fma.rn.f32x2 p, p, q, r; mov.b64 {%0, %1}, p;}"
      : "=f"(r.x), "=f"(r.y) : "f"(a.x), "f"(a.y), "f"(x.x), "f"(x.y), "f"(c.x), "f"(c.y));
  return r;
}
// Values 2 i and 2 i + 1 of a pack.
template <typename T, int V>
__device__ __forceinline__ float2 two_of(const Pack<T, V>& p, int i) {
  if constexpr (sizeof(T) == 4) return make_float2(p.x[2 * i], p.x[2 * i + 1]);
  else if constexpr (std::is_same<T, __half>::value) return __half22float2(reinterpret_cast<const __half2*>(p.x)[i]);
  else { const unsigned int w = reinterpret_cast<const unsigned int*>(p.x)[i]; return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u)); }
}
template <typename T, int V>
__device__ __forceinline__ void set_two(Pack<T, V>& p, int i, float2 v) {
  if constexpr (sizeof(T) == 4) { p.x[2 * i] = v.x; p.x[2 * i + 1] = v.y; }
  else if constexpr (std::is_same<T, __half>::value) reinterpret_cast<__half2*>(p.x)[i] = __floats2half2_rn(v.x, v.y);
  else reinterpret_cast<__nv_bfloat162*>(p.x)[i] = __floats2bfloat162_rn(v.x, v.y);
}

// A block has a few tokens and all heads: it computes every (token, pair)'s cosine and sine once, into shared memory; then a thread
// has one piece of a token (V pairs, or 2 V dims that only move), keeps its cosines and sines in registers and turns the piece
// in every groups-th head, kRotateFlight heads' loads in flight.  Bound by HBM where there is much to do, by latency where there is
// one token.  A 32K prompt of 40 heads of 128 dims in bf16: 671 MB in 114 us, 5.9 TB/s (with cosines computed by every thread for
// sixteen heads 179).
constexpr int kRotateThreads = 256, kRotateFlight = 4, kRotateTokens = 16;
template <typename T, int V, bool kPairs>
__global__ void __launch_bounds__(kRotateThreads, 3)
rotate_kernel(const __grid_constant__ RotateArgs a) {
  using P = Pack<T, V>;
  extern __shared__ float2 turn_s[];                   // [token][pair], padded to whole 16 bytes and off the banks of the next token
  const int tid = threadIdx.x, half = a.rot / 2, row = (half + 1) / 2 * 2 + 2;
  const long long token0 = (long long)blockIdx.x * a.block_tokens;
  const int here = (int)min((long long)a.block_tokens, a.all - token0);
  pdl_launch();
  pdl_wait();
  for (int x = tid; x < here * half; x += kRotateThreads) {
    float c, s;
    turn_of(a.pos[token0 + x / half], a.turns[x % half], c, s);
    turn_s[x / half * row + x % half] = make_float2(c * a.amplitude, s * a.amplitude * a.sign);
  }
  __syncthreads();
  const int piece = tid % a.pieces, k = tid / a.pieces % a.block_tokens, group = tid / (a.pieces * a.block_tokens);
  if (k >= here || group >= a.groups) return;
  const bool turned = piece < a.rot_pieces;
  if (!turned && a.in_place) return;
  const long long b = (token0 + k) / a.tokens, t = (token0 + k) % a.tokens;
  float2 cs[V];
  if (turned)
#pragma unroll
    for (int i = 0; i < V; ++i) cs[i] = turn_s[k * row + piece * V + i];
  // where the two packs of the piece lie
  const int d0 = !turned ? a.rot + (piece - a.rot_pieces) * 2 * V : kPairs ? piece * 2 * V : piece * V, d1 = turned && !kPairs ? d0 + half : d0 + V;
  const int step = a.groups * gridDim.y;
  for (int h = group + a.groups * blockIdx.y; h < a.heads; h += step * kRotateFlight) {
    P x[kRotateFlight], y[kRotateFlight];
#pragma unroll
    for (int f = 0; f < kRotateFlight; ++f)
      if (h + f * step < a.heads) {
        const int at = h + f * step, second = at >= a.x[0].heads;
        const RotateTensor& r = a.x[second];
        const T* from = static_cast<const T*>(r.in) + b * r.in_b + (at - (second ? a.x[0].heads : 0)) * r.in_h + t * r.in_t;
        x[f] = *reinterpret_cast<const P*>(from + d0);
        y[f] = *reinterpret_cast<const P*>(from + d1);
      }
#pragma unroll
    for (int f = 0; f < kRotateFlight; ++f)
      if (h + f * step < a.heads) {
        const int at = h + f * step, second = at >= a.x[0].heads;
        const RotateTensor& r = a.x[second];
        T* to = static_cast<T*>(r.out) + b * r.out_b + (at - (second ? a.x[0].heads : 0)) * r.out_h + t * r.out_t;
        if (turned) {
          if constexpr (V == 1) {
            const float u = to_float(x[f].x[0]), w = to_float(y[f].x[0]);
            x[f].x[0] = from_float<T>(fmaf(u, cs[0].x, -w * cs[0].y));
            y[f].x[0] = from_float<T>(fmaf(w, cs[0].x, u * cs[0].y));
          } else if constexpr (kPairs) {               // (u, w) -> c (u, w) + s (-w, u)
#pragma unroll
            for (int i = 0; i < V; ++i) {
              P& p = i < V / 2 ? x[f] : y[f];
              const float2 v = two_of(p, i % (V / 2));
              set_two(p, i % (V / 2), fma2(v, make_float2(cs[i].x, cs[i].x), mul2(make_float2(-v.y, v.x), make_float2(cs[i].y, cs[i].y))));
            }
          } else {
#pragma unroll
            for (int i = 0; i < V / 2; ++i) {
              const float2 u = two_of(x[f], i), w = two_of(y[f], i), c = make_float2(cs[2 * i].x, cs[2 * i + 1].x), s = make_float2(cs[2 * i].y, cs[2 * i + 1].y);
              set_two(x[f], i, fma2(u, c, mul2(w, make_float2(-s.x, -s.y))));
              set_two(y[f], i, fma2(w, c, mul2(u, s)));
            }
          }
        }
        *reinterpret_cast<P*>(to + d0) = x[f];
        *reinterpret_cast<P*>(to + d1) = y[f];
      }
  }
}

}  // namespace dkv
