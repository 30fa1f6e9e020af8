// Rotary positions: of a head's first rot_dim dims, every pair (a, b) is turned by the angle pos * f_i,
//   (a, b) -> A (a cos - b sin, a sin + b cos),
// pairs being dims (i, i + rot_dim/2) or (2i, 2i+1); the gradient is the same with sin negated (A times the inverse turn).
//
// Angles are computed in turns (f_i / 2 pi, in 64 bits on the host): position times turns is exact to 2^-53 of its size, its
// whole part is dropped, and what is left goes to sincospif in 32 bits.  A 32-bit angle would be off by 2^-24 of itself, 0.06
// radians at position 10^6.  The pair itself is turned in 32 bits and rounded once.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include "common.cuh"
#include "../../include/dkv.h"

namespace dkv {

// cos and sin of `turns` turns a position.
__device__ __forceinline__ void turn_of(int pos, double turns, float& c, float& s) {
  const double x = (double)pos * turns;
  sincospif((float)(2.0 * (x - rint(x))), &s, &c);
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
  long long threads;           // batch * tokens * pieces
  int tokens, pieces, rot_pieces, heads, heads_a_thread;
  int rot, pairs, in_place;    // pairs: neighbouring dims
  float amplitude, sign;
  double turns[128];
};

// A thread has one piece of a token (V pairs, or 2 V dims that only move) and turns it in heads_a_thread heads, so that cosines
// and sines stay in registers and kRotateFlight heads' loads are in flight.  Bound by HBM where there is much to do.
// grid (pieces of all tokens / threads, head groups).
constexpr int kRotateThreads = 128, kRotateFlight = 4;
template <typename T, int V>
__global__ void __launch_bounds__(kRotateThreads)
rotate_kernel(const __grid_constant__ RotateArgs a) {
  using P = Pack<T, V>;
  const long long id = (long long)blockIdx.x * kRotateThreads + threadIdx.x;
  pdl_launch();
  pdl_wait();
  if (id >= a.threads) return;
  const int piece = (int)(id % a.pieces);
  const long long token = id / a.pieces;
  const long long b = token / a.tokens, t = token % a.tokens;
  const bool turned = piece < a.rot_pieces;
  if (!turned && a.in_place) return;
  float c[V], s[V];
  int d0, d1;                  // where the two packs of the piece lie
  if (turned) {
    const int pos = a.pos[token];
#pragma unroll
    for (int i = 0; i < V; ++i) {
      turn_of(pos, a.turns[piece * V + i], c[i], s[i]);
      c[i] *= a.amplitude; s[i] *= a.amplitude * a.sign;
    }
    d0 = a.pairs ? piece * 2 * V : piece * V;
    d1 = a.pairs ? d0 + V : d0 + a.rot / 2;
  } else {
    d0 = a.rot + (piece - a.rot_pieces) * 2 * V;
    d1 = d0 + V;
  }
  const int h0 = blockIdx.y * a.heads_a_thread, h1 = min(a.heads, h0 + a.heads_a_thread);
  for (int h = h0; h < h1; h += kRotateFlight) {
    P x[kRotateFlight], y[kRotateFlight];
    T* to[kRotateFlight];
#pragma unroll
    for (int f = 0; f < kRotateFlight; ++f)
      if (h + f < h1) {
        const bool second = h + f >= a.x[0].heads;
        const RotateTensor& r = a.x[second];
        const int hh = h + f - (second ? a.x[0].heads : 0);
        const T* from = static_cast<const T*>(r.in) + b * r.in_b + hh * r.in_h + t * r.in_t;
        to[f] = static_cast<T*>(r.out) + b * r.out_b + hh * r.out_h + t * r.out_t;
        x[f] = *reinterpret_cast<const P*>(from + d0);
        y[f] = *reinterpret_cast<const P*>(from + d1);
      }
#pragma unroll
    for (int f = 0; f < kRotateFlight; ++f)
      if (h + f < h1) {
        if (turned) {
#pragma unroll
          for (int i = 0; i < V; ++i) {
            // pair i of the piece: (x[i], y[i]), or neighbours in x and then in y
            T& pa = a.pairs ? (2 * i < V ? x[f].x[(2 * i) % V] : y[f].x[(2 * i) % V]) : x[f].x[i];
            T& pb = V == 1 ? y[f].x[0] : a.pairs ? (2 * i < V ? x[f].x[(2 * i + 1) % V] : y[f].x[(2 * i + 1) % V]) : y[f].x[i];
            const float u = to_float(pa), w = to_float(pb);
            pa = from_float<T>(u * c[i] - w * s[i]);
            pb = from_float<T>(u * s[i] + w * c[i]);
          }
        }
        *reinterpret_cast<P*>(to[f] + d0) = x[f];
        *reinterpret_cast<P*>(to[f] + d1) = y[f];
      }
  }
}

}  // namespace dkv
