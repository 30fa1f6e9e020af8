// Attention of a few new queries a sequence over the rows of a cache in 8 bits (cache8.cuh):
//   out = sum_r p_r v_r / sum_r p_r,  p_r = exp(q . k_r / sqrt(D)),  rows r below the query's limit.
//
// What must move is every code once, D bytes of keys and D of values a row and head.  There are at most 64 query rows a head, 4
// or 8 in most models, so both products are warp-wide (mma.sync m16n8k16, fp16 in, fp32 sums): no 128-row tile to give to
// tcgen05.  Both code types are exact in fp16.  So are the queries, once a power of two has brought a row's largest number to 2^13 and
// above: what is 2^-17 of it and more keeps its 8 or 11 bits, what is smaller is off by 2^-38 of it.  Weights are split into two
// fp16 parts, 22 bits, which lie in the two halves of the 16-row operand where there are at most 8 query rows a head.
//   S = Q K^T   scaled by the page's key scale when it leaves the accumulators;
//   O = P V     a page's product is added to the result times its value scale, in units that follow the largest value scale met so far.
// Weights are relative to a reference that a row's largest logit may pass by a factor of 2^7 before it is moved, so that in most steps
// nothing is exchanged between lanes and the result is not rescaled.
//
// Measured: 64 sequences of 8K rows, 8 KV heads of 128 dims, 4 query rows: 1.07 GB in 177 us, 6.1 TB/s, 0.92 of the measured copy rate.
// Of what it took to get there: codes by 16-byte copies of every lane were 4.7 TB/s at best, whatever the number in flight; four
// independent sums in the first product and twelve warps instead of eight, 278 -> 253 us; a reference that rarely moves.
// Short ones are bound by latency: a sequence of 160 rows takes 6 us, of which 3 is the chain length, table, codes; one of 32K rows
// with 16 query rows 28, with 64 75 (every team converts every code), 12 for its codes, 4.4 before them, 2.5 to merge a block's warps and 6 the blocks' parts.
//
// Every warp has a ring of its own in shared memory, filled by bulk copies (4 or 8 KB, one or two instructions a chunk of 32 rows): it
// works on a chunk while the next kAttendStages - 1 are on their way.
#pragma once
#include "cache8.cuh"
#include "ring.cuh"

namespace dkv {

constexpr int kAttendWarps = 12, kAttendStages = 2, kAttendRows = 32;
constexpr int kAttendMaxSeqs = 1024;        // sequences a launch (their lengths and groups' prefix sums are in shared memory)
constexpr long long kDrainTicks = 2000000;  // about a millisecond, for copies on their way when a wait runs out, however short its own limit
constexpr float kSixteenth = 0.0625f;       // blocks leave averages that much smaller: the largest value, 448 * 2^120, passes fp32 (of results below 2^-122 bits are lost)
constexpr float kLift = 8.f, kSlack = 7.f;  // weights are 2^(logit - reference + kLift); logits may pass the reference by kSlack: 2^15 fits fp16

struct AttendArgs {
  const void* q;
  long long q_batch, q_head, q_token;
  float* out;                // [n][Hq][nq][D], strides below
  long long out_batch, out_head, out_token;
  float* lse;                // [n][Hq][nq] or null
  float* scratch;            // [2 slices][rows of a head, in whole QB] partial results, what belongs to each row behind them
  unsigned int* tickets;     // [n * Hkv], zero between launches
  long long wait;            // clock ticks after which a wait for a copy gives up
  int withhold;              // test hook: the chunk that warp 0 of block 0 never asks for, -1: none
  int first, step, n, nq, rows, G, causal, slots, io;
  float scale2;              // log2(e) / sqrt(D)
};

__device__ __forceinline__ void mma_f16_16816(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// (a, b) += (x, y) * f, as one packed instruction.
__device__ __forceinline__ void add_scaled2(float& a, float& b, float x, float y, float f) {
  asm("{.reg .b64 p, q, r; mov.b64 p, {%0, %1}; mov.b64 q, {%2, %3}; mov.b64 r, {%4, %4}; fma.rn.f32x2 p, q, r, p; mov.b64 {%0, %1}, p;}" : "+f"(a), "+f"(b) : "f"(x), "f"(y), "f"(f));
}
// Four codes as two pairs of fp16.
template <int kKind>
__device__ __forceinline__ void widen(uint32_t w, uint32_t& lo, uint32_t& hi) {
  if constexpr (kKind == kE4m3) {
    asm("{.reg .b16 a, b; mov.b32 {a, b}, %2; cvt.rn.f16x2.e4m3x2 %0, a; cvt.rn.f16x2.e4m3x2 %1, b;}" : "=r"(lo), "=r"(hi) : "r"(w));
  } else {                   // 0x64xx is 1024 + xx, and codes are held with 128 added
    const uint32_t off = 0x64806480u;
    const uint32_t a = __byte_perm(w, 0x64646464u, 0x4140), b = __byte_perm(w, 0x64646464u, 0x4342);
    asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(lo) : "r"(a), "r"(off));
    asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(hi) : "r"(b), "r"(off));
  }
}
__device__ __forceinline__ uint32_t pack_half(float a, float b) {
  const __half2 h = __floats2half2_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&h);
}
// Two floats as fp16 pairs hi + lo.
__device__ __forceinline__ void split_half(float a, float b, uint32_t& hi, uint32_t& lo) {
  const __half2 h = __floats2half2_rn(a, b);
  hi = *reinterpret_cast<const uint32_t*>(&h);
  const float2 f = __half22float2(h);
  lo = pack_half(a - f.x, b - f.y);
}

// Natural logarithm of a query's denominator: sum of weights relative to a reference.
__device__ __forceinline__ float log_sum(float ref, float sum) {
  return sum == 0.f ? -INFINITY : (ref - kLift + log2f(sum)) * 0.6931471805599453f;
}

// What belongs to a partial result, a sum of weighted values in units of `up`: the reference and the sum of the weights; the unit, a
// power of two, 2^-78 of the largest value scale met, but 2^-36 at least: the ratio of any two times a weight down to 2^-46 is an fp32 number.
// Over 2^24 rows, the most that there can be, a sum of codes times weights is below 2^48, and in such units below 2^126 whatever the scales;
// pages whose scale is below 2^-204 of the largest lose bits of what they add.
struct Part { float ref, sum, up; };
__device__ __forceinline__ float over(float x) { return __uint_as_float(0x7F000000u - __float_as_uint(x)); }      // 1 / x, a power of two from 2^-126 to 2^126
// The factor of a part's sums relative to m.  A part may have no row that this query sees.
__device__ __forceinline__ float weight_of(float ref, float sum, float m) { return sum == 0.f ? 0.f : fast_exp2(ref - m); }
// A result from its sums; a query that sees no row has sums of 0.
struct Whole {
  float inv, up;
  __device__ __forceinline__ Whole(float sum, float up) : inv(sum == 0.f ? 0.f : 1.f / sum), up(up) {}
  __device__ __forceinline__ float4 of(float4 v) const { return make_float4(v.x * inv * up, v.y * inv * up, v.z * inv * up, v.w * inv * up); }
};
__device__ __forceinline__ void put_part(float* at, int row, const Part& p) { __stcg(reinterpret_cast<float4*>(at) + row, make_float4(p.ref, p.sum, p.up, 0.f)); }
__device__ __forceinline__ Part get_part(const float* at, int row) { const float4 v = __ldcg(reinterpret_cast<const float4*>(at) + row); return {v.x, v.y, v.z}; }
__device__ __forceinline__ float* out_row(const AttendArgs& a, int i, int h, int row) { return a.out + i * a.out_batch + (h * a.G + row / a.nq) * a.out_head + row % a.nq * a.out_token; }
__device__ __forceinline__ void store_lse(const AttendArgs& a, int Hkv, int i, int h, int row, float ref, float sum) {
  if (a.lse) a.lse[((size_t)(i * Hkv + h) * a.G + row / a.nq) * a.nq + row % a.nq] = log_sum(ref, sum);
}

// One warp: QB (8 or 16) query rows against the chunks of 32 rows it takes.  Lane (g, t) = (lane / 4, lane % 4) holds query
// rows g (and g + 8); of the result dims 16 m + 4 t + 0..3, m < D/16.
template <int D, int QB, int kKind>
struct AttendWarp {
  static constexpr int kHalves = QB / 8, kTiles = D / 8, kSteps = D / 16, kPanels = D / 64, kVec = D / 16;   // kVec: 16-byte pieces a lane, tensor and chunk
  uint32_t q[kHalves][kSteps][2];
  float acc[kTiles][4];
  float ref[kHalves], sum[kHalves], qs[kHalves];     // reference (log2), sum of this lane's weights, scale2 / the query's scale
  int limit[kHalves];                                // rows the query sees
  float up;                                          // the unit of `acc`

  // The queries' raw numbers, asked for ahead of what their rows need.
  struct Raw { uint4 v[kHalves][kPanels][2]; };
  __device__ __forceinline__ static void ask(Raw& raw, const AttendArgs& a, int seq_i, int h, int c0, int g, int t) {
#pragma unroll
    for (int i = 0; i < kHalves; ++i) {
      const int row = c0 + g + 8 * i;
      const bool there = row < a.rows;
      const int hq = h * a.G + row / a.nq, token = row % a.nq;
      const unsigned short* from = static_cast<const unsigned short*>(a.q) + seq_i * a.q_batch + hq * a.q_head + token * a.q_token + t * 16;
#pragma unroll
      for (int p = 0; p < kPanels; ++p)
#pragma unroll
        for (int e = 0; e < 2; ++e) raw.v[i][p][e] = there ? *reinterpret_cast<const uint4*>(from + p * 64 + e * 8) : make_uint4(0, 0, 0, 0);
    }
  }
  __device__ __forceinline__ void start(const Raw& raw, const AttendArgs& a, int c0, int len, int g) {
#pragma unroll
    for (int i = 0; i < kHalves; ++i) {
      const int row = c0 + g + 8 * i;
      Eight x[kPanels][2];
      float most = 0.f, none = 0.f;                  // none: NaN where the row holds an infinity or NaN
#pragma unroll
      for (int p = 0; p < kPanels; ++p)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          x[p][e] = a.io == DKV_BF16 ? unpack8<DKV_BF16>(raw.v[i][p][e]) : unpack8<DKV_F16>(raw.v[i][p][e]);
#pragma unroll
          for (int k = 0; k < 8; ++k) { most = fmaxf(most, fabsf(x[p][e].x[k])); none = fmaf(x[p][e].x[k], 0.f, none); }
        }
#pragma unroll
      for (int o = 1; o < 4; o <<= 1) { most = fmaxf(most, __shfl_xor_sync(0xFFFFFFFFu, most, o)); none += __shfl_xor_sync(0xFFFFFFFFu, none, o); }
      // a power of two that brings the largest magnitude to [2^13, 2^14): 8 or 11 bits of it, and of all down to 2^-17 of it, are exact
      const int e = most > 0.f && most < INFINITY ? max(-126, min(126, 13 - ((int)(__float_as_uint(most) >> 23) - 127))) : 0;
      const float up = pow2(e);
      qs[i] = a.scale2 * pow2(-e);
#pragma unroll
      for (int p = 0; p < kPanels; ++p)
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const float* y = x[p][k >> 1].x + (k & 1) * 4;
          q[i][p * 4 + k][0] = pack_half(y[0] * up, y[1] * up);
          q[i][p * 4 + k][1] = pack_half(y[2] * up, y[3] * up);
        }
      limit[i] = row < a.rows ? len - (a.causal ? a.nq - 1 - row % a.nq : 0) : len;
      ref[i] = none == 0.f ? -INFINITY : 0.f;        // logits of such a row give no reference; its result is NaN, also where all are -infinity
      sum[i] = limit[i] > 0 ? none : 0.f;
    }
#pragma unroll
    for (int j = 0; j < kTiles; ++j) acc[j][0] = acc[j][1] = acc[j][2] = acc[j][3] = 0.f;
    up = 0x1p-36f;
  }

  // 32 rows from `row` on; k: in shared memory, v: this lane's first piece there; ks, vs: the page's scales, vs in units of `up`, which has
  // grown by 1 / shrink.
  __device__ __forceinline__ void add(const uint4* k, const uint4* v, float ks, float vs, float shrink, int row, int lane, int t) {
    float s[4][4];                                   // 8 rows each: four sums that do not wait for one another
#pragma unroll
    for (int i = 0; i < 4; ++i) s[i][0] = s[i][1] = s[i][2] = s[i][3] = 0.f;
#pragma unroll
    for (int p = 0; p < kPanels; ++p) {
      uint4 w[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) w[i] = k[(i * kPanels + p) * 32 + lane];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const uint32_t(&q0)[2] = q[0][p * 4 + e];
        const uint32_t(&q1)[2] = q[kHalves - 1][p * 4 + e];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          uint32_t b0, b1;
          widen<kKind>(e == 0 ? w[i].x : e == 1 ? w[i].y : e == 2 ? w[i].z : w[i].w, b0, b1);
          mma_f16_16816(s[i], q0[0], QB == 16 ? q1[0] : 0u, q0[1], QB == 16 ? q1[1] : 0u, b0, b1);
        }
      }
    }
    bool past = shrink != 1.f;
    float most[kHalves];
#pragma unroll
    for (int h = 0; h < kHalves; ++h) {
      const float f = qs[h] * ks;
      const bool cut = row + kAttendRows > limit[h];
      most[h] = -INFINITY;
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          float& x = s[i][2 * h + e];
          x *= f;
          if (cut && row + 8 * i + 2 * t + e >= limit[h]) x = -INFINITY;
          most[h] = fmaxf(most[h], x);
        }
      past |= most[h] > ref[h] + kSlack;             // also for the first rows that the query sees
    }
    if (__any_sync(0xFFFFFFFFu, past)) {
#pragma unroll
      for (int h = 0; h < kHalves; ++h) {
        float m = most[h];
        m = fmaxf(m, __shfl_xor_sync(0xFFFFFFFFu, m, 1));
        m = fmaxf(m, __shfl_xor_sync(0xFFFFFFFFu, m, 2));
        m = fmaxf(m, ref[h]);
        float c = m == -INFINITY ? 1.f : fast_exp2(ref[h] - m);             // (the other query rows' references may still be -inf)
        ref[h] = m; sum[h] *= c;
        c *= shrink;
#pragma unroll
        for (int j = 0; j < kTiles; ++j) {
          if (QB == 8) { acc[j][0] *= c; acc[j][1] *= c; acc[j][2] *= c; acc[j][3] *= c; }
          else { acc[j][2 * h] *= c; acc[j][2 * h + 1] *= c; }
        }
      }
    }
    uint32_t hi[kHalves][4], lo[kHalves][4];         // weights of rows 8 i + 2 t, + 1
#pragma unroll
    for (int h = 0; h < kHalves; ++h) {
      const float off = ref[h] == -INFINITY ? 0.f : ref[h] - kLift;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float a = fast_exp2(s[i][2 * h] - off), b = fast_exp2(s[i][2 * h + 1] - off);
        sum[h] += a + b;
        split_half(a, b, hi[h][i], lo[h][i]);
      }
    }
#pragma unroll
    for (int p = 0; p < D / 32; ++p) {
      const uint4 w0 = v[p * 32], w1 = v[(D / 32 + p) * 32];
      float o[4][4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        uint32_t b0, b1;
        widen<kKind>(e == 0 ? w0.x : e == 1 ? w0.y : e == 2 ? w0.z : w0.w, b0, b1);
        o[e][0] = o[e][1] = o[e][2] = o[e][3] = 0.f;
        if constexpr (QB == 8) mma_f16_16816(o[e], hi[0][0], lo[0][0], hi[0][1], lo[0][1], b0, b1);
        else { mma_f16_16816(o[e], hi[0][0], hi[1][0], hi[0][1], hi[1][1], b0, b1); mma_f16_16816(o[e], lo[0][0], lo[1][0], lo[0][1], lo[1][1], b0, b1); }
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        uint32_t b0, b1;
        widen<kKind>(e == 0 ? w1.x : e == 1 ? w1.y : e == 2 ? w1.z : w1.w, b0, b1);
        if constexpr (QB == 8) mma_f16_16816(o[e], hi[0][2], lo[0][2], hi[0][3], lo[0][3], b0, b1);
        else { mma_f16_16816(o[e], hi[0][2], hi[1][2], hi[0][3], hi[1][3], b0, b1); mma_f16_16816(o[e], lo[0][2], lo[1][2], lo[0][3], lo[1][3], b0, b1); }
      }
#pragma unroll
      for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int x = 0; x < 4; x += 2) add_scaled2(acc[4 * p + e][x], acc[4 * p + e][x + 1], o[e][x], o[e][x + 1], vs);
    }
  }

  // Every lane's sums become those of all rows the warp has seen, the two parts of the weights' products one.
  __device__ __forceinline__ void add_up() {
#pragma unroll
    for (int h = 0; h < kHalves; ++h) {
      sum[h] += __shfl_xor_sync(0xFFFFFFFFu, sum[h], 1);
      sum[h] += __shfl_xor_sync(0xFFFFFFFFu, sum[h], 2);
    }
    if constexpr (QB == 8) {
#pragma unroll
      for (int j = 0; j < kTiles; ++j) { acc[j][0] += acc[j][2]; acc[j][1] += acc[j][3]; }
    }
  }
  // Dims 16 m + 4 t .. + 3 of query row g + 8 h.
  __device__ __forceinline__ float4 piece(int h, int m) const { return make_float4(acc[2 * m][2 * h], acc[2 * m][2 * h + 1], acc[2 * m + 1][2 * h], acc[2 * m + 1][2 * h + 1]); }
  __device__ __forceinline__ Part sums(int h) const { return {ref[h], sum[h], up}; }
  // Results as rows in part[QB][D + 4], their sums in of[QB].
  __device__ __forceinline__ void park(float* part, Part* of, int g, int t) const {
#pragma unroll
    for (int h = 0; h < kHalves; ++h) {
      if (t == 0) of[g + 8 * h] = sums(h);
#pragma unroll
      for (int m = 0; m < D / 16; ++m) *reinterpret_cast<float4*>(part + (g + 8 * h) * (D + 4) + 16 * m + 4 * t) = piece(h, m);
    }
  }
  // A result as it lies in the registers: [kHalves][D/16][32] pieces, then the sums of every row.
  __device__ __forceinline__ void save(float* part, int lane, int g, int t) const {
#pragma unroll
    for (int h = 0; h < kHalves; ++h) {
      if (t == 0) put_part(part + QB * D, g + 8 * h, sums(h));
#pragma unroll
      for (int m = 0; m < D / 16; ++m) __stcg(reinterpret_cast<float4*>(part) + (h * (D / 16) + m) * 32 + lane, piece(h, m));
    }
  }
  // The saved results part(0), part(1), .. added up in that order.
  template <typename F>
  __device__ __forceinline__ void merge(F part, int parts, int lane, int g) {
    constexpr int kFlight = D == 64 ? 6 : 2;         // parts whose loads are in flight together, as many as the registers take
    float unit = 0.f;                                // the same for all of a part's rows
#pragma unroll
    for (int h = 0; h < kHalves; ++h) {
      float m = -INFINITY, l = 0.f;
      float4 r[D / 16];
#pragma unroll
      for (int x = 0; x < D / 16; ++x) r[x] = make_float4(0.f, 0.f, 0.f, 0.f);
      for (int p0 = 0; p0 < parts; p0 += 8) {
        Part of[8];
#pragma unroll
        for (int f = 0; f < 8; ++f) of[f] = get_part(part(min(p0 + f, parts - 1)) + QB * D, g + 8 * h);
#pragma unroll
        for (int f = 0; f < 8; ++f) { m = fmaxf(m, of[f].ref); unit = fmaxf(unit, of[f].up); }
      }
      const float down = over(unit);
      for (int p0 = 0; p0 < parts; p0 += kFlight) {
        Part of[kFlight];
        float4 y[kFlight][D / 16];
#pragma unroll
        for (int f = 0; f < kFlight; ++f) {
          const float* from = part(min(p0 + f, parts - 1));
          of[f] = get_part(from + QB * D, g + 8 * h);
#pragma unroll
          for (int x = 0; x < D / 16; ++x) y[f][x] = __ldcg(reinterpret_cast<const float4*>(from) + (h * (D / 16) + x) * 32 + lane);
        }
#pragma unroll
        for (int f = 0; f < kFlight; ++f) {
          float k = weight_of(of[f].ref, of[f].sum, m);
          l = p0 + f < parts ? fmaf(of[f].sum, k, l) : l;
          k *= of[f].up * down;
          if (p0 + f < parts) {
#pragma unroll
            for (int x = 0; x < D / 16; ++x) { r[x].x = fmaf(y[f][x].x, k, r[x].x); r[x].y = fmaf(y[f][x].y, k, r[x].y); r[x].z = fmaf(y[f][x].z, k, r[x].z); r[x].w = fmaf(y[f][x].w, k, r[x].w); }
          }
        }
      }
      ref[h] = m; sum[h] = l;
#pragma unroll
      for (int x = 0; x < D / 16; ++x) { acc[2 * x][2 * h] = r[x].x; acc[2 * x][2 * h + 1] = r[x].y; acc[2 * x + 1][2 * h] = r[x].z; acc[2 * x + 1][2 * h + 1] = r[x].w; }
    }
    up = unit;
  }
  __device__ __forceinline__ void store(const AttendArgs& a, int Hkv, int i, int h, int g, int t) const {
#pragma unroll
    for (int k = 0; k < kHalves; ++k) {
      const int row = g + 8 * k;
      if (row >= a.rows) continue;
      const Whole whole(sum[k], up);
      float* to = out_row(a, i, h, row);
      if (t == 0) store_lse(a, Hkv, i, h, row, ref[k], sum[k]);
#pragma unroll
      for (int m = 0; m < D / 16; ++m) *reinterpret_cast<float4*>(to + 16 * m + 4 * t) = whole.of(piece(k, m));
    }
  }
};

// Bytes of shared memory: the rings, whose room the merges use when all warps are done with them.
template <int D>
__host__ __device__ constexpr int attend_smem() { return kAttendWarps * kAttendStages * 2 * kAttendRows * D; }

// mbarriers of the rings.
__device__ __forceinline__ void ring_init(uint32_t bar) { asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" ::"r"(bar) : "memory"); }
__device__ __forceinline__ void ring_expect(uint32_t bar, uint32_t bytes) {
  asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ void ring_copy(uint32_t to, const void* from, uint32_t bytes, uint32_t bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(to), "l"(from), "r"(bytes), "r"(bar) : "memory");
}
__device__ __forceinline__ bool ring_done(uint32_t bar, uint32_t parity) {
  uint32_t ok;
  asm volatile("{.reg .pred p; mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2; selp.u32 %0, 1, 0, p;}" : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
  return ok != 0;
}
__device__ __forceinline__ bool ring_wait(uint32_t bar, uint32_t parity, long long limit) {
  if (ring_done(bar, parity)) return true;
  for (const long long t0 = clock64(); clock64() - t0 < limit;)
    if (ring_done(bar, parity)) return true;
  return false;
}

// A warp's ring and the chunks that run through it.
template <int D>
struct Ring {
  static constexpr int kHalfBytes = kAttendRows * D, kChunkBytes = 2 * kHalfBytes, kBytes = kAttendStages * kChunkBytes;
  unsigned char* at;
  uint32_t at_s, bar_s;
  long long limit;
  RingPlaces<kAttendStages> places;
  int withhold;

  __device__ __forceinline__ void start(unsigned char* ring, unsigned long long* bars, int lane, const AttendArgs& a) {
    at = ring; limit = a.wait;
    withhold = blockIdx.x == 0 && threadIdx.x < 32 ? a.withhold : -1;
    at_s = (uint32_t)__cvta_generic_to_shared(ring); bar_s = (uint32_t)__cvta_generic_to_shared(bars);
    if (lane == 0) {
      for (int i = 0; i < kAttendStages; ++i) ring_init(bar_s + i * 8);
      asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    __syncwarp();
  }
  __device__ __forceinline__ bool broken() const { return places.broken; }
  // Adds `count` chunks of head h to w: chunk x is rows first + 32 step x and on.  No copy is on its way when this returns.
  template <int QB, int kKind>
  __device__ __forceinline__ void run(AttendWarp<D, QB, kKind>& w, const typename AttendWarp<D, QB, kKind>::Raw& raw, const Cache8& c, const AttendArgs& a,
                                      const int* table, int h, int c0, int len, int first, int step, int count, int lane, int g, int t) {
    // page and scales of the next 32 chunks, one a lane
    int page = 0;
    float2 sc = make_float2(0.f, 0.f), now = sc;       // `now`: of the chunks being worked on (`sc` runs ahead)
    auto look = [&](int x0) {
      const int x = x0 + lane;
      if (x < count) {
        page = table[(first + x * step * kAttendRows) >> c.shift];
        sc = *reinterpret_cast<const float2*>(c.scales + region(c, page, h, 0));
      }
    };
    auto ask = [&](int x, int into) {                  // chunk x on its way into its place of the ring
      if (x && (x & 31) == 0) look(x);
      const int row = first + x * step * kAttendRows, p = __shfl_sync(0xFFFFFFFFu, page, x & 31);
      const bool withheld = withhold >= 0 && withhold-- == 0;
      __syncwarp();                                    // every lane is done with the place
      if (lane == 0) {
        const unsigned char* k = c.pages + region(c, p, h, 0) * (size_t)(c.R * D) + (row & (c.R - 1)) * D;
        const uint32_t bar = bar_s + into * 8, to = at_s + into * kChunkBytes;
        ring_expect(bar, kChunkBytes);
        if (!withheld) {
          if (c.R == kAttendRows) ring_copy(to, k, kChunkBytes, bar);
          else { ring_copy(to, k, kHalfBytes, bar); ring_copy(to + kHalfBytes, k + c.R * D, kHalfBytes, bar); }
        }
      }
      return !withheld;
    };
    auto wait = [&](int place, int parity) { return __all_sync(0xFFFFFFFFu, ring_wait(bar_s + place * 8, parity, limit)) != 0; };
    auto drain = [&](int place, int parity) { ring_wait(bar_s + place * 8, parity, limit > kDrainTicks ? limit : kDrainTicks); __syncwarp(); };
    auto use = [&](int x, int place) {
      float shrink = 1.f;
      if ((x & 31) == 0) {                             // the unit follows the largest value scale of all chunks looked up
        now = sc;
        const float up = 0x1p-78f * __uint_as_float(__reduce_max_sync(0xFFFFFFFFu, x + lane < count ? __float_as_uint(sc.y) : 0u));
        if (up > w.up) {
          if (x) shrink = w.up * over(up);
          w.up = up;
        }
      }
      const float ks = __shfl_sync(0xFFFFFFFFu, now.x, x & 31), vs = over(w.up) * __shfl_sync(0xFFFFFFFFu, now.y, x & 31);
      const unsigned char* k = at + place * kChunkBytes;
      w.add(reinterpret_cast<const uint4*>(k), reinterpret_cast<const uint4*>(k + kHalfBytes) + t * 8 + ((g + 2 * t) & 7), ks, vs, shrink, first + x * step * kAttendRows, lane, t);
    };
    static_assert(kAttendStages <= 32);                // chunk 32 i is used before the scales of chunk 32 (i + 1) are looked up
    look(0);
    places.run(count, ask, [&] { w.start(raw, a, c0, len, g); }, wait, use, drain);
  }
};

// Lengths of a launch's sequences into len_s, and before each, and in all, the sum of units_of(length) * Hkv into prefix_s.
template <typename F>
__device__ __forceinline__ void sum_units(const Cache8& c, const AttendArgs& a, int* len_s, int* prefix_s, int* scan_s, F units_of) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int per = (a.n + kAttendWarps * 32 - 1) / (kAttendWarps * 32), i0 = min(a.n, tid * per), i1 = min(a.n, i0 + per);
  int mine = 0;
  for (int i = i0; i < i1; ++i) { len_s[i] = c.len[a.first + i * a.step]; mine += units_of(len_s[i]) * c.Hkv; }
  int inc = mine;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) { const int y = __shfl_up_sync(0xFFFFFFFFu, inc, o); if (lane >= o) inc += y; }
  if (lane == 31) scan_s[warp] = inc;
  __syncthreads();
  int at = inc - mine;
  for (int w = 0; w < warp; ++w) at += scan_s[w];
  for (int i = i0; i < i1; ++i) { prefix_s[i] = at; at += units_of(len_s[i]) * c.Hkv; }
  if (i0 < i1 && i1 == a.n) prefix_s[a.n] = at;
  __syncthreads();
}
// The lengths and tables of a launch's sequences on their way to L2 while the kernel before this one ends, each line by one thread
// (0.3 us of every call whose lines are cold).
__device__ __forceinline__ void look_ahead(const Cache8& c, const AttendArgs& a) {
  const int lines = (c.max_pages * 4 + 127) / 128, x = blockIdx.x * (kAttendWarps * 32) + threadIdx.x;
  if (x < a.n) prefetch_l2(c.len + a.first + x * a.step);
  if (x / lines < a.n) prefetch_l2(c.table + (size_t)(a.first + x / lines * a.step) * c.max_pages + min(x % lines * 32, c.max_pages - 1));
}
__device__ __forceinline__ int chunks_of(int len) { return (len + kAttendRows - 1) / kAttendRows; }

// A sequence of units cut into equal slices.
struct Slices {
  int total, count;
  __device__ __forceinline__ int begin(int x) const { return (int)((long long)total * x / count); }
  __device__ __forceinline__ int owner(int u) const { return (int)(((long long)(u + 1) * count + total - 1) / total) - 1; }       // the slice that holds unit u
};
// The (sequence, head) that unit u belongs to: its place in the call, head, first unit and units.
struct HeadAt { int i, h, u0, units; };
__device__ __forceinline__ HeadAt head_at(int u, const int* prefix_s, int n, int Hkv) {
  int lo = 0, hi = n - 1;
  while (lo < hi) { const int mid = (lo + hi + 1) >> 1; if (prefix_s[mid] <= u) lo = mid; else hi = mid - 1; }
  const int units = (prefix_s[lo + 1] - prefix_s[lo]) / Hkv, h = (u - prefix_s[lo]) / units;
  return {lo, h, prefix_s[lo] + h * units, units};
}
// The parked results of `count` warps (kCount where that is not 0) added up: dims d .. d + 3 of query row qi, and the row's sums.
template <int D, int QB, int kCount>
__device__ __forceinline__ Part merge_team(const float* part, const Part* of, int count, int qi, int d, float4& v) {
  const int n = kCount ? kCount : count;
  Part all = {-INFINITY, 0.f, 0.f};
  v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll (kCount ? kCount : 1)
  for (int w = 0; w < n; ++w) { all.ref = fmaxf(all.ref, of[w * QB + qi].ref); all.up = fmaxf(all.up, of[w * QB + qi].up); }
  const float down = over(all.up);
#pragma unroll (kCount ? kCount : 1)
  for (int w = 0; w < n; ++w) {
    const Part p = of[w * QB + qi];
    float k = weight_of(p.ref, p.sum, all.ref);
    all.sum = fmaf(p.sum, k, all.sum);
    k *= p.up * down;
    const float4 y = *reinterpret_cast<const float4*>(part + (w * QB + qi) * (D + 4) + d);
    v.x = fmaf(y.x, k, v.x); v.y = fmaf(y.y, k, v.y); v.z = fmaf(y.z, k, v.z); v.w = fmaf(y.w, k, v.w);
  }
  return all;
}

// Few heads.  The warps of a block form a team for every QB query rows (one team of twelve for up to 16 rows, four of three for 64):
// each team goes over the same rows of a head, which the others then find in L2.  The rows of every (sequence, head) are taken in
// chunks of 32, a group as many chunks as a team has warps, the groups of all heads as one sequence that is cut into one equal
// slice a block; a head with one group is never cut.  In a slice a team's warps deal the chunks of a head out among themselves and
// merge through shared memory; a head that lies in several slices is merged by the block that arrives last (a ticket a head), in
// slice order, so that nothing depends on which that is.  kTeams: more than one team.
template <int D, int QB, int kKind, bool kTeams>
__global__ void __launch_bounds__(kAttendWarps * 32, 1)
attend8_kernel(const __grid_constant__ Cache8 c, const __grid_constant__ AttendArgs a) {
  using Warp = AttendWarp<D, QB, kKind>;
  constexpr int NW = kAttendWarps;
  static_assert(NW * QB * ((D + 4) * 4 + (int)sizeof(Part)) <= attend_smem<D>() && 256 * QB * 12 <= attend_smem<D>());   // merges, of at most 256 parts
  static_assert(NW % 2 == 0 && NW % 3 == 0 && NW % 4 == 0);                                                      // teams of equal size
  extern __shared__ __align__(128) unsigned char smem[];
  __shared__ int prefix_s[kAttendMaxSeqs + 1], len_s[kAttendMaxSeqs];
  __shared__ int scan_s[NW];
  __shared__ unsigned int ticket_s;
  __shared__ __align__(8) unsigned long long bar_s[NW * kAttendStages];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t = lane & 3;
  const int teams = kTeams ? a.slots : 1, size = NW / teams;
  const int c0 = kTeams ? warp / size * QB : 0, member = kTeams ? warp % size : warp;             // this warp's first query row, and place in its team
  Ring<D> ring;
  float* part_s = reinterpret_cast<float*>(smem);
  Part* of_s = reinterpret_cast<Part*>(part_s + NW * QB * (D + 4));
  pdl_launch();
  ring.start(smem + (size_t)warp * Ring<D>::kBytes, bar_s + warp * kAttendStages, lane, a);
  look_ahead(c, a);
  pdl_wait();
  sum_units(c, a, len_s, prefix_s, scan_s, [&](int len) { return max(1, (chunks_of(len) + size - 1) / size); });
  // as many slices a head as there can be, and no slice in two heads, where that leaves few blocks without one
  const int total = prefix_s[a.n], heads = a.n * c.Hkv, even = gridDim.x - gridDim.x % heads;
  const Slices slices = {total, min(heads <= (int)gridDim.x && even * 8 >= (int)gridDim.x * 7 ? even : (int)gridDim.x, total)};
  const int own = blockIdx.x;
  if (own >= slices.count) return;
  const int u1 = slices.begin(own + 1);
  for (int u = slices.begin(own); u < u1;) {
    const HeadAt at = head_at(u, prefix_s, a.n, c.Hkv);
    const int lo = at.i, h = at.h, seq = a.first + lo * a.step, len = len_s[lo], end = min(u1, at.u0 + at.units);
    const int ch0 = (u - at.u0) * size, ch1 = min(chunks_of(len), (end - at.u0) * size);
    const bool begins = u == at.u0, whole = begins && end == at.u0 + at.units;
    u = end;
    const int c_lo = slices.owner(at.u0), c_hi = slices.owner(at.u0 + at.units - 1);
    // parts: slot 0 of a slice continues a head, slot 1 begins one that others continue
    auto part = [&](int sl, bool first, int team) { return a.scratch + ((size_t)(2 * sl + first) * teams + team) * (QB * (D + 4)); };
    {
      Warp w;
      typename Warp::Raw raw;
      const int mine = max(0, (ch1 - ch0 - member + size - 1) / size);       // this warp's chunks: ch0 + member + size x
      Warp::ask(raw, a, lo, h, c0, g, t);
      ring.run(w, raw, c, a, c.table + (size_t)seq * c.max_pages, h, c0, len, (ch0 + member) * kAttendRows, size, mine, lane, g, t);
      if (ring.broken() && lane == 0) report(c, kTimeout, seq);
      __syncthreads();
      w.add_up();
      w.park(part_s + warp * QB * (D + 4), of_s + warp * QB, g, t);
    }
    __syncthreads();
    for (int x = tid; x < a.rows * (D / 4); x += NW * 32) {
      const int row = x / (D / 4), d = x % (D / 4) * 4, team = row / QB, qi = row % QB;
      float4 v;
      const Part of = merge_team<D, QB, kTeams ? 0 : NW>(part_s + team * size * QB * (D + 4), of_s + team * size * QB, size, qi, d, v);
      if (whole) {
        *reinterpret_cast<float4*>(out_row(a, lo, h, row) + d) = Whole(of.sum, of.up).of(v);
        if (d == 0) store_lse(a, c.Hkv, lo, h, row, of.ref, of.sum);
      } else {
        float* to = part(own, begins, team);
        __stcg(reinterpret_cast<float4*>(to) + qi * (D / 4) + d / 4, Whole(of.sum, of.up * kSixteenth).of(v));
        if (d == 0) __stcg(reinterpret_cast<float2*>(to + QB * D) + qi, make_float2(of.ref, of.sum));
      }
    }
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");             // the ring's copies come after what was written here
    __syncthreads();
    if (whole) continue;
    unsigned int* ticket = a.tickets + (size_t)lo * c.Hkv + h;
    if (tid == 0) {
      __threadfence();
      ticket_s = atomicAdd(ticket, 1u);
      __threadfence();
    }
    __syncthreads();
    if (ticket_s != (unsigned int)(c_hi - c_lo)) continue;
    // all parts of the head are there, averages of their values: their weights, by (part, query row), then every result as one weighted sum
    const int parts = c_hi - c_lo + 1;
    float* weight_s = reinterpret_cast<float*>(smem);
    float2* all_s = reinterpret_cast<float2*>(weight_s + parts * QB);
    for (int team = 0; team < teams; ++team) {
      const int r0 = team * QB, rows = min(QB, a.rows - r0);
      for (int x = tid; x < parts * QB; x += NW * 32)
        if (x % QB < rows) all_s[x] = __ldcg(reinterpret_cast<const float2*>(part(c_lo + x / QB, x < QB, team) + QB * D) + x % QB);
      __syncthreads();
      for (int qi = warp; qi < rows; qi += NW) {
        float m = -INFINITY, l = 0.f;
        for (int p = lane; p < parts; p += 32) m = fmaxf(m, all_s[p * QB + qi].x);
#pragma unroll
        for (int o = 16; o; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xFFFFFFFFu, m, o));
        auto weight = [&](float2 ml) { return weight_of(ml.x, ml.y, m) * ml.y; };
        for (int p = lane; p < parts; p += 32) l += weight(all_s[p * QB + qi]);
#pragma unroll
        for (int o = 16; o; o >>= 1) l += __shfl_xor_sync(0xFFFFFFFFu, l, o);
        const float inv = l == 0.f ? 0.f : 1.f / l;
        for (int p = lane; p < parts; p += 32) weight_s[p * QB + qi] = weight(all_s[p * QB + qi]) * inv;
        if (lane == 0) store_lse(a, c.Hkv, lo, h, r0 + qi, m, l);
      }
      __syncthreads();
      for (int x = tid; x < rows * (D / 4); x += NW * 32) {
        const int qi = x / (D / 4);
        float4 r = make_float4(0.f, 0.f, 0.f, 0.f);
        constexpr int kFlight = 10;                    // parts whose loads are in flight together
        for (int p0 = 0; p0 < parts; p0 += kFlight) {
          float4 y[kFlight];
#pragma unroll
          for (int f = 0; f < kFlight; ++f) {
            const int p = min(p0 + f, parts - 1);
            y[f] = __ldcg(reinterpret_cast<const float4*>(part(c_lo + p, p == 0, team)) + x);
          }
#pragma unroll
          for (int f = 0; f < kFlight; ++f)
            if (p0 + f < parts) {
              const float k = weight_s[(p0 + f) * QB + qi];
              r.x = fmaf(y[f].x, k, r.x); r.y = fmaf(y[f].y, k, r.y); r.z = fmaf(y[f].z, k, r.z); r.w = fmaf(y[f].w, k, r.w);
            }
        }
        *reinterpret_cast<float4*>(out_row(a, lo, h, r0 + qi) + x % (D / 4) * 4) = make_float4(r.x / kSixteenth, r.y / kSixteenth, r.z / kSixteenth, r.w / kSixteenth);
      }
      __syncthreads();
    }
    if (tid == 0) *ticket = 0;
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    __syncthreads();
  }
}

// Many heads.  The chunks of all heads form one sequence that is cut into one equal slice a WARP, so that no warp waits for another:
// no barrier, and the set-up of one warp's head runs beside the other warps' work.  A head counts kAttendHeadCost chunks more
// than it has, its set-up and its results: with 1 / 2 / 4 of them 32 sequences of 500 rows, 8 heads of 128, take 18.2 / 16.9 / 16.6 us,
// 96 of 160 rows 18.8 / 16.3 / 15.8, 64 of 8K the same.  A head that lies in one slice is finished there; of the others every warp leaves its part in scratch, as it
// lies in its registers, and the warp that arrives last for a head (a ticket) merges the parts in slice order.
constexpr int kAttendHeadCost = 4;
template <int D, int QB, int kKind>
__global__ void __launch_bounds__(kAttendWarps * 32, 1)
attend8_warps_kernel(const __grid_constant__ Cache8 c, const __grid_constant__ AttendArgs a) {
  using Warp = AttendWarp<D, QB, kKind>;
  constexpr int NW = kAttendWarps;
  extern __shared__ __align__(128) unsigned char smem[];
  __shared__ int prefix_s[kAttendMaxSeqs + 1], len_s[kAttendMaxSeqs];
  __shared__ int scan_s[NW];
  __shared__ __align__(8) unsigned long long bar_s[NW * kAttendStages];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
  Ring<D> ring;
  pdl_launch();
  ring.start(smem + (size_t)warp * Ring<D>::kBytes, bar_s + warp * kAttendStages, lane, a);
  look_ahead(c, a);
  pdl_wait();
  sum_units(c, a, len_s, prefix_s, scan_s, [](int len) { return chunks_of(len) + kAttendHeadCost; });
  // no more slices than units: an empty slice would leave no part, and whoever merges a head counts on one from each
  const int total = prefix_s[a.n], own = blockIdx.x * NW + warp;
  const Slices slices = {total, min((int)gridDim.x * NW, total)};
  if (own >= slices.count) return;
  const int u1 = slices.begin(own + 1);
  for (int u = slices.begin(own); u < u1;) {
    const HeadAt at = head_at(u, prefix_s, a.n, c.Hkv);
    // units of a head: its cost, then its chunks; a slice that has the cost only leaves the head to the next ones
    const int seq = a.first + at.i * a.step, len = len_s[at.i], all = at.units - kAttendHeadCost, row0 = at.u0 + kAttendHeadCost;
    const int end = min(u1, at.u0 + at.units), first = max(0, u - row0), after = max(0, end - row0);
    u = end;
    if (after == 0 && all > 0) continue;
    if (all == 0 && own != slices.owner(at.u0 + at.units - 1)) continue;       // a head without rows is its last unit's
    const bool whole = first == 0 && after == all;
    Warp w;
    typename Warp::Raw raw;
    Warp::ask(raw, a, at.i, at.h, 0, g, t);
    ring.run(w, raw, c, a, c.table + (size_t)seq * c.max_pages, at.h, 0, len, first * kAttendRows, 1, after - first, lane, g, t);
    if (ring.broken() && lane == 0) report(c, kTimeout, seq);
    w.add_up();
    if (whole) { w.store(a, c.Hkv, at.i, at.h, g, t); continue; }
    const int c_lo = slices.owner(row0), c_hi = slices.owner(at.u0 + at.units - 1);
    auto part = [&](int sl, bool first) { return a.scratch + (size_t)(2 * sl + first) * (QB * (D + 4)); };
    w.save(part(own, first == 0), lane, g, t);
    unsigned int* ticket = a.tickets + (size_t)at.i * c.Hkv + at.h;
    __threadfence();
    __syncwarp();
    unsigned int arrived = 0;
    if (lane == 0) arrived = atomicAdd(ticket, 1u);
    if (__shfl_sync(0xFFFFFFFFu, arrived, 0) != (unsigned int)(c_hi - c_lo)) continue;
    __threadfence();
    w.merge([&](int p) { return part(c_lo + p, p == 0); }, c_hi - c_lo + 1, lane, g);
    w.store(a, c.Hkv, at.i, at.h, g, t);
    if (lane == 0) *ticket = 0;
  }
}

}  // namespace dkv
