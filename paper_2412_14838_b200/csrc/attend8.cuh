// Attention of a few new queries a sequence over the rows of a cache in 8 bits (cache8.cuh):
//   out = sum_r p_r v_r / sum_r p_r,  p_r = exp(q . k_r / sqrt(D)),  rows r below the query's limit.
//
// What must move is every code once, D bytes of keys and D of values a row and head.  There are at most 64 query rows a head, 4
// or 8 in most models, so both products are warp-wide (mma.sync m16n8k16, fp16 in, fp32 sums): no 128-row tile to give to
// tcgen05.  Both code types are exact in fp16, and so are the queries once each is scaled by a power of two (8 or 11 bits of a
// row's largest magnitude down to 2^-24 below the rest's reach); weights are split into two fp16 parts, 22 bits.  The parts
// lie in the two halves of the 16-row operand where there are at most 8 query rows a head.
//   S = Q K^T   scaled by the page's key scale when it leaves the accumulators;
//   O = P V     a page's product is added to the result times its value scale.
// Weights are relative to a reference that a row's largest logit may pass by a factor of 2^7 before it is moved, so that in most steps
// nothing is exchanged between lanes and the result is not rescaled.
//
// Every warp has a ring of its own in shared memory, filled by bulk copies (4 or 8 KB, one or two instructions a chunk of 32 rows): it
// works on a chunk while the next kAttendStages - 1 are on their way.
#pragma once
#include "cache8.cuh"
#include "merge.cuh"

namespace dkv {

constexpr int kAttendWarps = 12, kAttendStages = 2, kAttendRows = 32;
constexpr int kAttendMaxSeqs = 1024;        // sequences a launch (their lengths and groups' prefix sums are in shared memory)
constexpr long long kAttendWait = 4000000000ll;  // clock ticks after which a wait for a copy gives up, about 2 s
constexpr float kLift = 8.f, kSlack = 7.f;  // weights are 2^(logit - reference + kLift); logits may pass the reference by kSlack: 2^15 fits fp16

struct AttendArgs {
  const void* q;
  long long q_batch, q_head, q_token;
  float* out;                // [n][Hq][nq][D], strides below
  long long out_batch, out_head, out_token;
  float* lse;                // [n][Hq][nq] or null
  float* scratch;            // [2 blocks][rows of a head, in whole QB] partial results, (reference, sum) behind them
  unsigned int* tickets;     // [n * Hkv], zero between launches
  int first, step, n, nq, rows, G, causal, slots;
  float scale2;              // log2(e) / sqrt(D)
};

__device__ __forceinline__ void mma_f16_16816(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// (a, b) += (x, y) * f, as one packed instruction.
__device__ __forceinline__ void fma2(float& a, float& b, float x, float y, float f) {
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

// One warp: QB (8 or 16) query rows against the chunks of 32 rows it takes.  Lane (g, t) = (lane / 4, lane % 4) holds query
// rows g (and g + 8); of the result dims 16 m + 4 t + 0..3, m < D/16.
template <int D, int QB, int kKind>
struct AttendWarp {
  static constexpr int kHalves = QB / 8, kTiles = D / 8, kSteps = D / 16, kPanels = D / 64, kVec = D / 16;   // kVec: 16-byte pieces a lane, tensor and chunk
  uint32_t q[kHalves][kSteps][2];
  float acc[kTiles][4];
  float ref[kHalves], sum[kHalves], qs[kHalves];     // reference (log2), sum of this lane's weights, scale2 / the query's scale
  int limit[kHalves];                                // rows the query sees

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
  __device__ __forceinline__ void start(const Raw& raw, const AttendArgs& a, int c0, int len, int io, int g) {
#pragma unroll
    for (int i = 0; i < kHalves; ++i) {
      const int row = c0 + g + 8 * i;
      Eight x[kPanels][2];
      float most = 0.f, none = 0.f;                  // none: NaN where the row holds an infinity or NaN
#pragma unroll
      for (int p = 0; p < kPanels; ++p)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          x[p][e] = unpack8(raw.v[i][p][e], io);
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
      ref[i] = none == 0.f ? -INFINITY : 0.f;        // logits of such a row give no reference; its result shall be NaN
      sum[i] = 0.f;
    }
#pragma unroll
    for (int j = 0; j < kTiles; ++j) acc[j][0] = acc[j][1] = acc[j][2] = acc[j][3] = 0.f;
  }

  // 32 rows from `row` on; k: in shared memory, v: this lane's first piece there; ks, vs: the page's scales.
  __device__ __forceinline__ void add(const uint4* k, const uint4* v, float ks, float vs, int row, int lane, int t) {
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
    bool past = false;
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
        const float c = m == -INFINITY ? 1.f : fast_exp2(ref[h] - m);       // (the other query rows' references may still be -inf)
        ref[h] = m; sum[h] *= c;
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
        for (int x = 0; x < 4; x += 2) fma2(acc[4 * p + e][x], acc[4 * p + e][x + 1], o[e][x], o[e][x + 1], vs);
    }
  }

  // Results as rows in part[QB][D + 4], (reference, sum) in ml[QB].
  __device__ __forceinline__ void park(float* part, float2* ml, int g, int t) {
#pragma unroll
    for (int h = 0; h < kHalves; ++h) {
      sum[h] += __shfl_xor_sync(0xFFFFFFFFu, sum[h], 1);
      sum[h] += __shfl_xor_sync(0xFFFFFFFFu, sum[h], 2);
      if (t == 0) ml[g + 8 * h] = make_float2(ref[h], sum[h]);
#pragma unroll
      for (int m = 0; m < D / 16; ++m) {
        float4 o;
        if (QB == 8) o = make_float4(acc[2 * m][0] + acc[2 * m][2], acc[2 * m][1] + acc[2 * m][3], acc[2 * m + 1][0] + acc[2 * m + 1][2], acc[2 * m + 1][1] + acc[2 * m + 1][3]);
        else o = make_float4(acc[2 * m][2 * h], acc[2 * m][2 * h + 1], acc[2 * m + 1][2 * h], acc[2 * m + 1][2 * h + 1]);
        *reinterpret_cast<float4*>(part + (g + 8 * h) * (D + 4) + 16 * m + 4 * t) = o;
      }
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
__device__ __forceinline__ bool ring_wait(uint32_t bar, uint32_t parity) {
  if (ring_done(bar, parity)) return true;
  for (const long long t0 = clock64(); clock64() - t0 < kAttendWait;)
    if (ring_done(bar, parity)) return true;
  return false;
}

// The rows of every (sequence, head) are taken in chunks of 32, kAttendWarps chunks a group, the groups of all heads as one sequence
// that is cut into one equal slice a block; a head with one group is never cut.  In a slice the warps deal the chunks of a head
// out among themselves and merge through shared memory; a head that lies in several slices is merged by the block that arrives
// last (a ticket a head), in slice order, so that nothing depends on which that is.
template <int D, int QB, int kKind>
__global__ void __launch_bounds__(kAttendWarps * 32, 1)
attend8_kernel(const __grid_constant__ Cache8 c, const __grid_constant__ AttendArgs a) {
  using Warp = AttendWarp<D, QB, kKind>;
  constexpr int NW = kAttendWarps, ST = kAttendStages, kHalfBytes = kAttendRows * D, kChunkBytes = 2 * kHalfBytes;
  static_assert(NW * QB * (D + 4) * 4 + NW * QB * 8 <= attend_smem<D>() && 256 * QB * 12 <= attend_smem<D>());   // merges, of at most 256 parts
  extern __shared__ __align__(128) unsigned char smem[];
  __shared__ int prefix_s[kAttendMaxSeqs + 1], len_s[kAttendMaxSeqs];
  __shared__ int scan_s[NW];
  __shared__ unsigned int ticket_s;
  __shared__ __align__(8) unsigned long long bar_s[NW * ST];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t = lane & 3;
  unsigned char* ring = smem + (size_t)warp * ST * kChunkBytes;
  const uint32_t ring_at = (uint32_t)__cvta_generic_to_shared(ring), bar_at = (uint32_t)__cvta_generic_to_shared(bar_s + warp * ST);
  float* part_s = reinterpret_cast<float*>(smem);
  float2* ml_s = reinterpret_cast<float2*>(part_s + NW * QB * (D + 4));
  pdl_launch();
  if (lane == 0) {
    for (int i = 0; i < ST; ++i) ring_init(bar_at + i * 8);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  __syncwarp();
  pdl_wait();
  auto chunks_of = [&](int len) { return (len + kAttendRows - 1) / kAttendRows; };
  auto groups_of = [&](int len) { return max(1, (chunks_of(len) + NW - 1) / NW) * c.Hkv; };
  {
    const int per = (a.n + NW * 32 - 1) / (NW * 32), i0 = min(a.n, tid * per), i1 = min(a.n, i0 + per);
    int mine = 0;
    for (int i = i0; i < i1; ++i) { len_s[i] = c.len[a.first + i * a.step]; mine += groups_of(len_s[i]); }
    int inc = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) { const int y = __shfl_up_sync(0xFFFFFFFFu, inc, o); if (lane >= o) inc += y; }
    if (lane == 31) scan_s[warp] = inc;
    __syncthreads();
    int at = inc - mine;
    for (int w = 0; w < warp; ++w) at += scan_s[w];
    for (int i = i0; i < i1; ++i) { prefix_s[i] = at; at += groups_of(len_s[i]); }
    if (i0 < i1 && i1 == a.n) prefix_s[a.n] = at;
    __syncthreads();
  }
  const int total = prefix_s[a.n], slices = min((int)gridDim.x, total), own = blockIdx.x;
  if (own >= slices) return;
  auto slice = [&](int x) { return (int)((long long)total * x / slices); };
  auto owner = [&](int u) { return (int)(((long long)(u + 1) * slices + total - 1) / total) - 1; };     // the slice that holds group u
  const int u1 = slice(own + 1), passes = (a.rows + QB - 1) / QB;
  int stage = 0, phase = 0;                            // of the next chunk this warp waits for
  bool broken = false;                                 // a wait ran out: nothing more is asked for or waited for
  for (int u = slice(own); u < u1;) {
    int lo = 0, hi = a.n - 1;
    while (lo < hi) { const int mid = (lo + hi + 1) >> 1; if (prefix_s[mid] <= u) lo = mid; else hi = mid - 1; }
    const int groups = (prefix_s[lo + 1] - prefix_s[lo]) / c.Hkv, h = (u - prefix_s[lo]) / groups, u0 = prefix_s[lo] + h * groups;
    const int seq = a.first + lo * a.step, len = len_s[lo], end = min(u1, u0 + groups);
    const int ch0 = (u - u0) * NW, ch1 = min(chunks_of(len), (end - u0) * NW);
    const bool begins = u == u0, whole = begins && end == u0 + groups;
    const int* table = c.table + (size_t)seq * c.max_pages;
    u = end;
    const int c_lo = owner(u0), c_hi = owner(u0 + groups - 1);
    // parts: slot 0 of a slice continues a head, slot 1 begins one that others continue
    auto part = [&](int sl, bool first, int pass) { return a.scratch + ((size_t)(2 * sl + first) * a.slots + pass) * (QB * (D + 2)); };
    for (int pass = 0; pass < passes; ++pass) {
      Warp w;
      typename Warp::Raw raw;
      const int c0 = pass * QB, mine = max(0, (ch1 - ch0 - warp + NW - 1) / NW);      // this warp's chunks: ch0 + warp + NW x
      Warp::ask(raw, a, lo, h, c0, g, t);
      // page and scales of the next 32 chunks, one a lane
      int page = 0;
      float2 sc = make_float2(0.f, 0.f);
      auto look = [&](int x0) {
        const int x = x0 + lane;
        if (x < mine) {
          page = table[(ch0 + warp + NW * x) * kAttendRows / c.R];
          sc = *reinterpret_cast<const float2*>(c.scales + region(c, page, h, 0));
        }
      };
      auto fetch = [&](int x, int into) {              // chunk x on its way into its place of the ring
        if (x >= mine || broken) return;
        const int row = (ch0 + warp + NW * x) * kAttendRows;
        const int p = __shfl_sync(0xFFFFFFFFu, page, x & 31);
        if (lane == 0) {
          const unsigned char* k = c.pages + region(c, p, h, 0) * (size_t)(c.R * D) + (row % c.R) * D;
          const uint32_t bar = bar_at + into * 8, to = ring_at + into * kChunkBytes;
          ring_expect(bar, kChunkBytes);
          if (c.R == kAttendRows) ring_copy(to, k, kChunkBytes, bar);
          else { ring_copy(to, k, kHalfBytes, bar); ring_copy(to + kHalfBytes, k + c.R * D, kHalfBytes, bar); }
        }
      };
      look(0);
#pragma unroll
      for (int x = 0; x < ST - 1; ++x) fetch(x, (stage + x) % ST);
      w.start(raw, a, c0, len, c.io, g);
      float2 now = sc;                                 // scales of the chunks being worked on (`sc` runs ahead)
      for (int x = 0; x < mine; ++x) {
        if ((x & 31) == 0) now = sc;
        if (((x + ST - 1) & 31) == 0) look(x + ST - 1);
        __syncwarp();                                  // every lane is done with the place that is filled next
        fetch(x + ST - 1, (stage + ST - 1) % ST);
        if (!broken) broken = !__all_sync(0xFFFFFFFFu, ring_wait(bar_at + stage * 8, phase));
        const float ks = __shfl_sync(0xFFFFFFFFu, now.x, x & 31), vs = __shfl_sync(0xFFFFFFFFu, now.y, x & 31);
        const unsigned char* at = ring + stage * kChunkBytes;
        if (!broken) w.add(reinterpret_cast<const uint4*>(at), reinterpret_cast<const uint4*>(at + kHalfBytes) + t * 8 + ((g + 2 * t) & 7), ks, vs, (ch0 + warp + NW * x) * kAttendRows, lane, t);
        if (++stage == ST) { stage = 0; phase ^= 1; }
      }
      if (broken && lane == 0) report(c, kTimeout, seq);
      __syncthreads();
      w.park(part_s + warp * QB * (D + 4), ml_s + warp * QB, g, t);
      __syncthreads();
      const int pieces = min(QB, a.rows - c0) * (D / 4);
      for (int x = tid; x < pieces; x += NW * 32) {
        float4 v;
        const float2 ml = merge_warps<D, QB, NW>(part_s, ml_s, x, v);
        const int qi = x / (D / 4), d = x % (D / 4) * 4, row = c0 + qi, hq = h * a.G + row / a.nq, token = row % a.nq;
        if (whole) {
          const float inv = ml.y == 0.f ? 0.f : 1.f / ml.y;
          *reinterpret_cast<float4*>(a.out + lo * a.out_batch + hq * a.out_head + token * a.out_token + d) = make_float4(v.x * inv, v.y * inv, v.z * inv, v.w * inv);
          if (a.lse && d == 0) a.lse[((size_t)lo * c.Hkv * a.G + hq) * a.nq + token] = log_sum(ml.x, ml.y);
        } else {
          float* to = part(own, begins, pass);
          __stcg(reinterpret_cast<float4*>(to) + x, v);
          if (d == 0) __stcg(reinterpret_cast<float2*>(to + QB * D) + qi, ml);
        }
      }
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");     // the ring's copies come after what was written here
      __syncthreads();
    }
    if (whole) continue;
    unsigned int* ticket = a.tickets + (size_t)lo * c.Hkv + h;
    if (tid == 0) {
      __threadfence();
      ticket_s = atomicAdd(ticket, 1u);
      __threadfence();
    }
    __syncthreads();
    if (ticket_s != (unsigned int)(c_hi - c_lo)) continue;
    // all parts of the head are there: their weights, by (part, query row), then every result as one weighted sum
    const int parts = c_hi - c_lo + 1;
    float* weight_s = reinterpret_cast<float*>(smem);
    float2* all_s = reinterpret_cast<float2*>(weight_s + parts * QB);
    for (int pass = 0; pass < passes; ++pass) {
      const int c0 = pass * QB, rows = min(QB, a.rows - c0);
      for (int x = tid; x < parts * QB; x += NW * 32)
        if (x % QB < rows) all_s[x] = __ldcg(reinterpret_cast<const float2*>(part(c_lo + x / QB, x < QB, pass) + QB * D) + x % QB);
      __syncthreads();
      for (int qi = warp; qi < rows; qi += NW) {
        float m = -INFINITY, l = 0.f;
        for (int p = lane; p < parts; p += 32) m = fmaxf(m, all_s[p * QB + qi].x);
#pragma unroll
        for (int o = 16; o; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xFFFFFFFFu, m, o));
        auto weight = [&](float2 ml) { return ml.y == 0.f ? 0.f : fast_exp2(ml.x - m); };      // (a part may have no row that this query sees)
        for (int p = lane; p < parts; p += 32) l += weight(all_s[p * QB + qi]) * all_s[p * QB + qi].y;
#pragma unroll
        for (int o = 16; o; o >>= 1) l += __shfl_xor_sync(0xFFFFFFFFu, l, o);
        const float inv = l == 0.f ? 0.f : 1.f / l;
        for (int p = lane; p < parts; p += 32) weight_s[p * QB + qi] = weight(all_s[p * QB + qi]) * inv;
        const int row = c0 + qi;
        if (a.lse && lane == 0) a.lse[((size_t)lo * c.Hkv * a.G + h * a.G + row / a.nq) * a.nq + row % a.nq] = log_sum(m, l);
      }
      __syncthreads();
      for (int x = tid; x < rows * (D / 4); x += NW * 32) {
        const int qi = x / (D / 4), row = c0 + qi, hq = h * a.G + row / a.nq, token = row % a.nq;
        float4 r = make_float4(0.f, 0.f, 0.f, 0.f);
        constexpr int kFlight = 10;                    // parts whose loads are in flight together
        for (int p0 = 0; p0 < parts; p0 += kFlight) {
          float4 y[kFlight];
#pragma unroll
          for (int f = 0; f < kFlight; ++f) {
            const int p = min(p0 + f, parts - 1);
            y[f] = __ldcg(reinterpret_cast<const float4*>(part(c_lo + p, p == 0, pass)) + x);
          }
#pragma unroll
          for (int f = 0; f < kFlight; ++f)
            if (p0 + f < parts) {
              const float k = weight_s[(p0 + f) * QB + qi];
              r.x = fmaf(y[f].x, k, r.x); r.y = fmaf(y[f].y, k, r.y); r.z = fmaf(y[f].z, k, r.z); r.w = fmaf(y[f].w, k, r.w);
            }
        }
        *reinterpret_cast<float4*>(a.out + lo * a.out_batch + hq * a.out_head + token * a.out_token + x % (D / 4) * 4) = r;
      }
      __syncthreads();
    }
    if (tid == 0) *ticket = 0;
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    __syncthreads();
  }
  if (broken)                                          // what is still on its way ends before the block does
    for (int i = 0; i < ST; ++i) ring_wait(bar_at + i * 8, i < stage ? phase ^ 1 : phase);
}

}  // namespace dkv
