// A cache of pages that holds keys and values in 8 bits: its format, rows in and out, and the pages' own operations.
//
// A page holds R rows (R = 32, 64 or 128) of every KV head of one sequence.  Per page, head and tensor (keys, values) there
// are R*D codes and one scale, a power of two: value = code * scale, codes being e4m3 numbers or int8.  A power of two costs
// e4m3 nothing (it has an exponent of its own) and int8 up to one bit, and it makes every value exactly a 16-bit number, a
// scale that grows while rows are added exact for e4m3 (but for what becomes subnormal) and one rounding for int8, and all
// arithmetic on scales free of rounding.
//
// Codes lie in the order in which a warp of the attention kernel takes them as operands of m16n8k16, so that its loads are
// 512 consecutive bytes and need neither shared memory nor a transposition (attend8.cuh):
//   keys    per 16 rows: [half of 8 rows][panel of 64 dims][row][64 dims];
//   values  per 16 rows: [32 dims][row pair t = (row % 8) / 2][place][word w][row half][row parity], place (g + 2 t) % 8 being dim
//           32 p + 16 (w / 2) + 4 (g / 2) + 2 (w % 2) + g % 2: one 32-bit word is the operand of one dim and four rows, a row lies
//           in 128 bytes of every 512, and eight lanes that read together find their 16 bytes in different banks.
// int8 codes are held with 128 added, as bytes that a permutation turns into fp16 numbers.
#pragma once
#include <cuda_fp8.h>
#include "common.cuh"
#include "rotary.cuh"

namespace dkv {

constexpr int kE4m3 = 0, kInt8 = 1;
// Status bits a kernel leaves (dkv_cache8_status).
constexpr int kNoPages = 1, kTableFull = 2, kNoRoom = 4, kBadArgument = 8, kNotFinite = 16, kTimeout = 32;

// What kernels see of a cache.
struct Cache8 {
  unsigned char* pages;      // [page][Hkv][2][R*D]
  float* scales;             // [page][Hkv][2]
  int* table;                // [sequence][max_pages]
  int* len;                  // [sequence] rows held
  int* held;                 // [sequence] pages held
  int* refs;                 // [page] sequences that hold it; 0: free
  unsigned int* free;        // bit per page: free
  int* hint;                 // no word of `free` before this one has a bit set
  int* status;               // [0] bits, [1] lowest sequence concerned
  int Hkv, D, R, max_pages, n_pages, kind, io;
};

__device__ __forceinline__ void report(const Cache8& c, int bit, int seq) {
  atomicOr(&c.status[0], bit);
  atomicMin(&c.status[1], seq);
}
__device__ __forceinline__ size_t region(const Cache8& c, int page, int h, int which) { return ((size_t)page * c.Hkv + h) * 2 + which; }

// Place of a code within its region: row r, dim d.
template <int D>
__device__ __forceinline__ int key_at(int r, int d) { return (r >> 4) * 16 * D + ((r >> 3) & 1) * 8 * D + (d >> 6) * 512 + (r & 7) * 64 + (d & 63); }
template <int D>
__device__ __forceinline__ int value_at(int r, int d) {
  const int u = d & 15, t = (r & 7) >> 1, g = 2 * (u >> 2) + (u & 1), w = 2 * ((d >> 4) & 1) + ((u >> 1) & 1);
  return (r >> 4) * 16 * D + (d >> 5) * 512 + t * 128 + ((g + 2 * t) & 7) * 16 + w * 4 + ((r >> 3) & 1) * 2 + (r & 1);
}

// Exponent of the smallest power of two s >= 2^-126 with most <= largest code * s; most is finite and not negative.
// 448 = 0x1.Cp8, 127 = 0x1.FCp6.
__device__ __forceinline__ int scale_exponent(float most, int kind) {
  const unsigned int b = __float_as_uint(most);
  const int e = (int)(b >> 23) - 127, m = (int)(b & 0x7FFFFFu);
  return max(-126, kind == kE4m3 ? e - 8 + (m > 0x600000) : e - 6 + (m > 0x7E0000));
}
__device__ __forceinline__ float pow2(int e) { return __uint_as_float((unsigned int)(e + 127) << 23); }       // -126 <= e <= 127
__device__ __forceinline__ int exponent_of(float s) { return (int)(__float_as_uint(s) >> 23) - 127; }          // of a power of two

// Codes of two numbers already divided by their scale: clamped, nearest, ties to even, NaN as 0.
__device__ __forceinline__ unsigned int code_pair(float a, float b, int kind) {
  a = a == a ? a : 0.f; b = b == b ? b : 0.f;
  if (kind == kE4m3) return __nv_cvt_float2_to_fp8x2(make_float2(a, b), __NV_SATFINITE, __NV_E4M3);
  const int x = __float2int_rn(fminf(fmaxf(a, -127.f), 127.f)), y = __float2int_rn(fminf(fmaxf(b, -127.f), 127.f));
  return (x + 128) | (y + 128) << 8;
}
__device__ __forceinline__ float code_value(unsigned int byte, int kind) {
  if (kind == kInt8) return (float)((int)byte - 128);
  return __half2float(__half(__nv_cvt_fp8_to_halfraw((__nv_fp8_storage_t)byte, __NV_E4M3)));
}

// A 16-bit number of the caller's type.
__device__ __forceinline__ float load16(unsigned int bits, int io) {
  return io == DKV_BF16 ? __uint_as_float(bits << 16) : __half2float(__ushort_as_half((unsigned short)bits));
}
__device__ __forceinline__ unsigned int store16(float x, int io) {
  if (io == DKV_BF16) return __bfloat16_as_ushort(__float2bfloat16_rn(fminf(fmaxf(x, -3.3895313892515355e38f), 3.3895313892515355e38f)));
  return __half_as_ushort(__float2half_rn(fminf(fmaxf(x, -65504.f), 65504.f)));
}

// Eight numbers of one row.
struct Eight { float x[8]; };
__device__ __forceinline__ Eight unpack8(uint4 v, int io) {
  Eight e;
  const unsigned int w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) { e.x[2 * i] = load16(w[i] & 0xFFFF, io); e.x[2 * i + 1] = load16(w[i] >> 16, io); }
  return e;
}

// Largest of a value per thread over the block.
__device__ __forceinline__ float block_max(float v, float* warp_s) {
#pragma unroll
  for (int o = 16; o; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xFFFFFFFFu, v, o));
  if ((threadIdx.x & 31) == 0) warp_s[threadIdx.x >> 5] = v;
  __syncthreads();
  v = warp_s[0];
  for (int w = 1; w < (int)blockDim.x / 32; ++w) v = fmaxf(v, warp_s[w]);
  return v;
}

// Codes of eight dims d..d+7 of row r into a region.
template <int D>
__device__ __forceinline__ void put8(unsigned char* to, int r, int d, const Eight& e, float inv, int which, int kind) {
  unsigned int c[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) c[i] = code_pair(e.x[2 * i] * inv, e.x[2 * i + 1] * inv, kind);
  if (which == 0) {
    *reinterpret_cast<uint2*>(to + key_at<D>(r, d)) = make_uint2(c[0] | c[1] << 16, c[2] | c[3] << 16);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) to[value_at<D>(r, d + i)] = (unsigned char)(c[i >> 1] >> (i & 1) * 8);
  }
}
template <int D>
__device__ __forceinline__ Eight get8(const unsigned char* from, int r, int d, float scale, int which, int kind) {
  Eight e;
  if (which == 0) {
    const uint2 v = *reinterpret_cast<const uint2*>(from + key_at<D>(r, d));
#pragma unroll
    for (int i = 0; i < 8; ++i) e.x[i] = code_value(((i < 4 ? v.x : v.y) >> (i & 3) * 8) & 0xFF, kind) * scale;
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) e.x[i] = code_value(from[value_at<D>(r, d + i)], kind) * scale;
  }
  return e;
}

// ---- rows in ------------------------------------------------------------------------------------------------------------

struct Rows8 { const void* data; long long batch, head, token; };     // strides in elements

struct AppendArgs {
  Rows8 k, v;
  const int* rows;           // [n] rows of every sequence, or null: `cap` each
  const int* pos0;           // [n] position of the first new key, where keys are turned
  unsigned int* tickets;     // [n], zero between launches
  int first, step, cap;
  int rot, pairs, vec;       // vec: rot/2 is a multiple of 8 (a piece's partner is a piece)
  float amplitude;
  double turns[128];
};

// The new rows of one page, head and tensor: their largest magnitude gives the scale, and where the page held rows before, the
// old scale is a lower bound for it; if it grows, the old codes are rounded again.  Bound by HBM (2 bytes in, 1 out) where rows
// are many and by latency where there is one.  A page is put together in shared memory and written as a whole, but for a few
// rows that join a page whose scale stays.  grid (pages a sequence can touch, 2 Hkv, n); the last block of a sequence to arrive
// (a ticket) makes the rows part of it.
constexpr int kRowThreads = 256;
template <int D, int R>
__global__ void __launch_bounds__(kRowThreads)
append8_kernel(const __grid_constant__ Cache8 c, const __grid_constant__ AppendArgs a) {
  constexpr int kPieces = R * D / 8, kPer = (kPieces + kRowThreads - 1) / kRowThreads;
  __shared__ __align__(16) unsigned char code_s[R * D];
  __shared__ float warp_s[kRowThreads / 32];
  const int tid = threadIdx.x, h = blockIdx.y >> 1, which = blockIdx.y & 1, i = blockIdx.z, seq = a.first + i * a.step;
  pdl_launch();
  pdl_wait();
  const int len = c.len[seq], held = c.held[seq], add = a.rows ? a.rows[i] : a.cap;
  const int* table = c.table + (size_t)seq * c.max_pages;
  const bool bad = add < 0 || add > a.cap;
  bool room = !bad && (long long)len + add <= (long long)held * R;
  if (room && add > 0 && len % R) room = c.refs[table[len / R]] == 1;
  if (!room || add == 0) {
    if (!room && tid == 0 && blockIdx.x == 0 && blockIdx.y == 0) report(c, bad ? kBadArgument : kNoRoom, seq);
    return;
  }
  const int slot = len / R + blockIdx.x, base = slot * R;
  const int r0 = max(0, len - base), r1 = min(R, len + add - base);          // the page's new rows
  if (r0 < r1) {
    const int page = table[slot];
    unsigned char* to = c.pages + region(c, page, h, which) * (size_t)(R * D);
    float* scale_p = c.scales + region(c, page, h, which);
    const Rows8& src = which ? a.v : a.k;
    const unsigned short* from = static_cast<const unsigned short*>(src.data) + i * src.batch + h * src.head;
    const int pieces = (r1 - r0) * (D / 8);
    Eight x[kPer];
    float most = 0.f;
    bool odd = false;
#pragma unroll
    for (int p = 0; p < kPer; ++p) {
      const int at = tid + p * kRowThreads;
      if (at < pieces) {
        const int r = r0 + at / (D / 8), d = at % (D / 8) * 8, row = base + r - len;
        const unsigned short* line = from + row * src.token;
        x[p] = unpack8(*reinterpret_cast<const uint4*>(line + d), c.io);
        if (which == 0 && d < a.rot) {
          const int pos = a.pos0[i] + row, half = a.rot / 2;
          if (a.pairs) {
#pragma unroll
            for (int e = 0; e < 8; e += 2)
              if (d + e < a.rot) {
                float cs, sn;
                turn_of(pos, a.turns[(d + e) / 2], cs, sn);
                const float u = x[p].x[e], w = x[p].x[e + 1];
                x[p].x[e] = a.amplitude * (u * cs - w * sn); x[p].x[e + 1] = a.amplitude * (u * sn + w * cs);
              }
          } else {
            Eight y;
            if (a.vec) y = unpack8(*reinterpret_cast<const uint4*>(line + (d < half ? d + half : d - half)), c.io);
#pragma unroll
            for (int e = 0; e < 8; ++e)
              if (d + e < a.rot) {
                const bool lower = d + e < half;
                if (!a.vec) y.x[e] = load16(line[lower ? d + e + half : d + e - half], c.io);
                float cs, sn;
                turn_of(pos, a.turns[lower ? d + e : d + e - half], cs, sn);
                x[p].x[e] = a.amplitude * (lower ? x[p].x[e] * cs - y.x[e] * sn : y.x[e] * sn + x[p].x[e] * cs);
              }
          }
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float m = fabsf(x[p].x[e]);
          if (m < INFINITY) most = fmaxf(most, m); else odd = true;
        }
      }
    }
    if (odd) report(c, kNotFinite, seq);
    int e = scale_exponent(block_max(most, warp_s), c.kind);
    const int was = r0 ? exponent_of(*scale_p) : e;
    e = max(e, was);
    const float inv = pow2(-e);
    if (r0 && e == was && pieces <= kRowThreads) {                           // a few rows beside others: straight to their places
      if (tid < pieces) put8<D>(to, r0 + tid / (D / 8), tid % (D / 8) * 8, x[0], inv, which, c.kind);
    } else {
      if (r0) {
        for (int q = tid; q < R * D / 16; q += kRowThreads) {
          uint4 v = reinterpret_cast<const uint4*>(to)[q];
          if (e != was) {
            const float f = pow2(max(-126, was - e));
            unsigned int* w = &v.x;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              const unsigned int o = w[k];
              w[k] = code_pair(code_value(o & 0xFF, c.kind) * f, code_value(o >> 8 & 0xFF, c.kind) * f, c.kind) |
                     code_pair(code_value(o >> 16 & 0xFF, c.kind) * f, code_value(o >> 24, c.kind) * f, c.kind) << 16;
            }
          }
          reinterpret_cast<uint4*>(code_s)[q] = v;
        }
      } else if (r1 < R) {                                                   // rows without a value yet
        for (int q = tid; q < R * D / 16; q += kRowThreads) reinterpret_cast<uint4*>(code_s)[q] = make_uint4(0, 0, 0, 0);
      }
      __syncthreads();
#pragma unroll
      for (int p = 0; p < kPer; ++p) {
        const int at = tid + p * kRowThreads;
        if (at < pieces) put8<D>(code_s, r0 + at / (D / 8), at % (D / 8) * 8, x[p], inv, which, c.kind);
      }
      __syncthreads();
      for (int q = tid; q < R * D / 16; q += kRowThreads) reinterpret_cast<uint4*>(to)[q] = reinterpret_cast<const uint4*>(code_s)[q];
    }
    if (tid == 0 && (!r0 || e != was)) *scale_p = pow2(e);
  }
  __syncthreads();                                                           // the whole block has read `len`
  if (tid == 0) {
    __threadfence();
    if (atomicAdd(&a.tickets[i], 1u) == gridDim.x * gridDim.y - 1) {
      a.tickets[i] = 0;
      c.len[seq] = len + add;
    }
  }
}

// ---- rows out -----------------------------------------------------------------------------------------------------------

struct ReadArgs { Rows8 k, v; int first, step, cap; };

// The rows of one page, head and tensor as 16-bit numbers; rows past the sequence's length are not written.  Bound by HBM.
// grid (pages of `cap` rows, 2 Hkv, n).
template <int D, int R>
__global__ void __launch_bounds__(kRowThreads)
read8_kernel(const __grid_constant__ Cache8 c, const __grid_constant__ ReadArgs a) {
  __shared__ __align__(16) unsigned char code_s[R * D];
  const int tid = threadIdx.x, h = blockIdx.y >> 1, which = blockIdx.y & 1, i = blockIdx.z, seq = a.first + i * a.step;
  pdl_launch();
  pdl_wait();
  const int base = blockIdx.x * R, rows = min(R, min(c.len[seq], a.cap) - base);
  if (rows <= 0) return;
  const int page = c.table[(size_t)seq * c.max_pages + blockIdx.x];
  const uint4* from = reinterpret_cast<const uint4*>(c.pages + region(c, page, h, which) * (size_t)(R * D));
  const float scale = c.scales[region(c, page, h, which)];
  for (int q = tid; q < R * D / 16; q += kRowThreads) reinterpret_cast<uint4*>(code_s)[q] = from[q];
  __syncthreads();
  const Rows8& dst = which ? a.v : a.k;
  unsigned short* to = static_cast<unsigned short*>(const_cast<void*>(dst.data)) + i * dst.batch + h * dst.head;
  for (int at = tid; at < rows * (D / 8); at += kRowThreads) {
    const int r = at / (D / 8), d = at % (D / 8) * 8;
    const Eight e = get8<D>(code_s, r, d, scale, which, c.kind);
    unsigned int w[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) w[k] = store16(e.x[2 * k], c.io) | store16(e.x[2 * k + 1], c.io) << 16;
    *reinterpret_cast<uint4*>(to + (base + r) * dst.token + d) = make_uint4(w[0], w[1], w[2], w[3]);
  }
}

// ---- pages --------------------------------------------------------------------------------------------------------------

constexpr int kPlanThreads = 1024;

struct PlanArgs {
  const int* count;          // [n] or null: `most` each
  int* prefix;               // [n + 1] scratch: pages that sequences before i need
  int* pick;                 // [n_pages] scratch: the pages found
  int* jobs;                 // [1 + 2 n] scratch: how many pages have to be copied, (from, to) of each
  int* new_table;            // [sequence][max_pages], compaction: the pages to be
  int* new_held;             // [sequence], compaction: how many, or -1: the sequence stays as it is
  int first, step, n, most;
};

// Sum over the block of one number per thread before this thread, and in all.
__device__ __forceinline__ long long block_scan(long long v, long long* warp_s, long long& total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  long long inc = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) { const long long y = __shfl_up_sync(0xFFFFFFFFu, inc, o); if (lane >= o) inc += y; }
  __syncthreads();                                                           // warp_s is free again
  if (lane == 31) warp_s[warp] = inc;
  __syncthreads();
  if (warp == 0) {
    long long s = lane < (int)blockDim.x / 32 ? warp_s[lane] : 0;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) { const long long y = __shfl_up_sync(0xFFFFFFFFu, s, o); if (lane >= o) s += y; }
    warp_s[lane] = s;
  }
  __syncthreads();
  total = warp_s[blockDim.x / 32 - 1];
  return inc - v + (warp ? warp_s[warp - 1] : 0);
}

// Pages for sequences that are to grow by count[i] rows (kCompact = false), or for the count[i] rows that a compaction keeps.
// Free pages are given out lowest first, in the order of the sequences: what a call does depends on nothing but the state it
// finds.  Where they do not last, the sequences from the first that cannot be served on get none.  A sequence that is to grow
// and whose last page is only partly filled and held by others too gets a page of its own, to be filled by copy_pages_kernel.
// One block: latency, a few us (one scan over the sequences, one over the words of `free` up to the last page given out).
template <bool kCompact>
__global__ void __launch_bounds__(kPlanThreads)
plan_pages_kernel(const __grid_constant__ Cache8 c, const __grid_constant__ PlanArgs a) {
  __shared__ long long warp_s[32];
  __shared__ int jobs_s;
  const int tid = threadIdx.x;
  pdl_launch();
  pdl_wait();
  if (tid == 0) jobs_s = 0;
  auto own_copy = [&](int seq, int len) { return len % c.R && c.refs[c.table[(size_t)seq * c.max_pages + len / c.R]] > 1; };
  int all = 0;
  for (int i0 = 0; i0 < a.n; i0 += kPlanThreads) {
    const int i = i0 + tid, seq = a.first + i * a.step;
    int need = 0;
    if (i < a.n) {
      const int count = a.count ? a.count[i] : a.most;
      if (kCompact) {
        const bool bad = count < 0 || count > a.most;
        if (bad) report(c, kBadArgument, seq);
        need = bad ? 0 : (int)(((long long)count + c.R - 1) / c.R);
        if (need > c.max_pages) { report(c, kTableFull, seq); need = 0; a.new_held[seq] = -1; }
        else a.new_held[seq] = bad ? -1 : need;
      } else {
        const int len = c.len[seq], held = c.held[seq];
        const long long pages = ((long long)len + count + c.R - 1) / c.R;
        if (count < 0) report(c, kBadArgument, seq);
        else if (pages > c.max_pages) report(c, kTableFull, seq);
        else if (count > 0) need = max(0, (int)pages - held) + own_copy(seq, len);
      }
    }
    long long total;                                                         // sums stop at n_pages + 1: more than there can be
    const long long before = block_scan(need, warp_s, total);
    if (i < a.n) a.prefix[i] = (int)min(all + before, c.n_pages + 1ll);
    all = (int)min(all + total, c.n_pages + 1ll);
  }
  if (tid == 0) { a.prefix[a.n] = all; if (!kCompact) a.jobs[0] = 0; }
  if (all == 0) return;
  // the lowest `all` free pages
  const int words = (c.n_pages + 31) / 32;
  int found = 0;
  for (int w0 = *c.hint; w0 < words && found < all; w0 += kPlanThreads) {
    const int w = w0 + tid;
    unsigned int bits = w < words ? c.free[w] : 0;
    long long total;
    int at = found + (int)block_scan(__popc(bits), warp_s, total);
    for (; bits && at < all; bits &= bits - 1) {
      if (at < c.n_pages) a.pick[at] = w * 32 + __ffs(bits) - 1;
      ++at;
    }
    found += (int)total;
  }
  __syncthreads();
  found = min(found, all);
  if (tid == 0 && found == all) *c.hint = a.pick[all - 1] >> 5;
  __syncthreads();
  for (int k = tid; k < found; k += kPlanThreads) {
    int lo = 0, hi = a.n - 1;                                                // the last sequence with prefix <= k
    while (lo < hi) { const int mid = (lo + hi + 1) >> 1; if (a.prefix[mid] <= k) lo = mid; else hi = mid - 1; }
    if (a.prefix[lo + 1] > found) continue;                                  // not served
    const int seq = a.first + lo * a.step, page = a.pick[k];
    int j = k - a.prefix[lo];
    if (kCompact) {
      a.new_table[(size_t)seq * c.max_pages + j] = page;
    } else {
      const int len = c.len[seq], held = c.held[seq];
      int* table = c.table + (size_t)seq * c.max_pages;
      // whether the sequence has its last page copied follows from how many pages it got: `refs` may have changed by now
      const int count = a.count ? a.count[lo] : a.most;
      const int grow = max(0, (int)(((long long)len + count + c.R - 1) / c.R) - held);
      const bool copies = a.prefix[lo + 1] - a.prefix[lo] > grow;
      if (copies && j == 0) {
        const int old = table[len / c.R], job = atomicAdd(&jobs_s, 1);
        a.jobs[1 + 2 * job] = old; a.jobs[2 + 2 * job] = page;
        table[len / c.R] = page;
        if (atomicSub(&c.refs[old], 1) == 1) { atomicOr(&c.free[old >> 5], 1u << (old & 31)); atomicMin(c.hint, old >> 5); }
      } else {
        table[held + j - copies] = page;
      }
    }
    c.refs[page] = 1;
    atomicAnd(&c.free[page >> 5], ~(1u << (page & 31)));
  }
  __syncthreads();
  for (int i = tid; i < a.n; i += kPlanThreads) {
    const int seq = a.first + i * a.step, need = a.prefix[i + 1] - a.prefix[i];
    if (need == 0) continue;
    if (a.prefix[i + 1] > found) {
      report(c, kNoPages, seq);
      if (kCompact) a.new_held[seq] = -1;
    } else if (!kCompact) {
      const int count = a.count ? a.count[i] : a.most;
      c.held[seq] = max(c.held[seq], (int)(((long long)c.len[seq] + count + c.R - 1) / c.R));
    }
  }
  if (!kCompact && tid == 0) a.jobs[0] = jobs_s;
}

// Pages that a sequence shared and is to write to: jobs[1 + 2 j] is copied to jobs[2 + 2 j], all heads.  Bound by HBM.
constexpr int kCopyThreads = 256;
__global__ void __launch_bounds__(kCopyThreads)
copy_pages_kernel(const __grid_constant__ Cache8 c, const int* jobs) {
  pdl_launch();
  pdl_wait();
  const int n = jobs[0], regions = c.Hkv * 2, vec = c.R * c.D / 16;
  for (long long at = blockIdx.x; at < (long long)n * regions; at += gridDim.x) {
    const int j = (int)(at / regions), r = (int)(at % regions);
    const size_t from = (size_t)jobs[1 + 2 * j] * regions + r, to = (size_t)jobs[2 + 2 * j] * regions + r;
    const uint4* s = reinterpret_cast<const uint4*>(c.pages) + from * vec;
    uint4* d = reinterpret_cast<uint4*>(c.pages) + to * vec;
    for (int q = threadIdx.x; q < vec; q += kCopyThreads) d[q] = s[q];
    if (threadIdx.x == 0) c.scales[to] = c.scales[from];
  }
}

// Gives back the pages [from, to) of a sequence's table.
__device__ __forceinline__ void let_go(const Cache8& c, const int* table, int from, int to) {
  for (int j = from + threadIdx.x; j < to; j += blockDim.x) {
    const int p = table[j];
    if (atomicSub(&c.refs[p], 1) == 1) { atomicOr(&c.free[p >> 5], 1u << (p & 31)); atomicMin(c.hint, p >> 5); }
  }
}

// Sequences cut to keep[i] rows, or by `drop` rows; pages behind them are given back.  grid (n).
constexpr int kSeqThreads = 128;
__global__ void __launch_bounds__(kSeqThreads)
trim8_kernel(const __grid_constant__ Cache8 c, int first, int step, const int* keep, int drop) {
  const int seq = first + blockIdx.x * step;
  pdl_launch();
  pdl_wait();
  const int len = c.len[seq], held = c.held[seq], want = keep ? keep[blockIdx.x] : len - drop;
  const int rows = max(0, min(len, want)), pages = (rows + c.R - 1) / c.R;
  if (keep && want < 0 && threadIdx.x == 0) report(c, kBadArgument, seq);
  let_go(c, c.table + (size_t)seq * c.max_pages, pages, held);
  __syncthreads();
  if (threadIdx.x == 0) { c.len[seq] = rows; c.held[seq] = pages; }
}

// Sequence `to` gives its pages back and then shares those of `from`.  No sequence is both: a source keeps its pages through
// the call, so no page that is shared here can become free meanwhile.  grid (n).
__global__ void __launch_bounds__(kSeqThreads)
fork8_kernel(const __grid_constant__ Cache8 c, int from0, int to0, int step) {
  const int from = from0 + blockIdx.x * step, to = to0 + blockIdx.x * step;
  pdl_launch();
  pdl_wait();
  const int* source = c.table + (size_t)from * c.max_pages;
  int* table = c.table + (size_t)to * c.max_pages;
  const int len = c.len[from], pages = (len + c.R - 1) / c.R;
  let_go(c, table, 0, c.held[to]);
  __syncthreads();
  for (int j = threadIdx.x; j < pages; j += kSeqThreads) {
    const int p = source[j];
    atomicAdd(&c.refs[p], 1);
    table[j] = p;
  }
  if (threadIdx.x == 0) { c.len[to] = len; c.held[to] = pages; }
}

struct CompactArgs {
  const int* idx;            // [n][Hkv][cols]
  const int* count;          // [n] or null: cols each
  const int* new_table;
  const int* new_held;
  int first, step, cols;
};

// One page, head and tensor of a compacted sequence: row j is row idx[j] of the sequence as it is; a new page takes the scale
// that its rows need.  grid (pages of `cols` rows, 2 Hkv, n).
template <int D, int R>
__global__ void __launch_bounds__(kRowThreads)
compact8_kernel(const __grid_constant__ Cache8 c, const __grid_constant__ CompactArgs a) {
  constexpr int kPieces = R * D / 8, kPer = (kPieces + kRowThreads - 1) / kRowThreads;
  __shared__ __align__(16) unsigned char code_s[R * D];
  __shared__ float warp_s[kRowThreads / 32];
  __shared__ int idx_s[R];
  const int tid = threadIdx.x, h = blockIdx.y >> 1, which = blockIdx.y & 1, i = blockIdx.z, seq = a.first + i * a.step;
  pdl_launch();
  pdl_wait();
  if ((int)blockIdx.x >= a.new_held[seq]) return;
  const int len = c.len[seq], base = blockIdx.x * R, rows = min(R, (a.count ? a.count[i] : a.cols) - base);
  const int* table = c.table + (size_t)seq * c.max_pages;
  for (int r = tid; r < rows; r += kRowThreads) {
    const int p = a.idx[((size_t)i * c.Hkv + h) * a.cols + base + r];
    const bool bad = p < 0 || p >= len;
    if (bad) report(c, kBadArgument, seq);
    idx_s[r] = bad ? -1 : p;
  }
  __syncthreads();
  Eight x[kPer];
  float most = 0.f;
#pragma unroll
  for (int p = 0; p < kPer; ++p) {
    const int at = tid + p * kRowThreads;
    if (at < rows * (D / 8)) {
      const int from = idx_s[at / (D / 8)], d = at % (D / 8) * 8;
      if (from >= 0) {
        const size_t reg = region(c, table[from / R], h, which);
        x[p] = get8<D>(c.pages + reg * (size_t)(R * D), from % R, d, c.scales[reg], which, c.kind);
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) x[p].x[e] = 0.f;
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) most = fmaxf(most, fabsf(x[p].x[e]));
    }
  }
  if (rows < R)
    for (int q = tid; q < R * D / 16; q += kRowThreads) reinterpret_cast<uint4*>(code_s)[q] = make_uint4(0, 0, 0, 0);
  const int e = scale_exponent(block_max(most, warp_s), c.kind);             // (a barrier: the zeros above are in place)
#pragma unroll
  for (int p = 0; p < kPer; ++p) {
    const int at = tid + p * kRowThreads;
    if (at < rows * (D / 8)) put8<D>(code_s, at / (D / 8), at % (D / 8) * 8, x[p], pow2(-e), which, c.kind);
  }
  __syncthreads();
  const size_t reg = region(c, a.new_table[(size_t)seq * c.max_pages + blockIdx.x], h, which);
  uint4* to = reinterpret_cast<uint4*>(c.pages + reg * (size_t)(R * D));
  for (int q = tid; q < R * D / 16; q += kRowThreads) to[q] = reinterpret_cast<const uint4*>(code_s)[q];
  if (tid == 0) c.scales[reg] = pow2(e);
}

// The compacted sequences take the place of the old ones.  grid (n).
__global__ void __launch_bounds__(kSeqThreads)
install8_kernel(const __grid_constant__ Cache8 c, const __grid_constant__ CompactArgs a) {
  const int seq = a.first + blockIdx.x * a.step;
  pdl_launch();
  pdl_wait();
  const int pages = a.new_held[seq];
  if (pages < 0) return;
  int* table = c.table + (size_t)seq * c.max_pages;
  let_go(c, table, 0, c.held[seq]);
  __syncthreads();
  for (int j = threadIdx.x; j < pages; j += kSeqThreads) table[j] = a.new_table[(size_t)seq * c.max_pages + j];
  if (threadIdx.x == 0) { c.held[seq] = pages; c.len[seq] = a.count ? a.count[blockIdx.x] : a.cols; }
}

}  // namespace dkv
