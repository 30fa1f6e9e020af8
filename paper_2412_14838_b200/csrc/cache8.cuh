// A cache of pages that holds keys and values in 8 bits: its format, rows in and out, and the pages' own operations.
//
// A page holds R rows (R = 32, 64 or 128) of every KV head of one sequence.  Per page, head and tensor (keys, values) there
// are R*D codes and one scale, a power of two: value = code * scale, codes being e4m3 numbers or int8.  A power of two costs
// e4m3 nothing (it has an exponent of its own) and int8 up to one bit, and it makes every value exactly a 16-bit number, a
// scale that grows while rows are added exact for e4m3 (but for what becomes subnormal) and one rounding for int8, and all
// arithmetic on scales free of rounding.
//
// Codes lie in the order in which a warp of the attention kernel takes them as operands of m16n8k16, so that 32 rows are one or two
// runs of memory for a bulk copy, and every lane finds its operands in 16 bytes without a transposition (attend8.cuh):
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
  int Hkv, D, R, shift, max_pages, n_pages;     // R = 2^shift
};

__device__ __forceinline__ void report(const Cache8& c, int bit, int seq) {
  atomicOr(&c.status[0], bit);
  atomicMin(&c.status[1], seq);
}
__device__ __forceinline__ size_t region(const Cache8& c, int page, int h, int which) { return ((size_t)page * c.Hkv + h) * 2 + which; }

// Place of a key's code within its region: row r, dim d.
template <int D>
__device__ __forceinline__ int key_at(int r, int d) { return (r >> 4) * 16 * D + ((r >> 3) & 1) * 8 * D + (d >> 6) * 512 + (r & 7) * 64 + (d & 63); }
// Exponent, at least `low`, of the smallest power of two s with most <= largest code * s; most is finite and not negative, and subnormal
// only where `low` is above all that it could give (-132).  448 = 0x1.Cp8, 127 = 0x1.FCp6.
__device__ __forceinline__ int scale_exponent(float most, int kind, int low = -126) {
  const unsigned int b = __float_as_uint(most);
  const int e = (int)(b >> 23) - 127, m = (int)(b & 0x7FFFFFu);
  return max(low, kind == kE4m3 ? e - 8 + (m > 0x600000) : e - 6 + (m > 0x7E0000));
}
__device__ __forceinline__ float pow2(int e) { return __uint_as_float((unsigned int)(e + 127) << 23); }       // -126 <= e <= 127
__device__ __forceinline__ int exponent_of(float s) { return (int)(__float_as_uint(s) >> 23) - 127; }          // of a power of two

// Four numbers times inv, a power of two, as four codes: nearest, ties to even, beyond the largest the largest.  Not NaN; for int8
// the products are at most 127 in magnitude.
template <int kKind>
__device__ __forceinline__ unsigned int word_of(float a, float b, float c, float d, float inv) {
  if constexpr (kKind == kE4m3) {
    const unsigned int x = __nv_cvt_float2_to_fp8x2(make_float2(a * inv, b * inv), __NV_SATFINITE, __NV_E4M3);
    return x | (unsigned int)__nv_cvt_float2_to_fp8x2(make_float2(c * inv, d * inv), __NV_SATFINITE, __NV_E4M3) << 16;
  } else {                   // 1.5 * 2^23 + 128 + product: a float's last bit is 1 there, its last byte the code
    constexpr float off = 12582912.f + 128.f;
    auto bits = [&](float x) { return __float_as_uint(fmaf(x, inv, off)); };
    return __byte_perm(__byte_perm(bits(a), bits(b), 0x0040), __byte_perm(bits(c), bits(d), 0x0040), 0x5410);
  }
}
// Four codes as numbers, times scale.
template <int kKind>
__device__ __forceinline__ void values_of(unsigned int w, float scale, float* x) {
  if constexpr (kKind == kE4m3) {
    const __half2 lo = __half2(__nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(w & 0xFFFF), __NV_E4M3));
    const __half2 hi = __half2(__nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(w >> 16), __NV_E4M3));
    const float2 a = __half22float2(lo), b = __half22float2(hi);
    x[0] = a.x * scale; x[1] = a.y * scale; x[2] = b.x * scale; x[3] = b.y * scale;
  } else {                   // 2^23 + byte, less 2^23 + 128 (before the product, which a large scale would take beyond all floats)
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = (__uint_as_float(__byte_perm(w, 0x4B000000u, 0x7540 + i)) - (8388608.f + 128.f)) * scale;
  }
}

// Eight 16-bit numbers of the caller's type, and back.
struct Eight { float x[8]; };
template <int kIo>
__device__ __forceinline__ Eight unpack8(uint4 v) {
  Eight e;
  const unsigned int w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (kIo == DKV_BF16) { e.x[2 * i] = __uint_as_float(w[i] << 16); e.x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u); }
    else { const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w[i])); e.x[2 * i] = f.x; e.x[2 * i + 1] = f.y; }
  }
  return e;
}
template <int kIo>
__device__ __forceinline__ float load16(unsigned short v) {
  return kIo == DKV_BF16 ? __uint_as_float((unsigned int)v << 16) : __half2float(__ushort_as_half(v));
}
template <int kIo>
__device__ __forceinline__ uint4 pack8(const Eight& e) {       // a code's value may pass the type's largest number by a rounding
  unsigned int o[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    constexpr float most = kIo == DKV_BF16 ? 3.3895313892515355e38f : 65504.f;
    const float a = fminf(fmaxf(e.x[2 * i], -most), most), b = fminf(fmaxf(e.x[2 * i + 1], -most), most);
    if constexpr (kIo == DKV_BF16) { const __nv_bfloat162 h = __floats2bfloat162_rn(a, b); o[i] = *reinterpret_cast<const unsigned int*>(&h); }
    else { const __half2 h = __floats2half2_rn(a, b); o[i] = *reinterpret_cast<const unsigned int*>(&h); }
  }
  return make_uint4(o[0], o[1], o[2], o[3]);
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

// What a thread takes of a page: rows 16 blk + 2 t, + 1, + 8, + 9 and dims d..d+7, the four rows that share the words of values.
struct Quad { Eight row[4]; };
__device__ __forceinline__ int quad_row(int blk, int t, int k) { return blk * 16 + 2 * t + (k & 1) + 8 * (k >> 1); }
template <int D>
__device__ __forceinline__ int quad_values_at(int blk, int t, int d, int pair) {       // 8 bytes: dims d + {0, 2}, {1, 3}, {4, 6}, {5, 7}
  const int g = 2 * ((d & 15) >> 2) + pair;
  return blk * 16 * D + (d >> 5) * 512 + t * 128 + ((g + 2 * t) & 7) * 16 + ((d >> 4) & 1) * 8;
}
// Codes of a quad times inv into a region: keys of rows [from, to), values of all four rows.
template <int D, int kKind>
__device__ __forceinline__ void put_quad(unsigned char* at, int blk, int t, int d, const Quad& q, float inv, int which, int from, int to) {
  if (which == 0) {
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int r = quad_row(blk, t, k);
      const float* x = q.row[k].x;
      const uint2 w = make_uint2(word_of<kKind>(x[0], x[1], x[2], x[3], inv), word_of<kKind>(x[4], x[5], x[6], x[7], inv));
      if (r >= from && r < to) *reinterpret_cast<uint2*>(at + key_at<D>(r, d)) = w;
    }
  } else {
    auto dim = [&](int i) { return word_of<kKind>(q.row[0].x[i], q.row[1].x[i], q.row[2].x[i], q.row[3].x[i], inv); };
#pragma unroll
    for (int p = 0; p < 4; ++p) {
      const int i = 4 * (p >> 1) + (p & 1);
      *reinterpret_cast<uint2*>(at + quad_values_at<D>(blk, t, d, p)) = make_uint2(dim(i), dim(i + 2));
    }
  }
}
// Codes of eight dims of one row; other rows' codes stay.
template <int D, int kKind>
__device__ __forceinline__ void put_row(unsigned char* at, int r, int d, const Eight& x, float inv, int which) {
  const unsigned int c[2] = {word_of<kKind>(x.x[0], x.x[1], x.x[2], x.x[3], inv), word_of<kKind>(x.x[4], x.x[5], x.x[6], x.x[7], inv)};
  if (which == 0) {
    *reinterpret_cast<uint2*>(at + key_at<D>(r, d)) = make_uint2(c[0], c[1]);
  } else {
#pragma unroll
    for (int p = 0; p < 4; ++p) {
      unsigned char* w = at + quad_values_at<D>(r >> 4, (r & 7) >> 1, d, p) + (r >> 3 & 1) * 2 + (r & 1);
      w[0] = (unsigned char)(c[p >> 1] >> (p & 1) * 8); w[4] = (unsigned char)(c[p >> 1] >> ((p & 1) * 8 + 16));
    }
  }
}
// A quad's raw words: keys of rows below `to`, values of all rows.
struct QuadWords { uint2 v[4]; };
template <int D>
__device__ __forceinline__ QuadWords get_words(const unsigned char* at, int blk, int t, int d, int which, int to) {
  QuadWords q;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const int r = quad_row(blk, t, k);
    if (which) q.v[k] = *reinterpret_cast<const uint2*>(at + quad_values_at<D>(blk, t, d, k));
    else q.v[k] = r < to ? *reinterpret_cast<const uint2*>(at + key_at<D>(r, d)) : make_uint2(0, 0);
  }
  return q;
}
template <int kKind>
__device__ __forceinline__ Eight eight_of(uint2 w, float scale) {
  Eight e;
  values_of<kKind>(w.x, scale, e.x);
  values_of<kKind>(w.y, scale, e.x + 4);
  return e;
}
// All four rows of a quad as numbers.
template <int kKind>
__device__ __forceinline__ Quad quad_of(const QuadWords& w, float scale, int which) {
  Quad q;
  if (which == 0) {
#pragma unroll
    for (int k = 0; k < 4; ++k) q.row[k] = eight_of<kKind>(w.v[k], scale);
  } else {                   // a word is one dim of the four rows
#pragma unroll
    for (int p = 0; p < 4; ++p)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        float x[4];
        values_of<kKind>(e ? w.v[p].y : w.v[p].x, scale, x);
#pragma unroll
        for (int k = 0; k < 4; ++k) q.row[k].x[4 * (p >> 1) + (p & 1) + 2 * e] = x[k];
      }
  }
  return q;
}
// Row k of a quad of values: its eight bytes as two words of four dims.
__device__ __forceinline__ uint2 row_of_values(const QuadWords& w, int k) {
  auto four = [&](uint2 a, uint2 b) { return __byte_perm(__byte_perm(a.x, b.x, k | (k + 4) << 4), __byte_perm(a.y, b.y, k | (k + 4) << 4), 0x5410); };
  return make_uint2(four(w.v[0], w.v[1]), four(w.v[2], w.v[3]));
}

// ---- rows in ------------------------------------------------------------------------------------------------------------

struct Rows8 { const void* data; long long batch, head, token; };     // strides in elements

struct AppendArgs {
  Rows8 k, v;
  const int* rows;           // [n] rows of every sequence, or null: `cap` each
  const int* pos0;           // [n] position of the first new key, where keys are turned
  unsigned int* tickets;     // [n], zero between launches
  int first, step, cap, per;  // per: heads and tensors a block
  int rot, pairs, vec;       // vec: rot/2 is a multiple of 8 (a piece's partner is a piece)
  float amplitude;
  double turns[128];
};

// The largest magnitude of eight raw numbers so far, as bits of their type, two at a time: magnitudes order like integers, and
// infinities and NaN are above all numbers.
__device__ __forceinline__ unsigned int largest_bits(unsigned int most, uint4 v) {
  return __vmaxu2(__vmaxu2(most, __vmaxu2(v.x & 0x7FFF7FFFu, v.y & 0x7FFF7FFFu)), __vmaxu2(v.z & 0x7FFF7FFFu, v.w & 0x7FFF7FFFu));
}
template <int kIo>
__device__ __forceinline__ bool has_odd(unsigned int bits) {       // an infinity or NaN among them
  constexpr unsigned int inf = kIo == DKV_BF16 ? 0x7F80u : 0x7C00u;
  return (bits & 0xFFFF) >= inf || bits >> 16 >= inf;
}
template <int kIo>
__device__ __forceinline__ float largest_of(unsigned int bits) { return load16<kIo>((unsigned short)max(bits & 0xFFFF, bits >> 16)); }
// Turns eight dims d.. of a row; cs(i) gives (A cos, A sin) of pair i.  bits: the largest magnitude of the raw numbers that were used
// besides x's own, so far (largest_bits); all of them above, where they were not looked at.
template <int kIo, typename F>
__device__ __forceinline__ void turn_row(Eight& x, unsigned int& bits, const AppendArgs& a, const unsigned short* line, int d, F cs) {
  if (d >= a.rot) return;
  const int half = a.rot / 2;
  if (a.pairs) {
#pragma unroll
    for (int e = 0; e < 8; e += 2)
      if (d + e < a.rot) {
        const float2 f = cs((d + e) / 2);
        const float u = x.x[e], w = x.x[e + 1];
        x.x[e] = u * f.x - w * f.y; x.x[e + 1] = u * f.y + w * f.x;
      }
  } else {
    Eight y;
    if (a.vec) {
      const uint4 raw = *reinterpret_cast<const uint4*>(line + (d < half ? d + half : d - half));
      bits = largest_bits(bits, raw);
      y = unpack8<kIo>(raw);
    } else {
      bits = 0x7FFF7FFFu;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (d + e < a.rot) {
        const bool lower = d + e < half;
        if (!a.vec) y.x[e] = load16<kIo>(line[lower ? d + e + half : d + e - half]);
        const float2 f = cs(lower ? d + e : d + e - half);
        x.x[e] = lower ? x.x[e] * f.x - y.x[e] * f.y : y.x[e] * f.y + x.x[e] * f.x;
      }
  }
}
__device__ __forceinline__ float2 turned_by(const AppendArgs& a, int pos, int pair) {
  float c, s;
  turn_of(pos, a.turns[pair], c, s);
  return make_float2(a.amplitude * c, a.amplitude * s);
}
// The largest finite magnitude of eight numbers; NaN becomes 0.  Whether there were some that are not finite.
__device__ __forceinline__ bool settle(Eight& x, float& most) {
  bool odd = false;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const float m = fabsf(x.x[e]);
    if (m < INFINITY) most = fmaxf(most, m);
    else { odd = true; if (m != INFINITY) x.x[e] = 0.f; }
  }
  return odd;
}
// Settled numbers times inv, which brings all finite ones within the codes: what is infinite becomes the largest.
template <int kKind>
__device__ __forceinline__ void cut(Eight& x, float inv) {
  constexpr float most = kKind == kE4m3 ? 448.f : 127.f;
#pragma unroll
  for (int e = 0; e < 8; ++e) x.x[e] = fminf(fmaxf(x.x[e] * inv, -most), most);
}
// Whether `add` rows go behind the `len` rows of a sequence; if not, why (a status bit), else 0.
__device__ __forceinline__ int no_room(const Cache8& c, const AppendArgs& a, const int* table, int len, int held, int add) {
  if (add < 0 || add > a.cap) return kBadArgument;
  if ((long long)len + add > (long long)held << c.shift) return kNoRoom;
  return add > 0 && len & (c.R - 1) && c.refs[table[len >> c.shift]] != 1 ? kNoRoom : 0;
}

// Many rows: the new rows of one page, `per` heads and tensors one after the other.  Their largest magnitude gives the scale; where
// the page held rows before, the old scale is a lower bound for it and the old codes are rounded again.  A thread has one quad, from
// 16-bit numbers in registers straight to codes, and asks for the next one's rows before it works on this one's.  Bound by HBM (2
// bytes in, 1 out), but for the chain of loads at a block's start and the ticket at its end, which is why a block has several heads
// where there are blocks enough.  Angles are shared by all heads (shared memory, [R][rot/2]).  32 sequences of 544 rows, 8 heads of 128:
// 24 us for 107 MB (4.4 TB/s); a block a head and tensor took 44, a warp each 40, rings of cp.async in place of the registers that
// hold the next rows 31.  What bounds it is its instructions, some fourteen a number to begin with, half of that now.
// Keys turned in neighbouring pairs: 33 us for 100 MB (28 unturned); in halves 135 for 197 MB (43 unturned): the other half of a row
// is loaded when it is needed, not ahead.  grid (pages a sequence can touch,
// 2 Hkv / per, n); the last block of a sequence to arrive (a ticket) makes the rows part of it.
constexpr int kQuadThreads = 512;                                            // R * D / 32 threads, at most
template <int D, int kKind, int kIo, bool kTurn>
__global__ void __launch_bounds__(kTurn ? 640 : kQuadThreads)                // (640: five blocks of 128 threads an SM in place of four, 42 -> 36 us where keys are turned)
append8_kernel(const __grid_constant__ Cache8 c, const __grid_constant__ AppendArgs a) {
  extern __shared__ float2 turn_s[];
  __shared__ float warp_s[2][kQuadThreads / 32];
  const int R = c.R, tid = threadIdx.x, i = blockIdx.z, seq = a.first + i * a.step;
  const int d = tid % (D / 8) * 8, t = tid / (D / 8) % 4, blk = tid / (D / 2);
  pdl_launch();
  pdl_wait();
  const int len = c.len[seq], held = c.held[seq], add = a.rows ? a.rows[i] : a.cap;
  const int* table = c.table + (size_t)seq * c.max_pages;
  const int not_ok = no_room(c, a, table, len, held, add);
  if (not_ok || add == 0) {
    if (not_ok && tid == 0 && blockIdx.x == 0 && blockIdx.y == 0) report(c, not_ok, seq);
    return;
  }
  const int slot = (len >> c.shift) + blockIdx.x, base = slot << c.shift;
  const int r0 = max(0, len - base), r1 = min(R, len + add - base);          // the page's new rows
  if (r0 < r1) {
    const int page = table[slot], y0 = blockIdx.y * a.per, y1 = min(2 * c.Hkv, y0 + a.per);
    struct Raw { uint4 v[4]; };
    // the page's row 0 (which may lie before the source) in both tensors, and a quad's rows from there
    const unsigned short* from_k = static_cast<const unsigned short*>(a.k.data) + i * a.k.batch + (base - len) * a.k.token;
    const unsigned short* from_v = static_cast<const unsigned short*>(a.v.data) + i * a.v.batch + (base - len) * a.v.token;
    const long long token_k = a.k.token, token_v = a.v.token, head_k = a.k.head, head_v = a.v.head;
    auto is_new = [&](int k) { return quad_row(blk, t, k) >= r0 && quad_row(blk, t, k) < r1; };
    auto ask = [&](int y) {
      Raw raw;
      const long long token = y & 1 ? token_v : token_k;
      const unsigned short* from = (y & 1 ? from_v + (y >> 1) * head_v : from_k + (y >> 1) * head_k) + d;
#pragma unroll
      for (int k = 0; k < 4; ++k) raw.v[k] = is_new(k) ? *reinterpret_cast<const uint4*>(from + quad_row(blk, t, k) * token) : make_uint4(0, 0, 0, 0);
      return raw;
    };
    Raw raw = ask(y0);
    if (kTurn) {
      const int pos0 = a.pos0[i] + base - len;
      for (int x = tid; x < (r1 - r0) * (a.rot / 2); x += blockDim.x) {
        const int r = r0 + x / (a.rot / 2), pair = x % (a.rot / 2);
        turn_s[r * (a.rot / 2) + pair] = turned_by(a, pos0 + r, pair);
      }
      __syncthreads();
    }
    for (int y = y0; y < y1; ++y) {
      const int which = y & 1;
      const size_t reg = region(c, page, y >> 1, which);
      unsigned char* to = c.pages + reg * (size_t)(R * D);
      const Raw now = raw;
      if (y + 1 < y1) raw = ask(y + 1);
      const bool turned = kTurn && !which;
      Quad x;
      unsigned int bits = 0;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        bits = largest_bits(bits, now.v[k]);
        x.row[k] = unpack8<kIo>(now.v[k]);
        if (turned && is_new(k)) turn_row<kIo>(x.row[k], bits, a, from_k + (y >> 1) * head_k + quad_row(blk, t, k) * token_k, d, [&](int pair) { return turn_s[quad_row(blk, t, k) * (a.rot / 2) + pair]; });
      }
      float most = largest_of<kIo>(bits);
      bool odd = has_odd<kIo>(bits) || (turned && !(most * fabsf(a.amplitude) < 1e38f));       // turned numbers are at most twice as large: finite
      if (turned && !odd) {
        most = 0.f;
#pragma unroll
        for (int k = 0; k < 4; ++k)
#pragma unroll
          for (int e = 0; e < 8; ++e) most = fmaxf(most, fabsf(x.row[k].x[e]));
      }
      if (odd) {                                                             // some may not be finite
        most = 0.f;
        odd = false;
#pragma unroll
        for (int k = 0; k < 4; ++k) odd |= settle(x.row[k], most);
        if (odd) report(c, kNotFinite, seq);
      }
      int e = scale_exponent(block_max(most, warp_s[y & 1]), kKind), grown = 0;
      if (r0) {
        const int old = exponent_of(c.scales[reg]);
        grown = max(0, e - old);
        e = max(e, old);
      }
      float inv = pow2(-e);
      if (odd) {
#pragma unroll
        for (int k = 0; k < 4; ++k) cut<kKind>(x.row[k], inv);
        inv = 1.f;
      }
      if (r0) {                                                              // all rows in units of the new scale: an old value may be beyond fp32
        const Quad w = quad_of<kKind>(get_words<D>(to, blk, t, d, which, r0), pow2(max(-126, -grown)), which);
#pragma unroll
        for (int k = 0; k < 4; ++k)
#pragma unroll
          for (int i = 0; i < 8; ++i) x.row[k].x[i] = quad_row(blk, t, k) < r0 ? w.row[k].x[i] : x.row[k].x[i] * inv;
        inv = 1.f;
        __syncthreads();                                                     // the whole block has read the old scale
      }
      put_quad<D, kKind>(to, blk, t, d, x, inv, which, 0, r1);
      if (tid == 0) c.scales[reg] = pow2(e);
    }
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

// A few rows (at most kFewRows): a block a sequence, a warp for each head and tensor in turn, so that nothing waits on other blocks.
// Latency: the new rows are on their way while the sequence's length, its table and the page's scale are looked up one after the
// other; then every lane writes its eight codes of a row.  Only where the scale of a page with rows grows is the page read.  grid (n).
// 1 / 2 / 4 / 8 rows a sequence (8 heads of 128, us, with append8_kernel in brackets): 32 sequences 3.5 (4.7) / 3.5 (7.3) / 4.1 (7.3) /
// 5.1 (7.3), 128 sequences 3.4 (11.1) / 3.4 (13.4) / 3.9 (13.3) / 4.8 (13.5), one sequence of 8 rows 4.9 (4.1).
constexpr int kFewRows = 8, kFewWarps = 16;
template <int D, int kKind, int kIo>
__global__ void __launch_bounds__(kFewWarps * 32)
append8_few_kernel(const __grid_constant__ Cache8 c, const __grid_constant__ AppendArgs a) {
  const int R = c.R;
  constexpr int kPer = kFewRows * D / 256;                                   // pieces (a row, eight dims) of a lane
  const int lane = threadIdx.x & 31, i = blockIdx.x, seq = a.first + i * a.step;
  pdl_launch();
  pdl_wait();
  const int len = c.len[seq], held = c.held[seq], add = a.rows ? a.rows[i] : a.cap;
  const int* table = c.table + (size_t)seq * c.max_pages;
  bool ok = true;
  for (int hw = threadIdx.x >> 5; ok && hw < 2 * c.Hkv; hw += blockDim.x >> 5) {
    const int h = hw >> 1, which = hw & 1;
    const long long token = which ? a.v.token : a.k.token;
    const unsigned short* from = static_cast<const unsigned short*>(which ? a.v.data : a.k.data) + i * (which ? a.v.batch : a.k.batch) + h * (which ? a.v.head : a.k.head);
    Eight x[kPer];
    uint4 raw[kPer];
#pragma unroll
    for (int p = 0; p < kPer; ++p) {
      const int j = (lane + 32 * p) / (D / 8), d = (lane + 32 * p) % (D / 8) * 8;
      raw[p] = j < a.cap ? *reinterpret_cast<const uint4*>(from + j * token + d) : make_uint4(0, 0, 0, 0);
    }
    const int pos0 = a.rot && !which ? a.pos0[i] : 0;
    const int not_ok = no_room(c, a, table, len, held, add);
    if (not_ok || add == 0) {
      if (not_ok && threadIdx.x == 0) report(c, not_ok, seq);
      ok = false;
      break;
    }
#pragma unroll
    for (int p = 0; p < kPer; ++p) {
      const int j = (lane + 32 * p) / (D / 8), d = (lane + 32 * p) % (D / 8) * 8;
      x[p] = unpack8<kIo>(raw[p]);
      unsigned int bits = 0;
      if (a.rot && !which && j < add) turn_row<kIo>(x[p], bits, a, from + j * token, d, [&](int pair) { return turned_by(a, pos0 + j, pair); });
    }
    for (int base = len & -R; base < len + add; base += R) {
      const int r0 = max(0, len - base), r1 = min(R, len + add - base);
      const size_t reg = region(c, table[base >> c.shift], h, which);
      unsigned char* to = c.pages + reg * (size_t)(R * D);
      const float old = c.scales[reg];
      float most = 0.f;
      bool odd = false;
#pragma unroll
      for (int p = 0; p < kPer; ++p) {
        const int j = (lane + 32 * p) / (D / 8), r = len + j - base;
        if (j < add && r >= r0 && r < r1) odd |= settle(x[p], most);
      }
      if (odd) report(c, kNotFinite, seq);
#pragma unroll
      for (int o = 16; o; o >>= 1) most = fmaxf(most, __shfl_xor_sync(0xFFFFFFFFu, most, o));
      int e = scale_exponent(most, kKind);
      if (r0 && e > exponent_of(old)) {                                      // the page's older codes are rounded again
        for (int u = lane; u < R * D / 32; u += 32) {
          const int d = u % (D / 8) * 8, t = u / (D / 8) % 4, blk = u / (D / 2);
          if (quad_row(blk, t, 0) >= r0) continue;                           // (row 0 is a quad's lowest)
          put_quad<D, kKind>(to, blk, t, d, quad_of<kKind>(get_words<D>(to, blk, t, d, which, r0), old, which), pow2(-e), which, 0, r0);
        }
        __syncwarp();                                                        // the new rows share words with the old ones
      } else if (r0) {
        e = exponent_of(old);
      }
      const float inv = pow2(-e);
#pragma unroll
      for (int p = 0; p < kPer; ++p) {
        const int j = (lane + 32 * p) / (D / 8), d = (lane + 32 * p) % (D / 8) * 8, r = len + j - base;
        if (j < add && r >= r0 && r < r1) {
          cut<kKind>(x[p], inv);
          put_row<D, kKind>(to, r, d, x[p], 1.f, which);
        }
      }
      __syncwarp();                                                          // every lane has read the old scale
      if (lane == 0 && (!r0 || e != exponent_of(old))) c.scales[reg] = pow2(e);
    }
  }
  __syncthreads();                                                           // the whole block has read `len`
  if (threadIdx.x == 0 && ok) c.len[seq] = len + add;
}

// ---- rows out -----------------------------------------------------------------------------------------------------------

struct ReadArgs { Rows8 k, v; int first, step, cap; };

// The rows of one page, head and tensor as 16-bit numbers, a quad a thread; rows past the sequence's length are not written.
// Bound by HBM: 32 sequences of 544 rows, 8 heads of 128, 18.5 us for 107 MB (5.8 TB/s).  grid (pages of `cap` rows, 2 Hkv, n).
template <int D, int kKind, int kIo>
__global__ void __launch_bounds__(kQuadThreads)
read8_kernel(const __grid_constant__ Cache8 c, const __grid_constant__ ReadArgs a) {
  const int R = c.R, tid = threadIdx.x, h = blockIdx.y >> 1, which = blockIdx.y & 1, i = blockIdx.z, seq = a.first + i * a.step;
  const int d = tid % (D / 8) * 8, t = tid / (D / 8) % 4, blk = tid / (D / 2);
  pdl_launch();
  pdl_wait();
  const int base = blockIdx.x * R, rows = min(R, min(c.len[seq], a.cap) - base);
  if (rows <= 0) return;
  const size_t reg = region(c, c.table[(size_t)seq * c.max_pages + blockIdx.x], h, which);
  const QuadWords w = get_words<D>(c.pages + reg * (size_t)(R * D), blk, t, d, which, rows);
  const float scale = c.scales[reg];
  const long long token = which ? a.v.token : a.k.token;
  unsigned short* to = static_cast<unsigned short*>(const_cast<void*>(which ? a.v.data : a.k.data)) + i * (which ? a.v.batch : a.k.batch) +
                       h * (which ? a.v.head : a.k.head) + d;
  const Quad q = quad_of<kKind>(w, scale, which);
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const int r = quad_row(blk, t, k);
    if (r < rows) *reinterpret_cast<uint4*>(to + (base + r) * token) = pack8<kIo>(q.row[k]);
  }
}

// ---- pages --------------------------------------------------------------------------------------------------------------

constexpr int kPlanThreads = 1024, kPlanPicks = 4096;       // picks: pages found that shared memory holds

struct PlanArgs {
  const int* count;          // [n] or null: `most` each
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
// and whose last page is only partly filled and held by others too gets a page of its own, to be filled with that page's rows.
// One block plans: latency, a few us (one scan over the sequences, one over the words of `free` up to the last page given out).
template <bool kCompact>
__device__ __forceinline__ void plan_pages(const Cache8& c, const PlanArgs& a) {
  __shared__ long long warp_s[32];
  __shared__ int jobs_s, prefix_s[kPlanThreads + 1], len_s[kPlanThreads], held_s[kPlanThreads], copies_s[kPlanThreads], pick_s[kPlanPicks];
  const int tid = threadIdx.x;
  if (tid == 0) jobs_s = 0;
  auto pick = [&](int k) -> int& { return k < kPlanPicks ? pick_s[k] : a.pick[k]; };
  int hint = __ldcg(c.hint);                                                 // (asked for ahead of its use)
  // Sequences that are served get the pages given out one call after the other, kPlanThreads sequences at a time, as if in one.
  bool lasts = true;
  for (int i0 = 0; i0 < a.n; i0 += kPlanThreads) {
    const int i = i0 + tid, n = min(kPlanThreads, a.n - i0), seq = a.first + i * a.step;
    int need = 0, pages = 0;
    if (i < a.n) {
      const int count = a.count ? a.count[i] : a.most;
      if (kCompact) {
        pages = need = (int)(((long long)count + c.R - 1) >> c.shift);
        const bool bad = count < 0 || count > a.most, full = !bad && need > c.max_pages;
        if (bad || full) { report(c, bad ? kBadArgument : kTableFull, seq); need = 0; }
        a.new_held[seq] = bad || full ? -1 : need;
      } else {
        const int len = c.len[seq], held = c.held[seq];
        const long long all = ((long long)len + count + c.R - 1) >> c.shift;
        bool copies = false;
        if (count < 0) report(c, kBadArgument, seq);
        else if (all > c.max_pages) report(c, kTableFull, seq);
        else if (count > 0) {
          copies = len & (c.R - 1) && __ldcg(c.refs + __ldcg(c.table + (size_t)seq * c.max_pages + (len >> c.shift))) > 1;
          need = max(0, (int)all - held) + copies;
          pages = max(held, (int)all);
        }
        len_s[tid] = len; held_s[tid] = held; copies_s[tid] = copies;
      }
    }
    long long sum;                                                           // sums stop at n_pages + 1: more than there can be
    const long long before = block_scan(need, warp_s, sum);
    if (i < a.n) prefix_s[tid] = (int)min(before, c.n_pages + 1ll);
    const int all = (int)min(sum, c.n_pages + 1ll);
    if (tid == 0) prefix_s[n] = all;
    // the lowest `all` free pages
    const int words = (c.n_pages + 31) / 32;
    int found = 0;
    if (all && lasts)
      for (int w0 = hint; w0 < words && found < all; w0 += kPlanThreads) {
        const int w = w0 + tid;
        unsigned int bits = w < words ? __ldcg(c.free + w) : 0;
        long long here;
        int at = found + (int)block_scan(__popc(bits), warp_s, here);
        for (; bits && at < all; bits &= bits - 1) {
          if (at < c.n_pages) pick(at) = w * 32 + __ffs(bits) - 1;
          ++at;
        }
        found += (int)here;
      }
    __syncthreads();
    found = min(found, all);
    if (tid == 0 && all && found == all) *c.hint = pick(all - 1) >> 5;
    __syncthreads();
    for (int k = tid; k < found; k += kPlanThreads) {
      int lo = 0, hi = n - 1;                                                // the last sequence with prefix <= k
      while (lo < hi) { const int mid = (lo + hi + 1) >> 1; if (prefix_s[mid] <= k) lo = mid; else hi = mid - 1; }
      if (prefix_s[lo + 1] > found) continue;                                // not served
      const int s = a.first + (i0 + lo) * a.step, page = pick(k), j = k - prefix_s[lo];
      if (kCompact) {
        a.new_table[(size_t)s * c.max_pages + j] = page;
      } else {
        int* table = c.table + (size_t)s * c.max_pages;
        if (copies_s[lo] && j == 0) {
          const int at = len_s[lo] >> c.shift, old = table[at], job = atomicAdd(&jobs_s, 1);
          a.jobs[1 + 2 * job] = old; a.jobs[2 + 2 * job] = page;
          table[at] = page;
        } else {
          table[held_s[lo] + j - copies_s[lo]] = page;
        }
      }
      c.refs[page] = 1;
      atomicAnd(&c.free[page >> 5], ~(1u << (page & 31)));
    }
    __syncthreads();
    if (need) {
      if (prefix_s[tid + 1] > found) {
        report(c, kNoPages, seq);
        if (kCompact) a.new_held[seq] = -1;
      } else if (!kCompact) {
        c.held[seq] = pages;
      }
    }
    lasts = lasts && found == all;
    if (i0 + kPlanThreads < a.n) {
      __threadfence();                                                       // the next sequences find `free` and the table as they are now
      __syncthreads();
      hint = __ldcg(c.hint);
    }
  }
  if (!kCompact) {                                                           // shared pages are given up when all sequences have been planned
    for (int j = tid; j < jobs_s; j += kPlanThreads) {
      const int old = a.jobs[1 + 2 * j];
      if (atomicSub(&c.refs[old], 1) == 1) { atomicOr(&c.free[old >> 5], 1u << (old & 31)); atomicMin(c.hint, old >> 5); }
    }
    if (tid == 0) a.jobs[0] = jobs_s;
  }
}

// A cluster of kPlanBlocks: its first block plans, then all of them copy the pages that sequences shared and are to write to
// (jobs[1 + 2 j] to jobs[2 + 2 j], all heads), mostly none: a launch of its own for that cost every step 2 us more (32 sequences 4.9
// us, now 3.5).
constexpr int kPlanBlocks = 8;
__global__ void __launch_bounds__(kPlanThreads)
reserve8_kernel(const __grid_constant__ Cache8 c, const __grid_constant__ PlanArgs a) {
  pdl_launch();
  pdl_wait();
  if (blockIdx.x == 0) plan_pages<false>(c, a);
  __threadfence();
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
  const int n = __ldcg(a.jobs);
  const size_t vec = (size_t)c.Hkv * 2 * c.R * c.D / 16;                      // a page
  for (int j = 0; j < n; ++j) {
    const size_t from = __ldcg(a.jobs + 1 + 2 * j), to = __ldcg(a.jobs + 2 + 2 * j);
    const uint4* s = reinterpret_cast<const uint4*>(c.pages) + from * vec;
    uint4* d = reinterpret_cast<uint4*>(c.pages) + to * vec;
    for (size_t q = blockIdx.x * kPlanThreads + threadIdx.x; q < vec; q += kPlanBlocks * kPlanThreads) d[q] = s[q];
    for (int r = blockIdx.x * kPlanThreads + threadIdx.x; r < c.Hkv * 2; r += kPlanBlocks * kPlanThreads) c.scales[to * c.Hkv * 2 + r] = c.scales[from * c.Hkv * 2 + r];
  }
}
__global__ void __launch_bounds__(kPlanThreads)
plan_compact8_kernel(const __grid_constant__ Cache8 c, const __grid_constant__ PlanArgs a) {
  pdl_launch();
  pdl_wait();
  plan_pages<true>(c, a);
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
  unsigned int* tickets;     // [n], zero between launches
  int first, step, cols;
};

// One page and head of a compacted sequence: row j is row idx[j] of the sequence as it is; a new page takes the scales that its rows
// need.  A quad of keys and one of values a thread, all their loads in flight.  A row's values lie in 32 bytes of every 128, so four
// times their bytes are read: 28 sequences cut from up to 8K rows to 1000, 4 heads of 128, about 30 us for 66 MB in and 26 out, bound by
// the latency of its chain of loads (count, row numbers, table, codes).  grid (pages of `cols` rows,
// at least one, Hkv, n).
template <int D, int kKind>
__global__ void __launch_bounds__(kQuadThreads, 2)
compact8_kernel(const __grid_constant__ Cache8 c, const __grid_constant__ CompactArgs a) {
  __shared__ float warp_s[2][kQuadThreads / 32];
  __shared__ bool last_s;
  const int R = c.R, tid = threadIdx.x, h = blockIdx.y, i = blockIdx.z, seq = a.first + i * a.step;
  const int d = tid % (D / 8) * 8, t = tid / (D / 8) % 4, blk = tid / (D / 2);
  const int* idx = a.idx + ((size_t)i * c.Hkv + h) * a.cols + blockIdx.x * R;
  pdl_launch();
  pdl_wait();
  const int base = blockIdx.x * R;
  int from[4];                                                               // asked for with what says how many count
#pragma unroll
  for (int k = 0; k < 4; ++k) from[k] = base + quad_row(blk, t, k) < a.cols ? idx[quad_row(blk, t, k)] : -1;
  const int held = a.new_held[seq], len = c.len[seq], count = a.count ? a.count[i] : a.cols, rows = min(R, count - base);
  int* table = c.table + (size_t)seq * c.max_pages;
  if (held < 0) return;                                                      // the sequence stays as it is
  if ((int)blockIdx.x < held) {
    size_t reg[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const bool wanted = quad_row(blk, t, k) < rows, inside = wanted && from[k] >= 0 && from[k] < len;
      if (wanted && !inside) report(c, kBadArgument, seq);
      if (!inside) from[k] = -1;
      reg[k] = inside ? region(c, table[from[k] >> c.shift], h, 0) : 0;
    }
    uint2 key[4];
    QuadWords value[4];
    float2 scale[4];
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (from[k] >= 0) {
        const unsigned char* at = c.pages + reg[k] * (size_t)(R * D);
        const int r = from[k] & (R - 1);
        key[k] = *reinterpret_cast<const uint2*>(at + key_at<D>(r, d));
        value[k] = get_words<D>(at + R * D, r >> 4, (r & 7) >> 1, d, 1, R);
        scale[k] = *reinterpret_cast<const float2*>(c.scales + reg[k]);
        scale[k].x *= 0.0625f; scale[k].y *= 0.0625f;                        // the largest values, 448 * 2^120, pass fp32; the smallest, 2^-139 now, do not
      }
    const size_t to = region(c, a.new_table[(size_t)seq * c.max_pages + blockIdx.x], h, 0);
#pragma unroll
    for (int which = 0; which < 2; ++which) {
      Quad x;
      float most = 0.f;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        if (from[k] >= 0) {
          x.row[k] = eight_of<kKind>(which ? row_of_values(value[k], (from[k] & 1) + 2 * (from[k] >> 3 & 1)) : key[k], which ? scale[k].y : scale[k].x);
        } else {
#pragma unroll
          for (int e = 0; e < 8; ++e) x.row[k].x[e] = 0.f;
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) most = fmaxf(most, fabsf(x.row[k].x[e]));
      }
      const int e = scale_exponent(block_max(most, warp_s[which]), kKind, -130) + 4;
      if (e < -123)                                                          // 2^(4-e) would pass fp32
#pragma unroll
        for (int k = 0; k < 4; ++k)
#pragma unroll
          for (int i = 0; i < 8; ++i) x.row[k].x[i] *= 8.f;
      put_quad<D, kKind>(c.pages + (to + which) * (size_t)(R * D), blk, t, d, x, pow2(e < -123 ? 1 - e : 4 - e), which, 0, rows);
      if (tid == 0) c.scales[to + which] = pow2(e);
    }
  }
  // the last block of the sequence to arrive: nobody needs the old pages any more, the new ones take their place
  __syncthreads();
  if (tid == 0) {
    __threadfence();
    last_s = atomicAdd(&a.tickets[i], 1u) == gridDim.x * gridDim.y - 1;
  }
  __syncthreads();
  if (!last_s) return;
  const int* made = a.new_table + (size_t)seq * c.max_pages;
  let_go(c, table, 0, c.held[seq]);
  __syncthreads();
  for (int j = tid; j < held; j += blockDim.x) table[j] = made[j];
  if (tid == 0) { a.tickets[i] = 0; c.held[seq] = held; c.len[seq] = count; }
}

}  // namespace dkv
