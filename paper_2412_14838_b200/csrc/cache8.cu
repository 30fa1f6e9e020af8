// Host side of rotary positions and of the cache in 8 bits: argument checks, memory and launches of the entry points that
// include/dkv.h declares under "Generation after a compressed prompt".
#include <cuda_runtime.h>
#include <limits.h>
#include <math.h>
#include <stdint.h>
#include <stdlib.h>
#include <string.h>
#include <algorithm>
#include <atomic>
#include <new>
#include <type_traits>
#include <utility>
#include <vector>

#include "../../include/dkv.h"
#include "attend8.cuh"
#include "cache8.cuh"
#include "launch.cuh"
#include "rotary.cuh"

using namespace dkv;

struct dkv_cache8 {
  dkv_cache8_config cfg;
  int device, n_sms;
  Cache8 view;
  int *d_pick, *d_jobs, *d_new_table, *d_new_held;     // scratch of the calls on pages
  unsigned int* d_tickets;      // [n_seqs * Hkv], zero between launches
  float* d_scratch;             // parts of heads that lie in several blocks' slices
  long long launches;
  long long wait_cycles;        // dkv_cache8_set_wait_limit
  int withhold;                 // dkv_cache8_debug_withhold
  int last_cuda;
  void* memory;                 // all of the above
};

namespace {

inline cudaStream_t as_stream(void* s) { return reinterpret_cast<cudaStream_t>(s); }

int fail(dkv_cache8* c, cudaError_t e) {
  if (c) c->last_cuda = (int)e;
  cudaGetLastError();                          // reported once: see cuda_fail in dkv.cu
  return e == cudaErrorMemoryAllocation ? DKV_ERR_NOMEM : DKV_ERR_CUDA;
}
#define C8_CUDA(c, call) do { const cudaError_t e__ = (call); if (e__ != cudaSuccess) return fail(c, e__); } while (0)
#define C8_LAUNCH(c, call) do { C8_CUDA(c, call); (c)->launches++; } while (0)

int element_size(int type) { return type == DKV_F32 ? 4 : 2; }
bool aligned(const void* p, size_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }

// A tensor that can be addressed: sizes not negative, strides too, data aligned to its elements.
bool valid(const dkv_rows* r) {
  if (!r || r->type < DKV_BF16 || r->type > DKV_RAW16 || r->batch < 0 || r->heads < 0 || r->tokens < 0 || r->head_dim < 0) return false;
  if (r->batch_stride < 0 || r->head_stride < 0 || r->token_stride < 0) return false;
  const bool empty = !r->batch || !r->heads || !r->tokens || !r->head_dim;
  return empty || (r->data && aligned(r->data, element_size(r->type)));
}
bool same_shape(const dkv_rows& a, const dkv_rows& b) {
  return a.type == b.type && a.batch == b.batch && a.heads == b.heads && a.tokens == b.tokens && a.head_dim == b.head_dim;
}
// Strides of dimensions with one entry say nothing.
bool same_places(const dkv_rows& a, const dkv_rows& b) {
  return a.data == b.data && (a.batch == 1 || a.batch_stride == b.batch_stride) && (a.heads == 1 || a.head_stride == b.head_stride) &&
         (a.tokens == 1 || a.token_stride == b.token_stride);
}
bool vectors(const dkv_rows& r) {              // every row starts on a 16-byte boundary
  const int per = 16 / element_size(r.type);
  return aligned(r.data, 16) && (r.batch == 1 || r.batch_stride % per == 0) && (r.heads == 1 || r.head_stride % per == 0) &&
         (r.tokens == 1 || r.token_stride % per == 0);
}
bool valid(const dkv_rotary* r) {
  if (!r || r->head_dim < 2 || r->head_dim > 256 || r->head_dim % 2 || r->rot_dim < 2 || r->rot_dim > r->head_dim || r->rot_dim % 2) return false;
  double sum = r->amplitude;                   // infinite or NaN where any part of it is
  for (int i = 0; i < r->rot_dim / 2; ++i) sum += fabs(r->turns[i]);
  return (r->layout == DKV_ROTARY_HALF || r->layout == DKV_ROTARY_PAIRS) && isfinite(sum);
}

// ---- rotary positions ---------------------------------------------------------------------------------------------------
template <typename T, int V>
cudaError_t launch_rotate(RotateArgs& a, int head_dim, bool pairs, int sms, cudaStream_t st) {
  a.rot_pieces = a.rot / (2 * V);
  a.pieces = head_dim / (2 * V);
  // As many tokens a block as leave two blocks an SM, few heads' cosines being shared otherwise; the rest of its threads deal out heads.
  a.block_tokens = (int)std::max(1ll, std::min<long long>(std::min(kRotateTokens, kRotateThreads / a.pieces), a.all / (2 * sms)));
  a.groups = std::max(1, std::min(a.heads, kRotateThreads / (a.pieces * a.block_tokens)));
  const long long blocks = (a.all + a.block_tokens - 1) / a.block_tokens;
  if (blocks > INT_MAX) return cudaErrorInvalidValue;
  const int splits = (int)std::max(1ll, std::min<long long>((a.heads + a.groups - 1) / a.groups, sms / blocks));      // blocks that share a token's heads
  const size_t smem = (size_t)a.block_tokens * ((a.rot / 2 + 1) / 2 * 2 + 2) * sizeof(float2);
  return launch_pdl(pairs ? rotate_kernel<T, V, true> : rotate_kernel<T, V, false>, dim3((unsigned)blocks, splits), kRotateThreads, smem, 1, st, a);
}
template <typename T>
cudaError_t launch_rotate(RotateArgs& a, int head_dim, bool wide, bool pairs, int sms, cudaStream_t st) {
  return wide ? launch_rotate<T, 16 / (int)sizeof(T)>(a, head_dim, pairs, sms, st) : launch_rotate<T, 1>(a, head_dim, pairs, sms, st);
}
// Of the current device, asked for once a device: a launch's shape depends on it, its result does not.
int sm_count() {
  static std::atomic<int> known[64];
  int device = 0, n = 148;
  if (cudaGetDevice(&device) != cudaSuccess || device < 0 || device >= 64) return n;
  if ((n = known[device].load(std::memory_order_relaxed)) > 0) return n;
  if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, device) != cudaSuccess) return 148;
  known[device].store(n, std::memory_order_relaxed);
  return n;
}

// ---- the cache ----------------------------------------------------------------------------------------------------------
int validate(const dkv_cache8_config* c) {
  if (!c || c->n_pages < 1 || c->n_seqs < 1 || c->max_pages < 1 || c->n_q_heads < 1 || c->n_kv_heads < 1) return DKV_ERR_INVALID_ARG;
  if (c->n_q_heads % c->n_kv_heads != 0) return DKV_ERR_INVALID_ARG;
  if (c->kind != DKV_E4M3 && c->kind != DKV_INT8) return DKV_ERR_UNSUPPORTED;
  if (c->io != DKV_BF16 && c->io != DKV_F16) return DKV_ERR_UNSUPPORTED;
  if (c->head_dim != 64 && c->head_dim != 128) return DKV_ERR_UNSUPPORTED;
  if (c->page_rows != 32 && c->page_rows != 64 && c->page_rows != 128) return DKV_ERR_UNSUPPORTED;
  if (c->n_pages > 1 << 26 || c->n_seqs > 65535 || c->n_kv_heads > 32767 || (long long)c->max_pages * c->page_rows > 1 << 24) return DKV_ERR_UNSUPPORTED;
  return DKV_OK;
}

constexpr int kMostQueries = 64;               // query rows of a KV head

int attend_blocks(const dkv_cache8* c) { return std::min(c->n_sms, 256); }
// A slice a warp where there are more heads than blocks and the query rows fit one pass; else a slice a block.  Measured, 8 KV heads a
// sequence, 4 query rows of 128 dims (us, a slice a block / a warp): 8 sequences of 2000 rows 18.4 / 22.6, 16 of 2000 24.3 / 26.5, 16 of
// 8192 55.1 / 62.1, but 16 of 500 15.3 / 13.9; 32 of 500 22.9 / 18.2, 32 of 2000 38.1 / 37.8, 64 of 2000 60.8 / 57.9.  With few heads a
// single warp has to merge a great many parts: 1 sequence of 8192 rows 12.2 / 75.9.
bool attend_by_warps(const dkv_cache8* c, int n, int rows) { return rows <= 16 && (long long)n * c->cfg.n_kv_heads > attend_blocks(c); }
// Floats of scratch: two parts a slice, of 16 rows a warp or of all a block.
size_t attend_scratch(const dkv_cache8* c) {
  return (size_t)attend_blocks(c) * 2 * std::max(kAttendWarps * 16, kMostQueries) * (c->cfg.head_dim + 4);
}

template <int D, int QB, int kKind>
cudaError_t set_attend_smem() {
  cudaError_t e = cudaSuccess;
  for (auto kernel : {attend8_kernel<D, QB, kKind, false>, attend8_kernel<D, QB, kKind, QB == 16>, attend8_warps_kernel<D, QB, kKind>})
    if (e == cudaSuccess) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, attend_smem<D>());
  return e;
}
template <int D>
cudaError_t set_attend_smem(int kind) {
  cudaError_t e = kind == kE4m3 ? set_attend_smem<D, 8, kE4m3>() : set_attend_smem<D, 8, kInt8>();
  return e != cudaSuccess ? e : kind == kE4m3 ? set_attend_smem<D, 16, kE4m3>() : set_attend_smem<D, 16, kInt8>();
}

// The sequences of a call exist and the cache's device is the current one.
int check(const dkv_cache8* c, int first, int n, int step) {
  if (!c || n < 0) return DKV_ERR_INVALID_ARG;
  if (n > 0 && (first < 0 || step < 1 || first + (long long)(n - 1) * step >= c->cfg.n_seqs)) return DKV_ERR_INVALID_ARG;
  int device = -1;
  if (cudaGetDevice(&device) != cudaSuccess || device != c->device) return DKV_ERR_INVALID_ARG;
  return DKV_OK;
}
// Rows or queries of a call: `heads` heads of the cache's kind of 16-bit numbers, every row on a 16-byte boundary.
bool fits(const dkv_cache8* c, const dkv_rows* r, int n, int heads) {
  if (!valid(r) || (r->type != c->cfg.io && r->type != DKV_RAW16)) return false;
  return r->batch == n && r->heads == heads && r->head_dim == c->cfg.head_dim && vectors(*r);
}
Rows8 rows8(const dkv_rows* r) { return {r->data, r->batch_stride, r->head_stride, r->token_stride}; }

// Calls f with std::integral_constants of the cache's head size, kind of codes and type of rows.
template <typename F>
cudaError_t with_types(const dkv_cache8* c, F f) {
  auto types = [&](auto d, auto kind) { return c->cfg.io == DKV_BF16 ? f(d, kind, std::integral_constant<int, DKV_BF16>()) : f(d, kind, std::integral_constant<int, DKV_F16>()); };
  auto kinds = [&](auto d) { return c->cfg.kind == DKV_E4M3 ? types(d, std::integral_constant<int, kE4m3>()) : types(d, std::integral_constant<int, kInt8>()); };
  return c->cfg.head_dim == 64 ? kinds(std::integral_constant<int, 64>()) : kinds(std::integral_constant<int, 128>());
}
int quad_threads(const dkv_cache8* c) { return c->cfg.page_rows * c->cfg.head_dim / 32; }

template <int D, int QB, int kKind>
cudaError_t launch_attend(dkv_cache8* c, const AttendArgs& a, cudaStream_t st) {
  const bool warps = attend_by_warps(c, a.n, a.rows);
  return launch_pdl(warps ? attend8_warps_kernel<D, QB, kKind> : a.slots > 1 ? attend8_kernel<D, QB, kKind, QB == 16> : attend8_kernel<D, QB, kKind, false>, dim3(attend_blocks(c)), kAttendWarps * 32, (size_t)attend_smem<D>(), 1, st, c->view, a);
}
template <int D>
cudaError_t launch_attend(dkv_cache8* c, const AttendArgs& a, cudaStream_t st) {
  if (c->cfg.kind == DKV_E4M3) return a.rows <= 8 ? launch_attend<D, 8, kE4m3>(c, a, st) : launch_attend<D, 16, kE4m3>(c, a, st);
  return a.rows <= 8 ? launch_attend<D, 8, kInt8>(c, a, st) : launch_attend<D, 16, kInt8>(c, a, st);
}

}  // namespace

extern "C" {

int dkv_rotary_init(const dkv_rotary_config* cfg, dkv_rotary* out) {
  if (!cfg || !out) return DKV_ERR_INVALID_ARG;
  dkv_rotary r;
  memset(&r, 0, sizeof r);
  r.head_dim = cfg->head_dim; r.rot_dim = cfg->rot_dim; r.layout = cfg->layout; r.amplitude = 1.f;
  if (!valid(&r) || cfg->scaling < DKV_SCALING_NONE || cfg->scaling > DKV_SCALING_RAMP) return DKV_ERR_INVALID_ARG;
  const int rot = cfg->rot_dim, scaling = cfg->scaling;
  const bool banded = scaling == DKV_SCALING_WAVELENGTH || scaling == DKV_SCALING_RAMP;
  const double pi = 3.14159265358979323846, factor = scaling ? cfg->factor : 1.0;
  double theta = cfg->theta;
  if (!(theta > 0) || !(factor >= 1) || isinf(theta) || isinf(factor)) return DKV_ERR_INVALID_ARG;
  if (banded && (!(cfg->low > 0) || !(cfg->high > cfg->low) || !(cfg->trained_len > 0) || isinf(cfg->high) || isinf(cfg->trained_len))) return DKV_ERR_INVALID_ARG;
  if (scaling == DKV_SCALING_BASE) {
    if (rot == 2) return DKV_ERR_INVALID_ARG;
    theta *= pow(factor, (double)rot / (rot - 2));
  }
  double x = 0, y = 0;
  if (scaling == DKV_SCALING_RAMP) {
    if (theta == 1) return DKV_ERR_INVALID_ARG;                              // all pairs alike: no place makes so many turns
    auto place = [&](double turns) { return rot * log(cfg->trained_len / (2 * pi * turns)) / (2 * log(theta)); };
    x = std::max(0.0, floor(place(cfg->high)));
    y = std::min(rot - 1.0, ceil(place(cfg->low)));
    r.amplitude = (float)(0.1 * log(factor) + 1);
  }
  for (int i = 0; i < rot / 2; ++i) {
    double f = pow(theta, -2.0 * i / rot);
    if (scaling == DKV_SCALING_LINEAR) f /= factor;
    if (scaling == DKV_SCALING_WAVELENGTH) {
      const double turns = cfg->trained_len * f / (2 * pi), b = std::min(1.0, std::max(0.0, (turns - cfg->low) / (cfg->high - cfg->low)));
      f = f / factor * (1 - b) + f * b;
    }
    if (scaling == DKV_SCALING_RAMP) {
      const double ramp = std::min(1.0, std::max(0.0, (i - x) / std::max(y - x, 0.001)));
      f = f / factor * ramp + f * (1 - ramp);
    }
    r.turns[i] = f / (2 * pi);
    if (!isfinite(r.turns[i])) return DKV_ERR_INVALID_ARG;
  }
  *out = r;
  return DKV_OK;
}

int dkv_rotate(const dkv_rotary* r, const int32_t* pos, const dkv_rows* x, const dkv_rows* x_out, const dkv_rows* y, const dkv_rows* y_out,
               int32_t transpose, void* stream) {
  if (!valid(r) || !valid(x) || !valid(x_out) || !same_shape(*x, *x_out) || x->type == DKV_RAW16 || x->head_dim != r->head_dim) return DKV_ERR_INVALID_ARG;
  if (!y != !y_out) return DKV_ERR_INVALID_ARG;
  if (y && (!valid(y) || !valid(y_out) || !same_shape(*y, *y_out) || y->type != x->type || y->batch != x->batch || y->tokens != x->tokens ||
            y->head_dim != x->head_dim)) return DKV_ERR_INVALID_ARG;
  const dkv_rows *in[2] = {x, y}, *out[2] = {x_out, y_out};
  RotateArgs a;
  memset(&a, 0, sizeof a);
  bool wide = true, in_place = true;
  for (int i = 0; i < 2; ++i) {
    if (!in[i] || !in[i]->heads || !in[i]->batch || !in[i]->tokens) continue;
    if (in[i]->data == out[i]->data && !same_places(*in[i], *out[i])) return DKV_ERR_INVALID_ARG;
    a.x[i] = {in[i]->data, out[i]->data, in[i]->batch_stride, in[i]->head_stride, in[i]->token_stride,
              out[i]->batch_stride, out[i]->head_stride, out[i]->token_stride, in[i]->heads};
    if ((long long)a.heads + in[i]->heads > 65535) return DKV_ERR_INVALID_ARG;
    a.heads += in[i]->heads;
    wide = wide && vectors(*in[i]) && vectors(*out[i]);
    in_place = in_place && in[i]->data == out[i]->data;
  }
  if (!a.heads) return DKV_OK;
  if (!pos || !aligned(pos, 4)) return DKV_ERR_INVALID_ARG;
  const int per = 16 / element_size(x->type);
  wide = wide && r->rot_dim % (2 * per) == 0 && (r->head_dim - r->rot_dim) % (2 * per) == 0;
  a.pos = pos;
  a.all = (long long)x->batch * x->tokens; a.tokens = x->tokens;
  a.rot = r->rot_dim; a.in_place = in_place;
  const bool pairs = r->layout == DKV_ROTARY_PAIRS;
  const int sms = sm_count(), D = r->head_dim;
  a.amplitude = r->amplitude; a.sign = transpose ? -1.f : 1.f;
  memcpy(a.turns, r->turns, sizeof a.turns);
  cudaStream_t st = as_stream(stream);
  const cudaError_t e = x->type == DKV_F32 ? launch_rotate<float>(a, D, wide, pairs, sms, st) : x->type == DKV_F16 ? launch_rotate<__half>(a, D, wide, pairs, sms, st)
                                                                                                : launch_rotate<__nv_bfloat16>(a, D, wide, pairs, sms, st);
  return e == cudaSuccess ? DKV_OK : fail(nullptr, e);
}

int dkv_cache8_create(const dkv_cache8_config* cfg, dkv_cache8** out) {
  if (!out) return DKV_ERR_INVALID_ARG;
  *out = nullptr;
  const int rc = validate(cfg);
  if (rc) return rc;
  dkv_cache8* c = new (std::nothrow) dkv_cache8;
  if (!c) return DKV_ERR_NOMEM;
  memset(c, 0, sizeof *c);
  c->cfg = *cfg;
  Cache8& v = c->view;
  v.Hkv = cfg->n_kv_heads; v.D = cfg->head_dim; v.R = cfg->page_rows; v.max_pages = cfg->max_pages; v.n_pages = cfg->n_pages;
  v.shift = cfg->page_rows == 32 ? 5 : cfg->page_rows == 64 ? 6 : 7;
  c->wait_cycles = 4000000000ll;               // about 2 s
  c->withhold = -1;
  const size_t regions = (size_t)cfg->n_pages * cfg->n_kv_heads * 2, entries = (size_t)cfg->n_seqs * cfg->max_pages;
  const int words = (cfg->n_pages + 31) / 32;
  cudaError_t e = cudaGetDevice(&c->device);
#define TRY(call) if (e == cudaSuccess) e = (call)
  TRY(cudaDeviceGetAttribute(&c->n_sms, cudaDevAttrMultiProcessorCount, c->device));
  // one allocation: every part on a 256-byte boundary, zeros but for what follows below.  Every code is a number from the start:
  // what rows not yet written hold is multiplied by a weight of zero
  size_t bytes = 0;
  std::vector<std::pair<void**, size_t>> parts;
  auto part = [&](auto& p, size_t n) { parts.push_back({reinterpret_cast<void**>(&p), bytes}); bytes += (n * sizeof *p + 255) / 256 * 256; };
  try {
    part(v.pages, regions * cfg->page_rows * cfg->head_dim);
    part(v.scales, regions);
    part(v.table, entries);
    part(v.len, cfg->n_seqs);
    part(v.held, cfg->n_seqs);
    part(v.refs, cfg->n_pages);
    part(v.free, words);
    part(v.hint, 1);
    part(v.status, 2);
    part(c->d_pick, cfg->n_pages);
    part(c->d_jobs, 1 + 2 * (size_t)cfg->n_seqs);
    part(c->d_new_table, entries);
    part(c->d_new_held, cfg->n_seqs);
    part(c->d_tickets, (size_t)cfg->n_seqs * cfg->n_kv_heads);
    part(c->d_scratch, attend_scratch(c));
  } catch (const std::bad_alloc&) { delete c; return DKV_ERR_NOMEM; }
  TRY(cudaMalloc(&c->memory, bytes));
  if (e == cudaSuccess)
    for (const auto& p : parts) *p.first = static_cast<char*>(c->memory) + p.second;
  TRY(cudaMemset(c->memory, 0, bytes));
  if (e == cudaSuccess) {
    const int status[2] = {0, INT_MAX};
    e = cudaMemcpy(v.status, status, sizeof status, cudaMemcpyHostToDevice);
    TRY(cudaMemset(v.free, 0xFF, sizeof(int) * words));
    if (cfg->n_pages % 32) {                   // no page behind the last
      const unsigned int last = (1u << cfg->n_pages % 32) - 1;
      TRY(cudaMemcpy(v.free + words - 1, &last, sizeof last, cudaMemcpyHostToDevice));
    }
  }
  TRY(cudaStreamSynchronize(cudaStreamLegacy));
  TRY(cfg->head_dim == 64 ? set_attend_smem<64>(cfg->kind) : set_attend_smem<128>(cfg->kind));
  TRY(with_types(c, [](auto d, auto kind, auto io) {       // angles of a page's rows: the most that any cache has
    return cudaFuncSetAttribute(append8_kernel<decltype(d)::value, decltype(kind)::value, decltype(io)::value, true>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                128 * decltype(d)::value / 2 * (int)sizeof(float2));
  }));
#undef TRY
  if (e != cudaSuccess) {
    cudaGetLastError();
    cudaFree(c->memory);
    delete c;
    return e == cudaErrorMemoryAllocation ? DKV_ERR_NOMEM : DKV_ERR_CUDA;
  }
  *out = c;
  return DKV_OK;
}

int dkv_cache8_destroy(dkv_cache8* c) {
  if (!c) return DKV_ERR_INVALID_ARG;
  cudaDeviceSynchronize();
  cudaFree(c->memory);
  delete c;
  return DKV_OK;
}

int dkv_cache8_reserve(dkv_cache8* c, int32_t first, int32_t n, int32_t step, const int32_t* rows, int32_t add, void* stream) {
  if (int rc = check(c, first, n, step)) return rc;
  if (!aligned(rows, 4) || (!rows && add < 0)) return DKV_ERR_INVALID_ARG;
  if (n == 0) return DKV_OK;
  PlanArgs a = {rows, c->d_pick, c->d_jobs, nullptr, nullptr, first, step, n, add};
  C8_LAUNCH(c, launch_pdl(reserve8_kernel, dim3(kPlanBlocks), kPlanThreads, 0, kPlanBlocks, as_stream(stream), c->view, a));
  return DKV_OK;
}

int dkv_cache8_append(dkv_cache8* c, int32_t first, int32_t n, int32_t step, const dkv_rows* k, const dkv_rows* v, const int32_t* rows,
                      const dkv_rotary* rotary, const int32_t* pos0, void* stream) {
  if (int rc = check(c, first, n, step)) return rc;
  if (!fits(c, k, n, c->cfg.n_kv_heads) || !fits(c, v, n, c->cfg.n_kv_heads) || k->tokens != v->tokens || !aligned(rows, 4)) return DKV_ERR_INVALID_ARG;
  if (!rotary != !pos0 || (rotary && (!valid(rotary) || rotary->head_dim != c->cfg.head_dim || !aligned(pos0, 4)))) return DKV_ERR_INVALID_ARG;
  if (n == 0 || k->tokens == 0) return DKV_OK;
  AppendArgs a;
  memset(&a, 0, sizeof a);
  a.k = rows8(k); a.v = rows8(v); a.rows = rows; a.pos0 = pos0; a.tickets = c->d_tickets;
  a.first = first; a.step = step; a.cap = k->tokens;
  if (rotary) {
    a.rot = rotary->rot_dim; a.pairs = rotary->layout == DKV_ROTARY_PAIRS; a.vec = rotary->rot_dim % 16 == 0; a.amplitude = rotary->amplitude;
    memcpy(a.turns, rotary->turns, sizeof a.turns);
  }
  const int R = c->cfg.page_rows, pages = (int)std::min<long long>(((long long)k->tokens + R - 2) / R + 1, c->cfg.max_pages);
  // Heads and tensors a block: as many as leave four blocks an SM.
  const long long blocks = 2ll * c->cfg.n_kv_heads * pages * n;
  a.per = (int)std::min<long long>(2 * c->cfg.n_kv_heads, std::max(1ll, blocks / (4 * c->n_sms)));
  a.per = 2 * c->cfg.n_kv_heads / ((2 * c->cfg.n_kv_heads + a.per - 1) / a.per);
  C8_LAUNCH(c, with_types(c, [&](auto d, auto kind, auto io) {
    constexpr int D = decltype(d)::value, K = decltype(kind)::value, I = decltype(io)::value;
    if (k->tokens <= kFewRows) return launch_pdl(append8_few_kernel<D, K, I>, dim3(n), std::min(2 * c->cfg.n_kv_heads, kFewWarps) * 32, 0, 1, as_stream(stream), c->view, a);
    return launch_pdl(rotary ? append8_kernel<D, K, I, true> : append8_kernel<D, K, I, false>, dim3(pages, (2 * c->cfg.n_kv_heads + a.per - 1) / a.per, n), quad_threads(c), (size_t)R * a.rot / 2 * sizeof(float2), 1,
                      as_stream(stream), c->view, a);
  }));
  return DKV_OK;
}

int dkv_cache8_read(dkv_cache8* c, int32_t first, int32_t n, int32_t step, const dkv_rows* k_out, const dkv_rows* v_out, void* stream) {
  if (int rc = check(c, first, n, step)) return rc;
  if (!fits(c, k_out, n, c->cfg.n_kv_heads) || !fits(c, v_out, n, c->cfg.n_kv_heads) || k_out->tokens != v_out->tokens) return DKV_ERR_INVALID_ARG;
  if (n == 0 || k_out->tokens == 0) return DKV_OK;
  const ReadArgs a = {rows8(k_out), rows8(v_out), first, step, k_out->tokens};
  const int R = c->cfg.page_rows, pages = std::min((int)(((long long)k_out->tokens + R - 1) / R), c->cfg.max_pages);
  C8_LAUNCH(c, with_types(c, [&](auto d, auto kind, auto io) {
    return launch_pdl(read8_kernel<decltype(d)::value, decltype(kind)::value, decltype(io)::value>, dim3(pages, 2 * c->cfg.n_kv_heads, n), quad_threads(c), 0, 1,
                      as_stream(stream), c->view, a);
  }));
  return DKV_OK;
}

int dkv_cache8_attend(dkv_cache8* c, int32_t first, int32_t n, int32_t step, const dkv_rows* q, const dkv_rows* out, float* lse, int32_t causal,
                      void* stream) {
  if (int rc = check(c, first, n, step)) return rc;
  if (!fits(c, q, n, c->cfg.n_q_heads) || !valid(out) || out->type != DKV_F32 || !aligned(lse, 4)) return DKV_ERR_INVALID_ARG;
  if (out->batch != n || out->heads != q->heads || out->tokens != q->tokens || out->head_dim != q->head_dim || !vectors(*out)) return DKV_ERR_INVALID_ARG;
  const int G = c->cfg.n_q_heads / c->cfg.n_kv_heads;
  if ((long long)G * q->tokens > kMostQueries) return DKV_ERR_INVALID_ARG;
  if (n == 0 || q->tokens == 0) return DKV_OK;
  AttendArgs a;
  memset(&a, 0, sizeof a);
  a.q_batch = q->batch_stride; a.q_head = q->head_stride; a.q_token = q->token_stride;
  a.out_batch = out->batch_stride; a.out_head = out->head_stride; a.out_token = out->token_stride;
  a.scratch = c->d_scratch; a.tickets = c->d_tickets;
  a.step = step; a.nq = q->tokens; a.rows = G * q->tokens; a.G = G; a.causal = causal != 0; a.io = c->cfg.io; a.wait = c->wait_cycles; a.withhold = c->withhold;
  a.slots = (a.rows + (a.rows <= 8 ? 7 : 15)) / (a.rows <= 8 ? 8 : 16);
  a.scale2 = kLog2e / sqrtf((float)c->cfg.head_dim);
  // sequences a launch: their prefix sums fit shared memory, and their units (chunks, at most) 31 bits
  const long long units = (long long)c->cfg.n_kv_heads * (((long long)c->cfg.max_pages * c->cfg.page_rows) / kAttendRows + kAttendHeadCost);
  const int most = (int)std::max(1ll, std::min<long long>(kAttendMaxSeqs, INT_MAX / units));
  for (int i = 0; i < n; i += most) {
    a.n = std::min(most, n - i); a.first = first + i * step;
    a.q = static_cast<const char*>(q->data) + (size_t)i * a.q_batch * 2;
    a.out = static_cast<float*>(out->data) + (size_t)i * a.out_batch;
    a.lse = lse ? lse + (size_t)i * c->cfg.n_q_heads * a.nq : nullptr;
    C8_LAUNCH(c, c->cfg.head_dim == 64 ? launch_attend<64>(c, a, as_stream(stream)) : launch_attend<128>(c, a, as_stream(stream)));
  }
  return DKV_OK;
}

int dkv_cache8_fork(dkv_cache8* c, int32_t from, int32_t to, int32_t n, int32_t step, void* stream) {
  if (int rc = check(c, from, n, step)) return rc;
  if (int rc = check(c, to, n, step)) return rc;
  if (n == 0) return DKV_OK;
  const long long apart = (long long)to - from;                              // a common sequence: a whole number of steps, fewer than n
  if (apart % step == 0 && std::llabs(apart / step) < n) return DKV_ERR_INVALID_ARG;
  C8_LAUNCH(c, launch_pdl(fork8_kernel, dim3(n), kSeqThreads, 0, 1, as_stream(stream), c->view, (int)from, (int)to, (int)step));
  return DKV_OK;
}

int dkv_cache8_compact(dkv_cache8* c, int32_t first, int32_t n, int32_t step, const int32_t* idx, int32_t heads, int32_t cols, const int32_t* count,
                       void* stream) {
  if (int rc = check(c, first, n, step)) return rc;
  if (heads != c->cfg.n_kv_heads || cols < 0 || (cols && !idx) || !aligned(idx, 4) || !aligned(count, 4)) return DKV_ERR_INVALID_ARG;
  if (n == 0) return DKV_OK;
  const PlanArgs p = {count, c->d_pick, c->d_jobs, c->d_new_table, c->d_new_held, first, step, n, cols};
  const CompactArgs a = {idx, count, c->d_new_table, c->d_new_held, c->d_tickets, first, step, cols};
  cudaStream_t st = as_stream(stream);
  C8_LAUNCH(c, launch_pdl(plan_compact8_kernel, dim3(1), kPlanThreads, 0, 1, st, c->view, p));
  const int R = c->cfg.page_rows, pages = std::max(1, std::min((int)(((long long)cols + R - 1) / R), c->cfg.max_pages));
  C8_LAUNCH(c, with_types(c, [&](auto d, auto kind, auto) {
    return launch_pdl(compact8_kernel<decltype(d)::value, decltype(kind)::value>, dim3(pages, c->cfg.n_kv_heads, n), quad_threads(c), 0, 1, st, c->view, a);
  }));
  return DKV_OK;
}

int dkv_cache8_trim(dkv_cache8* c, int32_t first, int32_t n, int32_t step, const int32_t* keep, int32_t drop, void* stream) {
  if (int rc = check(c, first, n, step)) return rc;
  if (!aligned(keep, 4) || (!keep && drop < 0)) return DKV_ERR_INVALID_ARG;
  if (n == 0) return DKV_OK;
  C8_LAUNCH(c, launch_pdl(trim8_kernel, dim3(n), kSeqThreads, 0, 1, as_stream(stream), c->view, (int)first, (int)step, (const int*)keep, (int)drop));
  return DKV_OK;
}

int dkv_cache8_views(dkv_cache8* c, const int32_t** len, const int32_t** held, const int32_t** table, const int32_t** refs) {
  if (!c) return DKV_ERR_INVALID_ARG;
  if (len) *len = c->view.len;
  if (held) *held = c->view.held;
  if (table) *table = c->view.table;
  if (refs) *refs = c->view.refs;
  return DKV_OK;
}

int dkv_cache8_status(dkv_cache8* c, int32_t* host_status) {
  if (int rc = check(c, 0, 0, 1)) return rc;                                 // another device's kernels would be waited for, not the cache's
  if (!host_status) return DKV_ERR_INVALID_ARG;
  C8_CUDA(c, cudaDeviceSynchronize());
  int status[2];
  const int clear[2] = {0, INT_MAX}, words = (c->cfg.n_pages + 31) / 32;
  std::vector<unsigned int> bits;
  try { bits.resize(words); } catch (const std::bad_alloc&) { return DKV_ERR_NOMEM; }
  C8_CUDA(c, cudaMemcpy(status, c->view.status, sizeof status, cudaMemcpyDeviceToHost));
  C8_CUDA(c, cudaMemcpy(c->view.status, clear, sizeof clear, cudaMemcpyHostToDevice));
  C8_CUDA(c, cudaMemcpy(bits.data(), c->view.free, sizeof(int) * words, cudaMemcpyDeviceToHost));
  int pages = 0;
  for (unsigned int b : bits) pages += __builtin_popcount(b);
  memset(host_status, 0, sizeof(int32_t) * 8);
  host_status[0] = status[0];
  host_status[1] = status[1] == INT_MAX ? -1 : status[1];
  host_status[2] = pages;
  host_status[3] = (int32_t)(c->launches & 0xFFFFFFFF); host_status[4] = (int32_t)(c->launches >> 32);
  if (status[0] & kTimeout) return DKV_ERR_TIMEOUT;
  if (status[0] & (kNoPages | kTableFull)) return DKV_ERR_NOMEM;
  return status[0] & kNoRoom ? DKV_ERR_STATE : status[0] & kBadArgument ? DKV_ERR_INVALID_ARG : DKV_OK;
}

int dkv_cache8_set_wait_limit(dkv_cache8* c, int64_t clock_ticks) {
  if (!c || clock_ticks < 1000) return DKV_ERR_INVALID_ARG;
  c->wait_cycles = clock_ticks;
  return DKV_OK;
}

int dkv_cache8_debug_withhold(dkv_cache8* c, int32_t chunk) {
  if (!c) return DKV_ERR_INVALID_ARG;
  c->withhold = chunk < 0 ? -1 : chunk;
  return DKV_OK;
}

int dkv_cache8_last_cuda_error(dkv_cache8* c) { return c ? c->last_cuda : 0; }

}  // extern "C"
