// Native half of binding.py: turns the arguments of the calls a serving loop makes (torch tensors, numpy arrays,
// integer addresses, lists of them, streams) into the C ABI's pointers and makes the call without the GIL.
//
// Why it exists: a decoding step calls the library once per layer and a pass hands over five lists of per-layer
// tensors.  Taking every address through Python attribute look-ups and ctypes arrays costs about 0.3 us a tensor and
// 8 us a call (a 32-layer dkv_decode_attend: 40 us on the host for a kernel of a third of that); here a tensor's
// address is a field read.  Every function returns the library's code; binding.py raises on it.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <stdint.h>

#include <exception>

#include "../../include/dkv.h"

namespace {

constexpr Py_ssize_t kMaxList = 4096;       // longest list of per-layer tensors taken

// Address of a torch tensor, a ctypes structure, an integer, None (NULL), or of anything with data_ptr() (a tensor subclass may have its own)
// or a numpy-like .ctypes.data.
bool address(PyObject* x, void** out) {
  if (x == Py_None) { *out = nullptr; return true; }
  if (THPVariable_CheckExact(x)) { *out = THPVariable_Unpack(x).data_ptr(); return true; }
  if (PyObject_CheckBuffer(x) && PyObject_HasAttrString(x, "_fields_")) {       // a ctypes structure: its own memory
    Py_buffer b;
    if (PyObject_GetBuffer(x, &b, PyBUF_SIMPLE) < 0) return false;
    *out = b.buf;
    PyBuffer_Release(&b);
    return true;
  }
  PyObject* v = nullptr;
  if (PyLong_Check(x)) {
    v = x;
    Py_INCREF(v);
  } else if (PyObject_HasAttrString(x, "data_ptr")) {
    v = PyObject_CallMethod(x, "data_ptr", nullptr);
  } else if (PyObject_HasAttrString(x, "ctypes")) {
    PyObject* c = PyObject_GetAttrString(x, "ctypes");
    if (c) { v = PyObject_GetAttrString(c, "data"); Py_DECREF(c); }
  } else {
    PyErr_Format(PyExc_TypeError, "cannot take the address of %R", (PyObject*)Py_TYPE(x));
  }
  if (!v) return false;
  *out = PyLong_AsVoidPtr(v);
  Py_DECREF(v);
  return !PyErr_Occurred();
}

// None: torch's current stream; an integer: a cudaStream_t; else an object with .cuda_stream.
bool stream_of(PyObject* x, void** out) {
  if (x == Py_None) { *out = (void*)c10::cuda::getCurrentCUDAStream().stream(); return true; }
  if (PyLong_Check(x)) { *out = PyLong_AsVoidPtr(x); return !PyErr_Occurred(); }
  PyObject* v = PyObject_GetAttrString(x, "cuda_stream");
  if (!v) return false;
  *out = PyLong_AsVoidPtr(v);
  Py_DECREF(v);
  return !PyErr_Occurred();
}

// The addresses of a sequence's items.  The library reads one address a layer, whatever the length of the list: there
// are never fewer than DKV_MAX_LAYERS entries, and a list that is too short ends in NULLs, which the library refuses.
struct Addresses {
  void* few[DKV_MAX_LAYERS] = {};
  void** p = few;
  PyObject* items = nullptr;
  ~Addresses() {
    if (p != few) PyMem_Free(p);
    Py_XDECREF(items);
  }
  bool take(PyObject* seq) {
    items = PySequence_Fast(seq, "a sequence of tensors or addresses is expected");
    if (!items) return false;
    const Py_ssize_t n = PySequence_Fast_GET_SIZE(items);
    if (n > kMaxList) { PyErr_SetString(PyExc_ValueError, "too many tensors"); return false; }
    if (n > DKV_MAX_LAYERS) {
      void** more = static_cast<void**>(PyMem_Malloc(sizeof(void*) * n));
      if (!more) { PyErr_NoMemory(); return false; }
      p = more;
    }
    for (Py_ssize_t i = 0; i < n && i < PySequence_Fast_GET_SIZE(items); ++i)      // (an item's own code may shorten its list)
      if (!address(PySequence_Fast_GET_ITEM(items, i), &p[i])) return false;
    return true;
  }
};

// A 32-bit integer; one that does not fit is refused rather than cut to another layer or count.
bool number(PyObject* x, int32_t* out) {
  const long v = PyLong_AsLong(x);
  if (v == -1 && PyErr_Occurred()) return false;
  if (v != (int32_t)v) { PyErr_SetString(PyExc_OverflowError, "an integer does not fit 32 bits"); return false; }
  *out = (int32_t)v;
  return true;
}

// Every function: `n` arguments exactly, conversions by the lines given, then the call without the GIL.
#define DKV_PY(NAME, N, CONVERT, CALL)                                                        \
  PyObject* py_##NAME(PyObject*, PyObject* const* a, Py_ssize_t n) {                          \
    if (n != (N)) { PyErr_SetString(PyExc_TypeError, #NAME ": wrong number of arguments"); return nullptr; } \
    try {                                                                                     \
      CONVERT                                                                                 \
      int rc;                                                                                 \
      Py_BEGIN_ALLOW_THREADS                                                                  \
      rc = CALL;                                                                              \
      Py_END_ALLOW_THREADS                                                                    \
      return PyLong_FromLong(rc);                                                             \
    } catch (const std::exception& e) {                                                       \
      PyErr_SetString(PyExc_RuntimeError, e.what());                                          \
      return nullptr;                                                                         \
    }                                                                                         \
  }
#define CTX(I) void* cp_; if (!address(a[I], &cp_)) return nullptr; dkv_ctx* c = static_cast<dkv_ctx*>(cp_);
#define INT(V, I) int32_t V; if (!number(a[I], &V)) return nullptr;
#define PTR(V, I) void* V; if (!address(a[I], &V)) return nullptr;
#define SIZE(V, I) const uint64_t V = PyLong_AsUnsignedLongLong(a[I]); if (PyErr_Occurred()) return nullptr;
#define STREAM(I) void* st; if (!stream_of(a[I], &st)) return nullptr;
#define LIST(V, I) Addresses V; if (!V.take(a[I])) return nullptr;

DKV_PY(reset, 2, CTX(0) STREAM(1), dkv_reset(c, st))
DKV_PY(score, 6, CTX(0) INT(l, 1) PTR(q, 2) PTR(k, 3) PTR(o, 4) STREAM(5), dkv_score(c, l, q, k, (float*)o, st))
DKV_PY(score_lse, 7, CTX(0) INT(l, 1) PTR(q, 2) PTR(k, 3) PTR(e, 4) PTR(o, 5) STREAM(6),
       dkv_score_lse(c, l, q, k, (const float*)e, (float*)o, st))
DKV_PY(score_static, 5, PTR(cfg, 0) PTR(q, 1) PTR(k, 2) PTR(o, 3) STREAM(4),
       dkv_score_static((const dkv_config*)cfg, q, k, (float*)o, st))
DKV_PY(set_scores, 4, CTX(0) INT(l, 1) PTR(s, 2) STREAM(3), dkv_set_scores(c, l, (const float*)s, st))
DKV_PY(select_topk, 5, CTX(0) INT(l, 1) PTR(i, 2) PTR(r, 3) STREAM(4), dkv_select_topk(c, l, (int32_t*)i, (int32_t*)r, st))
DKV_PY(rebudget, 4, CTX(0) INT(l, 1) PTR(o, 2) STREAM(3), dkv_rebudget(c, l, (int32_t*)o, st))
DKV_PY(compact, 8, CTX(0) INT(l, 1) PTR(ks, 2) PTR(vs, 3) PTR(kb, 4) PTR(vb, 5) PTR(len, 6) STREAM(7),
       dkv_compact(c, l, ks, vs, kb, vb, (int32_t*)len, st))
DKV_PY(compact_all, 5, CTX(0) INT(l, 1) LIST(kb, 2) LIST(vb, 3) STREAM(4), dkv_compact_all(c, l, kb.p, vb.p, st))
DKV_PY(run_prefill_pass, 7, CTX(0) LIST(q, 1) LIST(k, 2) LIST(v, 3) LIST(kb, 4) LIST(vb, 5) STREAM(6),
       dkv_run_prefill_pass(c, q.p, k.p, v.p, kb.p, vb.p, st))
DKV_PY(run_prefill_pass_lse, 8, CTX(0) LIST(q, 1) LIST(k, 2) LIST(v, 3) LIST(e, 4) LIST(kb, 5) LIST(vb, 6) STREAM(7),
       dkv_run_prefill_pass_lse(c, q.p, k.p, v.p, (const float* const*)e.p, kb.p, vb.p, st))
DKV_PY(run_prefill_pass_host, 7, CTX(0) LIST(q, 1) LIST(k, 2) LIST(v, 3) LIST(kb, 4) LIST(vb, 5) PTR(o, 6),
       dkv_run_prefill_pass_host(c, q.p, k.p, v.p, kb.p, vb.p, (int32_t*)o))
DKV_PY(apply_policy, 4, CTX(0) INT(p, 1) PTR(o, 2) STREAM(3), dkv_apply_policy(c, p, (int32_t*)o, st))
DKV_PY(select_positions, 5, CTX(0) INT(l, 1) INT(s, 2) INT(r, 3) STREAM(4), dkv_select_positions(c, l, s, r, st))
DKV_PY(decode_attend, 9, CTX(0) INT(l, 1) INT(nl, 2) INT(nq, 3) LIST(q, 4) LIST(kb, 5) LIST(vb, 6) LIST(o, 7) STREAM(8),
       dkv_decode_attend(c, l, nl, nq, q.p, kb.p, vb.p, (float* const*)o.p, st))
DKV_PY(get_counts, 3, CTX(0) PTR(o, 1) STREAM(2), dkv_get_counts(c, (int32_t*)o, st))
DKV_PY(memcpy_to_host, 5, CTX(0) PTR(dst, 1) PTR(src, 2) SIZE(bytes, 3) STREAM(4), dkv_memcpy_to_host(c, dst, src, bytes, st))
DKV_PY(kept_sorted, 4, CTX(0) INT(l, 1) PTR(o, 2) STREAM(3), dkv_kept_sorted(c, l, (int32_t*)o, st))

// On the current device, where the calls that take tensors run.
bool here(const at::Tensor& t) { return t.is_cuda() && t.get_device() == c10::cuda::current_device(); }

// A strided tensor [batch, heads, tokens, head_dim] on the current GPU, None (NULL), or the address of a dkv_rows.  A tensor that has not
// this form becomes one without a type, which the library refuses.
struct Rows {
  dkv_rows own;
  const dkv_rows* p = nullptr;
  bool take(PyObject* x) {
    if (x == Py_None) return true;
    if (!THPVariable_Check(x)) {
      void* at;
      if (!address(x, &at)) return false;
      p = static_cast<const dkv_rows*>(at);
      return true;
    }
    const at::Tensor& t = THPVariable_Unpack(x);
    own = {};
    own.type = -1;
    p = &own;
    if (!here(t) || t.dim() != 4 || (t.size(3) > 1 && t.stride(3) != 1)) return true;
    int32_t size[4];
    for (int i = 0; i < 4; ++i) {
      if (t.size(i) > INT32_MAX) return true;
      size[i] = (int32_t)t.size(i);
    }
    switch (t.scalar_type()) {
      case at::kBFloat16: own.type = DKV_BF16; break;
      case at::kHalf: own.type = DKV_F16; break;
      case at::kFloat: own.type = DKV_F32; break;
      case at::kShort: case at::kUInt16: own.type = DKV_RAW16; break;
      default: return true;
    }
    own.data = t.data_ptr();
    own.batch = size[0]; own.heads = size[1]; own.tokens = size[2]; own.head_dim = size[3];
    own.batch_stride = t.stride(0); own.head_stride = t.stride(1); own.token_stride = t.stride(2);
    return true;
  }
};
// A contiguous tensor of `need` 32-bit numbers at least on the current GPU, None (NULL), or an address.  *bad: it is not that.
bool numbers(PyObject* x, c10::ScalarType type, int64_t need, void** out, bool* bad) {
  if (!THPVariable_Check(x)) return address(x, out);
  const at::Tensor& t = THPVariable_Unpack(x);
  *bad = *bad || !here(t) || t.scalar_type() != type || !t.is_contiguous() || t.numel() < need;
  *out = t.data_ptr();
  return true;
}
// Tokens of a batch in a tensor that take() accepted.
int64_t tokens_of(const Rows& r) { return r.p ? (int64_t)r.p->batch * r.p->tokens : 0; }

#define CACHE(I) void* cp_; if (!address(a[I], &cp_)) return nullptr; dkv_cache8* c = static_cast<dkv_cache8*>(cp_); bool bad = false; (void)bad;
#define ROWS(V, I) Rows V; if (!V.take(a[I])) return nullptr;
#define INTS(V, I, NEED) void* V##_p; if (!numbers(a[I], at::kInt, NEED, &V##_p, &bad)) return nullptr; const int32_t* V = static_cast<const int32_t*>(V##_p);
#define SEQS INT(first, 1) INT(n, 2) INT(step, 3)

DKV_PY(rotate, 8, bool bad = false; PTR(r, 0) ROWS(x, 2) ROWS(xo, 3) ROWS(y, 4) ROWS(yo, 5) INTS(pos, 1, tokens_of(x)) INT(tr, 6) STREAM(7),
       bad ? DKV_ERR_INVALID_ARG : dkv_rotate((const dkv_rotary*)r, pos, x.p, xo.p, y.p, yo.p, tr, st))
DKV_PY(cache8_reserve, 7, CACHE(0) SEQS INTS(rows, 4, n) INT(add, 5) STREAM(6),
       bad ? DKV_ERR_INVALID_ARG : dkv_cache8_reserve(c, first, n, step, rows, add, st))
DKV_PY(cache8_append, 10, CACHE(0) SEQS ROWS(k, 4) ROWS(v, 5) INTS(rows, 6, n) PTR(r, 7) INTS(pos, 8, n) STREAM(9),
       bad ? DKV_ERR_INVALID_ARG : dkv_cache8_append(c, first, n, step, k.p, v.p, rows, (const dkv_rotary*)r, pos, st))
DKV_PY(cache8_read, 7, CACHE(0) SEQS ROWS(k, 4) ROWS(v, 5) STREAM(6), dkv_cache8_read(c, first, n, step, k.p, v.p, st))
DKV_PY(cache8_attend, 9, CACHE(0) SEQS ROWS(q, 4) ROWS(o, 5)
       void* lse; if (!numbers(a[6], at::kFloat, q.p ? tokens_of(q) * q.p->heads : 0, &lse, &bad)) return nullptr; INT(causal, 7) STREAM(8),
       bad ? DKV_ERR_INVALID_ARG : dkv_cache8_attend(c, first, n, step, q.p, o.p, (float*)lse, causal, st))
DKV_PY(cache8_fork, 6, CACHE(0) INT(from, 1) INT(to, 2) INT(n, 3) INT(step, 4) STREAM(5), dkv_cache8_fork(c, from, to, n, step, st))
// idx: a tensor [n, heads, cols], or an address with `heads` and `cols`.
DKV_PY(cache8_compact, 9, CACHE(0) SEQS INTS(idx, 4, 0) INT(heads, 5) INT(cols, 6) INTS(count, 7, n) STREAM(8)
       if (THPVariable_Check(a[4])) {
         const at::Tensor& t = THPVariable_Unpack(a[4]);
         bad = bad || t.dim() != 3 || t.size(0) != n || t.size(1) > INT32_MAX || t.size(2) > INT32_MAX;
         if (!bad) { heads = (int32_t)t.size(1); cols = (int32_t)t.size(2); }
       },
       bad ? DKV_ERR_INVALID_ARG : dkv_cache8_compact(c, first, n, step, idx, heads, cols, count, st))
DKV_PY(cache8_trim, 7, CACHE(0) SEQS INTS(keep, 4, n) INT(drop, 5) STREAM(6),
       bad ? DKV_ERR_INVALID_ARG : dkv_cache8_trim(c, first, n, step, keep, drop, st))

#define ENTRY(NAME) {#NAME, (PyCFunction)(void*)py_##NAME, METH_FASTCALL, nullptr}
PyMethodDef kMethods[] = {
    ENTRY(reset), ENTRY(score), ENTRY(score_lse), ENTRY(score_static), ENTRY(set_scores), ENTRY(select_topk),
    ENTRY(rebudget), ENTRY(compact), ENTRY(compact_all), ENTRY(run_prefill_pass), ENTRY(run_prefill_pass_lse),
    ENTRY(run_prefill_pass_host), ENTRY(apply_policy), ENTRY(select_positions), ENTRY(decode_attend),
    ENTRY(get_counts), ENTRY(kept_sorted), ENTRY(memcpy_to_host), ENTRY(rotate), ENTRY(cache8_reserve), ENTRY(cache8_append),
    ENTRY(cache8_read), ENTRY(cache8_attend), ENTRY(cache8_fork), ENTRY(cache8_compact), ENTRY(cache8_trim), {nullptr, nullptr, 0, nullptr}};
PyModuleDef kModule = {PyModuleDef_HEAD_INIT, "_dkv_pycall", nullptr, -1, kMethods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__dkv_pycall(void) { return PyModule_Create(&kModule); }
