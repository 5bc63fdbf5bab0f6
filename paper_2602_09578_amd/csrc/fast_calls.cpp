// The Python binding's short way into the library for the calls of a decode loop: the same checks of types,
// extents, device and contiguity as in binding.py, made on the tensors themselves, and the call, in one step.
// A call whose arguments are not plainly right is not made here: None is returned and the binding goes its long
// way, which reports what is wrong.  (Host time of a call, long way and short: attention of 16 sequences 7.9 and 3.5 us,
// log-probabilities 5.8 and 3.0, prompt scatter 7.4 and 3.5; most of what is left is the launch.)
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <torch/csrc/autograd/python_variable.h>
#include <torch/version.h>

#include <exception>
#include <initializer_list>
#include <type_traits>

#include "marl_decode.h"

namespace {

PyObject* g_stream_of = nullptr;      // device index -> the current stream's handle
PyObject* g_attn_shape = nullptr;     // the ctypes structures' types
PyObject* g_prefill_shape = nullptr;
decltype(&marl_decode_attn) f_decode_attn;
decltype(&marl_token_logprobs) f_token_logprobs;
decltype(&marl_kv_append) f_kv_append;
decltype(&marl_sample_tokens) f_sample_tokens;
decltype(&marl_sample_tokens_top_p) f_sample_tokens_top_p;
decltype(&marl_prefill_attn) f_prefill_attn;
decltype(&marl_kv_write_prompt) f_kv_write_prompt;
decltype(&marl_decode_attn_fp8) f_decode_attn_fp8;
decltype(&marl_kv_append_fp8) f_kv_append_fp8;
decltype(&marl_kv_write_prompt_fp8) f_kv_write_prompt_fp8;
decltype(&marl_kv_read_pages_fp8) f_kv_read_pages_fp8;
decltype(&marl_qk_norm_rope) f_qk_norm_rope;
decltype(&marl_qk_norm_rope_backward) f_qk_norm_rope_backward;

struct Call {
  bool ok = true;
  int device = -1;   // of the first tensor

  // The data of a plain, contiguous device tensor of the given type and sizes (-1: any, at least that many dimensions are
  // there); null for None.
  const at::Tensor* tensor(PyObject* o, at::ScalarType type, std::initializer_list<int64_t> sizes) {
    if (!ok || !THPVariable_CheckExact(o)) return fail();
    const at::Tensor& t = THPVariable_Unpack(o);
    if (!t.is_cuda() || t.scalar_type() != type || !t.is_contiguous() || t.dim() != (int64_t)sizes.size()) return fail();
    int k = 0;
    for (int64_t n : sizes) {
      if (n >= 0 && t.size(k) != n) return fail();
      ++k;
    }
    if (device < 0) device = t.get_device();
    return &t;
  }
  template <class T = void>
  T* data(PyObject* o, at::ScalarType type, std::initializer_list<int64_t> sizes) {
    if (o == Py_None) return nullptr;
    const at::Tensor* t = tensor(o, type, sizes);
    return t ? static_cast<T*>(t->data_ptr()) : nullptr;
  }
  // rows [tokens, heads, D] whose heads are contiguous; tokens lie `stride` elements apart
  void* rows(PyObject* o, at::ScalarType type, int64_t tokens, int64_t heads, int64_t D, int64_t& stride) {
    stride = heads * D;
    if (!ok || !THPVariable_CheckExact(o)) { fail(); return nullptr; }
    const at::Tensor& t = THPVariable_Unpack(o);
    if (!t.is_cuda() || t.scalar_type() != type || t.dim() != 3 || t.size(0) != tokens || t.size(1) != heads || t.size(2) != D ||
        t.stride(2) != 1 || (heads > 1 && t.stride(1) != D)) { fail(); return nullptr; }
    if (tokens > 1) stride = t.stride(0);
    if (device < 0) device = t.get_device();
    return t.data_ptr();
  }
  // a workspace: bytes of any number
  void* bytes(PyObject* o, size_t& n) {
    n = 0;
    if (o == Py_None) return nullptr;
    const at::Tensor* t = tensor(o, at::kByte, {-1});
    if (!t) return nullptr;
    n = (size_t)t->numel();
    return t->data_ptr();
  }
  float number(PyObject* o) {
    const double v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) fail();
    return (float)v;
  }
  void* stream() {
    if (!ok || device < 0) { fail(); return nullptr; }
    PyObject* index = PyLong_FromLong(device);
    PyObject* r = index ? PyObject_CallFunctionObjArgs(g_stream_of, index, nullptr) : nullptr;
    Py_XDECREF(index);
    if (!r) { fail(); return nullptr; }
    void* st = PyLong_AsVoidPtr(r);
    Py_DECREF(r);
    if (PyErr_Occurred()) fail();
    return st;
  }
  const at::Tensor* fail() { ok = false; return nullptr; }
};

// The C structure behind a ctypes one of the given type (other objects may have as many bytes).
template <class S>
struct Struct {
  Py_buffer view{};
  bool ok;
  Struct(PyObject* o, PyObject* type)
      : ok(type && PyObject_TypeCheck(o, reinterpret_cast<PyTypeObject*>(type)) && PyObject_GetBuffer(o, &view, PyBUF_SIMPLE) == 0) {
    if (ok && view.len != (Py_ssize_t)sizeof(S)) { PyBuffer_Release(&view); ok = false; }
  }
  ~Struct() { if (ok) PyBuffer_Release(&view); }
  const S* get() const { return static_cast<const S*>(view.buf); }
};

PyObject* not_here() {
  PyErr_Clear();
  Py_RETURN_NONE;
}
// (torch reports some tensors without memory of their own by an exception)
template <class F>
PyObject* guarded(F&& f) {
  try {
    return f();
  } catch (...) {
    return not_here();
  }
}
struct WithoutGil {   // (given back also where the call ends by an exception)
  PyThreadState* state = PyEval_SaveThread();
  ~WithoutGil() { PyEval_RestoreThread(state); }
};
// An exception out of the library is the call's result: it may have enqueued work, so the call is not made again.
template <class F>
PyObject* finish(Call& c, F&& call) {
  if (!c.ok) return not_here();
  int rc;
  try {
    WithoutGil released;
    rc = call();
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
    return nullptr;
  } catch (...) {
    PyErr_SetString(PyExc_RuntimeError, "exception in the library");
    return nullptr;
  }
  return PyLong_FromLong(rc);
}

constexpr auto kBf16 = at::kBFloat16;
constexpr auto kI32 = at::kInt;
at::ScalarType out_type(int32_t out_dtype) { return out_dtype == MARL_OUT_BF16 ? kBf16 : at::kFloat; }

// shape, workspace, q, k_pages, v_pages, prefix_block_table, suffix_block_table, prefix_lens, suffix_lens, group_of_seq, scale, out
PyObject* decode_attn(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    if (n != 12 || !f_decode_attn) Py_RETURN_NONE;
    Struct<marl_attn_shape> s(a[0], g_attn_shape);
    if (!s.ok) return not_here();
    const marl_attn_shape& h = *s.get();
    if (a[1] == Py_None || a[11] == Py_None) return not_here();
    if (h.max_prefix_pages <= 0 || h.max_suffix_pages <= 0) return not_here();   // (tables whose extents are not looked at)
    Call c;
    void* out = c.data(a[11], out_type(h.out_dtype), {h.num_seqs, h.num_q_heads, 128});   // (first: the call's device)
    size_t bytes;
    void* ws = c.bytes(a[1], bytes);
    const void* q = c.data(a[2], kBf16, {h.num_seqs, h.num_q_heads, 128});
    const void* k = c.data(a[3], kBf16, {h.num_pages, h.num_kv_heads, 16, 128});
    const void* v = c.data(a[4], kBf16, {h.num_pages, h.num_kv_heads, 128, 16});
    const int32_t* pt = c.data<int32_t>(a[5], kI32, {h.num_groups, h.max_prefix_pages});
    const int32_t* st = c.data<int32_t>(a[6], kI32, {h.num_seqs, h.max_suffix_pages});
    const int32_t* pl = c.data<int32_t>(a[7], kI32, {h.num_groups});
    const int32_t* sl = c.data<int32_t>(a[8], kI32, {h.num_seqs});
    const int32_t* gs = c.data<int32_t>(a[9], kI32, {h.num_seqs});
    const float scale = c.number(a[10]);
    void* stream = c.stream();
    return finish(c, [&] { return f_decode_attn(&h, ws, bytes, q, k, v, pt, st, pl, sl, gs, scale, out, stream); });
  });
}

// logits, tokens, temperature, out, workspace
PyObject* token_logprobs(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    if (n != 5 || !f_token_logprobs) Py_RETURN_NONE;
    Call c;
    const at::Tensor* x = c.tensor(a[0], kBf16, {-1, -1});
    if (!x || a[1] == Py_None || a[3] == Py_None) return not_here();
    const int64_t rows = x->size(0), vocab = x->size(1);
    if (rows > INT32_MAX || vocab > INT32_MAX) return not_here();
    const int32_t* tokens = c.data<int32_t>(a[1], kI32, {rows});
    const float temperature = c.number(a[2]);
    float* out = c.data<float>(a[3], at::kFloat, {rows});
    size_t bytes;
    void* ws = c.bytes(a[4], bytes);
    void* stream = c.stream();
    return finish(c, [&] { return f_token_logprobs(x->data_ptr(), tokens, temperature, out, (int32_t)rows, (int32_t)vocab, ws, bytes, stream); });
  });
}

// logits, uniforms, temperature, top_p or None, out_tokens, out_logprobs, workspace (not with top_p)
PyObject* sample_tokens(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    if (n != 7 || !f_sample_tokens || !f_sample_tokens_top_p) Py_RETURN_NONE;
    Call c;
    const at::Tensor* x = c.tensor(a[0], kBf16, {-1, -1});
    const bool nucleus = a[3] != Py_None;
    if (!x || a[1] == Py_None || a[4] == Py_None || a[5] == Py_None || (!nucleus && a[6] == Py_None)) return not_here();
    const int64_t rows = x->size(0), vocab = x->size(1);
    if (rows > INT32_MAX || vocab > INT32_MAX) return not_here();
    const float* u = c.data<float>(a[1], at::kFloat, {rows});
    const float temperature = c.number(a[2]);
    int32_t* tokens = c.data<int32_t>(a[4], kI32, {rows});
    float* logprobs = c.data<float>(a[5], at::kFloat, {rows});
    const void* logits = x->data_ptr();
    if (nucleus) {
      const float top_p = c.number(a[3]);
      void* stream = c.stream();
      return finish(c, [&] { return f_sample_tokens_top_p(logits, u, temperature, top_p, tokens, logprobs, (int32_t)rows, (int32_t)vocab, stream); });
    }
    size_t bytes;
    void* ws = c.bytes(a[6], bytes);
    void* stream = c.stream();
    return finish(c, [&] { return f_sample_tokens(logits, u, temperature, tokens, logprobs, (int32_t)rows, (int32_t)vocab, ws, bytes, stream); });
  });
}

// shape, k_new, v_new, k_pages, v_pages, suffix_block_table, suffix_lens, flags
PyObject* kv_append(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    if (n != 8 || !f_kv_append) Py_RETURN_NONE;
    Struct<marl_attn_shape> s(a[0], g_attn_shape);
    if (!s.ok || a[3] == Py_None || a[7] != Py_None) return not_here();
    const marl_attn_shape& h = *s.get();
    Call c;
    void* k = c.data(a[3], kBf16, {h.num_pages, h.num_kv_heads, 16, 128});
    void* v = c.data(a[4], kBf16, {h.num_pages, h.num_kv_heads, 128, 16});
    const void* kn = c.data(a[1], kBf16, {h.num_seqs, h.num_kv_heads, 128});
    const void* vn = c.data(a[2], kBf16, {h.num_seqs, h.num_kv_heads, 128});
    const int32_t* st = c.data<int32_t>(a[5], kI32, {h.num_seqs, h.max_suffix_pages});
    int32_t* sl = c.data<int32_t>(a[6], kI32, {h.num_seqs});
    void* stream = c.stream();
    return finish(c, [&] { return f_kv_append(&h, kn, vn, k, v, st, sl, nullptr, stream); });
  });
}

// shape, workspace, q, k_pages, v_pages, prefix_block_table, q_start, q_pos0, scale, out
PyObject* prefill_attn(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    if (n != 10 || !f_prefill_attn) Py_RETURN_NONE;
    Struct<marl_prefill_shape> s(a[0], g_prefill_shape);
    if (!s.ok || a[1] == Py_None || a[2] == Py_None) return not_here();
    const marl_prefill_shape& h = *s.get();
    Call c;
    const void* q = c.data(a[2], kBf16, {h.num_tokens, h.num_q_heads, 128});   // (first: the call's device)
    size_t bytes;
    void* ws = c.bytes(a[1], bytes);
    const void* k = c.data(a[3], kBf16, {h.num_pages, h.num_kv_heads, 16, 128});
    const void* v = c.data(a[4], kBf16, {h.num_pages, h.num_kv_heads, 128, 16});
    const int32_t* pt = c.data<int32_t>(a[5], kI32, {h.num_groups, h.max_prefix_pages});
    const int32_t* qs = c.data<int32_t>(a[6], kI32, {(int64_t)h.num_groups + 1});
    const int32_t* qp = c.data<int32_t>(a[7], kI32, {h.num_groups});
    const float scale = c.number(a[8]);
    void* out = c.data(a[9], out_type(h.out_dtype), {h.num_tokens, h.num_q_heads, 128});
    void* stream = c.stream();
    return finish(c, [&] { return f_prefill_attn(&h, ws, bytes, q, k, v, pt, qs, qp, scale, out, stream); });
  });
}

// shape, k_new, v_new, k_pages, v_pages, prefix_block_table, q_start, q_pos0, flags
PyObject* kv_write_prompt(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    if (n != 9 || !f_kv_write_prompt) Py_RETURN_NONE;
    Struct<marl_prefill_shape> s(a[0], g_prefill_shape);
    if (!s.ok || a[1] == Py_None || a[8] != Py_None) return not_here();
    const marl_prefill_shape& h = *s.get();
    Call c;
    const void* kn = c.data(a[1], kBf16, {h.num_tokens, h.num_kv_heads, 128});   // (first: the call's device)
    const void* vn = c.data(a[2], kBf16, {h.num_tokens, h.num_kv_heads, 128});
    void* k = c.data(a[3], kBf16, {h.num_pages, h.num_kv_heads, 16, 128});
    void* v = c.data(a[4], kBf16, {h.num_pages, h.num_kv_heads, 128, 16});
    const int32_t* pt = c.data<int32_t>(a[5], kI32, {h.num_groups, h.max_prefix_pages});
    const int32_t* qs = c.data<int32_t>(a[6], kI32, {(int64_t)h.num_groups + 1});
    const int32_t* qp = c.data<int32_t>(a[7], kI32, {h.num_groups});
    void* stream = c.stream();
    return finish(c, [&] { return f_kv_write_prompt(&h, kn, vn, k, v, pt, qs, qp, nullptr, stream); });
  });
}

constexpr auto kFp8 = at::kFloat8_e4m3fn;
constexpr auto kI8 = at::kChar;

// shape, workspace, q, k_pages, v_pages, exponents, prefix_block_table, suffix_block_table, prefix_lens, suffix_lens, group_of_seq, scale, out
PyObject* decode_attn_fp8(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    if (n != 13 || !f_decode_attn_fp8) Py_RETURN_NONE;
    Struct<marl_attn_shape> s(a[0], g_attn_shape);
    if (!s.ok) return not_here();
    const marl_attn_shape& h = *s.get();
    for (int k = 1; k < 13; ++k)
      if (a[k] == Py_None) return not_here();
    if (h.max_prefix_pages <= 0 || h.max_suffix_pages <= 0) return not_here();   // (tables whose extents are not looked at)
    Call c;
    void* out = c.data(a[12], out_type(h.out_dtype), {h.num_seqs, h.num_q_heads, 128});   // (first: the call's device)
    size_t bytes;
    void* ws = c.bytes(a[1], bytes);
    const void* q = c.data(a[2], kBf16, {h.num_seqs, h.num_q_heads, 128});
    const void* k = c.data(a[3], kFp8, {h.num_pages, h.num_kv_heads, 16, 128});
    const void* v = c.data(a[4], kFp8, {h.num_pages, h.num_kv_heads, 128, 16});
    const int8_t* ex = c.data<int8_t>(a[5], kI8, {h.num_pages, h.num_kv_heads, 2, 16});
    const int32_t* pt = c.data<int32_t>(a[6], kI32, {h.num_groups, h.max_prefix_pages});
    const int32_t* st = c.data<int32_t>(a[7], kI32, {h.num_seqs, h.max_suffix_pages});
    const int32_t* pl = c.data<int32_t>(a[8], kI32, {h.num_groups});
    const int32_t* sl = c.data<int32_t>(a[9], kI32, {h.num_seqs});
    const int32_t* gs = c.data<int32_t>(a[10], kI32, {h.num_seqs});
    const float scale = c.number(a[11]);
    void* stream = c.stream();
    return finish(c, [&] { return f_decode_attn_fp8(&h, ws, bytes, q, k, v, ex, pt, st, pl, sl, gs, scale, out, stream); });
  });
}

// shape, k_new, v_new, k_pages, v_pages, exponents, suffix_block_table, suffix_lens, flags
PyObject* kv_append_fp8(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    if (n != 9 || !f_kv_append_fp8) Py_RETURN_NONE;
    Struct<marl_attn_shape> s(a[0], g_attn_shape);
    if (!s.ok || a[3] == Py_None || a[8] != Py_None) return not_here();
    const marl_attn_shape& h = *s.get();
    Call c;
    void* k = c.data(a[3], kFp8, {h.num_pages, h.num_kv_heads, 16, 128});   // (first: the call's device)
    void* v = c.data(a[4], kFp8, {h.num_pages, h.num_kv_heads, 128, 16});
    int8_t* ex = c.data<int8_t>(a[5], kI8, {h.num_pages, h.num_kv_heads, 2, 16});
    const void* kn = c.data(a[1], kBf16, {h.num_seqs, h.num_kv_heads, 128});
    const void* vn = c.data(a[2], kBf16, {h.num_seqs, h.num_kv_heads, 128});
    const int32_t* st = c.data<int32_t>(a[6], kI32, {h.num_seqs, h.max_suffix_pages});
    int32_t* sl = c.data<int32_t>(a[7], kI32, {h.num_seqs});
    void* stream = c.stream();
    return finish(c, [&] { return f_kv_append_fp8(&h, kn, vn, k, v, ex, st, sl, nullptr, stream); });
  });
}

// shape, k_new, v_new, k_pages, v_pages, exponents, prefix_block_table, q_start, q_pos0, flags
PyObject* kv_write_prompt_fp8(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    if (n != 10 || !f_kv_write_prompt_fp8) Py_RETURN_NONE;
    Struct<marl_prefill_shape> s(a[0], g_prefill_shape);
    if (!s.ok || a[1] == Py_None || a[9] != Py_None) return not_here();
    const marl_prefill_shape& h = *s.get();
    Call c;
    const void* kn = c.data(a[1], kBf16, {h.num_tokens, h.num_kv_heads, 128});   // (first: the call's device)
    const void* vn = c.data(a[2], kBf16, {h.num_tokens, h.num_kv_heads, 128});
    void* k = c.data(a[3], kFp8, {h.num_pages, h.num_kv_heads, 16, 128});
    void* v = c.data(a[4], kFp8, {h.num_pages, h.num_kv_heads, 128, 16});
    int8_t* ex = c.data<int8_t>(a[5], kI8, {h.num_pages, h.num_kv_heads, 2, 16});
    const int32_t* pt = c.data<int32_t>(a[6], kI32, {h.num_groups, h.max_prefix_pages});
    const int32_t* qs = c.data<int32_t>(a[7], kI32, {(int64_t)h.num_groups + 1});
    const int32_t* qp = c.data<int32_t>(a[8], kI32, {h.num_groups});
    void* stream = c.stream();
    return finish(c, [&] { return f_kv_write_prompt_fp8(&h, kn, vn, k, v, ex, pt, qs, qp, nullptr, stream); });
  });
}

// k_codes, v_codes, exponents, src, dst, k_pages, v_pages, flags
PyObject* kv_read_pages_fp8(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    if (n != 8 || !f_kv_read_pages_fp8 || a[7] != Py_None) return not_here();
    Call c;
    const at::Tensor* kc = c.tensor(a[0], kFp8, {-1, -1, 16, 128});
    const at::Tensor* kp = c.tensor(a[5], kBf16, {-1, -1, 16, 128});
    const at::Tensor* src = c.tensor(a[3], kI32, {-1});
    if (!c.ok || a[1] == Py_None || a[2] == Py_None || a[4] == Py_None || a[6] == Py_None) return not_here();
    const int64_t pages = kc->size(0), heads = kc->size(1), out_pages = kp->size(0), count = src->numel();
    if (kp->size(1) != heads || pages > INT32_MAX || heads > INT32_MAX || out_pages > INT32_MAX || count > INT32_MAX) return not_here();
    const void* vc = c.data(a[1], kFp8, {pages, heads, 128, 16});
    const int8_t* ex = c.data<int8_t>(a[2], kI8, {pages, heads, 2, 16});
    const int32_t* dst = c.data<int32_t>(a[4], kI32, {count});
    void* vp = c.data(a[6], kBf16, {out_pages, heads, 128, 16});
    void* stream = c.stream();
    return finish(c, [&] {
      return f_kv_read_pages_fp8((int32_t)heads, (int32_t)pages, kc->data_ptr(), vc, ex, (int32_t)out_pages, kp->data_ptr(), vp,
                                 static_cast<const int32_t*>(src->data_ptr()), dst, (int32_t)count, nullptr, stream);
    });
  });
}

// The shape of a norm and rotation call and its common operands: q, k, q_weight, k_weight, cos_sin, positions, eps at a[0 .. 6].
struct NormRope {
  marl_norm_rope_shape h{};
  at::ScalarType type = kBf16;
  int64_t T = 0, Hq = 0, Hkv = 0, D = 0;
  const void *q = nullptr, *k = nullptr, *qw = nullptr, *kw = nullptr;
  const float* cos_sin = nullptr;
  const int32_t* positions = nullptr;

  bool take(Call& c, PyObject* const* a, PyObject* adjacent) {
    if (!THPVariable_CheckExact(a[0]) || !THPVariable_CheckExact(a[1]) || !PyBool_Check(adjacent)) return false;
    const at::Tensor &tq = THPVariable_Unpack(a[0]), &tk = THPVariable_Unpack(a[1]);
    type = tq.scalar_type();
    if (tq.dim() != 3 || tk.dim() != 3 || (type != kBf16 && type != at::kFloat)) return false;
    T = tq.size(0);
    Hq = tq.size(1);
    Hkv = tk.size(1);
    D = tq.size(2);
    if (T > INT32_MAX || Hq > INT32_MAX || Hkv > INT32_MAX || D > INT32_MAX) return false;
    q = c.rows(a[0], type, T, Hq, D, h.q_stride);
    k = c.rows(a[1], type, T, Hkv, D, h.k_stride);
    qw = c.data(a[2], type, {D});
    kw = c.data(a[3], type, {D});
    if (a[4] != Py_None) {
      const at::Tensor* cs = c.tensor(a[4], at::kFloat, {-1, -1});
      if (!cs || cs->size(0) > INT32_MAX || cs->size(1) > D) return false;
      h.rotary_dim = (int32_t)cs->size(1);
      if (h.rotary_dim > 0) {
        if (a[5] == Py_None) return false;
        h.max_positions = (int32_t)cs->size(0);
        cos_sin = static_cast<const float*>(cs->data_ptr());
        positions = c.data<int32_t>(a[5], kI32, {T});
      }
    }
    h.num_tokens = (int32_t)T;
    h.num_q_heads = (int32_t)Hq;
    h.num_kv_heads = (int32_t)Hkv;
    h.head_dim = (int32_t)D;
    h.dtype = type == kBf16 ? MARL_OUT_BF16 : MARL_OUT_F32;
    h.adjacent_pairs = adjacent == Py_True;
    h.eps = c.number(a[6]);
    return c.ok;
  }
};

// q, k, q_weight, k_weight, cos_sin, positions, eps, q_out, k_out, adjacent_pairs, flags
PyObject* qk_norm_rope(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    if (n != 11 || !f_qk_norm_rope || a[10] != Py_None) return not_here();
    Call c;
    NormRope m;
    if (!m.take(c, a, a[9])) return not_here();
    void* qo = c.rows(a[7], m.type, m.T, m.Hq, m.D, m.h.q_out_stride);
    void* ko = c.rows(a[8], m.type, m.T, m.Hkv, m.D, m.h.k_out_stride);
    void* stream = c.stream();
    return finish(c, [&] { return f_qk_norm_rope(&m.h, m.q, m.k, m.qw, m.kw, m.cos_sin, m.positions, qo, ko, nullptr, stream); });
  });
}

// dq_out, dk_out, q, k, q_weight, k_weight, cos_sin, positions, eps, dq, dk, dq_weight, dk_weight, workspace, adjacent_pairs, flags
PyObject* qk_norm_rope_backward(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    if (n != 16 || !f_qk_norm_rope_backward || a[13] == Py_None || a[15] != Py_None) return not_here();
    Call c;
    NormRope m;
    if (!m.take(c, a + 2, a[14])) return not_here();
    const void* dqo = c.rows(a[0], m.type, m.T, m.Hq, m.D, m.h.q_out_stride);
    const void* dko = c.rows(a[1], m.type, m.T, m.Hkv, m.D, m.h.k_out_stride);
    void* dq = c.rows(a[9], m.type, m.T, m.Hq, m.D, m.h.dq_stride);
    void* dk = c.rows(a[10], m.type, m.T, m.Hkv, m.D, m.h.dk_stride);
    float* dqw = c.data<float>(a[11], at::kFloat, {m.D});
    float* dkw = c.data<float>(a[12], at::kFloat, {m.D});
    size_t bytes;
    void* ws = c.bytes(a[13], bytes);
    void* stream = c.stream();
    return finish(c, [&] {
      return f_qk_norm_rope_backward(&m.h, ws, bytes, dqo, dko, m.q, m.k, m.qw, m.kw, m.cos_sin, m.positions, dq, dk, dqw, dkw, nullptr, stream);
    });
  });
}

// bind(stream_of, types of the two shapes, addresses of the library's functions in the order of the declarations above; the
// last ones, from the scatter's on, may be left out and then stay what they are)
PyObject* bind(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (n < 9 || n > 16 || !PyType_Check(a[1]) || !PyType_Check(a[2])) {
    PyErr_SetString(PyExc_TypeError, "bind: a function, two types, six to thirteen addresses");
    return nullptr;
  }
  void* f[13] = {};
  for (int k = 0; k + 3 < n; ++k) {
    f[k] = PyLong_AsVoidPtr(a[k + 3]);
    if (PyErr_Occurred()) return nullptr;
  }
  PyObject** const kept[3] = {&g_stream_of, &g_attn_shape, &g_prefill_shape};
  for (int k = 0; k < 3; ++k) {
    Py_INCREF(a[k]);
    Py_XSETREF(*kept[k], a[k]);
  }
  f_decode_attn = reinterpret_cast<decltype(f_decode_attn)>(f[0]);
  f_token_logprobs = reinterpret_cast<decltype(f_token_logprobs)>(f[1]);
  f_kv_append = reinterpret_cast<decltype(f_kv_append)>(f[2]);
  f_sample_tokens = reinterpret_cast<decltype(f_sample_tokens)>(f[3]);
  f_sample_tokens_top_p = reinterpret_cast<decltype(f_sample_tokens_top_p)>(f[4]);
  f_prefill_attn = reinterpret_cast<decltype(f_prefill_attn)>(f[5]);
  auto last = [&](int k, auto& function) {
    if (k + 3 < n) function = reinterpret_cast<std::remove_reference_t<decltype(function)>>(f[k]);
  };
  last(6, f_kv_write_prompt);
  last(7, f_decode_attn_fp8);
  last(8, f_kv_append_fp8);
  last(9, f_kv_write_prompt_fp8);
  last(10, f_kv_read_pages_fp8);
  last(11, f_qk_norm_rope);
  last(12, f_qk_norm_rope_backward);
  Py_RETURN_NONE;
}

#define MARL_FAST(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(name)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {MARL_FAST(bind), MARL_FAST(decode_attn), MARL_FAST(token_logprobs), MARL_FAST(sample_tokens),
                         MARL_FAST(kv_append), MARL_FAST(prefill_attn), MARL_FAST(kv_write_prompt), MARL_FAST(decode_attn_fp8),
                         MARL_FAST(kv_append_fp8), MARL_FAST(kv_write_prompt_fp8), MARL_FAST(kv_read_pages_fp8), MARL_FAST(qk_norm_rope),
                         MARL_FAST(qk_norm_rope_backward), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "fast_calls", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit_fast_calls(void) {
  PyObject* m = PyModule_Create(&module);
  if (m && PyModule_AddStringConstant(m, "torch_version", TORCH_VERSION) != 0) Py_CLEAR(m);   // (tensors are read as this torch lays them out)
  if (m && PyModule_AddStringConstant(m, "sources", MARL_FAST_CALLS_SOURCES) != 0) Py_CLEAR(m);
  return m;
}
