// The Python side of include/wait_kv.h in C++: argument checks and marshalling.
// A serving step calls these a few times a layer.  With the checks in Python
// and ctypes, they took longer than the kernels of small calls: the rotation of
// one token's 32 heads of 128 took 6.3 us a call there, 4.4 here (1.7 on the
// GPU), rows of 128 tokens written and read back 16.0 there, 9.5 here (6.6 on
// the GPU), 630 tokens read 9.4 there, 5.6 here (4.6).  kv.py has the
// documentation and gives the library's entry points as addresses (bind), so
// that this module works with whichever build of it is loaded.
#include <Python.h>

#include <ATen/ATen.h>
#include <c10/core/GradMode.h>
#include <c10/util/Float8_e4m3fn.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/autograd/python_variable.h>

#include <algorithm>
#include <cmath>
#include <cstdarg>
#include <cstdio>
#include <cstring>
#include <exception>

#include "wait_kv.h"

namespace {

decltype(&wait_kv_rotary) f_rotary;
decltype(&wait_kv_append) f_append;
decltype(&wait_kv_read) f_read;
decltype(&wait_kv_attention_workspace_bytes) f_workspace;
decltype(&wait_kv_attention) f_attention;
PyObject *g_check, *g_stream, *g_device, *g_on;  // of binding.py and torch

// Raised in Python as ValueError; Python's own errors as they are.
struct Refused : std::exception {};

[[noreturn]] void refuse(const char *format, ...) {
  char text[256];
  va_list args;
  va_start(args, format);
  vsnprintf(text, sizeof text, format, args);
  va_end(args);
  PyErr_SetString(PyExc_ValueError, text);
  throw Refused();
}
void need(bool ok, const char *text) {
  if (!ok) refuse("%s", text);
}

// The body of a function: C++ exceptions become Python's.
template <class F>
PyObject *guarded(F &&body) noexcept {
  try {
    need(g_on, "not bound to the library");
    return body();
  } catch (const Refused &) {
    return nullptr;
  } catch (const std::exception &e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
    return nullptr;
  } catch (...) {
    PyErr_SetString(PyExc_RuntimeError, "unexpected C++ exception");
    return nullptr;
  }
}

const at::Tensor &tensor(PyObject *o, const char *name) {
  if (!THPVariable_Check(o)) {
    PyErr_Format(PyExc_TypeError, "%s must be a tensor", name);
    throw Refused();
  }
  return THPVariable_Unpack(o);
}
const at::Tensor *tensor_or_none(PyObject *o, const char *name) {
  return o == Py_None ? nullptr : &tensor(o, name);
}

// Results carry no gradients, so inputs that ask for them are refused rather than
// cut off.
void no_gradient(const at::Tensor &t, const char *name) {
  if (t.requires_grad() && c10::GradMode::is_enabled())
    refuse("%s requires a gradient, which these operators do not carry (detach it, or call under "
           "torch.no_grad())", name);
}

// Memory that a call has written counts a version, as PyTorch's own operators in
// place do, so that autograd does not use what it kept of the old contents.
void written(const at::Tensor &t) {
  if (!t.is_inference()) t.unsafeGetTensorImpl()->bump_version();
}

int kv_type(at::ScalarType t) {
  switch (t) {
    case at::kBFloat16: return WS_KV_BF16;
    case at::kHalf: return WS_KV_FP16;
    case at::kFloat: return WS_KV_FP32;
    case at::kFloat8_e4m3fn: return WS_KV_FP8;
    case at::kChar: return WS_KV_INT8;
    default: return -1;
  }
}
bool wide(int t) { return t >= WS_KV_BF16 && t <= WS_KV_FP32; }

int index_of(const at::Tensor &t) { return t.is_cuda() ? (int)t.get_device() : -1; }

// [tokens, heads, dim] on GPU `index`.
ws_kv_rows rows(const at::Tensor &t, const char *name, int index) {
  no_gradient(t, name);
  if (t.dim() != 3) refuse("%s must be [tokens, heads, dim]", name);
  const int type = kv_type(t.scalar_type());
  if (!wide(type)) refuse("%s must be bf16, fp16 or fp32", name);
  if (t.stride(2) != 1 && t.size(2) != 1) refuse("%s: a vector's elements must be contiguous", name);
  if (index_of(t) != index) refuse("%s must be on the same device", name);
  return {t.data_ptr(), t.stride(0), t.stride(1), type};
}

// Refuses an output whose rows share memory.
void apart(const at::Tensor &t, const char *name) {
  int64_t size[2] = {t.size(0), t.size(1)}, step[2] = {std::abs(t.stride(0)), std::abs(t.stride(1))};
  if (step[0] > step[1]) {
    std::swap(size[0], size[1]);
    std::swap(step[0], step[1]);
  }
  int64_t least = t.size(2);
  for (int i = 0; i < 2; ++i) {
    if (size[i] <= 1) continue;
    if (step[i] < least) refuse("%s: rows must not overlap", name);
    least = step[i] * (size[i] - 1) + least;
  }
}

ws_kv_turn turn(const at::Tensor *positions, const at::Tensor *table, int64_t n, int64_t dim,
                bool interleaved, int index) {
  need(positions && table, "a rotation needs positions and a table");
  no_gradient(*table, "table");
  need(table->dim() == 2 && table->scalar_type() == at::kFloat && table->is_contiguous(),
       "table must be [positions, part], fp32, contiguous");
  need(positions->dim() == 1 && positions->size(0) == n && positions->is_contiguous() &&
           (positions->scalar_type() == at::kLong || positions->scalar_type() == at::kInt),
       "positions must be one int64 or int32 a token, contiguous");
  const int64_t part = table->size(1);
  need(part % 2 == 0 && part >= 2 && part <= dim,
       "the table's part must be even, at least 2 and at most the head dimension");
  need(index_of(*positions) == index && index_of(*table) == index,
       "positions and table must be on the vectors' device");
  need(table->size(0) <= INT32_MAX, "the table has too many positions");
  return {table->data_ptr<float>(), positions->data_ptr(), positions->scalar_type() == at::kInt,
          (int32_t)table->size(0), (int32_t)part, interleaved};
}

ws_kv_cache cache_of(PyObject *o) {
  need(PyBytes_Check(o) && PyBytes_GET_SIZE(o) == (Py_ssize_t)sizeof(ws_kv_cache), "not a cache");
  ws_kv_cache c;
  memcpy(&c, PyBytes_AS_STRING(o), sizeof c);
  return c;
}

long whole(PyObject *o) {
  const long x = PyLong_AsLong(o);
  if (x == -1 && PyErr_Occurred()) throw Refused();
  return x;
}
bool truth(PyObject *o) {
  const int x = PyObject_IsTrue(o);
  if (x < 0) throw Refused();
  return x;
}

// The library's errors, as binding.py raises them.
void check(int rc) {
  if (!rc) return;
  PyObject *code = PyLong_FromLong(rc);
  PyObject *none = code ? PyObject_CallOneArg(g_check, code) : nullptr;
  Py_XDECREF(code);
  Py_XDECREF(none);
  if (!PyErr_Occurred()) PyErr_SetString(PyExc_RuntimeError, "wait_kv failed");
  throw Refused();
}

// call(stream) on GPU `index`, its current stream, other Python threads running.
template <class F>
void run(int index, F &&call) {
  need(index >= 0, "the operators run on the GPU");
  struct Ref {
    PyObject *o;
    ~Ref() { Py_XDECREF(o); }
  };
  Ref which{PyLong_FromLong(index)}, now{PyObject_CallNoArgs(g_device)};
  if (!which.o || !now.o) throw Refused();
  Ref guard{nullptr};
  if (PyLong_AsLong(now.o) != index) {  // with torch.cuda.device(index):
    guard.o = PyObject_CallOneArg(g_on, which.o);
    Ref in{guard.o ? PyObject_CallMethod(guard.o, "__enter__", nullptr) : nullptr};
    if (!in.o) throw Refused();
  }
  int rc = 0;
  Ref stream{PyObject_CallOneArg(g_stream, which.o)};
  void *s = stream.o ? PyLong_AsVoidPtr(stream.o) : nullptr;
  if (!PyErr_Occurred()) {
    Py_BEGIN_ALLOW_THREADS
    rc = call(s);
    Py_END_ALLOW_THREADS
  }
  if (guard.o) {
    PyObject *type, *value, *trace;
    PyErr_Fetch(&type, &value, &trace);
    Ref out{PyObject_CallMethod(guard.o, "__exit__", "OOO", Py_None, Py_None, Py_None)};
    if (type) PyErr_Restore(type, value, trace);
  }
  if (PyErr_Occurred()) throw Refused();
  check(rc);
}

#define ARGS(n) \
  if (nargs != n) { PyErr_SetString(PyExc_TypeError, "wrong number of arguments"); return nullptr; }

// rotary(x, positions, table, interleaved, inverse, out or None)
PyObject *rotary(PyObject *, PyObject *const *v, Py_ssize_t nargs) {
  ARGS(6)
  return guarded([&]() -> PyObject * {
    const at::Tensor &x = tensor(v[0], "x");
    const int index = index_of(x);
    const ws_kv_rows xr = rows(x, "x", index);
    const int64_t n = x.size(0), heads = x.size(1), dim = x.size(2);
    need(heads <= INT32_MAX && dim <= INT32_MAX, "x is too large");
    const ws_kv_turn t = turn(tensor_or_none(v[1], "positions"), tensor_or_none(v[2], "table"), n,
                              dim, truth(v[3]), index);
    at::Tensor out;
    if (v[5] == Py_None) {
      need(index >= 0, "the operators run on the GPU");
      out = at::empty_like(x);
    } else {
      out = tensor(v[5], "out");
      need(out.sizes() == x.sizes() && out.scalar_type() == x.scalar_type(),
           "out must have x's shape and type");
      apart(out, "out");
    }
    const ws_kv_rows o = rows(out, "out", index);
    const bool inverse = truth(v[4]);
    if (n && heads)
      run(index, [&](void *s) {
        return f_rotary(&xr, &o, n, (int32_t)heads, (int32_t)dim, &t, inverse, s);
      });
    if (v[5] != Py_None) {
      written(out);
      Py_INCREF(v[5]);
      return v[5];
    }
    return THPVariable_Wrap(std::move(out));
  });
}

// cache(k, v, k_scale or None, v_scale or None): the struct, as bytes
PyObject *cache(PyObject *, PyObject *const *v, Py_ssize_t nargs) {
  ARGS(4)
  return guarded([&]() -> PyObject * {
    const at::Tensor &k = tensor(v[0], "k"), &w = tensor(v[1], "v");
    const int type = kv_type(k.scalar_type());
    need(k.dim() == 4 && k.sizes() == w.sizes() && k.scalar_type() == w.scalar_type() &&
             type >= 0 && type != WS_KV_FP32 && k.is_contiguous() && w.is_contiguous() &&
             k.device() == w.device(),
         "k and v must both be [pages, kv_heads, page_size, dim] of bf16, fp16, float8_e4m3fn or "
         "int8, contiguous, on one device");
    for (int i = 0; i < 4; ++i) need(k.size(i) <= INT32_MAX, "the cache is too large");
    const at::Tensor *scale[2] = {tensor_or_none(v[2], "k_scale"), tensor_or_none(v[3], "v_scale")};
    // a cache outlives the mode that it is made in
    for (auto *t : {&k, &w, scale[0], scale[1]})
      need(!t || !t->requires_grad(), "a cache's tensors must not require a gradient");
    float *p[2] = {nullptr, nullptr};
    if (type == WS_KV_FP8 || type == WS_KV_INT8) {
      for (int i = 0; i < 2; ++i) {
        need(scale[i], "an 8-bit cache needs scales");
        const at::Tensor &t = *scale[i];
        need(t.dim() == 3 && t.sizes() == k.sizes().slice(0, 3) && t.scalar_type() == at::kFloat &&
                 t.is_contiguous() && t.device() == k.device(),
             "scales must be [pages, kv_heads, page_size], fp32, contiguous, on the cache's device");
        p[i] = t.data_ptr<float>();
      }
    } else {
      need(!scale[0] && !scale[1], "a 16-bit cache has no scales");
    }
    ws_kv_cache c{};
    c.k = k.data_ptr();
    c.v = w.data_ptr();
    c.k_scale = p[0];
    c.v_scale = p[1];
    c.pages = (int32_t)k.size(0);
    c.kv_heads = (int32_t)k.size(1);
    c.page_size = (int32_t)k.size(2);
    c.dim = (int32_t)k.size(3);
    c.type = type;
    return PyBytes_FromStringAndSize((const char *)&c, sizeof c);
  });
}

int64_t slots_of(const at::Tensor &t, int index) {
  need(t.dim() == 1 && t.scalar_type() == at::kLong && t.is_contiguous() && index_of(t) == index,
       "slots must be one int64 a token, contiguous, on the cache's device");
  return t.size(0);
}

// append(cache bytes, GPU, k, v, slots, positions or None, table or None, interleaved,
//        the cache's tensors)
PyObject *append(PyObject *, PyObject *const *v, Py_ssize_t nargs) {
  ARGS(9)
  return guarded([&]() -> PyObject * {
    const ws_kv_cache c = cache_of(v[0]);
    need(PyTuple_Check(v[8]), "not a cache");
    const int index = (int)whole(v[1]);
    const at::Tensor &k = tensor(v[2], "k"), &w = tensor(v[3], "v"), &slots = tensor(v[4], "slots");
    const ws_kv_rows kr = rows(k, "k", index), wr = rows(w, "v", index);
    const int64_t n = slots_of(slots, index);
    need(k.size(0) == n && k.size(1) == c.kv_heads && k.size(2) == c.dim && k.sizes() == w.sizes() &&
             kr.type == wr.type,
         "k and v must be [slots, kv_heads, dim] of one type");
    ws_kv_turn t;
    const bool turned = v[5] != Py_None || v[6] != Py_None;
    if (turned)
      t = turn(tensor_or_none(v[5], "positions"), tensor_or_none(v[6], "table"), n, c.dim,
               truth(v[7]), index);
    run(index, [&](void *s) {
      return f_append(&c, &kr, &wr, slots.data_ptr<int64_t>(), n, turned ? &t : nullptr, s);
    });
    for (Py_ssize_t i = 0; i < PyTuple_GET_SIZE(v[8]); ++i)
      if (auto *t = tensor_or_none(PyTuple_GET_ITEM(v[8], i), "the cache's")) written(*t);
    Py_RETURN_NONE;
  });
}

// read(cache bytes, GPU, slots, dtype, out k or None, out v or None): (k, v)
PyObject *read(PyObject *, PyObject *const *v, Py_ssize_t nargs) {
  ARGS(6)
  return guarded([&]() -> PyObject * {
    const ws_kv_cache c = cache_of(v[0]);
    const int index = (int)whole(v[1]);
    const at::Tensor &slots = tensor(v[2], "slots");
    const int64_t n = slots_of(slots, index);
    const int64_t shape[3] = {n, c.kv_heads, c.dim};
    at::Tensor out[2];
    const bool made = v[4] == Py_None;
    if (made) {
      need(THPDtype_Check(v[3]), "dtype must be bf16, fp16 or fp32");
      const at::ScalarType type = reinterpret_cast<THPDtype *>(v[3])->scalar_type;
      need(wide(kv_type(type)), "dtype must be bf16, fp16 or fp32");
      need(index >= 0, "the operators run on the GPU");
      for (auto &t : out) t = at::empty(shape, slots.options().dtype(type));
    } else {
      for (int i = 0; i < 2; ++i) {
        out[i] = tensor(v[4 + i], "out");
        need(out[i].sizes() == at::IntArrayRef(shape, 3) &&
                 out[i].scalar_type() == out[0].scalar_type(),
             "out must be two [slots, kv_heads, dim] of one type");
        apart(out[i], "out");
      }
    }
    const ws_kv_rows k = rows(out[0], "k", index), w = rows(out[1], "v", index);
    run(index, [&](void *s) { return f_read(&c, slots.data_ptr<int64_t>(), n, &k, &w, s); });
    PyObject *a, *b;
    if (made) {
      a = THPVariable_Wrap(std::move(out[0]));
      b = THPVariable_Wrap(std::move(out[1]));
    } else {
      for (const auto &t : out) written(t);
      Py_INCREF(a = v[4]);
      Py_INCREF(b = v[5]);
    }
    PyObject *pair = a && b ? PyTuple_Pack(2, a, b) : nullptr;
    Py_XDECREF(a);
    Py_XDECREF(b);
    return pair;
  });
}

// The batch and its workspace's bytes.
ws_kv_batch batch_of(const ws_kv_cache &c, int index, const at::Tensor &q, PyObject *const *v,
                     PyObject *max_q, PyObject *max_kv, PyObject *scale, bool causal,
                     PyObject *window, size_t *bytes) {
  const at::Tensor &pages = tensor(v[0], "pages"), &starts = tensor(v[1], "starts"),
                   &lens = tensor(v[2], "kv_lens");
  need(q.dim() == 3, "q must be [tokens, heads, dim]");
  need(pages.dim() == 2 && pages.scalar_type() == at::kInt &&
           (pages.size(1) <= 1 || pages.stride(1) == 1) && index_of(pages) == index,
       "pages must be [requests, pages], int32, rows contiguous, on the cache's device");
  const int64_t n_seq = pages.size(0), cols = pages.size(1), tokens = q.size(0), heads = q.size(1);
  for (auto *t : {&starts, &lens})
    need(t->dim() == 1 && t->size(0) == n_seq + (t == &starts) && t->scalar_type() == at::kInt &&
             t->is_contiguous() && index_of(*t) == index,
         "starts (one more than the requests) and kv_lens (one each) must be int32, contiguous, on "
         "the cache's device");
  need(q.size(2) == c.dim, "q and the cache must have one head dimension");
  need(heads >= 1 && c.kv_heads >= 1 && heads % c.kv_heads == 0, "heads must be a multiple of the cache's");
  need(n_seq < INT32_MAX && cols <= INT32_MAX && tokens <= INT32_MAX && heads <= INT32_MAX,
       "the batch is too large");
  const int64_t capacity = std::min<int64_t>(cols * c.page_size, INT32_MAX);
  auto bound = [](PyObject *o, int64_t most) {
    return o == Py_None ? most : std::min<int64_t>(whole(o), most);
  };
  ws_kv_batch b{};
  b.table = pages.data_ptr<int32_t>();
  b.table_stride = n_seq > 1 ? pages.stride(0) : cols;
  b.table_cols = (int32_t)cols;
  b.starts = starts.data_ptr<int32_t>();
  b.kv_lens = lens.data_ptr<int32_t>();
  b.n_seq = (int32_t)n_seq;
  b.n_tokens = (int32_t)tokens;
  b.heads = (int32_t)heads;
  if (scale == Py_None) {
    b.scale = (float)(1.0 / std::sqrt((double)c.dim));
  } else {
    b.scale = (float)PyFloat_AsDouble(scale);
    if (PyErr_Occurred()) throw Refused();
  }
  b.causal = causal;
  b.window = (int32_t)std::max<int64_t>(std::min<int64_t>(whole(window), INT32_MAX), -1);
  b.max_q_len = (int32_t)std::max<int64_t>(bound(max_q, tokens), -1);
  b.max_kv_len = (int32_t)std::max<int64_t>(bound(max_kv, capacity), -1);
  check(f_workspace(&c, &b, bytes));
  return b;
}

// attention_workspace_bytes(cache bytes, GPU, q, pages, starts, kv_lens, max_q, max_kv, window)
PyObject *attention_workspace_bytes(PyObject *, PyObject *const *v, Py_ssize_t nargs) {
  ARGS(9)
  return guarded([&]() -> PyObject * {
    const ws_kv_cache c = cache_of(v[0]);
    const int index = (int)whole(v[1]);
    size_t bytes = 0;
    batch_of(c, index, tensor(v[2], "q"), v + 3, v[6], v[7], Py_None, true, v[8], &bytes);
    return PyLong_FromSize_t(bytes);
  });
}

// attention(cache bytes, GPU, q, pages, starts, kv_lens, max_q, max_kv, scale, causal, window,
//           lse, out or None, workspace or None): out, or (out, lse)
PyObject *attention(PyObject *, PyObject *const *v, Py_ssize_t nargs) {
  ARGS(14)
  return guarded([&]() -> PyObject * {
    const ws_kv_cache c = cache_of(v[0]);
    const int index = (int)whole(v[1]);
    const at::Tensor &q = tensor(v[2], "q");
    const ws_kv_rows qr = rows(q, "q", index);
    need(qr.type != WS_KV_FP32, "q must be bf16 or fp16");
    need(c.type == WS_KV_FP8 || c.type == WS_KV_INT8 || c.type == qr.type,
         "q must have the type of a 16-bit cache");
    size_t bytes = 0;
    const ws_kv_batch b = batch_of(c, index, q, v + 3, v[6], v[7], v[8], truth(v[9]), v[10], &bytes);
    const bool want_lse = truth(v[11]);
    at::Tensor out, lse, space;
    if (v[12] == Py_None) {
      need(index >= 0, "the operators run on the GPU");
      out = at::empty_like(q);
    } else {
      out = tensor(v[12], "out");
      need(out.sizes() == q.sizes() && out.scalar_type() == q.scalar_type(),
           "out must have q's shape and type");
      apart(out, "out");
    }
    const ws_kv_rows o = rows(out, "out", index);
    if (want_lse) lse = at::empty({q.size(0), q.size(1)}, q.options().dtype(at::kFloat));
    void *ptr = nullptr;
    size_t have = 0;
    if (v[13] != Py_None) {
      const at::Tensor &t = tensor(v[13], "workspace");
      need(t.is_contiguous() && index_of(t) == index,
           "workspace must be contiguous, on the cache's device");
      ptr = t.data_ptr();
      have = t.nbytes();
    } else if (bytes) {
      space = at::empty({(int64_t)bytes}, q.options().dtype(at::kByte));
      ptr = space.data_ptr();
      have = bytes;
    }
    run(index, [&](void *s) {
      return f_attention(&c, &b, &qr, &o, want_lse ? lse.data_ptr<float>() : nullptr, ptr, have, s);
    });
    if (v[13] != Py_None) written(tensor(v[13], "workspace"));
    PyObject *a;
    if (v[12] == Py_None) {
      a = THPVariable_Wrap(std::move(out));
    } else {
      written(out);
      Py_INCREF(a = v[12]);
    }
    if (!want_lse || !a) return a;
    PyObject *z = THPVariable_Wrap(std::move(lse));
    PyObject *pair = z ? PyTuple_Pack(2, a, z) : nullptr;
    Py_DECREF(a);
    Py_XDECREF(z);
    return pair;
  });
}

// bind(addresses of the five entry points, binding._check, stream of a GPU, current GPU,
//      torch.cuda.device)
PyObject *bind(PyObject *, PyObject *const *v, Py_ssize_t nargs) {
  ARGS(9)
  void *p[5];
  for (int i = 0; i < 5; ++i) {
    p[i] = PyLong_AsVoidPtr(v[i]);
    if (PyErr_Occurred()) return nullptr;
  }
  f_rotary = reinterpret_cast<decltype(f_rotary)>(p[0]);
  f_append = reinterpret_cast<decltype(f_append)>(p[1]);
  f_read = reinterpret_cast<decltype(f_read)>(p[2]);
  f_workspace = reinterpret_cast<decltype(f_workspace)>(p[3]);
  f_attention = reinterpret_cast<decltype(f_attention)>(p[4]);
  PyObject **kept[4] = {&g_check, &g_stream, &g_device, &g_on};
  for (int i = 0; i < 4; ++i) {
    Py_INCREF(v[5 + i]);
    Py_XSETREF(*kept[i], v[5 + i]);
  }
  Py_RETURN_NONE;
}

#define METHOD(name) {#name, (PyCFunction)(void (*)(void))name, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {METHOD(bind),      METHOD(rotary),    METHOD(cache),
                         METHOD(append),    METHOD(read),      METHOD(attention_workspace_bytes),
                         METHOD(attention), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_kv", "Argument checks of kv.py.", -1, methods,
                      nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__kv(void) { return PyModule_Create(&module); }
