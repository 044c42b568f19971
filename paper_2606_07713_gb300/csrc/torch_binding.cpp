// PyTorch tensors in, C ABI calls out: the binding of the operators around attention.
//
// A decoding step makes several of these calls with kernels of a few microseconds each, so the
// checks and the marshalling are done here, in about a microsecond a call, and not in Python.
// Nothing is computed here; every entry point calls the function of its name in
// include/moa_attn.h and raises its error.
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <ATen/cuda/EmptyTensor.h>
#include <c10/cuda/CUDACachingAllocator.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cmath>
#include <cstdarg>
#include <cstdio>
#include <exception>
#include <string>

#include "../../include/moa_attn.h"

namespace {

PyObject* g_error = nullptr;  // MoaError of the package

// A Python exception to raise: `type` with a message, or (type null) one that is already set.
struct Raise {
  PyObject* type;
  std::string text;
};

[[noreturn]] void fail(PyObject* type, const char* fmt, ...) {
  char buf[384];
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(buf, sizeof(buf), fmt, ap);
  va_end(ap);
  throw Raise{type, buf};
}

void check(int status) {
  if (status == MOA_OK) return;
  PyObject* e = g_error ? PyObject_CallFunction(g_error, "is", status, moa_last_error()) : nullptr;
  if (e != nullptr) {
    PyErr_SetObject(g_error, e);
    Py_DECREF(e);
  } else if (!PyErr_Occurred()) {
    PyErr_Format(PyExc_RuntimeError, "status %d: %s", status, moa_last_error());
  }
  throw Raise{nullptr, ""};
}

std::string text(at::IntArrayRef s) {
  std::string r = "(";
  for (size_t i = 0; i < s.size(); ++i) r += (i ? ", " : "") + std::to_string(s[i]);
  return r + ")";
}

const at::Tensor& tensor(const char* what, const char* name, PyObject* o) {
  if (!THPVariable_Check(o)) fail(PyExc_TypeError, "%s: %s must be a tensor", what, name);
  return THPVariable_Unpack(o);
}

// A [B, H, N, d] tensor with unit stride along d: appends its (b, h, n) strides.
void heads(const char* what, const char* name, const at::Tensor& t, const at::Tensor* like,
           const int64_t* shape, int64_t* strides) {
  if (!t.is_cuda()) fail(PyExc_ValueError, "%s needs CUDA tensors (%s)", what, name);
  if (t.dim() != 4 || (t.size(3) > 1 && t.stride(3) != 1))
    fail(PyExc_ValueError, "%s: %s must be [B, H, N, d] with unit stride along d", what, name);
  if (shape != nullptr && t.sizes() != at::IntArrayRef(shape, 4))
    fail(PyExc_ValueError, "%s: %s must be %s, got %s", what, name, text(at::IntArrayRef(shape, 4)).c_str(),
         text(t.sizes()).c_str());
  if (like != nullptr) {
    if (t.scalar_type() != like->scalar_type())
      fail(PyExc_TypeError, "%s: %s must be %s, got %s", what, name, c10::toString(like->scalar_type()),
           c10::toString(t.scalar_type()));
    if (t.device() != like->device()) fail(PyExc_ValueError, "%s: tensors on different devices", what);
  }
  for (int i = 0; i < 3; ++i) strides[i] = t.stride(i);
}

void flat(const char* what, const char* name, const at::Tensor& t, at::ScalarType type, at::IntArrayRef shape,
          at::Device device) {
  if (t.scalar_type() != type)
    fail(PyExc_TypeError, "%s: %s must be %s, got %s", what, name, c10::toString(type), c10::toString(t.scalar_type()));
  if (t.sizes() != shape || !t.is_contiguous())
    fail(PyExc_ValueError, "%s: %s must be a contiguous %s tensor, got %s", what, name, text(shape).c_str(),
         text(t.sizes()).c_str());
  if (t.device() != device)
    fail(PyExc_ValueError, "%s: %s is on %s, not on %s", what, name, t.device().str().c_str(), device.str().c_str());
}

int code(const char* what, const at::Tensor& t) {
  if (t.scalar_type() == at::kBFloat16) return MOA_BF16;
  if (t.scalar_type() == at::kFloat) return MOA_FP32;
  fail(PyExc_TypeError, "%s: unsupported dtype %s; use torch.bfloat16 or torch.float32", what,
       c10::toString(t.scalar_type()));
}

double number(const char* what, const char* name, PyObject* o) {
  const double x = PyFloat_AsDouble(o);
  if (x == -1.0 && PyErr_Occurred()) {
    PyErr_Clear();
    fail(PyExc_TypeError, "%s: %s must be a number", what, name);
  }
  return x;
}
int64_t integer(const char* what, const char* name, PyObject* o) {
  const long long x = PyLong_AsLongLong(o);
  if (x == -1 && PyErr_Occurred()) {
    PyErr_Clear();
    fail(PyExc_TypeError, "%s: %s must be an integer", what, name);
  }
  return x;
}
bool truth(PyObject* o) {
  const int r = PyObject_IsTrue(o);
  if (r < 0) throw Raise{nullptr, ""};
  return r != 0;
}

// The call's device and stream: None is torch's current stream of the device, else an object with
// .cuda_stream.  Memory allocated inside belongs to that stream, so that it is not handed out again
// before the call's work on it is done.
struct Place {
  c10::cuda::CUDAGuard device;
  c10::cuda::OptionalCUDAStreamGuard guard;
  c10::cuda::CUDAStream stream;
  Place(PyObject* o, at::Device dev) : device(dev), stream(c10::cuda::getCurrentCUDAStream(dev.index())) {
    if (o == Py_None) return;
    PyObject* s = PyObject_GetAttrString(o, "cuda_stream");
    if (s == nullptr) throw Raise{nullptr, ""};
    void* p = PyLong_AsVoidPtr(s);
    Py_DECREF(s);
    if (p == nullptr && PyErr_Occurred()) throw Raise{nullptr, ""};
    if (p == static_cast<void*>(stream.stream())) return;
    stream = p == nullptr ? c10::cuda::getDefaultCUDAStream(dev.index())
                          : c10::cuda::getStreamFromExternal(static_cast<cudaStream_t>(p), dev.index());
    guard.reset_stream(stream);
  }
  void* raw() const { return stream.stream(); }
};

at::Tensor make(at::IntArrayRef size, at::ScalarType type, at::Device dev) {
  return at::Tensor(at::detail::empty_cuda(size, type, dev, std::nullopt));
}

// The workspace: what the caller gives, or memory of the call's stream for the time of the call.
struct Scratch {
  void* p = nullptr;
  size_t bytes = 0;
  bool mine = false;
  Scratch(const char* what, PyObject* given, size_t need, const Place& place) {
    if (given != Py_None) {
      const at::Tensor& t = tensor(what, "workspace", given);
      if (t.device() != place.stream.device() || !t.is_contiguous())
        fail(PyExc_ValueError, "%s: workspace must be a contiguous tensor on %s", what, place.stream.device().str().c_str());
      p = t.data_ptr(), bytes = t.nbytes();
      return;
    }
    bytes = need < 16 ? 16 : need;
    p = c10::cuda::CUDACachingAllocator::raw_alloc_with_stream(bytes, place.stream);
    mine = true;
  }
  ~Scratch() {
    if (mine) c10::cuda::CUDACachingAllocator::raw_delete(p);
  }
  Scratch(const Scratch&) = delete;
  Scratch& operator=(const Scratch&) = delete;
};

// Two tensors of `out` (a pair), or new contiguous ones of these shapes like `like`.
void outputs(const char* what, PyObject* out, at::ScalarType type, at::Device dev, const int64_t* a, const int64_t* b,
             at::Tensor* t) {
  if (out == Py_None) {
    t[0] = make(at::IntArrayRef(a, 4), type, dev);
    t[1] = make(at::IntArrayRef(b, 4), type, dev);
    return;
  }
  PyObject* s = PySequence_Fast(out, "out must be a pair of tensors");
  if (s == nullptr) throw Raise{nullptr, ""};
  const bool two = PySequence_Fast_GET_SIZE(s) == 2;
  PyObject* x = two ? PySequence_Fast_GET_ITEM(s, 0) : nullptr;
  PyObject* y = two ? PySequence_Fast_GET_ITEM(s, 1) : nullptr;
  const bool good = two && THPVariable_Check(x) && THPVariable_Check(y);
  if (good) {
    t[0] = THPVariable_Unpack(x);
    t[1] = THPVariable_Unpack(y);
  }
  Py_DECREF(s);
  if (!good) fail(PyExc_ValueError, "%s: out must be a pair of tensors", what);
}

PyObject* pair(const at::Tensor& a, const at::Tensor& b) {
  PyObject* r = PyTuple_New(2);
  if (r == nullptr) return nullptr;
  PyTuple_SET_ITEM(r, 0, THPVariable_Wrap(a));
  PyTuple_SET_ITEM(r, 1, THPVariable_Wrap(b));
  return r;
}

struct Norm {
  const at::Tensor *q, *k, *wq, *wk, *cos, *sin, *pos;
  int64_t B, Hq, Hk, N, d, rot, n_pos;
  int64_t qs[4], ks[4];   // shapes
  int64_t strides[18];
};

Norm norm_args(const char* what, PyObject* const* a) {
  Norm n{};
  n.q = &tensor(what, "q", a[0]), n.k = &tensor(what, "k", a[1]);
  n.wq = &tensor(what, "wq", a[2]), n.wk = &tensor(what, "wk", a[3]);
  n.cos = &tensor(what, "cos", a[4]), n.sin = &tensor(what, "sin", a[5]);
  n.pos = &tensor(what, "pos", a[6]);
  heads(what, "q", *n.q, nullptr, nullptr, n.strides);
  heads(what, "k", *n.k, n.q, nullptr, n.strides + 3);
  n.B = n.q->size(0), n.Hq = n.q->size(1), n.N = n.q->size(2), n.d = n.q->size(3), n.Hk = n.k->size(1);
  if (n.k->size(0) != n.B || n.k->size(2) != n.N || n.k->size(3) != n.d)
    fail(PyExc_ValueError, "%s: q and k must share B, N and d, got %s %s", what, text(n.q->sizes()).c_str(),
         text(n.k->sizes()).c_str());
  const at::Device dev = n.q->device();
  flat(what, "wq", *n.wq, n.q->scalar_type(), {n.d}, dev);
  flat(what, "wk", *n.wk, n.q->scalar_type(), {n.d}, dev);
  if (n.cos->dim() != 2) fail(PyExc_ValueError, "%s: cos must be [n_pos, d_rot / 2]", what);
  flat(what, "cos", *n.cos, at::kFloat, n.cos->sizes(), dev);
  flat(what, "sin", *n.sin, at::kFloat, n.cos->sizes(), dev);
  flat(what, "pos", *n.pos, at::kInt, {n.B, n.N}, dev);
  n.rot = 2 * n.cos->size(1), n.n_pos = n.cos->size(0);
  const int64_t qs[4] = {n.B, n.Hq, n.N, n.d}, ks[4] = {n.B, n.Hk, n.N, n.d};
  for (int i = 0; i < 4; ++i) n.qs[i] = qs[i], n.ks[i] = ks[i];
  return n;
}

const float* f32(const at::Tensor& t) { return static_cast<const float*>(t.data_ptr()); }
const int32_t* i32(const at::Tensor& t) { return static_cast<const int32_t*>(t.data_ptr()); }

// (q, k, wq, wk, cos, sin, pos, eps, interleaved, out, stream)
PyObject* qk_norm_rope(PyObject* const* a) {
  const char* what = "qk_norm_rope";
  Norm n = norm_args(what, a);
  const Place place(a[10], n.q->device());
  at::Tensor o[2];
  outputs(what, a[9], n.q->scalar_type(), n.q->device(), n.qs, n.ks, o);
  heads(what, "out[0]", o[0], n.q, n.qs, n.strides + 6);
  heads(what, "out[1]", o[1], n.q, n.ks, n.strides + 9);
  check(moa_qk_norm_rope(n.q->data_ptr(), n.k->data_ptr(), n.wq->data_ptr(), n.wk->data_ptr(), f32(*n.cos),
                         f32(*n.sin), i32(*n.pos), o[0].data_ptr(), o[1].data_ptr(), n.B, n.Hq, n.Hk, n.N, n.d, n.rot,
                         n.n_pos, n.strides, float(number(what, "eps", a[7])), truth(a[8]), code(what, *n.q),
                         place.raw()));
  return pair(o[0], o[1]);
}

// (q, k, wq, wk, cos, sin, pos, dqo, dko, eps, interleaved, out, workspace, stream)
PyObject* qk_norm_rope_bwd(PyObject* const* a) {
  const char* what = "qk_norm_rope_bwd";
  Norm n = norm_args(what, a);
  const at::Tensor &gq = tensor(what, "dqo", a[7]), &gk = tensor(what, "dko", a[8]);
  heads(what, "dqo", gq, n.q, n.qs, n.strides + 6);
  heads(what, "dko", gk, n.q, n.ks, n.strides + 9);
  const Place place(a[13], n.q->device());
  at::Tensor o[2];
  outputs(what, a[11], n.q->scalar_type(), n.q->device(), n.qs, n.ks, o);
  heads(what, "out[0]", o[0], n.q, n.qs, n.strides + 12);
  heads(what, "out[1]", o[1], n.q, n.ks, n.strides + 15);
  const int dtype = code(what, *n.q);
  at::Tensor dwq = make({n.d}, at::kFloat, n.q->device()), dwk = make({n.d}, at::kFloat, n.q->device());
  const Scratch ws(what, a[12], moa_qk_norm_rope_bwd_workspace_bytes(n.B, n.Hq, n.Hk, n.N, n.d), place);
  check(moa_qk_norm_rope_bwd(n.q->data_ptr(), n.k->data_ptr(), n.wq->data_ptr(), n.wk->data_ptr(), f32(*n.cos),
                             f32(*n.sin), i32(*n.pos), gq.data_ptr(), gk.data_ptr(), o[0].data_ptr(), o[1].data_ptr(),
                             static_cast<float*>(dwq.data_ptr()), static_cast<float*>(dwk.data_ptr()), n.B, n.Hq, n.Hk,
                             n.N, n.d, n.rot, n.n_pos, n.strides, float(number(what, "eps", a[9])), truth(a[10]), dtype,
                             ws.p, ws.bytes, place.raw()));
  PyObject* r = PyTuple_New(4);
  if (r == nullptr) return nullptr;
  const at::Tensor* t[4] = {&o[0], &o[1], &dwq, &dwk};
  for (int i = 0; i < 4; ++i) PyTuple_SET_ITEM(r, i, THPVariable_Wrap(*t[i]));
  return r;
}

struct Cache {
  const at::Tensor *pool, *pages;
  int64_t n_pages, H, page, max_pages, dv;
};

Cache cache_args(const char* what, PyObject* pool, PyObject* pages, int64_t B, int64_t dk, at::Device dev) {
  Cache c{};
  c.pool = &tensor(what, "pool", pool), c.pages = &tensor(what, "pages", pages);
  if (c.pool->dim() != 4 || c.pool->scalar_type() != at::kByte || !c.pool->is_contiguous() || c.pool->size(3) % 9 != 0)
    fail(PyExc_ValueError, "%s: pool must be a contiguous uint8 tensor as kv4_pool makes it", what);
  if (c.pool->device() != dev)
    fail(PyExc_ValueError, "%s: pool is on %s, not on %s", what, c.pool->device().str().c_str(), dev.str().c_str());
  if (c.pages->dim() != 2) fail(PyExc_ValueError, "%s: pages must be [B, max_pages]", what);
  flat(what, "pages", *c.pages, at::kInt, {B, c.pages->size(1)}, dev);
  c.dv = c.pool->size(3) / 9 - dk;
  if ((dk != 64 && dk != 128) || (c.dv != 64 && c.dv != 128))
    fail(PyExc_ValueError, "%s: the pool's rows do not fit d_k = %lld", what, (long long)dk);
  c.n_pages = c.pool->size(0), c.H = c.pool->size(1), c.page = 16 * c.pool->size(2), c.max_pages = c.pages->size(1);
  return c;
}

// (k, v, pool, pages, pos, stream)
PyObject* kv4_write(PyObject* const* a) {
  const char* what = "kv4_write";
  const at::Tensor &k = tensor(what, "k", a[0]), &v = tensor(what, "v", a[1]), &pos = tensor(what, "pos", a[4]);
  int64_t strides[6];
  heads(what, "k", k, nullptr, nullptr, strides);
  const int64_t B = k.size(0), H = k.size(1), N = k.size(2), dk = k.size(3);
  heads(what, "v", v, &k, nullptr, strides + 3);
  const Cache c = cache_args(what, a[2], a[3], B, dk, k.device());
  const int64_t vs[4] = {B, H, N, c.dv};
  if (c.H != H || v.sizes() != at::IntArrayRef(vs, 4))
    fail(PyExc_ValueError, "%s: k %s and v %s do not fit the pool (%lld heads, d_v = %lld)", what,
         text(k.sizes()).c_str(), text(v.sizes()).c_str(), (long long)c.H, (long long)c.dv);
  flat(what, "pos", pos, at::kInt, {B, N}, k.device());
  const Place place(a[5], k.device());
  check(moa_kv4_write(k.data_ptr(), v.data_ptr(), c.pool->data_ptr(), i32(*c.pages), i32(pos), B, H, N, dk, c.dv,
                      c.n_pages, c.page, c.max_pages, strides, code(what, k), place.raw()));
  Py_RETURN_NONE;
}

// (pool, pages, pos, d_k, k, v, stream): k and v given, or both None and a dtype code in their place
PyObject* kv4_read(PyObject* const* a) {
  const char* what = "kv4_read";
  const at::Tensor& pos = tensor(what, "pos", a[2]);
  if (pos.dim() != 2 || !pos.is_cuda()) fail(PyExc_ValueError, "%s: pos must be a CUDA [B, N] tensor", what);
  const int64_t B = pos.size(0), N = pos.size(1), dk = integer(what, "d_k", a[3]);
  const at::Device dev = pos.device();
  const Cache c = cache_args(what, a[0], a[1], B, dk, dev);
  flat(what, "pos", pos, at::kInt, {B, N}, dev);
  const int64_t ks[4] = {B, c.H, N, dk}, vs[4] = {B, c.H, N, c.dv};
  const Place place(a[6], dev);
  at::Tensor o[2];
  const at::ScalarType type = integer(what, "dtype", a[4]) == MOA_FP32 ? at::kFloat : at::kBFloat16;
  outputs(what, a[5], type, dev, ks, vs, o);
  if (o[0].device() != dev) fail(PyExc_ValueError, "%s: out is on another device", what);
  int64_t strides[6];
  heads(what, "k", o[0], nullptr, ks, strides);
  heads(what, "v", o[1], &o[0], vs, strides + 3);
  check(moa_kv4_read(o[0].data_ptr(), o[1].data_ptr(), c.pool->data_ptr(), i32(*c.pages), i32(pos), B, c.H, N, dk,
                     c.dv, c.n_pages, c.page, c.max_pages, strides, code(what, o[0]), place.raw()));
  return pair(o[0], o[1]);
}

// (q, pool, pages, lens, max_len, scale, causal, out, lse, workspace, stream); lse: None, or a tensor,
// or True to make one.  Returns o or (o, lse).
PyObject* kv4_attn(PyObject* const* a) {
  const bool with_lse = a[8] != Py_None;
  const char* what = with_lse ? "kv4_attn_lse" : "kv4_attn";
  const at::Tensor &q = tensor(what, "q", a[0]), &lens = tensor(what, "lens", a[3]);
  int64_t strides[6];
  heads(what, "q", q, nullptr, nullptr, strides);
  const int64_t B = q.size(0), Hq = q.size(1), N = q.size(2), dk = q.size(3);
  const at::Device dev = q.device();
  const Cache c = cache_args(what, a[1], a[2], B, dk, dev);
  flat(what, "lens", lens, at::kInt, {B}, dev);
  const int64_t max_len = a[4] == Py_None ? c.max_pages * c.page : integer(what, "max_len", a[4]);
  const float scale = a[5] == Py_None ? float(1.0 / std::sqrt(double(dk))) : float(number(what, "scale", a[5]));
  const int dtype = code(what, q);
  const Place place(a[10], dev);
  const int64_t os[4] = {B, Hq, N, c.dv};
  at::Tensor o = a[7] == Py_None ? make(at::IntArrayRef(os, 4), q.scalar_type(), dev) : tensor(what, "out", a[7]);
  heads(what, "out", o, &q, os, strides + 3);
  at::Tensor lse;
  if (a[8] == Py_True) {
    lse = make({B, Hq, N}, at::kFloat, dev);
  } else if (with_lse) {
    lse = tensor(what, "lse", a[8]);
    flat(what, "lse", lse, at::kFloat, {B, Hq, N}, dev);
  }
  const Scratch ws(what, a[9], moa_kv4_attn_workspace_bytes(B, Hq, c.H, N, dk, c.dv, max_len, dtype), place);
  check(moa_kv4_attn(q.data_ptr(), c.pool->data_ptr(), i32(*c.pages), i32(lens), o.data_ptr(),
                     with_lse ? static_cast<float*>(lse.data_ptr()) : nullptr, B, Hq, c.H, N, dk, c.dv, c.n_pages,
                     c.page, c.max_pages, max_len, strides, scale, truth(a[6]), dtype, ws.p, ws.bytes, place.raw()));
  return with_lse ? pair(o, lse) : THPVariable_Wrap(o);
}

// Runs an entry point on its positional arguments; no C++ exception leaves it.
template <PyObject* (*F)(PyObject* const*), int ARGS>
PyObject* entry(PyObject*, PyObject* const* args, Py_ssize_t n) {
  if (n != ARGS) {
    PyErr_Format(PyExc_TypeError, "%d arguments are wanted, %zd given", ARGS, n);
    return nullptr;
  }
  try {
    return F(args);
  } catch (const Raise& e) {
    if (e.type != nullptr) PyErr_SetString(e.type, e.text.c_str());
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
  } catch (...) {
    PyErr_SetString(PyExc_RuntimeError, "unknown C++ exception");
  }
  return nullptr;
}

PyObject* set_error(PyObject*, PyObject* type) {
  Py_INCREF(type);
  Py_XDECREF(g_error);
  g_error = type;
  Py_RETURN_NONE;
}

template <PyObject* (*F)(PyObject* const*), int ARGS>
PyMethodDef method(const char* name) {
  return {name, reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(&entry<F, ARGS>)), METH_FASTCALL, nullptr};
}

PyMethodDef g_methods[] = {method<qk_norm_rope, 11>("qk_norm_rope"),
                           method<qk_norm_rope_bwd, 14>("qk_norm_rope_bwd"),
                           method<kv4_write, 6>("kv4_write"),
                           method<kv4_read, 7>("kv4_read"),
                           method<kv4_attn, 11>("kv4_attn"),
                           {"set_error", set_error, METH_O, nullptr},
                           {nullptr, nullptr, 0, nullptr}};
PyModuleDef g_module = {PyModuleDef_HEAD_INIT, "moa_torch", nullptr, -1, g_methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

extern "C" __attribute__((visibility("default"))) PyObject* PyInit_moa_torch() { return PyModule_Create(&g_module); }
