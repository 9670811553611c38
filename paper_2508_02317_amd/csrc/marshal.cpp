// Argument marshalling of the calls that a generation step makes many times: the checks of libmoe.py's functions on torch tensors and the call
// into the C ABI, without the interpreter in between.  A small call is bound by the host: 256 tokens rotated take 4.5 us on the GPU
// (launch to launch), 9.1 to be enqueued through ctypes and 4.2 from here.
// Built as a Python extension module beside libmoe_gfx950.so; libmoe.py uses it where it has been built.
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <torch/csrc/autograd/python_variable.h>
#include <new>
#include <exception>
#include "moe.h"

namespace {

struct Refused {};                                     // a Python error is set
[[noreturn]] void refuse(PyObject* type, const char* fmt, const char* name) {
  PyErr_Format(type, fmt, name);
  throw Refused{};
}

const at::Tensor& tensor(PyObject* o, const char* name) {
  if (!THPVariable_Check(o)) refuse(PyExc_TypeError, "%s must be a tensor", name);
  return THPVariable_Unpack(o);
}
long whole(PyObject* o) {
  const long v = PyLong_AsLong(o);
  if (v == -1 && PyErr_Occurred()) throw Refused{};
  return v;
}
int whole32(PyObject* o) {
  const long v = whole(o);
  if (v != static_cast<int>(v)) {
    PyErr_SetString(PyExc_OverflowError, "an int argument does not fit 32 bits");
    throw Refused{};
  }
  return static_cast<int>(v);
}
bool truth(PyObject* o) {
  const int v = PyObject_IsTrue(o);
  if (v < 0) throw Refused{};
  return v != 0;
}
int size32(const at::Tensor& t, int dim) {             // sizes beyond 32 bits are not marshalled to something smaller
  const int64_t v = t.size(dim);
  if (v != static_cast<int>(v)) {
    PyErr_SetString(PyExc_ValueError, "a tensor's size does not fit 32 bits");
    throw Refused{};
  }
  return static_cast<int>(v);
}

// a contiguous device tensor of one type
const at::Tensor& flat(PyObject* o, at::ScalarType type, const char* type_name, const char* name) {
  const at::Tensor& t = tensor(o, name);
  if (!t.is_cuda() || !t.is_contiguous()) refuse(PyExc_ValueError, "%s must be a contiguous device tensor", name);
  if (t.scalar_type() != type) PyErr_Format(PyExc_TypeError, "%s must be %s", name, type_name), throw Refused{};
  return t;
}

// [tokens, heads, dim], heads contiguous
struct Heads {
  void* p = nullptr;
  int64_t st = 0, sh = 0;
  int tokens = 0, heads = 0, dim = 0;
  at::ScalarType type = at::kFloat;
  Heads() = default;
  Heads(PyObject* o, const char* name) {
    const at::Tensor& t = tensor(o, name);
    if (t.dim() != 3 || !t.is_cuda()) refuse(PyExc_ValueError, "%s must be a [tokens, heads, dim] device tensor", name);
    if (t.stride(2) != 1 && t.size(2) != 1) refuse(PyExc_ValueError, "%s: the elements of a head must be contiguous", name);
    p = t.data_ptr();
    tokens = size32(t, 0); heads = size32(t, 1); dim = size32(t, 2);
    st = tokens > 1 ? t.stride(0) : 0;                 // the stride of one token or one head is never taken
    sh = heads > 1 ? t.stride(1) : 0;
    type = t.scalar_type();
  }
  void like(int T, int H, int D, at::ScalarType want, const char* name) const {
    if (type != want) refuse(PyExc_TypeError, "%s has another element type", name);
    if (tokens != T || heads != H || dim != D)
      PyErr_Format(PyExc_ValueError, "%s must have shape (%d, %d, %d), got (%d, %d, %d)", name, T, H, D, tokens, heads, dim), throw Refused{};
  }
};

struct Table {
  const int32_t* positions = nullptr;
  const float *cos = nullptr, *sin = nullptr;
  int n_pos = 0, rot = 0;
  Table(PyObject* po, PyObject* co, PyObject* so, int T) {
    if (co == Py_None) return;
    const at::Tensor &c = flat(co, at::kFloat, "float32", "cos"), &s = flat(so, at::kFloat, "float32", "sin"), &p = flat(po, at::kInt, "int32", "positions");
    if (c.dim() != 2 || s.dim() != 2 || c.size(0) != s.size(0) || c.size(1) != s.size(1) || p.numel() != T) {
      PyErr_Format(PyExc_ValueError, "cos and sin must be [n_pos, rot / 2] and positions [%d]", T);
      throw Refused{};
    }
    positions = p.data_ptr<int32_t>(); cos = c.data_ptr<float>(); sin = s.data_ptr<float>();
    n_pos = size32(c, 0); rot = 2 * size32(c, 1);
  }
};

// What every function does around its own marshalling: a count of arguments, and no C++ exception past the interpreter.
template <class F> PyObject* call(Py_ssize_t got, Py_ssize_t want, F f) {
  if (got != want) {
    PyErr_Format(PyExc_TypeError, "%zd arguments, %zd expected", got, want);
    return nullptr;
  }
  try {
    return PyLong_FromLong(f());
  } catch (const Refused&) {
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
  } catch (...) {
    PyErr_SetString(PyExc_RuntimeError, "unknown C++ exception");
  }
  return nullptr;
}
void* stream_of(PyObject* o) { return reinterpret_cast<void*>(static_cast<intptr_t>(whole(o))); }
const moe_kv_cache_t* cache_of(PyObject* o) { return reinterpret_cast<const moe_kv_cache_t*>(static_cast<intptr_t>(whole(o))); }
at::ScalarType beside(const moe_kv_cache_t* c) { return c->dtype == MOE_F32 ? at::kFloat : at::kBFloat16; }

// rope(back, q, k, positions, cos, sin, interleaved, q_out, k_out, stream)
PyObject* rope(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return call(n, 10, [&]() -> long {
    Heads q, k, qo, ko;
    const bool has_q = a[1] != Py_None, has_k = a[2] != Py_None;
    if (has_q) q = Heads(a[1], "q");
    if (has_k) k = Heads(a[2], "k");
    if (!has_q && !has_k) refuse(PyExc_ValueError, "%s must be given", "q or k");
    const Heads& some = has_q ? q : k;
    if (some.type != at::kFloat && some.type != at::kBFloat16) refuse(PyExc_TypeError, "%s", "libmoe supports float32 and bfloat16 tensors");
    if (has_q) { qo = Heads(a[7], "q out"); qo.like(q.tokens, q.heads, q.dim, q.type, "q out"); }
    if (has_k) {
      k.like(some.tokens, k.heads, some.dim, some.type, "k");
      ko = Heads(a[8], "k out");
      ko.like(k.tokens, k.heads, k.dim, k.type, "k out");
    }
    const Table t(a[3], a[4], a[5], some.tokens);
    const int code = some.type == at::kFloat ? MOE_F32 : MOE_BF16;
    return (truth(a[0]) ? moe_rope_bwd : moe_rope_fwd)(q.p, q.st, q.sh, k.p, k.st, k.sh, code, some.tokens, q.heads, k.heads, some.dim, t.rot, t.positions, t.cos,
                                                       t.sin, t.n_pos, truth(a[6]), qo.p, qo.st, qo.sh, ko.p, ko.st, ko.sh, stream_of(a[9]));
  });
}

// kv_cache_write(cache, k, v, slots, q, positions, cos, sin, interleaved, q_out, stream)
PyObject* kv_cache_write(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return call(n, 11, [&]() -> long {
    const moe_kv_cache_t* c = cache_of(a[0]);
    const at::ScalarType type = beside(c);
    const Heads k(a[1], "k"), v(a[2], "v");
    const int T = k.tokens;
    k.like(T, c->heads, c->dim, type, "k");
    v.like(T, c->heads, c->dim, type, "v");
    const at::Tensor& slots = flat(a[3], at::kLong, "int64", "slots");
    if (slots.numel() != T) refuse(PyExc_ValueError, "%s must be one per token", "slots");
    Heads q, qo;
    if (a[4] != Py_None) {
      q = Heads(a[4], "q");
      q.like(T, q.heads, c->dim, type, "q");
      qo = Heads(a[9], "q_out");
      qo.like(T, q.heads, c->dim, type, "q_out");
    }
    const Table t(a[5], a[6], a[7], T);
    return moe_kv_cache_write(c, k.p, k.st, k.sh, v.p, v.st, v.sh, T, slots.data_ptr<int64_t>(), q.p, q.st, q.sh, q.heads, t.rot, t.positions, t.cos, t.sin, t.n_pos,
                              truth(a[8]), qo.p, qo.st, qo.sh, stream_of(a[10]));
  });
}

// kv_cache_read(cache, pages, row_start, first, k_out, v_out, stream)
PyObject* kv_cache_read(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return call(n, 7, [&]() -> long {
    const moe_kv_cache_t* c = cache_of(a[0]);
    const at::ScalarType type = beside(c);
    const at::Tensor &pages = flat(a[1], at::kInt, "int32", "pages"), &starts = flat(a[2], at::kInt, "int32", "row_start");
    if (pages.dim() != 2) refuse(PyExc_ValueError, "%s must be [sequences, max_pages]", "pages");
    const int B = size32(pages, 0);
    if (starts.numel() != static_cast<int64_t>(B) + 1) refuse(PyExc_ValueError, "%s must have one entry more than there are sequences", "row_start");
    const int32_t* first = nullptr;
    if (a[3] != Py_None) {
      const at::Tensor& t = flat(a[3], at::kInt, "int32", "first");
      if (t.numel() != B) refuse(PyExc_ValueError, "%s must be one per sequence", "first");
      first = t.data_ptr<int32_t>();
    }
    const char* type_name = type == at::kFloat ? "float32" : "bfloat16";
    const at::Tensor &k = flat(a[4], type, type_name, "k out"), &v = flat(a[5], type, type_name, "v out");
    if (k.dim() != 3 || k.size(1) != c->heads || k.size(2) != c->dim || v.sizes() != k.sizes()) {
      PyErr_Format(PyExc_ValueError, "out must be two tensors [rows, %d, %d]", c->heads, c->dim);
      throw Refused{};
    }
    return moe_kv_cache_read(c, pages.data_ptr<int32_t>(), size32(pages, 1), starts.data_ptr<int32_t>(), first, B, size32(k, 0), k.data_ptr(), v.data_ptr(),
                             stream_of(a[6]));
  });
}

// paged_attn_decode(cache, q, pages, lens, scale, window, out, lse, ws, stream)
PyObject* paged_attn_decode(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return call(n, 10, [&]() -> long {
    const moe_kv_cache_t* c = cache_of(a[0]);
    const at::ScalarType type = beside(c);
    const Heads q(a[1], "q");
    const int B = q.tokens, Hq = q.heads;
    q.like(B, Hq, c->dim, type, "q");
    const at::Tensor &pages = flat(a[2], at::kInt, "int32", "pages"), &lens = flat(a[3], at::kInt, "int32", "lens");
    if (pages.dim() != 2 || pages.size(0) != B || lens.numel() != B) {
      PyErr_Format(PyExc_ValueError, "pages must be [%d, max_pages] and lens [%d]", B, B);
      throw Refused{};
    }
    const double scale = PyFloat_AsDouble(a[4]);
    if (scale == -1.0 && PyErr_Occurred()) throw Refused{};
    const at::Tensor& out = flat(a[6], type, type == at::kFloat ? "float32" : "bfloat16", "out");
    if (out.dim() != 3 || out.size(0) != B || out.size(1) != Hq || out.size(2) != c->dim) refuse(PyExc_ValueError, "%s must have the shape of q", "out");
    float* lse = nullptr;
    if (a[7] != Py_None) {
      const at::Tensor& t = flat(a[7], at::kFloat, "float32", "lse");
      if (t.dim() != 2 || t.size(0) != B || t.size(1) != Hq) refuse(PyExc_ValueError, "%s must be one number per sequence and head", "lse");
      lse = t.data_ptr<float>();
    }
    const at::Tensor& ws = tensor(a[8], "ws");
    if (!ws.is_cuda() || !ws.is_contiguous()) refuse(PyExc_ValueError, "%s must be a contiguous device tensor", "ws");
    return moe_paged_attn_decode(q.p, q.st, q.sh, c, pages.data_ptr<int32_t>(), size32(pages, 1), lens.data_ptr<int32_t>(), B, Hq, static_cast<float>(scale),
                                 whole32(a[5]), out.data_ptr(), lse, ws.data_ptr(), ws.nbytes(), stream_of(a[9]));
  });
}

PyMethodDef kMethods[] = {
  {"rope", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(rope)), METH_FASTCALL, "(back, q, k, positions, cos, sin, interleaved, q_out, k_out, stream) -> status"},
  {"kv_cache_write", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(kv_cache_write)), METH_FASTCALL,
   "(cache, k, v, slots, q, positions, cos, sin, interleaved, q_out, stream) -> status"},
  {"kv_cache_read", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(kv_cache_read)), METH_FASTCALL, "(cache, pages, row_start, first, k_out, v_out, stream) -> status"},
  {"paged_attn_decode", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(paged_attn_decode)), METH_FASTCALL,
   "(cache, q, pages, lens, scale, window, out, lse, ws, stream) -> status"},
  {nullptr, nullptr, 0, nullptr}};
PyModuleDef kModule = {PyModuleDef_HEAD_INIT, "_marshal", "Marshalling of torch tensors into libmoe's C ABI.", -1, kMethods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__marshal(void) { return PyModule_Create(&kModule); }
