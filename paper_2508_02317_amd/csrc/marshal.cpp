// Argument marshalling of the calls that a generation or training step makes many times: the checks of libmoe.py's functions on torch tensors and the call
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

// ---- calls whose tensors all have to be on the current device -----------------------------------------------
// (The stream is the current device's, so a tensor of another one would be read without its own stream's order.)
struct Here {
  int device;
  explicit Here(PyObject* o) : device(whole32(o)) {}
  const at::Tensor& on(PyObject* o, const char* name) const {
    const at::Tensor& t = tensor(o, name);
    if (!t.is_cuda()) refuse(PyExc_ValueError, "%s must be a device tensor", name);
    if (t.get_device() != device) refuse(PyExc_ValueError, "%s is not on the current device", name);
    return t;
  }
  // contiguous, of one type and of n elements (n < 0: of any number); None: null
  const at::Tensor* flat_or_none(PyObject* o, at::ScalarType type, const char* type_name, int64_t n, const char* name) const {
    if (o == Py_None) return nullptr;
    const at::Tensor& t = on(o, name);
    flat(o, type, type_name, name);
    if (n >= 0 && t.numel() != n) PyErr_Format(PyExc_ValueError, "%s must have %lld elements", name, static_cast<long long>(n)), throw Refused{};
    return &t;
  }
  template <class T> T* numbers(PyObject* o, at::ScalarType type, const char* type_name, int64_t n, const char* name) const {
    const at::Tensor* t = flat_or_none(o, type, type_name, n, name);
    return t ? t->data_ptr<T>() : nullptr;
  }
  template <class T> T* needed(PyObject* o, at::ScalarType type, const char* type_name, int64_t n, const char* name) const {
    if (o == Py_None) refuse(PyExc_ValueError, "%s must be given", name);
    return numbers<T>(o, type, type_name, n, name);
  }
  // one byte an element: truth values or uint8
  const uint8_t* mask(PyObject* o, int64_t n, const char* name) const {
    if (o == Py_None) return nullptr;
    const at::Tensor& t = on(o, name);
    if (t.scalar_type() != at::kBool && t.scalar_type() != at::kByte) refuse(PyExc_TypeError, "%s must be bool or uint8", name);
    if (!t.is_contiguous() || t.numel() != n) refuse(PyExc_ValueError, "%s must be contiguous, one per token", name);
    return static_cast<const uint8_t*>(t.data_ptr());
  }
  Heads heads(PyObject* o, const char* name) const { on(o, name); return Heads(o, name); }
};

int code_of(at::ScalarType t) {
  if (t == at::kFloat) return MOE_F32;
  if (t == at::kBFloat16) return MOE_BF16;
  refuse(PyExc_TypeError, "%s", "libmoe supports float32 and bfloat16 tensors");
}

// [tokens, dim] or [tokens, heads, dim], rows contiguous
struct Rows {
  void* p = nullptr;
  int64_t st = 0, sh = 0;
  int tokens = 0, heads = 1, dim = 0, rank = 0;
  at::ScalarType type = at::kFloat;
  Rows() = default;
  Rows(const Here& here, PyObject* o, const char* name) {
    if (o == Py_None) return;
    const at::Tensor& t = here.on(o, name);
    rank = static_cast<int>(t.dim());
    if (rank != 2 && rank != 3) refuse(PyExc_ValueError, "%s must be [tokens, dim] or [tokens, heads, dim]", name);
    if (t.stride(rank - 1) != 1 && t.size(rank - 1) != 1) refuse(PyExc_ValueError, "%s: the elements of a row must be contiguous", name);
    p = t.data_ptr();
    tokens = size32(t, 0); heads = rank == 3 ? size32(t, 1) : 1; dim = size32(t, rank - 1);
    st = tokens > 1 ? t.stride(0) : 0;
    sh = heads > 1 ? t.stride(1) : 0;
    type = t.scalar_type();
  }
  void like(const Rows& o, const char* name) const {
    if (!rank) return;
    if (type != o.type) refuse(PyExc_TypeError, "%s has another element type", name);
    if (rank != o.rank || tokens != o.tokens || heads != o.heads || dim != o.dim) refuse(PyExc_ValueError, "%s has another shape", name);
  }
  void given(const char* name) const {
    if (!rank) refuse(PyExc_ValueError, "%s must be given", name);
  }
};

// weight and its kind: [dim] f32 or bf16 of one type, any of them None
struct Vectors {
  int code = MOE_F32;
  bool seen = false;
  void* add(const Here& here, PyObject* o, int dim, const char* name) {
    if (o == Py_None) return nullptr;
    const at::Tensor& t = here.on(o, name);
    const int c = code_of(t.scalar_type());
    if (seen && c != code) refuse(PyExc_TypeError, "%s has another type than the other weights", name);
    if (t.dim() != 1 || t.size(0) != dim || !t.is_contiguous()) refuse(PyExc_ValueError, "%s must be contiguous, one number per column", name);
    code = c;
    seen = true;
    return t.data_ptr();
  }
};

// norm_fwd(x, weight, bias, eps, rms, residual, y, sum, mean, rstd, stream, device)
PyObject* norm_fwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return call(n, 12, [&]() -> long {
    const Here here(a[11]);
    const Rows x(here, a[0], "x"), res(here, a[5], "residual"), y(here, a[6], "y"), sum(here, a[7], "h");
    x.given("x"); y.given("y");
    res.like(x, "residual"); y.like(x, "y"); sum.like(x, "h");
    const int code = code_of(x.type);
    Vectors v;
    const void *w = v.add(here, a[1], x.dim, "weight"), *b = v.add(here, a[2], x.dim, "bias");
    const double eps = PyFloat_AsDouble(a[3]);
    if (eps == -1.0 && PyErr_Occurred()) throw Refused{};
    const int64_t rows = static_cast<int64_t>(x.tokens) * x.heads;
    float *mean = here.numbers<float>(a[8], at::kFloat, "float32", rows, "mean"), *rstd = here.numbers<float>(a[9], at::kFloat, "float32", rows, "rstd");
    return moe_norm_fwd(x.p, x.st, x.sh, res.p, res.st, res.sh, code, x.tokens, x.heads, x.dim, truth(a[4]), w, b, v.code, static_cast<float>(eps), sum.p, sum.st, sum.sh, y.p,
                        y.st, y.sh, mean, rstd, stream_of(a[10]));
  });
}

// norm_bwd(dy, x, rstd, mean, weight, add, dx, dweight, dbias, ws, stream, device)
PyObject* norm_bwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return call(n, 12, [&]() -> long {
    const Here here(a[11]);
    const Rows dy(here, a[0], "dy"), x(here, a[1], "x"), add(here, a[5], "add"), dx(here, a[6], "dx");
    x.given("x"); dy.given("dy"); dx.given("dx");
    dy.like(x, "dy"); add.like(x, "add"); dx.like(x, "dx");
    const int code = code_of(x.type);
    const int64_t rows = static_cast<int64_t>(x.tokens) * x.heads;
    const float *rstd = here.needed<float>(a[2], at::kFloat, "float32", rows, "rstd"), *mean = here.numbers<float>(a[3], at::kFloat, "float32", rows, "mean");
    Vectors v;
    const void* w = v.add(here, a[4], x.dim, "weight");
    void *dw = v.add(here, a[7], x.dim, "dweight"), *db = v.add(here, a[8], x.dim, "dbias");
    void* ws = nullptr;
    size_t bytes = 0;
    if (a[9] != Py_None) {
      const at::Tensor& t = here.on(a[9], "ws");
      if (!t.is_contiguous()) refuse(PyExc_ValueError, "%s must be a contiguous device tensor", "ws");
      ws = t.data_ptr();
      bytes = t.nbytes();
    }
    return moe_norm_bwd(dy.p, dy.st, dy.sh, x.p, x.st, x.sh, code, x.tokens, x.heads, x.dim, mean, rstd, w, v.code, add.p, add.st, add.sh, dx.p, dx.st, dx.sh, dw, db, ws, bytes,
                        stream_of(a[10]));
  });
}

// positions [n_axes, T], the table, the axis of every pair (bytes)
struct AxesTable {
  const int32_t* positions = nullptr;
  const float *cos = nullptr, *sin = nullptr;
  const uint8_t* pair_axis = nullptr;
  int n_axes = 1, n_pos = 0, rot = 0;
  AxesTable(const Here& here, PyObject* po, PyObject* co, PyObject* so, PyObject* pair, int T) {
    if (!PyBytes_Check(pair)) refuse(PyExc_TypeError, "%s must be bytes, the axis of every pair", "pair_axis");
    if (po == Py_None || co == Py_None || so == Py_None) refuse(PyExc_ValueError, "%s must be given", "positions, cos and sin");
    const at::Tensor &c = *here.flat_or_none(co, at::kFloat, "float32", -1, "cos"), &s = *here.flat_or_none(so, at::kFloat, "float32", -1, "sin"),
                     &p = *here.flat_or_none(po, at::kInt, "int32", -1, "positions");
    if (c.dim() != 2 || s.sizes() != c.sizes() || p.dim() != 2 || p.size(1) != T) {
      PyErr_Format(PyExc_ValueError, "cos and sin must be [n_pos, rot / 2] and positions [axes, %d]", T);
      throw Refused{};
    }
    if (PyBytes_GET_SIZE(pair) != c.size(1)) refuse(PyExc_ValueError, "%s must have one entry per pair", "pair_axis");
    positions = p.data_ptr<int32_t>(); cos = c.data_ptr<float>(); sin = s.data_ptr<float>();
    pair_axis = reinterpret_cast<const uint8_t*>(PyBytes_AS_STRING(pair));
    n_axes = size32(p, 0); n_pos = size32(c, 0); rot = 2 * size32(c, 1);
  }
};

// rope_axes(back, q, k, positions, cos, sin, pair_axis, interleaved, q_out, k_out, stream, device)
PyObject* rope_axes(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return call(n, 12, [&]() -> long {
    const Here here(a[11]);
    Heads q, k, qo, ko;
    const bool has_q = a[1] != Py_None, has_k = a[2] != Py_None;
    if (!has_q && !has_k) refuse(PyExc_ValueError, "%s must be given", "q or k");
    if (has_q) q = here.heads(a[1], "q");
    if (has_k) k = here.heads(a[2], "k");
    const Heads& some = has_q ? q : k;
    const int code = code_of(some.type);
    if (has_q) { qo = here.heads(a[8], "q out"); qo.like(q.tokens, q.heads, q.dim, q.type, "q out"); }
    if (has_k) {
      k.like(some.tokens, k.heads, some.dim, some.type, "k");
      ko = here.heads(a[9], "k out");
      ko.like(k.tokens, k.heads, k.dim, k.type, "k out");
    }
    const AxesTable t(here, a[3], a[4], a[5], a[6], some.tokens);
    return (truth(a[0]) ? moe_rope_axes_bwd : moe_rope_axes_fwd)(q.p, q.st, q.sh, k.p, k.st, k.sh, code, some.tokens, q.heads, k.heads, some.dim, t.rot, t.positions, t.n_axes,
                                                                 t.pair_axis, t.cos, t.sin, t.n_pos, truth(a[7]), qo.p, qo.st, qo.sh, ko.p, ko.st, ko.sh, stream_of(a[10]));
  });
}

// kv_cache_write_axes(cache, cache_device, k, v, slots, q, positions, cos, sin, pair_axis, interleaved, q_out, stream, device)
PyObject* kv_cache_write_axes(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return call(n, 14, [&]() -> long {
    const Here here(a[13]);
    const moe_kv_cache_t* c = cache_of(a[0]);
    if (whole32(a[1]) != here.device) refuse(PyExc_ValueError, "%s is not on the current device", "cache");
    const at::ScalarType type = beside(c);
    const Heads k = here.heads(a[2], "k"), v = here.heads(a[3], "v");
    const int T = k.tokens;
    k.like(T, c->heads, c->dim, type, "k");
    v.like(T, c->heads, c->dim, type, "v");
    const int64_t* slots = here.needed<int64_t>(a[4], at::kLong, "int64", T, "slots");
    Heads q, qo;
    if (a[5] != Py_None) {
      q = here.heads(a[5], "q");
      q.like(T, q.heads, c->dim, type, "q");
      qo = here.heads(a[11], "q_out");
      qo.like(T, q.heads, c->dim, type, "q_out");
    }
    const AxesTable t(here, a[6], a[7], a[8], a[9], T);
    return moe_kv_cache_write_axes(c, k.p, k.st, k.sh, v.p, v.st, v.sh, T, slots, q.p, q.st, q.sh, q.heads, t.rot, t.positions, t.n_axes, t.pair_axis, t.cos, t.sin, t.n_pos,
                                   truth(a[10]), qo.p, qo.st, qo.sh, stream_of(a[12]));
  });
}

struct Logits {
  const float* p;
  int T, E;
  Logits(const Here& here, PyObject* o) {
    if (o == Py_None) refuse(PyExc_ValueError, "%s must be given", "logits");
    const at::Tensor& t = *here.flat_or_none(o, at::kFloat, "float32", -1, "logits");
    if (t.dim() != 2) refuse(PyExc_ValueError, "%s must be [tokens, experts]", "logits");
    p = t.data_ptr<float>(); T = size32(t, 0); E = size32(t, 1);
  }
};

// balance_loss_fwd(logits, topk_idx, valid, losses, counts, importance, lse, ws, stream, device)
PyObject* balance_loss_fwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return call(n, 10, [&]() -> long {
    const Here here(a[9]);
    const Logits z(here, a[0]);
    if (a[1] == Py_None) refuse(PyExc_ValueError, "%s must be given", "topk_idx");
    const at::Tensor& idx = *here.flat_or_none(a[1], at::kInt, "int32", -1, "topk_idx");
    if (idx.dim() != 2 || idx.size(0) != z.T) refuse(PyExc_ValueError, "%s must be [tokens, k]", "topk_idx");
    const uint8_t* valid = here.mask(a[2], z.T, "valid");
    float *losses = here.needed<float>(a[3], at::kFloat, "float32", 2, "losses"), *importance = here.needed<float>(a[5], at::kFloat, "float32", z.E, "importance"),
          *lse = here.needed<float>(a[6], at::kFloat, "float32", z.T, "lse");
    int32_t* counts = here.needed<int32_t>(a[4], at::kInt, "int32", static_cast<int64_t>(z.E) + 1, "counts");
    const at::Tensor& ws = here.on(a[7], "ws");
    if (!ws.is_contiguous()) refuse(PyExc_ValueError, "%s must be a contiguous device tensor", "ws");
    return moe_balance_loss_fwd(z.p, idx.data_ptr<int32_t>(), valid, z.T, z.E, size32(idx, 1), losses, counts, importance, lse, ws.data_ptr(), ws.nbytes(), stream_of(a[8]));
  });
}

// balance_loss_bwd(logits, counts, lse, k, balance, z, dlosses, valid, add, dlogits, stream, device)
PyObject* balance_loss_bwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return call(n, 12, [&]() -> long {
    const Here here(a[11]);
    const Logits z(here, a[0]);
    const int32_t* counts = here.needed<int32_t>(a[1], at::kInt, "int32", static_cast<int64_t>(z.E) + 1, "counts");
    const float* lse = here.needed<float>(a[2], at::kFloat, "float32", z.T, "lse");
    const double balance = PyFloat_AsDouble(a[4]), zw = PyFloat_AsDouble(a[5]);
    if (PyErr_Occurred()) throw Refused{};
    const float* dlosses = here.numbers<float>(a[6], at::kFloat, "float32", 2, "dlosses");
    const uint8_t* valid = here.mask(a[7], z.T, "valid");
    const int64_t all = static_cast<int64_t>(z.T) * z.E;
    const float* add = here.numbers<float>(a[8], at::kFloat, "float32", all, "add");
    float* out = here.needed<float>(a[9], at::kFloat, "float32", all, "dlogits");
    return moe_balance_loss_bwd(z.p, counts, lse, valid, z.T, z.E, whole32(a[3]), static_cast<float>(balance), static_cast<float>(zw), dlosses, add, out, stream_of(a[10]));
  });
}

PyMethodDef kMethods[] = {
  {"rope", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(rope)), METH_FASTCALL, "(back, q, k, positions, cos, sin, interleaved, q_out, k_out, stream) -> status"},
  {"kv_cache_write", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(kv_cache_write)), METH_FASTCALL,
   "(cache, k, v, slots, q, positions, cos, sin, interleaved, q_out, stream) -> status"},
  {"kv_cache_read", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(kv_cache_read)), METH_FASTCALL, "(cache, pages, row_start, first, k_out, v_out, stream) -> status"},
  {"paged_attn_decode", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(paged_attn_decode)), METH_FASTCALL,
   "(cache, q, pages, lens, scale, window, out, lse, ws, stream) -> status"},
  {"norm_fwd", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(norm_fwd)), METH_FASTCALL, "(x, weight, bias, eps, rms, residual, y, sum, mean, rstd, stream, device) -> status"},
  {"norm_bwd", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(norm_bwd)), METH_FASTCALL, "(dy, x, rstd, mean, weight, add, dx, dweight, dbias, ws, stream, device) -> status"},
  {"rope_axes", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(rope_axes)), METH_FASTCALL, "(back, q, k, positions, cos, sin, pair_axis, interleaved, q_out, k_out, stream, device) -> status"},
  {"kv_cache_write_axes", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(kv_cache_write_axes)), METH_FASTCALL, "(cache, cache_device, k, v, slots, q, positions, cos, sin, pair_axis, interleaved, q_out, stream, device) -> status"},
  {"balance_loss_fwd", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(balance_loss_fwd)), METH_FASTCALL, "(logits, topk_idx, valid, losses, counts, importance, lse, ws, stream, device) -> status"},
  {"balance_loss_bwd", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(balance_loss_bwd)), METH_FASTCALL, "(logits, counts, lse, k, balance, z, dlosses, valid, add, dlogits, stream, device) -> status"},
  {nullptr, nullptr, 0, nullptr}};
PyModuleDef kModule = {PyModuleDef_HEAD_INIT, "_marshal", "Marshalling of torch tensors into libmoe's C ABI.", -1, kMethods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__marshal(void) { return PyModule_Create(&kModule); }
