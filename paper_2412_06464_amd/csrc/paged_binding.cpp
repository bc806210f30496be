// What the Python binding of the attention layer (paged.py) asks of its tensors,
// read off them directly: checks and the byte images of gdn_paged.h's structures.
// The same reads through Python attributes cost 0.5 to 2 us each, several per
// call, where the kernel behind the call takes five.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <string.h>

#include <ATen/Functions.h>
#include <ATen/core/Tensor.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include "../../include/gdn_paged.h"

namespace {

using at::Tensor;

PyObject* fail(PyObject* type, const char* fmt, const char* a = "", const char* b = "") {
  PyErr_Format(type, fmt, a, b);
  return nullptr;
}

const Tensor* tensor(const char* name, PyObject* x) {
  if (THPVariable_Check(x)) return &THPVariable_Unpack(x);
  fail(PyExc_TypeError, "%s must be a tensor", name);
  return nullptr;
}

template <class T> PyObject* bytes(const T& x) {
  return PyBytes_FromStringAndSize((const char*)&x, sizeof x);
}

bool dtype_of(const Tensor& x, gdn_dtype* out) {
  if (x.scalar_type() == at::kFloat) *out = GDN_F32;
  else if (x.scalar_type() == at::kBFloat16) *out = GDN_BF16;
  else return false;
  return true;
}

bool four(const char* name, const Tensor& x) {
  if (x.dim() == 4) return true;
  fail(PyExc_ValueError, "%s must be [B, T, heads, d]", name);
  return false;
}

// gdn_rows of a [B, T, heads, d] tensor; false: an exception is set.
bool rows_of(const char* name, const Tensor& x, gdn_rows* out) {
  const auto n = x.sizes(), s = x.strides();
  if (s[3] != 1) {
    fail(PyExc_ValueError, "%s must be contiguous in its last dim", name);
    return false;
  }
  int64_t token = s[1];
  if (n[0] > 1 && s[0] != n[1] * token) {
    if (n[1] != 1) {
      fail(PyExc_ValueError, "%s: the rows of B must follow each other, T tokens apart", name);
      return false;
    }
    token = s[0];  // a token a row: the rows' own stride
  }
  out->data = x.data_ptr();
  out->token_stride = token;
  out->head_stride = s[2];
  return true;
}

// contiguous int32 on the device of `like`
bool ints_of(const char* name, const Tensor& x, const Tensor& like) {
  if (x.scalar_type() == at::kInt && x.get_device() == like.get_device() && x.is_contiguous())
    return true;
  fail(PyExc_ValueError, "%s must be contiguous int32 on the call's device", name);
  return false;
}

#define NAME(i)                                              \
  PyUnicode_AsUTF8(args[i]);                                 \
  if (PyErr_Occurred()) return nullptr

// first(name, x) -> gdn_rows: the tensor that a call's others have to match
PyObject* first(PyObject*, PyObject* const* args, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  if (n != 2) return fail(PyExc_TypeError, "first takes 2 arguments");
  const char* name = NAME(0);
  const Tensor* x = tensor(name, args[1]);
  if (!x || !four(name, *x)) return nullptr;
  gdn_dtype dt;
  if (!dtype_of(*x, &dt)) return fail(PyExc_TypeError, "%s must be float32 or bfloat16", name);
  if (x->get_device() < 0) return fail(PyExc_ValueError, "%s must be on the GPU", name);
  gdn_rows r;
  return rows_of(name, *x, &r) ? bytes(r) : nullptr;
  END_HANDLE_TH_ERRORS
}

// rows(name, x, first's name, first, heads or -1) -> gdn_rows
PyObject* rows(PyObject*, PyObject* const* args, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  if (n != 5) return fail(PyExc_TypeError, "rows takes 5 arguments");
  const char* name = NAME(0);
  const Tensor* x = tensor(name, args[1]);
  const char* other = NAME(2);
  const Tensor* y = x ? tensor(other, args[3]) : nullptr;
  if (!x || !y || !four(name, *x)) return nullptr;
  const int64_t heads = PyLong_AsLongLong(args[4]);
  if (PyErr_Occurred()) return nullptr;
  if (x->scalar_type() != y->scalar_type() || x->get_device() != y->get_device())
    return fail(PyExc_ValueError, "%s must have %s's dtype and device", name, other);
  if (x->size(0) != y->size(0) || x->size(1) != y->size(1) || x->size(3) != y->size(3))
    return fail(PyExc_ValueError, "%s must have %s's B, T and d", name, other);
  if (heads >= 0 && x->size(2) != heads)
    return PyErr_Format(PyExc_ValueError, "%s must have %lld heads", name, (long long)heads);
  gdn_rows r;
  return rows_of(name, *x, &r) ? bytes(r) : nullptr;
  END_HANDLE_TH_ERRORS
}

// like(x) -> (a new tensor shaped as x, its gdn_rows)
PyObject* like(PyObject*, PyObject* const* args, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  if (n != 1) return fail(PyExc_TypeError, "like takes 1 argument");
  const Tensor* x = tensor("x", args[0]);
  if (!x || !four("x", *x)) return nullptr;
  Tensor y = at::empty(x->sizes(), x->options().requires_grad(false));
  gdn_rows r;
  if (!rows_of("the output", y, &r)) return nullptr;
  PyObject* t = THPVariable_Wrap(std::move(y));
  PyObject* b = t ? bytes(r) : nullptr;
  PyObject* out = b ? PyTuple_Pack(2, t, b) : nullptr;
  Py_XDECREF(t);
  Py_XDECREF(b);
  return out;
  END_HANDLE_TH_ERRORS
}

// book(table, lens, refs, page_size, out or None, with_lens, extra) -> (gdn_book, dict of the
// outputs: those of `out`, the missing ones new, the pointer of the one named extra, which is
// shaped as refs ("map") or as lens)
PyObject* book(PyObject*, PyObject* const* args, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  if (n != 7) return fail(PyExc_TypeError, "book takes 7 arguments");
  const Tensor* table = tensor("table", args[0]);
  const Tensor* lens = table ? tensor("lens", args[1]) : nullptr;
  const Tensor* refs = lens ? tensor("refs", args[2]) : nullptr;
  if (!refs) return nullptr;
  const long page_size = PyLong_AsLong(args[3]);
  const int with_lens = PyObject_IsTrue(args[5]);
  const char* extra = NAME(6);
  if (table->dim() != 2) return fail(PyExc_ValueError, "table must be int32 [sequences, blocks]");
  if (refs->dim() != 1) return fail(PyExc_ValueError, "refs must be int32 [pages]");
  if (table->get_device() < 0) return fail(PyExc_ValueError, "table must be on the GPU");
  if (!ints_of("table", *table, *table) || !ints_of("lens", *lens, *table) ||
      !ints_of("refs", *refs, *table))
    return nullptr;
  if (lens->dim() != 1 || lens->size(0) != table->size(0))
    return fail(PyExc_ValueError, "lens must be int32 [sequences]");
  const int64_t most = 0x7fffffff;
  if (table->size(0) > most || table->size(1) > most || refs->size(0) > most ||
      page_size < INT32_MIN || page_size > most)
    return fail(PyExc_ValueError, "the table is too large");
  gdn_book b = {};
  b.S = (int32_t)table->size(0);
  b.max_blocks = (int32_t)table->size(1);
  b.num_pages = (int32_t)refs->size(0);
  b.page_size = (int32_t)page_size;
  b.table = table->data_ptr<int32_t>();
  b.lens = lens->data_ptr<int32_t>();
  b.refs = refs->data_ptr<int32_t>();
  PyObject* got = PyDict_New();
  if (!got) return nullptr;
  if (args[4] != Py_None && PyDict_Update(got, args[4]) < 0) {
    Py_DECREF(got);
    return nullptr;
  }
  const Tensor* like_extra = strcmp(extra, "map") == 0 ? refs : lens;
  struct Out {
    const char* name;
    const Tensor* like;
    int32_t* ptr;
  } outs[] = {{"table", table, nullptr}, {"refs", refs, nullptr}, {extra, like_extra, nullptr},
              {"lens", lens, nullptr}};
  for (int i = 0; i < (with_lens ? 4 : 3); ++i) {
    Out& o = outs[i];
    PyObject* have = PyDict_GetItemString(got, o.name);  // borrowed
    if (!have || have == Py_None) {
      PyObject* fresh = THPVariable_Wrap(at::empty(o.like->sizes(), o.like->options()));
      if (!fresh || PyDict_SetItemString(got, o.name, fresh) < 0) {
        Py_XDECREF(fresh);
        Py_DECREF(got);
        return nullptr;
      }
      Py_DECREF(fresh);
      have = fresh;  // held by the dict
    }
    const Tensor* x = tensor(o.name, have);
    if (!x || !ints_of(o.name, *x, *table) || x->sizes() != o.like->sizes()) {
      if (!PyErr_Occurred()) fail(PyExc_ValueError, "out: %s has the wrong shape", o.name);
      Py_DECREF(got);
      return nullptr;
    }
    o.ptr = x->data_ptr<int32_t>();
  }
  b.table_out = outs[0].ptr;
  b.refs_out = outs[1].ptr;
  b.lens_out = outs[3].ptr;
  PyObject* image = bytes(b);
  PyObject* ptr = image ? PyLong_FromVoidPtr(outs[2].ptr) : nullptr;
  PyObject* out = ptr ? PyTuple_Pack(3, image, got, ptr) : nullptr;
  Py_XDECREF(image);
  Py_XDECREF(ptr);
  Py_DECREF(got);
  return out;
  END_HANDLE_TH_ERRORS
}

// pool(pool, first) -> gdn_pool of a [parts, pages, ...] tensor whose pages are contiguous
PyObject* pool(PyObject*, PyObject* const* args, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  if (n != 2) return fail(PyExc_TypeError, "pool takes 2 arguments");
  const Tensor* x = tensor("pool", args[0]);
  const Tensor* y = x ? tensor("first", args[1]) : nullptr;
  if (!y) return nullptr;
  if (x->dim() < 3 || x->get_device() < 0 || x->get_device() != y->get_device())
    return fail(PyExc_ValueError, "pool must be a [parts, pages, ...] tensor on the GPU of the call");
  int64_t inner = 1;
  for (int64_t i = x->dim() - 1; i > 1; --i) {
    if (x->size(i) != 1 && x->stride(i) != inner)
      return fail(PyExc_ValueError, "pool must be contiguous within a page");
    inner *= x->size(i);
  }
  if (x->size(0) > 0x7fffffff || x->size(1) > 0x7fffffff)
    return fail(PyExc_ValueError, "too many pages");
  const int64_t e = x->element_size();
  gdn_pool p = {};
  p.data = x->data_ptr();
  p.parts = (int32_t)x->size(0);
  p.num_pages = (int32_t)x->size(1);
  p.part_stride = x->stride(0) * e;
  p.page_stride = x->stride(1) * e;
  p.page_bytes = inner * e;
  return bytes(p);
  END_HANDLE_TH_ERRORS
}

// ints(name, x, first, dims...) -> pointer of a contiguous int32 tensor of these dims (any: none)
PyObject* ints(PyObject*, PyObject* const* args, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  if (n < 3) return fail(PyExc_TypeError, "ints takes 3 arguments or more");
  const char* name = NAME(0);
  const Tensor* x = tensor(name, args[1]);
  const Tensor* y = x ? tensor("first", args[2]) : nullptr;
  if (!x || !y || !ints_of(name, *x, *y)) return nullptr;
  bool ok = n == 3 || x->dim() == n - 3;
  for (Py_ssize_t i = 3; ok && i < n; ++i) {
    const int64_t want = PyLong_AsLongLong(args[i]);
    if (PyErr_Occurred()) return nullptr;
    ok = x->size(i - 3) == want;
  }
  if (!ok) return fail(PyExc_ValueError, "%s has the wrong shape", name);
  return PyLong_FromVoidPtr(x->data_ptr());
  END_HANDLE_TH_ERRORS
}

// tokens(first, Hq, Hk, cu, cu_host) -> gdn_tokens (cu None: dense); None if the boundaries are
// not int32 tensors on the device and on the host as they are to be passed
PyObject* tokens(PyObject*, PyObject* const* args, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  if (n != 5) return fail(PyExc_TypeError, "tokens takes 5 arguments");
  const Tensor* x = tensor("first", args[0]);
  if (!x || !four("first", *x)) return nullptr;
  gdn_tokens t = {};
  t.B = (int32_t)x->size(0);
  t.T = (int32_t)x->size(1);
  t.d = (int32_t)x->size(3);
  if (x->size(0) != t.B || x->size(1) != t.T || x->size(3) != t.d)
    return fail(PyExc_ValueError, "too many tokens");
  t.Hq = (int32_t)PyLong_AsLong(args[1]);
  t.Hk = (int32_t)PyLong_AsLong(args[2]);
  if (PyErr_Occurred()) return nullptr;
  if (!dtype_of(*x, &t.dtype)) return fail(PyExc_TypeError, "%s must be float32 or bfloat16", "x");
  if (args[3] != Py_None) {
    if (!THPVariable_Check(args[3]) || !THPVariable_Check(args[4])) Py_RETURN_NONE;
    const Tensor &cu = THPVariable_Unpack(args[3]), &host = THPVariable_Unpack(args[4]);
    if (cu.scalar_type() != at::kInt || host.scalar_type() != at::kInt || cu.dim() != 1 ||
        host.dim() != 1 || cu.size(0) != host.size(0) || cu.size(0) < 1 ||
        cu.get_device() != x->get_device() || !host.device().is_cpu() || !cu.is_contiguous() ||
        !host.is_contiguous())
      Py_RETURN_NONE;
    t.num_seqs = (int32_t)(cu.size(0) - 1);
    t.cu_seqlens = cu.data_ptr<int32_t>();
    t.cu_seqlens_host = host.data_ptr<int32_t>();
  }
  return bytes(t);
  END_HANDLE_TH_ERRORS
}

// cache(first's name, first, k_pages, v_pages, table, kv_lens or None, sequences, skip or None) ->
// gdn_cache
PyObject* cache(PyObject*, PyObject* const* args, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  if (n != 8) return fail(PyExc_TypeError, "cache takes 8 arguments");
  const char* other = NAME(0);
  const Tensor* x = tensor(other, args[1]);
  const Tensor* k = x ? tensor("k_pages", args[2]) : nullptr;
  const Tensor* v = k ? tensor("v_pages", args[3]) : nullptr;
  const Tensor* table = v ? tensor("table", args[4]) : nullptr;
  if (!table || !four(other, *x)) return nullptr;
  const int64_t seqs = PyLong_AsLongLong(args[6]);
  if (PyErr_Occurred()) return nullptr;
  if (k->dim() != 4 || k->sizes() != v->sizes() || k->strides() != v->strides())
    return fail(PyExc_ValueError,
                "k_pages and v_pages must be [num_pages, Hk, page_size, d], alike in shape and "
                "strides");
  if (k->scalar_type() != x->scalar_type() || v->scalar_type() != x->scalar_type() ||
      k->get_device() != x->get_device() || v->get_device() != x->get_device())
    return fail(PyExc_ValueError, "k_pages and v_pages must have %s's dtype and device", other);
  if (k->size(3) != x->size(3) || k->stride(3) != 1)
    return fail(PyExc_ValueError, "k_pages and v_pages must have %s's d, contiguous", other);
  if (!ints_of("table", *table, *x)) return nullptr;
  if (table->dim() != 2 || table->size(0) != seqs)
    return PyErr_Format(PyExc_ValueError, "table must be int32 [%lld sequences, blocks]",
                        (long long)seqs);
  gdn_cache c = {};
  c.k = k->data_ptr();
  c.v = v->data_ptr();
  c.page_stride = k->stride(0);
  c.head_stride = k->stride(1);
  c.token_stride = k->stride(2);
  const int64_t most = 0x7fffffff;
  if (k->size(0) > most || k->size(2) > most || table->size(1) > most)
    return fail(PyExc_ValueError, "too many pages");
  c.num_pages = (int32_t)k->size(0);
  c.page_size = (int32_t)k->size(2);
  c.max_blocks = (int32_t)table->size(1);
  c.table = table->data_ptr<int32_t>();
  const struct {
    const char* name;
    PyObject* arg;
    const int32_t** to;
  } per_seq[] = {{"kv_lens", args[5], &c.kv_lens}, {"skip", args[7], &c.skip}};
  for (const auto& p : per_seq) {
    if (p.arg == Py_None) continue;
    const Tensor* y = tensor(p.name, p.arg);
    if (!y || !ints_of(p.name, *y, *x)) return nullptr;
    if (y->dim() != 1 || y->size(0) != seqs)
      return PyErr_Format(PyExc_ValueError, "%s must be int32 [%lld sequences]", p.name,
                          (long long)seqs);
    *p.to = y->data_ptr<int32_t>();
  }
  return bytes(c);
  END_HANDLE_TH_ERRORS
}

// rotary(turns, layout, scale, first) -> gdn_rotary
PyObject* rotary(PyObject*, PyObject* const* args, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  if (n != 4) return fail(PyExc_TypeError, "rotary takes 4 arguments");
  const Tensor* t = tensor("rotary.turns", args[0]);
  const Tensor* x = t ? tensor("first", args[3]) : nullptr;
  if (!x) return nullptr;
  if (t->get_device() != x->get_device() || t->scalar_type() != at::kDouble || t->dim() != 1 ||
      !t->is_contiguous() || t->size(0) > 0x3fffffff)
    return fail(PyExc_ValueError,
                "rotary.turns must be contiguous float64 [rot / 2] on the call's device");
  gdn_rotary r = {};
  r.rot = (int32_t)(2 * t->size(0));
  r.layout = (int32_t)PyLong_AsLong(args[1]);
  r.scale = (float)PyFloat_AsDouble(args[2]);
  if (PyErr_Occurred()) return nullptr;
  r.turns = t->data_ptr<double>();
  return bytes(r);
  END_HANDLE_TH_ERRORS
}

PyMethodDef methods[] = {
    {"first", (PyCFunction)(void*)first, METH_FASTCALL, nullptr},
    {"rows", (PyCFunction)(void*)rows, METH_FASTCALL, nullptr},
    {"like", (PyCFunction)(void*)like, METH_FASTCALL, nullptr},
    {"book", (PyCFunction)(void*)book, METH_FASTCALL, nullptr},
    {"pool", (PyCFunction)(void*)pool, METH_FASTCALL, nullptr},
    {"ints", (PyCFunction)(void*)ints, METH_FASTCALL, nullptr},
    {"tokens", (PyCFunction)(void*)tokens, METH_FASTCALL, nullptr},
    {"cache", (PyCFunction)(void*)cache, METH_FASTCALL, nullptr},
    {"rotary", (PyCFunction)(void*)rotary, METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_paged_binding", nullptr, -1, methods,
                      nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__paged_binding() { return PyModule_Create(&module); }
