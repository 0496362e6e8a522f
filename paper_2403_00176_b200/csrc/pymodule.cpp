// CPython module `_sod2calls`: the calls a program makes for every batch (bind, plan, run, output shapes, destroy), with
// their arguments taken straight from Python lists.  Through ctypes, building the argument arrays cost more than the
// calls themselves (the smallest fused group: 6 of 13 us a pass).  Marshalling only: every function hands its arguments
// to the C ABI of libsod2.so, releases the interpreter lock around it and returns its status.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <climits>
#include <cstdint>
#include <cstring>
#include <new>

#include "../../include/sod2.h"

namespace {

// Small argument arrays live on the stack.  They start out as zeros: a missing address is a null address.
template <class T, int N>
struct Buf {
  T local[N] = {};
  T* p = local;
  bool reserve(Py_ssize_t n) {
    if (n <= N) return true;
    p = new (std::nothrow) T[n]();
    if (!p) { p = local; PyErr_NoMemory(); return false; }
    return true;
  }
  ~Buf() { if (p != local) delete[] p; }
};

bool as_i64(PyObject* o, int64_t* out) {
  if (PyLong_CheckExact(o)) {
    *out = PyLong_AsLongLong(o);
  } else {
    PyObject* l = PyNumber_Long(o);
    if (!l) return false;
    *out = PyLong_AsLongLong(l);
    Py_DECREF(l);
  }
  return !(*out == -1 && PyErr_Occurred());
}

bool as_ptr(PyObject* o, void** out) {
  if (o == Py_None) { *out = nullptr; return true; }
  *out = PyLong_AsVoidPtr(o);
  return !(*out == nullptr && PyErr_Occurred());
}
// An entry of a list of addresses may also be a ctypes.c_void_p.
bool as_entry(PyObject* o, void** out) {
  if (o == Py_None || PyLong_Check(o)) return as_ptr(o, out);
  PyObject* v = PyObject_GetAttrString(o, "value");
  if (!v) {
    PyErr_Format(PyExc_TypeError, "an address is wanted, got %.100s", Py_TYPE(o)->tp_name);
    return false;
  }
  const bool ok = as_ptr(v, out);
  Py_DECREF(v);
  return ok;
}

// At least `least` entries: what the list lacks is null, and refused by the call.
template <int N>
bool as_ptrs(PyObject* seq, Buf<void*, N>* out, Py_ssize_t least) {
  PyObject* f = PySequence_Fast(seq, "a sequence of addresses is wanted");
  if (!f) return false;
  const Py_ssize_t n = PySequence_Fast_GET_SIZE(f);
  bool ok = out->reserve(n > least ? n : least);
  for (Py_ssize_t i = 0; ok && i < n; ++i) ok = as_entry(PySequence_Fast_GET_ITEM(f, i), &out->p[i]);
  Py_DECREF(f);
  return ok;
}

bool want(Py_ssize_t got, Py_ssize_t n) {
  if (got == n) return true;
  PyErr_Format(PyExc_TypeError, "%zd arguments are wanted, got %zd", n, got);
  return false;
}

// bind(graph, names, rows) -> (status, binding)
PyObject* py_bind(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (!want(n, 3)) return nullptr;
  void* g;
  if (!as_ptr(a[0], &g)) return nullptr;
  PyObject* names = PySequence_Fast(a[1], "a sequence of symbol names is wanted");
  if (!names) return nullptr;
  PyObject* rows = PySequence_Fast(a[2], "a sequence of rows is wanted");
  if (!rows) { Py_DECREF(names); return nullptr; }
  const Py_ssize_t n_sym = PySequence_Fast_GET_SIZE(names), n_req = PySequence_Fast_GET_SIZE(rows);
  Buf<const char*, 16> nm;
  Buf<int64_t, 128> val;
  bool ok = nm.reserve(n_sym) && val.reserve(n_sym * n_req);
  for (Py_ssize_t i = 0; ok && i < n_sym; ++i) ok = (nm.p[i] = PyUnicode_AsUTF8(PySequence_Fast_GET_ITEM(names, i))) != nullptr;
  for (Py_ssize_t r = 0; ok && r < n_req; ++r) {
    PyObject* row = PySequence_Fast(PySequence_Fast_GET_ITEM(rows, r), "a row of symbol values is wanted");
    if (!row) { ok = false; break; }
    if (PySequence_Fast_GET_SIZE(row) != n_sym) {
      PyErr_Format(PyExc_ValueError, "request %zd has %zd values for %zd symbols", r, PySequence_Fast_GET_SIZE(row), n_sym);
      ok = false;
    }
    for (Py_ssize_t i = 0; ok && i < n_sym; ++i) ok = as_i64(PySequence_Fast_GET_ITEM(row, i), &val.p[r * n_sym + i]);
    Py_DECREF(row);
  }
  PyObject* res = nullptr;
  if (ok) {
    sod2_binding* b = nullptr;
    int st;
    Py_BEGIN_ALLOW_THREADS
    st = sod2_bind_dims(static_cast<sod2_graph*>(g), static_cast<int>(n_req), static_cast<int>(n_sym), nm.p, val.p, &b);
    Py_END_ALLOW_THREADS
    res = Py_BuildValue("iN", st, PyLong_FromVoidPtr(b));
  }
  Py_DECREF(names);
  Py_DECREF(rows);
  return res;
}

// plan(graph, binding) -> (status, plan, arena bytes)
PyObject* py_plan(PyObject*, PyObject* const* a, Py_ssize_t n) {
  void *g, *b;
  if (!want(n, 2) || !as_ptr(a[0], &g) || !as_ptr(a[1], &b)) return nullptr;
  sod2_plan_t* p = nullptr;
  size_t bytes = 0;
  int st;
  Py_BEGIN_ALLOW_THREADS
  st = sod2_plan(static_cast<sod2_graph*>(g), static_cast<sod2_binding*>(b), &p, &bytes);
  Py_END_ALLOW_THREADS
  return Py_BuildValue("iNn", st, PyLong_FromVoidPtr(p), static_cast<Py_ssize_t>(bytes));
}

// run(how, plan, inputs, outputs, arena, arena bytes, stream, info) -> status; info: a writable buffer of sod2_run_info
PyObject* py_run(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (!want(n, 8)) return nullptr;
  int64_t how, bytes;
  void *p, *arena, *stream;
  Buf<void*, 64> in, out;
  int n_in = 0, n_out = 0;
  if (!as_i64(a[0], &how) || !as_ptr(a[1], &p)) return nullptr;
  sod2_plan_io_counts(static_cast<sod2_plan_t*>(p), &n_in, &n_out);
  if (!as_ptrs(a[2], &in, n_in) || !as_ptrs(a[3], &out, n_out) || !as_ptr(a[4], &arena) ||
      !as_i64(a[5], &bytes) || !as_ptr(a[6], &stream))
    return nullptr;
  Py_buffer info;
  if (PyObject_GetBuffer(a[7], &info, PyBUF_WRITABLE) != 0) return nullptr;
  if (info.len < static_cast<Py_ssize_t>(sizeof(sod2_run_info))) {
    PyBuffer_Release(&info);
    PyErr_SetString(PyExc_ValueError, "the run-info buffer is too small");
    return nullptr;
  }
  auto* fn = how == 0 ? sod2_run : how == 1 ? sod2_run_graph : sod2_run_exact;
  int st;
  Py_BEGIN_ALLOW_THREADS
  st = fn(static_cast<sod2_plan_t*>(p), in.p, out.p, arena, static_cast<size_t>(bytes), stream, static_cast<sod2_run_info*>(info.buf));
  Py_END_ALLOW_THREADS
  PyBuffer_Release(&info);
  return PyLong_FromLong(st);
}

// output_shape(plan, arena, stream, request, output) -> list of extents, or the status if it is not 0
PyObject* py_output_shape(PyObject*, PyObject* const* a, Py_ssize_t n) {
  void *p, *arena, *stream;
  int64_t r, o;
  if (!want(n, 5) || !as_ptr(a[0], &p) || !as_ptr(a[1], &arena) || !as_ptr(a[2], &stream) || !as_i64(a[3], &r) || !as_i64(a[4], &o)) return nullptr;
  int64_t dims[16];
  int rank = 0, st;
  Py_BEGIN_ALLOW_THREADS
  st = sod2_run_output_shape(static_cast<sod2_plan_t*>(p), arena, stream, static_cast<int>(r), static_cast<int>(o), dims, &rank);
  Py_END_ALLOW_THREADS
  if (st) return PyLong_FromLong(st);
  PyObject* l = PyList_New(rank);
  for (int i = 0; l && i < rank; ++i) PyList_SET_ITEM(l, i, PyLong_FromLongLong(dims[i]));
  return l;
}

PyObject* py_binding_destroy(PyObject*, PyObject* h) {
  void* p;
  if (!as_ptr(h, &p)) return nullptr;
  sod2_binding_destroy(static_cast<sod2_binding*>(p));
  Py_RETURN_NONE;
}
PyObject* py_plan_destroy(PyObject*, PyObject* h) {
  void* p;
  if (!as_ptr(h, &p)) return nullptr;
  Py_BEGIN_ALLOW_THREADS
  sod2_plan_destroy(static_cast<sod2_plan_t*>(p));
  Py_END_ALLOW_THREADS
  Py_RETURN_NONE;
}

// Arguments of the serving calls by a pattern: i an integer or an address (None: 0), d a number, 3 / 4 a tuple of an address and its
// strides (None: absent).  Strides of absent tensors are zero.
struct Arg { int64_t v[4] = {}; double d = 0; bool there = false; };
bool parse(PyObject* const* a, Py_ssize_t n, const char* pattern, Arg* out) {
  if (!want(n, static_cast<Py_ssize_t>(std::strlen(pattern)))) return false;
  for (Py_ssize_t i = 0; i < n; ++i) {
    const char kind = pattern[i];
    if (kind == 'd') {
      out[i].d = PyFloat_AsDouble(a[i]);
      if (out[i].d == -1.0 && PyErr_Occurred()) return false;
    } else if (a[i] == Py_None) {
    } else if (kind == 'i') {
      if (!as_i64(a[i], &out[i].v[0])) return false;
    } else {
      const Py_ssize_t m = kind - '0';
      if (!PyTuple_Check(a[i]) || PyTuple_GET_SIZE(a[i]) != m) {
        PyErr_Format(PyExc_TypeError, "argument %zd: a tuple of an address and %zd strides is wanted", i, m - 1);
        return false;
      }
      for (Py_ssize_t j = 0; j < m; ++j) if (!as_i64(PyTuple_GET_ITEM(a[i], j), &out[i].v[j])) return false;
      out[i].there = true;
    }
  }
  return true;
}
template <class T> T* addr(const Arg& a) { return reinterpret_cast<T*>(static_cast<intptr_t>(a.v[0])); }
// An int of the C interface: what does not fit becomes a value that every call refuses.
int narrow(const Arg& a) { return a.v[0] < INT_MIN || a.v[0] > INT_MAX ? INT_MIN : static_cast<int>(a.v[0]); }
struct RowsArg {
  sod2_rows r;
  bool there;
  explicit RowsArg(const Arg& a) : r{addr<void>(a), a.v[1], a.v[2]}, there(a.there) {}
  const sod2_rows* get() const { return there ? &r : nullptr; }
};
struct PagesArg {
  sod2_pages r;
  bool there;
  explicit PagesArg(const Arg& a) : r{addr<void>(a), a.v[1], a.v[2], a.v[3]}, there(a.there) {}
  const sod2_pages* get() const { return there ? &r : nullptr; }
};

// page_tables(sod2_page_tables' arguments) -> status
PyObject* py_page_tables(PyObject*, PyObject* const* a, Py_ssize_t n) {
  Arg x[18];
  if (!parse(a, n, "iiiiiiiiiiiiiiiiii", x)) return nullptr;
  int st;
  Py_BEGIN_ALLOW_THREADS
  st = sod2_page_tables(narrow(x[0]), x[1].v[0], narrow(x[2]), addr<int32_t>(x[3]), addr<int32_t>(x[4]), addr<int32_t>(x[5]), x[6].v[0], addr<int32_t>(x[7]),
                        addr<int32_t>(x[8]), x[9].v[0], x[10].v[0], addr<int32_t>(x[11]), addr<int32_t>(x[12]), addr<int64_t>(x[13]), addr<int32_t>(x[14]),
                        addr<int32_t>(x[15]), addr<int32_t>(x[16]), addr<void>(x[17]));
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(st);
}
// rope_store(dtype, tokens, heads, kv heads, dim, pairs, freq, axis, adjacent, positions, axis stride, q, q_out, k, k_out, v, k cache, v cache,
// pages, page size, slots, status, stream) -> status
PyObject* py_rope_store(PyObject*, PyObject* const* a, Py_ssize_t n) {
  Arg x[23];
  if (!parse(a, n, "iiiiiiiiiii3333344iiiii", x)) return nullptr;
  const RowsArg q(x[11]), qo(x[12]), k(x[13]), ko(x[14]), v(x[15]);
  const PagesArg kc(x[16]), vc(x[17]);
  int st;
  Py_BEGIN_ALLOW_THREADS
  st = sod2_rope_store(narrow(x[0]), x[1].v[0], narrow(x[2]), narrow(x[3]), narrow(x[4]), narrow(x[5]), addr<double>(x[6]), addr<uint8_t>(x[7]),
                       narrow(x[8]), addr<int32_t>(x[9]), x[10].v[0], q.get(), qo.get(), k.get(), ko.get(), v.get(), kc.get(), vc.get(), x[18].v[0],
                       narrow(x[19]), addr<int64_t>(x[20]), addr<int32_t>(x[21]), addr<void>(x[22]));
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(st);
}
// attention_prompt(sod2_attention_prompt's arguments) -> status
PyObject* py_attention_prompt(PyObject*, PyObject* const* a, Py_ssize_t n) {
  Arg x[16];
  if (!parse(a, n, "iiiiii3333idiiii", x)) return nullptr;
  const RowsArg q(x[6]), k(x[7]), v(x[8]), o(x[9]);
  int st;
  Py_BEGIN_ALLOW_THREADS
  st = sod2_attention_prompt(narrow(x[0]), narrow(x[1]), x[2].v[0], narrow(x[3]), narrow(x[4]), narrow(x[5]), q.get(), k.get(), v.get(), o.get(),
                             addr<int32_t>(x[10]), static_cast<float>(x[11].d), addr<void>(x[12]), x[13].v[0] < 0 ? 0 : static_cast<size_t>(x[13].v[0]),
                             addr<int32_t>(x[14]), addr<void>(x[15]));
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(st);
}
// attention_paged(sod2_attention_paged's arguments) -> status
PyObject* py_attention_paged(PyObject*, PyObject* const* a, Py_ssize_t n) {
  Arg x[23];
  if (!parse(a, n, "iiiiiii33ii44iiiiidiiii", x)) return nullptr;
  const RowsArg q(x[7]), o(x[8]);
  const PagesArg kc(x[11]), vc(x[12]);
  int st;
  Py_BEGIN_ALLOW_THREADS
  st = sod2_attention_paged(narrow(x[0]), narrow(x[1]), x[2].v[0], x[3].v[0], narrow(x[4]), narrow(x[5]), narrow(x[6]), q.get(), o.get(),
                            addr<int32_t>(x[9]), addr<int32_t>(x[10]), kc.get(), vc.get(), x[13].v[0], narrow(x[14]), addr<int32_t>(x[15]), x[16].v[0],
                            x[17].v[0], static_cast<float>(x[18].d), addr<void>(x[19]), x[20].v[0] < 0 ? 0 : static_cast<size_t>(x[20].v[0]),
                            addr<int32_t>(x[21]), addr<void>(x[22]));
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(st);
}

#define FAST(f) reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)(void)>(f))
PyMethodDef methods[] = {
    {"bind", FAST(py_bind), METH_FASTCALL, "sod2_bind_dims"},
    {"plan", FAST(py_plan), METH_FASTCALL, "sod2_plan"},
    {"run", FAST(py_run), METH_FASTCALL, "sod2_run (0), sod2_run_graph (1), sod2_run_exact (2)"},
    {"output_shape", FAST(py_output_shape), METH_FASTCALL, "sod2_run_output_shape"},
    {"page_tables", FAST(py_page_tables), METH_FASTCALL, "sod2_page_tables"},
    {"rope_store", FAST(py_rope_store), METH_FASTCALL, "sod2_rope_store"},
    {"attention_prompt", FAST(py_attention_prompt), METH_FASTCALL, "sod2_attention_prompt"},
    {"attention_paged", FAST(py_attention_paged), METH_FASTCALL, "sod2_attention_paged"},
    {"binding_destroy", py_binding_destroy, METH_O, "sod2_binding_destroy"},
    {"plan_destroy", py_plan_destroy, METH_O, "sod2_plan_destroy"},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_sod2calls", "per-batch calls into libsod2.so", -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__sod2calls(void) { return PyModule_Create(&module); }
