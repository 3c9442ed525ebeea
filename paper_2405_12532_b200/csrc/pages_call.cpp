// The paged cache's calls from Python without what ctypes and the interpreter take for them (4 to 10 us a call, as long as a decode
// step's kernels run): arguments are taken out of the tensors here. Marshalling only, like binding.py, which keeps every
// check and message: what is not plainly right here (None is returned then) goes its way.
#include <Python.h>

#include <ATen/ATen.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include "pyr.h"

namespace {

struct Calls {
  decltype(&pyr_pages_attn) attn;
  decltype(&pyr_pages_attn_blocks) attn_blocks;
  decltype(&pyr_pages_select) select;
  decltype(&pyr_pages_append) append;
  decltype(&pyr_pages_read) read;
};
Calls g_calls{};

struct Cache {
  pyr_pages_t* handle;
  int device;
  int64_t heads, dim;
};

Cache* cache_of(PyObject* x) { return static_cast<Cache*>(PyCapsule_GetPointer(x, "pyr_pages")); }

// A [n, rows, heads, D] tensor.
struct Rows {
  const at::Tensor* t = nullptr;
  int64_t n = 0, rows = 0, heads = 0, sb = 0, sn = 0, sh = 0;
  int dtype = -1;
  void* at = nullptr;
};
bool rows_of(const at::Tensor& t, const Cache& c, Rows* r) {
  if (t.dim() != 4 || !t.is_cuda() || t.get_device() != c.device || t.size(3) != c.dim || t.stride(3) != 1) return false;
  const auto type = t.scalar_type();
  r->dtype = type == at::kBFloat16 ? PYR_BF16 : type == at::kFloat ? PYR_F32 : -1;
  if (r->dtype < 0 || t.size(0) > INT32_MAX || t.size(1) > INT32_MAX || t.size(2) > INT32_MAX) return false;
  r->t = &t;
  r->n = t.size(0); r->rows = t.size(1); r->heads = t.size(2);
  r->sb = t.stride(0); r->sn = t.stride(1); r->sh = t.stride(2);
  r->at = t.data_ptr();
  return true;
}
bool rows_of(PyObject* x, const Cache& c, Rows* r) { return THPVariable_Check(x) && rows_of(THPVariable_Unpack(x), c, r); }
// Keys and values: alike in shape, type and strides.
bool pair_of(PyObject* k, PyObject* v, const Cache& c, Rows* a, Rows* b) {
  return rows_of(k, c, a) && rows_of(v, c, b) && a->heads == c.heads && a->t->sizes() == b->t->sizes() && a->dtype == b->dtype &&
         a->t->strides() == b->t->strides();
}
// n contiguous int32 entries, or None.
bool ids_of(PyObject* x, int64_t n, const Cache& c, const int32_t** ids) {
  *ids = nullptr;
  if (x == Py_None) return true;
  if (!THPVariable_Check(x)) return false;
  const at::Tensor& t = THPVariable_Unpack(x);
  if (t.scalar_type() != at::kInt || t.dim() != 1 || t.size(0) != n || !t.is_cuda() || t.get_device() != c.device || !t.is_contiguous()) return false;
  *ids = static_cast<const int32_t*>(t.data_ptr());
  return true;
}
// A contiguous int32 tensor [n, groups, rows].
bool index_of(PyObject* x, int64_t n, const Cache& c, const int32_t** at, int64_t* groups, int64_t* rows) {
  if (!THPVariable_Check(x)) return false;
  const at::Tensor& t = THPVariable_Unpack(x);
  if (t.scalar_type() != at::kInt || t.dim() != 3 || t.size(0) != n || !t.is_cuda() || t.get_device() != c.device || !t.is_contiguous()) return false;
  *at = static_cast<const int32_t*>(t.data_ptr());
  *groups = t.size(1); *rows = t.size(2);
  return *groups <= INT32_MAX && *rows <= INT32_MAX;
}
// The stream to launch on, if the cache's device is the current one.
bool stream_of(const Cache& c, void** stream) {
  if (c10::cuda::current_device() != c.device) return false;
  *stream = c10::cuda::getCurrentCUDAStream(c.device).stream();
  return true;
}
// A result tensor: the one that was passed, or a new one in *mine.
const at::Tensor* result_of(PyObject* x, const at::Tensor& like, at::Tensor* mine) {
  if (x != Py_None) return THPVariable_Check(x) ? &THPVariable_Unpack(x) : nullptr;
  *mine = at::empty_like(like);
  return mine;
}
PyObject* given_or(PyObject* x, at::Tensor&& mine) {
  if (x != Py_None) { Py_INCREF(x); return x; }
  return THPVariable_Wrap(std::move(mine));
}
// None: the caller's own path; a number: a status that is not 0.
PyObject* status_of(pyr_status_t st) { return PyLong_FromLong(st); }

// C++ exceptions become those that torch makes of them (out of memory: torch.OutOfMemoryError).
template <class F>
PyObject* guarded(F f) {
  HANDLE_TH_ERRORS
  at::AutoDispatchBelowADInplaceOrView below;
  return f();
  END_HANDLE_TH_ERRORS
}
// The library's call without the interpreter's lock, as through ctypes: a launch can wait for room in the queue, and what it waits for for a
// host function that wants the lock.
template <class F>
pyr_status_t unlocked(F f) {
  pyr_status_t st;
  Py_BEGIN_ALLOW_THREADS
  st = f();
  Py_END_ALLOW_THREADS
  return st;
}
#define PYR_ARGS(count) if (n_args != count) { PyErr_SetString(PyExc_TypeError, "wrong number of arguments"); return nullptr; } \
                        Cache* const c = cache_of(args[0]); if (!c) return nullptr

// cache, q, lists, slots (None: all rows), out (None: a new one), lse, softmax_scale -> out, or (out, lse)
PyObject* attn(PyObject*, PyObject* const* args, Py_ssize_t n_args) {
  PYR_ARGS(7);
  return guarded([&]() -> PyObject* {
    Rows q, o;
    const int32_t* lists;
    at::Tensor mine, lse;
    const double scale = PyFloat_AsDouble(args[6]);
    if (PyErr_Occurred()) { PyErr_Clear(); Py_RETURN_NONE; }
    void* stream;
    if (!rows_of(args[1], *c, &q) || !ids_of(args[2], q.n, *c, &lists) || !stream_of(*c, &stream)) Py_RETURN_NONE;
    const int32_t* slots = nullptr;
    int64_t n_slots = 0;
    if (args[3] != Py_None) {
      if (!THPVariable_Check(args[3])) Py_RETURN_NONE;
      const at::Tensor& s = THPVariable_Unpack(args[3]);
      if (s.scalar_type() != at::kInt || s.dim() != 4 || s.size(0) != q.n || s.size(1) != q.rows || s.size(2) != c->heads || s.size(3) > INT32_MAX ||
          !s.is_cuda() || s.get_device() != c->device || !s.is_contiguous())
        Py_RETURN_NONE;
      slots = static_cast<const int32_t*>(s.data_ptr());
      n_slots = s.size(3);
    }
    const at::Tensor* out = result_of(args[4], *q.t, &mine);
    if (!out || !rows_of(*out, *c, &o) || out->sizes() != q.t->sizes() || o.dtype != q.dtype) Py_RETURN_NONE;
    const int stats = PyObject_IsTrue(args[5]);
    if (stats < 0) { PyErr_Clear(); Py_RETURN_NONE; }
    if (stats) lse = at::empty({q.n, q.heads, q.rows}, q.t->options().dtype(at::kFloat));
    float* const l = stats ? static_cast<float*>(lse.data_ptr()) : nullptr;
    const bool all = args[3] == Py_None;
    const pyr_status_t st = unlocked([&] {
      return all ? g_calls.attn(c->handle, lists, (int32_t)q.n, q.at, q.sb, q.sn, q.sh, o.at, o.sb, o.sn, o.sh, l, (int32_t)q.rows, (int32_t)q.heads,
                                q.dtype, (float)scale, stream)
                 : g_calls.attn_blocks(c->handle, lists, (int32_t)q.n, slots, (int32_t)n_slots, q.at, q.sb, q.sn, q.sh, o.at, o.sb, o.sn, o.sh, l,
                                       (int32_t)q.rows, (int32_t)q.heads, q.dtype, (float)scale, stream);
    });
    if (st != PYR_OK) return status_of(st);
    PyObject* first = given_or(args[4], std::move(mine));
    if (!stats || !first) return first;
    PyObject* second = THPVariable_Wrap(std::move(lse));
    PyObject* both = second ? PyTuple_Pack(2, first, second) : nullptr;
    Py_DECREF(first);
    Py_XDECREF(second);
    return both;
  });
}

// cache, q, n_slots, lists, keep_first, keep_last, out (None: a new one) -> slots
PyObject* select(PyObject*, PyObject* const* args, Py_ssize_t n_args) {
  PYR_ARGS(7);
  return guarded([&]() -> PyObject* {
    Rows q;
    const int32_t* lists;
    const long n_slots = PyLong_AsLong(args[2]), first = PyLong_AsLong(args[4]), last = PyLong_AsLong(args[5]);
    if (PyErr_Occurred()) { PyErr_Clear(); Py_RETURN_NONE; }
    void* stream;
    if (n_slots < 1 || n_slots > INT32_MAX || first < 0 || first > n_slots || last < 0 || last > n_slots || !rows_of(args[1], *c, &q) ||
        !ids_of(args[3], q.n, *c, &lists) || !stream_of(*c, &stream))
      Py_RETURN_NONE;
    at::Tensor mine;
    const at::Tensor* out = &mine;
    if (args[6] == Py_None) {
      mine = at::empty({q.n, q.rows, c->heads, n_slots}, q.t->options().dtype(at::kInt));
    } else {
      if (!THPVariable_Check(args[6])) Py_RETURN_NONE;
      out = &THPVariable_Unpack(args[6]);
      if (out->scalar_type() != at::kInt || out->dim() != 4 || out->size(0) != q.n || out->size(1) != q.rows || out->size(2) != c->heads ||
          out->size(3) != n_slots || !out->is_cuda() || out->get_device() != c->device || !out->is_contiguous())
        Py_RETURN_NONE;
    }
    int32_t* const slots = static_cast<int32_t*>(out->data_ptr());
    const pyr_status_t st = unlocked([&] {
      return g_calls.select(c->handle, lists, (int32_t)q.n, q.at, q.sb, q.sn, q.sh, (int32_t)q.rows, (int32_t)q.heads, q.dtype, slots,
                            (int32_t)n_slots, (int32_t)first, (int32_t)last, stream);
    });
    return st != PYR_OK ? status_of(st) : given_or(args[6], std::move(mine));
  });
}

// cache, k, v, lists, first, pos, rope, q, q_out (None: a new one), idx, counts -> q_out, or 0 without queries
PyObject* append(PyObject*, PyObject* const* args, Py_ssize_t n_args) {
  PYR_ARGS(11);
  return guarded([&]() -> PyObject* {
    Rows k, v, q, o;
    pyr_append_t x{};
    void* stream;
    if (!pair_of(args[1], args[2], *c, &k, &v) || !ids_of(args[3], k.n, *c, &x.lists) || !ids_of(args[4], k.n, *c, &x.first) ||
        !ids_of(args[10], k.n, *c, &x.counts) || !stream_of(*c, &stream))
      Py_RETURN_NONE;
    int64_t groups = 1, rows = k.rows;
    if (args[9] != Py_None) {
      if (!index_of(args[9], k.n, *c, &x.idx, &groups, &rows)) Py_RETURN_NONE;
      x.idx_stride = k.n > 1 ? groups * rows : 0;
    }
    if (args[5] != Py_None) {
      int64_t pos_groups, pos_rows;
      if (!index_of(args[5], k.n, *c, &x.pos, &pos_groups, &pos_rows) || pos_groups != groups || pos_rows != rows || !THPVariable_Check(args[6]))
        Py_RETURN_NONE;
      const at::Tensor& rope = THPVariable_Unpack(args[6]);
      if (rope.scalar_type() != at::kFloat || rope.dim() != 2 || rope.size(1) != c->dim || rope.size(0) > INT32_MAX || !rope.is_cuda() ||
          rope.get_device() != c->device || !rope.is_contiguous())
        Py_RETURN_NONE;
      x.pos_stride = k.n > 1 ? groups * rows : 0;
      x.rope = static_cast<const float*>(rope.data_ptr());
      x.n_pos = (int32_t)rope.size(0);
    }
    at::Tensor mine;
    if (args[7] != Py_None) {
      if (!rows_of(args[7], *c, &q) || q.n != k.n || q.rows != rows || q.dtype != k.dtype) Py_RETURN_NONE;
      const at::Tensor* out = result_of(args[8], *q.t, &mine);
      if (!out || !rows_of(*out, *c, &o) || out->sizes() != q.t->sizes() || o.dtype != q.dtype) Py_RETURN_NONE;
      x.q = q.at; x.q_out = o.at; x.n_q_heads = (int32_t)q.heads;
      x.q_stride_b = q.sb; x.q_stride_n = q.sn; x.q_stride_h = q.sh;
      x.o_stride_b = o.sb; x.o_stride_n = o.sn; x.o_stride_h = o.sh;
    } else if (args[8] != Py_None) {
      Py_RETURN_NONE;
    }
    x.k = k.at; x.v = v.at;
    x.stride_b = k.sb; x.stride_n = k.sn; x.stride_h = k.sh;
    x.n = (int32_t)k.n; x.src_rows = (int32_t)k.rows; x.dtype = k.dtype; x.idx_groups = (int32_t)groups; x.n_rows = (int32_t)rows;
    const pyr_status_t st = unlocked([&] { return g_calls.append(c->handle, &x, stream); });
    return st != PYR_OK || args[7] == Py_None ? status_of(st) : given_or(args[8], std::move(mine));
  });
}

// cache, k, v, lists, first, counts -> 0
PyObject* read(PyObject*, PyObject* const* args, Py_ssize_t n_args) {
  PYR_ARGS(6);
  return guarded([&]() -> PyObject* {
    Rows k, v;
    const int32_t *lists, *first, *counts;
    void* stream;
    if (!pair_of(args[1], args[2], *c, &k, &v) || !ids_of(args[3], k.n, *c, &lists) || !ids_of(args[4], k.n, *c, &first) ||
        !ids_of(args[5], k.n, *c, &counts) || !stream_of(*c, &stream))
      Py_RETURN_NONE;
    return status_of(unlocked([&] {
      return g_calls.read(c->handle, lists, (int32_t)k.n, first, k.at, v.at, k.sb, k.sn, k.sh, k.dtype, counts, (int32_t)k.rows, stream);
    }));
  });
}

// Addresses of the library's functions, in the order of Calls.
PyObject* setup(PyObject*, PyObject* const* args, Py_ssize_t n_args) {
  void* at[5];
  if (n_args != 5) { PyErr_SetString(PyExc_TypeError, "five addresses"); return nullptr; }
  for (int i = 0; i < 5; ++i) at[i] = PyLong_AsVoidPtr(args[i]);
  if (PyErr_Occurred()) return nullptr;
  g_calls.attn = reinterpret_cast<decltype(g_calls.attn)>(at[0]);
  g_calls.attn_blocks = reinterpret_cast<decltype(g_calls.attn_blocks)>(at[1]);
  g_calls.select = reinterpret_cast<decltype(g_calls.select)>(at[2]);
  g_calls.append = reinterpret_cast<decltype(g_calls.append)>(at[3]);
  g_calls.read = reinterpret_cast<decltype(g_calls.read)>(at[4]);
  Py_RETURN_NONE;
}
// handle, device, KV heads, head_dim -> what the calls take first
PyObject* cache(PyObject*, PyObject* const* args, Py_ssize_t n_args) {
  if (n_args != 4) { PyErr_SetString(PyExc_TypeError, "handle, device, heads, dimensions"); return nullptr; }
  Cache x{static_cast<pyr_pages_t*>(PyLong_AsVoidPtr(args[0])), (int)PyLong_AsLong(args[1]), PyLong_AsLong(args[2]), PyLong_AsLong(args[3])};
  if (PyErr_Occurred()) return nullptr;
  return PyCapsule_New(new Cache(x), "pyr_pages", [](PyObject* p) { delete static_cast<Cache*>(PyCapsule_GetPointer(p, "pyr_pages")); });
}

// (the type that CPython's table has for every calling convention)
template <class F>
PyCFunction entry(F f) { return reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f)); }
PyMethodDef g_methods[] = {{"setup", entry(setup), METH_FASTCALL, nullptr},
                           {"cache", entry(cache), METH_FASTCALL, nullptr},
                           {"attn", entry(attn), METH_FASTCALL, nullptr},
                           {"select", entry(select), METH_FASTCALL, nullptr},
                           {"append", entry(append), METH_FASTCALL, nullptr},
                           {"read", entry(read), METH_FASTCALL, nullptr},
                           {nullptr, nullptr, 0, nullptr}};
PyModuleDef g_module = {PyModuleDef_HEAD_INIT, "_pages_call", nullptr, -1, g_methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__pages_call() { return PyModule_Create(&g_module); }
