// Python's side of the operators over a cache in pages: checks that tensors go together, and the call of the C entry point.
// A call of these operators takes the GPU 3 to 20 us; reading 10 tensors' shapes and strides attribute by attribute in Python
// took 8 to 13 us a call, and its caller waits for that. Here the tensors are read as what they are: 1.5 to 3 us.
// Every function takes the arguments of its Python namesake in order, then the device that they must lie on (-1: none, a machine
// without a GPU) and the stream; it returns the entry point's status, or -1 where the tensors do not go together, and Python says why.
#include <Python.h>
#include <dlfcn.h>
#include <torch/csrc/autograd/python_variable.h>

#include <algorithm>

#include "fsx.h"

namespace {

decltype(&fsx_rotary) f_rotary;
decltype(&fsx_paged_attention) f_paged_attention;
decltype(&fsx_page_bounds) f_page_bounds;
decltype(&fsx_page_select) f_page_select;
decltype(&fsx_pages_step) f_pages_step;
decltype(&fsx_pages_compact) f_pages_compact;
decltype(&fsx_pages_copy) f_pages_copy;

using Tensor = at::Tensor;
using c10::ScalarType;

// The arguments of a call, taken one after another
class Args {
 public:
  Args(PyObject* const* at, Py_ssize_t n, Py_ssize_t want) : at_(at), good(n == want) {
    if (good) {
      device_ = PyLong_AsLong(at[n - 2]);
      stream = PyLong_AsVoidPtr(at[n - 1]);
      if (PyErr_Occurred()) good = false;
    }
  }
  // a tensor on the call's device; `optional`: NULL for None
  const Tensor* tensor(bool optional = false) {
    if (!good) return nullptr;
    PyObject* o = *at_++;
    if (o == Py_None && optional) return nullptr;
    if (!THPVariable_Check(o)) {
      good = false;
      return nullptr;
    }
    const Tensor& t = THPVariable_Unpack(o);
    if (t.layout() != c10::kStrided || (t.is_cuda() ? t.get_device() : t.is_cpu() ? -1 : -2) != device_) good = false;
    if (good && t.numel() > 0 && t.data_ptr() == nullptr) good = false;  // throws where there is no memory behind the tensor
    return &t;
  }
  // the status word
  const Tensor* word() {
    const Tensor* t = tensor();
    if (good && (t->scalar_type() != ScalarType::Int || t->numel() < 1)) good = false;
    return t;
  }
  long long number() {
    if (!good) return 0;
    const long long v = PyLong_AsLongLong(*at_++);
    if (v == -1 && PyErr_Occurred()) good = false;
    return v;
  }
  int small() {
    const long long v = number();
    if (v < INT32_MIN || v > INT32_MAX) good = false;
    return static_cast<int>(v);
  }
  bool check(bool x) { return good = good && x; }

 private:
  PyObject* const* at_;
  long device_ = -1;

 public:
  bool good;
  void* stream = nullptr;
};

// Other threads run meanwhile: a full launch queue waits. Also where torch throws of a tensor, what catches it holds the lock again.
class Unlocked {
 public:
  Unlocked() : state_(PyEval_SaveThread()) {}
  ~Unlocked() { PyEval_RestoreThread(state_); }

 private:
  PyThreadState* state_;
};

template <typename F>
PyObject* answer(Args& a, F call) {
  if (!a.good) {
    PyErr_Clear();
    return PyLong_FromLong(-1);
  }
  long status;
  {
    Unlocked meanwhile;
    status = call();
  }
  return PyLong_FromLong(status);
}

int code_of(const Tensor& t) {
  switch (t.scalar_type()) {
    case ScalarType::Float: return FSX_F32;
    case ScalarType::BFloat16: return FSX_BF16;
    case ScalarType::Half: return FSX_F16;
    case ScalarType::Float8_e4m3fn:
    case ScalarType::Byte: return FSX_E4M3;
    default: return -1;
  }
}
bool is(const Tensor* t, ScalarType type, std::initializer_list<int64_t> shape) {
  return t->scalar_type() == type && t->sizes() == at::IntArrayRef(shape) && t->is_contiguous();
}
// sizes that the entry points take in 32 bits
bool fit(std::initializer_list<int64_t> sizes) { return std::max(sizes) <= INT32_MAX; }
// [rows, heads, head_dim] whose rows are contiguous
bool rows(const Tensor* t) {
  return t->dim() == 3 && t->stride(2) == 1 && (t->stride(1) == t->size(2) || t->size(1) == 1);
}
long long pitch(const Tensor* t) {
  return t->size(0) > 1 ? t->stride(0) : std::max<int64_t>(t->stride(0), t->size(1) * t->size(2));
}
template <typename T = void>
T* ptr(const Tensor* t) {
  return t ? static_cast<T*>(t->data_ptr()) : nullptr;
}
bool scales(const Tensor* k, const Tensor* v, int64_t kv_heads, int64_t n) {
  return k && v && is(k, ScalarType::Float, {kv_heads, n}) && is(v, ScalarType::Float, {kv_heads, n});
}
bool two_caches(const Tensor* k, const Tensor* v, int64_t head_dim) {
  return k->dim() == 3 && k->size(2) == head_dim && k->is_contiguous() && v->is_contiguous() && v->sizes() == k->sizes() &&
         v->scalar_type() == k->scalar_type() && code_of(*k) >= 0;
}

// q, k, positions, axis, rate, n_axes, layout, status, q_out, k_out, v, rows, k_cache, v_cache, k_scale, v_scale
PyObject* rotary(PyObject*, PyObject* const* args, Py_ssize_t n) {
  Args a(args, n, 18);
  const Tensor *q = a.tensor(true), *k = a.tensor(true), *pos = a.tensor();
  const int* axis = reinterpret_cast<const int*>(a.number());
  const double* rate = reinterpret_cast<const double*>(a.number());
  const int n_axes = a.small(), layout = a.small();
  const Tensor *status = a.word(), *q_out = a.tensor(true), *k_out = a.tensor(true), *v = a.tensor(true), *dst = a.tensor(true),
               *kc = a.tensor(true), *vc = a.tensor(true), *ks = a.tensor(true), *vs = a.tensor(true);
  const Tensor* any = q ? q : k;
  int64_t count = 0, heads = 0, kv_heads = 0, dim = 0;
  if (a.check(any && any->dim() == 3 && !q == !q_out && (k || (!k_out && !kc)) && !kc == !vc)) {
    count = any->size(0), heads = any->size(1), dim = any->size(2);
    a.check(pos->scalar_type() == ScalarType::Long && pos->dim() == 2 && pos->size(1) == count && pos->size(0) >= n_axes && pos->is_contiguous());
    if (q) a.check(q_out->sizes() == q->sizes() && q_out->scalar_type() == q->scalar_type() && rows(q) && rows(q_out));
    kv_heads = heads;
    if (k && a.check(k->dim() == 3 && k->size(0) == count && k->size(2) == dim && k->scalar_type() == any->scalar_type() && rows(k))) {
      kv_heads = k->size(1);
      if (k_out) a.check(k_out->sizes() == k->sizes() && k_out->scalar_type() == k->scalar_type() && rows(k_out));
      if (kc && a.check(v && two_caches(kc, vc, dim) && kc->size(1) == kv_heads && kc->size(0) > 0)) {
        a.check(v->sizes() == k->sizes() && v->scalar_type() == k->scalar_type() && rows(v) && (count < 2 || v->stride(0) == k->stride(0)));
        a.check(code_of(*kc) != FSX_E4M3 || scales(ks, vs, kv_heads, kc->size(0)));
        a.check(!dst || is(dst, ScalarType::Long, {count}));
      }
    }
  }
  return answer(a, [&] {
    const bool eight = kc && code_of(*kc) == FSX_E4M3;
    return f_rotary(ptr(q), q ? pitch(q) : 0, ptr(k), kc ? ptr(v) : nullptr, k ? pitch(k) : 0, code_of(*any), ptr<int64_t>(pos),
                    static_cast<int>(pos->size(0)), axis, rate, layout, count, static_cast<int>(heads), static_cast<int>(kv_heads),
                    static_cast<int>(dim), ptr(q_out), q_out ? pitch(q_out) : 0, ptr(k_out), k_out ? pitch(k_out) : 0, kc ? ptr<int64_t>(dst) : nullptr,
                    ptr(kc), ptr(vc), eight ? ptr<float>(ks) : nullptr, eight ? ptr<float>(vs) : nullptr, kc ? code_of(*kc) : code_of(*any),
                    kc ? kc->size(0) : 0, ptr<int>(status), a.stream);
  });
}

// q, k_cache, v_cache, table, lengths, page_rows, out, status, workspace, k_scale, v_scale, picked, lse
PyObject* paged_attention(PyObject*, PyObject* const* args, Py_ssize_t n) {
  Args a(args, n, 15);
  const Tensor *q = a.tensor(), *kc = a.tensor(), *vc = a.tensor(), *table = a.tensor(), *lengths = a.tensor();
  const int page_rows = a.small();
  const Tensor *out = a.tensor(), *status = a.word(), *ws = a.tensor(), *ks = a.tensor(true), *vs = a.tensor(true), *picked = a.tensor(true),
               *lse = a.tensor(true);
  int64_t B = 0, heads = 0, dim = 0;
  if (a.check(a.good && rows(q) && table->dim() == 2 && ws->is_contiguous())) {
    B = q->size(0), heads = q->size(1), dim = q->size(2);
    a.check(code_of(*q) >= 0 && out->scalar_type() == q->scalar_type() && out->sizes() == q->sizes() && out->is_contiguous() &&
            is(table, ScalarType::Int, {B, table->size(1)}) && is(lengths, ScalarType::Long, {B}) && two_caches(kc, vc, dim));
    a.check(a.good && (code_of(*kc) != FSX_E4M3 || scales(ks, vs, kc->size(1), kc->size(0))));
    a.check(a.good && (!picked || (picked->dim() == 3 && picked->size(2) > 0 && is(picked, ScalarType::Int, {B, kc->size(1), picked->size(2)}))));
    a.check(a.good && fit({B, table->size(1), picked ? picked->size(2) : 0}));
    a.check(!lse || is(lse, ScalarType::Float, {heads, B}));
  }
  return answer(a, [&] {
    const bool eight = code_of(*kc) == FSX_E4M3;
    return f_paged_attention(ptr(q), pitch(q), code_of(*q), ptr(kc), ptr(vc), eight ? ptr<float>(ks) : nullptr, eight ? ptr<float>(vs) : nullptr,
                             code_of(*kc), kc->size(0), page_rows, ptr<int32_t>(table), static_cast<int>(table->size(1)), ptr<int64_t>(lengths),
                             static_cast<int>(B), ptr<int32_t>(picked), picked ? static_cast<int>(picked->size(2)) : 0, static_cast<int>(heads),
                             static_cast<int>(kc->size(1)), static_cast<int>(dim), ptr(out), ptr<float>(lse), ptr(ws),
                             static_cast<size_t>(ws->numel() * ws->element_size()), ptr<int>(status), a.stream);
  });
}

// a table of requests, their lengths, and the bounds of `pages` pages
bool paged(const Tensor* table, const Tensor* lengths, const Tensor* bounds, const Tensor* scale, int64_t pages, int64_t kv_heads, int64_t dim) {
  return table->dim() == 2 && is(table, ScalarType::Int, {table->size(0), table->size(1)}) && is(lengths, ScalarType::Long, {table->size(0)}) &&
         is(bounds, ScalarType::Char, {pages, kv_heads, 2, dim}) && is(scale, ScalarType::Float, {kv_heads, pages}) &&
         fit({table->size(0), table->size(1)});
}

// k_cache, table, lengths, page_rows, bounds, bound_scale, status, k_scale, start
PyObject* page_bounds(PyObject*, PyObject* const* args, Py_ssize_t n) {
  Args a(args, n, 11);
  const Tensor *kc = a.tensor(), *table = a.tensor(), *lengths = a.tensor();
  const int page_rows = a.small();
  const Tensor *bounds = a.tensor(), *scale = a.tensor(), *status = a.word(), *ks = a.tensor(true), *start = a.tensor(true);
  a.check(a.good && page_rows > 0 && kc->dim() == 3 && kc->is_contiguous() && code_of(*kc) >= 0 &&
          paged(table, lengths, bounds, scale, kc->size(0) / page_rows, kc->size(1), kc->size(2)));
  a.check(a.good && (code_of(*kc) != FSX_E4M3 || (ks && is(ks, ScalarType::Float, {kc->size(1), kc->size(0)}))));
  a.check(a.good && (!start || is(start, ScalarType::Long, {table->size(0)})));
  return answer(a, [&] {
    return f_page_bounds(ptr(kc), code_of(*kc) == FSX_E4M3 ? ptr<float>(ks) : nullptr, code_of(*kc), kc->size(0), page_rows, ptr<int32_t>(table),
                         static_cast<int>(table->size(1)), ptr<int64_t>(lengths), ptr<int64_t>(start), static_cast<int>(table->size(0)),
                         static_cast<int>(kc->size(1)), static_cast<int>(kc->size(2)), ptr<int8_t>(bounds), ptr<float>(scale), ptr<int>(status), a.stream);
  });
}

// q, bounds, bound_scale, table, lengths, page_rows, picked, status, first, last
PyObject* page_select(PyObject*, PyObject* const* args, Py_ssize_t n) {
  Args a(args, n, 12);
  const Tensor *q = a.tensor(), *bounds = a.tensor(), *scale = a.tensor(), *table = a.tensor(), *lengths = a.tensor();
  const int page_rows = a.small();
  const Tensor *picked = a.tensor(), *status = a.word();
  const int first = a.small(), last = a.small();
  a.check(a.good && rows(q) && bounds->dim() == 4 && code_of(*q) >= 0 && q->size(2) == bounds->size(3) &&
          paged(table, lengths, bounds, scale, bounds->size(0), bounds->size(1), bounds->size(3)) && table->size(0) == q->size(0) &&
          picked->dim() == 3 && is(picked, ScalarType::Int, {q->size(0), bounds->size(1), picked->size(2)}) && fit({picked->size(2)}));
  return answer(a, [&] {
    return f_page_select(ptr(q), pitch(q), code_of(*q), ptr<int8_t>(bounds), ptr<float>(scale), bounds->size(0) * page_rows, page_rows,
                         ptr<int32_t>(table), static_cast<int>(table->size(1)), ptr<int64_t>(lengths), static_cast<int>(q->size(0)),
                         static_cast<int>(q->size(1)), static_cast<int>(bounds->size(1)), static_cast<int>(q->size(2)), first, last,
                         static_cast<int>(picked->size(2)), ptr<int32_t>(picked), ptr<int>(status), a.stream);
  });
}

// table, lengths, refs, new_offsets, page_rows, table_out, lengths_out, refs_out, rows, pairs, n_pairs, status, source
PyObject* pages_step(PyObject*, PyObject* const* args, Py_ssize_t n) {
  Args a(args, n, 15);
  const Tensor *table = a.tensor(), *lengths = a.tensor(), *refs = a.tensor(), *offsets = a.tensor();
  const int page_rows = a.small();
  const Tensor *table_out = a.tensor(), *lengths_out = a.tensor(), *refs_out = a.tensor(), *to = a.tensor(), *pairs = a.tensor(), *n_pairs = a.tensor(),
               *status = a.word(), *source = a.tensor(true);
  int64_t B_in = 0, B = 0, width = 0, pages = 0, total = 0;
  if (a.check(a.good && table->dim() == 2 && table_out->dim() == 2 && refs->dim() == 1 && to->dim() == 1)) {
    B_in = table->size(0), B = table_out->size(0), width = table->size(1), pages = refs->size(0), total = to->size(0);
    a.check(is(table, ScalarType::Int, {B_in, width}) && is(lengths, ScalarType::Long, {B_in}) && is(refs, ScalarType::Int, {pages}) &&
            is(offsets, ScalarType::Long, {B + 1}) && is(table_out, ScalarType::Int, {B, width}) && is(lengths_out, ScalarType::Long, {B}) &&
            is(refs_out, ScalarType::Int, {pages}) && is(to, ScalarType::Long, {total}) && is(pairs, ScalarType::Int, {B, 2}) &&
            is(n_pairs, ScalarType::Int, {1}) && (!source || is(source, ScalarType::Int, {B})) && fit({B_in, B, width, pages}));
  }
  return answer(a, [&] {
    return f_pages_step(ptr<int32_t>(table), ptr<int64_t>(lengths), ptr<int32_t>(refs), static_cast<int>(B_in), ptr<int32_t>(source),
                        ptr<int64_t>(offsets), static_cast<int>(B), total, static_cast<int>(width), static_cast<int>(pages), page_rows,
                        ptr<int32_t>(table_out), ptr<int64_t>(lengths_out), ptr<int32_t>(refs_out), ptr<int64_t>(to), ptr<int32_t>(pairs),
                        ptr<int32_t>(n_pairs), ptr<int>(status), a.stream);
  });
}

// table, lengths, refs, page_rows, table_out, refs_out, pairs, n_pairs, status
PyObject* pages_compact(PyObject*, PyObject* const* args, Py_ssize_t n) {
  Args a(args, n, 11);
  const Tensor *table = a.tensor(), *lengths = a.tensor(), *refs = a.tensor();
  const int page_rows = a.small();
  const Tensor *table_out = a.tensor(), *refs_out = a.tensor(), *pairs = a.tensor(), *n_pairs = a.tensor(), *status = a.word();
  int64_t B = 0, width = 0, pages = 0;
  if (a.check(a.good && table->dim() == 2 && refs->dim() == 1 && pairs->dim() == 2)) {
    B = table->size(0), width = table->size(1), pages = refs->size(0);
    a.check(is(table, ScalarType::Int, {B, width}) && is(lengths, ScalarType::Long, {B}) && is(refs, ScalarType::Int, {pages}) &&
            is(table_out, ScalarType::Int, {B, width}) && is(refs_out, ScalarType::Int, {pages}) &&
            is(pairs, ScalarType::Int, {pairs->size(0), 2}) && is(n_pairs, ScalarType::Int, {1}) && fit({B, width, pages, pairs->size(0)}));
  }
  return answer(a, [&] {
    return f_pages_compact(ptr<int32_t>(table), ptr<int64_t>(lengths), ptr<int32_t>(refs), static_cast<int>(B), static_cast<int>(width),
                           static_cast<int>(pages), page_rows, ptr<int32_t>(table_out), ptr<int32_t>(refs_out), ptr<int32_t>(pairs),
                           static_cast<int>(pairs->size(0)), ptr<int32_t>(n_pairs), ptr<int>(status), a.stream);
  });
}

// planes, n_planes, n_pages, pairs, n_pairs, status
PyObject* pages_copy(PyObject*, PyObject* const* args, Py_ssize_t n) {
  Args a(args, n, 8);
  const fsx_page_plane* planes = reinterpret_cast<const fsx_page_plane*>(a.number());
  const int n_planes = a.small(), n_pages = a.small();
  const Tensor *pairs = a.tensor(), *n_pairs = a.tensor(), *status = a.word();
  a.check(a.good && pairs->dim() == 2 && is(pairs, ScalarType::Int, {pairs->size(0), 2}) && is(n_pairs, ScalarType::Int, {1}) &&
          fit({pairs->size(0)}));
  return answer(a, [&] {
    return f_pages_copy(planes, n_planes, n_pages, ptr<int32_t>(pairs), ptr<int32_t>(n_pairs), static_cast<int>(pairs->size(0)), ptr<int>(status),
                        a.stream);
  });
}

// the library's path: its entry points, from the same library that ctypes holds
PyObject* bind(PyObject*, PyObject* path) {
  const char* at = PyUnicode_AsUTF8(path);
  if (!at) return nullptr;
  void* lib = dlopen(at, RTLD_NOW);
  if (!lib) return PyErr_Format(PyExc_RuntimeError, "%s", dlerror());
  const char* missing = nullptr;
  auto find = [&](auto& f, const char* name) {
    f = reinterpret_cast<std::decay_t<decltype(f)>>(dlsym(lib, name));
    if (!f) missing = name;
  };
  find(f_rotary, "fsx_rotary");
  find(f_paged_attention, "fsx_paged_attention");
  find(f_page_bounds, "fsx_page_bounds");
  find(f_page_select, "fsx_page_select");
  find(f_pages_step, "fsx_pages_step");
  find(f_pages_compact, "fsx_pages_compact");
  find(f_pages_copy, "fsx_pages_copy");
  if (missing) return PyErr_Format(PyExc_RuntimeError, "%s: no %s", at, missing);
  Py_RETURN_NONE;
}

// what torch throws of a tensor is a tensor that does not go with the call
template <PyObject* (*F)(PyObject*, PyObject* const*, Py_ssize_t)>
PyObject* guarded(PyObject* self, PyObject* const* args, Py_ssize_t n) {
  try {
    return F(self, args, n);
  } catch (...) {
    PyErr_Clear();
    return PyLong_FromLong(-1);
  }
}
template <PyObject* (*F)(PyObject*, PyObject* const*, Py_ssize_t)>
PyCFunction fast() {
  return reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(&guarded<F>));
}
PyMethodDef methods[] = {{"rotary", fast<&rotary>(), METH_FASTCALL, nullptr},
                         {"paged_attention", fast<&paged_attention>(), METH_FASTCALL, nullptr},
                         {"page_bounds", fast<&page_bounds>(), METH_FASTCALL, nullptr},
                         {"page_select", fast<&page_select>(), METH_FASTCALL, nullptr},
                         {"pages_step", fast<&pages_step>(), METH_FASTCALL, nullptr},
                         {"pages_compact", fast<&pages_compact>(), METH_FASTCALL, nullptr},
                         {"pages_copy", fast<&pages_copy>(), METH_FASTCALL, nullptr},
                         {"bind", &bind, METH_O, nullptr},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module_def = {PyModuleDef_HEAD_INIT, "_calls", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__calls() { return PyModule_Create(&module_def); }
