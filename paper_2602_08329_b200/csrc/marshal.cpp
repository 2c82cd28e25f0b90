// Python extension of the binding: what the calls of the library need to know of their tensors (addresses, strides) and
// the checks that go with it, read from the tensors directly, and the calls themselves.  A small decode call is
// bound by the host; asking a tensor for its type, shape, strides, device and address through its Python
// attributes costs a tenth of a microsecond each, five to ten microseconds a call, and ctypes another one.
// Argument marshalling only: no CUDA here, and the library's entry points are handed in by bind().
#include <Python.h>

#include <ATen/ATen.h>
#include <torch/csrc/autograd/python_variable.h>

#include <algorithm>
#include <cstdint>
#include <exception>

#include "../../include/prhs.h"

namespace {

// Raises AssertionError with the reason and leaves the function.
#define REQUIRE(cond, what)                           \
  do {                                                \
    if (!(cond)) {                                    \
      PyErr_SetString(PyExc_AssertionError, what);    \
      return nullptr;                                 \
    }                                                 \
  } while (0)

const at::Tensor* tensor(PyObject* o) { return THPVariable_Check(o) ? &THPVariable_Unpack(o) : nullptr; }
bool none(PyObject* o) { return o == Py_None; }
int64_t address(const at::Tensor& t) { return reinterpret_cast<int64_t>(t.data_ptr()); }
// -1: not on a CUDA device
int64_t device(const at::Tensor& t) { return t.is_cuda() ? (int64_t)t.get_device() : -1; }
bool is(const at::Tensor* t, at::ScalarType type, int64_t dev) { return t->scalar_type() == type && device(*t) == dev; }
bool same_layout(const at::Tensor& a, const at::Tensor& b) { return a.sizes() == b.sizes() && a.strides() == b.strides(); }

// integers and tensors of a call: n arguments, in order
bool count_is(Py_ssize_t nargs, Py_ssize_t n) {
  if (nargs == n) return true;
  PyErr_SetString(PyExc_TypeError, "wrong number of arguments");
  return false;
}

// kv_view(k, v, seq_lens, page_table | None): k, v, stride_outer, stride_head, table, table_stride, seq_lens, pages, batch, heads,
// span (positions that the cache, or a row of the page table, has), device (-1 where the block calls refuse the view), why they do
PyObject* kv_view(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  if (!count_is(nargs, 4)) return nullptr;
  const at::Tensor *k = tensor(a[0]), *v = tensor(a[1]), *lens = tensor(a[2]), *table = none(a[3]) ? nullptr : tensor(a[3]);
  REQUIRE(k && v && lens && (table || none(a[3])), "a tensor is missing");
  REQUIRE(k->scalar_type() == at::kBFloat16 && v->scalar_type() == at::kBFloat16, "k and v are bf16");
  REQUIRE(k->dim() >= 3 && k->size(-1) == 128 && k->strides() == v->strides() && k->stride(-1) == 1 && k->stride(-2) == 128,
          "rows of 128 contiguous elements, k and v alike");
  REQUIRE(lens->scalar_type() == at::kInt, "seq_lens is int32");
  REQUIRE(!table || (table->scalar_type() == at::kInt && table->dim() >= 1 && (table->dim() == 1 || table->stride(-1) == 1)),
          "the page table is int32 [batch][pages], its rows contiguous");
  // what the block calls ask of a view beyond that; the other calls take it as it is
  const bool paged = table != nullptr;
  const int64_t dev = device(*k);
  const char* why = nullptr;
  if (k->dim() != 4 || v->sizes() != k->sizes()) why = "k and v are alike, with four axes";
  else if (lens->dim() != 1 || !lens->is_contiguous()) why = "seq_lens is contiguous [batch]";
  else if (paged && (table->dim() != 2 || k->size(2) != 16)) why = "the page table is [batch][pages], of pages of 16 positions";
  else if (device(*v) != dev || device(*lens) != dev || (paged && device(*table) != dev) || dev < 0) why = "the tensors of a call are on one CUDA device";
  const int64_t batch = std::min(lens->numel(), paged ? table->size(0) : k->size(0));
  const int64_t span = !paged ? k->size(2) : table->dim() == 2 ? 16 * table->size(1) : 0;
  return Py_BuildValue("LLLLLLLLLLLLz", address(*k), address(*v), k->stride(0), k->stride(1), paged ? address(*table) : 0,
                       paged ? table->stride(0) : 0, address(*lens), paged ? k->size(0) : 0, batch, k->size(1), span, why ? -1 : dev, why);
}

// bytekv_view(k, v, k_scale, v_scale, k_tail, v_tail, seq_lens, page_table | None, max_seq_len): six addresses, stride_outer,
// stride_head, scale strides, table, seq_lens, table_stride, pages, format, batch, heads, cap, device
PyObject* bytekv_view(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  if (!count_is(nargs, 9)) return nullptr;
  const at::Tensor* t[8];
  for (int i = 0; i < 8; ++i) {
    t[i] = i == 7 && none(a[7]) ? nullptr : tensor(a[i]);
    REQUIRE(t[i] || (i == 7 && none(a[7])), "a tensor is missing");
  }
  const at::Tensor &k = *t[0], &v = *t[1], &ks = *t[2], &vs = *t[3], &kt = *t[4], &vt = *t[5], &lens = *t[6];
  const int64_t max_len = PyLong_AsLongLong(a[8]);
  if (max_len == -1 && PyErr_Occurred()) return nullptr;
  const at::ScalarType type = k.scalar_type();
  REQUIRE(type == at::kFloat8_e4m3fn || type == at::kFloat8_e5m2, "codes are float8_e4m3fn or float8_e5m2");
  const int64_t dev = device(k);
  REQUIRE(dev >= 0, "the tensors of a call are on one CUDA device");
  REQUIRE(is(&v, type, dev) && k.dim() == 4 && same_layout(k, v), "k and v codes are alike");
  REQUIRE(k.size(3) == 128 && k.stride(3) == 1 && k.stride(2) == 128 && k.size(2) % 16 == 0, "rows of 128 contiguous codes, whole blocks of 16");
  REQUIRE(is(&ks, at::kFloat, dev) && is(&vs, at::kFloat, dev) && same_layout(ks, vs), "scales are fp32 and alike");
  REQUIRE(is(&kt, at::kBFloat16, dev) && is(&vt, at::kBFloat16, dev) && kt.sizes() == vt.sizes(), "tails are bf16 and alike");
  REQUIRE(is(&lens, at::kInt, dev) && lens.dim() == 1 && lens.is_contiguous(), "seq_lens is int32 [batch]");
  const int64_t batch = lens.size(0);
  REQUIRE(kt.dim() == 4 && kt.size(0) >= batch && kt.size(1) == k.size(1) && kt.size(2) == 16 && kt.size(3) == 128 && kt.is_contiguous() &&
              vt.is_contiguous(), "tails are contiguous [batch][Hkv][16][128]");
  if (t[7]) {
    const at::Tensor& table = *t[7];
    REQUIRE(k.size(2) == 16 && ks.dim() == 2 && ks.size(0) == k.size(0) && ks.size(1) == k.size(1), "pages of 16 positions, a scale per page and head");
    REQUIRE(is(&table, at::kInt, dev) && table.dim() == 2 && table.stride(1) == 1 && table.size(0) >= batch, "the page table is int32 [batch][pages]");
  } else {
    REQUIRE(ks.dim() == 3 && ks.size(0) == k.size(0) && ks.size(1) == k.size(1) && ks.size(2) == k.size(2) / 16 && ks.stride(2) == 1,
            "scales are [batch][Hkv][cap / 16]");
    REQUIRE(k.size(0) >= batch && max_len <= k.size(2), "the cache holds the batch and max_seq_len positions");
  }
  return Py_BuildValue("LLLLLLLLLLLLLLLLLLL", address(k), address(v), address(ks), address(vs), address(kt), address(vt), k.stride(0),
                       k.stride(1), ks.stride(0), ks.stride(1), t[7] ? address(*t[7]) : 0, address(lens), t[7] ? t[7]->stride(0) : 0,
                       t[7] ? k.size(0) : 0, type == at::kFloat8_e5m2 ? 1 : 0, batch, k.size(1), t[7] ? 16 * t[7]->size(1) : k.size(2), dev);
}

// bounds_view(codes, scale): codes, scale, stride_outer, stride_head, outer size, heads, blocks (0: per page), device
PyObject* bounds_view(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  if (!count_is(nargs, 2)) return nullptr;
  const at::Tensor *c = tensor(a[0]), *s = tensor(a[1]);
  REQUIRE(c && s, "a tensor is missing");
  const int64_t d = c->dim(), dev = device(*c);
  REQUIRE(dev >= 0, "the tensors of a call are on one CUDA device");
  REQUIRE(is(c, at::kChar, dev) && is(s, at::kFloat, dev), "bounds are int8, their scales fp32");
  REQUIRE((d == 4 || d == 5) && s->dim() == d - 2 && c->size(d - 2) == 2 && c->size(d - 1) == 128 && c->sizes().slice(0, d - 2) == s->sizes(),
          "bounds are [..][2][128], scales [..]");
  REQUIRE(c->is_contiguous() && s->is_contiguous(), "bounds and scales are contiguous");
  return Py_BuildValue("LLLLLLLL", address(*c), address(*s), s->stride(0), s->stride(1), c->size(0), c->size(1), d == 5 ? c->size(2) : 0, dev);
}

// ------------------------------------------------------------------------------------ calls
// The entry points, in the order that bind() receives them.
struct Entries {
  decltype(&prhs_bytekv_append) bytekv_append;
  decltype(&prhs_bytekv_decode_attn) bytekv_decode_attn;
  decltype(&prhs_bytekv_sparse_decode_attn) bytekv_sparse_decode_attn;
  decltype(&prhs_block_bounds) block_bounds;
  decltype(&prhs_block_topk) block_topk;
  decltype(&prhs_block_decode_attn) block_decode_attn;
  decltype(&prhs_block_decode_step) block_decode_step;
} entry{};
static_assert(sizeof(Entries) == 7 * sizeof(void*), "bind() fills the entries in order");

PyObject* bind(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  if (!count_is(nargs, 7)) return nullptr;
  for (int i = 0; i < 7; ++i) {
    void* p = PyLong_AsVoidPtr(a[i]);
    if (PyErr_Occurred()) return nullptr;
    reinterpret_cast<void**>(&entry)[i] = p;
  }
  Py_RETURN_NONE;
}

// Integer and address arguments (PyErr_Occurred() once one is neither).
struct Args {
  PyObject* const* a;
  int64_t integer(int i) const { return PyLong_AsLongLong(a[i]); }
  template <typename T>
  T* pointer(int i) const { return static_cast<T*>(PyLong_AsVoidPtr(a[i])); }
};
// The interpreter's lock, given up for as long as this lives, whichever way its scope is left.
class Released {
 public:
  Released() : state_(PyEval_SaveThread()) {}
  ~Released() { PyEval_RestoreThread(state_); }
  Released(const Released&) = delete;
  Released& operator=(const Released&) = delete;

 private:
  PyThreadState* state_;
};
// The call with the interpreter released, as ctypes makes it; the status as a Python integer.  Tensors are read before.
template <typename F>
PyObject* status(F call) {
  prhs_status rc;
  {
    const Released released;
    rc = call();
  }
  return PyLong_FromLong(rc);
}

// A decode attention's q, out and out_lse (Python None: absent).
struct Io {
  const void* q;
  void* out;
  float* lse;
  // nullptr: the error is set
  PyObject* read(PyObject* oq, PyObject* oo, PyObject* ol, int64_t batch, int64_t heads, int64_t dev) {
    const at::Tensor *tq = tensor(oq), *to = none(oo) ? nullptr : tensor(oo), *tl = none(ol) ? nullptr : tensor(ol);
    REQUIRE(tq && (to || none(oo)) && (tl || none(ol)), "a tensor is missing");
    for (const at::Tensor* t : {tq, to})
      REQUIRE(!t || (is(t, at::kBFloat16, dev) && t->dim() == 3 && t->size(0) == batch && t->size(1) == heads && t->size(2) == 128 && t->is_contiguous()),
              "q and out are contiguous bf16 [batch][Hq][128] on the cache's device");
    REQUIRE(!tl || (is(tl, at::kFloat, dev) && tl->dim() == 2 && tl->size(0) == batch && tl->size(1) == heads && tl->is_contiguous()),
            "out_lse is contiguous fp32 [batch][Hq] on the cache's device");
    q = tq->data_ptr();
    out = to ? to->data_ptr() : nullptr;
    lse = tl ? static_cast<float*>(tl->data_ptr()) : nullptr;
    return Py_None;
  }
};
// Lists of entries or blocks, with their counts.
struct Lists {
  int32_t *lists, *count;
  int32_t stride;
  PyObject* read(PyObject* ol, PyObject* oc, int64_t batch, int64_t units, int64_t dev) {
    const at::Tensor *l = tensor(ol), *c = tensor(oc);
    REQUIRE(l && c, "a tensor is missing");
    REQUIRE(is(l, at::kInt, dev) && l->dim() == 3 && l->size(0) == batch && l->size(1) == units && l->is_contiguous() && l->size(2) <= INT32_MAX,
            "lists are contiguous int32 [batch][units][stride] on the cache's device");
    REQUIRE(is(c, at::kInt, dev) && c->dim() == 2 && c->size(0) == batch && c->size(1) == units && c->is_contiguous(),
            "counts are contiguous int32 [batch][units] on the cache's device");
    lists = static_cast<int32_t*>(l->data_ptr());
    count = static_cast<int32_t*>(c->data_ptr());
    stride = (int32_t)l->size(2);
    return Py_None;
  }
};

// bytekv_append(ctx, view, new_k, new_v, new_lens, batch, heads, device, max_new, stream)
PyObject* bytekv_append(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  if (!count_is(nargs, 10)) return nullptr;
  const Args v{a};
  prhs_ctx* ctx = v.pointer<prhs_ctx>(0);
  const prhs_bytekv_view* kv = v.pointer<prhs_bytekv_view>(1);
  const int64_t batch = v.integer(5), heads = v.integer(6), dev = v.integer(7), max_new = v.integer(8);
  void* stream = v.pointer<void>(9);
  if (PyErr_Occurred()) return nullptr;
  const at::Tensor *k = tensor(a[2]), *vv = tensor(a[3]), *n = tensor(a[4]);
  REQUIRE(k && vv && n, "a tensor is missing");
  REQUIRE(is(k, at::kBFloat16, dev) && is(vv, at::kBFloat16, dev) && same_layout(*k, *vv), "new rows are bf16 on the cache's device, k and v alike");
  REQUIRE(k->dim() == 4 && k->size(0) >= batch && k->size(1) == heads && k->size(3) == 128 && k->stride(3) == 1, "new rows are [batch][Hkv][rows][128]");
  REQUIRE(is(n, at::kInt, dev) && n->dim() == 1 && n->size(0) >= batch && n->is_contiguous(), "new_lens is int32 [batch] on the cache's device");
  REQUIRE(0 <= max_new && max_new <= k->size(2) && k->size(2) <= INT32_MAX, "max_new is at most the number of rows given");
  auto stride = [&](int i) { return k->size(i) > 1 ? k->stride(i) : 0; };     // that of an axis of one element is arbitrary
  const int64_t by_seq = stride(0), by_head = stride(1), by_row = stride(2);
  const void *new_k = k->data_ptr(), *new_v = vv->data_ptr();
  const int32_t* new_lens = static_cast<const int32_t*>(n->data_ptr());
  const int32_t rows = (int32_t)(max_new ? max_new : k->size(2));
  return status([&] { return entry.bytekv_append(ctx, kv, new_k, new_v, by_seq, by_head, by_row, new_lens, rows, (int32_t)batch, stream); });
}

// bytekv_decode_attn(ctx, view, q, out, out_lse, batch, heads, device, stream)
PyObject* bytekv_decode_attn(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  if (!count_is(nargs, 9)) return nullptr;
  const Args v{a};
  prhs_ctx* ctx = v.pointer<prhs_ctx>(0);
  const prhs_bytekv_view* kv = v.pointer<prhs_bytekv_view>(1);
  const int64_t batch = v.integer(5), heads = v.integer(6), dev = v.integer(7);
  void* stream = v.pointer<void>(8);
  if (PyErr_Occurred()) return nullptr;
  Io io;
  if (!io.read(a[2], a[3], a[4], batch, heads, dev)) return nullptr;
  return status([&] { return entry.bytekv_decode_attn(ctx, io.q, kv, (int32_t)batch, io.out, io.lse, stream); });
}

// bytekv_sparse_decode_attn(ctx, view, q, out, out_lse, batch, heads, device, stream, idx, count)
PyObject* bytekv_sparse_decode_attn(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  if (!count_is(nargs, 11)) return nullptr;
  const Args v{a};
  prhs_ctx* ctx = v.pointer<prhs_ctx>(0);
  const prhs_bytekv_view* kv = v.pointer<prhs_bytekv_view>(1);
  const int64_t batch = v.integer(5), heads = v.integer(6), dev = v.integer(7);
  void* stream = v.pointer<void>(8);
  if (PyErr_Occurred()) return nullptr;
  Io io;
  Lists l;
  if (!io.read(a[2], a[3], a[4], batch, heads, dev) || !l.read(a[9], a[10], batch, heads, dev)) return nullptr;
  return status([&] { return entry.bytekv_sparse_decode_attn(ctx, io.q, kv, l.lists, l.count, l.stride, (int32_t)batch, io.out, io.lse, stream); });
}

// block_bounds(ctx, view, bounds, first | None, max_new, batch, device, stream)
PyObject* block_bounds(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  if (!count_is(nargs, 8)) return nullptr;
  const Args v{a};
  prhs_ctx* ctx = v.pointer<prhs_ctx>(0);
  const prhs_kv_view* kv = v.pointer<prhs_kv_view>(1);
  const prhs_block_bounds_view* bounds = v.pointer<prhs_block_bounds_view>(2);
  const int64_t max_new = v.integer(4), batch = v.integer(5), dev = v.integer(6);
  void* stream = v.pointer<void>(7);
  if (PyErr_Occurred()) return nullptr;
  const at::Tensor* first = none(a[3]) ? nullptr : tensor(a[3]);
  REQUIRE(first || none(a[3]), "a tensor is missing");
  REQUIRE(!first || (is(first, at::kInt, dev) && first->dim() == 1 && first->size(0) >= batch && first->is_contiguous()),
          "first is int32 [batch] on the cache's device");
  const int32_t* at = first ? static_cast<const int32_t*>(first->data_ptr()) : nullptr;
  return status([&] { return entry.block_bounds(ctx, kv, bounds, at, (int32_t)max_new, (int32_t)batch, stream); });
}

// block_topk(ctx, view, bounds, sched, q, batch, heads, units, device, stream, blocks, count)
PyObject* block_topk(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  if (!count_is(nargs, 12)) return nullptr;
  const Args v{a};
  prhs_ctx* ctx = v.pointer<prhs_ctx>(0);
  const prhs_kv_view* kv = v.pointer<prhs_kv_view>(1);
  const prhs_block_bounds_view* bounds = v.pointer<prhs_block_bounds_view>(2);
  const prhs_block_schedule* sched = v.pointer<prhs_block_schedule>(3);
  const int64_t batch = v.integer(5), heads = v.integer(6), units = v.integer(7), dev = v.integer(8);
  void* stream = v.pointer<void>(9);
  if (PyErr_Occurred()) return nullptr;
  Io io;
  Lists l;
  if (!io.read(a[4], Py_None, Py_None, batch, heads, dev) || !l.read(a[10], a[11], batch, units, dev)) return nullptr;
  return status([&] { return entry.block_topk(ctx, io.q, kv, bounds, sched, (int32_t)batch, l.lists, l.stride, l.count, stream); });
}

// block_decode_attn(ctx, view, q, out, out_lse, batch, heads, units, device, stream, blocks, count, flags)
PyObject* block_decode_attn(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  if (!count_is(nargs, 13)) return nullptr;
  const Args v{a};
  prhs_ctx* ctx = v.pointer<prhs_ctx>(0);
  const prhs_kv_view* kv = v.pointer<prhs_kv_view>(1);
  const int64_t batch = v.integer(5), heads = v.integer(6), units = v.integer(7), dev = v.integer(8), flags = v.integer(12);
  void* stream = v.pointer<void>(9);
  if (PyErr_Occurred()) return nullptr;
  Io io;
  Lists l;
  if (!io.read(a[2], a[3], a[4], batch, heads, dev) || !l.read(a[10], a[11], batch, units, dev)) return nullptr;
  return status([&] {
    return entry.block_decode_attn(ctx, io.q, kv, l.lists, l.count, l.stride, (uint32_t)flags, (int32_t)batch, io.out, io.lse, stream);
  });
}

// block_decode_step(ctx, view, bounds, sched, q, out, out_lse, batch, heads, units, device, stream, blocks, count)
PyObject* block_decode_step(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  if (!count_is(nargs, 14)) return nullptr;
  const Args v{a};
  prhs_ctx* ctx = v.pointer<prhs_ctx>(0);
  const prhs_kv_view* kv = v.pointer<prhs_kv_view>(1);
  const prhs_block_bounds_view* bounds = v.pointer<prhs_block_bounds_view>(2);
  const prhs_block_schedule* sched = v.pointer<prhs_block_schedule>(3);
  const int64_t batch = v.integer(7), heads = v.integer(8), units = v.integer(9), dev = v.integer(10);
  void* stream = v.pointer<void>(11);
  if (PyErr_Occurred()) return nullptr;
  Io io;
  Lists l;
  if (!io.read(a[4], a[5], a[6], batch, heads, dev) || !l.read(a[12], a[13], batch, units, dev)) return nullptr;
  return status([&] {
    return entry.block_decode_step(ctx, io.q, kv, bounds, sched, (int32_t)batch, io.out, io.lse, l.lists, l.stride, l.count, stream);
  });
}

// torch's C++ exceptions (a tensor without storage or strides) as Python's: none may leave a C function.
template <PyObject* (*F)(PyObject*, PyObject* const*, Py_ssize_t)>
PyObject* guarded(PyObject* self, PyObject* const* a, Py_ssize_t nargs) noexcept {
  try {
    return F(self, a, nargs);
  } catch (const c10::Error& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what_without_backtrace());
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
  }
  return nullptr;
}

#define METHOD(name) {#name, (PyCFunction)(void*)guarded<name>, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {METHOD(kv_view), METHOD(bytekv_view), METHOD(bounds_view), METHOD(bind), METHOD(bytekv_append), METHOD(bytekv_decode_attn),
                         METHOD(bytekv_sparse_decode_attn), METHOD(block_bounds), METHOD(block_topk), METHOD(block_decode_attn),
                         METHOD(block_decode_step), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module_def = {PyModuleDef_HEAD_INIT, "_marshal", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

#ifndef PRHS_BUILT_FOR
#define PRHS_BUILT_FOR ""
#endif
// built_for: the torch and the python that this was compiled for (build.py looks for the text in the file)
PyMODINIT_FUNC PyInit__marshal() {
  PyObject* module = PyModule_Create(&module_def);
  if (module && PyModule_AddStringConstant(module, "built_for", PRHS_BUILT_FOR) < 0) Py_CLEAR(module);
  return module;
}
