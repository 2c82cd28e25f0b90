// Python extension of the binding: what the calls of the library need to know of their tensors (addresses, strides) and
// the checks that go with it, read from the tensors directly.  A small decode call is bound by the host; asking a
// tensor for its type, shape, strides, device and address through its Python attributes costs a tenth of a
// microsecond each, five to ten microseconds a call.  Argument marshalling only: no CUDA here.
#include <Python.h>

#include <ATen/ATen.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cstdint>

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
// cap, device (-1: host tensors, which no call takes)
PyObject* kv_view(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  if (!count_is(nargs, 4)) return nullptr;
  const at::Tensor *k = tensor(a[0]), *v = tensor(a[1]), *lens = tensor(a[2]), *table = none(a[3]) ? nullptr : tensor(a[3]);
  REQUIRE(k && v && lens && (table || none(a[3])), "a tensor is missing");
  REQUIRE(k->scalar_type() == at::kBFloat16 && v->scalar_type() == at::kBFloat16, "k and v are bf16");
  REQUIRE(k->dim() >= 3 && k->size(-1) == 128 && k->strides() == v->strides() && k->stride(-1) == 1 && k->stride(-2) == 128,
          "rows of 128 contiguous elements, k and v alike");
  REQUIRE(lens->scalar_type() == at::kInt, "seq_lens is int32");
  REQUIRE(!table || (table->scalar_type() == at::kInt && table->dim() == 2 && table->is_contiguous()), "the page table is contiguous int32 [batch][pages]");
  return Py_BuildValue("LLLLLLLLLLLL", address(*k), address(*v), k->stride(0), k->stride(1), table ? address(*table) : 0,
                       table ? table->stride(0) : 0, address(*lens), table ? k->size(0) : 0, lens->numel(), k->size(1),
                       table ? 0 : k->size(2), device(*k));
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
                       t[7] ? k.size(0) : 0, type == at::kFloat8_e5m2 ? 1 : 0, batch, k.size(1), t[7] ? 0 : k.size(2), dev);
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

// rows(new_k, new_v, new_lens, batch, heads, device, max_new): addresses of k, v and lens, strides (sequence, head, row), rows
PyObject* rows(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  if (!count_is(nargs, 7)) return nullptr;
  const at::Tensor *k = tensor(a[0]), *v = tensor(a[1]), *n = tensor(a[2]);
  REQUIRE(k && v && n, "a tensor is missing");
  const int64_t batch = PyLong_AsLongLong(a[3]), heads = PyLong_AsLongLong(a[4]), dev = PyLong_AsLongLong(a[5]), max_new = PyLong_AsLongLong(a[6]);
  if (PyErr_Occurred()) return nullptr;
  REQUIRE(is(k, at::kBFloat16, dev) && is(v, at::kBFloat16, dev) && same_layout(*k, *v), "new rows are bf16 on the cache's device, k and v alike");
  REQUIRE(k->dim() == 4 && k->size(0) >= batch && k->size(1) == heads && k->size(3) == 128 && k->stride(3) == 1, "new rows are [batch][Hkv][rows][128]");
  REQUIRE(is(n, at::kInt, dev) && n->dim() == 1 && n->size(0) >= batch && n->is_contiguous(), "new_lens is int32 [batch]");
  REQUIRE(0 <= max_new && max_new <= k->size(2), "max_new is at most the number of rows given");
  auto stride = [&](int i) { return k->size(i) > 1 ? k->stride(i) : 0; };     // that of an axis of one element is arbitrary
  return Py_BuildValue("LLLLLLL", address(*k), address(*v), address(*n), stride(0), stride(1), stride(2), k->size(2));
}

// io(q, out, out_lse | None, batch, heads, device): their addresses
PyObject* io(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  if (!count_is(nargs, 6)) return nullptr;
  const at::Tensor *q = tensor(a[0]), *out = none(a[1]) ? nullptr : tensor(a[1]), *lse = none(a[2]) ? nullptr : tensor(a[2]);
  REQUIRE(q && (out || none(a[1])) && (lse || none(a[2])), "a tensor is missing");
  const int64_t batch = PyLong_AsLongLong(a[3]), heads = PyLong_AsLongLong(a[4]), dev = PyLong_AsLongLong(a[5]);
  if (PyErr_Occurred()) return nullptr;
  for (const at::Tensor* t : {q, out})
    REQUIRE(!t || (is(t, at::kBFloat16, dev) && t->dim() == 3 && t->size(0) == batch && t->size(1) == heads && t->size(2) == 128 && t->is_contiguous()),
            "q and out are contiguous bf16 [batch][Hq][128] on the cache's device");
  REQUIRE(!lse || (is(lse, at::kFloat, dev) && lse->dim() == 2 && lse->size(0) == batch && lse->size(1) == heads && lse->is_contiguous()),
          "out_lse is contiguous fp32 [batch][Hq] on the cache's device");
  return Py_BuildValue("LLL", address(*q), out ? address(*out) : 0, lse ? address(*lse) : 0);
}

// lists(lists, count, batch, units, device): their addresses and the lists' stride
PyObject* lists(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  if (!count_is(nargs, 5)) return nullptr;
  const at::Tensor *l = tensor(a[0]), *c = tensor(a[1]);
  REQUIRE(l && c, "a tensor is missing");
  const int64_t batch = PyLong_AsLongLong(a[2]), units = PyLong_AsLongLong(a[3]), dev = PyLong_AsLongLong(a[4]);
  if (PyErr_Occurred()) return nullptr;
  REQUIRE(is(l, at::kInt, dev) && l->dim() == 3 && l->size(0) == batch && l->size(1) == units && l->is_contiguous(), "lists are contiguous int32 [batch][units][stride]");
  REQUIRE(is(c, at::kInt, dev) && c->dim() == 2 && c->size(0) == batch && c->size(1) == units && c->is_contiguous(), "counts are contiguous int32 [batch][units]");
  return Py_BuildValue("LLL", address(*l), address(*c), l->size(2));
}

PyMethodDef methods[] = {{"kv_view", (PyCFunction)(void*)kv_view, METH_FASTCALL, nullptr},
                         {"bytekv_view", (PyCFunction)(void*)bytekv_view, METH_FASTCALL, nullptr},
                         {"bounds_view", (PyCFunction)(void*)bounds_view, METH_FASTCALL, nullptr},
                         {"rows", (PyCFunction)(void*)rows, METH_FASTCALL, nullptr},
                         {"io", (PyCFunction)(void*)io, METH_FASTCALL, nullptr},
                         {"lists", (PyCFunction)(void*)lists, METH_FASTCALL, nullptr},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module_def = {PyModuleDef_HEAD_INIT, "_marshal", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__marshal() { return PyModule_Create(&module_def); }
