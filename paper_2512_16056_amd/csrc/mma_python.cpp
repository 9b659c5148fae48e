// The binding of the operators on the paged KV cache: tensors to the argument structs of include/mma.h.
// A decode step makes these calls once or twice a layer, so their set-up counts: from Python through
// ctypes an append takes 14.3 us of host time, 3.6 of them in the library; from here 8.3. Checks types,
// shapes and contiguity (ValueError); that pointers are device memory of the right size is the
// library's check. What a call returns and is not given is allocated here, on the current stream.
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <ATen/ops/empty.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cmath>

#include "../../include/mma.h"

namespace {

decltype(&mma_kv_append) g_append;
decltype(&mma_kv_attention) g_attention;
decltype(&mma_kv_attention_workspace) g_attention_workspace;
decltype(&mma_kv_commit) g_commit;
decltype(&mma_kv_evict) g_evict;
decltype(&mma_kv_evict_workspace) g_evict_workspace;
PyObject* g_check;    // (status, name): raises the library's error
PyObject* g_address;  // (object): its address

struct Refused {};  // a Python exception is set

#define REFUSE(...)                          \
  do {                                       \
    PyErr_Format(PyExc_ValueError, __VA_ARGS__); \
    throw Refused();                         \
  } while (0)

void check(mma_status_t s, const char* name) {
  if (s == MMA_OK) return;
  PyObject* r = PyObject_CallFunction(g_check, "is", static_cast<int>(s), name);
  Py_XDECREF(r);
  if (!PyErr_Occurred()) PyErr_SetString(PyExc_RuntimeError, name);
  throw Refused();
}

// The bytes of a ctypes object.
void* bytes_of(PyObject* o, Py_ssize_t least, const char* name) {
  Py_buffer b;
  if (PyObject_GetBuffer(o, &b, PyBUF_SIMPLE) != 0) throw Refused();
  void* p = b.buf;
  const Py_ssize_t n = b.len;
  PyBuffer_Release(&b);
  if (n < least) REFUSE("%s: %zd bytes are wanted, got %zd", name, least, n);
  return p;
}

uint64_t number(PyObject* o) {
  const unsigned long long v = PyLong_AsUnsignedLongLongMask(o);
  if (v == static_cast<unsigned long long>(-1) && PyErr_Occurred()) throw Refused();
  return v;
}

double real(PyObject* o) {
  const double v = PyFloat_AsDouble(o);
  if (v == -1.0 && PyErr_Occurred()) throw Refused();
  return v;
}

bool truth(PyObject* o) {
  const int v = PyObject_IsTrue(o);
  if (v < 0) throw Refused();
  return v != 0;
}

uint32_t count(PyObject* o, const char* name) {
  const long long v = PyLong_AsLongLong(o);
  if (v == -1 && PyErr_Occurred()) throw Refused();
  if (v < 0 || v > UINT32_MAX) REFUSE("%s: from 0 to 2^32 - 1 is wanted", name);
  return static_cast<uint32_t>(v);
}

uint32_t size32(int64_t n, const char* name) {
  if (n > UINT32_MAX) REFUSE("%s: a size above 2^32 - 1", name);
  return static_cast<uint32_t>(n);
}

const at::Tensor& tensor(PyObject* o, const char* name) {
  if (!THPVariable_Check(o)) REFUSE("%s: a tensor is wanted, got %s", name, Py_TYPE(o)->tp_name);
  return THPVariable_Unpack(o);
}

void* address(PyObject* o) {
  if (THPVariable_Check(o)) return THPVariable_Unpack(o).data_ptr();
  PyObject* r = PyObject_CallOneArg(g_address, o);
  if (!r) throw Refused();
  void* p = PyLong_AsVoidPtr(r);
  Py_DECREF(r);
  if (!p && PyErr_Occurred()) throw Refused();
  return p;
}

// A cache layer: raw bytes (an integer type) or the type that the cache holds, contiguous. What is no GPU tensor is the
// library's to refuse.
void* layer(PyObject* o, at::ScalarType type) {
  if (!THPVariable_Check(o)) return address(o);
  const at::Tensor& t = THPVariable_Unpack(o);
  if (t.is_cuda() && !(t.is_contiguous() && (c10::isIntegralType(t.scalar_type(), false) || t.scalar_type() == type)))
    REFUSE("layer: a contiguous tensor of %s or of bytes is wanted, got %s%s", c10::toString(type), c10::toString(t.scalar_type()),
           t.is_contiguous() ? "" : ", not contiguous");
  return t.data_ptr();
}

std::string text(at::IntArrayRef v) {
  std::string s = "[";
  for (size_t i = 0; i < v.size(); ++i) s += (i ? ", " : "") + std::to_string(v[i]);
  return s + "]";
}

// A contiguous GPU tensor; sizes of -1 are not looked at.
const at::Tensor& flat(PyObject* o, const char* name, at::ScalarType type, std::initializer_list<int64_t> sizes) {
  const at::Tensor& t = tensor(o, name);
  bool ok = t.scalar_type() == type && t.is_cuda() && t.is_contiguous() && t.dim() == static_cast<int64_t>(sizes.size());
  int64_t i = 0;
  for (int64_t n : sizes) ok = ok && (n < 0 || t.size(i) == n), ++i;
  if (!ok)
    REFUSE("%s: a contiguous %s GPU tensor of shape %s is wanted, got %s %s on %s", name, c10::toString(type),
           text(at::IntArrayRef(sizes)).c_str(), c10::toString(t.scalar_type()), text(t.sizes()).c_str(), t.device().str().c_str());
  return t;
}

template <class T>
T* flat_ptr(PyObject* o, const char* name, at::ScalarType type, std::initializer_list<int64_t> sizes) {
  return o == Py_None ? nullptr : static_cast<T*>(flat(o, name, type, sizes).data_ptr());
}

// [tokens][heads][dim] rows.
mma_rows_t rows(const at::Tensor& t, const char* name, at::ScalarType type, int64_t tokens, int64_t heads, int64_t dim) {
  if (t.dim() != 3 || t.size(0) != tokens || t.size(1) != heads || t.size(2) != dim || t.scalar_type() != type || !t.is_cuda())
    REFUSE("%s: %s of shape [%lld, %lld, %lld] on the GPU is wanted, got %s %s on %s", name, c10::toString(type),
           static_cast<long long>(tokens), static_cast<long long>(heads), static_cast<long long>(dim),
           c10::toString(t.scalar_type()), text(t.sizes()).c_str(), t.device().str().c_str());
  if (t.stride(2) != 1 && dim > 1) REFUSE("%s: the values of a head have to be contiguous, strides %s", name, text(t.strides()).c_str());
  return mma_rows_t{t.data_ptr(), static_cast<uint64_t>(t.stride(0)), static_cast<uint64_t>(t.stride(1))};
}

struct Common {
  const mma_kv_layout_t* layout;
  const mma_kv_seqs_t* seqs;
  Common(PyObject* lay, PyObject* s)
      : layout(static_cast<const mma_kv_layout_t*>(bytes_of(lay, sizeof(mma_kv_layout_t), "layout"))),
        seqs(reinterpret_cast<const mma_kv_seqs_t*>(number(s))) {}
};

struct Queries {
  const at::Tensor& t;
  at::ScalarType type;
  uint32_t kind, cache;
  at::ScalarType cache_type;
  int64_t n, heads;
  Queries(PyObject* q, const mma_kv_layout_t* l) : t(tensor(q, "q")), type(t.scalar_type()) {
    if ((type != at::kBFloat16 && type != at::kHalf) || t.dim() != 3 || t.size(2) != l->head_dim)
      REFUSE("q: [tokens][heads][%u] of bfloat16 or float16 is wanted, got %s %s", l->head_dim, c10::toString(type), text(t.sizes()).c_str());
    kind = type == at::kBFloat16 ? MMA_TYPE_BF16 : MMA_TYPE_F16;
    cache = l->elem_bytes == 1 ? MMA_TYPE_F8 : kind;
    cache_type = l->elem_bytes == 1 ? at::kFloat8_e4m3fn : type;
    n = t.size(0);
    heads = t.size(1);
  }
};

at::Tensor fresh(at::IntArrayRef sizes, at::ScalarType type, const at::Tensor& like) {
  return at::empty(sizes, like.options().dtype(type));
}

PyObject* append(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  HANDLE_TH_ERRORS
  if (nargs != 16) REFUSE("16 arguments");
  const Common c(a[0], a[2]);
  const Queries q(a[3], c.layout);
  const int64_t H = c.layout->kv_heads, D = c.layout->head_dim;
  const at::Tensor out = a[8] == Py_None ? fresh(q.t.sizes(), q.type, q.t) : tensor(a[8], "q_out");
  mma_kv_append_t x{};
  x.q = rows(q.t, "q", q.type, q.n, q.heads, D);
  x.k = rows(tensor(a[4], "k"), "k", q.type, q.n, H, D);
  x.v = rows(tensor(a[5], "v"), "v", q.type, q.n, H, D);
  x.q_out = rows(out, "q_out", q.type, q.n, q.heads, D);
  if (a[7] != Py_None) {
    const at::Tensor& t = flat(a[7], "rope", at::kFloat, {-1, -1});
    if (a[6] == Py_None) REFUSE("rope without positions");
    x.positions = flat_ptr<int32_t>(a[6], "positions", at::kInt, {q.n});
    x.rope = static_cast<const float*>(t.data_ptr());
    x.rope_rows = size32(t.size(0), "rope");
    x.rot_dim = size32(t.size(1), "rope");
  }
  x.interleaved = truth(a[9]);
  x.q_weight = flat_ptr<void>(a[10], "q_weight", q.type, {D});
  x.k_weight = flat_ptr<void>(a[11], "k_weight", q.type, {D});
  x.eps = static_cast<float>(real(a[12]));
  x.k_scale = flat_ptr<float>(a[13], "k_scale", at::kFloat, {H});
  x.v_scale = flat_ptr<float>(a[14], "v_scale", at::kFloat, {H});
  x.num_tokens = size32(q.n, "q");
  x.q_heads = size32(q.heads, "q");
  x.type = q.kind;
  x.cache_type = q.cache;
  check(g_append(c.layout, layer(a[1], q.cache_type), c.seqs, &x, reinterpret_cast<void*>(number(a[15]))), "mma_kv_append");
  return THPVariable_Wrap(out);
  } catch (const Refused&) {
    return nullptr;
  END_HANDLE_TH_ERRORS
}

PyObject* attention(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  HANDLE_TH_ERRORS
  if (nargs != 15) REFUSE("15 arguments");
  const Common c(a[0], a[2]);
  const Queries q(a[3], c.layout);
  const int64_t H = c.layout->kv_heads, D = c.layout->head_dim;
  const at::Tensor out = a[4] == Py_None ? fresh(q.t.sizes(), q.type, q.t) : tensor(a[4], "out");
  mma_kv_attention_t x{};
  x.q = rows(q.t, "q", q.type, q.n, q.heads, D);
  x.out = rows(out, "out", q.type, q.n, q.heads, D);
  x.scale = a[5] == Py_None ? static_cast<float>(1.0 / std::sqrt(static_cast<double>(D))) : static_cast<float>(real(a[5]));
  if (a[6] != Py_None) {
    const at::Tensor& t = flat(a[6], "tree", at::kLong, {q.n, -1});
    x.tree = static_cast<const uint64_t*>(t.data_ptr());
    x.tree_words = size32(t.size(1), "tree");
  }
  x.lse = flat_ptr<float>(a[7], "lse", at::kFloat, {q.n, q.heads});
  if (a[9] != Py_None) {
    const at::Tensor& t = flat(a[9], "scores_out", at::kFloat, {c.seqs->num_seqs, H, -1});
    x.scores_out = static_cast<float*>(t.data_ptr());
    x.scores_stride = size32(t.size(2), "scores_out");
    x.scores_in = flat_ptr<float>(a[8], "scores_in", at::kFloat, {c.seqs->num_seqs, H, t.size(2)});
  } else if (a[8] != Py_None) {
    REFUSE("scores_in without scores_out");
  }
  x.decay = static_cast<float>(real(a[10]));
  x.k_scale = flat_ptr<float>(a[11], "k_scale", at::kFloat, {H});
  x.v_scale = flat_ptr<float>(a[12], "v_scale", at::kFloat, {H});
  x.num_tokens = size32(q.n, "q");
  x.q_heads = size32(q.heads, "q");
  x.type = q.kind;
  x.cache_type = q.cache;
  at::Tensor own;
  if (a[13] != Py_None) {
    const at::Tensor& t = flat(a[13], "workspace", at::kByte, {-1});
    x.workspace = t.data_ptr();
    x.workspace_bytes = t.numel();
  } else {
    check(g_attention_workspace(c.layout, c.seqs, &x, &x.workspace_bytes), "mma_kv_attention_workspace");
    if (x.workspace_bytes) {
      own = fresh({static_cast<int64_t>(x.workspace_bytes)}, at::kByte, q.t);
      x.workspace = own.data_ptr();
    }
  }
  check(g_attention(c.layout, layer(a[1], q.cache_type), c.seqs, &x, reinterpret_cast<void*>(number(a[14]))), "mma_kv_attention");
  return THPVariable_Wrap(out);
  } catch (const Refused&) {
    return nullptr;
  END_HANDLE_TH_ERRORS
}

PyObject* commit(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  HANDLE_TH_ERRORS
  if (nargs != 9) REFUSE("9 arguments");
  const Common c(a[0], a[2]);
  const int64_t S = c.seqs->num_seqs;
  const Py_ssize_t table = static_cast<Py_ssize_t>(sizeof(void*)) * c.layout->num_layers;
  const at::Tensor& acc = flat(a[3], "accepted", at::kInt, {S, -1});
  const at::Tensor lens = a[7] == Py_None ? fresh({S}, at::kInt, acc) : flat(a[7], "lens", at::kInt, {S});
  mma_kv_commit_t x{};
  x.accepted = static_cast<const int32_t*>(acc.data_ptr());
  x.accepted_stride = size32(acc.size(1), "accepted");
  x.counts = flat_ptr<int32_t>(a[4], "counts", at::kInt, {S});
  x.lens_out = static_cast<int32_t*>(lens.data_ptr());
  if (a[5] != Py_None) {
    x.scores = static_cast<float* const*>(bytes_of(a[5], table, "scores"));
    x.scores_stride = count(a[6], "scores_stride");
  }
  void* const* layers = static_cast<void* const*>(bytes_of(a[1], table, "layers"));
  check(g_commit(c.layout, layers, c.seqs, &x, reinterpret_cast<void*>(number(a[8]))), "mma_kv_commit");
  return THPVariable_Wrap(lens);
  } catch (const Refused&) {
    return nullptr;
  END_HANDLE_TH_ERRORS
}

PyObject* evict(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  HANDLE_TH_ERRORS
  if (nargs != 13) REFUSE("13 arguments");
  const Common c(a[0], a[2]);
  const int64_t S = c.seqs->num_seqs, H = c.layout->kv_heads;
  const at::Tensor& dst = flat(a[3], "dst_table", at::kInt, {S, -1});
  const at::Tensor& scores = flat(a[4], "scores", at::kFloat, {S, H, -1});
  mma_kv_evict_t x{};
  x.keep = count(a[5], "keep");
  if (!x.keep) REFUSE("keep: at least 1");
  x.sinks = count(a[6], "sinks");
  x.recent = count(a[7], "recent");
  const at::Tensor entries = a[8] == Py_None ? fresh({S, H, x.keep}, at::kInt, scores) : flat(a[8], "entries", at::kInt, {S, H, x.keep});
  const at::Tensor kept = a[9] == Py_None ? fresh({S, H, x.keep}, at::kFloat, scores) : flat(a[9], "scores kept", at::kFloat, {S, H, x.keep});
  const at::Tensor lens = a[10] == Py_None ? fresh({S}, at::kInt, scores) : flat(a[10], "lens", at::kInt, {S});
  x.dst_table = static_cast<const int32_t*>(dst.data_ptr());
  x.dst_stride = size32(dst.size(1), "dst_table");
  x.scores = static_cast<const float*>(scores.data_ptr());
  x.scores_stride = size32(scores.size(2), "scores");
  x.entries = static_cast<int32_t*>(entries.data_ptr());
  x.scores_out = static_cast<float*>(kept.data_ptr());
  x.lens_out = static_cast<int32_t*>(lens.data_ptr());
  at::Tensor own;
  if (a[11] != Py_None) {
    const at::Tensor& t = flat(a[11], "workspace", at::kByte, {-1});
    x.workspace = t.data_ptr();
    x.workspace_bytes = t.numel();
  } else {
    check(g_evict_workspace(c.layout, c.seqs, &x.workspace_bytes), "mma_kv_evict_workspace");
    own = fresh({static_cast<int64_t>(x.workspace_bytes)}, at::kByte, scores);
    x.workspace = own.data_ptr();
  }
  check(g_evict(c.layout, address(a[1]), c.seqs, &x, reinterpret_cast<void*>(number(a[12]))), "mma_kv_evict");
  PyObject* r = PyTuple_New(3);
  if (!r) return nullptr;
  PyTuple_SET_ITEM(r, 0, THPVariable_Wrap(entries));
  PyTuple_SET_ITEM(r, 1, THPVariable_Wrap(kept));
  PyTuple_SET_ITEM(r, 2, THPVariable_Wrap(lens));
  return r;
  } catch (const Refused&) {
    return nullptr;
  END_HANDLE_TH_ERRORS
}

// The library's entry points and the two Python helpers.
PyObject* attach(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  if (nargs != 8) {
    PyErr_SetString(PyExc_ValueError, "8 arguments");
    return nullptr;
  }
  void* p[6];
  for (int i = 0; i < 6; ++i) {
    p[i] = PyLong_AsVoidPtr(a[i]);
    if (!p[i]) return PyErr_Occurred() ? nullptr : (PyErr_SetString(PyExc_ValueError, "NULL entry point"), nullptr);
  }
  g_append = reinterpret_cast<decltype(g_append)>(p[0]);
  g_attention = reinterpret_cast<decltype(g_attention)>(p[1]);
  g_attention_workspace = reinterpret_cast<decltype(g_attention_workspace)>(p[2]);
  g_commit = reinterpret_cast<decltype(g_commit)>(p[3]);
  g_evict = reinterpret_cast<decltype(g_evict)>(p[4]);
  g_evict_workspace = reinterpret_cast<decltype(g_evict_workspace)>(p[5]);
  Py_INCREF(a[6]);
  g_check = a[6];
  Py_INCREF(a[7]);
  g_address = a[7];
  Py_RETURN_NONE;
}

#define METHOD(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(&name)), METH_FASTCALL, nullptr}
PyMethodDef g_methods[] = {METHOD(attach), METHOD(append), METHOD(attention), METHOD(commit), METHOD(evict), {nullptr, nullptr, 0, nullptr}};
PyModuleDef g_module = {PyModuleDef_HEAD_INIT, "_kv_ops", nullptr, -1, g_methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__kv_ops() { return PyModule_Create(&g_module); }
