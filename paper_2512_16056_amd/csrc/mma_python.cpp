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
decltype(&mma_kv_attention_shaped) g_attention_shaped;
decltype(&mma_kv_attention_shaped_workspace) g_attention_shaped_workspace;
decltype(&mma_kv_commit) g_commit;
decltype(&mma_kv_evict) g_evict;
decltype(&mma_kv_evict_workspace) g_evict_workspace;
decltype(&mma_beam_select) g_beam_select;
decltype(&mma_beam_select_workspace) g_beam_select_workspace;
decltype(&mma_kv_fork) g_fork;
decltype(&mma_kv_fork_workspace) g_fork_workspace;
decltype(&mma_kv_compact) g_compact;
decltype(&mma_kv_compact_workspace) g_compact_workspace;
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
  if (nargs != 20) REFUSE("20 arguments");
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
  mma_kv_shape_t shape{};
  const double cap = real(a[15]);
  shape.softcap = static_cast<float>(cap);
  if (cap != 0 && shape.softcap == 0) shape.softcap = -1.0f;  // too small a number is refused, not taken for none
  shape.window = count(a[16], "window");
  shape.slopes = flat_ptr<float>(a[17], "slopes", at::kFloat, {q.heads});
  shape.prefix = flat_ptr<int32_t>(a[18], "prefix", at::kInt, {c.seqs->num_seqs});
  shape.max_prefix = a[19] == Py_None ? c.seqs->max_len : count(a[19], "max_prefix");
  const bool shaped = shape.softcap != 0 || shape.window || a[17] != Py_None || a[18] != Py_None;
  at::Tensor own;
  if (a[13] != Py_None) {
    const at::Tensor& t = flat(a[13], "workspace", at::kByte, {-1});
    x.workspace = t.data_ptr();
    x.workspace_bytes = t.numel();
  } else {
    if (shaped)
      check(g_attention_shaped_workspace(c.layout, c.seqs, &x, &shape, &x.workspace_bytes), "mma_kv_attention_shaped_workspace");
    else
      check(g_attention_workspace(c.layout, c.seqs, &x, &x.workspace_bytes), "mma_kv_attention_workspace");
    if (x.workspace_bytes) {
      own = fresh({static_cast<int64_t>(x.workspace_bytes)}, at::kByte, q.t);
      x.workspace = own.data_ptr();
    }
  }
  void* const stream = reinterpret_cast<void*>(number(a[14]));
  if (shaped)
    check(g_attention_shaped(c.layout, layer(a[1], q.cache_type), c.seqs, &x, &shape, stream), "mma_kv_attention_shaped");
  else
    check(g_attention(c.layout, layer(a[1], q.cache_type), c.seqs, &x, stream), "mma_kv_attention");
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

// A workspace that was given, or a new one.
struct Space {
  at::Tensor own;
  void* p = nullptr;
  uint64_t bytes = 0;
  template <class Need>
  Space(PyObject* given, const at::Tensor& like, Need need) {
    if (given != Py_None) {
      const at::Tensor& t = flat(given, "workspace", at::kByte, {-1});
      p = t.data_ptr();
      bytes = t.numel();
      return;
    }
    bytes = need();
    if (!bytes) return;
    own = fresh({static_cast<int64_t>(bytes)}, at::kByte, like);
    p = own.data_ptr();
  }
};

at::Tensor given_or(PyObject* o, const char* name, at::ScalarType type, std::initializer_list<int64_t> sizes, const at::Tensor& like) {
  return o == Py_None ? fresh(at::IntArrayRef(sizes), type, like) : flat(o, name, type, sizes);
}

PyObject* tuple_of(std::initializer_list<at::Tensor> tensors) {
  PyObject* r = PyTuple_New(static_cast<Py_ssize_t>(tensors.size()));
  if (!r) throw Refused();
  Py_ssize_t i = 0;
  for (const at::Tensor& t : tensors) PyTuple_SET_ITEM(r, i++, THPVariable_Wrap(t));
  return r;
}

PyObject* beam_select(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  HANDLE_TH_ERRORS
  if (nargs != 10) REFUSE("10 arguments");
  const at::Tensor& x = tensor(a[0], "logits");
  const at::Tensor& scores = flat(a[1], "scores", at::kFloat, {-1, -1});
  const int64_t batch = scores.size(0), beams = scores.size(1);
  mma_beam_select_t b{};
  if (x.scalar_type() == at::kBFloat16) b.type = MMA_TYPE_BF16;
  else if (x.scalar_type() == at::kHalf) b.type = MMA_TYPE_F16;
  else if (x.scalar_type() == at::kFloat) b.type = MMA_TYPE_F32;
  else REFUSE("logits: bfloat16, float16 or float32 is wanted, got %s", c10::toString(x.scalar_type()));
  const bool rows = x.dim() == 2 && x.size(0) == batch * beams;
  const bool items = x.dim() == 3 && x.size(0) == batch && x.size(1) == beams;
  if (!x.is_cuda() || !(rows || items))
    REFUSE("logits: [%lld, vocabulary] or [%lld, %lld, vocabulary] on the GPU is wanted, got %s on %s", static_cast<long long>(batch * beams),
           static_cast<long long>(batch), static_cast<long long>(beams), text(x.sizes()).c_str(), x.device().str().c_str());
  const int64_t vocab = x.size(x.dim() - 1);
  if (vocab > 1 && x.stride(x.dim() - 1) != 1) REFUSE("logits: a row's values have to be contiguous, strides %s", text(x.strides()).c_str());
  if (items && batch > 1 && beams > 1 && x.stride(0) != x.stride(1) * beams)
    REFUSE("logits: rows at one distance are wanted, strides %s", text(x.strides()).c_str());
  b.row_stride = static_cast<uint64_t>(rows ? x.stride(0) : beams > 1 ? x.stride(1) : x.stride(0));
  b.keep = count(a[2], "keep");
  if (!b.keep) REFUSE("keep: at least 1");
  if (a[3] != Py_None) {
    const at::Tensor& d = tensor(a[3], "done");
    b.done = static_cast<const uint8_t*>(flat(a[3], "done", d.scalar_type() == at::kBool ? at::kBool : at::kByte, {batch, beams}).data_ptr());
  }
  const double token = real(a[4]);
  if (!(token >= -2147483648.0 && token <= 2147483647.0 && token == std::floor(token))) REFUSE("done_token: a token is wanted");
  b.done_token = static_cast<int32_t>(token);
  b.logits = x.data_ptr();
  b.scores = static_cast<const float*>(scores.data_ptr());
  b.batch = size32(batch, "scores");
  b.beams = size32(beams, "scores");
  b.vocab = size32(vocab, "logits");
  const int64_t keep = b.keep;
  const at::Tensor tokens = given_or(a[5], "tokens", at::kInt, {batch, keep}, scores);
  const at::Tensor parents = given_or(a[6], "parents", at::kInt, {batch, keep}, scores);
  const at::Tensor best = given_or(a[7], "scores_out", at::kFloat, {batch, keep}, scores);
  b.tokens = static_cast<int32_t*>(tokens.data_ptr());
  b.parents = static_cast<int32_t*>(parents.data_ptr());
  b.scores_out = static_cast<float*>(best.data_ptr());
  const Space space(a[8], scores, [&] {
    uint64_t need = 0;
    check(g_beam_select_workspace(&b, &need), "mma_beam_select_workspace");
    return need;
  });
  b.workspace = space.p;
  b.workspace_bytes = space.bytes;
  check(g_beam_select(&b, reinterpret_cast<void*>(number(a[9]))), "mma_beam_select");
  return tuple_of({tokens, parents, best});
  } catch (const Refused&) {
    return nullptr;
  END_HANDLE_TH_ERRORS
}

PyObject* fork(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  HANDLE_TH_ERRORS
  if (nargs != 13) REFUSE("13 arguments");
  const Common c(a[0], a[2]);
  const Py_ssize_t table = static_cast<Py_ssize_t>(sizeof(void*)) * c.layout->num_layers;
  const at::Tensor& parents = flat(a[3], "parents", at::kInt, {-1});
  const int64_t n = parents.size(0), blocks = c.layout->gpu_num_blocks;
  const at::Tensor& refs = flat(a[4], "refs", at::kInt, {blocks});
  const int64_t width = a[6] == Py_None ? static_cast<int64_t>(c.seqs->table_stride) : count(a[6], "width");
  mma_kv_fork_t x{};
  x.parents = static_cast<const int32_t*>(parents.data_ptr());
  x.grow = flat_ptr<int32_t>(a[5], "grow", at::kInt, {n});
  x.refs = static_cast<const int32_t*>(refs.data_ptr());
  x.num_children = size32(n, "parents");
  x.out_stride = static_cast<uint32_t>(width);
  const at::Tensor out = given_or(a[7], "table", at::kInt, {n, width}, refs);
  const at::Tensor lens = given_or(a[8], "lens", at::kInt, {n}, refs);
  const at::Tensor counts = given_or(a[9], "refs_out", at::kInt, {blocks}, refs);
  const at::Tensor left = given_or(a[10], "free", at::kInt, {1}, refs);
  x.table_out = static_cast<int32_t*>(out.data_ptr());
  x.lens_out = static_cast<int32_t*>(lens.data_ptr());
  x.refs_out = static_cast<int32_t*>(counts.data_ptr());
  x.free_out = static_cast<int32_t*>(left.data_ptr());
  const Space space(a[11], refs, [&] {
    uint64_t need = 0;
    check(g_fork_workspace(&x, &need), "mma_kv_fork_workspace");
    return need;
  });
  x.workspace = space.p;
  x.workspace_bytes = space.bytes;
  void* const* layers = static_cast<void* const*>(bytes_of(a[1], table, "layers"));
  check(g_fork(c.layout, layers, c.seqs, &x, reinterpret_cast<void*>(number(a[12]))), "mma_kv_fork");
  return tuple_of({out, lens, counts, left});
  } catch (const Refused&) {
    return nullptr;
  END_HANDLE_TH_ERRORS
}

PyObject* compact(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  HANDLE_TH_ERRORS
  if (nargs != 10) REFUSE("10 arguments");
  const mma_kv_layout_t* layout = static_cast<const mma_kv_layout_t*>(bytes_of(a[0], sizeof(mma_kv_layout_t), "layout"));
  const at::Tensor& table = flat(a[2], "table", at::kInt, {-1, -1});
  const int64_t blocks = layout->gpu_num_blocks;
  const at::Tensor& refs = flat(a[3], "refs", at::kInt, {blocks});
  mma_kv_compact_t x{};
  x.block_table = static_cast<const int32_t*>(table.data_ptr());
  x.num_seqs = size32(table.size(0), "table");
  x.table_stride = size32(table.size(1), "table");
  x.refs = static_cast<const int32_t*>(refs.data_ptr());
  const at::Tensor out = given_or(a[4], "table_out", at::kInt, {table.size(0), table.size(1)}, refs);
  const at::Tensor counts = given_or(a[5], "refs_out", at::kInt, {blocks}, refs);
  const at::Tensor moved = given_or(a[6], "moved", at::kInt, {blocks}, refs);
  const at::Tensor held = given_or(a[7], "held", at::kInt, {1}, refs);
  x.table_out = static_cast<int32_t*>(out.data_ptr());
  x.refs_out = static_cast<int32_t*>(counts.data_ptr());
  x.moved = static_cast<int32_t*>(moved.data_ptr());
  x.held_out = static_cast<int32_t*>(held.data_ptr());
  const Space space(a[8], refs, [&] {
    uint64_t need = 0;
    check(g_compact_workspace(layout, &need), "mma_kv_compact_workspace");
    return need;
  });
  x.workspace = space.p;
  x.workspace_bytes = space.bytes;
  void* const* layers = static_cast<void* const*>(bytes_of(a[1], static_cast<Py_ssize_t>(sizeof(void*)) * layout->num_layers, "layers"));
  check(g_compact(layout, layers, &x, reinterpret_cast<void*>(number(a[9]))), "mma_kv_compact");
  return tuple_of({out, counts, moved, held});
  } catch (const Refused&) {
    return nullptr;
  END_HANDLE_TH_ERRORS
}

// The library's entry points and the two Python helpers.
PyObject* attach(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  constexpr int kEntries = 14;
  if (nargs != kEntries + 2) {
    PyErr_SetString(PyExc_ValueError, "the entry points and two helpers");
    return nullptr;
  }
  void* p[kEntries];
  for (int i = 0; i < kEntries; ++i) {
    p[i] = PyLong_AsVoidPtr(a[i]);
    if (!p[i]) return PyErr_Occurred() ? nullptr : (PyErr_SetString(PyExc_ValueError, "NULL entry point"), nullptr);
  }
  g_append = reinterpret_cast<decltype(g_append)>(p[0]);
  g_attention = reinterpret_cast<decltype(g_attention)>(p[1]);
  g_attention_workspace = reinterpret_cast<decltype(g_attention_workspace)>(p[2]);
  g_commit = reinterpret_cast<decltype(g_commit)>(p[3]);
  g_evict = reinterpret_cast<decltype(g_evict)>(p[4]);
  g_evict_workspace = reinterpret_cast<decltype(g_evict_workspace)>(p[5]);
  g_attention_shaped = reinterpret_cast<decltype(g_attention_shaped)>(p[6]);
  g_attention_shaped_workspace = reinterpret_cast<decltype(g_attention_shaped_workspace)>(p[7]);
  g_beam_select = reinterpret_cast<decltype(g_beam_select)>(p[8]);
  g_beam_select_workspace = reinterpret_cast<decltype(g_beam_select_workspace)>(p[9]);
  g_fork = reinterpret_cast<decltype(g_fork)>(p[10]);
  g_fork_workspace = reinterpret_cast<decltype(g_fork_workspace)>(p[11]);
  g_compact = reinterpret_cast<decltype(g_compact)>(p[12]);
  g_compact_workspace = reinterpret_cast<decltype(g_compact_workspace)>(p[13]);
  Py_INCREF(a[kEntries]);
  g_check = a[kEntries];
  Py_INCREF(a[kEntries + 1]);
  g_address = a[kEntries + 1];
  Py_RETURN_NONE;
}

#define METHOD(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(&name)), METH_FASTCALL, nullptr}
PyMethodDef g_methods[] = {METHOD(attach), METHOD(append), METHOD(attention), METHOD(commit), METHOD(evict),
                          METHOD(beam_select), METHOD(fork), METHOD(compact), {nullptr, nullptr, 0, nullptr}};
PyModuleDef g_module = {PyModuleDef_HEAD_INIT, "_kv_ops", nullptr, -1, g_methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__kv_ops() { return PyModule_Create(&g_module); }
