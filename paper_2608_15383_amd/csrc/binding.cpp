// Compiled half of the Python binding of exactmoe_serving.h and exactmoe_drafts.h:
// takes tensors, checks what the library cannot see in a pointer (types, shapes, strides,
// devices) and calls the C entry points, whose addresses and whose exception
// class Python hands over once (init).  Marshalling only.  A decode step's calls
// take 3 to 15 us on the GPU, and the same checks in Python took 5 to 8 us of a
// call, here less than one.
#include <Python.h>

#include <c10/core/DeviceGuard.h>
#include <torch/csrc/autograd/python_variable.h>

#include <initializer_list>
#include <stdexcept>
#include <string>
#include <vector>

#include "exactmoe_drafts.h"

namespace {

PyObject* g_error = nullptr;  // ExactMoEError(status, message)
decltype(&emoe_paged_append) g_append = nullptr;
decltype(&emoe_paged_attention) g_attention = nullptr;
decltype(&emoe_process_logits) g_logits = nullptr;
decltype(&emoe_decoder_forward_paged) g_decoder = nullptr;
decltype(&emoe_paged_append_axes) g_append_axes = nullptr;
decltype(&emoe_paged_tree_attention) g_tree = nullptr;
decltype(&emoe_accept_drafts) g_accept = nullptr;
decltype(&emoe_paged_compact) g_compact = nullptr;
decltype(&emoe_paged_fork) g_fork = nullptr;
decltype(&emoe_last_error) g_last_error = nullptr;

struct Refused : std::runtime_error {
  using std::runtime_error::runtime_error;
};

[[noreturn]] void refuse(const std::string& message) { throw Refused(message); }

enum Kind { kI32 = -1, kF64 = -2, kI64 = -3 };  // besides emoe_dtype

// The emoe_dtype of a tensor; 16-bit patterns without a type of their own are bf16.
int type_of(const at::Tensor& t, const char* name) {
  switch (t.scalar_type()) {
    case at::kFloat: return EMOE_F32;
    case at::kBFloat16:
    case at::kShort:
    case at::kUInt16: return EMOE_BF16;
    case at::kHalf: return EMOE_F16;
    case at::kFloat8_e4m3fn: return EMOE_E4M3;
    case at::kInt:
    case at::kUInt32: return kI32;
    case at::kDouble: return kF64;
    case at::kLong:
    case at::kUInt64: return kI64;
    default: refuse(std::string(name) + ": type " + c10::toString(t.scalar_type()) + " is not supported");
  }
}

const at::Tensor& tensor(PyObject* o, const char* name) {
  if (!THPVariable_Check(o)) refuse(std::string(name) + ": need a tensor");
  return THPVariable_Unpack(o);
}

std::string shape_text(const at::Tensor& t) {
  std::string s = "(";
  for (int64_t n : t.sizes()) s += std::to_string(n) + ", ";
  return s + ")";
}

constexpr int64_t kAny = -1;

// An optional tensor of this type, shape and device, dense along its last axis.
const at::Tensor* array(PyObject* o, const char* name, int type, std::initializer_list<int64_t> shape,
                        int device) {
  if (o == Py_None) return nullptr;
  const at::Tensor& t = tensor(o, name);
  if (type_of(t, name) != type)
    refuse(std::string(name) + ": type " + c10::toString(t.scalar_type()) + " does not fit");
  if (!t.is_cuda() || t.device().index() != device)
    refuse(std::string(name) + " is on " + t.device().str() + ", not on cuda:" + std::to_string(device));
  bool fits = t.dim() == (int64_t)shape.size();
  int64_t i = 0;
  for (int64_t want : shape) {
    fits = fits && (want == kAny || t.size(i) == want);
    ++i;
  }
  if (!fits) {
    std::string want = "(";
    for (int64_t n : shape) want += (n == kAny ? std::string("*") : std::to_string(n)) + ", ";
    refuse(std::string(name) + ": shape " + shape_text(t) + ", need " + want + ")");
  }
  if (t.size(-1) > 1 && t.stride(-1) != 1 && t.numel())
    refuse(std::string(name) + ": the last axis must be dense");
  return &t;
}

const at::Tensor& need(const at::Tensor* t, const char* name) {
  if (!t) refuse(std::string(name) + " is missing");
  return *t;
}

template <class T>
T* pointer(const at::Tensor* t) {
  return t ? static_cast<T*>(t->data_ptr()) : nullptr;
}

// [rows][heads][dim] with dense rows.
const at::Tensor& head_rows(PyObject* o, const char* name, int type, int64_t rows, int64_t heads,
                            int64_t dim, int device) {
  const at::Tensor& t = need(array(o, name, type, {rows, heads, dim}, device), name);
  if (heads > 1 && rows > 0 && t.stride(1) != dim)
    refuse(std::string(name) + ": the heads of a row must be dense");
  return t;
}

int32_t i32(int64_t v, const char* name) {
  if (v < INT32_MIN || v > INT32_MAX) refuse(std::string(name) + " of " + std::to_string(v) + " is out of range");
  return (int32_t)v;
}

int64_t number(PyObject* o, const char* name) {
  const long long v = PyLong_AsLongLong(o);
  if (v == -1 && PyErr_Occurred()) {
    PyErr_Clear();
    refuse(std::string(name) + ": need a whole number");
  }
  return v;
}

struct Workspace {
  void* p = nullptr;
  size_t bytes = 0;
  Workspace(PyObject* o, int device) {
    if (o == Py_None) return;
    const at::Tensor& t = tensor(o, "workspace");
    if (!t.is_cuda() || t.device().index() != device || !t.is_contiguous())
      refuse("workspace must be contiguous and on cuda:" + std::to_string(device));
    p = t.data_ptr();
    bytes = t.nbytes();
  }
};

// A PagedKV as Python hands it over: the address of its emoe_paged_kv and its device.
struct Kv {
  const emoe_paged_kv* view;
  int device;
  Kv(PyObject* address, PyObject* index)
      : view(reinterpret_cast<const emoe_paged_kv*>(number(address, "kv"))),
        device((int)number(index, "device")) {}
};

hipStream_t stream_of(PyObject* o) {
  return reinterpret_cast<hipStream_t>((uintptr_t)number(o, "stream"));
}

PyObject* done(int32_t status) {
  if (status == EMOE_OK) Py_RETURN_NONE;
  PyObject* args = Py_BuildValue("(is)", (int)status, g_last_error());
  if (args) {
    PyErr_SetObject(g_error, args);
    Py_DECREF(args);
  }
  return nullptr;
}

// Runs a call with `device` current; nothing is thrown past it.
template <class Call>
PyObject* guarded(Call call) {
  try {
    return done(call());
  } catch (const Refused& e) {
    PyObject* args = Py_BuildValue("(is)", (int)EMOE_EINVAL, e.what());
    if (args) {
      PyErr_SetObject(g_error, args);
      Py_DECREF(args);
    }
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
  } catch (...) {
    PyErr_SetString(PyExc_RuntimeError, "unknown exception");
  }
  return nullptr;
}

template <class Fn, class... Args>
int32_t on_device(int device, Fn fn, Args... args) {
  const c10::DeviceGuard guard(c10::Device(c10::DeviceType::CUDA, (c10::DeviceIndex)device));
  int32_t status;
  Py_BEGIN_ALLOW_THREADS
  status = fn(args...);
  Py_END_ALLOW_THREADS
  return status;
}

// What the appends have in common: (kv, device, q, k, v, positions, page_table, inv_freq, seqs, q_out,
// interleaved).
emoe_paged_append_args append_args(const Kv& kv, PyObject* const* a) {
  const int64_t hk = kv.view->n_kv_heads, d = kv.view->head_dim;
  const at::Tensor& k0 = tensor(a[3], "k");
  const int type = type_of(k0, "k");
  const int64_t n = k0.dim() ? k0.size(0) : 0;
  const at::Tensor& k = head_rows(a[3], "k", type, n, hk, d, kv.device);
  const at::Tensor& v = head_rows(a[4], "v", type, n, hk, d, kv.device);
  emoe_paged_append_args A{};
  A.k = k.data_ptr();
  A.k_stride = k.stride(0);
  A.v = v.data_ptr();
  A.v_stride = v.stride(0);
  if (a[2] != Py_None) {
    const at::Tensor& q0 = tensor(a[2], "q");
    const int64_t heads = q0.dim() == 3 ? q0.size(1) : 0;
    const at::Tensor& q = head_rows(a[2], "q", type, n, heads, d, kv.device);
    const at::Tensor& q_out = a[9] == Py_None ? q : head_rows(a[9], "q_out", type, n, heads, d, kv.device);
    A.q = q.data_ptr();
    A.q_stride = q.stride(0);
    A.q_out = q_out.data_ptr();
    A.q_out_stride = q_out.stride(0);
    A.n_heads = i32(heads, "heads");
  }
  A.positions = pointer<const int32_t>(&need(array(a[5], "positions", kI32, {n}, kv.device), "positions"));
  const at::Tensor& table = need(array(a[6], "page_table", kI32, {kAny, kAny}, kv.device), "page_table");
  const at::Tensor* freq = array(a[7], "inv_freq", kF64, {kAny}, kv.device);
  A.inv_freq = pointer<const double>(freq);
  A.seqs = pointer<const int32_t>(array(a[8], "seqs", kI32, {n}, kv.device));
  A.page_table = pointer<const int32_t>(&table);
  A.table_stride = table.stride(0);
  A.dtype = type;
  A.tokens = i32(n, "tokens");
  A.n_seqs = i32(table.size(0), "sequences");
  A.table_width = i32(table.size(1), "page_table");
  A.rotary_dim = freq ? i32(2 * freq->size(0), "inv_freq") : 0;
  A.interleaved = PyObject_IsTrue(a[10]);
  if (A.interleaved < 0) {
    PyErr_Clear();
    refuse("interleaved: need True or False");
  }
  return A;
}

// (kv .. interleaved, stream)
PyObject* paged_append(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  return guarded([&]() -> int32_t {
    if (n_args != 12) refuse("paged_append: 12 arguments");
    const Kv kv(a[0], a[1]);
    const emoe_paged_append_args A = append_args(kv, a);
    return on_device(kv.device, g_append, kv.view, &A, stream_of(a[11]));
  });
}

// (kv .. interleaved, angles, axes, stream)
PyObject* paged_append_axes(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  return guarded([&]() -> int32_t {
    if (n_args != 14) refuse("paged_append_axes: 14 arguments");
    const Kv kv(a[0], a[1]);
    const emoe_paged_append_args A = append_args(kv, a);
    const at::Tensor& angles = need(array(a[11], "angles", kI32, {A.tokens, kAny}, kv.device), "angles");
    emoe_paged_axes X{};
    X.angles = pointer<const int32_t>(&angles);
    X.axes = pointer<const int32_t>(array(a[12], "axes", kI32, {A.rotary_dim / 2}, kv.device));
    X.angle_stride = angles.stride(0);
    X.n_axes = i32(angles.size(1), "angles");
    return on_device(kv.device, g_append_axes, kv.view, &A, &X, stream_of(a[13]));
  });
}

// (kv, device, q, page_table, lengths, out, workspace, max_keys, seqs, scale, window, lse, stream)
PyObject* paged_attention(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  return guarded([&]() -> int32_t {
    if (n_args != 13) refuse("paged_attention: 13 arguments");
    const Kv kv(a[0], a[1]);
    const at::Tensor& q0 = tensor(a[2], "q");
    const int type = type_of(q0, "q");
    if (q0.dim() != 3) refuse("q: need 3 axes, got shape " + shape_text(q0));
    const int64_t rows = q0.size(0), heads = q0.size(1), d = kv.view->head_dim;
    const at::Tensor& q = head_rows(a[2], "q", type, rows, heads, d, kv.device);
    const at::Tensor& table = need(array(a[3], "page_table", kI32, {kAny, kAny}, kv.device), "page_table");
    const at::Tensor& out = head_rows(a[5], "out", type, rows, heads, d, kv.device);
    const at::Tensor* lse = array(a[11], "lse", EMOE_F32, {rows, heads}, kv.device);
    if (lse && !lse->is_contiguous()) refuse("lse must be contiguous");
    const Workspace ws(a[6], kv.device);
    emoe_paged_attention_args A{};
    A.q = q.data_ptr();
    A.out = out.data_ptr();
    A.lse = pointer<float>(lse);
    A.lengths = pointer<const int32_t>(&need(array(a[4], "lengths", kI32, {rows}, kv.device), "lengths"));
    A.seqs = pointer<const int32_t>(array(a[8], "seqs", kI32, {rows}, kv.device));
    A.page_table = pointer<const int32_t>(&table);
    A.q_stride = q.stride(0);
    A.out_stride = out.stride(0);
    A.table_stride = table.stride(0);
    const double scale = PyFloat_AsDouble(a[9]);
    if (scale == -1.0 && PyErr_Occurred()) {
      PyErr_Clear();
      refuse("scale: need a number");
    }
    A.scale = (float)scale;
    A.dtype = type;
    A.rows = i32(rows, "rows");
    A.n_heads = i32(heads, "heads");
    A.n_seqs = i32(table.size(0), "sequences");
    A.table_width = i32(table.size(1), "page_table");
    A.max_keys = i32(number(a[7], "max_keys"), "max_keys");
    A.window = i32(number(a[10], "window"), "window");
    return on_device(kv.device, g_attention, kv.view, &A, ws.p, ws.bytes, stream_of(a[12]));
  });
}

// What process_logits and the decoder have in common, from a[0 .. 10]: history, history_lengths,
// prompt_lengths, repetition, presence, frequency, bias_ids, bias_values, bias_counts, mask, mask_rows.
constexpr int kProcessing = 11;
void processing(PyObject* const* a, int64_t rows, int64_t vocab, int device, emoe_logits_args& A) {
  if (const at::Tensor* h = array(a[0], "history", kI32, {rows, kAny}, device)) {
    A.history = pointer<const int32_t>(h);
    A.history_stride = h->stride(0);
    A.history_width = i32(h->size(1), "history");
  }
  A.history_lengths = pointer<const int32_t>(array(a[1], "history_lengths", kI32, {rows}, device));
  A.prompt_lengths = pointer<const int32_t>(array(a[2], "prompt_lengths", kI32, {rows}, device));
  A.repetition = pointer<const float>(array(a[3], "repetition", EMOE_F32, {rows}, device));
  A.presence = pointer<const float>(array(a[4], "presence", EMOE_F32, {rows}, device));
  A.frequency = pointer<const float>(array(a[5], "frequency", EMOE_F32, {rows}, device));
  if (const at::Tensor* ids = array(a[6], "bias_ids", kI32, {rows, kAny}, device)) {
    const at::Tensor& values =
        need(array(a[7], "bias_values", EMOE_F32, {rows, ids->size(1)}, device), "bias_values");
    if (rows > 1 && ids->stride(0) != values.stride(0))
      refuse("bias_ids and bias_values have different row strides");
    A.bias_ids = pointer<const int32_t>(ids);
    A.bias_values = pointer<const float>(&values);
    A.bias_counts = pointer<const int32_t>(array(a[8], "bias_counts", kI32, {rows}, device));
    A.bias_stride = ids->stride(0);
    A.bias_width = i32(ids->size(1), "bias_ids");
  } else if (a[7] != Py_None || a[8] != Py_None) {
    refuse("bias_ids is missing");
  }
  if (const at::Tensor* m = array(a[9], "mask", kI32, {kAny, kAny}, device)) {
    if (m->size(1) * 32 < vocab)
      refuse("mask: " + std::to_string(m->size(1)) + " words for a vocabulary of " + std::to_string(vocab));
    A.mask = pointer<const uint32_t>(m);
    A.mask_stride = m->stride(0);
    A.n_masks = i32(m->size(0), "mask");
  }
  A.mask_rows = pointer<const int32_t>(array(a[10], "mask_rows", kI32, {rows}, device));
}

// (logits, out, workspace, next_token, processing.., stream)
PyObject* process_logits(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  return guarded([&]() -> int32_t {
    if (n_args != 5 + kProcessing) refuse("process_logits: 16 arguments");
    const at::Tensor& x = tensor(a[0], "logits");
    if (!x.is_cuda()) refuse("logits is on " + x.device().str());
    if (x.dim() != 2) refuse("logits: need 2 axes, got shape " + shape_text(x));
    const int device = x.device().index(), type = type_of(x, "logits");
    const int64_t rows = x.size(0), vocab = x.size(1);
    array(a[0], "logits", type, {rows, vocab}, device);
    const at::Tensor* out = array(a[1], "out", type, {rows, vocab}, device);
    if (!out) out = &x;
    const Workspace ws(a[2], device);
    emoe_logits_args A{};
    processing(a + 4, rows, vocab, device, A);
    A.logits = x.data_ptr();
    A.out = out->data_ptr();
    A.next_token = pointer<int32_t>(array(a[3], "next_token", kI32, {rows}, device));
    A.logits_stride = x.stride(0);
    A.out_stride = out->stride(0);
    A.dtype = type;
    A.rows = i32(rows, "rows");
    A.vocab = i32(vocab, "vocab");
    return on_device(device, g_logits, &A, ws.p, ws.bytes, stream_of(a[4 + kProcessing]));
  });
}

// (decoder, kv views, vocab, device, tokens, positions, page_table, logits, workspace, max_keys, seqs,
//  out_rows, next_token, stats or 0, processing.., stream)
PyObject* decoder_forward_paged(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  return guarded([&]() -> int32_t {
    if (n_args != 15 + kProcessing) refuse("decoder_forward_paged: 26 arguments");
    auto* dec = reinterpret_cast<emoe_decoder*>(number(a[0], "decoder"));
    auto* kv = reinterpret_cast<const emoe_paged_kv*>(number(a[1], "kv"));
    const int64_t vocab = number(a[2], "vocab");
    const int device = (int)number(a[3], "device");
    const at::Tensor& tokens = need(array(a[4], "tokens", kI32, {kAny}, device), "tokens");
    const int64_t n = tokens.size(0);
    const at::Tensor& table = need(array(a[6], "page_table", kI32, {kAny, kAny}, device), "page_table");
    const at::Tensor* out_rows = array(a[11], "out_rows", kI32, {kAny}, device);
    const int64_t rows = out_rows ? out_rows->size(0) : n;
    const at::Tensor& logits = need(array(a[7], "logits", EMOE_F32, {rows, vocab}, device), "logits");
    if (!logits.is_contiguous()) refuse("logits must be contiguous");
    const Workspace ws(a[8], device);
    emoe_decoder_batch B{};
    B.tokens = pointer<const int32_t>(&tokens);
    B.positions = pointer<const int32_t>(&need(array(a[5], "positions", kI32, {n}, device), "positions"));
    B.seqs = pointer<const int32_t>(array(a[10], "seqs", kI32, {n}, device));
    B.page_table = pointer<const int32_t>(&table);
    B.out_rows = pointer<const int32_t>(out_rows);
    B.table_stride = table.stride(0);
    B.n_tokens = i32(n, "tokens");
    B.n_seqs = i32(table.size(0), "sequences");
    B.table_width = i32(table.size(1), "page_table");
    B.n_out = i32(rows, "out_rows");
    B.max_keys = i32(number(a[9], "max_keys"), "max_keys");
    emoe_logits_args A{};
    processing(a + 14, rows, vocab, device, A);
    int32_t* next = pointer<int32_t>(array(a[12], "next_token", kI32, {rows}, device));
    auto* stats = reinterpret_cast<emoe_stats*>(number(a[13], "stats"));
    return on_device(device, g_decoder, dec, kv, &B, pointer<float>(&logits), &A, next, ws.p, ws.bytes,
                     stream_of(a[14 + kProcessing]), stats);
  });
}

float real(PyObject* o, const char* name) {
  const double v = PyFloat_AsDouble(o);
  if (v == -1.0 && PyErr_Occurred()) {
    PyErr_Clear();
    refuse(std::string(name) + ": need a number");
  }
  return (float)v;
}

// (kv, device, q, page_table, lengths, out, workspace, max_keys, max_nodes, tree, starts, seqs, scale, cap,
//  slopes, window, lse, stream)
PyObject* paged_tree_attention(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  return guarded([&]() -> int32_t {
    if (n_args != 18) refuse("paged_tree_attention: 18 arguments");
    const Kv kv(a[0], a[1]);
    const at::Tensor& q0 = tensor(a[2], "q");
    const int type = type_of(q0, "q");
    if (q0.dim() != 3) refuse("q: need 3 axes, got shape " + shape_text(q0));
    const int64_t rows = q0.size(0), heads = q0.size(1), d = kv.view->head_dim;
    const at::Tensor& q = head_rows(a[2], "q", type, rows, heads, d, kv.device);
    const at::Tensor& table = need(array(a[3], "page_table", kI32, {kAny, kAny}, kv.device), "page_table");
    const at::Tensor& lengths = need(array(a[4], "lengths", kI32, {kAny}, kv.device), "lengths");
    const int64_t trees = lengths.size(0);
    const at::Tensor& out = head_rows(a[5], "out", type, rows, heads, d, kv.device);
    const at::Tensor* lse = array(a[16], "lse", EMOE_F32, {rows, heads}, kv.device);
    if (lse && !lse->is_contiguous()) refuse("lse must be contiguous");
    const Workspace ws(a[6], kv.device);
    emoe_paged_tree_args A{};
    A.q = q.data_ptr();
    A.out = out.data_ptr();
    A.lse = pointer<float>(lse);
    A.lengths = pointer<const int32_t>(&lengths);
    A.tree = pointer<const uint64_t>(array(a[9], "tree", kI64, {rows}, kv.device));
    A.starts = pointer<const int32_t>(array(a[10], "starts", kI32, {trees + 1}, kv.device));
    A.seqs = pointer<const int32_t>(array(a[11], "seqs", kI32, {trees}, kv.device));
    A.slopes = pointer<const float>(array(a[14], "slopes", EMOE_F32, {heads}, kv.device));
    A.page_table = pointer<const int32_t>(&table);
    A.q_stride = q.stride(0);
    A.out_stride = out.stride(0);
    A.table_stride = table.stride(0);
    A.scale = real(a[12], "scale");
    A.cap = real(a[13], "cap");
    A.dtype = type;
    A.rows = i32(rows, "rows");
    A.trees = i32(trees, "trees");
    A.n_heads = i32(heads, "heads");
    A.n_seqs = i32(table.size(0), "sequences");
    A.table_width = i32(table.size(1), "page_table");
    A.max_keys = i32(number(a[7], "max_keys"), "max_keys");
    A.max_nodes = i32(number(a[8], "max_nodes"), "max_nodes");
    A.window = i32(number(a[15], "window"), "window");
    return on_device(kv.device, g_tree, kv.view, &A, ws.p, ws.bytes, stream_of(a[17]));
  });
}

// (tokens, chosen, lengths, path, accepted, new_tokens, new_lengths, tree, starts, stream)
PyObject* accept_drafts(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  return guarded([&]() -> int32_t {
    if (n_args != 10) refuse("accept_drafts: 10 arguments");
    const at::Tensor& t0 = tensor(a[0], "tokens");
    if (!t0.is_cuda()) refuse("tokens is on " + t0.device().str());
    const int device = t0.device().index();
    const at::Tensor& tokens = need(array(a[0], "tokens", kI32, {kAny}, device), "tokens");
    const int64_t rows = tokens.size(0);
    const at::Tensor& path = need(array(a[3], "path", kI32, {kAny, kAny}, device), "path");
    const int64_t trees = path.size(0), nodes = path.size(1);
    const at::Tensor* made = array(a[5], "new_tokens", kI32, {trees, nodes}, device);
    emoe_accept_args A{};
    A.tokens = pointer<const int32_t>(&tokens);
    A.chosen = pointer<const int32_t>(&need(array(a[1], "chosen", kI32, {rows}, device), "chosen"));
    A.lengths = pointer<const int32_t>(array(a[2], "lengths", kI32, {trees}, device));
    A.path = pointer<int32_t>(&path);
    A.accepted = pointer<int32_t>(&need(array(a[4], "accepted", kI32, {trees}, device), "accepted"));
    A.new_tokens = pointer<int32_t>(made);
    A.new_lengths = pointer<int32_t>(array(a[6], "new_lengths", kI32, {trees}, device));
    A.tree = pointer<const uint64_t>(array(a[7], "tree", kI64, {rows}, device));
    A.starts = pointer<const int32_t>(array(a[8], "starts", kI32, {trees + 1}, device));
    A.path_stride = path.stride(0);
    A.new_tokens_stride = made ? made->stride(0) : 0;
    A.rows = i32(rows, "rows");
    A.trees = i32(trees, "trees");
    A.max_nodes = i32(nodes, "path");
    return on_device(device, g_accept, &A, stream_of(a[9]));
  });
}

// The caches of a sequence of PagedKV (which class that is, Python says), all on `device`.  An address
// is taken from nothing else.
std::vector<emoe_paged_kv> layers(PyObject* o, PyObject* paged_kv, int device) {
  if (!PyList_Check(o) && !PyTuple_Check(o)) refuse("kvs: need a list of PagedKV");
  const Py_ssize_t n = PySequence_Fast_GET_SIZE(o);
  static PyObject* const names[2] = {PyUnicode_InternFromString("address"), PyUnicode_InternFromString("index")};
  std::vector<emoe_paged_kv> out;
  out.reserve((size_t)n);
  for (Py_ssize_t i = 0; i < n; ++i) {
    PyObject* item = PySequence_Fast_GET_ITEM(o, i);
    if (PyObject_IsInstance(item, paged_kv) != 1) {
      PyErr_Clear();
      refuse("kvs: need a list of PagedKV");
    }
    PyObject* address = PyObject_GetAttr(item, names[0]);
    PyObject* index = address ? PyObject_GetAttr(item, names[1]) : nullptr;
    int64_t at = 0, dev = -1;
    const bool good = index && PyLong_Check(address) && PyLong_Check(index);
    if (good) {
      at = PyLong_AsLongLong(address);
      dev = PyLong_AsLongLong(index);
    }
    Py_XDECREF(address);
    Py_XDECREF(index);
    PyErr_Clear();
    if (!good) refuse("kvs: need a list of PagedKV");
    if (dev != device) refuse("kvs: caches on more than one device");
    out.push_back(*reinterpret_cast<const emoe_paged_kv*>(at));
  }
  return out;
}

// (kvs, PagedKV, device, page_table, lengths, path, accepted, seqs, stream)
PyObject* paged_compact(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  return guarded([&]() -> int32_t {
    if (n_args != 9) refuse("paged_compact: 9 arguments");
    const int device = (int)number(a[2], "device");
    const std::vector<emoe_paged_kv> kvs = layers(a[0], a[1], device);
    const at::Tensor& table = need(array(a[3], "page_table", kI32, {kAny, kAny}, device), "page_table");
    const at::Tensor& path = need(array(a[5], "path", kI32, {kAny, kAny}, device), "path");
    const int64_t trees = path.size(0);
    emoe_compact_args A{};
    A.lengths = pointer<const int32_t>(&need(array(a[4], "lengths", kI32, {trees}, device), "lengths"));
    A.path = pointer<const int32_t>(&path);
    A.accepted = pointer<const int32_t>(&need(array(a[6], "accepted", kI32, {trees}, device), "accepted"));
    A.seqs = pointer<const int32_t>(array(a[7], "seqs", kI32, {trees}, device));
    A.page_table = pointer<const int32_t>(&table);
    A.path_stride = path.stride(0);
    A.table_stride = table.stride(0);
    A.trees = i32(trees, "trees");
    A.max_nodes = i32(path.size(1), "path");
    A.n_seqs = i32(table.size(0), "sequences");
    A.table_width = i32(table.size(1), "page_table");
    return on_device(device, g_compact, kvs.data(), (int32_t)kvs.size(), &A, stream_of(a[8]));
  });
}

// (kvs, PagedKV, device, page_table, parents, lengths, fresh, new_table, stream)
PyObject* paged_fork(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  return guarded([&]() -> int32_t {
    if (n_args != 9) refuse("paged_fork: 9 arguments");
    const int device = (int)number(a[2], "device");
    const std::vector<emoe_paged_kv> kvs = layers(a[0], a[1], device);
    const at::Tensor& table = need(array(a[3], "page_table", kI32, {kAny, kAny}, device), "page_table");
    const at::Tensor& parents = need(array(a[4], "parents", kI32, {kAny}, device), "parents");
    const int64_t forks = parents.size(0);
    const at::Tensor& to = need(array(a[7], "new_table", kI32, {forks, table.size(1)}, device), "new_table");
    emoe_fork_args A{};
    A.page_table = pointer<const int32_t>(&table);
    A.parents = pointer<const int32_t>(&parents);
    A.lengths = pointer<const int32_t>(&need(array(a[5], "lengths", kI32, {forks}, device), "lengths"));
    A.fresh = pointer<const int32_t>(array(a[6], "fresh", kI32, {forks}, device));
    A.new_table = pointer<int32_t>(&to);
    A.table_stride = table.stride(0);
    A.new_table_stride = to.stride(0);
    A.forks = i32(forks, "forks");
    A.n_seqs = i32(table.size(0), "sequences");
    A.table_width = i32(table.size(1), "page_table");
    return on_device(device, g_fork, kvs.data(), (int32_t)kvs.size(), &A, stream_of(a[8]));
  });
}

// (error class, addresses of emoe_last_error, _paged_append, _paged_attention, _process_logits,
//  _decoder_forward_paged, _paged_append_axes, _paged_tree_attention, _accept_drafts, _paged_compact,
//  _paged_fork)
PyObject* init(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  constexpr int kCalls = 10;
  if (n_args != 1 + kCalls) {
    PyErr_SetString(PyExc_TypeError, "init: 11 arguments");
    return nullptr;
  }
  uintptr_t at[kCalls];
  for (int i = 0; i < kCalls; ++i) {
    at[i] = (uintptr_t)PyLong_AsUnsignedLongLong(a[1 + i]);
    if (PyErr_Occurred()) return nullptr;
  }
  Py_INCREF(a[0]);
  Py_XDECREF(g_error);
  g_error = a[0];
  g_last_error = reinterpret_cast<decltype(g_last_error)>(at[0]);
  g_append = reinterpret_cast<decltype(g_append)>(at[1]);
  g_attention = reinterpret_cast<decltype(g_attention)>(at[2]);
  g_logits = reinterpret_cast<decltype(g_logits)>(at[3]);
  g_decoder = reinterpret_cast<decltype(g_decoder)>(at[4]);
  g_append_axes = reinterpret_cast<decltype(g_append_axes)>(at[5]);
  g_tree = reinterpret_cast<decltype(g_tree)>(at[6]);
  g_accept = reinterpret_cast<decltype(g_accept)>(at[7]);
  g_compact = reinterpret_cast<decltype(g_compact)>(at[8]);
  g_fork = reinterpret_cast<decltype(g_fork)>(at[9]);
  Py_RETURN_NONE;
}

#define FAST(f) {#f, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {FAST(init),           FAST(paged_append),          FAST(paged_attention),
                         FAST(process_logits), FAST(decoder_forward_paged),
                         FAST(paged_append_axes), FAST(paged_tree_attention), FAST(accept_drafts),
                         FAST(paged_compact),  FAST(paged_fork), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_binding", nullptr, -1, methods,
                      nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__binding() { return PyModule_Create(&module); }
