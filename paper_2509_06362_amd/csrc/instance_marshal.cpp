// Marshalling of the instance's calls: torch tensors to the structures of include/maaso_instance.h, with the checks that the
// binding makes of them.  A single token's calls run for a few microseconds; looking at a dozen tensors through the
// interpreter takes twice that, here a tenth.  Nothing is computed and nothing is kept.
#include <Python.h>

#include <c10/hip/HIPStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <string>

#include "../../include/maaso_instance.h"

namespace {

using Type = c10::ScalarType;

decltype(&maaso_kv_extend) call_extend;
decltype(&maaso_kv_fork) call_fork;
decltype(&maaso_kv_trim) call_trim;
decltype(&maaso_kv_compact) call_compact;
decltype(&maaso_kv_copy) call_copy;
decltype(&maaso_kv_append) call_append;
decltype(&maaso_kv_attention) call_attention;
decltype(&maaso_logits_adjust) call_logits;
decltype(&maaso_rows_quantize) call_quantize;
decltype(&maaso_scaled_product) call_product;
decltype(&maaso_expert_route) call_route;
decltype(&maaso_expert_product) call_experts;
decltype(&maaso_expert_combine) call_combine;

struct Refused {};  // the Python error is set

[[noreturn]] void refuse(const std::string& why) {
  PyErr_SetString(PyExc_AssertionError, why.c_str());
  throw Refused{};
}

const at::Tensor& tensor(PyObject* o) {
  if (!THPVariable_Check(o)) refuse(std::string("expected a tensor, got ") + Py_TYPE(o)->tp_name);
  return THPVariable_Unpack(o);
}

uint64_t whole(PyObject* o, uint64_t most = ~0ull) {
  PyObject* index = PyNumber_Index(o);
  if (!index) throw Refused{};
  const unsigned long long v = PyLong_AsUnsignedLongLong(index);
  Py_DECREF(index);
  if (v == ~0ull && PyErr_Occurred()) throw Refused{};
  if (v > most) refuse("a number out of range");
  return v;
}
uint32_t whole32(PyObject* o) { return (uint32_t)whole(o, 0xffffffffu); }
uint32_t whole32(int64_t v) {
  if (v < 0 || v > 0xffffffffll) refuse("a size out of range");
  return (uint32_t)v;
}

float real(PyObject* o) {
  const double v = PyFloat_AsDouble(o);
  if (v == -1.0 && PyErr_Occurred()) throw Refused{};
  return (float)v;
}

bool truth(PyObject* o) {
  const int v = PyObject_IsTrue(o);
  if (v < 0) throw Refused{};
  return v != 0;
}

template <typename T> T* address(PyObject* o) { return reinterpret_cast<T*>((uintptr_t)whole(o)); }

uint32_t type_of(const at::Tensor& t) {
  switch (t.scalar_type()) {
    case Type::BFloat16: return MAASO_BF16;
    case Type::Half: return MAASO_FP16;
    case Type::Float: return MAASO_FP32;
    case Type::Float8_e4m3fn: return MAASO_E4M3;
    case Type::Char: return MAASO_INT8;
    default: refuse(std::string(c10::toString(t.scalar_type())) + " is none of the library's types");
  }
}

// Device pointer of a contiguous tensor of this type, with `size` elements at least; None is NULL.
void* buffer(PyObject* o, Type type, int64_t size = 0) {
  if (o == Py_None) return nullptr;
  const at::Tensor& t = tensor(o);
  if (!t.is_cuda() || !t.is_contiguous()) refuse("device buffers must be contiguous GPU tensors");
  if (t.scalar_type() != type) refuse(std::string("expected ") + c10::toString(type) + ", got " + c10::toString(t.scalar_type()));
  if (t.numel() < size) refuse("expected " + std::to_string(size) + " elements, got " + std::to_string(t.numel()));
  return t.data_ptr();
}
int32_t* ints(PyObject* o, int64_t size = 0) { return static_cast<int32_t*>(buffer(o, Type::Int, size)); }
float* floats(PyObject* o, int64_t size = 0) { return static_cast<float*>(buffer(o, Type::Float, size)); }
int64_t elements(PyObject* o) { return o == Py_None ? 0 : tensor(o).numel(); }

// [tokens, heads, dim], a token's heads side by side; the elements between tokens go to `stride`.
void* heads(PyObject* o, Type type, int64_t n_tok, int64_t n_heads, int64_t dim, uint64_t& stride) {
  const at::Tensor& t = tensor(o);
  if (!t.is_cuda() || t.scalar_type() != type)
    refuse(std::string("expected a GPU tensor of ") + c10::toString(type) + ", got " + c10::toString(t.scalar_type()) + " on " + t.device().str());
  if (t.dim() != 3 || t.size(0) != n_tok || t.size(1) != n_heads || t.size(2) != dim)
    refuse("expected [" + std::to_string(n_tok) + ", " + std::to_string(n_heads) + ", " + std::to_string(dim) + "]");
  if (t.stride(2) != 1 || (n_heads > 1 && t.stride(1) != dim)) refuse("a token's heads must lie side by side");
  stride = (uint64_t)t.stride(0);
  return t.data_ptr();
}

// [rows, width], a row's elements side by side; the elements between rows go to `stride`.
void* rows_of(PyObject* o, Type type, int64_t n, int64_t width, uint64_t& stride) {
  const at::Tensor& t = tensor(o);
  if (!t.is_cuda() || t.scalar_type() != type)
    refuse(std::string("expected a GPU tensor of ") + c10::toString(type) + ", got " + c10::toString(t.scalar_type()) + " on " + t.device().str());
  if (t.dim() != 2 || t.size(0) != n || t.size(1) != width)
    refuse("expected [" + std::to_string(n) + ", " + std::to_string(width) + "]");
  if (t.stride(1) != 1 && width > 1) refuse("a row's elements must lie side by side");
  stride = (uint64_t)t.stride(0);
  return t.data_ptr();
}
const at::Tensor& matrix(PyObject* o, int64_t dims, const char* what) {
  const at::Tensor& t = tensor(o);
  if (t.dim() != dims) refuse(std::string("expected ") + what);
  return t;
}

void* stream(PyObject* o) {
  if (o == Py_None) return c10::hip::getCurrentHIPStream().stream();
  PyObject* handle = PyObject_GetAttrString(o, "cuda_stream");
  if (!handle) throw Refused{};
  void* s = PyLong_AsVoidPtr(handle);
  Py_DECREF(handle);
  if (!s && PyErr_Occurred()) throw Refused{};
  return s;
}

// What every entry does around its own part: count the arguments, call without the interpreter's lock, return the status.
template <typename Fill>
PyObject* entry(Py_ssize_t given, Py_ssize_t wanted, Fill fill) {
  try {
    if (given != wanted) refuse("expected " + std::to_string(wanted) + " arguments, got " + std::to_string(given));
    auto call = fill();
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = call();
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
  } catch (const Refused&) {
    return nullptr;
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
    return nullptr;
  }
}

using Args = PyObject* const*;
maaso_instance* instance_of(PyObject* o) {
  if (o == Py_None) return nullptr;  // (closed: the library refuses it)
  return address<maaso_instance>(o);
}

PyObject* extend(PyObject*, Args a, Py_ssize_t n) {
  return entry(n, 8, [=] {
    maaso_instance* inst = instance_of(a[0]);
    const auto* pages = address<const maaso_kv_pages>(a[1]);
    const int64_t rows = tensor(a[2]).numel(), tokens = tensor(a[4]).numel();
    const int32_t *row = ints(a[2]), *start = ints(a[3], rows + 1);
    auto* slot = static_cast<int64_t*>(buffer(a[4], Type::Long));
    int32_t *pos = ints(a[5], tokens), *copies = ints(a[6], 2 * rows);
    void* s = stream(a[7]);
    const uint32_t n_rows = whole32(rows), n_tok = whole32(tokens);
    return [=] { return call_extend(inst, pages, row, n_rows, start, n_tok, slot, pos, copies, s); };
  });
}

PyObject* fork_rows(PyObject*, Args a, Py_ssize_t n) {
  return entry(n, 5, [=] {
    maaso_instance* inst = instance_of(a[0]);
    const auto* pages = address<const maaso_kv_pages>(a[1]);
    const int64_t rows = tensor(a[3]).numel();
    const int32_t *parents = ints(a[2], rows), *children = ints(a[3]);
    void* s = stream(a[4]);
    const uint32_t n_rows = whole32(rows);
    return [=] { return call_fork(inst, pages, parents, children, n_rows, s); };
  });
}

PyObject* trim(PyObject*, Args a, Py_ssize_t n) {
  return entry(n, 5, [=] {
    maaso_instance* inst = instance_of(a[0]);
    const auto* pages = address<const maaso_kv_pages>(a[1]);
    const int64_t rows = tensor(a[2]).numel();
    const int32_t *row = ints(a[2]), *keep = ints(a[3], rows);
    void* s = stream(a[4]);
    const uint32_t n_rows = whole32(rows);
    return [=] { return call_trim(inst, pages, row, keep, n_rows, s); };
  });
}

PyObject* compact(PyObject*, Args a, Py_ssize_t n) {
  return entry(n, 7, [=] {
    maaso_instance* inst = instance_of(a[0]);
    const auto* pages = address<const maaso_kv_pages>(a[1]);
    int32_t *refs = ints(a[2], pages->n_pages), *table = ints(a[3], (int64_t)pages->n_rows * pages->width);
    int32_t *moves = ints(a[4], 2 * (int64_t)(pages->n_pages / 2u)), *live = ints(a[5], 1);
    void* s = stream(a[6]);
    return [=] { return call_compact(inst, pages, refs, table, moves, live, s); };
  });
}

PyObject* copy_pages(PyObject*, Args a, Py_ssize_t n) {
  return entry(n, 4, [=] {
    maaso_instance* inst = instance_of(a[0]);
    const auto* cache = address<const maaso_kv_cache>(a[1]);
    const int32_t* pairs = ints(a[2]);
    const uint32_t n_pairs = whole32(elements(a[2]) / 2);
    void* s = stream(a[3]);
    return [=] { return call_copy(inst, cache, pairs, n_pairs, s); };
  });
}

// (inst, cache, layer, q, k, v, q_out, slot, pos, cos_sin, q_weight, k_weight, eps, interleaved, stream)
PyObject* append(PyObject*, Args a, Py_ssize_t n) {
  return entry(n, 15, [=] {
    maaso_instance* inst = instance_of(a[0]);
    const auto* cache = address<const maaso_kv_cache>(a[1]);
    const uint32_t layer = whole32(a[2]);
    const at::Tensor& q = tensor(a[3]);
    if (q.dim() != 3) refuse("expected [tokens, heads, dim]");
    const Type type = q.scalar_type();
    const int64_t tokens = q.size(0), dim = cache->head_dim;
    maaso_kv_append_args p{};
    p.type = type_of(q);
    p.n_tok = whole32(tokens);
    p.n_heads = whole32(q.size(1));
    p.q = heads(a[3], type, tokens, q.size(1), dim, p.q_stride);
    p.k = heads(a[4], type, tokens, cache->n_kv_heads, dim, p.k_stride);
    p.v = heads(a[5], type, tokens, cache->n_kv_heads, dim, p.v_stride);
    p.q_out = heads(a[6], type, tokens, q.size(1), dim, p.q_out_stride);
    p.slot = static_cast<const int64_t*>(buffer(a[7], Type::Long, tokens));
    p.pos = ints(a[8], tokens);
    if (a[9] != Py_None) {
      const at::Tensor& t = tensor(a[9]);
      if (t.dim() != 2) refuse("cos_sin must be [positions, rotary]");
      p.cos_sin = floats(a[9]);
      p.n_pos = whole32(t.size(0));
      p.rotary = whole32(t.size(1));
    }
    p.q_weight = buffer(a[10], type, dim);
    p.k_weight = buffer(a[11], type, dim);
    p.eps = real(a[12]);
    p.interleaved = truth(a[13]);
    void* s = stream(a[14]);
    return [=] { return call_append(inst, cache, layer, &p, s); };
  });
}

// (inst, cache, pages, layer, q, out, q_start, scale, max_q, max_len, rows, group_start, shared, max_shared, total_len, lse, stream)
PyObject* attention(PyObject*, Args a, Py_ssize_t n) {
  return entry(n, 17, [=] {
    maaso_instance* inst = instance_of(a[0]);
    const auto* cache = address<const maaso_kv_cache>(a[1]);
    const auto* pages = address<const maaso_kv_pages>(a[2]);
    const uint32_t layer = whole32(a[3]);
    const at::Tensor& q = tensor(a[4]);
    if (q.dim() != 3) refuse("expected [tokens, heads, dim]");
    const Type type = q.scalar_type();
    const int64_t tokens = q.size(0), n_heads = q.size(1), sequences = tensor(a[6]).numel() - 1;
    const int64_t groups = a[11] == Py_None ? 0 : tensor(a[11]).numel() - 1;
    maaso_kv_attention_args p{};
    p.type = type_of(q);
    p.n_tok = whole32(tokens);
    p.n_heads = whole32(n_heads);
    p.n = whole32(sequences);
    p.n_groups = whole32(groups);
    p.q = heads(a[4], type, tokens, n_heads, cache->head_dim, p.q_stride);
    p.out = heads(a[5], type, tokens, n_heads, cache->head_dim, p.out_stride);
    p.q_start = ints(a[6]);
    p.scale = real(a[7]);
    p.max_q = whole32(a[8]);
    p.max_len = whole32(a[9]);
    p.rows = ints(a[10], sequences);
    p.group_start = ints(a[11]);
    p.shared = ints(a[12], groups);
    p.max_shared = whole32(a[13]);
    p.total_len = whole(a[14]);
    p.lse = floats(a[15], tokens * n_heads);
    void* s = stream(a[16]);
    return [=] { return call_attention(inst, cache, layer, pages, &p, s); };
  });
}

// (inst, logits, out, chosen, repetition, frequency, presence, temperature, history, history_start, bias_token, bias_value,
//  bias_start, mask, mask_row, stream)
PyObject* logits(PyObject*, Args a, Py_ssize_t n) {
  return entry(n, 16, [=] {
    maaso_instance* inst = instance_of(a[0]);
    const at::Tensor& x = tensor(a[1]);
    if (x.dim() != 2 || !x.is_cuda() || x.stride(1) != 1) refuse("a row's logits must lie side by side, on the GPU");
    const int64_t rows = x.size(0), vocab = x.size(1);
    maaso_logits_args p{};
    p.type = type_of(x);
    p.n = whole32(rows);
    p.vocab = whole32(vocab);
    p.logits = x.data_ptr();
    p.stride = (uint64_t)x.stride(0);
    p.out_type = MAASO_FP32;
    if (a[2] != Py_None) {
      const at::Tensor& y = tensor(a[2]);
      if (!y.is_cuda() || y.dim() != 2 || y.size(0) != rows || y.size(1) != vocab || y.stride(1) != 1)
        refuse("out must have the logits' shape, a row's elements side by side");
      p.out = y.data_ptr();
      p.out_type = type_of(y);
      p.out_stride = (uint64_t)y.stride(0);
    }
    p.chosen = ints(a[3], rows);
    p.repetition = floats(a[4], rows);
    p.frequency = floats(a[5], rows);
    p.presence = floats(a[6], rows);
    p.temperature = floats(a[7], rows);
    p.history = ints(a[8]);
    p.history_start = ints(a[9], rows + 1);
    p.n_history = whole32(elements(a[8]));
    p.n_bias = whole32(elements(a[10]));
    p.bias_token = ints(a[10]);
    p.bias_value = floats(a[11], p.n_bias);
    p.bias_start = ints(a[12], rows + 1);
    if (a[13] != Py_None) {
      const at::Tensor& m = tensor(a[13]);
      if (m.dim() != 2 || m.size(1) != (vocab + 31) / 32) refuse("a mask has a bit for each token");
      p.mask = reinterpret_cast<const uint32_t*>(ints(a[13]));
      p.n_mask = whole32(m.size(0));
    }
    p.mask_row = ints(a[14], rows);
    void* s = stream(a[15]);
    return [=] { return call_logits(inst, &p, s); };
  });
}

// (inst, x, q, scale, weight, norm, gated, eps, stream)
PyObject* quantize(PyObject*, Args a, Py_ssize_t n) {
  return entry(n, 9, [=] {
    maaso_instance* inst = instance_of(a[0]);
    const at::Tensor &x = matrix(a[1], 2, "x as [rows, width]"), &q = matrix(a[2], 2, "q as [rows, width]");
    maaso_rows_quantize_args p{};
    const bool norm = truth(a[5]), gated = truth(a[6]);
    if (norm && gated) refuse("rows are either normed or gated");
    const int64_t rows = x.size(0), width = q.size(1);
    p.type = type_of(x);
    p.form = norm ? MAASO_ROWS_NORM : gated ? MAASO_ROWS_GATED : MAASO_ROWS_PLAIN;
    p.n = whole32(rows);
    p.width = whole32(width);
    p.eps = real(a[7]);
    p.x = rows_of(a[1], x.scalar_type(), rows, gated ? 2 * width : width, p.x_stride);
    p.q = static_cast<int8_t*>(rows_of(a[2], Type::Char, rows, width, p.q_stride));
    p.scale = floats(a[3], rows);
    p.weight = buffer(a[4], x.scalar_type(), width);
    void* s = stream(a[8]);
    return [=] { return call_quantize(inst, &p, s); };
  });
}

// What both products have in common: a [rows, in], out [out rows, channels]; w's last two dimensions are looked at by the caller.
maaso_product product_of(PyObject* a, PyObject* a_scale, const at::Tensor& w, PyObject* w_scale, PyObject* out, PyObject* bias, PyObject* gated, int64_t experts) {
  maaso_product p{};
  const at::Tensor &x = matrix(a, 2, "a as [rows, in]"), &y = matrix(out, 2, "out as [rows, channels]");
  const int64_t rows = x.size(0), in = x.size(1), channels = w.size(-2);
  p.type = type_of(x);
  p.out_type = type_of(y);
  p.gated = truth(gated) ? 1u : 0u;
  if (!w.is_cuda() || w.scalar_type() != x.scalar_type()) refuse("w must be a GPU tensor of a's type");
  if (w.size(-1) != in || channels != y.size(1) * (p.gated ? 2 : 1)) refuse("w must have a row of a's width for each channel, twice as many where gated");
  if (w.stride(-1) != 1 && in > 1) refuse("a row's elements must lie side by side");
  p.n_a = whole32(rows);
  p.n_in = whole32(in);
  p.n_out = whole32(y.size(1));
  p.a = rows_of(a, x.scalar_type(), rows, in, p.a_stride);
  p.out = rows_of(out, y.scalar_type(), y.size(0), y.size(1), p.out_stride);
  p.w = w.data_ptr();
  p.w_stride = (uint64_t)w.stride(-2);
  p.a_scale = floats(a_scale, rows);
  p.w_scale = floats(w_scale, experts * channels);
  p.bias = floats(bias, experts * channels);
  return p;
}

// (inst, a, a_scale, w, w_scale, out, bias, gated, stream)
PyObject* scaled_product(PyObject*, Args a, Py_ssize_t n) {
  return entry(n, 9, [=] {
    maaso_instance* inst = instance_of(a[0]);
    const at::Tensor& w = matrix(a[3], 2, "w as [channels, in]");
    const maaso_product p = product_of(a[1], a[2], w, a[4], a[5], a[6], a[7], 1);
    if (tensor(a[5]).size(0) != tensor(a[1]).size(0)) refuse("out must have a's rows");
    void* s = stream(a[8]);
    return [=] { return call_product(inst, &p, s); };
  });
}

// (inst, a, a_scale, w, w_scale, out, start, token, bias, gated, stream)
PyObject* expert_product(PyObject*, Args a, Py_ssize_t n) {
  return entry(n, 11, [=] {
    maaso_instance* inst = instance_of(a[0]);
    const at::Tensor& w = matrix(a[3], 3, "w as [experts, channels, in]");
    maaso_expert_product_args p{};
    p.product = product_of(a[1], a[2], w, a[4], a[5], a[8], a[9], w.size(0));
    p.n_rows = whole32(tensor(a[5]).size(0));
    p.n_experts = whole32(w.size(0));
    p.expert_stride = (uint64_t)w.stride(0);
    p.start = ints(a[6], w.size(0) + 1);
    p.token = ints(a[7], p.n_rows);
    void* s = stream(a[10]);
    return [=] { return call_experts(inst, &p, s); };
  });
}

// (inst, logits, bias, expert, weight, start, token, place, sigmoid, renorm, scale, stream)
PyObject* route(PyObject*, Args a, Py_ssize_t n) {
  return entry(n, 12, [=] {
    maaso_instance* inst = instance_of(a[0]);
    const at::Tensor &x = matrix(a[1], 2, "logits as [tokens, experts]"), &e = matrix(a[3], 2, "expert as [tokens, chosen]");
    maaso_expert_route_args p{};
    const int64_t tokens = x.size(0), k = e.size(1);
    if (e.size(0) != tokens) refuse("expert must have a row for each token");
    p.type = type_of(x);
    p.n = whole32(tokens);
    p.n_experts = whole32(x.size(1));
    p.k = whole32(k);
    p.logits = rows_of(a[1], x.scalar_type(), tokens, x.size(1), p.stride);
    p.bias = floats(a[2], p.n_experts);
    p.expert = ints(a[3]);
    p.weight = floats(a[4], tokens * k);
    p.start = ints(a[5], x.size(1) + 1);
    p.token = ints(a[6], tokens * k);
    p.place = ints(a[7], tokens * k);
    p.sigmoid = truth(a[8]) ? 1u : 0u;
    p.renorm = truth(a[9]) ? 1u : 0u;
    p.scale = real(a[10]);
    void* s = stream(a[11]);
    return [=] { return call_route(inst, &p, s); };
  });
}

// (inst, y, place, weight, out, residual, stream)
PyObject* combine(PyObject*, Args a, Py_ssize_t n) {
  return entry(n, 7, [=] {
    maaso_instance* inst = instance_of(a[0]);
    const at::Tensor &y = matrix(a[1], 2, "y as [rows, width]"), &place = matrix(a[2], 2, "place as [tokens, chosen]");
    maaso_expert_combine_args p{};
    const Type type = y.scalar_type();
    const int64_t tokens = place.size(0), width = y.size(1);
    p.type = type_of(y);
    p.n = whole32(tokens);
    p.k = whole32(place.size(1));
    p.width = whole32(width);
    p.n_rows = whole32(y.size(0));
    p.y = rows_of(a[1], type, y.size(0), width, p.y_stride);
    p.out = rows_of(a[4], type, tokens, width, p.out_stride);
    if (a[5] != Py_None) p.residual = rows_of(a[5], type, tokens, width, p.residual_stride);
    p.place = ints(a[2]);
    p.weight = floats(a[3], tokens * place.size(1));
    void* s = stream(a[6]);
    return [=] { return call_combine(inst, &p, s); };
  });
}

// The library's entry points, as addresses, in the order of the declarations above.
PyObject* bind(PyObject*, Args a, Py_ssize_t n) {
  return entry(n, 13, [=] {
    auto at = [&](int k) { return (uintptr_t)whole(a[k]); };
    call_extend = reinterpret_cast<decltype(call_extend)>(at(0));
    call_fork = reinterpret_cast<decltype(call_fork)>(at(1));
    call_trim = reinterpret_cast<decltype(call_trim)>(at(2));
    call_compact = reinterpret_cast<decltype(call_compact)>(at(3));
    call_copy = reinterpret_cast<decltype(call_copy)>(at(4));
    call_append = reinterpret_cast<decltype(call_append)>(at(5));
    call_attention = reinterpret_cast<decltype(call_attention)>(at(6));
    call_logits = reinterpret_cast<decltype(call_logits)>(at(7));
    call_quantize = reinterpret_cast<decltype(call_quantize)>(at(8));
    call_product = reinterpret_cast<decltype(call_product)>(at(9));
    call_route = reinterpret_cast<decltype(call_route)>(at(10));
    call_experts = reinterpret_cast<decltype(call_experts)>(at(11));
    call_combine = reinterpret_cast<decltype(call_combine)>(at(12));
    return [] { return 0; };
  });
}

template <PyObject* (*F)(PyObject*, Args, Py_ssize_t)>
PyMethodDef method(const char* name) {
  return {name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(F)), METH_FASTCALL, nullptr};
}

PyMethodDef methods[] = {method<bind>("bind"), method<extend>("extend"), method<fork_rows>("fork"), method<trim>("trim"),
                         method<compact>("compact"), method<copy_pages>("copy"), method<append>("append"),
                         method<attention>("attention"), method<logits>("logits"), method<quantize>("quantize"),
                         method<scaled_product>("scaled_product"), method<expert_product>("expert_product"), method<route>("route"),
                         method<combine>("combine"), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__marshal() { return PyModule_Create(&module); }
