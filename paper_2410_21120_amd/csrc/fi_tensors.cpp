// Python extension: the decoder operators on PyTorch tensors.  Argument marshalling only: every tensor's type, device, shape and strides are checked, the
// struct of the C entry point is filled and the call made on the tensors' device.  A decoding step is a handful of launches of a few microseconds, which
// the same checks in Python do not keep up with (the host's time for norms and rotation of one token 11.0 us, here 3.6, nearly all of it the launch).
#include <Python.h>

#include <ATen/ATen.h>
#include <c10/core/DeviceGuard.h>
#include <c10/core/GradMode.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cmath>
#include <cstdarg>
#include <cstdint>
#include <cstdio>
#include <initializer_list>
#include <optional>
#include <string>

#include "../../include/fusedinf.h"

namespace {

using Shape = std::initializer_list<int64_t>;

struct Refusal {   // becomes a Python exception
  PyObject* type;
  std::string text;
};
struct Raised {};   // one is set already
[[noreturn]] void refuse(PyObject* type, const char* format, ...) {
  char text[400];
  va_list args;
  va_start(args, format);
  vsnprintf(text, sizeof text, format, args);
  va_end(args);
  throw Refusal{type, text};
}

// What bind() was given: the library's entry points and what Python does for the rare cases.
struct {
  fi_status (*qk_norm_rope)(const fi_qk_norm_rope_args*, void*);
  fi_status (*prompt_attention)(const fi_prompt_attention_args*, void*);
  fi_status (*tree_attention)(const fi_tree_attention_args*, void*);
  fi_status (*q4_matmul)(const fi_q4_matmul_args*, void*);
  fi_status (*tree_workspace)(const fi_tree_attention_args*, uint64_t*);
  fi_status (*q4_workspace)(const fi_q4_matmul_args*, uint64_t*);
  PyObject *check;    // check(status, entry point's name): raises
  PyObject *stream;   // stream(device index): the current one as a number
  PyObject *room;     // room(shape, type, stream, device index): a tensor from the memory that torch keeps for that stream
} py;

// The operators have no gradients: a call that would have to be recorded for one is refused.
const at::Tensor& tensor(PyObject* o, const char* name) {
  if (!THPVariable_Check(o)) refuse(PyExc_TypeError, "%s is no tensor", name);
  const at::Tensor& t = THPVariable_Unpack(o);
  if (t.requires_grad() && c10::GradMode::is_enabled()) refuse(PyExc_ValueError, "%s requires a gradient, and there is none: detach it, or call under torch.no_grad()", name);
  if (t._fw_grad(0).defined()) refuse(PyExc_ValueError, "%s has a tangent, and there is no forward derivative: detach it", name);
  if (t.is_neg()) refuse(PyExc_ValueError, "%s is a negated view: resolve_neg() makes its values", name);
  return t;
}
int32_t int32(int64_t v, const char* name) {
  if (v < INT32_MIN || v > INT32_MAX) refuse(PyExc_ValueError, "%s: %lld does not fit 32 bits", name, (long long)v);
  return (int32_t)v;
}
int64_t integer(PyObject* o) {
  const long long v = PyLong_AsLongLong(o);
  if (v == -1 && PyErr_Occurred()) throw Raised{};
  return v;
}
double number(PyObject* o) {
  const double v = PyFloat_AsDouble(o);
  if (v == -1.0 && PyErr_Occurred()) throw Raised{};
  return v;
}
bool truth(PyObject* o) {
  const int v = PyObject_IsTrue(o);
  if (v < 0) throw Raised{};
  return v != 0;
}

// The type and device that a call's tensors share.
struct Call {
  at::ScalarType type;
  int index;

  Call(const at::Tensor& t, const char* name) : type(t.scalar_type()), index((int)t.get_device()) {
    if (type != at::kBFloat16 && type != at::kFloat) refuse(PyExc_TypeError, "%s: %s, bfloat16 and float32 are covered", name, c10::toString(type));
    if (!t.is_cuda()) refuse(PyExc_ValueError, "%s is not in device memory", name);
  }
  int32_t dtype() const { return type == at::kFloat ? FI_F32 : FI_BF16; }

  [[noreturn]] void misfit(const at::Tensor& t, const char* name, at::ScalarType want, Shape shape, const char* more) const {
    auto list = [](auto&& v) {
      std::string s;
      for (int64_t x : v) s += (s.empty() ? "" : ", ") + std::to_string(x);
      return "(" + s + ")";
    };
    refuse(PyExc_ValueError, "%s: %s %s strides %s on %s, %s%s %s on device %d is wanted", name, c10::toString(t.scalar_type()), list(t.sizes()).c_str(),
           list(t.strides()).c_str(), t.device().str().c_str(), more, c10::toString(want), list(shape).c_str(), index);
  }
  bool fits(const at::Tensor& t, at::ScalarType want, Shape shape) const {
    return t.scalar_type() == want && t.is_cuda() && t.get_device() == index && t.sizes() == at::IntArrayRef(shape);
  }
  // A tensor whose last dimension is contiguous: its address; the other strides, in elements.
  void* rows(const at::Tensor& t, const char* name, at::ScalarType want, Shape shape, int64_t* strides) const {
    if (!fits(t, want, shape) || (t.stride(-1) != 1 && t.size(-1) > 1)) misfit(t, name, want, shape, "contiguous in its last dimension ");
    for (size_t i = 0; i + 1 < shape.size(); ++i) strides[i] = t.stride((int64_t)i);
    return t.data_ptr();
  }
  void* rows(const at::Tensor& t, const char* name, Shape shape, int64_t* strides) const { return rows(t, name, type, shape, strides); }
  template <typename T>
  T* plain(const at::Tensor& t, const char* name, at::ScalarType want, Shape shape) const {
    if (!fits(t, want, shape) || !t.is_contiguous()) misfit(t, name, want, shape, "contiguous ");
    return static_cast<T*>(t.data_ptr());
  }
  // Memory for a call on `stream` (None: the current one).  It has to come from what torch keeps for that stream: a block that another stream's pool hands out may
  // have been freed a moment ago with kernels of that other stream, for which nothing makes this one wait, still at work on it.
  at::Tensor room(at::ScalarType kind, Shape shape, PyObject* stream) const {
    if (stream == Py_None) return at::empty(at::IntArrayRef(shape), at::TensorOptions().dtype(kind).device(at::Device(at::kCUDA, (c10::DeviceIndex)index)));
    PyObject* const sizes = PyTuple_New((Py_ssize_t)shape.size());
    if (!sizes) throw Raised{};
    Py_ssize_t i = 0;
    for (int64_t n : shape) PyTuple_SET_ITEM(sizes, i++, PyLong_FromLongLong(n));
    PyObject* const o = PyObject_CallFunction(py.room, "NsOi", sizes, c10::toString(kind), stream, index);
    if (!o) throw Raised{};
    const at::Tensor made = THPVariable_Unpack(o);
    Py_DECREF(o);
    return made;
  }
  // A caller's output, or one made here.
  at::Tensor output(PyObject* o, const char* name, Shape shape, PyObject* stream) const {
    if (o != Py_None) return tensor(o, name);
    return room(type, shape, stream);
  }

  template <typename Args>
  void check(fi_status status, const char* name, const Args*) const {
    if (status == FI_OK) return;
    PyObject* const r = PyObject_CallFunction(py.check, "is", (int)status, name);
    Py_XDECREF(r);
    if (r) PyErr_Format(PyExc_RuntimeError, "%s: status %d", name, (int)status);
    throw Raised{};
  }
  // Makes the call on the tensors' device and the given stream, or the current one.
  template <typename Args>
  void make(fi_status (*entry)(const Args*, void*), const char* name, const Args& args, PyObject* stream) const {
    const c10::DeviceGuard guard(c10::Device(c10::DeviceType::CUDA, (c10::DeviceIndex)index));
    PyObject* const now = stream == Py_None ? PyObject_CallFunction(py.stream, "i", index) : (Py_INCREF(stream), stream);
    if (!now) throw Raised{};
    void* const s = PyLong_AsVoidPtr(now);
    Py_DECREF(now);
    if (!s && PyErr_Occurred()) throw Raised{};
    fi_status status;
    Py_BEGIN_ALLOW_THREADS
    status = entry(&args, s);
    Py_END_ALLOW_THREADS
    check(status, name, &args);
  }
  // Puts the caller's workspace, or one made here, into args; it has to live until the call is made.
  template <typename Args>
  at::Tensor workspace(fi_status (*needed)(const Args*, uint64_t*), const char* name, Args& args, PyObject* given, PyObject* stream) const {
    at::Tensor w;
    if (given != Py_None) {
      w = tensor(given, "workspace");
      if (w.scalar_type() != at::kByte || !w.is_cuda() || w.get_device() != index || !w.is_contiguous()) misfit(w, "workspace", at::kByte, {w.numel()}, "contiguous ");
    } else {
      uint64_t need = 0;
      check(needed(&args, &need), name, &args);
      if (!need) return w;
      w = room(at::kByte, {(int64_t)need}, stream);
    }
    args.workspace = w.data_ptr();
    args.workspace_bytes = (uint64_t)w.numel();
    return w;
  }
};

PyObject* returned(PyObject* given, const at::Tensor& t) {
  if (given == Py_None) return THPVariable_Wrap(t);
  if (!t.is_inference()) t.unsafeGetTensorImpl()->bump_version();   // (tells autograd that the values of a caller's output have changed)
  Py_INCREF(given);
  return given;
}

// Arguments in the order of the Python functions.
PyObject* qk_norm_rope(PyObject* const* arg) {
  const at::Tensor &q = tensor(arg[0], "q"), &k = tensor(arg[1], "k"), &positions = tensor(arg[3], "positions"), &inv_freq = tensor(arg[4], "inv_freq");
  const bool has_v = arg[2] != Py_None, paged = arg[10] != Py_None;
  const Call c(q, "q");
  if (q.dim() != 3 || k.dim() != 3 || positions.dim() < 1 || positions.dim() > 2 || inv_freq.dim() != 1)
    refuse(PyExc_ValueError, "q and k are [tokens, heads, head dim], positions [tokens] or [tokens, axes], inv_freq [pairs]");
  const int64_t tokens = q.size(0), heads = q.size(1), dim = q.size(2), kv_heads = k.size(1), pairs = inv_freq.size(0), axes = positions.dim() == 2 ? positions.size(1) : 1;
  fi_qk_norm_rope_args a = {};
  a.dtype = c.dtype();
  a.tokens = int32(tokens, "tokens");
  a.q_heads = int32(heads, "q heads");
  a.kv_heads = int32(kv_heads, "kv heads");
  a.head_dim = int32(dim, "head dim");
  a.rot_dim = int32(2 * pairs, "rotated values");
  a.interleaved = truth(arg[8]);
  int64_t sections = 1;
  if (arg[9] == Py_None) {
    a.sections[0] = a.rot_dim / 2;
  } else {
    PyObject* const list = PySequence_Fast(arg[9], "sections: pairs of every axis");
    if (!list) throw Raised{};
    sections = PySequence_Fast_GET_SIZE(list);
    for (int i = 0; i < sections && i < FI_MAX_AXES; ++i) {
      const long long n = PyLong_AsLongLong(PySequence_Fast_GET_ITEM(list, i));
      if (n < INT32_MIN || n > INT32_MAX || (n == -1 && PyErr_Occurred())) {
        Py_DECREF(list);
        if (PyErr_Occurred()) throw Raised{};
        refuse(PyExc_ValueError, "a section of %lld pairs", n);
      }
      a.sections[i] = (int32_t)n;
    }
    Py_DECREF(list);
  }
  if (sections != axes || axes < 1 || axes > FI_MAX_AXES) refuse(PyExc_ValueError, "%lld sections for %lld axes, 1 to %d are covered", (long long)sections, (long long)axes, FI_MAX_AXES);
  a.n_axes = (int32_t)axes;
  a.eps = (float)number(arg[7]);
  a.q = c.rows(q, "q", {tokens, heads, dim}, a.q_strides);
  a.k = c.rows(k, "k", {tokens, kv_heads, dim}, a.k_strides);
  if (arg[5] != Py_None) a.q_weight = c.plain<float>(tensor(arg[5], "q_weight"), "q_weight", at::kFloat, {dim});
  if (arg[6] != Py_None) a.k_weight = c.plain<float>(tensor(arg[6], "k_weight"), "k_weight", at::kFloat, {dim});
  a.positions = positions.dim() == 1 ? c.plain<int32_t>(positions, "positions", at::kInt, {tokens}) : c.plain<int32_t>(positions, "positions", at::kInt, {tokens, axes});
  a.inv_freq = c.plain<float>(inv_freq, "inv_freq", at::kFloat, {pairs});
  const at::Tensor q_out = c.output(arg[11], "q_out", {tokens, heads, dim}, arg[14]);
  a.q_out = c.rows(q_out, "q_out", {tokens, heads, dim}, a.q_out_strides);
  at::Tensor k_out, v_out;
  if (paged) {
    if (arg[12] == Py_None || tensor(arg[12], "k_out").dim() != 4 || (has_v && arg[13] == Py_None))
      refuse(PyExc_ValueError, "with slots, k_out and v_out are caches [pages, page size, kv heads, head dim]");
    k_out = tensor(arg[12], "k_out");
    const int64_t pages = k_out.size(0), page = k_out.size(1);
    a.page_size = int32(page, "page size");
    a.n_slots = pages * page;
    a.slots = c.plain<int64_t>(tensor(arg[10], "slots"), "slots", at::kLong, {tokens});
    a.k_out = c.rows(k_out, "k_out", {pages, page, kv_heads, dim}, a.k_out_strides);
    if (has_v) v_out = tensor(arg[13], "v_out"), a.v_out = c.rows(v_out, "v_out", {pages, page, kv_heads, dim}, a.v_out_strides);
  } else {
    k_out = c.output(arg[12], "k_out", {tokens, kv_heads, dim}, arg[14]);
    a.k_out = c.rows(k_out, "k_out", {tokens, kv_heads, dim}, a.k_out_strides + 1);
    if (has_v) v_out = c.output(arg[13], "v_out", {tokens, kv_heads, dim}, arg[14]), a.v_out = c.rows(v_out, "v_out", {tokens, kv_heads, dim}, a.v_out_strides + 1);
  }
  if (has_v) a.v = c.rows(tensor(arg[2], "v"), "v", {tokens, kv_heads, dim}, a.v_strides);
  c.make(py.qk_norm_rope, "fi_qk_norm_rope", a, arg[14]);
  return Py_BuildValue("(NNN)", returned(arg[11], q_out), returned(arg[12], k_out), has_v ? returned(arg[13], v_out) : (Py_INCREF(Py_None), Py_None));
}

PyObject* prompt_attention(PyObject* const* arg) {
  const at::Tensor &q = tensor(arg[0], "q"), &k = tensor(arg[1], "k"), &v = tensor(arg[2], "v"), &cu_q = tensor(arg[3], "cu_q");
  const Call c(q, "q");
  if (q.dim() != 3 || k.dim() != 3 || cu_q.dim() != 1 || cu_q.size(0) < 1) refuse(PyExc_ValueError, "q, k and v are [tokens, heads, head dim], cu_q is [sequences + 1]");
  const int64_t tokens = q.size(0), heads = q.size(1), dim = q.size(2), keys = k.size(0), kv_heads = k.size(1), ends = cu_q.size(0);
  fi_prompt_attention_args a = {};
  a.dtype = c.dtype();
  a.n_seqs = int32(ends - 1, "sequences");
  a.q_heads = int32(heads, "q heads");
  a.kv_heads = int32(kv_heads, "kv heads");
  a.head_dim = int32(dim, "head dim");
  a.causal = truth(arg[5]);
  a.scale = (float)(arg[6] == Py_None ? std::pow((double)dim, -0.5) : number(arg[6]));
  a.q_tokens = tokens;
  a.k_tokens = keys;
  a.q = c.rows(q, "q", {tokens, heads, dim}, a.q_strides);
  a.k = c.rows(k, "k", {keys, kv_heads, dim}, a.k_strides);
  a.v = c.rows(v, "v", {keys, kv_heads, dim}, a.v_strides);
  a.cu_q = c.plain<int32_t>(cu_q, "cu_q", at::kInt, {ends});
  a.cu_k = arg[4] == Py_None ? a.cu_q : c.plain<int32_t>(tensor(arg[4], "cu_k"), "cu_k", at::kInt, {ends});
  const at::Tensor out = c.output(arg[7], "out", {tokens, heads, dim}, arg[8]);
  a.out = c.rows(out, "out", {tokens, heads, dim}, a.out_strides);
  c.make(py.prompt_attention, "fi_prompt_attention", a, arg[8]);
  return returned(arg[7], out);
}

PyObject* tree_attention(PyObject* const* arg) {
  const at::Tensor &q = tensor(arg[0], "q"), &k = tensor(arg[1], "k_cache"), &v = tensor(arg[2], "v_cache"), &table = tensor(arg[3], "block_table"),
                   &cached = tensor(arg[4], "cached"), &cu = tensor(arg[5], "cu_nodes");
  const Call c(q, "q");
  if (q.dim() != 3 || k.dim() != 4 || table.dim() != 2 || cu.dim() != 1 || cu.size(0) < 1)
    refuse(PyExc_ValueError, "q is [nodes, heads, head dim], the caches [pages, page size, heads, head dim], block_table [sequences, columns], cu_nodes [sequences + 1]");
  const int64_t nodes = q.size(0), heads = q.size(1), dim = q.size(2), pages = k.size(0), page = k.size(1), kv_heads = k.size(2), seqs = cu.size(0) - 1, columns = table.size(1);
  fi_tree_attention_args a = {};
  a.dtype = c.dtype();
  a.n_seqs = int32(seqs, "sequences");
  a.q_heads = int32(heads, "q heads");
  a.kv_heads = int32(kv_heads, "kv heads");
  a.head_dim = int32(dim, "head dim");
  a.page_size = int32(page, "page size");
  a.n_pages = int32(pages, "pages");
  a.table_columns = int32(columns, "block_table's columns");
  a.scale = (float)(arg[7] == Py_None ? std::pow((double)dim, -0.5) : number(arg[7]));
  a.max_nodes = int32(arg[8] == Py_None ? nodes : integer(arg[8]), "max_nodes");
  const int64_t places = page * columns;
  a.max_length = arg[9] == Py_None ? (int32_t)(places < INT32_MAX ? places : INT32_MAX) : int32(integer(arg[9]), "max_length");
  a.nodes = nodes;
  a.block_table = static_cast<int32_t*>(c.rows(table, "block_table", at::kInt, {seqs, columns}, &a.table_stride));
  if (arg[6] != Py_None) {
    const at::Tensor& mask = tensor(arg[6], "mask");
    const int64_t words = mask.dim() ? mask.size(-1) : 0;
    a.mask = c.plain<uint64_t>(mask, "mask", at::kLong, {nodes, words});
    if (words < 1) refuse(PyExc_ValueError, "a mask of no words: None is the mask of chains");   // (its address is null, as None's)
    a.mask_words = int32(words, "mask words");
  }
  a.q = c.rows(q, "q", {nodes, heads, dim}, a.q_strides);
  a.k_cache = c.rows(k, "k_cache", {pages, page, kv_heads, dim}, a.k_strides);
  a.v_cache = c.rows(v, "v_cache", {pages, page, kv_heads, dim}, a.v_strides);
  a.cached = c.plain<int32_t>(cached, "cached", at::kInt, {seqs});
  a.cu_nodes = c.plain<int32_t>(cu, "cu_nodes", at::kInt, {seqs + 1});
  const at::Tensor out = c.output(arg[10], "out", {nodes, heads, dim}, arg[12]);
  a.out = c.rows(out, "out", {nodes, heads, dim}, a.out_strides);
  const at::Tensor workspace = c.workspace(py.tree_workspace, "fi_tree_attention_workspace", a, arg[11], arg[12]);
  c.make(py.tree_attention, "fi_tree_attention", a, arg[12]);
  return returned(arg[10], out);
}

PyObject* q4_matmul(PyObject* const* arg) {
  const at::Tensor &x = tensor(arg[0], "x"), &w = tensor(arg[1], "w"), &scales = tensor(arg[2], "scales");
  const Call c(x, "x");
  if (x.dim() != 2 || w.dim() != 2 || scales.dim() != 2) refuse(PyExc_ValueError, "x is [rows, inputs], w [outputs, inputs / 2], scales [outputs, groups]");
  const int64_t rows = x.size(0), inputs = x.size(1), outputs = w.size(0), groups = scales.size(1);
  const int64_t group = arg[4] != Py_None ? integer(arg[4]) : groups ? inputs / groups : 128;
  if (inputs % 2 || groups * group != inputs) refuse(PyExc_ValueError, "%lld inputs do not make %lld groups of %lld", (long long)inputs, (long long)groups, (long long)group);
  fi_q4_matmul_args a = {};
  a.dtype = c.dtype();
  a.rows = int32(rows, "rows");
  a.inputs = int32(inputs, "inputs");
  a.outputs = int32(outputs, "outputs");
  a.group = int32(group, "group");
  a.x = c.rows(x, "x", {rows, inputs}, &a.x_stride);
  a.w = static_cast<uint8_t*>(c.rows(w, "w", at::kByte, {outputs, inputs / 2}, &a.w_stride));
  a.scales = static_cast<float*>(c.rows(scales, "scales", at::kFloat, {outputs, groups}, &a.scales_stride));
  if (arg[3] != Py_None) a.zeros = static_cast<uint8_t*>(c.rows(tensor(arg[3], "zeros"), "zeros", at::kByte, {outputs, groups}, &a.zeros_stride));
  const at::Tensor out = c.output(arg[5], "out", {rows, outputs}, arg[7]);
  a.out = c.rows(out, "out", {rows, outputs}, &a.out_stride);
  const at::Tensor workspace = c.workspace(py.q4_workspace, "fi_q4_matmul_workspace", a, arg[6], arg[7]);
  c.make(py.q4_matmul, "fi_q4_matmul", a, arg[7]);
  return returned(arg[5], out);
}

template <PyObject* (*F)(PyObject* const*), int N>
PyObject* guarded(PyObject*, PyObject* const* arg, Py_ssize_t n) {
  if (n != N) return PyErr_Format(PyExc_TypeError, "%d arguments, not %zd", N, n);
  if (!py.check) return PyErr_Format(PyExc_RuntimeError, "bind() comes first");
  try {
    return F(arg);
  } catch (const Raised&) {
  } catch (const Refusal& r) {
    PyErr_SetString(r.type, r.text.c_str());
  } catch (const std::exception& e) {
    if (!PyErr_Occurred()) PyErr_SetString(PyExc_RuntimeError, e.what());
  }
  return nullptr;
}

// bind(addresses of the six entry points, check, stream, room)
PyObject* bind(PyObject*, PyObject* const* arg, Py_ssize_t n) {
  if (n != 9) return PyErr_Format(PyExc_TypeError, "9 arguments, not %zd", n);
  void* at[6];
  for (int i = 0; i < 6; ++i) {
    at[i] = PyLong_AsVoidPtr(arg[i]);
    if (!at[i]) return PyErr_Occurred() ? nullptr : PyErr_Format(PyExc_ValueError, "entry point %d is null", i);
  }
  py.qk_norm_rope = reinterpret_cast<decltype(py.qk_norm_rope)>(at[0]);
  py.prompt_attention = reinterpret_cast<decltype(py.prompt_attention)>(at[1]);
  py.tree_attention = reinterpret_cast<decltype(py.tree_attention)>(at[2]);
  py.q4_matmul = reinterpret_cast<decltype(py.q4_matmul)>(at[3]);
  py.tree_workspace = reinterpret_cast<decltype(py.tree_workspace)>(at[4]);
  py.q4_workspace = reinterpret_cast<decltype(py.q4_workspace)>(at[5]);
  for (int i = 6; i < 9; ++i) Py_INCREF(arg[i]);   // (for the life of the process)
  py.check = arg[6];
  py.stream = arg[7];
  py.room = arg[8];
  Py_RETURN_NONE;
}

#define FAST(f) reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(&f))
PyMethodDef methods[] = {
    {"bind", FAST(bind), METH_FASTCALL, nullptr},
    {"qk_norm_rope", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(&guarded<qk_norm_rope, 15>)), METH_FASTCALL, nullptr},
    {"prompt_attention", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(&guarded<prompt_attention, 9>)), METH_FASTCALL, nullptr},
    {"tree_attention", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(&guarded<tree_attention, 13>)), METH_FASTCALL, nullptr},
    {"q4_matmul", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(&guarded<q4_matmul, 8>)), METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_tensors", "The decoder operators on tensors (see operators.py).", -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__tensors() { return PyModule_Create(&module); }
