// Argument marshalling of the operators of a speculative step, for torch tensors: checks their shapes and types and calls the C ABI on
// torch's current stream.  In Python the same took 11 to 16 us a call, several times what the smallest kernels take; here it
// takes about one.  Nothing is computed here and nothing kept between calls.
#include <ATen/ops/empty.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include "../../include/blink.h"
#include "ops.h"

namespace {

// The arguments of one call, unpacked in order; the first error is kept as Python's.
struct Args {
  PyObject* const* arg;
  Py_ssize_t n, at = 0;
  c10::DeviceIndex device = -1;
  bool ok = true;

  Args(PyObject* const* a, Py_ssize_t have, Py_ssize_t want) : arg(a), n(have) {
    if (have != want) fail(PyExc_TypeError, "%zd arguments instead of %zd", have, want);
  }
  template <typename... A>
  void fail(PyObject* kind, const char* format, A... a) {
    if (ok) PyErr_Format(kind, format, a...);
    ok = false;
  }
  void need(bool fine, const char* what) {
    if (!fine) fail(PyExc_ValueError, "%s", what);
  }
  PyObject* next() {
    static PyObject* none = Py_None;
    return ok && at < n ? arg[at++] : none;
  }
  long integer() {
    PyObject* o = next();
    if (!ok) return 0;
    const long v = PyLong_AsLong(o);
    if (v == -1 && PyErr_Occurred()) ok = false;
    if (v > 0x7fffffffl || v < -0x7fffffffl) fail(PyExc_ValueError, "%ld is no 32-bit number", v);
    return v;
  }
  // null: None, where that is allowed
  const at::Tensor* tensor(const char* what, bool optional = false) {
    PyObject* o = next();
    if (!ok || (optional && o == Py_None)) return nullptr;
    if (!THPVariable_Check(o)) {
      fail(PyExc_ValueError, "%s: a tensor", what);
      return nullptr;
    }
    const at::Tensor* t = &THPVariable_Unpack(o);
    if (!t->is_cuda()) fail(PyExc_ValueError, "%s: on the host; the operators run on a CUDA device", what);
    else if (device < 0) device = t->get_device();
    else if (t->get_device() != device) fail(PyExc_ValueError, "%s: on CUDA device %d, others on %d", what, (int)t->get_device(), (int)device);
    return t;
  }
  const at::Tensor* vector(const char* what, at::ScalarType type, int64_t size = -1, bool optional = false) {
    const at::Tensor* t = tensor(what, optional);
    if (ok && t && (t->scalar_type() != type || t->dim() != 1 || !t->is_contiguous() || (size >= 0 && t->numel() != size))) {
      if (size >= 0) fail(PyExc_ValueError, "%s: contiguous %s vector of %lld", what, c10::toString(type), (long long)size);
      else fail(PyExc_ValueError, "%s: contiguous %s vector", what, c10::toString(type));
    }
    return t;
  }
  const at::Tensor* ints(const char* what, int64_t size = -1, bool optional = false) { return vector(what, at::kInt, size, optional); }
  const at::Tensor* floats(const char* what, int64_t size, bool optional = false) { return vector(what, at::kFloat, size, optional); }
  const at::Tensor* table(int64_t rows) {
    const at::Tensor* t = tensor("block_table");
    if (ok && (t->scalar_type() != at::kInt || t->dim() != 2 || t->size(0) != rows || !t->is_contiguous()))
      fail(PyExc_ValueError, "block_table: contiguous Int [%lld][stride]", (long long)rows);
    return t;
  }
  // [rows][cols], elements of a row next to one another; rows < 0: any number
  const at::Tensor* matrix(const char* what, int64_t rows, int64_t cols, at::ScalarType type, int64_t* stride, bool optional = false) {
    const at::Tensor* t = tensor(what, optional);
    *stride = cols;
    if (!ok || !t) return t;
    if (t->dim() != 2 || t->scalar_type() != type || (rows >= 0 && t->size(0) != rows) || (cols >= 0 && t->size(1) != cols) || (t->stride(1) != 1 && t->size(1) > 1)) {
      if (cols >= 0) fail(PyExc_ValueError, "%s: [%s][%lld] of %s, elements of a row next to one another", what, rows >= 0 ? std::to_string(rows).c_str() : "rows",
                          (long long)cols, c10::toString(type));
      else fail(PyExc_ValueError, "%s: [rows][columns] of %s, elements of a row next to one another", what, c10::toString(type));
    } else {
      *stride = t->size(0) > 1 ? t->stride(0) : t->size(1);   // (of a single row it may be anything)
    }
    return t;
  }
};

const void* at_of(const at::Tensor* t) { return t ? t->const_data_ptr() : nullptr; }
template <typename T>
const T* in(const at::Tensor* t) { return static_cast<const T*>(at_of(t)); }
template <typename T>
T* out(const at::Tensor* t) { return t ? static_cast<T*>(t->data_ptr()) : nullptr; }

// A model shape (synth.ModelCfg or its like).
bool model_of(Args& a, blink_model_cfg* m) {
  PyObject* o = a.next();
  if (!a.ok) return false;
  static const char* const names[] = {"n_layers", "d_model", "n_q_heads", "n_kv_heads", "head_dim", "d_ff", "vocab", "n_experts", "top_k_experts"};
  static PyObject* keys[12];
  if (!keys[11]) {
    for (int i = 0; i < 9; ++i) keys[i] = PyUnicode_InternFromString(names[i]);
    keys[9] = PyUnicode_InternFromString("rope_theta");
    keys[10] = PyUnicode_InternFromString("rms_eps");
    keys[11] = PyUnicode_InternFromString("dtype");
  }
  *m = {};
  m->size = sizeof(*m);
  int32_t* const to[] = {&m->n_layers, &m->d_model, &m->n_q_heads, &m->n_kv_heads, &m->head_dim, &m->d_ff, &m->vocab, &m->n_experts, &m->top_k_experts};
  for (int i = 0; i < 12 && a.ok; ++i) {
    PyObject* v = PyObject_GetAttr(o, keys[i]);
    if (!v) {
      a.ok = false;
      break;
    }
    if (i < 9) {
      const long n = PyLong_AsLong(v);
      *to[i] = (int32_t)n;
      if (!PyErr_Occurred() && n != *to[i]) a.fail(PyExc_ValueError, "%s: %ld is no 32-bit number", names[i], n);
    } else if (i == 9) m->rope_theta = (float)PyFloat_AsDouble(v);
    else if (i == 10) m->rms_eps = (float)PyFloat_AsDouble(v);
    else if (PyUnicode_Check(v) && PyUnicode_CompareWithASCIIString(v, "bf16") == 0) m->dtype = BLINK_DTYPE_BF16;
    else if (PyUnicode_Check(v) && PyUnicode_CompareWithASCIIString(v, "fp32") == 0) m->dtype = BLINK_DTYPE_FP32;
    else a.fail(PyExc_ValueError, "dtype: %R, neither 'bf16' nor 'fp32'", v);
    Py_DECREF(v);
    if (PyErr_Occurred()) a.ok = false;
  }
  return a.ok;
}

at::ScalarType type_of(const blink_model_cfg& m) { return m.dtype == BLINK_DTYPE_BF16 ? at::kBFloat16 : at::kFloat; }

// The pool as it was carved out: elements of the model's type, or bytes.  One that says its shape has the model's.
blink_kv_pool pool_of(Args& a, const blink_model_cfg& m) {
  const at::Tensor* t = a.tensor("kv_pool");
  if (!a.ok) return {};
  a.need(t->is_contiguous(), "kv_pool: contiguous");
  if (t->scalar_type() != type_of(m) && t->scalar_type() != at::kByte)
    a.fail(PyExc_ValueError, "kv_pool: of %s, neither the model's %s nor bytes", c10::toString(t->scalar_type()), c10::toString(type_of(m)));
  if (t->dim() == 6 && t->scalar_type() != at::kByte) {
    const int64_t want[6] = {m.n_layers, 2, t->size(2), m.n_kv_heads, 16, m.head_dim};
    for (int i = 0; i < 6; ++i)
      if (t->size(i) != want[i]) a.fail(PyExc_ValueError, "kv_pool: [layers][2][blocks][kv heads][16][head_dim] of the model has %lld elements in dimension %d, not %lld",
                                        (long long)want[i], i, (long long)t->size(i));
  }
  return {sizeof(blink_kv_pool), 16, t->data_ptr(), (uint64_t)t->nbytes()};
}

at::Tensor make(at::IntArrayRef size, at::ScalarType type, const Args& a) {
  return at::empty(size, at::TensorOptions().dtype(type).device(at::Device(at::kCUDA, a.device)));
}

// f(stream) with the arguments' device current; the error code as a Python number
template <typename F>
PyObject* call(const Args& a, F f) {
  const c10::cuda::CUDAGuard guard(a.device);
  return PyLong_FromLong(f(static_cast<void*>(c10::cuda::getCurrentCUDAStream(a.device).stream())));
}

// ctx_len, new_len, blocks_held, free_blocks, free_count, block_table, then the seven outputs -> error code
PyObject* build_tables(PyObject*, PyObject* const* arg, Py_ssize_t nargs) {
  Args a(arg, nargs, 13);
  const at::Tensor* ctx = a.ints("ctx_len");
  const int64_t n = a.ok ? ctx->numel() : 0;
  const at::Tensor *add = a.ints("new_len", n), *held = a.ints("blocks_held", n), *free_blocks = a.ints("free_blocks"), *count = a.ints("free_count", 1);
  const at::Tensor* table = a.table(n);
  const at::Tensor *row_start = a.ints("row_start", n + 1), *kv_len = a.ints("kv_len", n), *positions = a.ints("positions");
  const int64_t rows = a.ok ? positions->numel() : 0;
  const at::Tensor *slots = a.ints("slot_map", rows), *held_out = a.ints("blocks_held", n), *count_out = a.ints("free_count", 1), *status = a.ints("status", 1);
  if (a.ok) a.need(std::max({n, rows, table->size(1), free_blocks->numel()}) <= 0x7fffffff, "sizes beyond 31 bits");
  if (!a.ok) return nullptr;
  return call(a, [&](void* stream) {
    return blink_build_tables(in<int32_t>(ctx), in<int32_t>(add), in<int32_t>(held), (int)n, in<int32_t>(free_blocks), (int)free_blocks->numel(), in<int32_t>(count),
                              out<int32_t>(table), (int)table->size(1), (int)rows, out<int32_t>(held_out), out<int32_t>(count_out), out<int32_t>(row_start),
                              out<int32_t>(kv_len), out<int32_t>(positions), out<int32_t>(slots), out<int32_t>(status), stream);
  });
}

// model, kv_pool, layer, qkv, q_gain, k_gain, positions, slot_map, out -> error code
PyObject* qk_norm_rope(PyObject*, PyObject* const* arg, Py_ssize_t nargs) {
  Args a(arg, nargs, 9);
  blink_model_cfg m;
  if (!model_of(a, &m)) return nullptr;
  const blink_kv_pool kv = pool_of(a, m);
  const long layer = a.integer();
  const int64_t q_dim = (int64_t)m.n_q_heads * m.head_dim;
  int64_t stride = 0, out_stride = 0;
  const at::Tensor* probe = a.ok && a.at < a.n && THPVariable_Check(a.arg[a.at]) ? &THPVariable_Unpack(a.arg[a.at]) : nullptr;
  const bool f32 = probe && probe->scalar_type() == at::kFloat;
  const at::Tensor* qkv = a.matrix("qkv", -1, q_dim + 2ll * m.n_kv_heads * m.head_dim, f32 ? at::kFloat : type_of(m), &stride);
  const int64_t rows = a.ok ? qkv->size(0) : 0;
  const at::Tensor *qg = a.floats("q_gain", m.head_dim, true), *kg = a.floats("k_gain", m.head_dim, true);
  const at::Tensor *positions = a.ints("positions", rows), *slots = a.ints("slot_map", rows);
  const at::Tensor* q = a.matrix("out", rows, q_dim, type_of(m), &out_stride);
  if (a.ok) a.need(rows <= 0x7fffffff, "rows beyond 31 bits");
  if (!a.ok) return nullptr;
  if (rows == 0) return PyLong_FromLong(BLINK_OK);
  return call(a, [&](void* stream) {
    return blink_qk_norm_rope(&m, &kv, (int)layer, at_of(qkv), f32 ? BLINK_DTYPE_FP32 : BLINK_DTYPE_BF16, stride, in<float>(qg), in<float>(kg), in<int32_t>(positions),
                              in<int32_t>(slots), (int)rows, out<void>(q), out_stride, stream);
  });
}

// model, kv_pool, layer, q, row_start, kv_len, block_table, window, sinks, max_new, out, workspace or None -> error code
PyObject* window_attention(PyObject*, PyObject* const* arg, Py_ssize_t nargs) {
  Args a(arg, nargs, 12);
  blink_model_cfg m;
  if (!model_of(a, &m)) return nullptr;
  const blink_kv_pool kv = pool_of(a, m);
  const long layer = a.integer();
  const int64_t q_dim = (int64_t)m.n_q_heads * m.head_dim;
  int64_t stride = 0, out_stride = 0;
  const at::Tensor* q = a.matrix("q", -1, q_dim, type_of(m), &stride);
  const at::Tensor *row_start = a.ints("row_start"), *kv_len = a.ints("kv_len");
  const int64_t n = a.ok ? kv_len->numel() : 0, rows = a.ok ? q->size(0) : 0;
  if (a.ok) a.need(row_start->numel() == n + 1, "row_start: one more than kv_len");
  const at::Tensor* table = a.table(n);
  const long window = a.integer(), sinks = a.integer(), max_new = a.integer();
  const at::Tensor* o = a.matrix("out", rows, q_dim, type_of(m), &out_stride);
  const at::Tensor* given = a.tensor("workspace", true);
  if (a.ok && given) a.need(given->is_contiguous(), "workspace: contiguous");
  if (a.ok) a.need(std::max({n, rows, table->size(1)}) <= 0x7fffffff, "sizes beyond 31 bits");
  if (!a.ok) return nullptr;
  at::Tensor mine;
  if (!given) {
    mine = make({(int64_t)blink_window_attention_workspace(&m, (int)max_new)}, at::kByte, a);
    given = &mine;
  }
  return call(a, [&](void* stream) {
    return blink_window_attention(&m, &kv, (int)layer, at_of(q), stride, (int)rows, in<int32_t>(row_start), in<int32_t>(kv_len), (int)n, in<int32_t>(table),
                                  (int)table->size(1), (int)window, (int)sinks, (int)max_new, out<void>(o), out_stride, out<void>(given), given->nbytes(), stream);
  });
}

// logits, row_start, draft_tokens, draft_probs or None, temperature, u_accept, u_pick, out_tokens, n_accepted, workspace or None, 1 when the tokens'
// memory is new -> error code
PyObject* verify_drafts(PyObject*, PyObject* const* arg, Py_ssize_t nargs) {
  Args a(arg, nargs, 11);
  int64_t stride = 0, probs_stride = 0;
  const at::Tensor* z = a.matrix("logits", -1, -1, at::kFloat, &stride);
  const int64_t rows = a.ok ? z->size(0) : 0, vocab = a.ok ? z->size(1) : 0;
  const at::Tensor *row_start = a.ints("row_start"), *draft = a.ints("draft_tokens", rows);
  const at::Tensor* probs = a.matrix("draft_probs", rows, vocab, at::kFloat, &probs_stride, true);
  const int64_t n = a.ok ? row_start->numel() - 1 : 0;
  const at::Tensor *T = a.floats("temperature", n), *ua = a.floats("u_accept", rows), *up = a.floats("u_pick", n);
  const at::Tensor *tokens = a.ints("out_tokens", rows), *accepted = a.ints("n_accepted", n), *given = a.tensor("workspace", true);
  const bool clear = a.integer() != 0;
  if (a.ok && given) a.need(given->is_contiguous(), "workspace: contiguous");
  if (a.ok) a.need(std::max({n, rows, vocab}) <= 0x7fffffff, "sizes beyond 31 bits");
  if (!a.ok) return nullptr;
  at::Tensor mine;
  if (!given) {
    mine = make({(int64_t)blink_verify_workspace((int)rows, (int)n, (int)vocab)}, at::kByte, a);
    given = &mine;
  }
  return call(a, [&](void* stream) {
    return blink::verify_drafts(in<float>(z), stride, (int)rows, (int)vocab, in<int32_t>(row_start), (int)n, in<int32_t>(draft), in<float>(probs), probs_stride, in<float>(T),
                                in<float>(ua), in<float>(up), out<int32_t>(tokens), out<int32_t>(accepted), out<void>(given), given->nbytes(), clear, stream);
  });
}

// What torch throws (no memory for a workspace) becomes Python's.
template <PyObject* (*F)(PyObject*, PyObject* const*, Py_ssize_t)>
PyObject* guarded(PyObject* self, PyObject* const* arg, Py_ssize_t n) {
  try {
    return F(self, arg, n);
  } catch (const std::exception& e) {
    if (!PyErr_Occurred()) PyErr_SetString(PyExc_RuntimeError, e.what());
  } catch (...) {
    if (!PyErr_Occurred()) PyErr_SetString(PyExc_RuntimeError, "unknown C++ exception");
  }
  return nullptr;
}

#define BLINK_FAST(f) {#f, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(guarded<f>)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {BLINK_FAST(build_tables), BLINK_FAST(qk_norm_rope), BLINK_FAST(window_attention), BLINK_FAST(verify_drafts), {nullptr, nullptr, 0, nullptr}};
#undef BLINK_FAST
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal", "Argument marshalling of the operators of a speculative step.", -1, methods};

}  // namespace

PyMODINIT_FUNC PyInit__marshal() {
  PyObject* m = PyModule_Create(&module);
  if (m && PyModule_AddStringConstant(m, "built", "built for " BLINK_BUILT_FOR ".") != 0) {
    Py_DECREF(m);
    return nullptr;
  }
  return m;
}
