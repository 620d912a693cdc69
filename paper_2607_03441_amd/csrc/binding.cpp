// Native argument marshalling of the Python binding for the calls that take a list of problems: one
// decoding step passes 64 problems of four tensors, an adapter step 256 parameters, and reading those
// tensors attribute by attribute from Python took 145 and 350 us a call, several times the GPU's work;
// and for the calls of a decoding step on the cache, whose few microseconds a dozen Python operations would pass.
// Each function checks and raises exactly as its caller documents and returns the library's status.
#include <Python.h>

#include <c10/core/DeviceGuard.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <ATen/ops/empty.h>

#include <cmath>
#include <optional>
#include <vector>

#include "attt.h"

namespace {

// A Python error is set; unwinds to the module function's handler.
struct PyError {};

[[noreturn]] void raise(PyObject* type, const char* fmt, const char* arg = "") {
  PyErr_Format(type, fmt, arg);
  throw PyError{};
}

// What a call reads, held until it returns: the problems, and the tensors that their mappings hand out.
// Only then may the allocator give their memory to the call's own workspace, whatever the caller's
// objects do meanwhile (a sequence may make its problems on access).
struct Held {
  std::vector<PyObject*> v;
  ~Held() {
    for (PyObject* o : v) Py_DECREF(o);
  }
  PyObject* keep(PyObject* o) {  // takes over the caller's reference
    if (!o) throw PyError{};
    try {
      v.push_back(o);
    } catch (...) {
      Py_DECREF(o);
      throw;
    }
    return o;
  }
};

// The problems of a call: a tuple of their own. Like len(), this refuses what has no length (a generator).
PyObject* list(Held& held, PyObject* seq) {
  const Py_ssize_t n = PyObject_Size(seq);
  if (n < 0) throw PyError{};
  held.v.reserve(1 + 8 * (size_t)n);
  return held.keep(PySequence_Tuple(seq));
}

// A mapping's entry; nullptr when `optional` and absent.
PyObject* item(Held& held, PyObject* map, PyObject* key, bool optional = false) {
  if (PyDict_CheckExact(map)) {
    PyObject* v = PyDict_GetItemWithError(map, key);
    if (v) {
      Py_INCREF(v);
      return held.keep(v);
    }
    if (optional && !PyErr_Occurred()) return nullptr;
    if (!PyErr_Occurred()) PyErr_SetObject(PyExc_KeyError, key);
    throw PyError{};
  }
  return held.keep(optional ? PyObject_CallMethod(map, "get", "O", key) : PyObject_GetItem(map, key));
}

const at::Tensor& tensor(PyObject* o, const char* name) {
  if (!THPVariable_Check(o)) raise(PyExc_TypeError, "%s must be a tensor", name);
  return THPVariable_Unpack(o);
}

const at::Tensor& device_tensor(PyObject* o, const char* name) {
  const at::Tensor& t = tensor(o, name);
  if (!t.is_cuda() || !t.is_contiguous()) raise(PyExc_ValueError, "%s must be a contiguous device tensor", name);
  return t;
}

int64_t dim(const at::Tensor& t, int64_t d) {
  if (d >= t.dim()) raise(PyExc_IndexError, "tuple index out of range");
  return t.size(d);
}

PyObject *k_x, *k_dy, *k_A, *k_B, *k_dA, *k_dB, *k_y, *k_scale, *k_param, *k_grad, *k_param_bf16;

// What float() takes, a number's text too; a TypeError for the rest.
float number(Held& held, PyObject* o) {
  PyObject* f = PyNumber_Float(o);
  if (!f && PyErr_ExceptionMatches(PyExc_ValueError)) PyErr_Format(PyExc_TypeError, "%R is not a number", o);
  return (float)PyFloat_AS_DOUBLE(held.keep(f));
}

float scale_of(Held& held, PyObject* map) { return number(held, item(held, map, k_scale)); }

// The library plans, launches and, the first time, loads its code: other Python threads run meanwhile. The
// tensors stay held, and nothing of Python is touched.
template <class F>
auto without_gil(F f) {
  struct Released {
    PyThreadState* state = PyEval_SaveThread();
    ~Released() { PyEval_RestoreThread(state); }
  } released;
  return f();
}

void* stream() { return c10::hip::getCurrentHIPStream().stream(); }

std::vector<attt_lora_problem> lora_problems(Held& held, PyObject* seq, bool check, at::ScalarType* dt, at::Device* dev) {
  PyObject* f = list(held, seq);
  const Py_ssize_t n = PyTuple_GET_SIZE(f);
  std::vector<attt_lora_problem> v(n);
  for (Py_ssize_t i = 0; i < n; ++i) {
    PyObject* p = PyTuple_GET_ITEM(f, i);
    auto get = [&](PyObject* key, const char* name) -> const at::Tensor& {
      PyObject* o = item(held, p, key);
      return check ? device_tensor(o, name) : tensor(o, name);
    };
    const at::Tensor &x = get(k_x, "x"), &dy = get(k_dy, "dy"), &A = get(k_A, "A"), &B = get(k_B, "B"),
                     &dA = get(k_dA, "dA"), &dB = get(k_dB, "dB");
    if (i == 0 && dt) *dt = x.scalar_type();
    if (i == 0 && dev) *dev = x.device();
    v[i] = {x.data_ptr(), dy.data_ptr(), A.data_ptr(), B.data_ptr(), static_cast<float*>(dA.data_ptr()),
            static_cast<float*>(dB.data_ptr()), dim(x, 0), dim(x, 1), dim(dy, 1), (int32_t)dim(A, 0), scale_of(held, p)};
  }
  return v;
}

// lora_workspace_size(problems, dtype) -> (status, bytes)
PyObject* lora_workspace_size(PyObject* args) {
  Held held;
  PyObject* seq;
  int dtype;
  if (!PyArg_ParseTuple(args, "Oi", &seq, &dtype)) throw PyError{};
  const auto v = lora_problems(held, seq, false, nullptr, nullptr);
  size_t need = 0;
  const attt_status st = without_gil([&] { return attt_lora_workspace_size(v.data(), (int32_t)v.size(), dtype, &need); });
  return Py_BuildValue("in", (int)st, (Py_ssize_t)need);
}

// lora_grad(problems, workspace or None) -> status
PyObject* lora_grad(PyObject* args) {
  Held held;
  PyObject *seq, *ws_obj;
  if (!PyArg_ParseTuple(args, "OO", &seq, &ws_obj)) throw PyError{};
  at::ScalarType dt = at::kFloat;
  at::Device dev(at::kCPU);
  const auto v = lora_problems(held, seq, true, &dt, &dev);
  if (v.empty()) return PyLong_FromLong(ATTT_OK);
  if (dt != at::kFloat && dt != at::kBFloat16)
    raise(PyExc_TypeError, "unsupported dtype torch.%s (float32 or bfloat16)", c10::toString(dt));
  const int32_t dtype = dt == at::kBFloat16 ? ATTT_BF16 : ATTT_F32;
  size_t need = 0;
  attt_status st = without_gil([&] { return attt_lora_workspace_size(v.data(), (int32_t)v.size(), dtype, &need); });
  if (st) return PyLong_FromLong(st);
  at::Tensor ws;
  if (ws_obj != Py_None) ws = tensor(ws_obj, "workspace");
  void* s = stream();
  st = without_gil([&] {
    if (!ws.defined() || ws.numel() < (int64_t)need)
      ws = at::empty({(int64_t)(need > 256 ? need : 256)}, at::TensorOptions().dtype(at::kByte).device(dev));
    return attt_lora_grad(v.data(), (int32_t)v.size(), dtype, ws.data_ptr(), (size_t)ws.numel(), s);
  });
  return PyLong_FromLong(st);
}

// lora_sgd_step(params, lr, zero_grad) -> status
PyObject* lora_sgd_step(PyObject* args) {
  Held held;
  PyObject *seq, *lr_obj;
  int zero;
  if (!PyArg_ParseTuple(args, "OOp", &seq, &lr_obj, &zero)) throw PyError{};
  const float lr = number(held, lr_obj);
  PyObject* f = list(held, seq);
  const Py_ssize_t n = PyTuple_GET_SIZE(f);
  std::vector<attt_lora_param> v(n);
  for (Py_ssize_t i = 0; i < n; ++i) {
    PyObject* p = PyTuple_GET_ITEM(f, i);
    const at::Tensor &P = device_tensor(item(held, p, k_param), "param"), &G = device_tensor(item(held, p, k_grad), "grad");
    if (P.scalar_type() != at::kFloat || G.scalar_type() != at::kFloat || G.numel() != P.numel())
      raise(PyExc_ValueError, "param and grad must be float32 tensors of equal size");
    void* copy = nullptr;
    PyObject* b = item(held, p, k_param_bf16, true);
    if (b && b != Py_None) {
      const at::Tensor& Pb = device_tensor(b, "param_bf16");
      if (Pb.scalar_type() != at::kBFloat16 || Pb.numel() != P.numel())
        raise(PyExc_ValueError, "param_bf16 must be a bfloat16 tensor of the param's size");
      copy = Pb.data_ptr();
    }
    v[i] = {static_cast<float*>(P.data_ptr()), static_cast<float*>(G.data_ptr()), copy, P.numel()};
  }
  void* s = stream();
  return PyLong_FromLong(without_gil([&] { return attt_lora_sgd_step(v.data(), (int32_t)n, lr, zero, s); }));
}

// lora_forward(problems) -> status
PyObject* lora_forward(PyObject* args) {
  Held held;
  PyObject* seq;
  if (!PyArg_ParseTuple(args, "O", &seq)) throw PyError{};
  PyObject* f = list(held, seq);
  const Py_ssize_t n = PyTuple_GET_SIZE(f);
  std::vector<attt_lora_fwd_problem> v(n);
  for (Py_ssize_t i = 0; i < n; ++i) {
    PyObject* p = PyTuple_GET_ITEM(f, i);
    auto get = [&](PyObject* key, const char* name) -> const at::Tensor& {
      const at::Tensor& t = device_tensor(item(held, p, key), name);
      if (t.scalar_type() != at::kBFloat16 || t.dim() != 2) raise(PyExc_ValueError, "%s must be a 2-D bfloat16 tensor", name);
      return t;
    };
    const at::Tensor &x = get(k_x, "x"), &y = get(k_y, "y"), &A = get(k_A, "A"), &B = get(k_B, "B");
    v[i] = {x.data_ptr(), y.data_ptr(), A.data_ptr(), B.data_ptr(), x.size(0), x.size(1), y.size(1), (int32_t)A.size(0),
            scale_of(held, p)};
  }
  void* s = stream();
  return PyLong_FromLong(without_gil([&] { return attt_lora_forward(v.data(), (int32_t)n, s); }));
}

// lora_hot_swap(pairs) -> status
PyObject* lora_hot_swap(PyObject* args) {
  Held held;
  PyObject* seq;
  if (!PyArg_ParseTuple(args, "O", &seq)) throw PyError{};
  PyObject* f = list(held, seq);
  const Py_ssize_t n = PyTuple_GET_SIZE(f);
  std::vector<attt_lora_swap_item> v(n);
  for (Py_ssize_t i = 0; i < n; ++i) {
    PyObject* pair = held.keep(PySequence_Tuple(PyTuple_GET_ITEM(f, i)));
    if (PyTuple_GET_SIZE(pair) != 2) raise(PyExc_ValueError, "a pair must be (src, dst)");
    const at::Tensor &src = device_tensor(PyTuple_GET_ITEM(pair, 0), "src"),
                     &dst = device_tensor(PyTuple_GET_ITEM(pair, 1), "dst");
    if (src.scalar_type() != at::kFloat || dst.scalar_type() != at::kBFloat16 || src.numel() != dst.numel())
      raise(PyExc_ValueError, "src must be float32 and dst bfloat16 of the same numel");
    v[i] = {static_cast<const float*>(src.data_ptr()), dst.data_ptr(), src.numel()};
  }
  void* s = stream();
  return PyLong_FromLong(without_gil([&] { return attt_lora_hot_swap(v.data(), (int32_t)n, s); }));
}

// ---- calls on single tensors: attention, the 4-bit cache, log-probabilities ---------------------------

// A contiguous device tensor of a dtype and shape (-1: any), on the device of those before it.
struct Checked {
  std::optional<at::Device> device;

  const at::Tensor& operator()(PyObject* o, const char* name, at::ScalarType dt, std::initializer_list<int64_t> shape) {
    const at::Tensor& t = device_tensor(o, name);
    if (t.scalar_type() != dt) {
      PyErr_Format(PyExc_TypeError, "%s must be %s", name, lower(dt));
      throw PyError{};
    }
    bool fits = t.dim() == (int64_t)shape.size();
    int64_t d = 0;
    for (int64_t n : shape) {
      fits = fits && (n < 0 || t.size(d) == n);
      ++d;
    }
    if (!fits) raise(PyExc_ValueError, "%s has a shape that does not fit the other arguments", name);
    if (device && *device != t.device()) raise(PyExc_ValueError, "%s is on another device than the arguments before it", name);
    device = t.device();
    return t;
  }
  static const char* lower(at::ScalarType dt) {
    return dt == at::kFloat ? "float32" : dt == at::kBFloat16 ? "bfloat16" : dt == at::kInt ? "int32" : "uint8";
  }
};

// Host offsets [E + 1]: an int64 array, or any sequence of integers; None: not given.
struct Offsets {
  std::vector<int64_t> v;
  const int64_t* data() const { return v.empty() ? nullptr : v.data(); }
  int32_t count(int64_t none) const { return v.empty() ? (int32_t)none : (int32_t)(v.size() - 1); }

  Offsets(Held& held, PyObject* o) {
    if (o == Py_None) return;
    Py_buffer b;
    if (PyObject_CheckBuffer(o) && PyObject_GetBuffer(o, &b, PyBUF_FORMAT | PyBUF_ND) == 0) {
      const bool plain = b.ndim == 1 && b.itemsize == 8 && b.format && (b.format[0] == 'l' || b.format[0] == 'q') && !b.format[1];
      if (plain) v.assign(static_cast<const int64_t*>(b.buf), static_cast<const int64_t*>(b.buf) + b.shape[0]);
      PyBuffer_Release(&b);
      if (plain) {
        check();
        return;
      }
    }
    PyErr_Clear();  // a strided array: item by item
    PyObject* f = held.keep(PySequence_Tuple(o));
    v.resize(PyTuple_GET_SIZE(f));
    for (size_t i = 0; i < v.size(); ++i) {
      PyObject* n = held.keep(PyNumber_Index(PyTuple_GET_ITEM(f, i)));
      v[i] = PyLong_AsLongLong(n);
      if (v[i] == -1 && PyErr_Occurred()) throw PyError{};
    }
    check();
  }
  void check() const {
    if (v.empty()) raise(PyExc_ValueError, "offsets need at least one entry");
    if (v.size() > INT32_MAX) raise(PyExc_ValueError, "too many offsets");
  }
};

// The members of an `out` tuple of n tensors, or nothing.
PyObject* const* members(Held& held, PyObject* out, Py_ssize_t n) {
  if (out == Py_None) return nullptr;
  PyObject* f = held.keep(PySequence_Tuple(out));
  if (PyTuple_GET_SIZE(f) != n) raise(PyExc_ValueError, "out has another number of tensors than the call returns");
  return &PyTuple_GET_ITEM(f, 0);
}

at::Tensor empty(at::IntArrayRef shape, at::ScalarType dt, at::Device dev) {
  return at::empty(shape, at::TensorOptions().dtype(dt).device(dev));
}

// The caller's workspace where it is large enough, or one of the call's own.
struct Workspace {
  at::Tensor t;
  void take(PyObject* o, Checked& check) {
    if (o != Py_None) t = check(o, "workspace", at::kByte, {-1});
  }
  void need(size_t bytes, at::Device dev) {
    if (bytes && (!t.defined() || (size_t)t.numel() < bytes)) t = empty({(int64_t)bytes}, at::kByte, dev);
  }
  void* data() const { return t.defined() ? t.data_ptr() : nullptr; }
  size_t bytes() const { return t.defined() ? (size_t)t.numel() : 0; }
};

void* stream(at::Device dev) { return c10::hip::getCurrentHIPStream(dev.index()).stream(); }

float scale_or(Held& held, PyObject* o, int64_t head_dim) {
  return o == Py_None ? (float)(1.0 / std::sqrt((double)head_dim)) : number(held, o);
}

PyObject* wrap(const at::Tensor& t) {
  if (t.defined()) return THPVariable_Wrap(t);
  Py_RETURN_NONE;
}

// attention_fwd(q, k, v, row_offsets, scale, out) -> (status, o, lse)
PyObject* attention_fwd(PyObject* args) {
  Held held;
  PyObject *q_, *k_, *v_, *off_, *scale_, *out_;
  if (!PyArg_ParseTuple(args, "OOOOOO", &q_, &k_, &v_, &off_, &scale_, &out_)) throw PyError{};
  Checked check;
  const at::Tensor& q = check(q_, "q", at::kBFloat16, {-1, -1, -1});
  const int64_t N = q.size(0), H = q.size(1), D = q.size(2);
  const at::Tensor& k = check(k_, "k", at::kBFloat16, {N, -1, D});
  const int64_t kv = k.size(1);
  const at::Tensor& v = check(v_, "v", at::kBFloat16, {N, kv, D});
  const Offsets off(held, off_);
  const float scale = scale_or(held, scale_, D);
  at::Tensor o, lse;
  if (PyObject* const* m = members(held, out_, 2)) {
    o = check(m[0], "out[0]", at::kBFloat16, {N, H, D});
    lse = check(m[1], "out[1]", at::kFloat, {H, N});
  }
  const attt_status st = without_gil([&] {
    const at::Device dev = *check.device;
    const c10::DeviceGuard guard(dev);
    if (!o.defined()) o = empty({N, H, D}, at::kBFloat16, dev), lse = empty({H, N}, at::kFloat, dev);
    return attt_attention_fwd(q.data_ptr(), k.data_ptr(), v.data_ptr(), off.data(), off.count(1), N, (int32_t)H, (int32_t)kv,
                              (int32_t)D, scale, o.data_ptr(), static_cast<float*>(lse.data_ptr()), stream(dev));
  });
  return Py_BuildValue("iNN", (int)st, wrap(o), wrap(lse));
}

// attention_bwd_saved(q, k, v, o, lse, dout, row_offsets, scale, out, workspace) -> (status, dq, dk, dv, dsum)
PyObject* attention_bwd_saved(PyObject* args) {
  Held held;
  PyObject *q_, *k_, *v_, *o_, *lse_, *do_, *off_, *scale_, *out_, *ws_;
  if (!PyArg_ParseTuple(args, "OOOOOOOOOO", &q_, &k_, &v_, &o_, &lse_, &do_, &off_, &scale_, &out_, &ws_)) throw PyError{};
  Checked check;
  const at::Tensor& q = check(q_, "q", at::kBFloat16, {-1, -1, -1});
  const int64_t N = q.size(0), H = q.size(1), D = q.size(2);
  const at::Tensor& k = check(k_, "k", at::kBFloat16, {N, -1, D});
  const int64_t kv = k.size(1);
  const at::Tensor& v = check(v_, "v", at::kBFloat16, {N, kv, D});
  const at::Tensor& o = check(o_, "o", at::kBFloat16, {N, H, D});
  const at::Tensor& lse = check(lse_, "lse", at::kFloat, {H, N});
  const at::Tensor& dout = check(do_, "dout", at::kBFloat16, {N, H, D});
  const Offsets off(held, off_);
  const float scale = scale_or(held, scale_, D);
  at::Tensor dq, dk, dv, dsum;
  if (PyObject* const* m = members(held, out_, 4)) {
    dq = check(m[0], "out[0]", at::kBFloat16, {N, H, D});
    dk = check(m[1], "out[1]", at::kBFloat16, {N, kv, D});
    dv = check(m[2], "out[2]", at::kBFloat16, {N, kv, D});
    dsum = check(m[3], "out[3]", at::kFloat, {H, N});
  }
  Workspace ws;
  ws.take(ws_, check);
  const attt_status st = without_gil([&]() -> attt_status {
    const at::Device dev = *check.device;
    const c10::DeviceGuard guard(dev);
    if (!dq.defined()) {
      dq = empty({N, H, D}, at::kBFloat16, dev);
      dk = empty({N, kv, D}, at::kBFloat16, dev);
      dv = empty({N, kv, D}, at::kBFloat16, dev);
      dsum = empty({H, N}, at::kFloat, dev);
    }
    size_t need = 0;
    if (attt_status e = attt_attention_workspace_size(off.data(), off.count(1), N, (int32_t)H, (int32_t)kv, (int32_t)D, &need))
      return e;
    try {
      ws.need(need, dev);
    } catch (const c10::OutOfMemoryError&) {  // the call does without
      ws.t = at::Tensor();
    }
    return attt_attention_bwd_saved(q.data_ptr(), k.data_ptr(), v.data_ptr(), o.data_ptr(),
                                    static_cast<const float*>(lse.data_ptr()), dout.data_ptr(), off.data(), off.count(1), N,
                                    (int32_t)H, (int32_t)kv, (int32_t)D, scale, dq.data_ptr(), dk.data_ptr(), dv.data_ptr(),
                                    static_cast<float*>(dsum.data_ptr()), need ? ws.data() : nullptr, need ? ws.bytes() : 0,
                                    stream(dev));
  });
  return Py_BuildValue("iNNNN", (int)st, wrap(dq), wrap(dk), wrap(dv), wrap(dsum));
}

// kv4_append(cache, k, v, page_table, lengths, row_offsets, want_held, out) -> (status, k_held, v_held)
PyObject* kv4_append(PyObject* args) {
  Held held;
  PyObject *cache_, *k_, *v_, *table_, *len_, *off_, *out_;
  int want;
  if (!PyArg_ParseTuple(args, "OOOOOOpO", &cache_, &k_, &v_, &table_, &len_, &off_, &want, &out_)) throw PyError{};
  Checked check;
  const at::Tensor& k = check(k_, "k", at::kBFloat16, {-1, -1, -1});
  const int64_t N = k.size(0), kv = k.size(1), D = k.size(2);
  const at::Tensor& v = check(v_, "v", at::kBFloat16, {N, kv, D});
  const at::Tensor& cache = check(cache_, "cache", at::kByte, {-1, kv, ATTT_KV4_RECORD_BYTES});
  const at::Tensor& len = check(len_, "lengths", at::kInt, {-1});
  const at::Tensor& table = check(table_, "page_table", at::kInt, {len.size(0), -1});
  const Offsets off(held, off_);
  if (off.count(len.size(0)) != len.size(0)) raise(PyExc_ValueError, "one length per sequence");
  at::Tensor kh, vh;
  if (PyObject* const* m = members(held, out_, 2)) {
    kh = check(m[0], "out[0]", at::kBFloat16, {N, kv, D});
    vh = check(m[1], "out[1]", at::kBFloat16, {N, kv, D});
  }
  const attt_status st = without_gil([&] {
    const at::Device dev = *check.device;
    const c10::DeviceGuard guard(dev);
    if (want && !kh.defined()) kh = empty({N, kv, D}, at::kBFloat16, dev), vh = empty({N, kv, D}, at::kBFloat16, dev);
    return attt_kv4_append(cache.data_ptr(), cache.size(0), k.data_ptr(), v.data_ptr(), static_cast<const int32_t*>(table.data_ptr()),
                           table.size(1), static_cast<const int32_t*>(len.data_ptr()), off.data(), (int32_t)len.size(0), N,
                           (int32_t)kv, (int32_t)D, kh.defined() ? kh.data_ptr() : nullptr,
                           vh.defined() ? vh.data_ptr() : nullptr, stream(dev));
  });
  return Py_BuildValue("iNN", (int)st, wrap(kh), wrap(vh));
}

// kv4_attention(q, cache, page_table, lengths, row_offsets, scale, max_length, out, workspace) -> (status, o, lse)
PyObject* kv4_attention(PyObject* args) {
  Held held;
  PyObject *q_, *cache_, *table_, *len_, *off_, *scale_, *most_, *out_, *ws_;
  if (!PyArg_ParseTuple(args, "OOOOOOOOO", &q_, &cache_, &table_, &len_, &off_, &scale_, &most_, &out_, &ws_)) throw PyError{};
  Checked check;
  const at::Tensor& q = check(q_, "q", at::kBFloat16, {-1, -1, -1});
  const int64_t N = q.size(0), H = q.size(1), D = q.size(2);
  const at::Tensor& cache = check(cache_, "cache", at::kByte, {-1, -1, ATTT_KV4_RECORD_BYTES});
  const int64_t kv = cache.size(1);
  const at::Tensor& len = check(len_, "lengths", at::kInt, {-1});
  const at::Tensor& table = check(table_, "page_table", at::kInt, {len.size(0), -1});
  const Offsets off(held, off_);
  if (off.count(len.size(0)) != len.size(0)) raise(PyExc_ValueError, "one length per sequence");
  const float scale = scale_or(held, scale_, D);
  int64_t most = table.size(1) * ATTT_KV4_PAGE_TOKENS;
  if (most_ != Py_None) {
    most = PyLong_AsLongLong(held.keep(PyNumber_Index(most_)));
    if (most == -1 && PyErr_Occurred()) throw PyError{};
  }
  at::Tensor o, lse;
  if (PyObject* const* m = members(held, out_, 2)) {
    o = check(m[0], "out[0]", at::kBFloat16, {N, H, D});
    lse = check(m[1], "out[1]", at::kFloat, {H, N});
  }
  Workspace ws;
  ws.take(ws_, check);
  const attt_status st = without_gil([&]() -> attt_status {
    const at::Device dev = *check.device;
    const c10::DeviceGuard guard(dev);
    if (!o.defined()) o = empty({N, H, D}, at::kBFloat16, dev), lse = empty({H, N}, at::kFloat, dev);
    size_t need = 0;
    if (attt_status e = attt_kv4_attention_workspace_size(off.data(), (int32_t)len.size(0), N, (int32_t)H, (int32_t)kv,
                                                          (int32_t)D, most, &need))
      return e;
    ws.need(need, dev);
    return attt_kv4_attention(q.data_ptr(), cache.data_ptr(), cache.size(0), static_cast<const int32_t*>(table.data_ptr()),
                              table.size(1), static_cast<const int32_t*>(len.data_ptr()), off.data(), (int32_t)len.size(0), N,
                              (int32_t)H, (int32_t)kv, (int32_t)D, most, scale, o.data_ptr(),
                              static_cast<float*>(lse.data_ptr()), ws.data(), ws.bytes(), stream(dev));
  });
  return Py_BuildValue("iNN", (int)st, wrap(o), wrap(lse));
}

// token_logprobs(hidden, lm_head, labels, top, out, workspace) -> (status, logp, entropy, top_ids, top_logp)
PyObject* token_logprobs(PyObject* args) {
  Held held;
  PyObject *h_, *w_, *y_, *out_, *ws_;
  int top;
  if (!PyArg_ParseTuple(args, "OOOiOO", &h_, &w_, &y_, &top, &out_, &ws_)) throw PyError{};
  Checked check;
  const at::ScalarType dt = tensor(h_, "hidden").scalar_type();
  if (dt != at::kFloat && dt != at::kBFloat16)
    raise(PyExc_TypeError, "unsupported dtype torch.%s (float32 or bfloat16)", c10::toString(dt));
  const int32_t dtype = dt == at::kBFloat16 ? ATTT_BF16 : ATTT_F32;
  const at::Tensor& h = check(h_, "hidden", dt, {-1, -1});
  const int64_t N = h.size(0), d = h.size(1);
  const at::Tensor& w = check(w_, "lm_head", dt, {-1, d});
  const int64_t V = w.size(0);
  const at::Tensor& y = check(y_, "labels", at::kInt, {N});
  at::Tensor logp, entropy, ids, lp;
  if (PyObject* const* m = members(held, out_, top > 0 ? 4 : 2)) {
    logp = check(m[0], "out[0]", at::kFloat, {N});
    if (m[1] != Py_None) entropy = check(m[1], "out[1]", at::kFloat, {N});
    if (top > 0) ids = check(m[2], "out[2]", at::kInt, {N, top}), lp = check(m[3], "out[3]", at::kFloat, {N, top});
  }
  Workspace ws;
  ws.take(ws_, check);
  const attt_status st = without_gil([&]() -> attt_status {
    const at::Device dev = *check.device;
    const c10::DeviceGuard guard(dev);
    size_t need = 0;
    if (attt_status e = attt_logprobs_workspace_size(N, d, V, dtype, top, &need)) return e;
    if (!logp.defined()) {
      logp = empty({N}, at::kFloat, dev);
      entropy = empty({N}, at::kFloat, dev);
      if (top > 0) ids = empty({N, top}, at::kInt, dev), lp = empty({N, top}, at::kFloat, dev);
    }
    ws.need(need, dev);
    auto f = [](const at::Tensor& t) { return t.defined() ? static_cast<float*>(t.data_ptr()) : nullptr; };
    return attt_token_logprobs(h.data_ptr(), w.data_ptr(), static_cast<const int32_t*>(y.data_ptr()), N, d, V, dtype, top,
                               f(logp), f(entropy), ids.defined() ? static_cast<int32_t*>(ids.data_ptr()) : nullptr, f(lp),
                               ws.data(), ws.bytes(), stream(dev));
  });
  return Py_BuildValue("iNNNN", (int)st, wrap(logp), wrap(entropy), wrap(ids), wrap(lp));
}

// No C++ exception leaves a module function; torch's become the Python errors they are elsewhere (its
// OutOfMemoryError among them).
template <PyObject* (*Fn)(PyObject*)>
PyObject* guarded(PyObject*, PyObject* args) {
  HANDLE_TH_ERRORS
  try {
    return Fn(args);
  } catch (const PyError&) {
    return nullptr;
  }
  END_HANDLE_TH_ERRORS
}

PyMethodDef kMethods[] = {{"lora_workspace_size", guarded<lora_workspace_size>, METH_VARARGS, nullptr},
                          {"lora_grad", guarded<lora_grad>, METH_VARARGS, nullptr},
                          {"lora_sgd_step", guarded<lora_sgd_step>, METH_VARARGS, nullptr},
                          {"lora_forward", guarded<lora_forward>, METH_VARARGS, nullptr},
                          {"lora_hot_swap", guarded<lora_hot_swap>, METH_VARARGS, nullptr},
                          {"attention_fwd", guarded<attention_fwd>, METH_VARARGS, nullptr},
                          {"attention_bwd_saved", guarded<attention_bwd_saved>, METH_VARARGS, nullptr},
                          {"kv4_append", guarded<kv4_append>, METH_VARARGS, nullptr},
                          {"kv4_attention", guarded<kv4_attention>, METH_VARARGS, nullptr},
                          {"token_logprobs", guarded<token_logprobs>, METH_VARARGS, nullptr},
                          {nullptr, nullptr, 0, nullptr}};

PyModuleDef kModule = {PyModuleDef_HEAD_INIT, "_binding", "argument marshalling of libattt.so's calls", -1, kMethods,
                       nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__binding(void) {
  struct {
    PyObject** at;
    const char* name;
  } keys[] = {{&k_x, "x"},   {&k_dy, "dy"}, {&k_A, "A"},         {&k_B, "B"},         {&k_dA, "dA"},   {&k_dB, "dB"},
              {&k_y, "y"},   {&k_scale, "scale"}, {&k_param, "param"}, {&k_grad, "grad"}, {&k_param_bf16, "param_bf16"}};
  for (auto& k : keys)
    if (!(*k.at = PyUnicode_InternFromString(k.name))) return nullptr;
  return PyModule_Create(&kModule);
}
