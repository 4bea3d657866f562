// The binding of the paged cache's entry points (smetric_kv.h): tensors checked and their
// addresses, shapes and strides handed on, on the current stream of the current device, which has
// to be all tensors' device.
//
// A single token's calls are bound by this: a launch takes 2.7 us, and reading a tensor's type,
// shape, strides and address from Python takes 0.6 us each, five of them in an append (8.6 us
// a call through ctypes, where the kernel itself takes less than three).
#include <Python.h>

#include <c10/hip/HIPFunctions.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include "smetric_kv.h"

namespace {

struct Refused {  // a Python exception that has been set
};
[[noreturn]] void refuse(PyObject *type, const char *format, const char *name) {
  PyErr_Format(type, format, name);
  throw Refused{};
}
[[noreturn]] void refuse_type(const char *name, const char *what) {
  PyErr_Format(PyExc_TypeError, "%s: expected a %s CUDA tensor", name, what);
  throw Refused{};
}

const char *name_of(at::ScalarType t) {
  return t == at::kBFloat16 ? "bfloat16" : t == at::kHalf ? "float16" : t == at::kFloat ? "float32"
         : t == at::kInt ? "int32" : t == at::kLong ? "int64" : "differently typed";
}
// The device of a call: its first tensor's, and every other one's.
struct Device {
  int64_t index = -1;
  void holds(int64_t i, const char *name) {
    if (index < 0) index = i;
    if (i != index) refuse(PyExc_ValueError, "%s: on another device than the call's other tensors", name);
  }
};
const at::Tensor &tensor(Device &d, PyObject *o, at::ScalarType type, const char *name) {
  if (!THPVariable_Check(o)) refuse_type(name, name_of(type));
  const at::Tensor &t = THPVariable_Unpack(o);
  if (t.scalar_type() != type || !t.is_cuda() || t.layout() != at::kStrided) refuse_type(name, name_of(type));
  d.holds(t.get_device(), name);
  return t;
}
// Contiguous, or NULL for None.
template <typename T>
T *array(Device &d, PyObject *o, at::ScalarType type, const char *name) {
  if (o == Py_None) return nullptr;
  const at::Tensor &t = tensor(d, o, type, name);
  if (!t.is_contiguous()) refuse(PyExc_TypeError, "%s: expected a contiguous CUDA tensor", name);
  return static_cast<T *>(t.data_ptr());
}

// The activations' type, which every other one has to have.
at::ScalarType activations(PyObject *o, const char *name) {
  if (THPVariable_Check(o)) {
    const at::Tensor &t = THPVariable_Unpack(o);
    if ((t.scalar_type() == at::kBFloat16 || t.scalar_type() == at::kHalf) && t.dim() == 3 && t.is_cuda()) return t.scalar_type();
  }
  refuse(PyExc_TypeError, "%s: expected a bfloat16 or float16 CUDA tensor [tokens, heads, head_dim]", name);
}
int32_t code_of(at::ScalarType t) { return t == at::kBFloat16 ? SMETRIC_BF16 : SMETRIC_F16; }

// An activation [tokens, heads, head_dim]; heads < 0: any number.
struct Heads : smetric_heads {
  int64_t tokens, heads, dim;
};
Heads heads(Device &dev, PyObject *o, at::ScalarType type, const char *name, int64_t tokens, int64_t n_heads, int64_t dim) {
  const at::Tensor &t = tensor(dev, o, type, name);
  const bool fits = t.dim() == 3 && (tokens < 0 || t.size(0) == tokens) && (n_heads < 0 || t.size(1) == n_heads) &&
                    (dim < 0 || t.size(2) == dim);
  if (!fits || t.stride(2) != 1) {
    if (tokens < 0 || n_heads < 0 || dim < 0)
      refuse(PyExc_ValueError, "%s: expected [tokens, heads, head_dim] with contiguous components", name);
    PyErr_Format(PyExc_ValueError, "%s: expected shape (%lld, %lld, %lld) with contiguous components", name,
                 (long long)tokens, (long long)n_heads, (long long)dim);
    throw Refused{};
  }
  Heads h;
  h.data = t.data_ptr();
  h.token_stride = t.stride(0);
  h.head_stride = t.stride(1);
  h.tokens = t.size(0);
  h.heads = t.size(1);
  h.dim = t.size(2);
  return h;
}

void check_weight(PyObject *o, at::ScalarType type, int64_t dim, const char *name) {
  if (o == Py_None) return;
  if (!THPVariable_Check(o) || THPVariable_Unpack(o).scalar_type() != type || THPVariable_Unpack(o).numel() != dim) {
    PyErr_Format(PyExc_ValueError, "%s: expected %lld values of %s", name, (long long)dim, name_of(type));
    throw Refused{};
  }
}
const int32_t *positions_of(Device &d, PyObject *o, int64_t tokens) {
  const int32_t *p = array<const int32_t>(d, o, at::kInt, "positions");
  if (p || o != Py_None) {
    if (THPVariable_Unpack(o).numel() != tokens) refuse(PyExc_ValueError, "%s: expected one per token", "positions");
  }
  return p;
}
smetric_batch batch_of(Device &d, PyObject *table, PyObject *q_off, PyObject *kv_len, int64_t tokens) {
  if (!THPVariable_Check(table) || THPVariable_Unpack(table).dim() != 2)
    refuse(PyExc_TypeError, "%s: expected an int32 CUDA matrix", "page_table");
  const at::Tensor &t = tensor(d, table, at::kInt, "page_table");
  smetric_batch b;
  b.q_off = array<const int64_t>(d, q_off, at::kLong, "q_off");
  b.kv_len = array<const int32_t>(d, kv_len, at::kInt, "kv_len");
  if (q_off == Py_None || kv_len == Py_None) refuse(PyExc_TypeError, "%s: expected CUDA tensors", "q_off and kv_len");
  const int64_t n_req = THPVariable_Unpack(kv_len).numel(), width = t.size(1);
  if (t.size(0) != n_req || (width > 1 && t.stride(1) != 1))
    refuse(PyExc_ValueError, "%s: expected a row of contiguous entries per request", "page_table");
  if (THPVariable_Unpack(q_off).numel() != n_req + 1)
    refuse(PyExc_ValueError, "%s: expected one entry more than kv_len", "q_off");
  if (n_req > INT32_MAX || width > INT32_MAX) refuse(PyExc_ValueError, "%s: too large", "page_table");
  b.table = static_cast<const int32_t *>(t.data_ptr());
  b.table_stride = n_req < 2 && t.stride(0) < width ? width : t.stride(0);
  b.max_pages = int32_t(width);
  b.n_req = int32_t(n_req);
  b.n_tokens = tokens;
  return b;
}

int64_t whole(PyObject *o) {
  const long long x = PyLong_AsLongLong(o);
  if (x == -1 && PyErr_Occurred()) throw Refused{};
  return x;
}
int32_t whole32(PyObject *o) {
  const int64_t x = whole(o);
  if (x < INT32_MIN || x > INT32_MAX) refuse(PyExc_OverflowError, "%s does not fit 32 bits", "argument");
  return int32_t(x);
}
void same_device(Device &d, PyObject *index, const char *name) {  // of what comes by address; -1: nothing
  const int64_t i = whole(index);
  if (i >= 0) d.holds(i, name);
}
template <typename T>
T *address(PyObject *o) {
  return reinterpret_cast<T *>(uintptr_t(whole(o)));
}
hipStream_t stream(const Device &d) {
  const c10::DeviceIndex now = c10::hip::current_device();
  if (d.index >= 0 && d.index != now) refuse(PyExc_ValueError, "%s: not on the current device", "tensors");
  return c10::hip::getCurrentHIPStream(now).stream();
}

// Runs f(args), which returns the call's status; no C++ exception leaves.
template <typename F>
PyObject *guarded(Py_ssize_t n, Py_ssize_t want, F f) {
  try {
    if (n != want) refuse(PyExc_TypeError, "%s of arguments", "wrong number");
    return PyLong_FromLong(f());
  } catch (const Refused &) {
  } catch (const std::exception &e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
  }
  return nullptr;
}
// The entry point without the interpreter's lock: a full queue makes a launch wait.
template <typename F>
int unlocked(F f) {
  int rc;
  Py_BEGIN_ALLOW_THREADS
  rc = f();
  Py_END_ALLOW_THREADS
  return rc;
}

// (q, k, rotary's address, q_weight, k_weight, positions, q_out, k_out, status, rotary's device or -1)
PyObject *qk_rotate(PyObject *, PyObject *const *a, Py_ssize_t n) {
  return guarded(n, 10, [&] {
    Device d;
    const at::ScalarType type = activations(a[0], "q");
    const Heads q = heads(d, a[0], type, "q", -1, -1, -1), k = heads(d, a[1], type, "k", q.tokens, -1, q.dim);
    const Heads q_out = heads(d, a[6], type, "q_out", q.tokens, q.heads, q.dim);
    const Heads k_out = heads(d, a[7], type, "k_out", q.tokens, k.heads, q.dim);
    check_weight(a[3], type, q.dim, "q_weight");
    check_weight(a[4], type, q.dim, "k_weight");
    const auto *rotary = address<const smetric_rotary>(a[2]);
    const int32_t *positions = positions_of(d, a[5], q.tokens);
    int32_t *status = array<int32_t>(d, a[8], at::kInt, "status");
    same_device(d, a[9], "rotary");
    const hipStream_t s = stream(d);
    return unlocked([&] {
      return smetric_qk_rotate(code_of(type), int32_t(q.dim), q.tokens, rotary, positions, int32_t(q.heads), &q, &q_out,
                               int32_t(k.heads), &k, &k_out, status, s);
    });
  });
}

// (cache's address, page_table, q_off, kv_len, k, v, q, q_out, rotary's address or 0, q_weight,
// k_weight, positions, status, cache's device, rotary's or -1)
PyObject *append(PyObject *, PyObject *const *a, Py_ssize_t n) {
  return guarded(n, 15, [&] {
    Device d;
    same_device(d, a[13], "cache");
    same_device(d, a[14], "rotary");
    const auto *cache = address<const smetric_kv_cache>(a[0]);
    const at::ScalarType type = activations(a[4], "k");
    const Heads k = heads(d, a[4], type, "k", -1, cache->n_kv_heads, cache->head_dim);
    const Heads v = heads(d, a[5], type, "v", k.tokens, k.heads, k.dim);
    const smetric_batch batch = batch_of(d, a[1], a[2], a[3], k.tokens);
    const auto *rotary = address<const smetric_rotary>(a[8]);
    check_weight(a[9], type, k.dim, "q_weight");
    check_weight(a[10], type, k.dim, "k_weight");
    const int32_t *positions = positions_of(d, a[11], k.tokens);
    int32_t *status = array<int32_t>(d, a[12], at::kInt, "status");
    const bool queries = a[6] != Py_None;
    Heads q{}, q_out{};
    if (queries) {
      q = heads(d, a[6], type, "q", k.tokens, -1, k.dim);
      q_out = heads(d, a[7], type, "q_out", k.tokens, q.heads, k.dim);
    }
    const hipStream_t s = stream(d);
    return unlocked([&] {
      return smetric_kv_append(code_of(type), cache, &batch, rotary, positions, queries ? int32_t(q.heads) : 0,
                               queries ? &q : nullptr, queries ? &q_out : nullptr, &k, &v, status, s);
    });
  });
}

// (q_off, kv_len, n_req, n_tokens, n_q_heads, n_kv_heads, head_dim, max_new, window, plan's
// address, bytes, status, plan's device)
PyObject *make_plan(PyObject *, PyObject *const *a, Py_ssize_t n) {
  return guarded(n, 13, [&] {
    Device d;
    same_device(d, a[12], "plan");
    const auto *q_off = array<const int64_t>(d, a[0], at::kLong, "q_off");
    const auto *kv_len = array<const int32_t>(d, a[1], at::kInt, "kv_len");
    const int64_t n_req = whole32(a[2]);
    if (a[0] == Py_None || a[1] == Py_None) refuse(PyExc_TypeError, "%s: expected CUDA tensors", "q_off and kv_len");
    if (THPVariable_Unpack(a[1]).numel() != n_req || THPVariable_Unpack(a[0]).numel() != n_req + 1)
      refuse(PyExc_ValueError, "%s: not of the plan's requests", "q_off, kv_len");
    int32_t *status = array<int32_t>(d, a[11], at::kInt, "status");
    const int64_t tokens = whole(a[3]), bytes = whole(a[10]);
    const int32_t n_q = whole32(a[4]), n_kv = whole32(a[5]), dim = whole32(a[6]), max_new = whole32(a[7]), window = whole32(a[8]);
    void *plan = address<void>(a[9]);
    const hipStream_t s = stream(d);
    return unlocked([&] {
      return smetric_attend_plan(q_off, kv_len, int32_t(n_req), tokens, n_q, n_kv, dim, max_new, window, plan, uint64_t(bytes),
                                 status, s);
    });
  });
}

// (q, out, lse, cache's address, page_table, q_off, kv_len, n_tokens, n_q_heads, scale, max_new, window, plan's
// address, bytes, workspace's address, bytes, status, cache's device, plan's)
PyObject *attend(PyObject *, PyObject *const *a, Py_ssize_t n) {
  return guarded(n, 19, [&] {
    Device d;
    same_device(d, a[17], "cache");
    same_device(d, a[18], "plan");
    const auto *cache = address<const smetric_kv_cache>(a[3]);
    const at::ScalarType type = activations(a[0], "q");
    const int64_t tokens = whole(a[7]);
    const int32_t n_q = whole32(a[8]);
    const Heads q = heads(d, a[0], type, "q", tokens, n_q, cache->head_dim);
    const Heads out = heads(d, a[1], type, "out", tokens, n_q, cache->head_dim);
    float *lse = array<float>(d, a[2], at::kFloat, "lse");
    if (a[2] != Py_None) {
      const at::Tensor &t = THPVariable_Unpack(a[2]);
      if (t.dim() != 2 || t.size(0) != tokens || t.size(1) != n_q)
        refuse(PyExc_ValueError, "%s: expected one per token and query head", "lse");
    }
    const smetric_batch batch = batch_of(d, a[4], a[5], a[6], tokens);
    const double scale = PyFloat_AsDouble(a[9]);
    if (scale == -1.0 && PyErr_Occurred()) throw Refused{};
    const int32_t max_new = whole32(a[10]), window = whole32(a[11]);
    const void *plan = address<const void>(a[12]);
    void *workspace = address<void>(a[14]);
    const uint64_t plan_bytes = uint64_t(whole(a[13])), ws_bytes = uint64_t(whole(a[15]));
    int32_t *status = array<int32_t>(d, a[16], at::kInt, "status");
    const hipStream_t s = stream(d);
    return unlocked([&] {
      return smetric_attend(code_of(type), cache, &batch, n_q, &q, &out, lse, float(scale), max_new, window, plan, plan_bytes,
                            workspace, ws_bytes, status, s);
    });
  });
}

#define CALL(f) #f, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f)), METH_FASTCALL, nullptr
PyMethodDef methods[] = {{CALL(qk_rotate)}, {CALL(append)}, {CALL(make_plan)}, {CALL(attend)}, {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_kv_calls", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__kv_calls() { return PyModule_Create(&module); }
