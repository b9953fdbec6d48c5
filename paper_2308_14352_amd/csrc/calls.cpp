// The calls of the operators beside the layer from Python, without the interpreter between a call and its launch: the checks of the
// tensors, the outputs' memory and the C ABI call of include/moeq.h in one native function each. A call of a few rows is a kernel or two
// of 3 us; marshalled in Python it took 8 to 10 us of the host's time, of which 3 are the launch. binding.py holds the public functions
// with their documentation; the library's entry points come from it as addresses, so that both use the same library.
#include <torch/csrc/Dtype.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <ATen/EmptyTensor.h>
#include <ATen/ops/empty.h>

#include <algorithm>
#include <initializer_list>

#include "moeq.h"

namespace {

struct Entry {
  decltype(&moe_sort_bytes) sort_bytes;
  decltype(&moe_sort_pairs) sort_pairs;
  decltype(&moe_gather_rows) gather_rows;
  decltype(&moe_combine_rows) combine_rows;
  decltype(&moe_combine_rows_backward) combine_rows_backward;
  decltype(&moe_adapters_workspace_bytes) adapters_workspace_bytes;
  decltype(&moe_adapters_forward) adapters_forward;
  decltype(&moe_adapters_backward) adapters_backward;
  decltype(&moe_distill_workspace_bytes) distill_workspace_bytes;
  decltype(&moe_distill_forward) distill_forward;
  decltype(&moe_distill_backward) distill_backward;
  decltype(&moe_distill_loss_grad) distill_loss_grad;
} lib;
PyObject* error_class = nullptr;      // binding.MoeqError(status, what)
PyObject* current_stream = nullptr;   // index of a device -> the handle of torch's current stream there; raises MoeqError if another is current

using at::Tensor;

// A refused call; ends in MoeqError.
struct Refused { int status; };
inline void need(bool ok) { if (!ok) throw Refused{MOEQ_EINVAL}; }
// The library's call, without the interpreter's lock (a launch waits where the queue is full).
template <typename F>
inline void run(F&& f) {
  struct Unlocked {
    PyThreadState* held = PyEval_SaveThread();
    ~Unlocked() { PyEval_RestoreThread(held); }
  };
  int status;
  {
    Unlocked u;
    status = f();
  }
  if (status != MOEQ_OK) throw Refused{status};
}

PyObject* refuse(const Refused& r, const char* what) {
  PyObject* e = PyObject_CallFunction(error_class, "is", r.status, what);
  if (e) {
    PyErr_SetObject(error_class, e);
    Py_DECREF(e);
  }
  return nullptr;
}

inline const Tensor& tensor(PyObject* o) {
  need(THPVariable_Check(o));
  return THPVariable_Unpack(o);
}
inline const Tensor* tensor_or_none(PyObject* o) { return o == Py_None ? nullptr : &tensor(o); }
inline int64_t whole(PyObject* o) {
  const long long v = PyLong_AsLongLong(o);
  if (v == -1 && PyErr_Occurred()) throw python_error();
  return v;
}
inline int32_t whole32(PyObject* o) {
  const int64_t v = whole(o);
  need(v >= INT32_MIN && v <= INT32_MAX);
  return (int32_t)v;
}
inline void* address(PyObject* o) { return (void*)whole(o); }
// The current stream of the device that a call's tensors are on: all of them (those that are there) on one, which has to be the current
// device, for the launches go to that.
inline void* stream_of(const Tensor& t, std::initializer_list<const Tensor*> others) {
  for (const Tensor* o : others) need(!o || !o->defined() || o->device() == t.device());
  PyObject* index = PyLong_FromLong(t.get_device());
  PyObject* s = index ? PyObject_CallFunctionObjArgs(current_stream, index, nullptr) : nullptr;
  Py_XDECREF(index);
  if (!s) throw python_error();
  const long long v = PyLong_AsLongLong(s);
  Py_DECREF(s);
  if (v == -1 && PyErr_Occurred()) throw python_error();
  return (void*)v;
}
inline void* data(const Tensor& t) { return t.data_ptr(); }
template <typename T>
inline T* data(const Tensor* t) { return t ? (T*)t->data_ptr() : nullptr; }

inline int32_t type_of(at::ScalarType t) {
  need(t == at::kFloat || t == at::kBFloat16 || t == at::kHalf);
  return t == at::kFloat ? MOEQ_F32 : t == at::kBFloat16 ? MOEQ_BF16 : MOEQ_F16;
}
inline int32_t size32(int64_t n) {
  need(n <= INT32_MAX);
  return (int32_t)n;
}
// The row stride of a [rows][cols] tensor with contiguous rows.
inline int64_t matrix(const Tensor& t, int64_t rows, int64_t cols) {
  need(t.is_cuda() && t.dim() == 2 && t.size(0) == rows && t.size(1) == cols && (cols == 1 || t.stride(1) == 1));
  return t.stride(0);
}
inline void plain(const Tensor& t, at::IntArrayRef shape, at::ScalarType type) {
  need(t.is_cuda() && t.scalar_type() == type && t.sizes() == shape && t.is_contiguous());
}
inline Tensor empty(at::IntArrayRef shape, at::ScalarType type, const Tensor& like) {
  return at::empty(shape, at::TensorOptions().dtype(type).device(like.device()));
}
inline PyObject* give(Tensor t) { return THPVariable_Wrap(std::move(t)); }
template <typename... P>
PyObject* give_tuple(P... objects) {
  constexpr int n = sizeof...(P);
  PyObject* list[] = {objects...};
  PyObject* t = nullptr;
  bool ok = true;
  for (PyObject* o : list) ok = ok && o;
  if (ok && (t = PyTuple_New(n)))
    for (int i = 0; i < n; ++i) PyTuple_SET_ITEM(t, i, list[i]);
  else
    for (PyObject* o : list) Py_XDECREF(o);
  return t;
}
// The same tensor again where the caller passed it.
inline PyObject* again(PyObject* o) {
  Py_INCREF(o);
  return o;
}

#define CALL(name, count)                                                        \
  PyObject* name##_body(PyObject* const* a);                                     \
  PyObject* name(PyObject*, PyObject* const* a, Py_ssize_t n) {                  \
    HANDLE_TH_ERRORS                                                             \
    try {                                                                        \
      need(n == count);                                                          \
      return name##_body(a);                                                     \
    } catch (const Refused& r) {                                                 \
      return refuse(r, "moe_" #name);                                            \
    }                                                                            \
    END_HANDLE_TH_ERRORS                                                         \
  }                                                                              \
  PyObject* name##_body(PyObject* const* a)

// idx, n_experts -> offsets, order, slot, n_tokens, top_k, n_experts
CALL(sort_pairs, 2) {
  const Tensor& idx = tensor(a[0]);
  const int64_t E = whole32(a[1]);
  need(idx.dim() == 2 && E > 0);
  const int64_t T = idx.size(0), k = idx.size(1), P = T * k;
  plain(idx, {T, k}, at::kInt);
  const size_t ws = lib.sort_bytes(size32(T), size32(k), (int32_t)E);
  const Tensor buf = empty({E + 1 + 2 * P + (int64_t)ws / 4}, at::kInt, idx);
  int32_t* at = (int32_t*)data(buf);
  void* stream = stream_of(idx, {});
  run([&] { return lib.sort_pairs((const int32_t*)data(idx), (int32_t)T, (int32_t)k, (int32_t)E, at, at + E + 1, at + E + 1 + P, at + E + 1 + 2 * P, ws, stream); });
  return give_tuple(give(buf.narrow(0, 0, E + 1)), give(buf.narrow(0, E + 1, P)), give(buf.narrow(0, E + 1 + P, P)), PyLong_FromLongLong(T), PyLong_FromLongLong(k), again(a[1]));
}

// slot, n_tokens, top_k, x, rows or None -> rows
CALL(gather_rows, 5) {
  const Tensor &slot = tensor(a[0]), &x = tensor(a[3]);
  const int64_t T = whole32(a[1]), k = whole32(a[2]);
  need(x.dim() == 2);
  const int64_t d = x.size(1), xs = matrix(x, T, d);
  plain(slot, {T * k}, at::kInt);
  const Tensor rows = a[4] == Py_None ? empty({T * k, d}, x.scalar_type(), x) : tensor(a[4]);
  need(rows.scalar_type() == x.scalar_type());
  void* stream = stream_of(slot, {&x, &rows});
  run([&] { return lib.gather_rows((const int32_t*)data(slot), (int32_t)T, (int32_t)k, size32(d), type_of(x.scalar_type()), data(x), xs, data(rows), matrix(rows, T * k, d), stream); });
  return a[4] == Py_None ? give(rows) : again(a[4]);
}

// slot, n_tokens, top_k, rows, gate or None, dtype or None, y or None -> y
CALL(combine_rows, 7) {
  const Tensor &slot = tensor(a[0]), &rows = tensor(a[3]), *gate = tensor_or_none(a[4]);
  const int64_t T = whole32(a[1]), k = whole32(a[2]);
  need(rows.dim() == 2 && (a[5] == Py_None || THPDtype_Check(a[5])));
  const int64_t d = rows.size(1), rs = matrix(rows, T * k, d);
  plain(slot, {T * k}, at::kInt);
  if (gate) plain(*gate, {T, k}, at::kFloat);
  const at::ScalarType type = a[5] != Py_None ? ((THPDtype*)a[5])->scalar_type : a[6] != Py_None ? tensor(a[6]).scalar_type() : rows.scalar_type();
  const Tensor y = a[6] == Py_None ? empty({T, d}, type, rows) : tensor(a[6]);
  need(y.scalar_type() == type);
  void* stream = stream_of(slot, {&rows, gate, &y});
  run([&] { return lib.combine_rows((const int32_t*)data(slot), data<const float>(gate), (int32_t)T, (int32_t)k, size32(d), type_of(rows.scalar_type()), data(rows), rs, type_of(type),
                        data(y), matrix(y, T, d), stream); });
  return a[6] == Py_None ? give(y) : again(a[6]);
}

// slot, n_tokens, top_k, dy, rows, gate or None, drows or None -> drows, dgate
CALL(combine_rows_backward, 7) {
  const Tensor &slot = tensor(a[0]), &dy = tensor(a[3]), &rows = tensor(a[4]), *gate = tensor_or_none(a[5]);
  const int64_t T = whole32(a[1]), k = whole32(a[2]);
  need(rows.dim() == 2);
  const int64_t d = rows.size(1), rs = matrix(rows, T * k, d), ys = matrix(dy, T, d);
  plain(slot, {T * k}, at::kInt);
  if (gate) plain(*gate, {T, k}, at::kFloat);
  const Tensor drows = a[6] == Py_None ? empty({T * k, d}, rows.scalar_type(), rows) : tensor(a[6]), dgate = empty({T, k}, at::kFloat, rows);
  need(drows.scalar_type() == rows.scalar_type());
  void* stream = stream_of(slot, {&dy, &rows, gate, &drows});
  run([&] { return lib.combine_rows_backward((const int32_t*)data(slot), data<const float>(gate), (int32_t)T, (int32_t)k, size32(d), type_of(rows.scalar_type()), data(rows), rs,
                                 type_of(dy.scalar_type()), data(dy), ys, data(drows), matrix(drows, T * k, d), (float*)data(dgate), stream); });
  return give_tuple(a[6] == Py_None ? give(drows) : again(a[6]), give(dgate));
}

// The workspace that is passed, or one for this call alone: from the allocator, on the stream that the call runs on, so that calls on
// other streams, of other threads (the interpreter's lock is not held around a call's launches) or in a graph have each their own.
// (Past the dispatcher, which at::empty goes through: 0.4 us less of a call of nine rows of the host's time.)
Tensor workspace(PyObject* o, const moeq_adapters* L, int64_t T, bool backward, const Tensor& like) {
  if (o == Py_None) {
    static at::Allocator* const memory = empty({1}, at::kByte, like).storage().allocator();      // (that of torch's own tensors)
    const int64_t bytes = std::max<int64_t>(lib.adapters_workspace_bytes(L, size32(T), backward), 16);
    return Tensor(at::detail::empty_generic({bytes}, memory, c10::DispatchKeySet(c10::DispatchKey::CUDA), at::kByte, c10::nullopt));
  }
  const Tensor& ws = tensor(o);
  need(ws.is_cuda() && ws.is_contiguous() && ws.scalar_type() == at::kByte);
  return ws;
}

// handle, x, ids, base or None, y or None, ws or None, the adapters' weights -> y, ws
CALL(adapters_forward, 7) {
  const moeq_adapters* L = (const moeq_adapters*)address(a[0]);
  const Tensor &x = tensor(a[1]), &ids = tensor(a[2]), *base = tensor_or_none(a[3]), &weights = tensor(a[6]);
  need(x.dim() == 2 && type_of(x.scalar_type()) == L->dtype);
  const int64_t T = x.size(0), xs = matrix(x, T, L->d_in);
  plain(ids, {T}, at::kInt);
  const Tensor ws = workspace(a[5], L, T, false, x);
  const Tensor y = a[4] != Py_None ? tensor(a[4]) : empty({T, L->d_out}, base ? base->scalar_type() : x.scalar_type(), x);
  need(!base || base->scalar_type() == y.scalar_type());
  void* stream = stream_of(x, {&weights, &ids, base, &ws, &y});
  run([&] { return lib.adapters_forward(L, data(x), xs, (const int32_t*)data(ids), size32(T), data<const void>(base), base ? matrix(*base, T, L->d_out) : 0, type_of(y.scalar_type()), data(y),
                            matrix(y, T, L->d_out), data(ws), ws.numel(), stream); });
  return give_tuple(a[4] == Py_None ? give(y) : again(a[4]), give(ws));
}

// handle, x, ids, dy, dx_base or None, dx or None, whether dx is wanted, ws or None, the adapters' weights -> dx or None, dA, dB, ws
CALL(adapters_backward, 9) {
  const moeq_adapters* L = (const moeq_adapters*)address(a[0]);
  const Tensor &x = tensor(a[1]), &ids = tensor(a[2]), &dy = tensor(a[3]), *base = tensor_or_none(a[4]), &weights = tensor(a[8]);
  need(x.dim() == 2 && type_of(x.scalar_type()) == L->dtype);
  const int64_t T = x.size(0), xs = matrix(x, T, L->d_in), ys = matrix(dy, T, L->d_out);
  plain(ids, {T}, at::kInt);
  const Tensor ws = workspace(a[7], L, T, true, x);
  const bool mine = a[5] == Py_None && a[6] == Py_True;
  const Tensor dx = a[5] != Py_None ? tensor(a[5]) : mine ? empty({T, L->d_in}, dy.scalar_type(), x) : Tensor();
  need(!dx.defined() || dx.scalar_type() == dy.scalar_type());
  need(!base || base->scalar_type() == dy.scalar_type());
  const Tensor dA = empty({L->n_adapters, L->rank, L->d_in}, at::kFloat, x), dB = empty({L->n_adapters, L->d_out, L->rank}, at::kFloat, x);
  void* stream = stream_of(x, {&weights, &ids, &dy, base, &ws, &dx});
  run([&] { return lib.adapters_backward(L, data(x), xs, (const int32_t*)data(ids), size32(T), type_of(dy.scalar_type()), data(dy), ys, data<const void>(base), base ? matrix(*base, T, L->d_in) : 0,
                             dx.defined() ? data(dx) : nullptr, dx.defined() ? matrix(dx, T, L->d_in) : 0, (float*)data(dA), (float*)data(dB), data(ws), ws.numel(), stream); });
  return give_tuple(mine ? give(dx) : again(a[5]), give(dA), give(dB), give(ws));
}

struct Teacher { int64_t T, V, K, stride; int32_t type; const Tensor *logits, *idx, *top, *weight; float temperature; };
Teacher teacher(PyObject* const* a) {      // logits, top_idx, top_logits, temperature, weight or None
  Teacher t{};
  t.logits = &tensor(a[0]), t.idx = &tensor(a[1]), t.top = &tensor(a[2]), t.weight = tensor_or_none(a[4]);
  need(t.logits->dim() == 2 && t.idx->dim() == 2);
  t.T = t.logits->size(0), t.V = t.logits->size(1), t.K = t.idx->size(1), t.stride = matrix(*t.logits, t.T, t.V), t.type = type_of(t.logits->scalar_type());
  size32(t.T), size32(t.V), size32(t.K);
  plain(*t.idx, {t.T, t.K}, at::kInt);
  plain(*t.top, {t.T, t.K}, at::kFloat);
  if (t.weight) plain(*t.weight, {t.T}, at::kFloat);
  const double tau = PyFloat_AsDouble(a[3]);
  if (tau == -1.0 && PyErr_Occurred()) throw python_error();
  t.temperature = (float)tau;
  return t;
}

// logits, top_idx, top_logits, temperature, weight or None -> loss, lse
CALL(distill_forward, 5) {
  const Teacher t = teacher(a);
  const size_t ws = lib.distill_workspace_bytes(t.T, t.V, t.type);
  const Tensor buf = empty({2 * t.T + (int64_t)(ws + 3) / 4 + 1}, at::kFloat, *t.logits);      // (loss, lse, and the workspace at the next 8 bytes)
  float *at = (float*)data(buf), *scratch = at + (2 * t.T + 1) / 2 * 2;
  void* stream = stream_of(*t.logits, {t.idx, t.top, t.weight});
  run([&] { return lib.distill_forward(data(*t.logits), t.stride, t.type, t.T, t.V, (const int32_t*)data(*t.idx), (const float*)data(*t.top), t.K, t.temperature, data<const float>(t.weight), at,
                           at + t.T, scratch, ws, stream); });
  return give_tuple(give(buf.narrow(0, 0, t.T)), give(buf.narrow(0, t.T, t.T)));
}

// logits, top_idx, top_logits, temperature, weight or None, lse, dloss, dlogits or None -> dlogits
CALL(distill_backward, 8) {
  const Teacher t = teacher(a);
  const Tensor &lse = tensor(a[5]), &dloss = tensor(a[6]);
  plain(lse, {t.T}, at::kFloat);
  plain(dloss, {t.T}, at::kFloat);
  const Tensor dz = a[7] == Py_None ? empty({t.T, t.V}, t.logits->scalar_type(), *t.logits) : tensor(a[7]);
  need(dz.scalar_type() == t.logits->scalar_type());
  void* stream = stream_of(*t.logits, {t.idx, t.top, t.weight, &lse, &dloss, &dz});
  run([&] { return lib.distill_backward(data(*t.logits), t.stride, t.type, t.T, t.V, (const int32_t*)data(*t.idx), (const float*)data(*t.top), t.K, t.temperature, data<const float>(t.weight),
                            (const float*)data(lse), (const float*)data(dloss), data(dz), matrix(dz, t.T, t.V), stream); });
  return a[7] == Py_None ? give(dz) : again(a[7]);
}

// logits, top_idx, top_logits, temperature, weight or None, dlogits or None -> loss, dlogits
CALL(distill_loss_grad, 6) {
  const Teacher t = teacher(a);
  const size_t ws = lib.distill_workspace_bytes(t.T, t.V, t.type);
  const Tensor buf = empty({t.T + (int64_t)(ws + 3) / 4 + 1}, at::kFloat, *t.logits);
  const Tensor dz = a[5] == Py_None ? empty({t.T, t.V}, t.logits->scalar_type(), *t.logits) : tensor(a[5]);
  need(dz.scalar_type() == t.logits->scalar_type());
  float *at = (float*)data(buf), *scratch = at + (t.T + 1) / 2 * 2;
  void* stream = stream_of(*t.logits, {t.idx, t.top, t.weight, &dz});
  run([&] { return lib.distill_loss_grad(data(*t.logits), t.stride, t.type, t.T, t.V, (const int32_t*)data(*t.idx), (const float*)data(*t.top), t.K, t.temperature, data<const float>(t.weight), at,
                             data(dz), matrix(dz, t.T, t.V), scratch, ws, stream); });
  return give_tuple(give(buf.narrow(0, 0, t.T)), a[5] == Py_None ? give(dz) : again(a[5]));
}

// MoeqError, the function that gives the current stream of a device, then the addresses of the library's entry points in the order of Entry.
PyObject* bind(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  constexpr int kEntries = sizeof(Entry) / sizeof(void*);
  if (n != 2 + kEntries) return PyErr_Format(PyExc_TypeError, "bind: %d entry points wanted", kEntries);
  void* at[kEntries];
  for (int i = 0; i < kEntries; ++i) at[i] = address(a[2 + i]);
  memcpy(&lib, at, sizeof(lib));
  Py_INCREF(a[0]);
  Py_INCREF(a[1]);
  Py_XDECREF(error_class);
  Py_XDECREF(current_stream);
  error_class = a[0];
  current_stream = a[1];
  Py_RETURN_NONE;
  END_HANDLE_TH_ERRORS
}

#define METHOD(name) {#name, (PyCFunction)(void (*)(void))name, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {METHOD(bind), METHOD(sort_pairs), METHOD(gather_rows), METHOD(combine_rows), METHOD(combine_rows_backward), METHOD(adapters_forward), METHOD(adapters_backward),
                         METHOD(distill_forward), METHOD(distill_backward), METHOD(distill_loss_grad), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_calls", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__calls(void) { return PyModule_Create(&module); }
