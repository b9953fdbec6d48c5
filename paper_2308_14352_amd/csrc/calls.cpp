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
#include <vector>

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
  decltype(&moe_block_norms_forward) block_norms_forward;
  decltype(&moe_block_norms_workspace_bytes) block_norms_workspace_bytes;
  decltype(&moe_block_norms_backward) block_norms_backward;
  decltype(&moe_pack8) pack8;
  decltype(&moe_unpack8) unpack8;
  decltype(&moe_gated_ffn_workspace_bytes) gated_ffn_workspace_bytes;
  decltype(&moe_gated_ffn_forward) gated_ffn_forward;
  decltype(&moe_gated_ffn_backward) gated_ffn_backward;
  decltype(&moe_q8_pitch) q8_pitch;
  decltype(&moe_quantize_rows) quantize_rows;
  decltype(&moe_matmul_q8_workspace_bytes) matmul_q8_workspace_bytes;
  decltype(&moe_matmul_q8) matmul_q8;
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

inline float real(PyObject* o) {
  const double v = PyFloat_AsDouble(o);
  if (v == -1.0 && PyErr_Occurred()) throw python_error();
  return (float)v;
}
inline at::ScalarType type_or(PyObject* o, at::ScalarType otherwise) {
  need(o == Py_None || THPDtype_Check(o));
  return o == Py_None ? otherwise : ((THPDtype*)o)->scalar_type;
}
inline const float* vector(const Tensor* t, int64_t n) {      // fp32 [n], or none
  if (t) plain(*t, {n}, at::kFloat);
  return data<const float>(t);
}
// What a call writes for itself between its kernels, from the allocator on the stream of the call; the smallest for calls that need none.
inline Tensor scratch(size_t bytes, const Tensor& like) { return empty({(int64_t)std::max<size_t>(bytes, 16)}, at::kByte, like); }

// f, r, gate, w_after, w_before (each or None), residual_scale, eps, dtype of n or None, y or None, n or None -> y, n or None
CALL(block_norms_forward, 10) {
  const Tensor &f = tensor(a[0]), &r = tensor(a[1]), *gate = tensor_or_none(a[2]), *after = tensor_or_none(a[3]), *before = tensor_or_none(a[4]);
  need(f.dim() == 2 && (before || a[9] == Py_None));
  const int64_t T = f.size(0), d = f.size(1), fs = matrix(f, T, d), rs = matrix(r, T, d);
  const at::ScalarType type = type_or(a[7], a[9] != Py_None ? tensor(a[9]).scalar_type() : r.scalar_type());
  const Tensor y = a[8] == Py_None ? empty({T, d}, r.scalar_type(), f) : tensor(a[8]);
  const Tensor n = a[9] != Py_None ? tensor(a[9]) : before ? empty({T, d}, type, f) : Tensor();
  need(y.scalar_type() == r.scalar_type() && (!n.defined() || n.scalar_type() == type));
  const float scale = real(a[5]), eps = real(a[6]), *g = vector(gate, T), *wa = vector(after, d), *wb = vector(before, d);
  void* stream = stream_of(f, {&r, gate, after, before, &y, &n});
  run([&] {
    return lib.block_norms_forward(size32(T), size32(d), scale, eps, type_of(f.scalar_type()), data(f), fs, type_of(r.scalar_type()), data(r), rs, g, wa, wb, data(y), matrix(y, T, d), type_of(type), n.defined() ? data(n) : nullptr, n.defined() ? matrix(n, T, d) : 0, stream);
  });
  return give_tuple(a[8] == Py_None ? give(y) : again(a[8]), a[9] == Py_None && before ? give(n) : again(a[9]));
}

// f, y or None, dy, dn or None, gate, w_after, w_before (each or None), residual_scale, eps, df or None, dr or None -> df, dr, dgate, dw_after, dw_before (each of the last or None)
CALL(block_norms_backward, 11) {
  const Tensor &f = tensor(a[0]), *y = tensor_or_none(a[1]), &dy = tensor(a[2]), *dn = tensor_or_none(a[3]);
  const Tensor *gate = tensor_or_none(a[4]), *after = tensor_or_none(a[5]), *before = tensor_or_none(a[6]);
  need(f.dim() == 2 && (!before || (y && dn && y->scalar_type() == dy.scalar_type())));
  const int64_t T = f.size(0), d = f.size(1), fs = matrix(f, T, d), ds = matrix(dy, T, d);
  if (!before) y = dn = nullptr;      // (not read)
  const Tensor df = a[9] == Py_None ? empty({T, d}, f.scalar_type(), f) : tensor(a[9]), dr = a[10] == Py_None ? empty({T, d}, dy.scalar_type(), f) : tensor(a[10]);
  need(df.scalar_type() == f.scalar_type() && dr.scalar_type() == dy.scalar_type());
  const Tensor dgate = gate ? empty({T}, at::kFloat, f) : Tensor(), da = after ? empty({d}, at::kFloat, f) : Tensor(), db = before ? empty({d}, at::kFloat, f) : Tensor();
  const size_t bytes = after || before ? lib.block_norms_workspace_bytes(size32(T), size32(d)) : 0;
  const Tensor ws = scratch(bytes, f);
  const int64_t ys = y ? matrix(*y, T, d) : 0, ns = dn ? matrix(*dn, T, d) : 0;
  const float scale = real(a[7]), eps = real(a[8]), *g = vector(gate, T), *wa = vector(after, d), *wb = vector(before, d);
  const auto at = [](const Tensor& t) { return t.defined() ? (float*)t.data_ptr() : nullptr; };
  void* stream = stream_of(f, {y, &dy, dn, gate, after, before, &df, &dr});
  run([&] {
    return lib.block_norms_backward(size32(T), size32(d), scale, eps, type_of(f.scalar_type()), data(f), fs, type_of(dy.scalar_type()), data<const void>(y), ys, data(dy), ds,
                                    dn ? type_of(dn->scalar_type()) : type_of(dy.scalar_type()), data<const void>(dn), ns, g, wa, wb, data(df), matrix(df, T, d), data(dr), matrix(dr, T, d),
                                    at(dgate), at(da), at(db), data(ws), ws.numel(), stream);
  });
  const auto some = [](const Tensor& t) { return t.defined() ? give(t) : again(Py_None); };
  return give_tuple(a[9] == Py_None ? give(df) : again(a[9]), a[10] == Py_None ? give(dr) : again(a[10]), some(dgate), some(da), some(db));
}

inline int64_t pack_blocks(int64_t d) { return (d + 31) / 32; }

// x, codes or None, exps or None -> codes, exps
CALL(pack8, 3) {
  const Tensor& x = tensor(a[0]);
  need(x.dim() == 2 && (a[1] == Py_None) == (a[2] == Py_None));
  const int64_t T = x.size(0), d = x.size(1), xs = matrix(x, T, d);
  const Tensor codes = a[1] == Py_None ? empty({T, d}, at::kChar, x) : tensor(a[1]), exps = a[2] == Py_None ? empty({T, pack_blocks(d)}, at::kChar, x) : tensor(a[2]);
  plain(codes, {T, d}, at::kChar);
  plain(exps, {T, pack_blocks(d)}, at::kChar);
  void* stream = stream_of(x, {&codes, &exps});
  run([&] { return lib.pack8(data(x), xs, type_of(x.scalar_type()), size32(T), size32(d), (int8_t*)data(codes), (int8_t*)data(exps), stream); });
  return give_tuple(a[1] == Py_None ? give(codes) : again(a[1]), a[2] == Py_None ? give(exps) : again(a[2]));
}

// codes [..., d], exps [..., blocks], dtype, x or None -> x
CALL(unpack8, 4) {
  const Tensor &codes = tensor(a[0]), &exps = tensor(a[1]);
  need(codes.dim() >= 1 && THPDtype_Check(a[2]));
  const int64_t d = codes.size(-1), T = d > 0 ? codes.numel() / d : 0;
  plain(codes, codes.sizes(), at::kChar);
  std::vector<int64_t> shape = codes.sizes().vec();
  shape.back() = pack_blocks(d);
  plain(exps, shape, at::kChar);
  const at::ScalarType type = ((THPDtype*)a[2])->scalar_type;
  const Tensor x = a[3] == Py_None ? empty(codes.sizes(), type, codes) : tensor(a[3]);
  need(x.scalar_type() == type && (a[3] == Py_None || x.dim() == 2));
  const int64_t xs = a[3] == Py_None ? d : matrix(x, T, d);
  void* stream = stream_of(codes, {&exps, &x});
  run([&] { return lib.unpack8((const int8_t*)data(codes), (const int8_t*)data(exps), size32(T), size32(d), type_of(type), data(x), xs, stream); });
  return a[3] == Py_None ? give(x) : again(a[3]);
}

// handle, x, base or None, dtype of y or None, y or None, keep, ws or None, a weight -> y, what is kept of a and b or None, its exponents or None
CALL(gated_ffn_forward, 8) {
  const moeq_gated_ffn* L = (const moeq_gated_ffn*)address(a[0]);
  const Tensor &x = tensor(a[1]), *base = tensor_or_none(a[2]), &weight = tensor(a[7]);
  const int32_t keep = whole32(a[5]);
  need(x.dim() == 2 && type_of(x.scalar_type()) == L->dtype);
  const int64_t T = x.size(0), xs = matrix(x, T, L->d_model), F = L->d_ff;
  const at::ScalarType type = type_or(a[3], a[4] != Py_None ? tensor(a[4]).scalar_type() : base ? base->scalar_type() : x.scalar_type());
  const Tensor y = a[4] != Py_None ? tensor(a[4]) : empty({T, L->d_model}, type, x);
  need(y.scalar_type() == type && (!base || base->scalar_type() == type));
  const Tensor ab = keep == MOEQ_KEEP_NONE ? Tensor() : empty({2, T, F}, keep == MOEQ_KEEP_8 ? at::kChar : x.scalar_type(), x);
  const Tensor exps = keep == MOEQ_KEEP_8 ? empty({2, T, pack_blocks(F)}, at::kChar, x) : Tensor();
  const Tensor ws = a[6] != Py_None ? tensor(a[6]) : scratch(lib.gated_ffn_workspace_bytes(L, size32(T), 0, 0, keep), x);
  need(ws.is_contiguous() && ws.scalar_type() == at::kByte);
  const int64_t bs = base ? matrix(*base, T, L->d_model) : 0, ys = matrix(y, T, L->d_model);
  void* stream = stream_of(x, {base, &y, &ws, &weight});
  run([&] {
    return lib.gated_ffn_forward(L, data(x), xs, size32(T), data<const void>(base), bs, type_of(type), data(y), ys, keep, ab.defined() ? data(ab) : nullptr,
                                 exps.defined() ? (int8_t*)data(exps) : nullptr, data(ws), ws.numel(), stream);
  });
  const auto some = [](const Tensor& t) { return t.defined() ? give(t) : again(Py_None); };
  return give_tuple(a[4] == Py_None ? give(y) : again(a[4]), some(ab), some(exps));
}

// handle, x or its codes, None or its exponents, dy, keep, ab or codes or None, exponents or None, dx or None, whether dx is wanted, ws or None, a weight
// -> dx or None, dw_in, dw_gate, dw_out
CALL(gated_ffn_backward, 11) {
  const moeq_gated_ffn* L = (const moeq_gated_ffn*)address(a[0]);
  const Tensor &x = tensor(a[1]), *xe = tensor_or_none(a[2]), &dy = tensor(a[3]), *ab = tensor_or_none(a[5]), *abe = tensor_or_none(a[6]), &weight = tensor(a[10]);
  const int32_t keep = whole32(a[4]);
  need(dy.dim() == 2 && type_of(dy.scalar_type()) == L->dtype);
  const int64_t T = dy.size(0), D = L->d_model, F = L->d_ff, ds = matrix(dy, T, D);
  int64_t xs = 0;
  if (xe) {
    plain(x, {T, D}, at::kChar);
    plain(*xe, {T, pack_blocks(D)}, at::kChar);
  } else {
    need(x.scalar_type() == dy.scalar_type());
    xs = matrix(x, T, D);
  }
  need((ab != nullptr) == (keep != MOEQ_KEEP_NONE) && (abe != nullptr) == (keep == MOEQ_KEEP_8));
  if (ab) plain(*ab, {2, T, F}, keep == MOEQ_KEEP_8 ? at::kChar : dy.scalar_type());
  if (abe) plain(*abe, {2, T, pack_blocks(F)}, at::kChar);
  const bool mine = a[7] == Py_None && a[8] == Py_True;
  const Tensor dx = a[7] != Py_None ? tensor(a[7]) : mine ? empty({T, D}, dy.scalar_type(), dy) : Tensor();
  need(!dx.defined() || dx.scalar_type() == dy.scalar_type());
  const Tensor d_in = empty({F, D}, dy.scalar_type(), dy), d_gate = empty({F, D}, dy.scalar_type(), dy), d_out = empty({D, F}, dy.scalar_type(), dy);
  const Tensor ws = a[9] != Py_None ? tensor(a[9]) : scratch(lib.gated_ffn_workspace_bytes(L, size32(T), 1, xe != nullptr, keep), dy);
  need(ws.is_contiguous() && ws.scalar_type() == at::kByte);
  const int64_t dxs = dx.defined() ? matrix(dx, T, D) : 0;
  void* stream = stream_of(dy, {&x, xe, ab, abe, &dx, &ws, &weight});
  run([&] {
    return lib.gated_ffn_backward(L, xe ? nullptr : data(x), xs, xe ? (const int8_t*)data(x) : nullptr, data<const int8_t>(xe), size32(T), data(dy), ds, keep, data<const void>(ab),
                                  data<const int8_t>(abe), dx.defined() ? data(dx) : nullptr, dxs, data(d_in), data(d_gate), data(d_out), data(ws), ws.numel(), stream);
  });
  return give_tuple(mine ? give(dx) : again(a[7]), give(d_in), give(d_gate), give(d_out));
}

// x -> codes [T][pitch], scale
CALL(quantize_rows, 1) {
  const Tensor& x = tensor(a[0]);
  need(x.dim() == 2 && x.size(1) > 0);
  const int64_t T = x.size(0), d = x.size(1), xs = matrix(x, T, d);
  const Tensor codes = empty({T, lib.q8_pitch(size32(d))}, at::kChar, x), scale = empty({T}, at::kFloat, x);
  void* stream = stream_of(x, {});
  run([&] { return lib.quantize_rows(data(x), xs, type_of(x.scalar_type()), size32(T), (int32_t)d, (int8_t*)data(codes), (float*)data(scale), stream); });
  return give_tuple(give(codes), give(scale));
}

// k, codes and scale of x, codes and scale of w, base or None, dtype or None, y or None -> y
CALL(matmul_q8, 8) {
  const int32_t k = whole32(a[0]);
  const Tensor &x = tensor(a[1]), &xs = tensor(a[2]), &w = tensor(a[3]), &ws = tensor(a[4]), *base = tensor_or_none(a[5]);
  need(k > 0 && x.dim() == 2 && w.dim() == 2);
  const int64_t T = x.size(0), N = w.size(0), pitch = lib.q8_pitch(k);
  plain(x, {T, pitch}, at::kChar);
  plain(w, {N, pitch}, at::kChar);
  plain(xs, {T}, at::kFloat);
  plain(ws, {N}, at::kFloat);
  const at::ScalarType type = type_or(a[6], a[7] != Py_None ? tensor(a[7]).scalar_type() : base ? base->scalar_type() : at::kFloat);
  const Tensor y = a[7] != Py_None ? tensor(a[7]) : empty({T, N}, type, x);
  need(y.scalar_type() == type && (!base || base->scalar_type() == type));
  const Tensor room = scratch(lib.matmul_q8_workspace_bytes(size32(T), size32(N), k), x);
  const int64_t bs = base ? matrix(*base, T, N) : 0, ys = matrix(y, T, N);
  void* stream = stream_of(x, {&xs, &w, &ws, base, &y});
  run([&] {
    return lib.matmul_q8((const int8_t*)data(x), (const float*)data(xs), (int32_t)T, (const int8_t*)data(w), (const float*)data(ws), (int32_t)N, k, data<const void>(base), bs, type_of(type),
                         data(y), ys, data(room), room.numel(), stream);
  });
  return a[7] == Py_None ? give(y) : again(a[7]);
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
                         METHOD(distill_forward), METHOD(distill_backward), METHOD(distill_loss_grad), METHOD(block_norms_forward), METHOD(block_norms_backward), METHOD(pack8), METHOD(unpack8), METHOD(gated_ffn_forward),
                         METHOD(gated_ffn_backward), METHOD(quantize_rows), METHOD(matmul_q8), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_calls", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__calls(void) { return PyModule_Create(&module); }
