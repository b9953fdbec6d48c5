// Host side of the operators beside the layer: argument checks (all before the first HIP call) and launches.
#include "operators.h"

#include <initializer_list>

using namespace moeq;

namespace {

inline moeq_status done(hipError_t e) { return e == hipSuccess ? MOEQ_OK : MOEQ_EDEVICE; }
inline bool type_ok(int32_t t) { return t == MOEQ_F32 || t == MOEQ_BF16 || t == MOEQ_F16; }
inline bool aligned(const void* p, size_t a) { return ((uintptr_t)p & (a - 1)) == 0; }
// A strided matrix in memory, for the checks of outputs against inputs.
struct Block { const void* p; int64_t rows, stride, width; int32_t dtype; };
// Whether two may share a byte. Slices of the columns of one buffer (the same stride in bytes, or a single row) are compared within a row.
bool overlap(const Block& a, const Block& b) {
  if (!a.p || !b.p || a.rows == 0 || b.rows == 0) return false;
  const int64_t ea = dtype_bytes(a.dtype), eb = dtype_bytes(b.dtype);
  const uintptr_t x = (uintptr_t)a.p, y = (uintptr_t)b.p;
  if (!(x < y + (uintptr_t)(((b.rows - 1) * b.stride + b.width) * eb) && y < x + (uintptr_t)(((a.rows - 1) * a.stride + a.width) * ea)))
    return false;
  // (the stride of a single row says nothing)
  const int64_t pitch = a.rows > 1 ? a.stride * ea : b.rows > 1 ? b.stride * eb : 0;
  if (pitch > 0 && (b.rows == 1 || pitch == b.stride * eb)) {
    const int64_t at = ((int64_t)(y - x) % pitch + pitch) % pitch;      // where b's rows begin in a's
    return at < a.width * ea || at + b.width * eb > pitch;
  }
  return true;
}
// n contiguous elements of 4 bytes.
inline Block vec(const void* p, int64_t n) { return Block{p, n > 0, n, n, MOEQ_F32}; }
// Whether the outputs share no byte with the inputs or with each other (those that are null, or of no rows, with none).
bool apart(std::initializer_list<Block> out, std::initializer_list<Block> in) {
  for (const Block* o = out.begin(); o != out.end(); ++o) {
    for (const Block& i : in)
      if (overlap(i, *o)) return false;
    for (const Block* p = o + 1; p != out.end(); ++p)
      if (overlap(*p, *o)) return false;
  }
  return true;
}
// Whether an input may be used beside an output that it may also be itself.
inline bool apart_or_same(const Block& in, const Block& out) {
  return !overlap(in, out) || (in.p == out.p && (in.rows == 1 || in.stride == out.stride) && in.dtype == out.dtype);
}
// A matrix of n rows: there, aligned to its elements, its rows either apart or (inputs only) all the same one; a single row has any stride.
inline bool matrix_ok(const void* p, int64_t rows, int64_t stride, int64_t width, int32_t dtype, bool input) {
  if (rows == 0) return true;
  return p && aligned(p, dtype_bytes(dtype)) &&
         (rows == 1 || ((stride >= width || (input && stride == 0)) && stride <= (int64_t)1 << 32));
}
constexpr int64_t kMaxPairs = (int64_t)1 << 28;

moeq_status rows_ok(const int32_t* slot, int32_t n_tokens, int32_t top_k, int32_t d) {
  if (n_tokens < 0 || top_k <= 0 || d <= 0 || (n_tokens && (!slot || !aligned(slot, 4)))) return MOEQ_EINVAL;
  if ((int64_t)n_tokens * top_k > kMaxPairs) return MOEQ_EUNSUPPORTED;
  return MOEQ_OK;
}

moeq_status adapters_ok(const moeq_adapters* a, int32_t n_tokens, int32_t out_dtype) {
  if (!a || a->n_adapters <= 0 || a->rank <= 0 || a->d_in <= 0 || a->d_out <= 0 || n_tokens < 0) return MOEQ_EINVAL;
  if (!type_ok(a->dtype) || (out_dtype != a->dtype && out_dtype != MOEQ_F32)) return MOEQ_EINVAL;
  if (a->rank > kAdapterMaxRank || a->n_adapters > kSortMaxExperts || a->d_in > 32768 || a->d_out > 32768 || n_tokens > 65535)
    return MOEQ_EUNSUPPORTED;
  const size_t e = dtype_bytes(a->dtype);
  if (!a->a || !a->b || !a->scale || !aligned(a->a, e) || !aligned(a->b, e) || !aligned(a->scale, 4)) return MOEQ_EINVAL;
  return MOEQ_OK;
}

inline Block a_of(const moeq_adapters& L) { return Block{L.a, (int64_t)L.n_adapters * L.rank, L.d_in, L.d_in, L.dtype}; }
inline Block b_of(const moeq_adapters& L) { return Block{L.b, (int64_t)L.n_adapters * L.d_out, L.rank, L.rank, L.dtype}; }

AdapterArgs adapter_args(const moeq_adapters* a, int32_t n_tokens, int32_t out_dtype) {
  AdapterArgs p = {};
  p.n = a->n_adapters, p.rank = a->rank, p.d_in = a->d_in, p.d_out = a->d_out, p.dtype = a->dtype, p.out_dtype = out_dtype;
  p.T = n_tokens, p.A = a->a, p.B = a->b, p.scale = a->scale;
  return p;
}

moeq_status distill_ok(const DistillArgs& a, const void* ws, size_t ws_bytes, bool grad, bool stats) {
  if (a.T < 0 || a.V <= 0 || a.K <= 0 || !type_ok(a.dtype) || !(a.temperature > 0.f) || a.temperature > 1e30f || a.temperature < 1e-30f)
    return MOEQ_EINVAL;
  if (a.K > kDistillMaxTop || a.T > (1 << 24)) return MOEQ_EUNSUPPORTED;
  if (a.T == 0) return MOEQ_OK;
  if (!matrix_ok(a.logits, a.T, a.stride, a.V, a.dtype, true)) return MOEQ_EINVAL;
  if (!a.top_idx || !a.top_logits || !aligned(a.top_idx, 4) || !aligned(a.top_logits, 4) || !aligned(a.weight, 4)) return MOEQ_EINVAL;
  if (grad && !matrix_ok(a.dlogits, a.T, a.dstride, a.V, a.dtype, false)) return MOEQ_EINVAL;
  const int64_t entries = (int64_t)a.T * a.K;
  if (!apart({{a.dlogits, a.T, a.dstride, a.V, a.dtype}, vec(a.loss, a.T), vec(a.lse, a.T)},
             {{a.logits, a.T, a.stride, a.V, a.dtype}, vec(a.top_idx, entries), vec(a.top_logits, entries), vec(a.weight, a.T),
              vec(a.lse_in, a.T), vec(a.dloss, a.T)}))
    return MOEQ_EINVAL;
  if (stats) {
    const size_t need = distill_ws_bytes(a.T, a.V, a.dtype);
    if (need && (!ws || ws_bytes < need)) return MOEQ_EWORKSPACE;
    if (need && !aligned(ws, 8)) return MOEQ_EINVAL;
  }
  return MOEQ_OK;
}

DistillArgs distill_args(const void* logits, int64_t stride, int32_t dtype, int32_t T, int32_t V, const int32_t* idx,
                         const float* top, int32_t K, float temperature, const float* weight) {
  DistillArgs a = {};
  a.logits = logits, a.stride = stride, a.dtype = dtype, a.T = T, a.V = V, a.K = K, a.top_idx = idx, a.top_logits = top;
  a.temperature = temperature, a.weight = weight;
  return a;
}

}  // namespace

extern "C" {

size_t moe_sort_bytes(int32_t n_tokens, int32_t top_k, int32_t n_experts) {
  if (n_tokens <= 0 || top_k <= 0 || n_experts <= 0 || n_experts > kSortMaxExperts || (int64_t)n_tokens * top_k > kMaxPairs) return 0;
  return sort_ws_bytes((int64_t)n_tokens * top_k, n_experts);
}

moeq_status moe_sort_pairs(const int32_t* idx, int32_t n_tokens, int32_t top_k, int32_t n_experts, int32_t* offsets, int32_t* order,
                           int32_t* slot, void* ws, size_t ws_bytes, void* stream) {
  if (n_tokens < 0 || top_k <= 0 || n_experts <= 0 || !offsets || !aligned(offsets, 4)) return MOEQ_EINVAL;
  if (n_tokens && (!idx || !order || !slot || !aligned(idx, 4) || !aligned(order, 4) || !aligned(slot, 4))) return MOEQ_EINVAL;
  const int64_t pairs = (int64_t)n_tokens * top_k;
  if (n_experts > kSortMaxExperts || pairs > kMaxPairs) return MOEQ_EUNSUPPORTED;
  if (!apart({vec(offsets, n_experts + 1), vec(order, pairs), vec(slot, pairs)}, {vec(idx, pairs)})) return MOEQ_EINVAL;
  const size_t need = sort_ws_bytes(pairs, n_experts);
  if (need && (!ws || ws_bytes < need)) return MOEQ_EWORKSPACE;
  if (need && !aligned(ws, 4)) return MOEQ_EINVAL;
  return done(launch_sort_pairs(idx, pairs, n_experts, offsets, order, slot, ws, (hipStream_t)stream));
}

moeq_status moe_gather_rows(const int32_t* slot, int32_t n_tokens, int32_t top_k, int32_t d, int32_t dtype, const void* x,
                            int64_t x_stride, void* rows, int64_t rows_stride, void* stream) {
  if (moeq_status s = rows_ok(slot, n_tokens, top_k, d); s != MOEQ_OK) return s;
  if (!type_ok(dtype) || !matrix_ok(x, n_tokens, x_stride, d, dtype, true)) return MOEQ_EINVAL;
  if (!matrix_ok(rows, (int64_t)n_tokens * top_k, rows_stride, d, dtype, false)) return MOEQ_EINVAL;
  const int64_t pairs = (int64_t)n_tokens * top_k;
  if (!apart({{rows, pairs, rows_stride, d, dtype}}, {{x, n_tokens, x_stride, d, dtype}, vec(slot, pairs)})) return MOEQ_EINVAL;
  if (n_tokens == 0) return MOEQ_OK;
  RowsArgs a = {};
  a.slot = slot, a.T = n_tokens, a.k = top_k, a.d = d, a.a = x, a.a_stride = x_stride, a.out = rows, a.out_stride = rows_stride;
  return done(launch_gather_rows(a, dtype, (hipStream_t)stream));
}

moeq_status moe_combine_rows(const int32_t* slot, const float* gate_opt, int32_t n_tokens, int32_t top_k, int32_t d, int32_t dtype,
                             const void* rows, int64_t rows_stride, int32_t y_dtype, void* y, int64_t y_stride, void* stream) {
  if (moeq_status s = rows_ok(slot, n_tokens, top_k, d); s != MOEQ_OK) return s;
  if (!type_ok(dtype) || (y_dtype != dtype && y_dtype != MOEQ_F32) || !aligned(gate_opt, 4)) return MOEQ_EINVAL;
  if (!matrix_ok(rows, (int64_t)n_tokens * top_k, rows_stride, d, dtype, true)) return MOEQ_EINVAL;
  if (!matrix_ok(y, n_tokens, y_stride, d, y_dtype, false)) return MOEQ_EINVAL;
  const int64_t pairs = (int64_t)n_tokens * top_k;
  if (!apart({{y, n_tokens, y_stride, d, y_dtype}}, {{rows, pairs, rows_stride, d, dtype}, vec(slot, pairs), vec(gate_opt, pairs)})) return MOEQ_EINVAL;
  if (n_tokens == 0) return MOEQ_OK;
  RowsArgs a = {};
  a.slot = slot, a.gate = gate_opt, a.T = n_tokens, a.k = top_k, a.d = d, a.a = rows, a.a_stride = rows_stride, a.out = y, a.out_stride = y_stride;
  return done(launch_combine_rows(a, dtype, y_dtype, (hipStream_t)stream));
}

moeq_status moe_combine_rows_backward(const int32_t* slot, const float* gate_opt, int32_t n_tokens, int32_t top_k, int32_t d,
                                      int32_t dtype, const void* rows, int64_t rows_stride, int32_t dy_dtype, const void* dy,
                                      int64_t dy_stride, void* drows, int64_t drows_stride, float* dgate_opt, void* stream) {
  if (moeq_status s = rows_ok(slot, n_tokens, top_k, d); s != MOEQ_OK) return s;
  if (!type_ok(dtype) || (dy_dtype != dtype && dy_dtype != MOEQ_F32) || !aligned(gate_opt, 4) || !aligned(dgate_opt, 4)) return MOEQ_EINVAL;
  const int64_t pairs = (int64_t)n_tokens * top_k;
  if (dgate_opt && !matrix_ok(rows, pairs, rows_stride, d, dtype, true)) return MOEQ_EINVAL;
  if (!matrix_ok(dy, n_tokens, dy_stride, d, dy_dtype, true) || !matrix_ok(drows, pairs, drows_stride, d, dtype, false)) return MOEQ_EINVAL;
  if (!apart({{drows, pairs, drows_stride, d, dtype}, vec(dgate_opt, pairs)},
             {{dgate_opt ? rows : nullptr, pairs, rows_stride, d, dtype}, {dy, n_tokens, dy_stride, d, dy_dtype}, vec(slot, pairs), vec(gate_opt, pairs)}))
    return MOEQ_EINVAL;
  if (n_tokens == 0) return MOEQ_OK;
  RowsArgs a = {};
  a.slot = slot, a.gate = gate_opt, a.T = n_tokens, a.k = top_k, a.d = d, a.a = rows, a.a_stride = rows_stride, a.dy = dy, a.dy_stride = dy_stride;
  a.out = drows, a.out_stride = drows_stride, a.dgate = dgate_opt;
  return done(launch_combine_rows_backward(a, dtype, dy_dtype, (hipStream_t)stream));
}

size_t moe_adapters_workspace_bytes(const moeq_adapters* adapters, int32_t max_tokens, int32_t backward) {
  if (adapters_ok(adapters, max_tokens, MOEQ_F32) != MOEQ_OK) return 0;
  return adapter_ws_bytes(adapter_args(adapters, max_tokens, MOEQ_F32), backward != 0);
}

moeq_status moe_adapters_forward(const moeq_adapters* adapters, const void* x, int64_t x_stride, const int32_t* ids, int32_t n_tokens,
                                 const void* base_opt, int64_t base_stride, int32_t y_dtype, void* y, int64_t y_stride, void* ws,
                                 size_t ws_bytes, void* stream) {
  if (moeq_status s = adapters_ok(adapters, n_tokens, y_dtype); s != MOEQ_OK) return s;
  if (n_tokens == 0) return MOEQ_OK;
  const moeq_adapters& L = *adapters;
  if (!ids || !aligned(ids, 4) || !matrix_ok(x, n_tokens, x_stride, L.d_in, L.dtype, true) ||
      !matrix_ok(y, n_tokens, y_stride, L.d_out, y_dtype, false))
    return MOEQ_EINVAL;
  if (base_opt && !matrix_ok(base_opt, n_tokens, base_stride, L.d_out, y_dtype, true)) return MOEQ_EINVAL;
  const Block out{y, n_tokens, y_stride, L.d_out, y_dtype};
  if (!apart({out}, {{x, n_tokens, x_stride, L.d_in, L.dtype}, vec(ids, n_tokens), a_of(L), b_of(L), vec(L.scale, L.n_adapters)}) ||
      !apart_or_same({base_opt, n_tokens, base_stride, L.d_out, y_dtype}, out))
    return MOEQ_EINVAL;
  AdapterArgs p = adapter_args(adapters, n_tokens, y_dtype);
  p.x = x, p.x_stride = x_stride, p.ids = ids, p.base = base_opt, p.base_stride = base_stride, p.out = y, p.out_stride = y_stride, p.ws = ws;
  const size_t need = adapter_ws_bytes(p, false);
  if (!ws || ws_bytes < need) return MOEQ_EWORKSPACE;
  if (!aligned(ws, 16)) return MOEQ_EINVAL;
  return done(launch_adapters_forward(p, (hipStream_t)stream));
}

moeq_status moe_adapters_backward(const moeq_adapters* adapters, const void* x, int64_t x_stride, const int32_t* ids, int32_t n_tokens,
                                  int32_t dy_dtype, const void* dy, int64_t dy_stride, const void* dx_base_opt, int64_t dx_base_stride,
                                  void* dx_opt, int64_t dx_stride, float* dA, float* dB, void* ws, size_t ws_bytes, void* stream) {
  if (moeq_status s = adapters_ok(adapters, n_tokens, dy_dtype); s != MOEQ_OK) return s;
  const moeq_adapters& L = *adapters;
  if (!dA || !dB || !aligned(dA, 4) || !aligned(dB, 4)) return MOEQ_EINVAL;
  if (n_tokens && (!ids || !aligned(ids, 4))) return MOEQ_EINVAL;
  if (!matrix_ok(x, n_tokens, x_stride, L.d_in, L.dtype, true) || !matrix_ok(dy, n_tokens, dy_stride, L.d_out, dy_dtype, true)) return MOEQ_EINVAL;
  if (dx_opt) {
    if (!matrix_ok(dx_opt, n_tokens, dx_stride, L.d_in, dy_dtype, false)) return MOEQ_EINVAL;
    if (dx_base_opt && !matrix_ok(dx_base_opt, n_tokens, dx_base_stride, L.d_in, dy_dtype, true)) return MOEQ_EINVAL;
  }
  const Block dx{dx_opt, n_tokens, dx_stride, L.d_in, dy_dtype}, base{dx_opt ? dx_base_opt : nullptr, n_tokens, dx_base_stride, L.d_in, dy_dtype};
  const Block da = vec(dA, (int64_t)L.n_adapters * L.rank * L.d_in), db = vec(dB, (int64_t)L.n_adapters * L.rank * L.d_out);
  if (!apart({dx, da, db}, {{x, n_tokens, x_stride, L.d_in, L.dtype}, {dy, n_tokens, dy_stride, L.d_out, dy_dtype}, vec(ids, n_tokens), a_of(L), b_of(L),
                            vec(L.scale, L.n_adapters)}) ||
      overlap(base, da) || overlap(base, db) || !apart_or_same(base, dx))
    return MOEQ_EINVAL;
  AdapterArgs p = adapter_args(adapters, n_tokens, dy_dtype);
  p.x = x, p.x_stride = x_stride, p.ids = ids, p.dy = dy, p.dy_stride = dy_stride, p.base = dx_base_opt, p.base_stride = dx_base_stride;
  p.out = dx_opt, p.out_stride = dx_stride, p.dA = dA, p.dB = dB, p.ws = ws;
  const size_t need = adapter_ws_bytes(p, true);
  if (need && (!ws || ws_bytes < need)) return MOEQ_EWORKSPACE;
  if (need && !aligned(ws, 16)) return MOEQ_EINVAL;
  return done(launch_adapters_backward(p, (hipStream_t)stream));
}

size_t moe_distill_workspace_bytes(int32_t max_tokens, int32_t vocab, int32_t dtype) {
  if (max_tokens <= 0 || vocab <= 0 || !type_ok(dtype)) return 0;
  return distill_ws_bytes(max_tokens, vocab, dtype);
}

moeq_status moe_distill_forward(const void* logits, int64_t stride, int32_t dtype, int32_t n_tokens, int32_t vocab,
                                const int32_t* top_idx, const float* top_logits, int32_t top, float temperature,
                                const float* weight_opt, float* loss, float* lse_opt, void* ws, size_t ws_bytes, void* stream) {
  DistillArgs a = distill_args(logits, stride, dtype, n_tokens, vocab, top_idx, top_logits, top, temperature, weight_opt);
  a.loss = loss, a.lse = lse_opt, a.ws = ws;
  if (moeq_status s = distill_ok(a, ws, ws_bytes, false, true); s != MOEQ_OK) return s;
  if (n_tokens == 0) return MOEQ_OK;
  if (!loss || !aligned(loss, 4) || !aligned(lse_opt, 4)) return MOEQ_EINVAL;
  return done(launch_distill_forward(a, (hipStream_t)stream));
}

moeq_status moe_distill_backward(const void* logits, int64_t stride, int32_t dtype, int32_t n_tokens, int32_t vocab,
                                 const int32_t* top_idx, const float* top_logits, int32_t top, float temperature,
                                 const float* weight_opt, const float* lse, const float* dloss, void* dlogits, int64_t dstride,
                                 void* stream) {
  DistillArgs a = distill_args(logits, stride, dtype, n_tokens, vocab, top_idx, top_logits, top, temperature, weight_opt);
  a.dlogits = dlogits, a.dstride = dstride, a.lse_in = lse, a.dloss = dloss;
  if (moeq_status s = distill_ok(a, nullptr, 0, true, false); s != MOEQ_OK) return s;
  if (n_tokens == 0) return MOEQ_OK;
  if (!lse || !dloss || !aligned(lse, 4) || !aligned(dloss, 4)) return MOEQ_EINVAL;
  return done(launch_distill_backward(a, (hipStream_t)stream));
}

moeq_status moe_distill_loss_grad(const void* logits, int64_t stride, int32_t dtype, int32_t n_tokens, int32_t vocab,
                                  const int32_t* top_idx, const float* top_logits, int32_t top, float temperature,
                                  const float* weight_opt, float* loss, void* dlogits, int64_t dstride, void* ws, size_t ws_bytes,
                                  void* stream) {
  DistillArgs a = distill_args(logits, stride, dtype, n_tokens, vocab, top_idx, top_logits, top, temperature, weight_opt);
  a.dlogits = dlogits, a.dstride = dstride, a.loss = loss, a.ws = ws;
  if (moeq_status s = distill_ok(a, ws, ws_bytes, true, true); s != MOEQ_OK) return s;
  if (n_tokens == 0) return MOEQ_OK;
  if (!loss || !aligned(loss, 4)) return MOEQ_EINVAL;
  return done(launch_distill_loss_grad(a, (hipStream_t)stream));
}

}  // extern "C"
