// Host side of the operators beside the layer: argument checks (all before the first HIP call) and launches.
#include "operators.h"

#include <algorithm>
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
// n contiguous bytes.
inline Block codes_of(const void* p, int64_t n) { return Block{p, n > 0, n, n, kByteType}; }
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

moeq_status norms_ok(const NormsArgs& a) {
  if (a.T < 0 || a.d <= 0 || !type_ok(a.f_dtype) || !type_ok(a.r_dtype) || !type_ok(a.n_dtype)) return MOEQ_EINVAL;
  if (!(a.eps >= 0.f) || a.eps > 1e30f || !(a.alpha >= -1e30f && a.alpha <= 1e30f)) return MOEQ_EINVAL;
  int32_t half = MOEQ_F32;
  for (int32_t t : {a.f_dtype, a.r_dtype, a.n_dtype}) {
    if (t == MOEQ_F32) continue;
    if (half != MOEQ_F32 && half != t) return MOEQ_EINVAL;
    half = t;
  }
  if (a.d > kNormsMaxWidth) return MOEQ_EUNSUPPORTED;
  if (!aligned(a.gate, 4) || !aligned(a.w_after, 4) || !aligned(a.w_before, 4)) return MOEQ_EINVAL;
  return matrix_ok(a.f, a.T, a.f_stride, a.d, a.f_dtype, true) ? MOEQ_OK : MOEQ_EINVAL;
}

moeq_status ffn_ok(const moeq_gated_ffn* f, int32_t n_tokens, int32_t keep) {
  if (!f || f->d_model <= 0 || f->d_ff <= 0 || !type_ok(f->dtype) || n_tokens < 0) return MOEQ_EINVAL;
  if (keep != MOEQ_KEEP_NONE && keep != MOEQ_KEEP_OWN && keep != MOEQ_KEEP_8) return MOEQ_EINVAL;
  if (f->d_model > kFfnMaxWidth || f->d_ff > kFfnMaxWidth || n_tokens > kProductMaxRows || (int64_t)n_tokens * 2 * std::max(f->d_model, f->d_ff) > kProductMaxOut)
    return MOEQ_EUNSUPPORTED;
  const size_t e = dtype_bytes(f->dtype);
  if (!f->w_in || !f->w_gate || !f->w_out || !aligned(f->w_in, e) || !aligned(f->w_gate, e) || !aligned(f->w_out, e)) return MOEQ_EINVAL;
  return MOEQ_OK;
}
FfnArgs ffn_args(const moeq_gated_ffn* f, int32_t n_tokens, int32_t keep) {
  FfnArgs a = {};
  a.T = n_tokens, a.D = f->d_model, a.F = f->d_ff, a.dtype = f->dtype, a.w_in = f->w_in, a.w_gate = f->w_gate, a.w_out = f->w_out, a.keep = keep;
  return a;
}
// What is kept of a and b, and of one of them the exponents.
Block ab_of(const FfnArgs& a, const void* ab) {
  const int64_t n = (int64_t)2 * a.T * a.F;
  return a.keep == MOEQ_KEEP_NONE ? Block{} : a.keep == MOEQ_KEEP_8 ? codes_of(ab, n) : Block{ab, n > 0, n, n, a.dtype};
}
Block exps_of(const FfnArgs& a, const void* exps) {
  return a.keep == MOEQ_KEEP_8 ? codes_of(exps, (int64_t)2 * a.T * ((a.F + kPackBlock - 1) / kPackBlock)) : Block{};
}
bool kept_ok(const FfnArgs& a, const void* ab, const void* exps) {
  if (a.T == 0 || a.keep == MOEQ_KEEP_NONE) return true;
  return ab && (a.keep == MOEQ_KEEP_8 ? exps != nullptr : aligned(ab, dtype_bytes(a.dtype)));
}
inline Block weight_of(const FfnArgs& a, const void* w) { return Block{w, 1, (int64_t)a.D * a.F, (int64_t)a.D * a.F, a.dtype}; }

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

moeq_status moe_block_norms_forward(int32_t n_tokens, int32_t d, float residual_scale, float eps, int32_t f_dtype, const void* f,
                                    int64_t f_stride, int32_t r_dtype, const void* r, int64_t r_stride, const float* gate_opt,
                                    const float* w_after_opt, const float* w_before_opt, void* y, int64_t y_stride, int32_t n_dtype,
                                    void* n, int64_t n_stride, void* stream) {
  NormsArgs a = {};
  a.T = n_tokens, a.d = d, a.alpha = residual_scale, a.eps = eps, a.f_dtype = f_dtype, a.r_dtype = r_dtype, a.n_dtype = n_dtype;
  a.f = f, a.f_stride = f_stride, a.r = r, a.r_stride = r_stride, a.gate = gate_opt, a.w_after = w_after_opt, a.w_before = w_before_opt;
  a.out_y = y, a.out_y_stride = y_stride, a.out_n = w_before_opt ? n : nullptr, a.out_n_stride = n_stride;
  if (moeq_status s = norms_ok(a); s != MOEQ_OK) return s;
  if (!matrix_ok(r, n_tokens, r_stride, d, r_dtype, true) || !matrix_ok(y, n_tokens, y_stride, d, r_dtype, false)) return MOEQ_EINVAL;
  if (w_before_opt && !matrix_ok(n, n_tokens, n_stride, d, n_dtype, false)) return MOEQ_EINVAL;
  const Block by{y, n_tokens, y_stride, d, r_dtype}, bn{a.out_n, n_tokens, n_stride, d, n_dtype}, bf{f, n_tokens, f_stride, d, f_dtype},
      br{r, n_tokens, r_stride, d, r_dtype};
  if (!apart({by, bn}, {vec(gate_opt, n_tokens), vec(w_after_opt, d), vec(w_before_opt, d)}) || overlap(bf, by) || overlap(br, bn) ||
      !apart_or_same(br, by) || !apart_or_same(bf, bn))
    return MOEQ_EINVAL;
  if (n_tokens == 0) return MOEQ_OK;
  return done(launch_norms_forward(a, (hipStream_t)stream));
}

size_t moe_block_norms_workspace_bytes(int32_t max_tokens, int32_t d) {
  return max_tokens <= 0 || d <= 0 || d > kNormsMaxWidth ? 0 : norms_ws_bytes(max_tokens, d);
}

moeq_status moe_block_norms_backward(int32_t n_tokens, int32_t d, float residual_scale, float eps, int32_t f_dtype, const void* f,
                                     int64_t f_stride, int32_t r_dtype, const void* y, int64_t y_stride, const void* dy,
                                     int64_t dy_stride, int32_t n_dtype, const void* dn, int64_t dn_stride, const float* gate_opt,
                                     const float* w_after_opt, const float* w_before_opt, void* df, int64_t df_stride, void* dr,
                                     int64_t dr_stride, float* dgate, float* dw_after, float* dw_before, void* ws, size_t ws_bytes,
                                     void* stream) {
  NormsArgs a = {};
  a.T = n_tokens, a.d = d, a.alpha = residual_scale, a.eps = eps, a.f_dtype = f_dtype, a.r_dtype = r_dtype, a.n_dtype = n_dtype;
  a.f = f, a.f_stride = f_stride, a.y = w_before_opt ? y : nullptr, a.y_stride = y_stride, a.dy = dy, a.dy_stride = dy_stride;
  a.dn = w_before_opt ? dn : nullptr, a.dn_stride = dn_stride, a.gate = gate_opt, a.w_after = w_after_opt, a.w_before = w_before_opt;
  a.out_y = dr, a.out_y_stride = dr_stride, a.out_n = df, a.out_n_stride = df_stride;
  a.dgate = gate_opt ? dgate : nullptr, a.dw_after = w_after_opt ? dw_after : nullptr, a.dw_before = w_before_opt ? dw_before : nullptr, a.ws = (float*)ws;
  if (moeq_status s = norms_ok(a); s != MOEQ_OK) return s;
  if (!matrix_ok(dy, n_tokens, dy_stride, d, r_dtype, true) || !matrix_ok(df, n_tokens, df_stride, d, f_dtype, false) ||
      !matrix_ok(dr, n_tokens, dr_stride, d, r_dtype, false))
    return MOEQ_EINVAL;
  if (w_before_opt && (!matrix_ok(y, n_tokens, y_stride, d, r_dtype, true) || !matrix_ok(dn, n_tokens, dn_stride, d, n_dtype, true))) return MOEQ_EINVAL;
  if ((gate_opt && n_tokens && !a.dgate) || (w_after_opt && !a.dw_after) || (w_before_opt && !a.dw_before)) return MOEQ_EINVAL;
  if (!aligned(a.dgate, 4) || !aligned(a.dw_after, 4) || !aligned(a.dw_before, 4)) return MOEQ_EINVAL;
  if (!apart({{df, n_tokens, df_stride, d, f_dtype}, {dr, n_tokens, dr_stride, d, r_dtype}, vec(a.dgate, n_tokens), vec(a.dw_after, d), vec(a.dw_before, d)},
             {{f, n_tokens, f_stride, d, f_dtype}, {a.y, n_tokens, y_stride, d, r_dtype}, {dy, n_tokens, dy_stride, d, r_dtype},
              {a.dn, n_tokens, dn_stride, d, n_dtype}, vec(gate_opt, n_tokens), vec(w_after_opt, d), vec(w_before_opt, d)}))
    return MOEQ_EINVAL;
  if (n_tokens && (w_after_opt || w_before_opt)) {
    if (!ws || ws_bytes < norms_ws_bytes(n_tokens, d)) return MOEQ_EWORKSPACE;
    if (!aligned(ws, 16)) return MOEQ_EINVAL;
  }
  return done(launch_norms_backward(a, (hipStream_t)stream));
}

moeq_status moe_pack8(const void* x, int64_t x_stride, int32_t dtype, int32_t rows, int32_t d, int8_t* codes, int8_t* exps, void* stream) {
  if (rows < 0 || d <= 0 || !type_ok(dtype) || !matrix_ok(x, rows, x_stride, d, dtype, true) || (rows && (!codes || !exps))) return MOEQ_EINVAL;
  if (d > kPackMaxWidth) return MOEQ_EUNSUPPORTED;
  const Block c = codes_of(codes, (int64_t)rows * d), e = codes_of(exps, (int64_t)rows * ((d + kPackBlock - 1) / kPackBlock));
  if (!apart({c, e}, {{x, rows, x_stride, d, dtype}})) return MOEQ_EINVAL;
  if (rows == 0) return MOEQ_OK;
  Rows8Args a = {};
  a.T = rows, a.d = d, a.dtype = dtype, a.x = x, a.x_stride = x_stride, a.codes = codes, a.exps = exps;
  return done(launch_pack8(a, (hipStream_t)stream));
}

moeq_status moe_unpack8(const int8_t* codes, const int8_t* exps, int32_t rows, int32_t d, int32_t dtype, void* x, int64_t x_stride, void* stream) {
  if (rows < 0 || d <= 0 || !type_ok(dtype) || !matrix_ok(x, rows, x_stride, d, dtype, false) || (rows && (!codes || !exps))) return MOEQ_EINVAL;
  if (d > kPackMaxWidth) return MOEQ_EUNSUPPORTED;
  if (!apart({{x, rows, x_stride, d, dtype}},
             {codes_of(codes, (int64_t)rows * d), codes_of(exps, (int64_t)rows * ((d + kPackBlock - 1) / kPackBlock))}))
    return MOEQ_EINVAL;
  if (rows == 0) return MOEQ_OK;
  Rows8Args a = {};
  a.T = rows, a.d = d, a.dtype = dtype, a.out = x, a.out_stride = x_stride, a.codes = (int8_t*)codes, a.exps = (int8_t*)exps;
  return done(launch_unpack8(a, (hipStream_t)stream));
}

size_t moe_gated_ffn_workspace_bytes(const moeq_gated_ffn* ffn, int32_t max_tokens, int32_t backward, int32_t x_packed, int32_t keep) {
  if (ffn_ok(ffn, max_tokens, keep) != MOEQ_OK || max_tokens == 0) return 0;
  FfnArgs a = ffn_args(ffn, max_tokens, keep);
  a.x_codes = x_packed ? (const int8_t*)ffn : nullptr;      // (whether there are any is all that counts)
  return ffn_ws_bytes(a, backward != 0);
}

moeq_status moe_gated_ffn_forward(const moeq_gated_ffn* ffn, const void* x, int64_t x_stride, int32_t n_tokens, const void* base_opt,
                                  int64_t base_stride, int32_t y_dtype, void* y, int64_t y_stride, int32_t keep, void* ab, int8_t* ab_exps,
                                  void* ws, size_t ws_bytes, void* stream) {
  if (moeq_status s = ffn_ok(ffn, n_tokens, keep); s != MOEQ_OK) return s;
  if (y_dtype != ffn->dtype && y_dtype != MOEQ_F32) return MOEQ_EINVAL;
  if (n_tokens == 0) return MOEQ_OK;
  FfnArgs a = ffn_args(ffn, n_tokens, keep);
  a.x = x, a.x_stride = x_stride, a.base = base_opt, a.base_stride = base_stride, a.y_dtype = y_dtype, a.y = y, a.y_stride = y_stride, a.ws = ws;
  if (keep != MOEQ_KEEP_NONE) a.ab = ab, a.ab_exps = keep == MOEQ_KEEP_8 ? ab_exps : nullptr;
  if (!matrix_ok(x, n_tokens, x_stride, a.D, a.dtype, true) || !matrix_ok(y, n_tokens, y_stride, a.D, y_dtype, false) || !kept_ok(a, ab, ab_exps)) return MOEQ_EINVAL;
  if (base_opt && !matrix_ok(base_opt, n_tokens, base_stride, a.D, y_dtype, true)) return MOEQ_EINVAL;
  const Block out{y, n_tokens, y_stride, a.D, y_dtype}, base{base_opt, n_tokens, base_stride, a.D, y_dtype}, kab = ab_of(a, ab), kexps = exps_of(a, ab_exps);
  if (!apart({out, kab, kexps}, {{x, n_tokens, x_stride, a.D, a.dtype}, weight_of(a, a.w_in), weight_of(a, a.w_gate), weight_of(a, a.w_out)}) ||
      !apart_or_same(base, out) || overlap(base, kab) || overlap(base, kexps))
    return MOEQ_EINVAL;
  if (!ws || ws_bytes < ffn_ws_bytes(a, false)) return MOEQ_EWORKSPACE;
  if (!aligned(ws, 256)) return MOEQ_EINVAL;
  return done(launch_ffn_forward(a, (hipStream_t)stream));
}

moeq_status moe_gated_ffn_backward(const moeq_gated_ffn* ffn, const void* x, int64_t x_stride, const int8_t* x_codes, const int8_t* x_exps,
                                   int32_t n_tokens, const void* dy, int64_t dy_stride, int32_t keep, const void* ab, const int8_t* ab_exps,
                                   void* dx_opt, int64_t dx_stride, void* dw_in, void* dw_gate, void* dw_out, void* ws, size_t ws_bytes,
                                   void* stream) {
  if (moeq_status s = ffn_ok(ffn, n_tokens, keep); s != MOEQ_OK) return s;
  FfnArgs a = ffn_args(ffn, n_tokens, keep);
  const size_t e = dtype_bytes(a.dtype);
  a.x = x, a.x_stride = x_stride, a.x_codes = x_codes, a.x_exps = x_exps, a.dy = dy, a.dy_stride = dy_stride, a.dx = dx_opt, a.dx_stride = dx_stride;
  if (keep != MOEQ_KEEP_NONE) a.ab = (void*)ab, a.ab_exps = keep == MOEQ_KEEP_8 ? (int8_t*)ab_exps : nullptr;
  a.dw_in = dw_in, a.dw_gate = dw_gate, a.dw_out = dw_out, a.ws = ws;
  if (!dw_in || !dw_gate || !dw_out || !aligned(dw_in, e) || !aligned(dw_gate, e) || !aligned(dw_out, e)) return MOEQ_EINVAL;
  if (n_tokens && ((x != nullptr) == (x_codes != nullptr) || (x_codes && !x_exps))) return MOEQ_EINVAL;
  if ((x && !matrix_ok(x, n_tokens, x_stride, a.D, a.dtype, true)) || !matrix_ok(dy, n_tokens, dy_stride, a.D, a.dtype, true) || !kept_ok(a, ab, ab_exps)) return MOEQ_EINVAL;
  if (dx_opt && !matrix_ok(dx_opt, n_tokens, dx_stride, a.D, a.dtype, false)) return MOEQ_EINVAL;
  const int64_t blocks = (a.D + kPackBlock - 1) / kPackBlock;
  if (!apart({{dx_opt, n_tokens, dx_stride, a.D, a.dtype}, weight_of(a, dw_in), weight_of(a, dw_gate), weight_of(a, dw_out)},
             {{x, n_tokens, x_stride, a.D, a.dtype}, codes_of(x_codes, (int64_t)n_tokens * a.D), codes_of(x_exps, n_tokens * blocks),
              {dy, n_tokens, dy_stride, a.D, a.dtype}, ab_of(a, ab), exps_of(a, ab_exps), weight_of(a, a.w_in), weight_of(a, a.w_gate), weight_of(a, a.w_out)}))
    return MOEQ_EINVAL;
  if (n_tokens) {
    if (!ws || ws_bytes < ffn_ws_bytes(a, true)) return MOEQ_EWORKSPACE;
    if (!aligned(ws, 256)) return MOEQ_EINVAL;
  }
  return done(launch_ffn_backward(a, (hipStream_t)stream));
}

int64_t moe_q8_pitch(int32_t d) { return d <= 0 ? 0 : q8_pitch(d); }

moeq_status moe_quantize_rows(const void* x, int64_t x_stride, int32_t dtype, int32_t rows, int32_t d, int8_t* codes, float* scale, void* stream) {
  if (rows < 0 || d <= 0 || !type_ok(dtype) || !matrix_ok(x, rows, x_stride, d, dtype, true)) return MOEQ_EINVAL;
  if (d > kQuantMaxWidth) return MOEQ_EUNSUPPORTED;
  if (rows && (!codes || !scale || !aligned(codes, 16) || !aligned(scale, 4))) return MOEQ_EINVAL;
  if (!apart({codes_of(codes, rows * q8_pitch(d)), vec(scale, rows)}, {{x, rows, x_stride, d, dtype}})) return MOEQ_EINVAL;
  if (rows == 0) return MOEQ_OK;
  Rows8Args a = {};
  a.T = rows, a.d = d, a.dtype = dtype, a.x = x, a.x_stride = x_stride, a.codes = codes, a.scale = scale;
  return done(launch_quantize_rows(a, (hipStream_t)stream));
}

size_t moe_matmul_q8_workspace_bytes(int32_t max_tokens, int32_t n_out, int32_t k) {
  if (max_tokens <= 0 || n_out <= 0 || k <= 0 || k > kQuantMaxWidth || max_tokens > kProductMaxRows || n_out > kProductMaxRows) return 0;
  return q8_ws_bytes(max_tokens, n_out, k);
}

moeq_status moe_matmul_q8(const int8_t* x, const float* x_scale, int32_t n_tokens, const int8_t* w, const float* w_scale, int32_t n_out,
                          int32_t k, const void* base_opt, int64_t base_stride, int32_t dtype, void* y, int64_t y_stride, void* ws,
                          size_t ws_bytes, void* stream) {
  if (n_tokens < 0 || n_out <= 0 || k <= 0 || !type_ok(dtype) || !w || !w_scale || !aligned(w, 16) || !aligned(w_scale, 4)) return MOEQ_EINVAL;
  if (k > kQuantMaxWidth || n_tokens > kProductMaxRows || n_out > kProductMaxRows || (int64_t)n_tokens * n_out > kProductMaxOut) return MOEQ_EUNSUPPORTED;
  if (n_tokens == 0) return MOEQ_OK;
  if (!x || !x_scale || !aligned(x, 16) || !aligned(x_scale, 4) || !matrix_ok(y, n_tokens, y_stride, n_out, dtype, false)) return MOEQ_EINVAL;
  if (base_opt && !matrix_ok(base_opt, n_tokens, base_stride, n_out, dtype, true)) return MOEQ_EINVAL;
  const Block out{y, n_tokens, y_stride, n_out, dtype};
  if (!apart({out}, {codes_of(x, n_tokens * q8_pitch(k)), vec(x_scale, n_tokens), codes_of(w, n_out * q8_pitch(k)), vec(w_scale, n_out)}) ||
      !apart_or_same({base_opt, n_tokens, base_stride, n_out, dtype}, out))
    return MOEQ_EINVAL;
  const size_t need = q8_ws_bytes(n_tokens, n_out, k);
  if (need && (!ws || ws_bytes < need)) return MOEQ_EWORKSPACE;
  if (need && !aligned(ws, 16)) return MOEQ_EINVAL;
  Q8Args a = {};
  a.T = n_tokens, a.N = n_out, a.K = k, a.dtype = dtype, a.x = x, a.w = w, a.x_scale = x_scale, a.w_scale = w_scale;
  a.base = base_opt, a.base_stride = base_stride, a.y = y, a.y_stride = y_stride, a.ws = ws;
  return done(launch_matmul_q8(a, (hipStream_t)stream));
}

}  // extern "C"
