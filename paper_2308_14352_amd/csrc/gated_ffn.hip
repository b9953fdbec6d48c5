// The gated feed-forward block's kernels for bf16, and the choice of the type (ffn_core.h has what they do).
#include "ffn_core.h"

namespace moeq {

size_t ffn_ws_bytes(const FfnArgs& a, bool backward) { return tiles::FfnPlan(a, backward).bytes; }

hipError_t launch_ffn_forward(const FfnArgs& a, hipStream_t st) {
  if (a.dtype == MOEQ_F16) return ffn_forward_f16(a, st);
  if (a.dtype == MOEQ_F32) return ffn_forward_f32(a, st);
  return tiles::ffn_forward<__bf16>(a, st);
}
hipError_t launch_ffn_backward(const FfnArgs& a, hipStream_t st) {
  if (a.dtype == MOEQ_F16) return ffn_backward_f16(a, st);
  if (a.dtype == MOEQ_F32) return ffn_backward_f32(a, st);
  return tiles::ffn_backward<__bf16>(a, st);
}

}  // namespace moeq
