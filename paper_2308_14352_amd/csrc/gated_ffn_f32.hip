// The gated feed-forward block's kernels for fp32 (ffn_core.h has what they do).
#include "ffn_core.h"

namespace moeq {

hipError_t ffn_forward_f32(const FfnArgs& a, hipStream_t st) { return tiles::ffn_forward<float>(a, st); }
hipError_t ffn_backward_f32(const FfnArgs& a, hipStream_t st) { return tiles::ffn_backward<float>(a, st); }

}  // namespace moeq
