// The gated feed-forward block's kernels for fp16 (ffn_core.h has what they do).
#include "ffn_core.h"

namespace moeq {

hipError_t ffn_forward_f16(const FfnArgs& a, hipStream_t st) { return tiles::ffn_forward<_Float16>(a, st); }
hipError_t ffn_backward_f16(const FfnArgs& a, hipStream_t st) { return tiles::ffn_backward<_Float16>(a, st); }

}  // namespace moeq
