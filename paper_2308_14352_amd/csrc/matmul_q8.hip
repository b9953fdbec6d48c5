// A product in 8-bit integers: rows of x and of w as codes with a scale each (k_quantize_rows),
//   y[t][n] = base[t][n] + scale_x[t] scale_w[n] sum over k of x[t][k] w[n][k].
// The sums are whole numbers in 32 bits (K <= 65536 codes of at most 128 each: below 2^30), so that no order of adding changes them.
#include "tiles.h"

namespace moeq {
namespace {

using namespace tiles;

template <typename O>
struct Scaled {
  O* y;
  int64_t stride;
  const O* base;
  int64_t base_stride;
  const float *xs, *ws;
  int32_t T, N;
  __device__ __forceinline__ void block(int, int m, int n, int half, const i32x16& c) const {
    if (m >= T) return;
    const float s = xs[m];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int at = column(n, half, q);
      if (at >= N) continue;
      float v[4], w[4], b[4] = {};
      load4(w, ws, at, N);
      if (base) load4(b, base + m * base_stride, at, N);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float p = (float)c[4 * q + i] * (s * w[i]);
        v[i] = base ? b[i] + p : p;
      }
      store4(y + m * stride, at, N, v);
    }
  }
};

}  // namespace

size_t q8_ws_bytes(int32_t, int32_t, int32_t) { return 0; }

hipError_t launch_matmul_q8(const Q8Args& a, hipStream_t st) {
  return with_type(a.dtype, [&](auto o) {
    using O = decltype(o);
    const int32_t pitch = (int32_t)q8_pitch(a.K);
    Product p = {Side{{(const char*)a.x, nullptr}, pitch, a.T, pitch}, Side{{(const char*)a.w, nullptr}, pitch, a.N, pitch}, pitch / kStepBytes, 0};
    Scaled<O> e = {(O*)a.y, a.y_stride, (const O*)a.base, a.base_stride, a.x_scale, a.w_scale, a.T, a.N};
    return launch_tile<int8_t, true, true, kOne>(p, a.T, a.N, 1, e, st);
  });
}

}  // namespace moeq
