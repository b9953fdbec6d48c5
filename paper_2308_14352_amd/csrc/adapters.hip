// Low-rank adapters of many requests beside a shared projection: y[t] = base[t] + scale_a B_a A_a x[t] with a = ids[t], and the
// gradient. A [n][r][d_in], B [n][d_out][r]; a row whose id is outside [0, n) has no adapter.
//   forward   h = scale_a A_a x,   y = base + B_a h
//   backward  g = scale_a B_a^T dy,   dx = dx_base + A_a^T g,   dA_a = sum of g x^T,   dB_a = sum of dy h^T
#include "operators.h"

namespace moeq {
namespace {

constexpr int kThreads = 256;

__device__ __forceinline__ float block_sum(float v, float* part) {
#pragma unroll
  for (int m = 1; m < 64; m <<= 1) v += __shfl_xor(v, m);
  if (threadIdx.x % 64 == 0) part[threadIdx.x / 64] = v;
  __syncthreads();
  v = (part[0] + part[1]) + (part[2] + part[3]);
  __syncthreads();
  return v;
}

// h[t][j] = scale * sum of in[t][i] * W(j, i): W = A (rows of r), or B read across its rows (TRANS).
template <typename X, typename W, bool TRANS>
__global__ __launch_bounds__(kThreads) void k_shrink(AdapterArgs P, const void* in, int64_t stride, int d, float* h) {
  __shared__ float part[4];
  const int t = blockIdx.x, a = P.ids[t], r = P.rank;
  const bool on = (uint32_t)a < (uint32_t)P.n;
  for (int j = 0; j < r; ++j) {
    float sum = 0.f;
    if (on)
      for (int i = threadIdx.x; i < d; i += kThreads) {
        const W* w = (const W*)(TRANS ? P.B : P.A) + (int64_t)a * r * d + (TRANS ? (int64_t)i * r + j : (int64_t)j * d + i);
        sum = fmaf((float)((const X*)in)[t * stride + i], (float)*w, sum);
      }
    sum = block_sum(sum, part);
    if (threadIdx.x == 0) h[(int64_t)t * r + j] = on ? sum * P.scale[a] : 0.f;
  }
}

// out[t][i] = base + sum of h[t][j] * W(i, j): W = B (rows of d_out), or A read across its rows (TRANS).
template <typename Y, typename W, bool TRANS>
__global__ __launch_bounds__(kThreads) void k_expand(AdapterArgs P, const float* h, int d) {
  const int t = blockIdx.y, i = blockIdx.x * kThreads + threadIdx.x, a = P.ids[t], r = P.rank;
  if (i >= d) return;
  float sum = 0.f;
  if ((uint32_t)a < (uint32_t)P.n)
    for (int j = 0; j < r; ++j) {
      const W* w = (const W*)(TRANS ? P.A : P.B) + (int64_t)a * r * d + (TRANS ? (int64_t)j * d + i : (int64_t)i * r + j);
      sum = fmaf(h[(int64_t)t * r + j], (float)*w, sum);
    }
  const float base = P.base ? (float)((const Y*)P.base)[t * P.base_stride + i] : 0.f;
  ((Y*)P.out)[t * P.out_stride + i] = (Y)(base + sum);
}

// dW of adapter blockIdx.z, rank index blockIdx.y: dA[a][j][i] = sum of h[t][j] * in[t][i] (TRANS: at dB[a][i][j]).
template <typename X, bool TRANS>
__global__ __launch_bounds__(kThreads) void k_wgrad(AdapterArgs P, const void* in, int64_t stride, int d, const float* h, float* out) {
  const int i = blockIdx.x * kThreads + threadIdx.x, j = blockIdx.y, a = blockIdx.z, r = P.rank;
  if (i >= d) return;
  float sum = 0.f;
  for (int t = 0; t < P.T; ++t)
    if (P.ids[t] == a) sum = fmaf(h[(int64_t)t * r + j], (float)((const X*)in)[t * stride + i], sum);
  out[(int64_t)a * r * d + (TRANS ? (int64_t)i * r + j : (int64_t)j * d + i)] = sum;
}

template <typename F>
hipError_t with_types(const AdapterArgs& a, F&& f) {
  return with_type(a.dtype, [&](auto tag) { return a.out_dtype == MOEQ_F32 ? f(tag, float{}) : f(tag, tag); });
}

}  // namespace

size_t adapter_ws_bytes(const AdapterArgs& a, bool backward) { return (size_t)a.T * a.rank * 4 * (backward ? 2 : 1); }

hipError_t launch_adapters_forward(const AdapterArgs& a, hipStream_t st) {
  if (a.T == 0) return hipSuccess;
  return with_types(a, [&](auto tag, auto ytag) {
    using W = decltype(tag);
    using Y = decltype(ytag);
    float* h = (float*)a.ws;
    hipLaunchKernelGGL((k_shrink<W, W, false>), dim3(a.T), dim3(kThreads), 0, st, a, a.x, a.x_stride, a.d_in, h);
    hipLaunchKernelGGL((k_expand<Y, W, false>), dim3((a.d_out + kThreads - 1) / kThreads, a.T), dim3(kThreads), 0, st, a, h, a.d_out);
    return hipGetLastError();
  });
}

hipError_t launch_adapters_backward(const AdapterArgs& a, hipStream_t st) {
  return with_types(a, [&](auto tag, auto ytag) {
    using W = decltype(tag);
    using Y = decltype(ytag);
    float *h = (float*)a.ws, *g = h + (size_t)a.T * a.rank;
    if (a.T) {
      hipLaunchKernelGGL((k_shrink<W, W, false>), dim3(a.T), dim3(kThreads), 0, st, a, a.x, a.x_stride, a.d_in, h);
      hipLaunchKernelGGL((k_shrink<Y, W, true>), dim3(a.T), dim3(kThreads), 0, st, a, a.dy, a.dy_stride, a.d_out, g);
      if (a.out) hipLaunchKernelGGL((k_expand<Y, W, true>), dim3((a.d_in + kThreads - 1) / kThreads, a.T), dim3(kThreads), 0, st, a, g, a.d_in);
    }
    hipLaunchKernelGGL((k_wgrad<W, false>), dim3((a.d_in + kThreads - 1) / kThreads, a.rank, a.n), dim3(kThreads), 0, st, a, a.x, a.x_stride, a.d_in, g, a.dA);
    hipLaunchKernelGGL((k_wgrad<Y, true>), dim3((a.d_out + kThreads - 1) / kThreads, a.rank, a.n), dim3(kThreads), 0, st, a, a.dy, a.dy_stride, a.d_out, h, a.dB);
    return hipGetLastError();
  });
}

}  // namespace moeq
