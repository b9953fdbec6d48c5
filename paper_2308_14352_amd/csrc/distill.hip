// Distillation from a teacher's top logits. Of a row with student logits z [V], teacher logits u at K indices, temperature tau and
// weight w: s = z / tau, q = softmax(s), p = softmax(u / tau) over the entries that have an index,
//   loss = w tau^2 sum_j p_j (log p_j - s[idx_j] + lse(s)),   dloss/dz = w tau (q - p at the indices).
// A row of weight 0, or without a teacher's entry, has no loss and no gradient.
#include "operators.h"

namespace moeq {
namespace {

constexpr int kThreads = 256;

template <bool MAX>
__device__ __forceinline__ float block_fold(float v, float* part) {
  const int waves = blockDim.x / 64;
#pragma unroll
  for (int m = 1; m < 64; m <<= 1) {
    const float o = __shfl_xor(v, m);
    v = MAX ? fmaxf(v, o) : v + o;
  }
  __syncthreads();
  if (threadIdx.x % 64 == 0) part[threadIdx.x / 64] = v;
  __syncthreads();
  v = part[0];
  for (int w = 1; w < waves; ++w) v = MAX ? fmaxf(v, part[w]) : v + part[w];
  return v;
}

// A logit of minus infinity has no probability, also where a whole row has none.
__device__ __forceinline__ float prob(float z, float it, float lse) { return z == -INFINITY ? 0.f : expf(z * it - lse); }

template <typename T>
__global__ __launch_bounds__(kThreads) void k_distill(DistillArgs A, bool grad) {
  __shared__ float part[16];
  const int t = blockIdx.x, V = A.V, K = A.K;
  const T* z = (const T*)A.logits + (int64_t)t * A.stride;
  const int32_t* idx = A.top_idx + (int64_t)t * K;
  const float* u = A.top_logits + (int64_t)t * K;
  const float it = 1.f / A.temperature;
  float w = A.weight ? A.weight[t] : 1.f, lse;
  if (A.lse_in) {
    lse = A.lse_in[t];
    w *= A.dloss[t];
  } else {
    float m = -INFINITY, s = 0.f;
    for (int i = threadIdx.x; i < V; i += kThreads) m = fmaxf(m, (float)z[i]);
    m = block_fold<true>(m, part);
    const float m0 = m == -INFINITY ? 0.f : m;
    for (int i = threadIdx.x; i < V; i += kThreads) s += expf(((float)z[i] - m0) * it);
    lse = logf(block_fold<false>(s, part)) + m0 * it;
    if (A.lse && threadIdx.x == 0) A.lse[t] = lse;
  }
  float top = -INFINITY, sum = 0.f;
  for (int j = threadIdx.x; j < K; j += kThreads)
    if ((uint32_t)idx[j] < (uint32_t)V) top = fmaxf(top, u[j]);
  top = block_fold<true>(top, part);
  const bool none = w == 0.f || top == -INFINITY;
  for (int j = threadIdx.x; j < K; j += kThreads)
    if ((uint32_t)idx[j] < (uint32_t)V && !none) sum += expf((u[j] - top) * it);
  sum = block_fold<false>(sum, part);
  if (A.loss) {
    float l = 0.f;
    for (int j = threadIdx.x; j < K; j += kThreads)
      if ((uint32_t)idx[j] < (uint32_t)V && !none) {
        const float lp = (u[j] - top) * it - logf(sum), p = expf(lp);
        const float zj = (float)z[idx[j]];
        if (p > 0.f) l += zj == -INFINITY ? INFINITY : p * (lp - (zj * it - lse));
      }
    l = block_fold<false>(l, part);
    if (threadIdx.x == 0) A.loss[t] = none ? 0.f : w * A.temperature * A.temperature * l;
  }
  if (!grad) return;
  T* dz = (T*)A.dlogits + (int64_t)t * A.dstride;
  const float c = w * A.temperature;
  for (int i = threadIdx.x; i < V; i += kThreads) dz[i] = none ? (T)0.f : (T)(c * prob((float)z[i], it, lse));
  __syncthreads();
  for (int j = threadIdx.x; j < K; j += kThreads) {
    if (none || (uint32_t)idx[j] >= (uint32_t)V) continue;
    float p = 0.f;
    for (int i = 0; i < K; ++i)
      if (idx[i] == idx[j]) p += expf((u[i] - top) * it) / sum;
    dz[idx[j]] = (T)(c * (prob((float)z[idx[j]], it, lse) - p));
  }
}

hipError_t launch(const DistillArgs& a, bool grad, hipStream_t st) {
  if (a.T == 0) return hipSuccess;
  return with_type(a.dtype, [&](auto tag) {
    hipLaunchKernelGGL(k_distill<decltype(tag)>, dim3(a.T), dim3(kThreads), 0, st, a, grad);
    return hipGetLastError();
  });
}

}  // namespace

size_t distill_ws_bytes(int32_t, int32_t, int32_t) { return 0; }
hipError_t launch_distill_forward(const DistillArgs& a, hipStream_t st) { return launch(a, false, st); }
hipError_t launch_distill_backward(const DistillArgs& a, hipStream_t st) { return launch(a, true, st); }
hipError_t launch_distill_loss_grad(const DistillArgs& a, hipStream_t st) { return launch(a, true, st); }

}  // namespace moeq
