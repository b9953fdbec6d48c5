// Shared by the operators beside the layer (dispatch.hip, adapters.hip, distill.hip) and their host side (operators.cpp): the
// launchers' arguments, and on the device the three element types with loads and stores of 16 bytes at any element's address.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "moeq.h"

namespace moeq {

inline int dtype_bytes(int32_t t) { return t == MOEQ_F32 ? 4 : 2; }
// Workgroups of a launch: the threads of a dimension of the grid have to be fewer than 2^32. Calls of more are several launches.
constexpr int32_t launch_groups(int32_t threads) { return (int32_t)(0xffffffffu / (uint32_t)threads); }

// ---- dispatch.hip ----
constexpr int32_t kSortMaxExperts = 1024;
size_t sort_ws_bytes(int64_t pairs, int32_t experts);
hipError_t launch_sort_pairs(const int32_t* idx, int64_t pairs, int32_t experts, int32_t* offsets, int32_t* order, int32_t* slot,
                             void* ws, hipStream_t st);
struct RowsArgs {
  const int32_t* slot;      // [T][k]
  const float* gate;        // [T][k] or null (ones)
  int32_t T, k, d;
  int32_t first;            // token of the launch's first thread
  const void* a;            // gather: x; combine: rows; backward: rows
  int64_t a_stride;
  const void* dy;           // backward only
  int64_t dy_stride;
  void* out;                // gather: rows; combine: y; backward: drows
  int64_t out_stride;
  float* dgate;             // backward only, or null
};
hipError_t launch_gather_rows(const RowsArgs& a, int32_t dtype, hipStream_t st);
hipError_t launch_combine_rows(const RowsArgs& a, int32_t dtype, int32_t y_dtype, hipStream_t st);
hipError_t launch_combine_rows_backward(const RowsArgs& a, int32_t dtype, int32_t dy_dtype, hipStream_t st);

// ---- adapters.hip ----
constexpr int32_t kAdapterMaxRank = 64;
struct AdapterArgs {
  int32_t n, rank, d_in, d_out, dtype, out_dtype, T;
  const void *A, *B;
  const float* scale;
  const void* x;      int64_t x_stride;
  const int32_t* ids;
  const void* dy;     int64_t dy_stride;      // backward
  const void* base;   int64_t base_stride;    // of y, or of dx in the backward pass; may be null
  void* out;          int64_t out_stride;     // y, or dx in the backward pass (null: not wanted)
  float *dA, *dB;                             // backward
  void* ws;
};
size_t adapter_ws_bytes(const AdapterArgs& a, bool backward);
hipError_t launch_adapters_forward(const AdapterArgs& a, hipStream_t st);
hipError_t launch_adapters_backward(const AdapterArgs& a, hipStream_t st);

// ---- distill.hip ----
constexpr int32_t kDistillMaxTop = 1024;
struct DistillArgs {
  const void* logits;  int64_t stride;
  int32_t dtype, T, V, K;
  const int32_t* top_idx;      // [T][K]
  const float* top_logits;     // [T][K]
  float temperature;
  const float* weight;         // [T] or null
  const float* lse_in;         // backward from saved sums
  const float* dloss;          // [T], backward from saved sums
  float *loss, *lse;
  void* dlogits;       int64_t dstride;
  void* ws;
};
size_t distill_ws_bytes(int32_t T, int32_t V, int32_t dtype);
hipError_t launch_distill_forward(const DistillArgs& a, hipStream_t st);
hipError_t launch_distill_backward(const DistillArgs& a, hipStream_t st);
hipError_t launch_distill_loss_grad(const DistillArgs& a, hipStream_t st);

#ifdef __HIPCC__
template <typename F>
inline auto with_type(int32_t dtype, F&& f) {
  if (dtype == MOEQ_BF16) return f(__bf16{});
  if (dtype == MOEQ_F16) return f(_Float16{});
  return f(float{});
}

// N consecutive elements at an address aligned to an element only: global memory takes any of them with wide accesses.
template <int N, typename T>
__device__ __forceinline__ void load_n(float (&v)[N], const T* p) {
  T t[N];
  __builtin_memcpy(t, p, sizeof(t));
#pragma unroll
  for (int i = 0; i < N; ++i) v[i] = (float)t[i];
}
template <int N, typename T>
__device__ __forceinline__ void store_n(T* p, const float (&v)[N]) {
  T t[N];
#pragma unroll
  for (int i = 0; i < N; ++i) t[i] = (T)v[i];      // (to nearest even)
  __builtin_memcpy(p, t, sizeof(t));
}
// 16 bytes that the kernel does not come back to. With the non-temporal hint they go to memory at once; without it they lie in the L2 of
// the XCD until the end of the kernel, which then waits for their way out (2048 bf16 rows of 4096 copied twice each: 16.1 / 9.5 us).
__device__ __forceinline__ void stream_out(void* p, const void* v) {
  typedef uint32_t words __attribute__((ext_vector_type(4)));
  typedef words anywhere __attribute__((aligned(2)));
  words w;
  __builtin_memcpy(&w, v, 16);
  __builtin_nontemporal_store(w, (anywhere*)p);
}
// N elements, in pieces of 16 bytes where they are as many.
template <int N, typename T>
__device__ __forceinline__ void stream_n(T* p, const float (&v)[N]) {
  if constexpr (N * sizeof(T) % 16 == 0) {
    T t[N];
#pragma unroll
    for (int i = 0; i < N; ++i) t[i] = (T)v[i];
#pragma unroll
    for (int i = 0; i < (int)(N * sizeof(T) / 16); ++i) stream_out((char*)p + 16 * i, (const char*)t + 16 * i);
  } else {
    store_n(p, v);
  }
}
#endif

}  // namespace moeq
