// (Token, choice) pairs sorted by expert, the tokens' rows copied into that order, and expert rows combined back into tokens with
// the gradient of that. Pair i = token * k + choice; order[p] is the pair in place p, slot[i] the place of pair i; pairs without an
// expert (an index outside [0, E)) come last, as ~pair and ~place, have rows of zeros and add nothing.
#include <type_traits>

#include "sort_core.h"

namespace moeq {
namespace {

constexpr int64_t kSortOne = 16384;      // pairs that one workgroup sorts alone
constexpr int64_t kSortChunk = 4096;     // pairs of a workgroup beyond

__global__ __launch_bounds__(1024) void k_sort_one(const int32_t* __restrict__ idx, int pairs, int run, int E,
                                                   int32_t* __restrict__ offsets, int32_t* __restrict__ order, int32_t* __restrict__ slot) {
  __shared__ int cnt[kSortCounts], place[kSortMaxExperts + 1];
  sort_pairs(idx, pairs, run, E, cnt, [&](int e, int n) { place[e] = n; },
             [&] {
               if (threadIdx.x < 64) {
                 sort_scan(E, place);
                 for (int e = threadIdx.x; e <= E; e += 64) offsets[e] = place[e];
               }
             },
             [&](int i, int number, int e) {
               const int p = place[e] + number;
               order[p] = e < E ? i : ~i;
               slot[i] = e < E ? p : ~p;
             });
}

__global__ __launch_bounds__(1024) void k_sort_count(const int32_t* __restrict__ idx, int64_t pairs, int E, int32_t* __restrict__ counts) {
  __shared__ int cnt[kSortMaxExperts + 1];
  for (int e = threadIdx.x; e <= E; e += blockDim.x) cnt[e] = 0;
  __syncthreads();
  const int64_t a = blockIdx.x * kSortChunk, b = min(a + kSortChunk, pairs);
  for (int64_t i = a + threadIdx.x; i < b; i += blockDim.x) atomicAdd(&cnt[bin_of(idx[i], E)], 1);
  __syncthreads();
  for (int e = threadIdx.x; e <= E; e += blockDim.x) counts[(int64_t)blockIdx.x * (E + 1) + e] = cnt[e];
}

__global__ __launch_bounds__(1024) void k_sort_chunk(const int32_t* __restrict__ idx, int64_t pairs, int run, int E,
                                                     const int32_t* __restrict__ counts, int32_t* __restrict__ offsets,
                                                     int32_t* __restrict__ order, int32_t* __restrict__ slot) {
  __shared__ int cnt[kSortCounts], place[kSortMaxExperts + 1], ahead[kSortMaxExperts + 1];
  const int chunks = gridDim.x, me = blockIdx.x;
  const int64_t a = me * kSortChunk;
  sort_pairs(idx + a, (int)min(kSortChunk, pairs - a), run, E, cnt,
             [&](int e, int) {
               int before = 0, all = 0;
#pragma unroll 8
               for (int c = 0; c < chunks; ++c) {
                 const int v = counts[(int64_t)c * (E + 1) + e];
                 before += c < me ? v : 0;
                 all += v;
               }
               place[e] = all;
               ahead[e] = before;
             },
             [&] {
               if (threadIdx.x < 64) {
                 sort_scan(E, place);
                 for (int e = threadIdx.x; e <= E; e += 64) {
                   if (me == 0) offsets[e] = place[e];
                   ahead[e] += place[e];
                 }
               }
             },
             [&](int i, int number, int e) {
               const int p = ahead[e] + number, pair = (int)a + i;
               order[p] = e < E ? pair : ~pair;
               slot[pair] = e < E ? p : ~p;
             });
}

// ---- rows. G threads take a token's row in pieces of VE elements.
__device__ __forceinline__ int place_of(int s, int pairs) { return s < 0 ? ~s : s; }
// Whether an entry of slot points to a row at all (entries come from the caller).
__device__ __forceinline__ bool has_row(int s, int pairs) { return (uint32_t)place_of(s, pairs) < (uint32_t)pairs; }

template <typename T, int G>
__global__ __launch_bounds__(256) void k_gather_rows(RowsArgs A) {
  constexpr int VE = 16 / sizeof(T);
  const int t = blockIdx.x * (256 / G) + threadIdx.x / G;
  if (t >= A.T) return;
  const T* x = (const T*)A.a + (int64_t)t * A.a_stride;
  for (int c = (threadIdx.x % G) * VE; c < A.d; c += G * VE) {
    const int n = min(VE, A.d - c);
    float v[VE], z[VE] = {};
    load_some(v, x + c, n);
    for (int j = 0; j < A.k; ++j) {
      const int s = A.slot[(int64_t)t * A.k + j];
      if (!has_row(s, A.T * A.k)) continue;
      T* to = (T*)A.out + (int64_t)place_of(s, 0) * A.out_stride + c;
      store_some(to, s >= 0 ? v : z, n);
    }
  }
}

// y[t] = sum of gate * row over the token's choices, in their order, in fp32.
template <typename T, typename Y, int G>
__global__ __launch_bounds__(256) void k_combine_rows(RowsArgs A) {
  constexpr int VE = 16 / (sizeof(T) < sizeof(Y) ? sizeof(T) : sizeof(Y));
  const int t = blockIdx.x * (256 / G) + threadIdx.x / G;
  if (t >= A.T) return;
  const int64_t i0 = (int64_t)t * A.k;
  for (int c = (threadIdx.x % G) * VE; c < A.d; c += G * VE) {
    const int n = min(VE, A.d - c);
    float acc[VE] = {};
    for (int j = 0; j < A.k; ++j) {
      const int s = A.slot[i0 + j];
      if (s < 0 || !has_row(s, A.T * A.k)) continue;
      const float g = A.gate ? A.gate[i0 + j] : 1.f;
      float v[VE];
      load_some(v, (const T*)A.a + (int64_t)s * A.a_stride + c, n);
#pragma unroll
      for (int i = 0; i < VE; ++i) acc[i] = fmaf(g, v[i], acc[i]);
    }
    store_some((Y*)A.out + (int64_t)t * A.out_stride + c, acc, n);
  }
}

// drows = gate * dy, dgate = dy . row, of all choices of a token.
template <typename T, typename Y, int G>
__global__ __launch_bounds__(256) void k_combine_grad(RowsArgs A) {
  constexpr int VE = 16 / (sizeof(T) < sizeof(Y) ? sizeof(T) : sizeof(Y));
  __shared__ float part[4];
  const int t = blockIdx.x * (256 / G) + threadIdx.x / G, me = threadIdx.x % G;
  if (t >= A.T) return;
  const Y* dy = (const Y*)A.dy + (int64_t)t * A.dy_stride;
  for (int j = 0; j < A.k; ++j) {
    const int64_t i = (int64_t)t * A.k + j;
    const int s = A.slot[i];
    const bool row = has_row(s, A.T * A.k), kept = row && s >= 0;
    const float g = !kept ? 0.f : A.gate ? A.gate[i] : 1.f;
    float sum = 0.f;
    if (row)
      for (int c = me * VE; c < A.d; c += G * VE) {
        const int n = min(VE, A.d - c);
        float v[VE] = {}, r[VE], o[VE] = {};
        if (kept) {
          load_some(v, dy + c, n);
          if (A.dgate) {
            load_some(r, (const T*)A.a + (int64_t)s * A.a_stride + c, n);
#pragma unroll
            for (int e = 0; e < VE; ++e) sum = fmaf(v[e], r[e], sum);
          }
#pragma unroll
          for (int e = 0; e < VE; ++e) o[e] = g * v[e];
        }
        store_some((T*)A.out + (int64_t)place_of(s, 0) * A.out_stride + c, o, n);
      }
    if (!A.dgate) continue;
#pragma unroll
    for (int m = 1; m < (G < 64 ? G : 64); m <<= 1) sum += __shfl_xor(sum, m);
    if (G == 256) {
      if (threadIdx.x % 64 == 0) part[threadIdx.x / 64] = sum;
      __syncthreads();
      sum = (part[0] + part[1]) + (part[2] + part[3]);
      __syncthreads();
    }
    if (me == 0) A.dgate[i] = kept ? sum : 0.f;
  }
}

// Threads of a token: as many as its row has pieces of 16 bytes, as far as there are such groups.
template <typename F>
hipError_t by_width(int d, int ve, F&& f) {
  const int pieces = (d + ve - 1) / ve;
  if (pieces <= 16) return f(std::integral_constant<int, 16>{});
  if (pieces <= 128) return f(std::integral_constant<int, 64>{});
  return f(std::integral_constant<int, 256>{});
}

}  // namespace

size_t sort_ws_bytes(int64_t pairs, int32_t experts) {
  return pairs <= kSortOne ? 0 : (size_t)((pairs + kSortChunk - 1) / kSortChunk) * (size_t)(experts + 1) * 4;
}

hipError_t launch_sort_pairs(const int32_t* idx, int64_t pairs, int32_t experts, int32_t* offsets, int32_t* order, int32_t* slot,
                             void* ws, hipStream_t st) {
  const bool one = pairs <= kSortOne;
  const int64_t span = one ? pairs : kSortChunk;
  const int waves = sort_waves(span, experts);
  const int run = (int)((span + waves * 64 - 1) / (waves * 64) * 64);
  if (one) {
    hipLaunchKernelGGL(k_sort_one, dim3(1), dim3(waves * 64), 0, st, idx, (int)pairs, run, experts, offsets, order, slot);
    return hipGetLastError();
  }
  const int chunks = (int)((pairs + kSortChunk - 1) / kSortChunk);
  hipLaunchKernelGGL(k_sort_count, dim3(chunks), dim3(1024), 0, st, idx, pairs, experts, (int32_t*)ws);
  if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  hipLaunchKernelGGL(k_sort_chunk, dim3(chunks), dim3(waves * 64), 0, st, idx, pairs, run, experts, (const int32_t*)ws, offsets, order, slot);
  return hipGetLastError();
}

hipError_t launch_gather_rows(const RowsArgs& a, int32_t dtype, hipStream_t st) {
  return with_type(dtype, [&](auto tag) {
    using T = decltype(tag);
    return by_width(a.d, 16 / sizeof(T), [&](auto g) {
      constexpr int G = decltype(g)::value;
      hipLaunchKernelGGL((k_gather_rows<T, G>), dim3((a.T + 256 / G - 1) / (256 / G)), dim3(256), 0, st, a);
      return hipGetLastError();
    });
  });
}

// T x Y: the rows' type with itself, or with fp32 tokens.
template <typename F>
static hipError_t with_types(int32_t dtype, int32_t y_dtype, F&& f) {
  return with_type(dtype, [&](auto tag) {
    return y_dtype == MOEQ_F32 ? f(tag, float{}) : f(tag, tag);
  });
}

hipError_t launch_combine_rows(const RowsArgs& a, int32_t dtype, int32_t y_dtype, hipStream_t st) {
  return with_types(dtype, y_dtype, [&](auto tag, auto ytag) {
    using T = decltype(tag);
    using Y = decltype(ytag);
    return by_width(a.d, 16 / sizeof(T), [&](auto g) {
      constexpr int G = decltype(g)::value;
      hipLaunchKernelGGL((k_combine_rows<T, Y, G>), dim3((a.T + 256 / G - 1) / (256 / G)), dim3(256), 0, st, a);
      return hipGetLastError();
    });
  });
}

hipError_t launch_combine_rows_backward(const RowsArgs& a, int32_t dtype, int32_t dy_dtype, hipStream_t st) {
  return with_types(dtype, dy_dtype, [&](auto tag, auto ytag) {
    using T = decltype(tag);
    using Y = decltype(ytag);
    return by_width(a.d, 16 / sizeof(T), [&](auto g) {
      constexpr int G = decltype(g)::value;
      hipLaunchKernelGGL((k_combine_grad<T, Y, G>), dim3((a.T + 256 / G - 1) / (256 / G)), dim3(256), 0, st, a);
      return hipGetLastError();
    });
  });
}

}  // namespace moeq
