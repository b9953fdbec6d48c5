// The stable counting sort of indices into a range, by a workgroup: shared by the pairs of a routing (dispatch.hip) and the rows of
// adapters (adapters.hip). In an unnamed namespace: each translation unit gets its own copy.
#pragma once
#include "operators.h"

namespace moeq {
namespace {

// ---- the sort: stable, by counting. A wavefront owns a run of consecutive pairs, so a pair's place is the sum of: the pairs of
// smaller experts, those of its expert in the runs before, and those before it in the run (64 at a time, by ballots on the bits of
// the expert). All counts are integers, so the order never depends on timing.
constexpr int kSortCounts = 8208;        // counters in LDS: 16 wavefronts x 513 bins or 8 x 1025

inline int sort_waves(int64_t pairs, int32_t experts) {
  const int most = experts <= 512 ? 16 : 8;
  const int64_t need = (pairs + 63) / 64;
  return need < 1 ? 1 : need < most ? (int)need : most;
}

__device__ __forceinline__ int key_of(const int32_t* idx, int64_t i, int E) {
  const int e = idx[i];
  return (uint32_t)e < (uint32_t)E ? e : E;
}

// Counts of this workgroup's pairs [first, last) into cnt[wave][bin].
__device__ __forceinline__ void sort_count(const int32_t* idx, int64_t first, int64_t last, int64_t run, int E, int* cnt) {
  const int waves = blockDim.x >> 6, wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  for (int i = threadIdx.x; i < waves * (E + 1); i += blockDim.x) cnt[i] = 0;
  __syncthreads();
  const int64_t a = first + wave * run, b = min(a + run, last);
  for (int64_t i = a + lane; i < b; i += 64) atomicAdd(&cnt[wave * (E + 1) + key_of(idx, i, E)], 1);
  __syncthreads();
}

// cnt[wave][bin] becomes the place of the wavefront's next pair of that bin: place[bin] + the counts of the wavefronts before.
// put(pair, place, bin) takes them.
template <typename Put>
__device__ __forceinline__ void sort_place(const int32_t* idx, int64_t first, int64_t last, int64_t run, int E, const int* place,
                                           int* cnt, Put&& put) {
  const int waves = blockDim.x >> 6, wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  for (int e = threadIdx.x; e <= E; e += blockDim.x) {
    int at = place[e];
    for (int w = 0; w < waves; ++w) {
      const int n = cnt[w * (E + 1) + e];
      cnt[w * (E + 1) + e] = at;
      at += n;
    }
  }
  __syncthreads();
  const int bits = 32 - __builtin_clz(E);
  const int64_t a = first + wave * run, b = min(a + run, last);
  for (int64_t i0 = a; i0 < b; i0 += 64) {
    const int64_t i = i0 + lane;
    const bool in = i < b;
    const int key = in ? key_of(idx, i, E) : 0;
    uint64_t same = __ballot(in);
    for (int j = 0; j < bits; ++j) {
      const bool one = (key >> j) & 1;
      const uint64_t m = __ballot(one);
      same &= one ? m : ~m;
    }
    if (in) {
      const int rank = __popcll(same & ((1ull << lane) - 1));
      int* next = &cnt[wave * (E + 1) + key];
      const int p = *next + rank;
      __builtin_amdgcn_wave_barrier();                 // every lane has read before the first of the bin counts on
      if (rank == 0) *next = p + __popcll(same);
      put((int)i, p, key);
    }
    __builtin_amdgcn_wave_barrier();
  }
}

// Counts of all wavefronts together.
__device__ __forceinline__ int sort_total(const int* cnt, int E, int e) {
  const int waves = blockDim.x >> 6;
  int n = 0;
  for (int w = 0; w < waves; ++w) n += cnt[w * (E + 1) + e];
  return n;
}

// place[bin] = the sum of the totals before it; by the first wavefront.
__device__ __forceinline__ void sort_scan(int E, int* place) {
  if (threadIdx.x < 64) {
    const int lane = threadIdx.x, per = (E + 1 + 63) / 64, a = lane * per, b = min(a + per, E + 1);
    int sum = 0;
    for (int e = a; e < b; ++e) sum += place[e];
    int before = sum;
    for (int s = 1; s < 64; s <<= 1) {
      const int v = __shfl_up(before, s);
      if (lane >= s) before += v;
    }
    before -= sum;
    for (int e = a; e < b; ++e) {
      const int n = place[e];
      place[e] = before;
      before += n;
    }
  }
  __syncthreads();
}

}  // namespace
}  // namespace moeq
