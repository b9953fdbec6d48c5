// The stable counting sort of indices into a range, by a workgroup: shared by the pairs of a routing (dispatch.hip) and the rows of
// adapters (adapters.hip). In an unnamed namespace: each translation unit gets its own copy.
#pragma once
#include "operators.h"

namespace moeq {
namespace {

// A wavefront owns a run of consecutive pairs, so a pair's place is the sum of: the pairs of smaller bins, those of its bin in the
// runs before, and those before it in the run (64 at a time, by ballots on the bits of the bin). All counts are integers, so the
// order never depends on timing. The run is gone through twice by the same loop, once to count and once to place: what a launch
// executes once costs some 200 cycles per 64 bytes of code, so that loops unrolled to keep what was counted in registers took longer.
// A pair's number in its run and bin is kept in LDS for the second time.
constexpr int kSortKept = 8192;          // pairs of a workgroup, at most
struct SortShared {
  int cnt[4112];                         // 16 wavefronts x 257 bins, 8 x 513 or 4 x 1025
  uint16_t number[kSortKept];
};

inline int sort_waves(int64_t pairs, int32_t experts) {
  const int most = experts <= 256 ? 16 : experts <= 512 ? 8 : 4;
  const int64_t need = (pairs + 63) / 64;
  return need < 1 ? 1 : need < most ? (int)need : most;
}

__device__ __forceinline__ int bin_of(int e, int E) { return (uint32_t)e < (uint32_t)E ? e : E; }

// The sum of the lanes up to this one, within rows of 16 and beyond, by moves between lanes that are part of the addition (through LDS
// a step is some 100 cycles).
template <int CTRL, int ROWS>
__device__ __forceinline__ int add_from(int v) { return v + __builtin_amdgcn_update_dpp(0, v, CTRL, ROWS, 0xf, false); }
__device__ __forceinline__ int row_sum_to(int v) {
  v = add_from<0x111, 0xf>(v);
  v = add_from<0x112, 0xf>(v);
  v = add_from<0x114, 0xf>(v);
  return add_from<0x118, 0xf>(v);
}
__device__ __forceinline__ int wave_sum_to(int v) {
  v = row_sum_to(v);
  v = add_from<0x142, 0xa>(v);        // the last lane of rows 0 and 2 to rows 1 and 3
  return add_from<0x143, 0xc>(v);     // lane 31 to rows 2 and 3
}

// v[bin] = the sum of the values before it, by the calling wavefront.
__device__ __forceinline__ void sort_scan(int E, int* v) {
  const int lane = threadIdx.x & 63;
  int before = 0;
  for (int e0 = 0; e0 <= E; e0 += 64) {
    const int e = e0 + lane, n = e <= E ? v[e] : 0, at = wave_sum_to(n);
    if (e <= E) v[e] = before + at - n;
    before += __builtin_amdgcn_readlane(at, 63);
  }
}

// The pairs idx[0, n) of a workgroup, n <= kSortKept, `run` of them a wavefront. After counting, totals(bin, count) is called for every bin by one
// thread, then starts() by all (with barriers before and behind), then put(pair, number, bin) for every pair with its number in the bin.
template <typename Totals, typename Starts, typename Put>
__device__ __forceinline__ void sort_pairs(const int32_t* idx, int n, int run, int E, SortShared& sh, Totals&& totals, Starts&& starts, Put&& put) {
  const int waves = blockDim.x >> 6, wave = threadIdx.x >> 6, lane = threadIdx.x & 63, bits = 32 - __builtin_clz(E);
  const int a = wave * run, b = min(a + run, n);
  int *cnt = sh.cnt, *mine = cnt + wave * (E + 1);
  constexpr int kNext = 4;                      // 64 pairs that are on their way ahead of those worked on
  int next[kNext];
  auto request = [&](int i) { return idx[min(i + lane, n - 1)]; };
  if (a < b)
#pragma unroll
    for (int j = 0; j < kNext; ++j) next[j] = request(a + 64 * j);
  for (int i = threadIdx.x; i < waves * (E + 1); i += blockDim.x) cnt[i] = 0;
  __syncthreads();
  for (int placing = 0;; ++placing) {
    for (int i0 = a; i0 < b; i0 += 64) {
      const int i = i0 + lane, key = bin_of(next[0], E);
      const bool in = i < b;
#pragma unroll
      for (int j = 0; j + 1 < kNext; ++j) next[j] = next[j + 1];
      next[kNext - 1] = request(i0 + 64 * kNext);
      if (placing) {
        if (in) put(i, mine[key] + sh.number[i], key);
        continue;
      }
      // the lanes that hold the same bin; runs of one bin, as sorted ids have them, are seen at once
      uint64_t same = __ballot(in);
      if (__ballot(in && key != __builtin_amdgcn_readfirstlane(key)))
        for (int j = 0; j < bits; ++j) {
          const int one = __builtin_amdgcn_sbfe(key, j, 1);              // 0 or -1
          const uint64_t m = __ballot(one);
          same &= ~(m ^ (uint64_t)(int64_t)one);
        }
      if (in) {
        const int rank = __popcll(same & ((1ull << lane) - 1)), at = mine[key] + rank;
        __builtin_amdgcn_wave_barrier();                 // every lane has read before the first of the bin counts on
        if (rank == 0) mine[key] = at + __popcll(same);
        sh.number[i] = (uint16_t)at;
      }
      __builtin_amdgcn_wave_barrier();
    }
    if (placing) return;
    if (a < b)
#pragma unroll
      for (int j = 0; j < kNext; ++j) next[j] = request(a + 64 * j);
    __syncthreads();
    // 16 lanes take the counts of a bin (of one wavefront: a lane), which become the numbers of the wavefronts' first pairs in it
    const int shift = waves > 1 ? 4 : 0;
    for (int i = threadIdx.x; i < (E + 1) << shift; i += blockDim.x) {
      const int w = shift ? i & 15 : 0, e = i >> shift, c = w < waves ? cnt[w * (E + 1) + e] : 0;
      const int at = shift ? row_sum_to(c) : c;
      if (w < waves) cnt[w * (E + 1) + e] = at - c;
      if (w == (1 << shift) - 1) totals(e, at);
    }
    __syncthreads();
    starts();
    __syncthreads();
  }
}

// Sorts of several workgroups: a chunk's pairs of every bin (counts [chunks][E + 1]), and from those, a bin's pairs in all chunks and in
// the ones ahead of `me`.
constexpr int64_t kSortChunk = 4096;     // pairs
static_assert(kSortChunk <= kSortKept);
__global__ __launch_bounds__(1024) void k_sort_count(const int32_t* __restrict__ idx, int64_t pairs, int E, int32_t* __restrict__ counts) {
  __shared__ int cnt[kSortMaxExperts + 1];
  for (int e = threadIdx.x; e <= E; e += blockDim.x) cnt[e] = 0;
  __syncthreads();
  const int64_t a = blockIdx.x * kSortChunk, b = min(a + kSortChunk, pairs);
  for (int64_t i = a + threadIdx.x; i < b; i += blockDim.x) atomicAdd(&cnt[bin_of(idx[i], E)], 1);
  __syncthreads();
  for (int e = threadIdx.x; e <= E; e += blockDim.x) counts[(int64_t)blockIdx.x * (E + 1) + e] = cnt[e];
}

__device__ __forceinline__ int count_all(const int32_t* __restrict__ counts, int chunks, int me, int E, int e, int& ahead) {
  int before = 0, all = 0;
#pragma unroll 8
  for (int c = 0; c < chunks; ++c) {
    const int v = counts[(int64_t)c * (E + 1) + e];
    before += c < me ? v : 0;
    all += v;
  }
  ahead = before;
  return all;
}

}  // namespace
}  // namespace moeq
