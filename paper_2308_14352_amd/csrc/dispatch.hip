// (Token, choice) pairs sorted by expert, the tokens' rows copied into that order, and expert rows combined back into tokens with
// the gradient of that. Pair i = token * k + choice; order[p] is the pair in place p, slot[i] the place of pair i; pairs without an
// expert (an index outside [0, E)) come last, as ~pair and ~place, have rows of zeros and add nothing.
#include <algorithm>
#include <type_traits>

#include "sort_core.h"

namespace moeq {
namespace {

// Pairs that one workgroup sorts alone; beyond, they go in chunks, and a kernel that counts goes ahead. us alone / in chunks:
// 4096 pairs of 8 experts 5.9 / 8.3, of 128 8.1 / 10.6; 6144 7.5 / 8.6 and 10.6 / 11.5; 8192 9.1 / 8.9 and 13.0 / 11.7; 32768 36 / 9.1.
constexpr int64_t kSortOne = 6144;
static_assert(kSortOne <= kSortKept);

__global__ __launch_bounds__(1024) void k_sort_one(const int32_t* __restrict__ idx, int pairs, int run, int E,
                                                   int32_t* __restrict__ offsets, int32_t* __restrict__ order, int32_t* __restrict__ slot) {
  __shared__ SortShared sh;
  __shared__ int place[kSortMaxExperts + 1];
  sort_pairs(idx, pairs, run, E, sh, [&](int e, int n) { place[e] = n; },
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

// Every workgroup adds up the counts of all chunks, which is quadratic in them, or a kernel ahead turns the counts into the pairs ahead of
// a chunk and writes the bins' totals behind them. us without / with it: 8 experts, 96 chunks 16.4 / 17.1, 128 18.0 / 16.9, 4096 1552 /
// 112; 64 experts, 64 chunks 18.8 / 18.9, 96 20.8 / 20.0; 256 experts, 16 chunks 19.5 / 20.8, 20 23.3 / 20.8, 4096 12371 / 188; 1024 experts, 6
// chunks 91 / 52, 2048 16734 / 221.
bool counts_scanned(int64_t chunks, int experts) { return chunks > 96 || chunks * (experts + 1) > 5000; }

__global__ __launch_bounds__(1024) void k_sort_scan(int32_t* __restrict__ counts, int chunks, int E) {
  __shared__ int sum[16][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, e = blockIdx.x * 64 + lane;
  const int span = (chunks + 15) / 16, a = wave * span, b = min(a + span, chunks);      // the wavefront's chunks; a bin a lane
  int32_t* at = counts + min(e, E);
  int n = 0;
#pragma unroll 8
  for (int c = a; c < b; ++c) n += at[(int64_t)c * (E + 1)];
  sum[wave][lane] = n;
  __syncthreads();
  int before = 0;
  for (int w = 0; w < wave; ++w) before += sum[w][lane];
  if (wave == 15 && e <= E) at[(int64_t)chunks * (E + 1)] = before + n;
  for (int c0 = a; c0 < b; c0 += 16) {
    int v[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] = at[(int64_t)min(c0 + i, b - 1) * (E + 1)];
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      if (c0 + i < b && e <= E) at[(int64_t)(c0 + i) * (E + 1)] = before;
      before += v[i];
    }
  }
}

template <bool SCANNED>
__global__ __launch_bounds__(1024) void k_sort_chunk(const int32_t* __restrict__ idx, int64_t pairs, int run, int E,
                                                     const int32_t* __restrict__ counts, int32_t* __restrict__ offsets,
                                                     int32_t* __restrict__ order, int32_t* __restrict__ slot) {
  __shared__ SortShared sh;
  __shared__ int place[kSortMaxExperts + 1], ahead[kSortMaxExperts + 1];
  const int chunks = gridDim.x, me = blockIdx.x;
  const int64_t a = me * kSortChunk;
  sort_pairs(idx + a, (int)min(kSortChunk, pairs - a), run, E, sh,
             [&](int e, int) {
               if constexpr (SCANNED) {
                 place[e] = counts[(int64_t)chunks * (E + 1) + e];
                 ahead[e] = counts[(int64_t)me * (E + 1) + e];
               } else {
                 place[e] = count_all(counts, chunks, me, E, e, ahead[e]);
               }
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

// ---- rows. Memory bounds all three: every row is read once and written once, the sums are registers of the thread that holds the
// piece. 2048 bf16 rows of 4096 to two places each: 9.3 us, 5.4 TB/s; 1117 tokens from two fp32 rows of 1024: 3.6 us; the gradient of
// 8192 tokens with two rows of 4096: 61 us, 5.5 TB/s (a large copy: 5.2).
// G threads take a token's row in pieces of VE elements, KB of its choices at a time. Loads stand in straight lines at
// addresses that exist (of dropped pairs: their place's, of entries that point nowhere: the first row's), so that they are on their way
// together; what they bring is not used then. A row's last piece, where the width is no multiple of VE, begins before its place and is
// read and written twice alike; rows shorter than a piece go element by element. ----
struct Choice { int place; bool row, kept; float gate; };      // row: has a place at all (entries come from the caller)

template <int KB>
__device__ __forceinline__ void take_choices(const RowsArgs& A, int t, int j0, Choice (&c)[KB]) {
  const int pairs = A.T * A.k;
#pragma unroll
  for (int j = 0; j < KB; ++j) {
    const int64_t i = (int64_t)t * A.k + min(j0 + j, A.k - 1);
    const int s = A.slot[i], place = s < 0 ? ~s : s;
    c[j].row = place < pairs && j0 + j < A.k;
    c[j].kept = s >= 0 && c[j].row;
    c[j].place = place < pairs ? place : 0;
    c[j].gate = A.gate ? A.gate[i] : 1.f;
  }
}
// The threads' pieces of a row of d elements: f(first element, elements) with compile-time VE where the row has as many.
template <int VE, int G, typename F>
__device__ __forceinline__ void for_pieces(int d, F&& f) {
  if (d >= VE) {
    for (int c = (threadIdx.x % G) * VE; c < d; c += G * VE) f(min(c, d - VE), std::integral_constant<int, VE>{}, min(c, d - VE) == c);
  } else {
    for (int c = threadIdx.x % G; c < d; c += G) f(c, std::integral_constant<int, 1>{}, true);
  }
}

template <typename T, int G, int KB>
__global__ __launch_bounds__(256) void k_gather_rows(RowsArgs A) {
  const int t = A.first + blockIdx.x * (256 / G) + threadIdx.x / G;
  if (t >= A.T) return;
  const T* x = (const T*)A.a + (int64_t)t * A.a_stride;
  for (int j0 = 0; j0 < A.k; j0 += KB) {
    Choice ch[KB];
    take_choices(A, t, j0, ch);
    // (two pieces on their way together: a thread has two or four of a wide row, and the whole call is one round of workgroups)
    constexpr int VE = 16 / sizeof(T);
    if (A.d >= VE) {
      for (int c = (threadIdx.x % G) * VE; c < A.d; c += 2 * G * VE) {
        T v[2][VE], z[VE] = {};
        const int at[2] = {min(c, A.d - VE), min(c + G * VE, A.d - VE)};
#pragma unroll
        for (int i = 0; i < 2; ++i) __builtin_memcpy(v[i], x + at[i], 16);
#pragma unroll
        for (int i = 0; i < 2; ++i)
          if (i == 0 || c + G * VE < A.d)
#pragma unroll
            for (int j = 0; j < KB; ++j)
              if (ch[j].row) stream_out((T*)A.out + (int64_t)ch[j].place * A.out_stride + at[i], ch[j].kept ? v[i] : z);
      }
    } else {
      for (int c = threadIdx.x % G; c < A.d; c += G)
#pragma unroll
        for (int j = 0; j < KB; ++j)
          if (ch[j].row) ((T*)A.out)[(int64_t)ch[j].place * A.out_stride + c] = ch[j].kept ? x[c] : (T)0.f;
    }
  }
}

// y[t] = sum of gate * row over the token's choices, in their order, in fp32.
template <typename T, typename Y, int G, int KB>
__global__ __launch_bounds__(256) void k_combine_rows(RowsArgs A) {
  const int t = A.first + blockIdx.x * (256 / G) + threadIdx.x / G;
  if (t >= A.T) return;
  Choice ch[KB];
  take_choices(A, t, 0, ch);
  for_pieces<16 / (sizeof(T) < sizeof(Y) ? sizeof(T) : sizeof(Y)), G>(A.d, [&](int c, auto size, bool) {
    constexpr int N = decltype(size)::value;
    float acc[N] = {};
    auto add = [&](const Choice (&ch)[KB]) {
      float v[KB][N];
#pragma unroll
      for (int j = 0; j < KB; ++j) load_n(v[j], (const T*)A.a + (int64_t)ch[j].place * A.a_stride + c);
#pragma unroll
      for (int j = 0; j < KB; ++j)
#pragma unroll
        for (int i = 0; i < N; ++i) acc[i] = ch[j].kept ? fmaf(ch[j].gate, v[j][i], acc[i]) : acc[i];
    };
    add(ch);
    for (int j0 = KB; j0 < A.k; j0 += KB) {
      Choice more[KB];
      take_choices(A, t, j0, more);
      add(more);
    }
    stream_n((Y*)A.out + (int64_t)t * A.out_stride + c, acc);
  });
}

// drows = gate * dy, dgate = dy . row, of all choices of a token.
template <typename T, typename Y, int G, int KB>
__global__ __launch_bounds__(256) void k_combine_grad(RowsArgs A) {
  __shared__ float part[4][KB];
  const int t = A.first + blockIdx.x * (256 / G) + threadIdx.x / G, me = threadIdx.x % G;
  if (t >= A.T) return;                       // (G = 256: the whole workgroup)
  const Y* dy = (const Y*)A.dy + (int64_t)t * A.dy_stride;
  for (int j0 = 0; j0 < A.k; j0 += KB) {
    Choice ch[KB];
    take_choices(A, t, j0, ch);
    float sum[KB] = {};
    for_pieces<16 / (sizeof(T) < sizeof(Y) ? sizeof(T) : sizeof(Y)), G>(A.d, [&](int c, auto size, bool whole) {
      constexpr int N = decltype(size)::value;
      float v[N], r[KB][N] = {};
      load_n(v, dy + c);
      if (A.dgate)
#pragma unroll
        for (int j = 0; j < KB; ++j) load_n(r[j], (const T*)A.a + (int64_t)ch[j].place * A.a_stride + c);
#pragma unroll
      for (int j = 0; j < KB; ++j) {
        float o[N];
        // (elements that the piece before has as well count once: those from the piece's own place on)
        const int first = whole ? 0 : N - A.d % N;
#pragma unroll
        for (int i = 0; i < N; ++i) {
          sum[j] = i >= first ? fmaf(v[i], r[j][i], sum[j]) : sum[j];
          o[i] = ch[j].kept ? ch[j].gate * v[i] : 0.f;
        }
        if (ch[j].row) stream_n((T*)A.out + (int64_t)ch[j].place * A.out_stride + c, o);
      }
    });
    if (!A.dgate) continue;
#pragma unroll
    for (int j = 0; j < KB; ++j)
#pragma unroll
      for (int m = 1; m < (G < 64 ? G : 64); m <<= 1) sum[j] += __shfl_xor(sum[j], m);
    if (G == 256) {
      __syncthreads();
      if (threadIdx.x % 64 == 0)
#pragma unroll
        for (int j = 0; j < KB; ++j) part[threadIdx.x / 64][j] = sum[j];
      __syncthreads();
#pragma unroll
      for (int j = 0; j < KB; ++j) sum[j] = (part[0][j] + part[1][j]) + (part[2][j] + part[3][j]);
    }
#pragma unroll
    for (int j = 0; j < KB; ++j)
      if (me == 0 && j0 + j < A.k) A.dgate[(int64_t)t * A.k + j0 + j] = ch[j].kept ? sum[j] : 0.f;
  }
}

// Threads of a token by its row's pieces of 16 bytes: 16 up to 16, 64 up to 128, 256 beyond. us of the gradient with the next larger
// group / this one / the next smaller: 8192 rows of 96 pieces 15.0 / 12.7 / -, of 256 - / 34.0 / 46.1; 2048 rows of 48 5.2 / 3.9 / 4.5.
// Choices at a time: all up to four.
template <typename F>
hipError_t by_width(int d, int k, int ve, F&& f) {
  const int pieces = (d + ve - 1) / ve;
  auto with_k = [&](auto g) {
    if (k == 1) return f(g, std::integral_constant<int, 1>{});
    if (k == 2) return f(g, std::integral_constant<int, 2>{});
    return f(g, std::integral_constant<int, 4>{});
  };
  if (pieces <= 16) return with_k(std::integral_constant<int, 16>{});
  if (pieces <= 128) return with_k(std::integral_constant<int, 64>{});
  return with_k(std::integral_constant<int, 256>{});
}

// The tokens of a call, `per` a workgroup of 256 threads: f(arguments, workgroups) for every launch.
template <typename F>
hipError_t in_launches(RowsArgs a, int per, F&& f) {
  for (a.first = 0; a.first < a.T;) {
    const int groups = std::min((a.T - a.first + per - 1) / per, launch_groups(256));
    f(a, groups);
    if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    a.first += groups * per;
  }
  return hipSuccess;
}

}  // namespace

size_t sort_ws_bytes(int64_t pairs, int32_t experts) {
  if (pairs <= kSortOne) return 0;
  const int64_t chunks = (pairs + kSortChunk - 1) / kSortChunk;
  return (size_t)(chunks + counts_scanned(chunks, experts)) * (size_t)(experts + 1) * 4;
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
  if (counts_scanned(chunks, experts)) {
    hipLaunchKernelGGL(k_sort_scan, dim3(experts / 64 + 1), dim3(1024), 0, st, (int32_t*)ws, chunks, experts);
    if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    hipLaunchKernelGGL(k_sort_chunk<true>, dim3(chunks), dim3(waves * 64), 0, st, idx, pairs, run, experts, (const int32_t*)ws, offsets, order, slot);
  } else {
    hipLaunchKernelGGL(k_sort_chunk<false>, dim3(chunks), dim3(waves * 64), 0, st, idx, pairs, run, experts, (const int32_t*)ws, offsets, order, slot);
  }
  return hipGetLastError();
}

hipError_t launch_gather_rows(const RowsArgs& a, int32_t dtype, hipStream_t st) {
  return with_type(dtype, [&](auto tag) {
    using T = decltype(tag);
    return by_width(a.d, a.k, 16 / sizeof(T), [&](auto g, auto kb) {
      constexpr int G = decltype(g)::value, KB = decltype(kb)::value;
      return in_launches(a, 256 / G, [&](const RowsArgs& b, int groups) {
        hipLaunchKernelGGL((k_gather_rows<T, G, KB>), dim3(groups), dim3(256), 0, st, b);
      });
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
    return by_width(a.d, a.k, 16 / sizeof(T), [&](auto g, auto kb) {
      constexpr int G = decltype(g)::value, KB = decltype(kb)::value;
      return in_launches(a, 256 / G, [&](const RowsArgs& b, int groups) {
        hipLaunchKernelGGL((k_combine_rows<T, Y, G, KB>), dim3(groups), dim3(256), 0, st, b);
      });
    });
  });
}

hipError_t launch_combine_rows_backward(const RowsArgs& a, int32_t dtype, int32_t dy_dtype, hipStream_t st) {
  return with_types(dtype, dy_dtype, [&](auto tag, auto ytag) {
    using T = decltype(tag);
    using Y = decltype(ytag);
    return by_width(a.d, a.k, 16 / sizeof(T), [&](auto g, auto kb) {
      constexpr int G = decltype(g)::value, KB = decltype(kb)::value;
      return in_launches(a, 256 / G, [&](const RowsArgs& b, int groups) {
        hipLaunchKernelGGL((k_combine_grad<T, Y, G, KB>), dim3(groups), dim3(256), 0, st, b);
      });
    });
  });
}

}  // namespace moeq
