// Distillation from a teacher's top logits. Of a row with student logits z [V], teacher logits u at K indices, temperature tau and
// weight w: s = z / tau, q = softmax(s), p = softmax(u / tau) over the entries that have an index,
//   loss = w tau^2 sum_j p_j (log p_j - s[idx_j] + lse(s)),   dloss/dz = w tau (q - p at the indices).
// A row of weight 0, or without a teacher's entry, has no loss and no gradient.
//
// One pass over a row: it is held in registers (up to 256 KB) between the maximum, the sum and the gradient, every thread with a maximum
// and a sum of its own that are joined once. Longer rows, and calls of few rows, are cut into chunks of a workgroup each: a kernel writes
// every chunk's maximum and sum, and the next joins them and goes on (the second reading of a row comes from the cache where it fits).
// Memory bounds it: 4096 rows of 32000 bf16 logits to loss and gradient 105 us, 5.0 TB/s of one reading and one writing; the gradient of
// 1000 rows of 50257 fp16 logits, a fifth of them masked, 33.4 us, 5.4 TB/s; the losses of 2048 bf16 rows of 32000 26 us, 5.0 TB/s. Few
// rows are latency: 13 of 131072 fp32 logits take 4.7 us for the chunks and 3.8 for their join (the teacher's entries, one wavefront).
// Differences z - max are taken before the scaling, so that where the row's maximum is known (the loss, and the gradient that comes with
// it) a probability's error does not grow with the size of the logits. The gradient from a saved log-sum-exp takes that for the origin, an
// fp32 number, for which a probability is off by some 2^-23 |lse|: beyond kFarLse the row's maximum and sum are taken again. The gradient is
// written without the teacher's part first; its K elements are written again behind a barrier.
#include <algorithm>
#include <type_traits>

#include "operators.h"

namespace moeq {
namespace {

constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;

// ---- folds over a wavefront, by moves between lanes that are part of the operation ----
template <int CTRL, int ROWS>
__device__ __forceinline__ float from_lane(float v, float none) {
  return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(__builtin_bit_cast(int, none), __builtin_bit_cast(int, v), CTRL, ROWS, 0xf, false));
}
template <typename Op>
__device__ __forceinline__ float fold(float v, float none, Op op) {
  v = op(v, from_lane<0x111, 0xf>(v, none));
  v = op(v, from_lane<0x112, 0xf>(v, none));
  v = op(v, from_lane<0x114, 0xf>(v, none));
  v = op(v, from_lane<0x118, 0xf>(v, none));
  v = op(v, from_lane<0x142, 0xa>(v, none));      // the last lane of rows 0 and 2 to rows 1 and 3
  v = op(v, from_lane<0x143, 0xc>(v, none));      // lane 31 to rows 2 and 3
  return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), 63));
}
__device__ __forceinline__ float wave_max(float v) { return fold(v, -INFINITY, [](float a, float b) { return fmaxf(a, b); }); }
__device__ __forceinline__ float wave_sum(float v) { return fold(v, 0.f, [](float a, float b) { return a + b; }); }

// A maximum of logits and the sum of exp2((z - max) c) that belongs to it; minus infinity counts from 0.
struct Stat { float m, s; };
__device__ __forceinline__ float origin(float m) { return m == -INFINITY ? 0.f : m; }
// The sum from another maximum on. That of nothing but minus infinities is 0 (NaNs: NaN) from any: not times exp2 of how far 0 is above m.
__device__ __forceinline__ float rescale(Stat a, float m, float c) {
  return a.m == -INFINITY ? a.s : a.s * __builtin_amdgcn_exp2f((a.m - m) * c);
}

// ---- a row as vectors of 16 bytes that lie on a multiple of 16 in the gradient (in the logits, where there is none), with single
// elements before the first and behind the last: rows of an odd length begin anywhere, and a store across two lines is two of them ----
template <typename T>
struct Span {
  static constexpr int VE = 16 / sizeof(T);
  int V, head, n;        // elements, those before the first vector, vectors
  __device__ __forceinline__ Span(const T* at, int V) : V(V) {
    head = min((int)(-(uintptr_t)at % 16 / sizeof(T)), V);
    n = (V - head) / VE;
  }
  __device__ __forceinline__ int singles() const { return V - n * VE; }
  __device__ __forceinline__ int single(int i) const { return i < head ? i : i + n * VE; }      // element of the i-th single one
};

// ---- a piece of a row in registers: vectors of 16 bytes, v = thread + i threads ----
template <typename T, int NV>
struct Held {
  static constexpr int VE = 16 / sizeof(T);
  struct Words { uint32_t w[4]; } raw[NV];
  __device__ __forceinline__ void load(const T* z, int n, int threads) {      // n: vectors, at least one
#pragma unroll
    for (int i = 0; i < NV; ++i) __builtin_memcpy(raw[i].w, z + (int64_t)min((int)threadIdx.x + i * threads, n - 1) * VE, 16);
  }
  // As fp32, anew every time: kept from one use to the next the values would take twice the registers of 16-bit logits.
  __device__ __forceinline__ void get(int i, float (&v)[VE]) const {
    Words r = raw[i];
    if constexpr (sizeof(T) == 2) {
#pragma unroll
      for (int e = 0; e < 4; ++e) asm volatile("" : "+v"(r.w[e]));
    }
    T t[VE];
    __builtin_memcpy(t, r.w, 16);
#pragma unroll
    for (int e = 0; e < VE; ++e) v[e] = (float)t[e];
  }
};

// The statistics of a workgroup's piece: n vectors in `held` and `rest` single elements behind them (`last` for the threads below).
template <typename T, int NV>
__device__ __forceinline__ Stat piece_stat(const Held<T, NV>& held, int n, int threads, bool rest, float last, float c, Stat* sh) {
  constexpr int VE = Held<T, NV>::VE;
  Stat a{-INFINITY, 0.f};
#pragma unroll
  for (int i = 0; i < NV; ++i)
    if ((int)threadIdx.x + i * threads < n) {
      float v[VE];
      held.get(i, v);
#pragma unroll
      for (int e = 0; e < VE; ++e) a.m = fmaxf(a.m, v[e]);
    }
  if (rest) a.m = fmaxf(a.m, last);
  const float m = wave_max(a.m), o = origin(m);      // (one maximum a wavefront: no thread rescales)
#pragma unroll
  for (int i = 0; i < NV; ++i)
    if ((int)threadIdx.x + i * threads < n) {
      float v[VE];
      held.get(i, v);
#pragma unroll
      for (int e = 0; e < VE; ++e) a.s += __builtin_amdgcn_exp2f((v[e] - o) * c);
    }
  if (rest) a.s += __builtin_amdgcn_exp2f((last - o) * c);
  a.s = wave_sum(a.s);
  if (threadIdx.x % 64 == 0) sh[threadIdx.x / 64] = Stat{m, a.s};
  __syncthreads();
  Stat all{-INFINITY, 0.f};
  for (int w = 0; w < threads / 64; ++w) all.m = fmaxf(all.m, sh[w].m);
  for (int w = 0; w < threads / 64; ++w) all.s += rescale(sh[w], all.m, c);
  return all;
}
// Several pieces' statistics as one, by a wavefront.
__device__ __forceinline__ Stat join(const Stat* part, int n, float c) {
  float m = -INFINITY, s = 0.f;
  for (int i = threadIdx.x % 64; i < n; i += 64) m = fmaxf(m, part[i].m);
  m = wave_max(m);
  for (int i = threadIdx.x % 64; i < n; i += 64) s += rescale(part[i], m, c);
  return Stat{m, wave_sum(s)};
}

// ---- the teacher's entries of a row, in LDS: index (-1: none), probability, logit of the student ----
struct Teacher {
  int idx[kDistillMaxTop];
  float p[kDistillMaxTop], z[kDistillMaxTop];
  bool any;
};
// By the first wavefront (a barrier has to follow). Returns sum of p log p, in all its lanes. A row has a teacher where an entry is not
// minus infinity; a NaN or plus infinity among them makes every p a NaN, which goes into both sums (only p = 0 is left out of them).
template <typename T>
__device__ __forceinline__ float take_teacher(const DistillArgs& A, int t, const T* z, Teacher& sh) {
  const int lane = threadIdx.x & 63;
  const float it = 1.f / A.temperature;
  const int32_t* idx = A.top_idx + (int64_t)t * A.K;
  const float* u = A.top_logits + (int64_t)t * A.K;
  float top = -INFINITY, sum = 0.f, plogp = 0.f;
  for (int j = lane; j < A.K; j += 64) {
    const int i = idx[j];
    const bool ok = (uint32_t)i < (uint32_t)A.V;
    sh.idx[j] = ok ? i : -1;
    sh.p[j] = ok ? u[j] : -INFINITY;
    sh.z[j] = ok ? (float)z[i] : 0.f;
    top = ok ? fmaxf(top, u[j]) : top;
  }
  top = wave_max(top);
  const float o = origin(top);
  for (int j = lane; j < A.K; j += 64) {
    const float e = __builtin_amdgcn_exp2f((sh.p[j] - o) * it * kLog2e);
    sum += e;
  }
  sum = wave_sum(sum);
  const bool any = sum != 0.f;      // (0: no entry, or minus infinities alone; the largest finite one adds 1)
  const float log_sum = __builtin_amdgcn_logf(sum) * kLn2;
  for (int j = lane; j < A.K; j += 64) {
    const float lp = (sh.p[j] - o) * it - log_sum, p = __builtin_amdgcn_exp2f(lp * kLog2e);
    plogp += p != 0.f ? p * lp : 0.f;
    sh.p[j] = any ? p : 0.f;
  }
  if (lane == 0) sh.any = any;
  return wave_sum(plogp);
}
// The loss from there, by the first wavefront: w tau^2 (sum p log p - sum p ((z_j - m) / tau - log S)). The temperature is multiplied twice: its
// square is no fp32 number below 1e-19.
__device__ __forceinline__ float row_loss(const DistillArgs& A, const Teacher& sh, Stat st, float w, float plogp) {
  const float it = 1.f / A.temperature, o = origin(st.m), log_s = __builtin_amdgcn_logf(st.s) * kLn2;
  float cross = 0.f;
  for (int j = threadIdx.x & 63; j < A.K; j += 64)
    if (sh.p[j] != 0.f) cross += sh.z[j] == -INFINITY ? -INFINITY : sh.p[j] * ((sh.z[j] - o) * it - log_s);
  cross = wave_sum(cross);
  return sh.any && w != 0.f ? w * (A.temperature * (A.temperature * (plogp - cross))) : 0.f;
}
// The teacher's elements of a gradient in columns [c0, c1): scale * (q - p), q = exp2((z - o) c) * inv.
template <typename T>
__device__ __forceinline__ void put_teacher(const DistillArgs& A, const Teacher& sh, T* dz, int c0, int c1, float o, float c, float inv, float scale) {
  for (int j = threadIdx.x; j < A.K; j += blockDim.x) {
    const int at = sh.idx[j];
    if (at < c0 || at >= c1) continue;
    float p = 0.f;      // (an index that comes twice counts twice, and is written twice alike)
    for (int i = 0; i < A.K; ++i) p += sh.idx[i] == at ? sh.p[i] : 0.f;
    const float q = __builtin_amdgcn_exp2f((sh.z[j] - o) * c) * inv;
    dz[at] = (T)(scale * (q - p));
  }
}
// The gradient without the teacher's part.
template <typename T, int NV>
__device__ __forceinline__ void put_piece(const Held<T, NV>& held, T* dz, int n, int threads, bool rest, float last, T* dlast, float o, float c, float by) {
  constexpr int VE = Held<T, NV>::VE;
#pragma unroll
  for (int i = 0; i < NV; ++i)
    if ((int)threadIdx.x + i * threads < n) {
      float v[VE];
      held.get(i, v);
#pragma unroll
      for (int e = 0; e < VE; ++e) v[e] = __builtin_amdgcn_exp2f((v[e] - o) * c) * by;
      stream_n(dz + ((int)threadIdx.x + i * threads) * VE, v);
    }
  if (rest) *dlast = (T)(__builtin_amdgcn_exp2f((last - o) * c) * by);
}
template <typename T>
__device__ __forceinline__ void put_zeros(T* dz, int n, bool rest, T* dlast) {
  constexpr int VE = 16 / sizeof(T);
  const float zero[VE] = {};
  for (int i = threadIdx.x; i < n; i += blockDim.x) stream_n(dz + (int64_t)i * VE, zero);
  if (rest) *dlast = (T)0.f;
}
// Before elements are written again by other threads: the workgroup's stores have arrived.
__device__ __forceinline__ void stores_done() {
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
}

// ---- a row a workgroup: loss, log-sum-exp and gradient, whichever are wanted ----
// 512 threads with eight vectors each for rows of up to 64 KB: four workgroups a compute unit, so that some read while others write.
template <typename T, int THREADS, int NV>
__global__ __launch_bounds__(THREADS) void k_distill_row(DistillArgs A) {
  __shared__ Teacher teacher;
  __shared__ Stat sh[THREADS / 64];
  const int t = blockIdx.x;
  const T* z = (const T*)A.logits + (int64_t)t * A.stride;
  T* dz = A.dlogits ? (T*)A.dlogits + (int64_t)t * A.dstride : nullptr;
  const Span<T> row(dz ? dz : z, A.V);
  const bool rest = (int)threadIdx.x < row.singles();
  const int single = row.single(threadIdx.x);
  const float w = A.weight ? A.weight[t] : 1.f, c = kLog2e / A.temperature;
  if (w == 0.f && !A.lse) {
    if (threadIdx.x == 0) A.loss[t] = 0.f;
    if (dz) put_zeros(dz + row.head, row.n, rest, dz + single);
    return;
  }
  Held<T, NV> held;
  if (row.n) held.load(z + row.head, row.n, THREADS);
  const float last = rest ? (float)z[single] : 0.f;
  const float plogp = threadIdx.x < 64 ? take_teacher(A, t, z, teacher) : 0.f;
  const Stat st = piece_stat(held, row.n, THREADS, rest, last, c, sh);
  if (threadIdx.x < 64) {
    const float loss = row_loss(A, teacher, st, w, plogp);
    if (threadIdx.x == 0) {
      A.loss[t] = loss;
      if (A.lse) A.lse[t] = origin(st.m) / A.temperature + __builtin_amdgcn_logf(st.s) * kLn2;
    }
  }
  if (!dz) return;
  if (!teacher.any) return put_zeros(dz + row.head, row.n, rest, dz + single);
  const float o = origin(st.m), inv = st.s == 0.f ? 0.f : 1.f / st.s, scale = w * A.temperature;
  put_piece(held, dz + row.head, row.n, THREADS, rest, last, dz + single, o, c, inv * scale);
  stores_done();
  put_teacher(A, teacher, dz, 0, A.V, o, c, inv, scale);
}

// A saved log-sum-exp beyond which it is not used: 2^-23 |lse| is half a step of the 16-bit types there. In rows of the type's lowest value
// alone it cannot tell log V, and below temperature 1 it may be no finite number.
constexpr float kFarLse = 4096.f;
// The statistics of a whole row, by a workgroup (rows of that kind are rare, and every chunk's workgroup goes through all of theirs).
template <typename T>
__device__ __forceinline__ Stat row_stat(const T* z, int V, float c, Stat* sh) {
  float m = -INFINITY, s = 0.f;
#pragma unroll 1
  for (int64_t i = threadIdx.x; i < V; i += blockDim.x) m = fmaxf(m, (float)z[i]);
  m = wave_max(m);
#pragma unroll 1
  for (int64_t i = threadIdx.x; i < V; i += blockDim.x) s += __builtin_amdgcn_exp2f(((float)z[i] - origin(m)) * c);
  s = wave_sum(s);
  if (threadIdx.x % 64 == 0) sh[threadIdx.x / 64] = Stat{m, s};
  __syncthreads();
  return join(sh, blockDim.x / 64, c);
}

// ---- rows in chunks of a workgroup: vectors [chunk * per, ...); the single elements with the last chunk ----
constexpr int kChunkThreads = 256, kChunkVectors = 8;

template <typename T>
__global__ __launch_bounds__(kChunkThreads) void k_distill_stat(DistillArgs A, int per) {
  __shared__ Stat sh[kChunkThreads / 64];
  const int t = blockIdx.y;
  if (A.weight && !A.lse && A.weight[t] == 0.f) return;
  const T* z = (const T*)A.logits + (int64_t)t * A.stride;
  const Span<T> row(z, A.V);
  const int first = blockIdx.x * per, n = min(per, row.n - first);
  Held<T, kChunkVectors> held;
  if (n > 0) held.load(z + row.head + (int64_t)first * Span<T>::VE, n, kChunkThreads);
  const bool rest = blockIdx.x + 1 == gridDim.x && (int)threadIdx.x < row.singles();
  const Stat st = piece_stat(held, n, kChunkThreads, rest, rest ? (float)z[row.single(threadIdx.x)] : 0.f, kLog2e / A.temperature, sh);
  if (threadIdx.x == 0) ((Stat*)A.ws)[(int64_t)t * gridDim.x + blockIdx.x] = st;
}

// Loss and log-sum-exp of a row, a wavefront each, from its chunks' statistics.
template <typename T>
__global__ __launch_bounds__(64) void k_distill_join(DistillArgs A, int chunks) {
  __shared__ Teacher teacher;
  const int t = blockIdx.x;
  const float w = A.weight ? A.weight[t] : 1.f;
  const float plogp = take_teacher(A, t, (const T*)A.logits + (int64_t)t * A.stride, teacher);
  const Stat st = join((const Stat*)A.ws + (int64_t)t * chunks, chunks, kLog2e / A.temperature);
  __syncthreads();
  const float loss = row_loss(A, teacher, st, w, plogp);
  if (threadIdx.x == 0) {
    A.loss[t] = loss;
    if (A.lse) A.lse[t] = origin(st.m) / A.temperature + __builtin_amdgcn_logf(st.s) * kLn2;
  }
}

// The gradient of a chunk: from the chunks' statistics (with the loss, by the first one), or from a saved log-sum-exp.
template <typename T, bool SAVED>
__global__ __launch_bounds__(kChunkThreads) void k_distill_grad(DistillArgs A, int per, int chunks) {
  __shared__ Teacher teacher;
  __shared__ Stat sh[SAVED ? kChunkThreads / 64 : 1];
  const int t = blockIdx.y;
  const T* z = (const T*)A.logits + (int64_t)t * A.stride;
  T* dz = (T*)A.dlogits + (int64_t)t * A.dstride;
  const Span<T> row(dz, A.V);
  const int first = blockIdx.x * per, n = min(per, row.n - first), at = row.head + first * Span<T>::VE;
  const bool rest = blockIdx.x + 1 == gridDim.x && (int)threadIdx.x < row.singles();
  const int single = row.single(threadIdx.x);
  float w = A.weight ? A.weight[t] : 1.f;
  const float c = kLog2e / A.temperature;
  if (w == 0.f) {
    if (!SAVED && blockIdx.x == 0 && threadIdx.x == 0) A.loss[t] = 0.f;
    return put_zeros(dz + at, n, rest, dz + single);
  }
  Held<T, kChunkVectors> held;
  if (n > 0) held.load(z + at, n, kChunkThreads);
  const float last = rest ? (float)z[single] : 0.f;
  if (threadIdx.x < 64) {
    const float plogp = take_teacher(A, t, z, teacher);
    if constexpr (!SAVED) {
      const Stat st = join((const Stat*)A.ws + (int64_t)t * chunks, chunks, c);
      if (threadIdx.x == 0) sh[0] = st;
      if (blockIdx.x == 0) {
        const float loss = row_loss(A, teacher, st, w, plogp);
        if (threadIdx.x == 0) A.loss[t] = loss;
      }
    }
  }
  __syncthreads();
  if (!teacher.any) return put_zeros(dz + at, n, rest, dz + single);
  float o, inv, scale = w * A.temperature;
  if constexpr (SAVED) {
    // exp(z / tau - lse): the sum's logarithm as an origin of the logits, and nothing left to divide by
    const float lse = A.lse_in[t];
    o = lse * A.temperature, inv = 1.f;
    scale *= A.dloss[t];
    if (fabsf(lse) > kFarLse) {
      const Stat st = row_stat(z, A.V, c, sh);
      o = origin(st.m), inv = st.s == 0.f ? 0.f : 1.f / st.s;
    }
  } else {
    o = origin(sh[0].m), inv = sh[0].s == 0.f ? 0.f : 1.f / sh[0].s;
  }
  put_piece(held, dz + at, n, kChunkThreads, rest, last, dz + single, o, c, inv * scale);
  stores_done();
  // the teacher's entries among this chunk's vectors, and, with the last chunk, among the single elements
  put_teacher(A, teacher, dz, at, at + max(n, 0) * Span<T>::VE, o, c, inv, scale);
  if (blockIdx.x + 1 == gridDim.x) {
    put_teacher(A, teacher, dz, 0, row.head, o, c, inv, scale);
    put_teacher(A, teacher, dz, row.head + row.n * Span<T>::VE, A.V, o, c, inv, scale);
  }
}

// ---- host side ----
// Vectors of a chunk and their number in a row: full chunks, or shorter ones (of a vector a thread or more) where the rows are too few
// to give every compute unit four workgroups.
struct Chunks { int per, n; };
constexpr int64_t kFewChunks = 1024;      // of all rows
int64_t vectors_of(int32_t V, int32_t dtype) { return std::max<int64_t>(1, V / (16 / dtype_bytes(dtype))); }
int64_t full_chunks(int64_t vectors) { return (vectors + kChunkThreads * kChunkVectors - 1) / (kChunkThreads * kChunkVectors); }
Chunks chunks_of(int32_t T, int32_t V, int32_t dtype) {
  const int64_t all = vectors_of(V, dtype);
  int64_t n = full_chunks(all);
  while (n * T < kFewChunks && all / (2 * n) >= kChunkThreads) n *= 2;
  const int64_t per = (all + n - 1) / n;
  return Chunks{(int)per, (int)((all + per - 1) / per)};
}
// Rows that go a workgroup each, held in its registers: those of up to 128 KB, and for a gradient, which the chunks read the logits
// twice for, those of up to 256 KB where they are enough for the chip. us by rows / in chunks, loss and with the gradient: 32000 bf16
// x 16 rows 5.2 / 6.4, 8.1 / 8.5, x 1024 14.9 / 17.7, 28.8 / 36.1; 32000 fp32 x 64 5.6 / 7.4, 8.7 / 11.0, x 1024 30.7 / 28.5,
// 53 / 68; 128000 bf16 x 64 11.4 / 9.3, 18.7 / 13.6, x 128 12.8 / 12.0, 20.2 / 20.3, x 1024 62 / 53, 110 / 135.
bool by_rows(int32_t T, int32_t V, int32_t dtype, bool gradient) {
  const int64_t all = V / (16 / dtype_bytes(dtype));
  return all <= 8192 || (gradient && all <= 16384 && T >= 128);
}

// Rows of one launch of the chunked kernels (the grid's second dimension).
constexpr int32_t kRowsOfLaunch = 65535;
template <typename F>
hipError_t in_launches(DistillArgs a, int32_t most, F&& f) {
  while (a.T > 0) {
    DistillArgs b = a;
    b.T = std::min(a.T, most);
    if (hipError_t e = f(b); e != hipSuccess) return e;
    const int64_t sz = dtype_bytes(a.dtype), k = b.T;
    a.T -= b.T;
    a.logits = (const char*)a.logits + k * a.stride * sz;
    a.top_idx += k * a.K, a.top_logits += k * a.K;
    if (a.weight) a.weight += k;
    if (a.lse_in) a.lse_in += k;
    if (a.dloss) a.dloss += k;
    if (a.loss) a.loss += k;
    if (a.lse) a.lse += k;
    if (a.dlogits) a.dlogits = (char*)a.dlogits + k * a.dstride * sz;
  }
  return hipSuccess;
}

template <typename T>
hipError_t launch_rows(const DistillArgs& a, hipStream_t st) {
  const int all = a.V / (16 / (int)sizeof(T)), threads = all <= 1024 ? 256 : all <= 4096 ? 512 : 1024;
  return in_launches(a, launch_groups(threads), [&](const DistillArgs& b) {
    if (all <= 1024) hipLaunchKernelGGL((k_distill_row<T, 256, 4>), dim3(b.T), dim3(256), 0, st, b);
    else if (all <= 4096) hipLaunchKernelGGL((k_distill_row<T, 512, 8>), dim3(b.T), dim3(512), 0, st, b);
    else if (all <= 8192) hipLaunchKernelGGL((k_distill_row<T, 1024, 8>), dim3(b.T), dim3(1024), 0, st, b);
    else hipLaunchKernelGGL((k_distill_row<T, 1024, 16>), dim3(b.T), dim3(1024), 0, st, b);
    return hipGetLastError();
  });
}

}  // namespace

size_t distill_ws_bytes(int32_t T, int32_t V, int32_t dtype) {
  if (T <= 0 || by_rows(T, V, dtype, false)) return 0;
  // (room for as many rows and for any fewer: those in shorter chunks have less than twice kFewChunks of them)
  return (size_t)std::max<int64_t>(std::min(T, kRowsOfLaunch) * full_chunks(vectors_of(V, dtype)), 2 * kFewChunks) * sizeof(Stat);
}

hipError_t launch_distill_forward(const DistillArgs& a, hipStream_t st) {
  return with_type(a.dtype, [&](auto tag) {
    using T = decltype(tag);
    if (by_rows(a.T, a.V, a.dtype, false)) return launch_rows<T>(a, st);
    const Chunks k = chunks_of(a.T, a.V, a.dtype);
    return in_launches(a, kRowsOfLaunch, [&](const DistillArgs& b) {
      hipLaunchKernelGGL(k_distill_stat<T>, dim3(k.n, b.T), dim3(kChunkThreads), 0, st, b, k.per);
      hipLaunchKernelGGL(k_distill_join<T>, dim3(b.T), dim3(64), 0, st, b, k.n);
      return hipGetLastError();
    });
  });
}

hipError_t launch_distill_backward(const DistillArgs& a, hipStream_t st) {
  return with_type(a.dtype, [&](auto tag) {
    using T = decltype(tag);
    const Chunks k = chunks_of(a.T, a.V, a.dtype);
    return in_launches(a, kRowsOfLaunch, [&](const DistillArgs& b) {
      hipLaunchKernelGGL((k_distill_grad<T, true>), dim3(k.n, b.T), dim3(kChunkThreads), 0, st, b, k.per, k.n);
      return hipGetLastError();
    });
  });
}

hipError_t launch_distill_loss_grad(const DistillArgs& a, hipStream_t st) {
  return with_type(a.dtype, [&](auto tag) {
    using T = decltype(tag);
    if (by_rows(a.T, a.V, a.dtype, true)) return launch_rows<T>(a, st);
    const Chunks k = chunks_of(a.T, a.V, a.dtype);
    return in_launches(a, kRowsOfLaunch, [&](const DistillArgs& b) {
      hipLaunchKernelGGL(k_distill_stat<T>, dim3(k.n, b.T), dim3(kChunkThreads), 0, st, b, k.per);
      hipLaunchKernelGGL((k_distill_grad<T, false>), dim3(k.n, b.T), dim3(kChunkThreads), 0, st, b, k.per, k.n);
      return hipGetLastError();
    });
  });
}

}  // namespace moeq
