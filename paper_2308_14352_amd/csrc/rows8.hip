// Tensors in 8 bits, two forms.
//
// Packed (what training keeps between its passes): blocks of 32 columns of a row share a power of two,
//   e = floor(log2(largest |v|)) - 6, at least -126 (fp16: -24), code = rint(v 2^-e) in [-127, 127], value = code 2^e,
// so that a value has 7 bits and a sign, which every element type holds exactly: what is unpacked is the value itself, and matrix products
// take it without a further rounding. A block with a NaN or an infinity is NaN altogether (its exponent is kPackNan).
//
// Rows for products in 8-bit integers: a scale for each row, scale = max |x| / 127 (at least 2^-126), code = rint(x / scale) with the
// quotient of fp32. A row with a NaN or an infinity has the scale NaN and codes of zero. Rows lie a multiple of 128 bytes apart, zeros
// behind the last column: the product reads them by whole cache lines.
//
// Memory bounds all three: 8192 rows of 4096 bf16 packed in 20.9 us (4.8 TB/s), unpacked in 15 (6.6, the codes from the cache), to rows of
// codes in 22.9 (4.4); a few rows are a launch's latency, 3.4 to 4.4.
#include <algorithm>

#include "operators.h"

namespace moeq {
namespace {

constexpr uint32_t kInfinity = 0x7f800000u;
__device__ __forceinline__ uint32_t magnitude(float v) { return __builtin_bit_cast(uint32_t, v) & 0x7fffffffu; }      // (ordered as the values are, infinity and NaN on top)
__device__ __forceinline__ float power(int e) { return __builtin_bit_cast(float, (uint32_t)(e + 127) << 23); }         // 2^e, -126 <= e <= 127

// N elements of a row of d at column c (zeros behind its end).
template <int N, typename T>
__device__ __forceinline__ void load_part(float (&v)[N], const T* row, int c, int d) {
  if (c + N <= d) {
    load_n(v, row + c);
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = c + i < d ? (float)row[c + i] : 0.f;
  }
}

// ---- packed: a thread has 16 bytes of the elements, 4 or 8 lanes a block; U pieces a thread are in flight together. A piece is as many
// elements, so that a wavefront reads 1 KB in a row and the largest of a block is two or three exchanges away ----
constexpr int kThreads = 256;
template <typename T> constexpr int kE = 16 / sizeof(T);
template <typename T> constexpr int kLanes = kPackBlock / kE<T>;

struct PackGrid { int32_t d, per_row; uint32_t first_row, pieces; };      // pieces of a row (whole blocks), of the launch

template <typename T, int U>
__global__ __launch_bounds__(kThreads) void k_pack8(Rows8Args a, PackGrid g) {
  constexpr int E = kE<T>;
  const uint32_t nb = (a.d + kPackBlock - 1) / kPackBlock;
  float v[U][E];
  uint32_t row[U];
  int c[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const uint32_t i = (blockIdx.x * U + u) * kThreads + threadIdx.x, r = i / g.per_row;
    row[u] = g.first_row + r;
    c[u] = i < g.pieces ? (int)(i - r * g.per_row) * E : a.d;
    if (c[u] < a.d) {
      load_part(v[u], (const T*)a.x + row[u] * a.x_stride, c[u], a.d);
    } else {
#pragma unroll
      for (int j = 0; j < E; ++j) v[u][j] = 0.f;
    }
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    uint32_t top = 0;
#pragma unroll
    for (int j = 0; j < E; ++j) top = max(top, magnitude(v[u][j]));
    for (int s = 1; s < kLanes<T>; s *= 2) top = max(top, (uint32_t)__shfl_xor((int)top, s));
    if (c[u] >= a.d && c[u] % kPackBlock == 0) continue;      // (no block at all)
    const bool nan = top >= kInfinity;
    const int e = max((int)(top >> 23) - 127 - 6, std::is_same<T, _Float16>::value ? -24 : -126);
    const float up = nan ? 0.f : power(-e);
    int8_t code[E];
#pragma unroll
    for (int j = 0; j < E; ++j) code[j] = nan ? 0 : (int8_t)fminf(fmaxf(rintf(v[u][j] * up), -127.f), 127.f);
    int8_t* to = a.codes + (int64_t)row[u] * a.d + c[u];
    if (c[u] + E <= a.d) {
      __builtin_memcpy(to, code, E);
    } else {
#pragma unroll
      for (int j = 0; j < E; ++j)
        if (c[u] + j < a.d) to[j] = code[j];
    }
    if (c[u] % kPackBlock == 0) a.exps[(int64_t)row[u] * nb + c[u] / kPackBlock] = (int8_t)(nan ? kPackNan : e);
  }
}

template <typename T, int U>
__global__ __launch_bounds__(kThreads) void k_unpack8(Rows8Args a, PackGrid g) {
  constexpr int E = kE<T>;
  const uint32_t nb = (a.d + kPackBlock - 1) / kPackBlock;
  int8_t code[U][E], e[U];
  uint32_t row[U];
  int c[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const uint32_t i = (blockIdx.x * U + u) * kThreads + threadIdx.x, r = i / g.per_row;
    row[u] = g.first_row + r;
    c[u] = i < g.pieces ? (int)(i - r * g.per_row) * E : a.d;
    if (c[u] >= a.d) continue;
    const int8_t* from = a.codes + (int64_t)row[u] * a.d + c[u];
    if (c[u] + E <= a.d) {
      __builtin_memcpy(code[u], from, E);
    } else {
#pragma unroll
      for (int j = 0; j < E; ++j) code[u][j] = c[u] + j < a.d ? from[j] : 0;
    }
    e[u] = a.exps[(int64_t)row[u] * nb + c[u] / kPackBlock];
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    if (c[u] >= a.d) continue;
    const float unit = e[u] == kPackNan ? __builtin_nanf("") : power(e[u]);
    float v[E];
#pragma unroll
    for (int j = 0; j < E; ++j) v[j] = (float)code[u][j] * unit;
    T* to = (T*)a.out + row[u] * a.out_stride + c[u];
    if (c[u] + E <= a.d) {
      stream_n(to, v);
    } else {
#pragma unroll
      for (int j = 0; j < E; ++j)
        if (c[u] + j < a.d) to[j] = (T)v[j];
    }
  }
}

// Launches of fewer than 2^31 pieces each.
template <typename T, typename K>
hipError_t by_pieces(const Rows8Args& a, int unroll, hipStream_t st, K kernel) {
  const int64_t per_row = (int64_t)(a.d + kPackBlock - 1) / kPackBlock * kLanes<T>;
  const int64_t rows = std::max<int64_t>(((int64_t)1 << 31) / per_row - 1, 1);
  for (int64_t r = 0; r < a.T; r += rows) {
    const int64_t pieces = std::min<int64_t>(rows, a.T - r) * per_row;
    kernel<<<(uint32_t)((pieces + kThreads * unroll - 1) / (kThreads * unroll)), kThreads, 0, st>>>(a, PackGrid{a.d, (int32_t)per_row, (uint32_t)r, (uint32_t)pieces});
    if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  }
  return hipSuccess;
}

// ---- rows: W wavefronts a row, which is in registers between its largest element and the codes ----
template <typename T, int W, int NV>
__global__ __launch_bounds__(W == 1 ? 256 : 64 * W) void k_quantize_rows(Rows8Args a, int64_t pitch) {
  constexpr int VE = 8, kRows = W == 1 ? 4 : 1;
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, at = W == 1 ? lane : threadIdx.x;
  __shared__ uint32_t sh[W];
  for (int64_t row = (int64_t)blockIdx.x * kRows + (W == 1 ? wave : 0); row < a.T; row += (int64_t)gridDim.x * kRows) {
    float v[NV][VE];
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < NV; ++i) load_part(v[i], (const T*)a.x + row * a.x_stride, (at + i * 64 * W) * VE, a.d);
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int j = 0; j < VE; ++j) top = max(top, magnitude(v[i][j]));
    for (int s = 1; s < 64; s *= 2) top = max(top, (uint32_t)__shfl_xor((int)top, s));
    if constexpr (W > 1) {
      if (lane == 0) sh[wave] = top;
      __syncthreads();
#pragma unroll
      for (int w = 0; w < W; ++w) top = max(top, sh[w]);
      __syncthreads();
    }
    const bool nan = top >= kInfinity;
    const float scale = fmaxf(__builtin_bit_cast(float, top) / 127.f, 0x1p-126f);
    if (at == 0) a.scale[row] = nan ? __builtin_nanf("") : scale;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = (at + i * 64 * W) * VE;
      if (c >= pitch) continue;
      int8_t code[VE];
#pragma unroll
      for (int j = 0; j < VE; ++j) code[j] = nan ? 0 : (int8_t)rintf(v[i][j] / scale);      // (|quotient| <= 127 and a rounding)
      __builtin_memcpy(a.codes + row * pitch + c, code, VE);
    }
  }
}

}  // namespace

hipError_t launch_pack8(const Rows8Args& a, hipStream_t st) {
  return with_type(a.dtype, [&](auto t) { return by_pieces<decltype(t)>(a, 2, st, k_pack8<decltype(t), 2>); });
}

hipError_t launch_unpack8(const Rows8Args& a, hipStream_t st) {
  return with_type(a.dtype, [&](auto t) { return by_pieces<decltype(t)>(a, 2, st, k_unpack8<decltype(t), 2>); });
}

hipError_t launch_quantize_rows(const Rows8Args& a, hipStream_t st) {
  const int64_t pitch = q8_pitch(a.d);
  return with_type(a.dtype, [&](auto t) {
    using T = decltype(t);
    auto go = [&](auto kernel, int rows, int threads) {
      kernel<<<(uint32_t)std::min<int64_t>((a.T + rows - 1) / rows, 1 << 20), threads, 0, st>>>(a, pitch);
      return hipGetLastError();
    };
    if (pitch <= 512) return go(k_quantize_rows<T, 1, 1>, 4, 256);
    if (pitch <= 1024) return go(k_quantize_rows<T, 1, 2>, 4, 256);
    if (pitch <= 2048) return go(k_quantize_rows<T, 4, 1>, 1, 256);
    if (pitch <= 4096) return go(k_quantize_rows<T, 4, 2>, 1, 256);
    if (pitch <= 8192) return go(k_quantize_rows<T, 4, 4>, 1, 256);
    if (pitch <= 16384) return go(k_quantize_rows<T, 8, 4>, 1, 512);
    if (pitch <= 32768) return go(k_quantize_rows<T, 16, 4>, 1, 1024);
    return go(k_quantize_rows<T, 16, 8>, 1, 1024);
  });
}

}  // namespace moeq
