// Low-rank adapters of many requests beside a shared projection: y[t] = base[t] + scale_a B_a A_a x[t] with a = ids[t], and the
// gradient. A [n][r][d_in], B [n][d_out][r]; a row whose id is outside [0, n) has no adapter.
//   forward   h = scale_a A_a x,   y = base + B_a h
//   backward  g = scale_a B_a^T dy,   dx = dx_base + A_a^T g,   dA_a = sum of g x^T,   dB_a = sum of dy h^T
// Everything runs on the bf16 (fp16) matrix instructions with operands from memory straight to registers; memory bounds it: 2 r
// operations a byte are far below what the matrix cores do beside a stream of the rows.
//
// Precision. A fp32 operand is cut into three bf16 pieces of 8 bits each by truncation, a fp16 one into two, both exactly; the
// products of pieces whose places add up to 2 or less are taken (those left out are below 2^-23 of the product) and summed in fp32.
// bf16 with bf16 and fp16 with fp16 are one product. h and g are held as three pieces.
//
// Order of the rows. k_adapter_plan sorts them by adapter, every adapter's rows padded to whole tiles of TP (places; rowof[place] is
// the row or -1). Calls of up to kInlineTokens rows find their tiles by themselves: the tile b holds row b's adapter and those of
// its rows from b on, where b is each 16th of them.
#include <algorithm>

#include "sort_core.h"

namespace moeq {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr int kInlineTokens = 64;

// ---- operands of the matrix instructions ----
template <typename T> constexpr int kPieces = sizeof(T) == 4 ? 3 : std::is_same<T, _Float16>::value ? 2 : 1;

struct Bits8 { uint32_t w[4]; };      // eight 16-bit elements

__device__ __forceinline__ uint32_t high_halves(uint32_t lo, uint32_t hi) { return __builtin_amdgcn_perm(hi, lo, 0x07060302u); }

// The upper 16 bits of eight fp32 values as bf16, which are then taken off the values.
__device__ __forceinline__ bf16x8 peel(float (&v)[8]) {
  Bits8 b;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t x = __builtin_bit_cast(uint32_t, v[2 * i]), y = __builtin_bit_cast(uint32_t, v[2 * i + 1]);
    b.w[i] = high_halves(x, y);
    v[2 * i] -= __builtin_bit_cast(float, x & 0xffff0000u);
    v[2 * i + 1] -= __builtin_bit_cast(float, y & 0xffff0000u);
  }
  return __builtin_bit_cast(bf16x8, b);
}
// Eight elements as pieces.
template <typename T>
__device__ __forceinline__ void cut(const T (&v)[8], bf16x8 (&p)[kPieces<T>]) {
  if constexpr (kPieces<T> == 1) {
    __builtin_memcpy(&p[0], v, 16);
  } else {
    float f[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = (float)v[i];
#pragma unroll
    for (int i = 0; i < kPieces<T>; ++i) p[i] = peel(f);
  }
}

__device__ __forceinline__ f32x4 mma(bf16x8 a, bf16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
// Operands of several pieces: the rows of the product from a, the columns from b.
template <int NA, int NB>
__device__ __forceinline__ f32x4 mma(const bf16x8 (&a)[NA], const bf16x8 (&b)[NB], f32x4 c) {
#pragma unroll
  for (int i = NA - 1; i >= 0; --i)
#pragma unroll
    for (int j = NB - 1; j >= 0; --j)
      if (i + j <= 2) c = mma(a[i], b[j], c);
  return c;
}

template <typename T>
__device__ __forceinline__ void load8(T (&v)[8], const T* p) { __builtin_memcpy(v, p, sizeof(v)); }
template <typename T>
__device__ __forceinline__ void load8_some(T (&v)[8], const T* p, int n) {
  if (n >= 8) return load8(v, p);
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = i < n ? p[i] : (T)0.f;
}

// ---- the plan ----
struct Segment { int32_t a, from, to, part; };      // rows of an adapter in places [from, to); part: index of its partial sums, or -1
struct Plan {
  int32_t *rowof, *tile_adapter;      // [places], [places / TP]: the adapter of a tile, n: none, -1: not used
  Segment* segments;                  // backward: the work items of the weights' gradients
  Segment* split;                     // adapters of several segments: {adapter, first part, number of parts}
  int32_t places, tiles, n_segments, n_split, seg_rows;
};

__global__ __launch_bounds__(1024) void k_adapter_plan(const int32_t* __restrict__ ids, int T, int64_t run, int n, int TP, Plan plan) {
  __shared__ int cnt[kSortCounts], start[kSortMaxExperts + 2], total[kSortMaxExperts + 2], segs[kSortMaxExperts + 2], parts[kSortMaxExperts + 2], n_split;
  if (threadIdx.x == 0) n_split = 0;
  sort_count(ids, 0, T, run, n, cnt);
  for (int e = threadIdx.x; e <= n; e += blockDim.x) {
    total[e] = sort_total(cnt, n, e);
    start[e] = (total[e] + TP - 1) / TP * TP;
    const int s = max(1, (start[e] + plan.seg_rows - 1) / max(1, plan.seg_rows));
    segs[e] = s;
    parts[e] = s > 1 && e < n ? s : 0;
  }
  __syncthreads();
  sort_scan(n, start);
  const int end = start[n] + (total[n] + TP - 1) / TP * TP;
  for (int e = threadIdx.x; e <= n; e += blockDim.x)
    for (int i = total[e]; i % TP; ++i) plan.rowof[start[e] + i] = -1;
  // the bin of a place: the last one that starts at or before it
  auto bin_of = [&](const int* from, int at) {
    int lo = 0, hi = n + 1;
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (from[mid] <= at) lo = mid; else hi = mid;
    }
    return lo;
  };
  for (int i = threadIdx.x; i < plan.tiles; i += blockDim.x) plan.tile_adapter[i] = i * TP < end ? bin_of(start, i * TP) : -1;
  if (plan.segments) {
    sort_scan(n, segs);
    sort_scan(n, parts);
    for (int i = threadIdx.x; i < plan.n_segments; i += blockDim.x) {
      const int a = bin_of(segs, i);
      Segment s{-1, 0, 0, -1};
      if (a < n) {
        const int k = i - segs[a], rows = (total[a] + TP - 1) / TP * TP, many = segs[a + 1] - segs[a];
        s.a = a;
        s.from = start[a] + k * plan.seg_rows;
        s.to = start[a] + min((k + 1) * plan.seg_rows, rows);
        if (many > 1) s.part = parts[a] + k;
      }
      plan.segments[i] = s;
    }
    for (int a = threadIdx.x; a < n; a += blockDim.x)       // (in any order: each is added up by itself)
      if (segs[a + 1] - segs[a] > 1) plan.split[atomicAdd(&n_split, 1)] = Segment{a, parts[a], segs[a + 1] - segs[a], 0};
    __syncthreads();
    for (int i = n_split + threadIdx.x; i < plan.n_split; i += blockDim.x) plan.split[i] = Segment{-1, 0, 0, 0};
  }
  sort_place(ids, 0, T, run, n, start, cnt, [&](int i, int p, int) { plan.rowof[p] = i; });
}

// The tile of a workgroup: its adapter (n: none; -1: nothing to do) and its rows, 16 MT of them from place 16 MT tile.
template <int ROWS>
__device__ __forceinline__ int find_tile(const Plan& plan, const int32_t* ids, int T, int n, int TP, int tile, int* rows) {
  if (plan.tile_adapter) {
    const int a = plan.tile_adapter[tile * ROWS / TP];
    if (threadIdx.x < ROWS) rows[threadIdx.x] = a < 0 ? -1 : plan.rowof[tile * ROWS + threadIdx.x];
    __syncthreads();
    return a;
  }
  const int lane = threadIdx.x & 63;
  const int id = lane < T ? key_of(ids, lane, n) : -1, mine = __builtin_amdgcn_readlane(id, tile);
  const uint64_t same = __ballot(id == mine);
  const int before = __popcll(same & ((1ull << tile) - 1));
  if (before % 16) return -1;
  if (threadIdx.x < 16) rows[threadIdx.x] = -1;
  __syncthreads();
  if (threadIdx.x < 64 && id == mine) {
    const int k = __popcll(same & ((1ull << lane) - 1)) - before;
    if (k >= 0 && k < 16) rows[k] = lane;
  }
  __syncthreads();
  return mine;
}

// h as bf16 pieces in the two orders that the products need: by place (rank contiguous, RK of it, zeros beyond the rank), and by
// rank (places contiguous).
struct Pieces {
  uint16_t* by_place;      // [places][3][RK] or null
  uint16_t* by_rank;       // [3][16 RT][places] or null
  int32_t RK, RR, places;
};

// ---- h = scale * (rows) A^T: products of 16 (rank) x 16 MT (rows), the columns split over the wavefronts ----
// A rank index: of wavefront lane m of the product's rows and tile j. Beyond the rank the last ones are computed again.
template <int RT>
__device__ __forceinline__ int rank_of(int m, int j, int rank) { return min(RT * m, rank - RT) + j; }

constexpr int kShrinkWaves = 8;

template <typename X, typename W, int RT, int MT, bool TRANS>
struct Shrink {
  static constexpr bool kSame16 = std::is_same<X, W>::value && sizeof(X) == 2;
  static constexpr int KS = sizeof(X) == 2 && sizeof(W) == 2 ? 2 : 1;      // 32-column steps of a unit: 128 bytes of a row
  struct Unit { X x[KS][MT][8]; W w[KS][RT][8]; };

  const X* xrow[MT];
  const W* wrow;
  int64_t wstep;
  int d, rank, m, q;

  template <bool TAIL>
  __device__ __forceinline__ void load(Unit& u, int unit) const {
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      const int c = (unit * KS + s) * 32 + 8 * q, left = d - c;
#pragma unroll
      for (int t = 0; t < MT; ++t) {
        if (TAIL) load8_some(u.x[s][t], xrow[t] + c, left); else load8(u.x[s][t], xrow[t] + c);
      }
      if constexpr (!TRANS) {
#pragma unroll
        for (int j = 0; j < RT; ++j) {
          const W* p = wrow + (int64_t)rank_of<RT>(m, j, rank) * d + c;
          if (TAIL) load8_some(u.w[s][j], p, left); else load8(u.w[s][j], p);
        }
      } else {
        const W* p = wrow + (int64_t)c * rank + rank_of<RT>(m, 0, rank);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          W v[RT] = {};
          if (!TAIL || e < left) __builtin_memcpy(v, p + e * rank, sizeof(v));
#pragma unroll
          for (int j = 0; j < RT; ++j) u.w[s][j][e] = v[j];
        }
      }
    }
  }
  __device__ __forceinline__ void multiply(const Unit& u, f32x4 (&acc)[RT][MT]) const {
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      if constexpr (std::is_same<X, _Float16>::value && kSame16) {
#pragma unroll
        for (int j = 0; j < RT; ++j)
#pragma unroll
          for (int t = 0; t < MT; ++t) {
            f16x8 a, b;
            __builtin_memcpy(&a, u.w[s][j], 16);
            __builtin_memcpy(&b, u.x[s][t], 16);
            acc[j][t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, acc[j][t], 0, 0, 0);
          }
      } else {
        bf16x8 a[RT][kPieces<W>], b[MT][kPieces<X>];
#pragma unroll
        for (int j = 0; j < RT; ++j) cut(u.w[s][j], a[j]);
#pragma unroll
        for (int t = 0; t < MT; ++t) cut(u.x[s][t], b[t]);
#pragma unroll
        for (int j = 0; j < RT; ++j)
#pragma unroll
          for (int t = 0; t < MT; ++t) acc[j][t] = mma(a[j], b[t], acc[j][t]);
      }
    }
  }
};

template <typename X, typename W, int RT, int MT, bool TRANS>
__device__ __forceinline__ void shrink(const AdapterArgs& P, const Plan& plan, int TP, const void* in, int64_t stride, int d, const Pieces& h,
                                       f32x4* red, int* rows) {
  using S = Shrink<X, W, RT, MT, TRANS>;
  const int tile = blockIdx.x, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int a = find_tile<16 * MT>(plan, P.ids, P.T, P.n, TP, tile, rows);
  if (a < 0 || a == P.n) return;
  S s;
  s.d = d, s.rank = P.rank, s.m = lane & 15, s.q = lane >> 4;
#pragma unroll
  for (int t = 0; t < MT; ++t) s.xrow[t] = (const X*)in + max(rows[16 * t + s.m], 0) * stride;      // (columns of the product do not meet: padding may hold any row)
  s.wrow = (const W*)(TRANS ? P.B : P.A) + (int64_t)a * P.rank * d;
  f32x4 acc[RT][MT] = {};
  const int width = 32 * S::KS, whole = d / width;
  typename S::Unit u[2];
  int k = wave;
  if (k < whole) s.template load<false>(u[0], k);
  while (k < whole) {
    const int k1 = k + kShrinkWaves;
    if (k1 < whole) s.template load<false>(u[1], k1);
    s.multiply(u[0], acc);
    if (k1 >= whole) break;
    k = k1 + kShrinkWaves;
    if (k < whole) s.template load<false>(u[0], k);
    s.multiply(u[1], acc);
  }
  if (whole * width < d && wave == whole % kShrinkWaves) {
    s.template load<true>(u[0], whole);
    s.multiply(u[0], acc);
  }
#pragma unroll
  for (int half = 1; half >= 0; --half) {                      // eight wavefronts to four, and those below
    if (wave / (kShrinkWaves / 2) == half)
#pragma unroll
      for (int j = 0; j < RT; ++j)
#pragma unroll
        for (int t = 0; t < MT; ++t) {
          f32x4& v = red[(((wave % (kShrinkWaves / 2)) * RT + j) * MT + t) * 64 + lane];
          v = half ? acc[j][t] : acc[j][t] + v;
        }
    __syncthreads();
  }
  const float scale = P.scale[a];
  for (int i = threadIdx.x; i < RT * MT * 64; i += blockDim.x) {
    const int l = i & 63, t = (i >> 6) % MT, j = (i >> 6) / MT, row = rows[16 * t + (l & 15)], place = (tile * MT + t) * 16 + (l & 15);
    f32x4 v = red[i];
#pragma unroll
    for (int w = 1; w < kShrinkWaves / 2; ++w) v += red[w * RT * MT * 64 + i];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int r = rank_of<RT>(4 * (l >> 4) + e, j, P.rank);      // (an index that comes twice has the same sums twice)
      float f = row < 0 ? 0.f : v[e] * scale;
#pragma unroll
      for (int p = 0; p < 3; ++p) {
        const uint32_t b = __builtin_bit_cast(uint32_t, f);
        f -= __builtin_bit_cast(float, b & 0xffff0000u);
        if (h.by_place) h.by_place[((int64_t)place * 3 + p) * h.RK + r] = b >> 16;
        if (h.by_rank) h.by_rank[(int64_t)(p * h.RR + r) * h.places + place] = b >> 16;
      }
    }
  }
  if (h.by_place)
    for (int i = threadIdx.x; i < 48 * MT * (h.RK - P.rank); i += blockDim.x)
      h.by_place[((int64_t)tile * MT * 48 + i / (h.RK - P.rank)) * h.RK + P.rank + i % (h.RK - P.rank)] = 0;
}

template <typename W, int RT, int MT>
__global__ __launch_bounds__(kShrinkWaves * 64) void k_adapter_down(AdapterArgs P, Plan plan, int TP, Pieces h) {
  __shared__ f32x4 red[kShrinkWaves / 2 * RT * MT * 64];
  __shared__ int rows[16 * MT];
  shrink<W, W, RT, MT, false>(P, plan, TP, P.x, P.x_stride, P.d_in, h, red, rows);
}
// Backward: h of the rows of x in the first half of the grid's second dimension, g of those of dy in the other.
template <typename W, typename Y, int RT, int MT>
__global__ __launch_bounds__(kShrinkWaves * 64) void k_adapter_down_both(AdapterArgs P, Plan plan, int TP, Pieces h, Pieces g) {
  __shared__ f32x4 red[kShrinkWaves / 2 * RT * MT * 64];
  __shared__ int rows[16 * MT];
  if (blockIdx.y == 0) shrink<W, W, RT, MT, false>(P, plan, TP, P.x, P.x_stride, P.d_in, h, red, rows);
  else shrink<Y, W, RT, MT, true>(P, plan, TP, P.dy, P.dy_stride, P.d_out, g, red, rows);
}

// ---- out = base + h B^T (TRANS: + g A): a wavefront holds the weights of 16 NJ columns and takes 16 rows at a time ----
// Column of the product's row 4 q + i of tile j: four lanes store 64 consecutive bytes.
template <typename Y, int NJ>
__device__ __forceinline__ int column_of(int m, int j) {
  constexpr int VE = 16 / sizeof(Y);
  return 4 * VE * ((m & 3) * (NJ / VE) + j / VE) + VE * (m >> 2) + j % VE;
}

template <typename Y, typename W, int RKS, int NJ, bool TRANS>
__global__ __launch_bounds__(256) void k_adapter_up(AdapterArgs P, Plan plan, int TP, Pieces h, int d, int per) {
  constexpr int VE = 16 / sizeof(Y), NW = kPieces<W>;
  __shared__ int rows[16];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, m = lane & 15, q = lane >> 4;
  const int c0 = (blockIdx.x * 4 + wave) * 16 * NJ, rank = P.rank;
  bf16x8 w[NJ][RKS][NW];
  int held = -1;
  for (int tile = blockIdx.y * per; tile < (int)(blockIdx.y + 1) * per && tile < plan.places / 16; ++tile) {
    __syncthreads();
    const int a = find_tile<16>(plan, P.ids, P.T, P.n, TP, tile, rows);
    if (a < 0) { if (plan.tile_adapter) return; continue; }
    if (c0 >= d) continue;
    f32x4 acc[NJ] = {};
    if (a < P.n) {
      if (a != held) {
        held = a;
        const W* W0 = (const W*)(TRANS ? P.A : P.B) + (int64_t)a * rank * d;
#pragma unroll
        for (int s = 0; s < RKS; ++s) {
          const int r0 = 32 * s + 8 * q;
          if constexpr (!TRANS) {
#pragma unroll
            for (int j = 0; j < NJ; ++j) {
              W v[8] = {};
              if (r0 < rank) load8_some(v, W0 + (int64_t)min(c0 + column_of<Y, NJ>(m, j), d - 1) * rank + r0, rank - r0);
              cut(v, w[j][s]);
            }
          } else {
#pragma unroll
            for (int j0 = 0; j0 < NJ; j0 += 4) {
              const int c = c0 + column_of<Y, NJ>(m, j0);
              W v[4][8] = {};
#pragma unroll
              for (int e = 0; e < 8; ++e)
                if (r0 + e < rank) {
                  const W* p = W0 + (int64_t)(r0 + e) * d + c;
                  W u[4] = {};
                  if (c + 4 <= d) {
                    __builtin_memcpy(u, p, sizeof(u));
                  } else {
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                      if (c + j < d) u[j] = p[j];
                  }
#pragma unroll
                  for (int j = 0; j < 4; ++j) v[j][e] = u[j];
                }
#pragma unroll
              for (int j = 0; j < 4; ++j) cut(v[j], w[j0 + j][s]);
            }
          }
        }
      }
      const uint16_t* hp = h.by_place + (int64_t)(tile * 16 + m) * 3 * h.RK + 8 * q;
      bf16x8 b[RKS][3];
#pragma unroll
      for (int s = 0; s < RKS; ++s)
#pragma unroll
        for (int p = 0; p < 3; ++p) __builtin_memcpy(&b[s][p], hp + p * h.RK + 32 * s, 16);
#pragma unroll
      for (int s = 0; s < RKS; ++s)
#pragma unroll
        for (int j = 0; j < NJ; ++j) acc[j] = mma(w[j][s], b[s], acc[j]);
    }
    const int row = rows[m];
    if (row >= 0)
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int g = 0; g < NJ / VE; ++g) {
          const int c = c0 + column_of<Y, NJ>(4 * q + i, g * VE), n = d - c;
          if (n <= 0) continue;
          float v[VE] = {};
          if (P.base) load_some(v, (const Y*)P.base + row * P.base_stride + c, n);
#pragma unroll
          for (int e = 0; e < VE; ++e) v[e] += acc[g * VE + e][i];
          store_some((Y*)P.out + row * P.out_stride + c, v, n);
        }
  }
}

// ---- dA = sum of g x^T, dB = sum of h dy^T: products of 16 (rank) x 16 NJ (columns), the places split over the wavefronts ----
// A lane holds NJ adjacent columns (16 bytes) of eight rows; a tile's operand is one column of all eight.
template <typename X, int RT, bool TRANS>
__device__ __forceinline__ void weight_grad(const AdapterArgs& P, const Plan& plan, const Pieces& h, const void* in, int64_t stride, int d,
                                            int slice, float* out, float* part, f32x4* red) {
  constexpr int NJ = 16 / sizeof(X);
  const Segment seg = plan.segments[blockIdx.y];
  if (seg.a < 0) return;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, m = lane & 15, q = lane >> 4, rank = P.rank;
  const int c0 = slice * 16 * NJ, c = c0 + NJ * m, left = d - c;
  const X* x = (const X*)in + c;
  f32x4 acc[RT][NJ] = {};
  for (int p = seg.from + 32 * wave; p < seg.to; p += 128) {
    int row[8];
    __builtin_memcpy(row, plan.rowof + p + 8 * q, 32);
    X v[8][NJ] = {};
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (row[e] >= 0) {
        const X* at = x + row[e] * stride;
        if (left >= NJ) {
          __builtin_memcpy(v[e], at, 16);
        } else {
#pragma unroll
          for (int j = 0; j < NJ; ++j)
            if (j < left) v[e][j] = at[j];
        }
      }
    bf16x8 a[RT][3];
#pragma unroll
    for (int t = 0; t < RT; ++t)
#pragma unroll
      for (int k = 0; k < 3; ++k) {
        const int r = min(4 * RT * (m >> 2) + 4 * t + (m & 3), rank - 1);      // (rows of the product do not meet)
        __builtin_memcpy(&a[t][k], h.by_rank + (int64_t)(k * h.RR + r) * h.places + p + 8 * q, 16);
      }
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
      X u[8];
      bf16x8 b[kPieces<X>];
#pragma unroll
      for (int e = 0; e < 8; ++e) u[e] = v[e][j];
      cut(u, b);
#pragma unroll
      for (int t = 0; t < RT; ++t) acc[t][j] = mma(a[t], b, acc[t][j]);
    }
  }
  // four wavefronts to two, and those in the stores
  constexpr int kTiles = RT * NJ * 64;
  if (wave >= 2)
#pragma unroll
    for (int t = 0; t < RT; ++t)
#pragma unroll
      for (int j = 0; j < NJ; ++j) red[(wave - 2) * kTiles + (t * NJ + j) * 64 + lane] = acc[t][j];
  __syncthreads();
  if (wave < 2)
#pragma unroll
    for (int t = 0; t < RT; ++t)
#pragma unroll
      for (int j = 0; j < NJ; ++j) {
        f32x4& v = red[wave * kTiles + (t * NJ + j) * 64 + lane];
        v = acc[t][j] + v;
      }
  __syncthreads();
  float* to = seg.part < 0 ? out + (int64_t)seg.a * rank * d : part + (int64_t)seg.part * rank * (P.d_in + P.d_out);
  for (int i = threadIdx.x; i < kTiles; i += 256) {
    // columns one after the other (dA), or the four rank indices of a column and those of its other tiles (dB)
    const int k = TRANS ? i / (4 * RT) : i % (16 * NJ), rt = TRANS ? i % (4 * RT) : i / (16 * NJ);
    const int qq = rt / RT, t = rt % RT, r = 4 * rt, at = (t * NJ + k % NJ) * 64 + qq * 16 + k / NJ, col = c0 + k;
    if (col >= d) continue;
    const f32x4 v = red[at] + red[kTiles + at];
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (r + e < rank) to[TRANS ? (int64_t)col * rank + r + e : (int64_t)(r + e) * d + col] = v[e];
  }
}

template <typename W, typename Y, int RT>
__global__ __launch_bounds__(256) void k_adapter_weights(AdapterArgs P, Plan plan, Pieces h, Pieces g, int slices_a, float* part) {
  constexpr int NJ = 16 / sizeof(W) > 16 / sizeof(Y) ? 16 / sizeof(W) : 16 / sizeof(Y);
  __shared__ f32x4 red[2 * RT * NJ * 64];
  const int s = blockIdx.x;
  if (s < slices_a) weight_grad<W, RT, false>(P, plan, g, P.x, P.x_stride, P.d_in, s, P.dA, part, red);
  else weight_grad<Y, RT, true>(P, plan, h, P.dy, P.dy_stride, P.d_out, s - slices_a, P.dB, part + (int64_t)P.rank * P.d_in, red);
}

// Adapters of several segments: their partial sums added up in order.
__global__ __launch_bounds__(256) void k_adapter_join(AdapterArgs P, Plan plan, const float* __restrict__ part) {
  const Segment s = plan.split[blockIdx.y];
  if (s.a < 0) return;
  const int64_t na = (int64_t)P.rank * P.d_in, nb = (int64_t)P.rank * P.d_out, all = na + nb;
  for (int64_t i = blockIdx.x * 256 + threadIdx.x; i < all; i += (int64_t)gridDim.x * 256) {
    float v = 0.f;
    for (int k = 0; k < s.to; ++k) v += part[(s.from + k) * all + i];
    if (i < na) P.dA[s.a * na + i] = v; else P.dB[s.a * nb + i - na] = v;
  }
}

// ---- host side ----
struct Setup {
  Plan plan;
  Pieces h, g;
  float* part;
  int TP, RT, RKS;
  size_t total;
};

// Rows of a segment of the weights' gradients: 1024, fewer where that leaves too few workgroups for the chip, more in long calls
// (the partial sums are rank x (d_in + d_out) floats a segment).
int segment_rows(const AdapterArgs& a) {
  const int64_t slices = (a.d_in + 127) / 128 + (a.d_out + 127) / 128;
  int rows = 1024;
  while (rows > 256 && slices * ((a.T + rows - 1) / rows) < 512) rows /= 2;
  while ((a.T + rows - 1) / rows > 16) rows *= 2;
  return rows;
}

Setup set_up(const AdapterArgs& a, bool backward) {
  Setup s = {};
  const bool inl = !backward && a.T <= kInlineTokens;
  s.RT = a.rank <= 16 ? 1 : a.rank <= 32 ? 2 : 4;
  s.RKS = a.rank <= 32 ? 1 : 2;
  s.TP = backward ? 32 : 16;
  Plan& p = s.plan;
  // every bin that has rows adds at most a tile less a row of padding
  const int pad = (s.TP - 1) * std::min(a.T, a.n + 1);
  p.places = inl ? 16 * a.T : (a.T + pad) / s.TP * s.TP;
  p.tiles = p.places / s.TP;
  // what is set aside never falls with the number of rows, so that the workspace of a call serves the smaller ones
  const int room = inl || backward ? p.places : std::max(p.places, 16 * kInlineTokens);
  const int room_split = std::min(16, a.T / 256) + pad / 256 + 1;
  size_t at = 0;
  auto take = [&](size_t bytes) {
    char* q = a.ws ? (char*)a.ws + at : nullptr;
    at += (bytes + 255) / 256 * 256;
    return (void*)q;
  };
  if (!inl) {
    p.rowof = (int32_t*)take((size_t)room * 4);
    p.tile_adapter = (int32_t*)take((size_t)room / s.TP * 4);
  }
  const int RK = 32 * s.RKS, RR = 16 * s.RT;
  auto pieces = [&](bool by_place, bool by_rank) {
    Pieces h{nullptr, nullptr, RK, RR, p.places};
    if (by_place) h.by_place = (uint16_t*)take((size_t)room * 3 * RK * 2);
    if (by_rank) h.by_rank = (uint16_t*)take((size_t)room * 3 * RR * 2);
    return h;
  };
  if (!backward) {
    s.h = pieces(true, false);
  } else {
    p.seg_rows = segment_rows(a);
    p.n_segments = a.n + 1 + p.places / p.seg_rows;
    p.n_split = p.places / p.seg_rows;
    p.segments = (Segment*)take((size_t)(a.n + 1 + room_split) * sizeof(Segment));
    p.split = (Segment*)take((size_t)room_split * sizeof(Segment));
    s.h = pieces(false, true);
    s.g = pieces(a.out || !a.ws, true);
    // (segments of at least 256 rows, at most 16 of them in the rows themselves: segment_rows)
    s.part = (float*)take((size_t)2 * room_split * a.rank * (a.d_in + a.d_out) * 4);
  }
  s.total = at;
  return s;
}

hipError_t launch_plan(const AdapterArgs& a, const Setup& s, hipStream_t st) {
  if (!s.plan.tile_adapter) return hipSuccess;
  const int waves = sort_waves(a.T, a.n);
  const int64_t run = (a.T + waves * 64 - 1) / (waves * 64) * 64;
  hipLaunchKernelGGL(k_adapter_plan, dim3(1), dim3(waves * 64), 0, st, a.ids, a.T, run, a.n, s.TP, s.plan);
  return hipGetLastError();
}

template <typename F>
hipError_t with_types(const AdapterArgs& a, F&& f) {
  return with_type(a.dtype, [&](auto tag) { return a.out_dtype == MOEQ_F32 ? f(tag, float{}) : f(tag, tag); });
}
template <typename F>
hipError_t with_rank(int RT, F&& f) {
  if (RT == 1) return f(std::integral_constant<int, 1>{});
  if (RT == 2) return f(std::integral_constant<int, 2>{});
  return f(std::integral_constant<int, 4>{});
}

// Rows and columns of the expanding kernel: 16-row tiles of a workgroup, which then loads its weights once for them.
template <typename Y, typename W, int RKS, bool TRANS>
hipError_t launch_up(const AdapterArgs& a, const Setup& s, const Pieces& h, int d, hipStream_t st) {
  constexpr int NJ = sizeof(W) == 4 ? 4 : 8;
  const int cols = (d + 64 * NJ - 1) / (64 * NJ), tiles = s.plan.places / 16;
  int per = 1;
  while (s.plan.tile_adapter && per < 4 && (int64_t)cols * tiles / (2 * per) >= 1024) per *= 2;
  hipLaunchKernelGGL((k_adapter_up<Y, W, RKS, NJ, TRANS>), dim3(cols, (tiles + per - 1) / per), dim3(256), 0, st, a, s.plan, s.TP, h, d, per);
  return hipGetLastError();
}

}  // namespace

size_t adapter_ws_bytes(const AdapterArgs& a, bool backward) {
  AdapterArgs b = a;
  b.ws = nullptr;
  const size_t forward = set_up(b, false).total;
  return backward ? std::max(forward, set_up(b, true).total) : forward;       // (what serves the backward pass serves both)
}

hipError_t launch_adapters_forward(const AdapterArgs& a, hipStream_t st) {
  if (a.T == 0) return hipSuccess;
  const Setup s = set_up(a, false);
  if (hipError_t e = launch_plan(a, s, st); e != hipSuccess) return e;
  return with_types(a, [&](auto tag, auto ytag) {
    using W = decltype(tag);
    using Y = decltype(ytag);
    return with_rank(s.RT, [&](auto rt) {
      constexpr int RT = decltype(rt)::value, RKS = RT == 4 ? 2 : 1, MT = 1;
      hipLaunchKernelGGL((k_adapter_down<W, RT, MT>), dim3(s.plan.places / (16 * MT)), dim3(kShrinkWaves * 64), 0, st, a, s.plan, s.TP, s.h);
      if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
      return launch_up<Y, W, RKS, false>(a, s, s.h, a.d_out, st);
    });
  });
}

hipError_t launch_adapters_backward(const AdapterArgs& a, hipStream_t st) {
  const Setup s = set_up(a, true);
  if (hipError_t e = launch_plan(a, s, st); e != hipSuccess) return e;
  return with_types(a, [&](auto tag, auto ytag) {
    using W = decltype(tag);
    using Y = decltype(ytag);
    return with_rank(s.RT, [&](auto rt) {
      constexpr int RT = decltype(rt)::value, RKS = RT == 4 ? 2 : 1, MT = 2;
      if (a.T) {
        hipLaunchKernelGGL((k_adapter_down_both<W, Y, RT, MT>), dim3(s.plan.places / (16 * MT), 2), dim3(kShrinkWaves * 64), 0, st, a, s.plan, s.TP, s.h, s.g);
        if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
        if (a.out)
          if (hipError_t e = launch_up<Y, W, RKS, true>(a, s, s.g, a.d_in, st); e != hipSuccess) return e;
      }
      const int sa = (a.d_in + 16 * (16 / sizeof(W)) - 1) / (16 * (16 / (int)sizeof(W))), sb = (a.d_out + 16 * (16 / (int)sizeof(Y)) - 1) / (16 * (16 / (int)sizeof(Y)));
      hipLaunchKernelGGL((k_adapter_weights<W, Y, RT>), dim3(sa + sb, s.plan.n_segments), dim3(256), 0, st, a, s.plan, s.h, s.g, sa, s.part);
      if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
      if (s.plan.n_split) {
        const int64_t all = (int64_t)a.rank * (a.d_in + a.d_out);
        hipLaunchKernelGGL(k_adapter_join, dim3((unsigned)std::min<int64_t>((all + 255) / 256, 1024), s.plan.n_split), dim3(256), 0, st, a, s.plan, s.part);
      }
      return hipGetLastError();
    });
  });
}

}  // namespace moeq
