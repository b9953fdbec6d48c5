// Low-rank adapters of many requests beside a shared projection: y[t] = base[t] + scale_a B_a A_a x[t] with a = ids[t], and the
// gradient. A [n][r][d_in], B [n][d_out][r]; a row whose id is outside [0, n) has no adapter.
//   forward   h = scale_a A_a x,   y = base + B_a h
//   backward  g = scale_a B_a^T dy,   dx = dx_base + A_a^T g,   dA_a = sum of g x^T,   dB_a = sum of dy h^T
// Everything runs on the bf16 (fp16) matrix instructions with operands from memory straight to registers; memory bounds it: 2 r
// operations a byte are far below what the matrix cores do beside a stream of the rows.
//
// Precision. A fp32 operand is cut into three bf16 pieces of 8 bits each by truncation, a fp16 one into two, both exactly; the
// products of pieces whose places add up to 2 or less are taken (those left out are below 2^-23 of the product) and summed in fp32.
// bf16 with bf16 and fp16 with fp16 are one product. h and g are held in fp32 and cut where they are operands, or kept as three pieces.
//
// What bounds it, at 8192 bf16 rows of 4096 with eight adapters of rank 32: the plan 9 us (one workgroup's ballots), both narrowing
// products 42 (268 MB through the L1 caches, rows and weights alike: a compute unit receives some 26 KB a us; with the weights left out
// it took 34, without the rows 21), pieces 5, the weights' gradients 37 and 5 for their join (134 MB, part of it still in the cache of
// the memory side), the widening product 36 (134 MB, 3.8 TB/s). 4100 rows forward with 24 adapters of rank 16 and fp32 outputs: plan 8,
// narrowing 15, widening 33 (4.1 TB/s). Nine rows: 4.6 and 5.2, latency.
//
// Requests. Loads stand in straight lines without conditions, at addresses that are moved into the matrix where a piece would pass its
// end (and what comes twice by that meets a zero or is not stored): behind a condition the compiler waits for every load under way
// instead of counting them.
//
// Order of the rows. k_adapter_plan sorts them by adapter, every adapter's rows padded to whole tiles of TP (places; rowof[place] is
// the row, or ~row in padding, where row is one of the same adapter: it is read again and counts nothing). Calls of up to
// kInlineTokens rows find their tiles by themselves: the tile b holds row b's adapter and those of its rows from b on, where b is each
// 16th of them.
#include <algorithm>

#include "sort_core.h"

namespace moeq {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

// Rows of a call without a plan: a wavefront sees the ids of all at once. us of calls of 4096 columns without / with: 1 row 9.1 / 11.6,
// 32 rows of 32 adapters 9.7 / 12.5, 64 12.1 / 13.4.
constexpr int kInlineTokens = 64;
// Rows that one workgroup plans alone; beyond, chunks of them do, and a launch ahead of them counts. us of forward calls of 4096 columns,
// alone / in chunks: 12288 rows of 8 adapters 92 / 88, 16384 of 64 128 / 118, of 1024 columns 58 / 47 (8192 ids, the sort by itself: 9.1 /
// 8.9).
constexpr int kPlanOne = 8192;
static_assert(kPlanOne <= kSortKept);

// ---- operands of the matrix instructions: eight elements as they lie in memory, 4 words (16-bit types) or 8 ----
template <typename T> constexpr int kPieces = sizeof(T) == 4 ? 3 : std::is_same<T, _Float16>::value ? 2 : 1;
template <typename T> constexpr int kWords = 2 * sizeof(T);
template <typename T> struct Eight { uint32_t w[kWords<T>]; };

__device__ __forceinline__ uint32_t low_halves(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x05040100u); }
__device__ __forceinline__ uint32_t high_halves(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x07060302u); }

// The upper 16 bits of eight fp32 values as bf16, which are then taken off the values.
__device__ __forceinline__ bf16x8 peel(float (&v)[8]) {
  Eight<__bf16> b;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t x = __builtin_bit_cast(uint32_t, v[2 * i]), y = __builtin_bit_cast(uint32_t, v[2 * i + 1]);
    b.w[i] = high_halves(x, y);
    v[2 * i] -= __builtin_bit_cast(float, x & 0xffff0000u);
    v[2 * i + 1] -= __builtin_bit_cast(float, y & 0xffff0000u);
  }
  return __builtin_bit_cast(bf16x8, b);
}
__device__ __forceinline__ void cut(float (&f)[8], bf16x8 (&p)[3]) {
#pragma unroll
  for (int i = 0; i < 3; ++i) p[i] = peel(f);
}
// Eight elements as pieces.
template <typename T>
__device__ __forceinline__ void cut(const Eight<T>& v, bf16x8 (&p)[kPieces<T>]) {
  if constexpr (kPieces<T> == 1) {
    p[0] = __builtin_bit_cast(bf16x8, v);
  } else {
    float f[8];
    if constexpr (sizeof(T) == 4) {
#pragma unroll
      for (int i = 0; i < 8; ++i) f[i] = __builtin_bit_cast(float, v.w[i]);
    } else {
      const f16x8 h = __builtin_bit_cast(f16x8, v);
#pragma unroll
      for (int i = 0; i < 8; ++i) f[i] = (float)h[i];
    }
#pragma unroll
    for (int i = 0; i < kPieces<T>; ++i) p[i] = peel(f);
  }
}
// Operand j of the N that lie beside each other in eight rows of memory: v[e] holds N elements of row e.
template <typename T, int N>
__device__ __forceinline__ Eight<T> column(const uint32_t (&v)[8][(N * sizeof(T) + 3) / 4], int j) {
  Eight<T> r;
  if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int e = 0; e < 8; ++e) r.w[e] = v[e][j];
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) r.w[i] = j % 2 ? high_halves(v[2 * i][j / 2], v[2 * i + 1][j / 2]) : low_halves(v[2 * i][j / 2], v[2 * i + 1][j / 2]);
  }
  return r;
}
template <typename T, int N>
__device__ __forceinline__ void load_words(uint32_t (&v)[(N * sizeof(T) + 3) / 4], const T* p) {
  if constexpr (N * sizeof(T) == 2) {
    uint16_t u;
    __builtin_memcpy(&u, p, 2);
    v[0] = u;
  } else {
    __builtin_memcpy(v, p, N * sizeof(T));
  }
}

// Matrix instructions work on all lanes, whatever is masked off, and a short branch that no lane takes may be run masked instead of
// jumped over: every condition around them has to be one that the compiler knows to be the same for the whole wavefront.
__device__ __forceinline__ int wave_index() { return __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); }

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

// ---- the plan ----
struct Segment { int32_t a, from, to, part; };      // rows of an adapter in places [from, to); part: index of its partial sums, or -1
struct Plan {
  int32_t *rowof, *tile_adapter;      // [places], [places / TP]: the adapter of a tile, n: none, -1: not used
  Segment* segments;                  // backward: the work items of the weights' gradients
  Segment* split;                     // adapters of several segments: {adapter, first part, number of parts}
  int32_t* counts;                    // [chunks][n + 1]
  int32_t places, tiles, n_segments, n_split, seg_shift;
};

template <bool CHUNKS>
__global__ __launch_bounds__(1024) void k_adapter_plan(const int32_t* __restrict__ ids, int T, int run, int n, int TP, Plan plan) {
  __shared__ SortShared sh;
  __shared__ int ahead[CHUNKS ? kSortMaxExperts + 1 : 1];
  const int first = CHUNKS ? blockIdx.x * (int)kSortChunk : 0;
  __shared__ int start[kSortMaxExperts + 1], total[kSortMaxExperts + 1], segs[kSortMaxExperts + 1], parts[kSortMaxExperts + 1], n_split;
  if (threadIdx.x == 0) n_split = 0;
  // the bin of a place: the last one that starts at or before it
  auto last_at = [&](const int* from, int at) {
    int lo = 0, hi = n + 1;
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      const bool in = from[mid] <= at;
      lo = in ? mid : lo;
      hi = in ? hi : mid;
    }
    return lo;
  };
  sort_pairs(ids + first, CHUNKS ? min((int)kSortChunk, T - first) : T, run, n, sh,
             [&](int e, int all) {
               if (CHUNKS) all = count_all(plan.counts, gridDim.x, blockIdx.x, n, e, ahead[e]);
               const int rows = (all + TP - 1) & -TP, s = max(1, (rows + (1 << plan.seg_shift) - 1) >> plan.seg_shift);
               total[e] = all;
               start[e] = rows;
               segs[e] = s;
               parts[e] = s > 1 && e < n ? s : 0;
             },
             [&] {
               // three scans by three wavefronts (by one after the other in workgroups of fewer)
               const int waves = blockDim.x >> 6, wave = threadIdx.x >> 6;
               for (int k = wave; k < (plan.segments ? 3 : 1); k += waves) sort_scan(n, k == 0 ? start : k == 1 ? segs : parts);
             },
             [&](int i, int number, int e) {
               if (CHUNKS) i += first, number += ahead[e];
               const int p = start[e] + number;
               plan.rowof[p] = i;
               if (number == 0)
                 for (int k = total[e], end = (k + TP - 1) & -TP; k < end; ++k) plan.rowof[p + k] = ~i;
             });
  const int end = start[n] + ((total[n] + TP - 1) & -TP);
  for (int i = blockIdx.x * blockDim.x + threadIdx.x; i < plan.tiles; i += gridDim.x * blockDim.x) plan.tile_adapter[i] = i * TP < end ? last_at(start, i * TP) : -1;
  if (plan.segments && blockIdx.x == 0) {
    for (int i = threadIdx.x; i < plan.n_segments; i += blockDim.x) {
      const int a = last_at(segs, i);
      Segment s{-1, 0, 0, -1};
      if (a < n) {
        const int k = i - segs[a], rows = (total[a] + TP - 1) & -TP, many = segs[a + 1] - segs[a];
        s.a = a;
        s.from = start[a] + (k << plan.seg_shift);
        s.to = start[a] + min((k + 1) << plan.seg_shift, rows);
        if (many > 1) {
          s.part = parts[a] + k;
          if (k == 0) plan.split[atomicAdd(&n_split, 1)] = Segment{a, parts[a], many, 0};      // (in any order: each is added up by itself)
        }
      }
      plan.segments[i] = s;
    }
    __syncthreads();
    for (int i = n_split + threadIdx.x; i < plan.n_split; i += blockDim.x) plan.split[i] = Segment{-1, 0, 0, 0};
  }
}

// A tile of 16 rows: its adapter (n: none; -1: nothing to do), and for every lane the row of a place of its own (~row: padding). By
// every wavefront for itself.
template <bool FEW>
__device__ __forceinline__ int find_tile(const Plan& plan, const int32_t* ids, int T, int n, int TP, int tile) {
  if constexpr (!FEW) return plan.tile_adapter[tile * 16 / TP];
  const int lane = threadIdx.x & 63, id = lane < T ? bin_of(ids[lane], n) : -1, mine = __builtin_amdgcn_readlane(id, tile);
  return __popcll(__ballot(id == mine) & ((1ull << tile) - 1)) % 16 ? -1 : mine;
}
template <bool FEW>
__device__ __forceinline__ int find_row(const Plan& plan, const int32_t* ids, int T, int n, int tile, int place) {
  if constexpr (!FEW) return plan.rowof[tile * 16 + place];
  const int lane = threadIdx.x & 63, id = lane < T ? bin_of(ids[lane], n) : -1, mine = __builtin_amdgcn_readlane(id, tile);
  // the tile's rows send their numbers to the lanes that stand for their places; a lane that gets none reads 0
  const int k = __popcll(__ballot(id == mine) & ~((1ull << tile) - 1) & ((1ull << lane) - 1)), to = id == mine && lane >= tile && k < 16 ? k : 63;
  const int got = __builtin_amdgcn_ds_permute(4 * to, to < 63 ? lane + 1 : 0);      // (lanes that send none send 0 to a lane that nobody asks)
  return __shfl(got, place) - 1;
}
__device__ __forceinline__ int real_row(int row) { return row ^ (row >> 31); }

// h on its way from the narrowing to the widening products: in fp32 by place, one part per share of the columns, and as bf16 pieces by
// rank (places contiguous), as the weights' gradients need it.
struct Pieces {
  float* parts;            // [splits][places][RR]
  uint16_t* by_rank;       // [3][RR][places], backward
  int32_t RR, places, splits;
};
// Slots of the widening product's operands, in groups of eight: the rank index that a slot takes its weights from. The last group, where
// the rank is no multiple of eight, begins before its place, so that eight elements can be read; a rank below eight takes its last four,
// or single ones. h is zero in the slots that come twice by that.
__device__ __forceinline__ int slot_source(int slot, int rank) {
  const int e = slot & 7;
  return rank >= 8 ? min(slot - e, rank - 8) + e : rank >= 4 ? (e < 4 ? e : rank - 8 + e) : min(e, rank - 1);
}
__device__ __forceinline__ int slot_of(int r, int rank) {
  const int g = r & ~7;
  return rank >= 8 ? (g + 8 <= rank ? r : g + r - (rank - 8)) : rank >= 4 ? (r < 4 ? r : r + 8 - rank) : r;
}

// ---- h = scale * (rows) A^T: products of 16 (rank) x 16 MT (rows), the columns split over the wavefronts (and workgroups) ----
// A rank index: of lane m of the product's rows and tile j. Beyond the rank the last ones are computed again.
template <int RT>
__device__ __forceinline__ int rank_of(int m, int j, int rank) { return min(RT * m, rank - RT) + j; }

// 16-bit operands of two steps of 32 columns. A load takes eight rows of 128 bytes (a whole line of the cache) instead of sixteen of 64:
// lanes of m < 8 hold the first step's piece of rows m and m + 8, those of m >= 8 the second's of rows m - 8 and m; half of them change places.
__device__ __forceinline__ void exchange(uint32_t (&a)[4], uint32_t (&b)[4]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t x = a[i], y = b[i];
    a[i] = __builtin_amdgcn_update_dpp(x, y, 0x128, 0xf, 0xc, false);      // lanes 8..15 of a row of 16: from the lane 8 below
    b[i] = __builtin_amdgcn_update_dpp(y, x, 0x128, 0xf, 0x3, false);
  }
}

template <typename X, typename W, int RT, int MT, bool TRANS>
struct Shrink {
  static constexpr bool kHalf = std::is_same<X, _Float16>::value && std::is_same<W, _Float16>::value;
  static constexpr int KS = sizeof(X) == 2 && sizeof(W) == 2 ? 2 : 1;      // 32-column steps of a unit: 128 bytes of a row
  static constexpr bool kLines = KS == 2;
  static constexpr int kWidth = 32 * KS;
  // units that are under way in a wavefront: some 64 registers of them
  static constexpr int kRegs = KS * (MT * kWords<X> + (TRANS ? 8 * ((RT * (int)sizeof(W) + 3) / 4) : RT * kWords<W>)), DEPTH = kRegs <= 16 ? 4 : kRegs <= 24 ? 3 : kRegs <= 48 ? 2 : 1;
  struct Unit {
    Eight<X> x[KS][MT];
    Eight<W> w[TRANS ? 1 : KS][TRANS ? 1 : RT];
    uint32_t t[TRANS ? KS : 1][8][(RT * sizeof(W) + 3) / 4];
  };

  const X* xrow[MT][KS];      // rows of the lane's loads
  const W* wrow;
  int d, rank, m, q;

  // the row (of 16) and the column of load s
  __device__ __forceinline__ int row_of(int s) const { return kLines ? 8 * s + (m & 7) : m; }
  __device__ __forceinline__ int column_of(int unit, int s) const { return unit * kWidth + 8 * q + (kLines ? 32 * (m >> 3) : 32 * s); }

  __device__ __forceinline__ void load(Unit& u, int unit) const {
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      const int c = min(column_of(unit, s), d - 8);
#pragma unroll
      for (int t = 0; t < MT; ++t) load_words<X, 8>(u.x[s][t].w, xrow[t][s] + c);
      if constexpr (!TRANS) {
#pragma unroll
        for (int j = 0; j < RT; ++j) load_words<W, 8>(u.w[s][j].w, wrow + (int64_t)rank_of<RT>(row_of(s), j, rank) * d + c);
      } else {
        const W* p = wrow + (int64_t)min(unit * kWidth + 32 * s + 8 * q, d - 8) * rank + rank_of<RT>(m, 0, rank);
#pragma unroll
        for (int e = 0; e < 8; ++e) load_words<W, RT>(u.t[s][e], p + e * rank);
      }
    }
  }
  __device__ __forceinline__ void multiply(Unit& u, int unit, f32x4 (&acc)[RT][MT]) const {
    if ((unit + 1) * kWidth > d) {
      // the last columns: what was read before a piece's own place counts nothing
#pragma unroll
      for (int s = 0; s < KS; ++s) {
        const int c = column_of(unit, s), lead = c - min(c, d - 8);
#pragma unroll
        for (int t = 0; t < MT; ++t)
#pragma unroll
          for (int i = 0; i < kWords<X>; ++i) {
            const uint32_t keep = sizeof(X) == 4 ? (i >= lead ? ~0u : 0u) : (2 * i >= lead ? 0xffffu : 0u) | (2 * i + 1 >= lead ? 0xffff0000u : 0u);
            u.x[s][t].w[i] &= keep;
          }
      }
    }
    if constexpr (kLines) {
#pragma unroll
      for (int t = 0; t < MT; ++t) exchange(u.x[0][t].w, u.x[1][t].w);
      if constexpr (!TRANS)
#pragma unroll
        for (int j = 0; j < RT; ++j) exchange(u.w[0][j].w, u.w[1][j].w);
    }
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      Eight<W> w[RT];
#pragma unroll
      for (int j = 0; j < RT; ++j) {
        if constexpr (TRANS) w[j] = column<W, RT>(u.t[s], j); else w[j] = u.w[s][j];
      }
      if constexpr (kHalf) {
#pragma unroll
        for (int j = 0; j < RT; ++j)
#pragma unroll
          for (int t = 0; t < MT; ++t)
            acc[j][t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, w[j]), __builtin_bit_cast(f16x8, u.x[s][t]), acc[j][t], 0, 0, 0);
      } else {
        bf16x8 a[RT][kPieces<W>], b[MT][kPieces<X>];
#pragma unroll
        for (int j = 0; j < RT; ++j) cut(w[j], a[j]);
#pragma unroll
        for (int t = 0; t < MT; ++t) cut(u.x[s][t], b[t]);
#pragma unroll
        for (int j = 0; j < RT; ++j)
#pragma unroll
          for (int t = 0; t < MT; ++t) acc[j][t] = mma(a[j], b[t], acc[j][t]);
      }
    }
  }
  // The units first, first + step, ... below end.
  __device__ __forceinline__ void run(int first, int step, int end, f32x4 (&acc)[RT][MT]) const {
    const int n = first < end ? (end - first + step - 1) / step : 0, full = n / DEPTH, rest = n - full * DEPTH;
    Unit u[DEPTH];
    int at = first;
    if (full) {
#pragma unroll
      for (int i = 0; i < DEPTH; ++i) load(u[i], at + i * step);
      for (int k = 1; k < full; ++k) {
#pragma unroll
        for (int i = 0; i < DEPTH; ++i, at += step) {
          multiply(u[i], at, acc);
          load(u[i], at + DEPTH * step);
        }
      }
#pragma unroll
      for (int i = 0; i < DEPTH; ++i, at += step) multiply(u[i], at, acc);
    }
    if (rest) {
#pragma unroll
      for (int i = 0; i < DEPTH - 1; ++i) load(u[i], at + (i < rest ? i : 0) * step);
#pragma unroll
      for (int i = 0; i < DEPTH - 1; ++i)
        if (i < rest) multiply(u[i], at + i * step, acc);
    }
  }
};

// split: which share of the columns, of h.splits. PIECES: the pieces by rank as well (of all columns).
template <typename X, typename W, int RT, int MT, bool TRANS, int WAVES, bool FEW, bool PIECES>
__device__ __forceinline__ void shrink(const AdapterArgs& P, const Plan& plan, int TP, const void* in, int64_t stride, int d, const Pieces& h,
                                       int split, f32x4* red) {
  using S = Shrink<X, W, RT, MT, TRANS>;
  const int tile = blockIdx.x * MT, lane = threadIdx.x & 63, wave = wave_index();
  S s;
  s.d = d, s.rank = P.rank, s.m = lane & 15, s.q = lane >> 4;
  int rows[MT];
#pragma unroll
  for (int t = 0; t < MT; ++t) {
    rows[t] = find_row<FEW>(plan, P.ids, P.T, P.n, tile + t, s.m);
#pragma unroll
    for (int k = 0; k < S::KS; ++k)      // (columns of the product do not meet: padding may hold any row)
      s.xrow[t][k] = (const X*)in + real_row(S::kLines ? find_row<FEW>(plan, P.ids, P.T, P.n, tile + t, s.row_of(k)) : rows[t]) * stride;
  }
  const int a = find_tile<FEW>(plan, P.ids, P.T, P.n, TP, tile);
  if (a < 0 || a == P.n) return;
  s.wrow = (const W*)(TRANS ? P.B : P.A) + (int64_t)a * P.rank * d;
  const float scale = P.scale[a];
  f32x4 acc[RT][MT] = {};
  s.run(split * WAVES + wave, WAVES * h.splits, (d + S::kWidth - 1) / S::kWidth, acc);
#pragma unroll
  for (int half = 1; half >= 0; --half) {                      // the upper half of the wavefronts, and the lower one added to it
    if (wave / (WAVES / 2) == half)
#pragma unroll
      for (int j = 0; j < RT; ++j)
#pragma unroll
        for (int t = 0; t < MT; ++t) {
          f32x4& v = red[(((wave % (WAVES / 2)) * RT + j) * MT + t) * 64 + lane];
          v = half ? acc[j][t] : acc[j][t] + v;
        }
    __syncthreads();
  }
  for (int i = threadIdx.x; i < RT * MT * 64; i += WAVES * 64) {
    const int t = (i >> 6) % MT, j = (i >> 6) / MT, place = (tile + t) * 16 + s.m;
    int row = rows[0];
#pragma unroll
    for (int k = 1; k < MT; ++k) row = t == k ? rows[k] : row;
    f32x4 v = red[i];
#pragma unroll
    for (int w = 1; w < WAVES / 2; ++w) v += red[w * RT * MT * 64 + i];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int r = rank_of<RT>(4 * s.q + e, j, P.rank);      // (an index that comes twice has the same sums twice)
      float f = row < 0 ? 0.f : v[e] * scale;
      h.parts[((int64_t)split * h.places + place) * h.RR + r] = f;
      if constexpr (PIECES)
#pragma unroll
        for (int p = 0; p < 3; ++p) {
          const uint32_t b = __builtin_bit_cast(uint32_t, f);
          f -= __builtin_bit_cast(float, b & 0xffff0000u);
          h.by_rank[(int64_t)(p * h.RR + r) * h.places + place] = b >> 16;
        }
    }
  }
}

template <typename W, int RT, int MT, bool FEW>
__global__ __launch_bounds__(256) void k_adapter_down(AdapterArgs P, Plan plan, int TP, Pieces h) {
  __shared__ f32x4 red[2 * RT * MT * 64];
  shrink<W, W, RT, MT, false, 4, FEW, false>(P, plan, TP, P.x, P.x_stride, P.d_in, h, blockIdx.y, red);
}
// Backward: h of the rows of x in the first half of the grid's second dimension, g of those of dy in the other.
template <typename W, typename Y, int RT, int MT, bool WHOLE>
__global__ __launch_bounds__(256) void k_adapter_down_both(AdapterArgs P, Plan plan, int TP, Pieces h, Pieces g) {
  __shared__ f32x4 red[2 * RT * MT * 64];
  if ((int)blockIdx.y < h.splits) shrink<W, W, RT, MT, false, 4, false, WHOLE>(P, plan, TP, P.x, P.x_stride, P.d_in, h, blockIdx.y, red);
  else shrink<Y, W, RT, MT, true, 4, false, WHOLE>(P, plan, TP, P.dy, P.dy_stride, P.d_out, g, blockIdx.y - h.splits, red);
}

// The parts of h (of g) added up in order: as pieces by rank, and in fp32 in the place of the first part. 32 places a workgroup.
__global__ __launch_bounds__(256) void k_adapter_pieces(Pieces h, Pieces g) {
  __shared__ float sum[32 * 65];
  const Pieces p = blockIdx.y ? g : h;
  const int first = blockIdx.x * 32, shift = 31 - __builtin_clz(p.RR);
  float* from = p.parts + (int64_t)first * p.RR;
  const int64_t step = (int64_t)p.places * p.RR;
  for (int i = threadIdx.x * 4; i < 32 * p.RR; i += 1024) {
    f32x4 v[8] = {}, s = {};
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = *(const f32x4*)(from + min(k, p.splits - 1) * step + i);
#pragma unroll
    for (int k = 0; k < 8; ++k)
#pragma unroll
      for (int e = 0; e < 4; ++e) s[e] += k < p.splits ? v[k][e] : 0.f;
    if (p.splits > 1) *(f32x4*)(from + i) = s;
#pragma unroll
    for (int e = 0; e < 4; ++e) sum[(i >> shift) * 65 + (i & (p.RR - 1)) + e] = s[e];
  }
  __syncthreads();
  for (int i = threadIdx.x; i < 32 * p.RR; i += 256) {
    const int place = i & 31, r = i >> 5;
    float f = sum[place * 65 + r];
#pragma unroll
    for (int k = 0; k < 3; ++k) {
      const uint32_t b = __builtin_bit_cast(uint32_t, f);
      f -= __builtin_bit_cast(float, b & 0xffff0000u);
      p.by_rank[(int64_t)(k * p.RR + r) * p.places + first + place] = b >> 16;
    }
  }
}

// ---- out = base + h B^T (TRANS: + g A): a wavefront takes 16 NJ columns of `per` tiles of 16 rows, one after the other with the same
// weights (tiles on their way together would be twice the code, which a launch of few rows fetches once for each workgroup's sake) ----
// A lane holds groups of VE columns, 16 bytes of the output, of four rows: sixteen lanes read and store 256 consecutive bytes. A group
// that would pass the last column begins before it.

// Eight slots from `at` on of a row of `rank` elements. KIND: 0 for ranks of eight and more, 1 of four and more, 2 below (the choice is
// made once, around all loads).
template <typename T, int KIND>
__device__ __forceinline__ void load_slots(uint32_t (&w)[kWords<T>], const T* row, int at, int rank) {
  if constexpr (KIND == 0) {
    load_words<T, 8>(w, row + min(at, rank - 8));
  } else if constexpr (KIND == 1) {
    __builtin_memcpy(w, row, 4 * sizeof(T));
    __builtin_memcpy(w + kWords<T> / 2, row + rank - 4, 4 * sizeof(T));
  } else {
    T v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = row[min(e, rank - 1)];
    __builtin_memcpy(w, v, sizeof(v));
  }
}
template <typename F>
__device__ __forceinline__ void by_rank_kind(int rank, F&& f) {
  if (rank >= 8) f(std::integral_constant<int, 0>{});
  else if (rank >= 4) f(std::integral_constant<int, 1>{});
  else f(std::integral_constant<int, 2>{});
}

template <typename Y, typename W, int RKS, int NJ, bool TRANS, bool FEW>
__global__ __launch_bounds__(256, RKS == 1 ? 3 : 2) void k_adapter_up(AdapterArgs P, Plan plan, int TP, Pieces h, int d, int per) {
  constexpr int VE = 16 / sizeof(Y), NG = NJ / VE;
  const int lane = threadIdx.x & 63, c0 = (blockIdx.x * 4 + wave_index()) * 16 * NJ, m = lane & 15, q = lane >> 4, rank = P.rank;
  if (c0 >= d) return;
  const int first = blockIdx.y * per, a = find_tile<FEW>(plan, P.ids, P.T, P.n, TP, first);
  if (a < 0) return;
  auto group = [&](int g) { return c0 + 16 * VE * g + VE * m; };

  // weights: eight slots of a column (a row of B), or four columns of eight slots (rows of A)
  const W* W0 = (const W*)(TRANS ? P.A : P.B) + (int64_t)min(a, P.n - 1) * rank * d;
  Eight<W> w[TRANS ? 1 : RKS][TRANS ? 1 : NJ];
  uint32_t wt[TRANS ? RKS : 1][TRANS ? NJ / 4 : 1][8][sizeof(W)];
  if constexpr (!TRANS) {
    by_rank_kind(rank, [&](auto kind) {
#pragma unroll
      for (int s = 0; s < RKS; ++s)
#pragma unroll
        for (int j = 0; j < NJ; ++j)
          load_slots<W, decltype(kind)::value>(w[s][j].w, W0 + (int64_t)(min(group(j / VE), d - VE) + j % VE) * rank, 32 * s + 8 * q, rank);
    });
  } else {
#pragma unroll
    for (int s = 0; s < RKS; ++s)
#pragma unroll
      for (int g = 0; g < NJ / 4; ++g)
#pragma unroll
        for (int e = 0; e < 8; ++e)
          load_words<W, 4>(wt[s][g][e], W0 + (int64_t)slot_source(32 * s + 8 * q + e, rank) * d + min(group(g * 4 / VE), d - VE) + g * 4 % VE);
  }
  uint32_t once[RKS] = {};      // a bit for each of the lane's slots that is not a repetition
#pragma unroll
  for (int s = 0; s < RKS; ++s)
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int slot = 32 * s + 8 * q + e;
      once[s] |= (slot_of(slot_source(slot, rank), rank) == slot ? 1u : 0u) << e;
    }
#pragma unroll 1
  for (int tile = first; tile < first + per; ++tile) {
    int rows[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) rows[i] = find_row<FEW>(plan, P.ids, P.T, P.n, tile, 4 * q + i);
    struct Group { uint32_t w[4]; } base[4][NG] = {};
    if (P.base)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const Y* from = (const Y*)P.base + real_row(rows[i]) * P.base_stride;
#pragma unroll
        for (int g = 0; g < NG; ++g) __builtin_memcpy(base[i][g].w, from + min(group(g), d - VE), 16);
      }
    f32x4 acc[NJ] = {};
    if (a < P.n) {
      bf16x8 b[RKS][3];
      float f[RKS][8] = {};
      by_rank_kind(rank, [&](auto kind) {
        const float* from = h.parts + (int64_t)(tile * 16 + m) * h.RR;
        auto add = [&](int first, auto count) {      // parts from `first` on, those past the last one read again and not added
          constexpr int N = decltype(count)::value;
          Eight<float> v[N][RKS];
#pragma unroll
          for (int k = 0; k < N; ++k)
#pragma unroll
            for (int s = 0; s < RKS; ++s)
              load_slots<float, decltype(kind)::value>(v[k][s].w, from + min(first + k, h.splits - 1) * (int64_t)h.places * h.RR, 32 * s + 8 * q, rank);
#pragma unroll
          for (int k = 0; k < N; ++k)
#pragma unroll
            for (int s = 0; s < RKS; ++s)
#pragma unroll
              for (int e = 0; e < 8; ++e) f[s][e] += first + k < h.splits ? __builtin_bit_cast(float, v[k][s].w[e]) : 0.f;
        };
        if (h.splits == 1) add(0, std::integral_constant<int, 1>{});
        else
          for (int k = 0; k < h.splits; k += 4) add(k, std::integral_constant<int, 4>{});
      });
#pragma unroll
      for (int s = 0; s < RKS; ++s) {
#pragma unroll
        for (int e = 0; e < 8; ++e) f[s][e] = (once[s] >> e) & 1 ? f[s][e] : 0.f;
        cut(f[s], b[s]);
      }
#pragma unroll
      for (int s = 0; s < RKS; ++s)
#pragma unroll
        for (int j = 0; j < NJ; ++j) {
          Eight<W> v;
          if constexpr (TRANS) v = column<W, 4>(wt[s][j / 4], j % 4); else v = w[s][j];
          if constexpr (std::is_same<W, _Float16>::value) {      // (cut anew for every tile: the pieces of all would not fit the registers)
#pragma unroll
            for (int i = 0; i < 4; ++i) asm volatile("" : "+v"(v.w[i]));
          }
          bf16x8 p[kPieces<W>];
          cut(v, p);
          acc[j] = mma(b[s], p, acc[j]);
        }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (rows[i] < 0) continue;
      Y* out = (Y*)P.out + rows[i] * P.out_stride;
#pragma unroll
      for (int g = 0; g < NG; ++g) {
        const int c = group(g), at = min(c, d - VE);
        Y v[VE];
        __builtin_memcpy(v, base[i][g].w, 16);
#pragma unroll
        for (int e = 0; e < VE; ++e) v[e] = (Y)(acc[g * VE + e][i] + (float)v[e]);
        if (at == c) {
          stream_out(out + c, v);
        } else {
#pragma unroll
          for (int e = 0; e < VE; ++e)
            if (at + e >= c) out[at + e] = v[e];
        }
      }
    }
  }
}

// ---- dA = sum of g x^T, dB = sum of h dy^T: products of 16 (rank) x 16 NJ (columns), the places split over the wavefronts ----
// A lane holds NJ adjacent columns (16 bytes) of eight rows; a tile's operand is one column of all eight, put together from the rows'
// words by one byte permutation a word: no transposition through LDS. Sums of different wavefronts and segments meet in a fixed order.
template <typename X, int RT, bool TRANS>
__device__ __forceinline__ void weight_grad(const AdapterArgs& P, const Plan& plan, const Pieces& h, const void* in, int64_t stride, int d,
                                            int slice, float* out, float* part, f32x4* red) {
  constexpr int NJ = 16 / sizeof(X);
  const Segment seg = plan.segments[blockIdx.y];
  if (seg.a < 0) return;
  const int lane = threadIdx.x & 63, wave = wave_index(), m = lane & 15, q = lane >> 4, rank = P.rank;
  float* to = seg.part < 0 ? out + (int64_t)seg.a * rank * d : part + (int64_t)seg.part * rank * (P.d_in + P.d_out);
  // (lanes past the last column take the last ones again, with the same sums)
  const int c0 = slice * 16 * NJ;
  const X* x = (const X*)in + min(c0 + NJ * m, d - NJ);
  f32x4 acc[RT][NJ] = {};
  // The rows of a step are requested a step ahead, their numbers two; h with the rows where there are registers for that.
  constexpr bool kAhead = RT < 4;
  struct Step { uint32_t v[8][4]; bf16x8 a[kAhead ? RT : 1][3]; };
  auto numbers = [&](int (&row)[8], int p) { __builtin_memcpy(row, plan.rowof + min(p, seg.to - 32) + 8 * q, 32); };
  auto request_h = [&](bf16x8 (&a)[RT][3], int p) {
#pragma unroll
    for (int t = 0; t < RT; ++t)
#pragma unroll
      for (int k = 0; k < 3; ++k) {
        const int r = min(4 * RT * (m >> 2) + 4 * t + (m & 3), rank - 1);      // (rows of the product do not meet)
        __builtin_memcpy(&a[t][k], h.by_rank + (int64_t)(k * h.RR + r) * h.places + min(p, seg.to - 32) + 8 * q, 16);
      }
  };
  auto request = [&](Step& s, const int (&row)[8], int p) {
#pragma unroll
    for (int e = 0; e < 8; ++e) __builtin_memcpy(s.v[e], x + (row[e] ^ (row[e] >> 31)) * stride, 16);
    if constexpr (kAhead) request_h(s.a, p);
  };
  auto multiply = [&](const Step& s, const bf16x8 (&a)[RT][3]) {
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
      bf16x8 b[kPieces<X>];
      cut(column<X, NJ>(s.v, j), b);
#pragma unroll
      for (int t = 0; t < RT; ++t) acc[t][j] = mma(a[t], b, acc[t][j]);
    }
  };
  const int first = seg.from + 32 * wave;
  if (first < seg.to) {
    int row[8];
    Step next;
    numbers(row, first);
    request(next, row, first);
    numbers(row, first + 128);
    for (int p = first; p < seg.to; p += 128) {
      const Step now = next;
      if constexpr (kAhead) {
        request(next, row, p + 128);
        numbers(row, p + 256);
        multiply(now, now.a);
      } else {
        bf16x8 a[RT][3];
        request_h(a, p);
        request(next, row, p + 128);
        numbers(row, p + 256);
        multiply(now, a);
      }
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
  for (int i = threadIdx.x; i < kTiles; i += 256) {
    // columns one after the other (dA), or the four rank indices of a column and those of its other tiles (dB)
    const int k = TRANS ? i / (4 * RT) : i % (16 * NJ), rt = TRANS ? i % (4 * RT) : i / (16 * NJ);
    const int qq = rt / RT, t = rt % RT, r = 4 * rt, at = (t * NJ + k % NJ) * 64 + qq * 16 + k / NJ, col = min(c0 + k / NJ * NJ, d - NJ) + k % NJ;
    const f32x4 v = red[at] + red[kTiles + at];
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (r + e < rank) to[TRANS ? (int64_t)col * rank + r + e : (int64_t)(r + e) * d + col] = v[e];
  }
}

template <typename W, typename Y, int RT>
__global__ __launch_bounds__(256, RT < 4 ? 2 : 1) void k_adapter_weights(AdapterArgs P, Plan plan, Pieces h, Pieces g, int slices_a, float* part) {
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

// ---- rows of less than 16 bytes' worth of elements (d_in or d_out below 8): a thread or a workgroup an element, in fp32 ----
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
__global__ __launch_bounds__(kThreads) void k_narrow_down(AdapterArgs P, const void* in, int64_t stride, int d, float* h) {
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
__global__ __launch_bounds__(kThreads) void k_narrow_up(AdapterArgs P, const float* h, int d) {
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
__global__ __launch_bounds__(kThreads) void k_narrow_weights(AdapterArgs P, const void* in, int64_t stride, int d, const float* h, float* out) {
  const int i = blockIdx.x * kThreads + threadIdx.x, j = blockIdx.y, a = blockIdx.z, r = P.rank;
  if (i >= d) return;
  float sum = 0.f;
  for (int t = 0; t < P.T; ++t)
    if (P.ids[t] == a) sum = fmaf(h[(int64_t)t * r + j], (float)((const X*)in)[t * stride + i], sum);
  out[(int64_t)a * r * d + (TRANS ? (int64_t)i * r + j : (int64_t)j * d + i)] = sum;
}

// ---- host side ----
enum Form { kNarrow, kFew, kSorted };
struct Setup {
  Form form;
  Plan plan;
  Pieces h, g;
  float *part, *narrow_h, *narrow_g;
  int TP, RT, MT;
  size_t total;
};

// Rows of a segment of the weights' gradients, as a power of two: 1024, fewer where that leaves too few workgroups for the chip (but not
// in calls that are one segment, which need no sums to be joined: a launch less), more in long calls (the partial sums are
// rank x (d_in + d_out) floats a segment). us of the gradient with segments of 256 / 512 / 1024 rows, rank 16: one adapter, 2048 rows of 256
// columns 24.2 / 26.0 / 31.8, of 1024 29.4 / 31.4 / 36.7, 4096 rows of 1024 36.1 / 36.3 / 41.0, four adapters 42.3 / 42.7 / 48.8 (rank 32): few
// columns want more workgroups. Of eight adapters whose rows are hardly more than a segment each the sums to join cost more: 2048 rows of
// 2048 columns 38.9 / 37.1 / 36.8, of 4096 (rank 32) 56.1 / 51.4 / 51.1, 4096 rows 77.3 / 77.9 / 70.9. The rule goes by the columns alone:
// how the rows spread is not known on the host.
int segment_shift(const AdapterArgs& a) {
  const int64_t slices = (a.d_in + 127) / 128 + (a.d_out + 127) / 128;
  int k = 10;
  while (k > 8 && a.T > 1024 && slices * ((a.T >> k) + 1) < 512) --k;
  while ((a.T >> k) >= 16) ++k;
  return k;
}

// Shares k of the columns in the narrowing products, each a workgroup of four wavefronts, while the chip has fewer than two workgroups a
// compute unit. A row's units of 128 bytes fall on 4 k wavefronts and what reads the result adds k sums, so k grows as the square root of
// the units: 2 of 1024 bf16 columns, 4 of 4096, 8 of 8192 and more. us of a forward call with one share more in the doubling / this /
// one less: 256 rows of 4096 15.3 / 13.9 / -, 8 rows 9.5 / 8.8 / -, 8 rows of 14336 - / 10.4 / 12.0, 512 of 1024 - / 14.7 / 17.2. The
// backward pass has a launch that adds the shares, none where there is one, and twice the workgroups, for it takes both products. us of the
// gradient with two or more shares by this rule / with one: 777 rows of 4096 31.0 / 33.4, 4096 rows 77.5 / 80.6, 8192 115.1 / 117.8; 2048 rows
// of 2048 39.3 / 35.6, 4096 55.5 / 54.6, 12000 rows of 4096 163 / 154; up to 1024 columns one.
inline int column_splits(const AdapterArgs& a, int d, int tiles, bool backward) {
  const int units = a.dtype == MOEQ_F32 ? (d + 31) / 32 : (d + 63) / 64;
  int k = 1;
  while (k < 8 && units >= (backward ? 32 * k : 8 * k * k) && tiles * k < 512) k *= 2;
  return k;
}

Setup set_up(const AdapterArgs& a, bool backward) {
  Setup s = {};
  s.form = a.d_in < 8 || a.d_out < 8 ? kNarrow : !backward && a.T <= kInlineTokens ? kFew : kSorted;
  s.RT = a.rank <= 16 ? 1 : a.rank <= 32 ? 2 : 4;
  size_t at = 0;
  auto take = [&](size_t bytes) {
    char* q = a.ws ? (char*)a.ws + at : nullptr;
    at += (bytes + 255) / 256 * 256;
    return (void*)q;
  };
  const int RR = 16 * s.RT;
  if (s.form == kNarrow) {
    s.narrow_h = (float*)take((size_t)a.T * a.rank * 4);
    if (backward) s.narrow_g = (float*)take((size_t)a.T * a.rank * 4);
  } else if (s.form == kFew) {
    s.h = Pieces{(float*)take((size_t)8 * a.T * 16 * RR * 4), nullptr, RR, 16 * a.T, column_splits(a, a.d_in, a.T, false)};
  } else {
    Plan& p = s.plan;
    // Rows of a tile: as many as share the weights that are read for them, unless that is mostly padding or leaves compute units without
    // work. us of calls of 4096 columns by tiles of 16 / 32 / 64, rows x adapters: rank 16, 128 x 32 15.1 / 17.2 / 23.2, 1024 x 32 22.3
    // / 22.8 / 25.3, 6144 x 256 74 / 69 / 84, 8192 x 64 83 / 74 / 80, 8192 x 8 74 / 63 / 67, 16384 x 8 135 / 124 / 114; rank 64, 4096 x
    // 8 81 / 70 / 92, 8192 x 8 126 / 115 / 110 (one line for all ranks: 8192 rows lose 4 us at rank 16 and gain 5 at 64). Backward, 8192 x 8 - / 101 / 104, 16384 x 64 - / 213 / 215, 32768 x 8 - / 400 / 392.
    // The narrowing products take 16 MT rows at a time, two or four times their rank at most.
    s.TP = backward ? (a.T >= 16384 && a.T >= 512 * (int64_t)a.n ? 64 : 32)
                    : a.T < 64 * (int64_t)a.n && a.T < 4096 ? 16 : a.T < 256 * (int64_t)a.n || a.T < 8192 ? 32 : 64;
    s.MT = s.TP == 64 ? (s.RT == 1 || backward ? 2 : 4) : s.TP / 16;
    // every bin that has rows adds at most a tile less a row of padding (room: of the largest tile)
    const int pad = (s.TP - 1) * std::min(a.T, a.n + 1), most = 63 * std::min(a.T, a.n + 1), room = a.T + most, room_split = std::min(16, a.T / 256) + most / 256 + 1;
    p.places = (a.T + pad) / s.TP * s.TP;
    p.tiles = p.places / s.TP;
    p.rowof = (int32_t*)take((size_t)room * 4);
    p.tile_adapter = (int32_t*)take((size_t)room / 16 * 4 + 4);
    if (a.T > kPlanOne) p.counts = (int32_t*)take((size_t)((a.T + kSortChunk - 1) / kSortChunk) * (a.n + 1) * 4);
    if (!backward) {
      s.h = Pieces{nullptr, nullptr, RR, p.places, column_splits(a, a.d_in, p.tiles, false)};
      // (several shares only of less than 512 tiles)
      s.h.parts = (float*)take((size_t)std::max(room, 8 * std::min(room, 512 * 64)) * RR * 4);
    } else {
      p.seg_shift = segment_shift(a);
      p.n_segments = a.n + 1 + (p.places >> p.seg_shift);
      p.n_split = a.T <= 1 << p.seg_shift ? 0 : p.places >> p.seg_shift;
      p.segments = (Segment*)take((size_t)(a.n + 1 + room_split) * sizeof(Segment));
      p.split = (Segment*)take((size_t)room_split * sizeof(Segment));
      s.h = Pieces{nullptr, (uint16_t*)take((size_t)room * 3 * RR * 2), RR, p.places, column_splits(a, std::min(a.d_in, a.d_out), p.tiles, true)};
      s.g = s.h;
      s.g.by_rank = (uint16_t*)take((size_t)room * 3 * RR * 2);
      s.h.parts = (float*)take((size_t)std::max(room, 8 * std::min(room, 512 * 64)) * RR * 4);
      s.g.parts = (float*)take((size_t)std::max(room, 8 * std::min(room, 512 * 64)) * RR * 4);
      // (segments of at least 256 rows, at most 16 of them in the rows themselves: segment_shift)
      s.part = (float*)take((size_t)2 * room_split * a.rank * (a.d_in + a.d_out) * 4);
    }
  }
  s.total = at;
  return s;
}

hipError_t launch_plan(const AdapterArgs& a, const Setup& s, hipStream_t st) {
  const bool one = a.T <= kPlanOne;
  const int span = one ? a.T : (int)kSortChunk, waves = sort_waves(span, a.n);
  const int run = (span + waves * 64 - 1) / (waves * 64) * 64;
  if (one) {
    hipLaunchKernelGGL(k_adapter_plan<false>, dim3(1), dim3(waves * 64), 0, st, a.ids, a.T, run, a.n, s.TP, s.plan);
    return hipGetLastError();
  }
  const int chunks = (int)((a.T + kSortChunk - 1) / kSortChunk);
  hipLaunchKernelGGL(k_sort_count, dim3(chunks), dim3(1024), 0, st, a.ids, (int64_t)a.T, a.n, s.plan.counts);
  if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  hipLaunchKernelGGL(k_adapter_plan<true>, dim3(chunks), dim3(waves * 64), 0, st, a.ids, a.T, run, a.n, s.TP, s.plan);
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

template <typename Y, typename W, int RKS, bool TRANS, bool FEW>
hipError_t launch_up(const AdapterArgs& a, const Setup& s, const Pieces& h, int d, hipStream_t st) {
  constexpr int NJ = sizeof(W) == 4 ? 4 : 8;
  const int per = FEW ? 1 : s.TP / 16;
  hipLaunchKernelGGL((k_adapter_up<Y, W, RKS, NJ, TRANS, FEW>), dim3((d + 64 * NJ - 1) / (64 * NJ), FEW ? a.T : s.plan.tiles), dim3(256), 0, st, a, s.plan, s.TP, h, d, per);
  return hipGetLastError();
}
template <typename W, int RT, int MT, bool FEW>
hipError_t launch_down(const AdapterArgs& a, const Setup& s, hipStream_t st) {
  hipLaunchKernelGGL((k_adapter_down<W, RT, MT, FEW>), dim3(FEW ? a.T : s.plan.places / (16 * MT), s.h.splits), dim3(256), 0, st, a, s.plan, s.TP, s.h);
  return hipGetLastError();
}

hipError_t narrow_forward(const AdapterArgs& a, const Setup& s, hipStream_t st) {
  return with_types(a, [&](auto tag, auto ytag) {
    using W = decltype(tag);
    using Y = decltype(ytag);
    hipLaunchKernelGGL((k_narrow_down<W, W, false>), dim3(a.T), dim3(kThreads), 0, st, a, a.x, a.x_stride, a.d_in, s.narrow_h);
    hipLaunchKernelGGL((k_narrow_up<Y, W, false>), dim3((a.d_out + kThreads - 1) / kThreads, a.T), dim3(kThreads), 0, st, a, s.narrow_h, a.d_out);
    return hipGetLastError();
  });
}
hipError_t narrow_backward(const AdapterArgs& a, const Setup& s, hipStream_t st) {
  return with_types(a, [&](auto tag, auto ytag) {
    using W = decltype(tag);
    using Y = decltype(ytag);
    if (a.T) {
      hipLaunchKernelGGL((k_narrow_down<W, W, false>), dim3(a.T), dim3(kThreads), 0, st, a, a.x, a.x_stride, a.d_in, s.narrow_h);
      hipLaunchKernelGGL((k_narrow_down<Y, W, true>), dim3(a.T), dim3(kThreads), 0, st, a, a.dy, a.dy_stride, a.d_out, s.narrow_g);
      if (a.out) hipLaunchKernelGGL((k_narrow_up<Y, W, true>), dim3((a.d_in + kThreads - 1) / kThreads, a.T), dim3(kThreads), 0, st, a, s.narrow_g, a.d_in);
    }
    hipLaunchKernelGGL((k_narrow_weights<W, false>), dim3((a.d_in + kThreads - 1) / kThreads, a.rank, a.n), dim3(kThreads), 0, st, a, a.x, a.x_stride, a.d_in, s.narrow_g, a.dA);
    hipLaunchKernelGGL((k_narrow_weights<Y, true>), dim3((a.d_out + kThreads - 1) / kThreads, a.rank, a.n), dim3(kThreads), 0, st, a, a.dy, a.dy_stride, a.d_out, s.narrow_h, a.dB);
    return hipGetLastError();
  });
}

}  // namespace

size_t adapter_ws_bytes(const AdapterArgs& a, bool backward) {
  AdapterArgs b = a;
  b.ws = nullptr;
  // (what serves the backward pass serves both, and what serves many rows the few that take another form)
  size_t n = set_up(b, false).total;
  if (backward) n = std::max(n, set_up(b, true).total);
  b.T = std::min(b.T, kInlineTokens);
  return std::max(n, set_up(b, false).total);
}

hipError_t launch_adapters_forward(const AdapterArgs& a, hipStream_t st) {
  if (a.T == 0) return hipSuccess;
  const Setup s = set_up(a, false);
  if (s.form == kNarrow) return narrow_forward(a, s, st);
  if (s.form == kSorted)
    if (hipError_t e = launch_plan(a, s, st); e != hipSuccess) return e;
  return with_types(a, [&](auto tag, auto ytag) {
    using W = decltype(tag);
    using Y = decltype(ytag);
    return with_rank(s.RT, [&](auto rt) {
      constexpr int RT = decltype(rt)::value, RKS = RT == 4 ? 2 : 1;
      hipError_t e = s.form == kFew ? launch_down<W, RT, 1, true>(a, s, st) : s.MT == 1 ? launch_down<W, RT, 1, false>(a, s, st)
                   : s.MT == 2 || RT == 1 ? launch_down<W, RT, 2, false>(a, s, st) : launch_down<W, RT, RT == 1 ? 2 : 4, false>(a, s, st);
      if (e != hipSuccess) return e;
      if (s.form == kFew) return launch_up<Y, W, RKS, false, true>(a, s, s.h, a.d_out, st);
      return launch_up<Y, W, RKS, false, false>(a, s, s.h, a.d_out, st);
    });
  });
}

hipError_t launch_adapters_backward(const AdapterArgs& a, hipStream_t st) {
  const Setup s = set_up(a, true);
  if (s.form == kNarrow) return narrow_backward(a, s, st);
  if (hipError_t e = launch_plan(a, s, st); e != hipSuccess) return e;
  return with_types(a, [&](auto tag, auto ytag) {
    using W = decltype(tag);
    using Y = decltype(ytag);
    return with_rank(s.RT, [&](auto rt) {
      constexpr int RT = decltype(rt)::value, RKS = RT == 4 ? 2 : 1, MT = 2;
      if (a.T) {
        const dim3 grid(s.plan.places / (16 * MT), 2 * s.h.splits);
        if (s.h.splits == 1) hipLaunchKernelGGL((k_adapter_down_both<W, Y, RT, MT, true>), grid, dim3(256), 0, st, a, s.plan, s.TP, s.h, s.g);
        else hipLaunchKernelGGL((k_adapter_down_both<W, Y, RT, MT, false>), grid, dim3(256), 0, st, a, s.plan, s.TP, s.h, s.g);
        if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
        if (s.h.splits > 1) hipLaunchKernelGGL(k_adapter_pieces, dim3(s.plan.places / 32, 2), dim3(256), 0, st, s.h, s.g);
        if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
      }
      // (the weights' gradients first: what the products before them read of x and dy may still be in the cache)
      const int sa = (a.d_in + 256 / (int)sizeof(W) - 1) / (256 / (int)sizeof(W)), sb = (a.d_out + 256 / (int)sizeof(Y) - 1) / (256 / (int)sizeof(Y));
      hipLaunchKernelGGL((k_adapter_weights<W, Y, RT>), dim3(sa + sb, s.plan.n_segments), dim3(256), 0, st, a, s.plan, s.h, s.g, sa, s.part);
      if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
      if (s.plan.n_split) {
        const int64_t all = (int64_t)a.rank * (a.d_in + a.d_out);
        hipLaunchKernelGGL(k_adapter_join, dim3((unsigned)std::min<int64_t>((all + 255) / 256, 1024), s.plan.n_split), dim3(256), 0, st, a, s.plan, s.part);
        if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
      }
      if (!a.T || !a.out) return hipSuccess;
      Pieces g = s.g;
      g.splits = 1;
      return launch_up<Y, W, RKS, true, false>(a, s, g, a.d_in, st);
    });
  });
}

}  // namespace moeq
