// What the kernels of the experts' products share: matrix instructions, an expert's places, the cut of the ragged rows into
// tiles, exact division by a constant.
#pragma once

#include <type_traits>

#include "common.hpp"
#include "experts.hpp"

namespace topk {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef f16 f16x8 __attribute__((ext_vector_type(8)));
template <class T>
struct FragmentOf;
template <>
struct FragmentOf<bf16> {
  using type = bf16x8;
};
template <>
struct FragmentOf<f16> {
  using type = f16x8;
};
template <>
struct FragmentOf<float> {
  using type = f32x4;
};
// 16 bytes of k of one row
template <class T>
using Fragment = typename FragmentOf<T>::type;

// 32 x 32 outputs += 32 bytes of k: lane l holds the 16 bytes of k at (l / 32) * 16 of row l % 32 of either operand.
// (float32 takes four instructions, `q`, of one k per lane; which k meets which is the same on both sides.)  Outputs: lane l has
// column l % 32 (a row of the second operand) and, in registers 4 i .. 4 i + 3, rows 8 i + 4 (l / 32) .. of the first.
// The instructions of 16 x 16 outputs reach 1.3 PFLOP/s of bfloat16 and 126 TFLOP/s of float32 on registers alone, these 2.1 PFLOP/s
// and 155 TFLOP/s.
template <class T>
constexpr int kMma = sizeof(T) == 4 ? 4 : 1;
__device__ __forceinline__ f32x16 mma(int, bf16x8 a, bf16x8 b, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ f32x16 mma(int, f16x8 a, f16x8 b, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ f32x16 mma(int q, f32x4 a, f32x4 b, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x2f32(a[q], b[q], c, 0, 0, 0);
}

// x / d for 0 <= x < 2^31: with s = ceil(log2 d) and M = floor(2^(31 + s) / d) + 1, M d = 2^(31 + s) + e with 0 < e <= 2^s, so
// x M / 2^(31 + s) exceeds x / d by less than 1 / d.
struct Divisor {
  uint32_t mul;
  int shift;
};
inline Divisor divisor(int64_t d) {
  int s = 0;
  while ((int64_t(1) << s) < d) ++s;
  return {uint32_t((uint64_t(1) << (31 + s)) / uint64_t(d) + 1), 31 + s};
}
__device__ __forceinline__ int quotient(int x, const Divisor& d) { return int((uint64_t(uint32_t(x)) * d.mul) >> d.shift); }

// [begin, end) of expert e, inside [0, slots) whatever the array holds
__device__ __forceinline__ void places(const int32_t* offset, int e, int64_t slots, int64_t* begin, int64_t* end) {
  *begin = min(max(int64_t(offset[e]), int64_t(0)), slots);
  *end = min(max(int64_t(offset[e + 1]), *begin), slots);
}

constexpr int kDies = 8;

// The experts' rows are cut into tiles of `size` rows, one expert after the other, and every tile of rows meets
// `col_tiles` tiles of columns.  These pairs are dealt to the dies in runs of neighbouring ones (workgroups go to the dies in
// turn): what neighbours share is read by one die's cache, and every die gets a share of every kind of expert.  Eight runs per
// die where there are pairs enough, 32 pairs (a die's compute units) at most.
struct Found {
  int expert;
  int64_t begin, end;      // rows
  int64_t col;             // tile of columns
};
constexpr int kRunMost = 32;
// pair number of workgroup b, `total` or more where there is none
__device__ __forceinline__ int64_t dealt(int64_t b, int64_t total) {
  const int64_t run = min(max(total / (8 * kDies), int64_t(1)), int64_t(kRunMost));
  const int64_t die = b % kDies, i = b / kDies;
  return (i / run * kDies + die) * run + i % run;
}
// Expert, rows and columns of a workgroup's pair, false where there is none.  All threads of the workgroup call it.
template <int kThreads>
__device__ __forceinline__ bool find_tile(const int32_t* offset, int n, int64_t slots, int64_t block, int64_t col_tiles, int size,
                                          Found* f) {
  __shared__ int64_t wave_total[kThreads / kWave];
  __shared__ Found found;
  constexpr int kOwn = kExpertsMax / kThreads;
  const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = tid / kWave;
  int64_t b[kOwn], e[kOwn], mine = 0;
#pragma unroll
  for (int i = 0; i < kOwn; ++i) {
    b[i] = e[i] = 0;
    if (tid * kOwn + i < n) places(offset, tid * kOwn + i, slots, &b[i], &e[i]);
    mine += (e[i] - b[i] + size - 1) / size;
  }
  int64_t scan = mine;
  for (int off = 1; off < kWave; off <<= 1) {
    const int64_t v = __shfl_up(scan, off, kWave);
    if (lane >= off) scan += v;
  }
  if (lane == kWave - 1) wave_total[wave] = scan;
  if (tid == 0) found.expert = -1;
  __syncthreads();
  int64_t start = scan - mine, total = 0;
  for (int w = 0; w < kThreads / kWave; ++w) {
    if (w < wave) start += wave_total[w];
    total += wave_total[w];
  }
  // tiles of rows run fastest within an expert: they share its columns of W
  const int64_t pair = dealt(block, total * col_tiles);
#pragma unroll
  for (int i = 0; i < kOwn; ++i) {
    const int64_t tiles = (e[i] - b[i] + size - 1) / size;
    if (pair >= start * col_tiles && pair < (start + tiles) * col_tiles) {
      const int64_t in = pair - start * col_tiles, first = b[i] + in % tiles * size;
      found = Found{tid * kOwn + i, first, min(first + size, e[i]), in / tiles};
    }
    start += tiles;
  }
  __syncthreads();
  *f = found;
  return f->expert >= 0;
}

// forward and dx: rows of A are places, B is W[e] seen as [n][k] (contiguous in k or in n).  With what a kernel takes beside it, 128
// bytes: arguments of one more line cost the smallest calls 0.3 to 0.5 us.
struct RowsArgs {
  const void* a;
  int64_t a_stride;
  const int32_t* source;
  Divisor div;
  int64_t limit;
  const void* w;
  int64_t w_expert, w_stride;
  const int32_t* offset;
  int64_t slots;
  int n;
  uint32_t first;          // number of the launch's first workgroup
  int64_t cols, depth, col_tiles;
  void* c;
};
static_assert(sizeof(RowsArgs) + sizeof(int) <= 128, "two lines of arguments");
// dW: k runs over an expert's places; one of the two operands goes through `source`
struct WeightArgs {
  const void *a, *b;
  int64_t a_stride, b_stride;
  const int32_t *a_source, *b_source;
  Divisor div;
  int64_t a_limit, b_limit;
  const int32_t* offset;
  int64_t slots;
  int n;
  uint32_t first;          // number of the launch's first workgroup
  int64_t m, cols;
  void* c;
  // tiles, and those of a die (split_tiles)
  int64_t m_tiles = 0, col_tiles = 0, die_m = 0, die_cols = 0;
};
// Every die gets an eighth of every expert's tiles, since experts differ in their rows: a rectangle of the tiles, that of 1 x 8, 2 x
// 4, 4 x 2 or 8 x 1 such rectangles that reads least, or an eighth of the tiles in row order (die_cols 0) where rectangles would
// leave a die more than a sixteenth above that.  Returns the number of workgroups.
inline int64_t split_tiles(WeightArgs* g, int64_t rows, int64_t cols) {
  g->m_tiles = (g->m + rows - 1) / rows;
  g->col_tiles = (g->cols + cols - 1) / cols;
  const int64_t tiles = g->m_tiles * g->col_tiles;
  int64_t share = (tiles + kDies - 1) / kDies, best = 0;
  g->die_m = share;
  for (int d = 1; d <= kDies; d *= 2) {
    const int64_t m = (g->m_tiles + d - 1) / d, c = (g->col_tiles + kDies / d - 1) / (kDies / d);
    const int64_t read = m * rows + c * cols;
    if (m * c * kDies * 16 > tiles * 17 || (best != 0 && read >= best)) continue;
    best = read;
    g->die_m = m;
    g->die_cols = c;
    share = m * c;
  }
  return g->n * share * kDies;
}
// Expert and tile of workgroup b, false where there is none.
__device__ __forceinline__ bool find_weight_tile(const WeightArgs& g, uint32_t b, int* expert, int64_t* m, int64_t* col) {
  const uint32_t die = b % kDies, i = b / kDies, cols = uint32_t(g.col_tiles), die_m = uint32_t(g.die_m);
  if (g.die_cols == 0) {
    const uint32_t e = i / die_m, tile = die * die_m + i - e * die_m;
    *expert = int(e);
    *m = tile / cols;
    *col = tile % cols;
  } else {
    const uint32_t die_cols = uint32_t(g.die_cols), share = die_m * die_cols, across = (cols + die_cols - 1) / die_cols;
    const uint32_t e = i / share, at = i - e * share;
    *expert = int(e);
    *m = die / across * die_m + at / die_cols;
    *col = die % across * die_cols + at % die_cols;
  }
  return *m < g.m_tiles && *col < g.col_tiles;
}
// workgroups for all pairs: as many tiles of rows as there can be, and room for the last runs
inline int64_t rows_blocks(const RowsArgs& g, int size) {
  return (g.slots / size + min(int64_t(g.n), g.slots)) * g.col_tiles + kDies * kRunMost;
}
// launch(g, grid) for workgroups 0 .. blocks - 1 of kThreads threads, in as many launches as that takes (of whole turns of the
// dies).  Returns -1 where their numbers do not fit 32 bits.
template <int kThreads, class ARGS, class LAUNCH>
int in_launches(ARGS g, int64_t blocks, LAUNCH launch) {
  constexpr int64_t kMost = (int64_t(1) << 31) / kThreads;
  static_assert(kMost % kDies == 0, "workgroup b is on die b % kDies");
  if (blocks >= (int64_t(1) << 32)) return -1;
  for (int64_t b = 0; b < blocks; b += kMost) {
    g.first = uint32_t(b);
    launch(g, dim3(unsigned(min(blocks - b, kMost))));
  }
  return 0;
}

// few rows per expert, limit > 0; W contiguous in n: of 32 columns at least
int launch_rows_few(int type, const RowsArgs& g, bool k_contiguous, hipStream_t stream);
int launch_rows_large(int type, RowsArgs g, bool k_contiguous, hipStream_t stream);
// tiles of expert_product_tiles.hip; kWideDirect: dW of whole, aligned parts only.  float32 takes kSmall
enum TileKind { kSmall, kMiddle, kWideDirect };
int launch_rows_tiles(int type, const RowsArgs& g, bool k_contiguous, TileKind kind, hipStream_t stream);
int launch_weight_tiles(int type, const WeightArgs& g, TileKind kind, hipStream_t stream);

}  // namespace topk
