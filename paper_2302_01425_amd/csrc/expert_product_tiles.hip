// The experts' products (expert_product.hip) by workgroups of four wavefronts: dW, and forward and dx of rows of any alignment
// and of few tiles.
//
// Wide, 128 x 256: 64 x 128 float32 sums per wavefront, 12 fragments of 1 KB read from LDS feed 32 matrix instructions.  A step
// is 64 bytes of k, 24 KB of LDS for both operands, so that two workgroups share a compute unit and one multiplies while the
// other begins, ends or waits: an expert's rows (the k of dW) are few.  For dW of whole, aligned parts, which are loaded
// straight to LDS two steps ahead (three images).
// Middle, 128 x 128 (steps of 128 bytes for rows, which are read along k, of 64 for dW), and Small, 64 x 64 (of 128 bytes), of
// any alignment: operands pass through registers, two steps ahead, to two images; two and four workgroups share a compute
// unit.  Small is for float32, whose matrix instructions take 16 times as long for the same fragments, and where larger tiles
// would leave compute units without work.  What binds the others is the first cache: 16 bytes at any address take twice the
// time of aligned ones (8192 tokens x 2, 8 experts, 2001 -> 3001, bfloat16: 411 us, less than half of that
// without the loads).
#include "expert_tiles.hpp"

namespace topk {
namespace {

constexpr int kThreads = 256;

template <class T>
using Wide = Tile<T, 128, 256, 64>;
template <class T, int STEP>
using Middle = Tile<T, 128, 128, STEP>;
template <class T>
using Small = Tile<T, 64, 64, 128>;

// Sums over `depth` k.  LISTED: rows of k are looked up in `table`, which is filled on the way.
template <class TILE, class IA, class IB, bool LISTED, class LA, class LB>
__device__ __forceinline__ void sum_direct(char* lds, const LA& a, const LB& b, const Table& table, int64_t depth,
                                           typename TILE::Sums& acc) {
  constexpr int kLoads = IA::kParts + IB::kParts;
  const uint32_t lds0 = lds_address(lds);
  const auto fill = [&](int64_t k0) {
    if constexpr (LISTED) {
      if ((k0 & (kTable - 1)) == 0) table.fill<kThreads>(k0, depth);
    }
  };
  const auto there = [&](int64_t k0) {
    if constexpr (LISTED) return table.bits(k0);
    else return 0u;
  };
  const auto issue = [&](int i, int64_t k0, uint32_t bits, int stage) {   // (steps behind the last are loaded as zeros)
    if (i < IA::kParts) a.issue_part(i, k0, depth, lds0 + stage * TILE::kStageBytes, bits);
    else b.issue_part(i - IA::kParts, k0, depth, lds0 + stage * TILE::kStageBytes + IA::kBytes, bits);
  };
#pragma unroll
  for (int stage = 0; stage < 2; ++stage) {
    fill(stage * IA::kStepK);
#pragma unroll
    for (int i = 0; i < kLoads; ++i) issue(i, stage * IA::kStepK, there(stage * IA::kStepK), stage);
  }
  int stage = 0;
  for (int64_t k0 = 0; k0 < depth; k0 += IA::kStepK) {
    wait_stage<kLoads>();
    fill(k0 + 2 * IA::kStepK);
    const uint32_t bits = there(k0 + 2 * IA::kStepK);
    const int other = stage == 0 ? 2 : stage - 1;
    multiply<TILE, IA, IB>(lds + stage * TILE::kStageBytes, acc, [&](int turn, int turns) {
#pragma unroll
      for (int i = turn * kLoads / turns; i < (turn + 1) * kLoads / turns; ++i) issue(i, k0 + 2 * IA::kStepK, bits, other);
      __builtin_amdgcn_sched_barrier(0);
    });
    stage = stage == 2 ? 0 : stage + 1;
  }
  wait_stage<0>();           // (no load may reach LDS that is another workgroup's by then)
}

// float32 sums of four steps, 128 k, are added to the others' as a whole: a sum over k then has roundings of k / 128 additions,
// and those of 128, instead of k in a row.  (16-bit outputs are rounded by more than either.)
template <class TILE, class IA, class IB, bool LISTED, class LA, class LB>
__device__ __forceinline__ void sum_staged(char* lds, LA& a, LB& b, const Table& table, int64_t depth,
                                           typename TILE::Sums& sums) {
  constexpr bool kApart = sizeof(typename TILE::T) == 4;
  typename TILE::Sums part;
  typename TILE::Sums& acc = kApart ? part : sums;
  if constexpr (kApart) clear(part);
  const auto add_part = [&]() {
#pragma unroll
    for (int i = 0; i < TILE::MI; ++i)
#pragma unroll
      for (int j = 0; j < TILE::NJ; ++j) sums[i][j] += part[i][j];
    clear(part);
  };
  const auto load = [&](int set, int64_t k0) {
    if constexpr (LISTED) {
      if ((k0 & (kTable - 1)) == 0) table.fill<kThreads>(k0, depth);
    }
    a.load(set, k0, depth);
    b.load(set, k0, depth);
  };
  load(0, 0);
  load(1, IA::kStepK);
  for (int64_t k0 = 0; k0 < depth; k0 += 2 * IA::kStepK) {
#pragma unroll
    for (int set = 0; set < 2; ++set) {
      const int64_t k = k0 + set * IA::kStepK;
      if (set == 1 && k >= depth) break;
      // (the image that is written was read two steps ago, and a barrier lies between)
      char* image = lds + set * TILE::kStageBytes;
      a.store(set, image, k, depth);
      b.store(set, image + IA::kBytes, k, depth);
      __syncthreads();
      load(set, k + 2 * IA::kStepK);
      multiply<TILE, IA, IB>(image, acc, [](int, int) {});
    }
    if (kApart && (k0 & (2 * IA::kStepK)) != 0) add_part();
  }
  if constexpr (kApart) add_part();
}

template <class TILE, bool B_KC, bool TINY>
__global__ __launch_bounds__(kThreads, 2) void rows_tiles_kernel(RowsArgs g) {
  using T = typename TILE::T;
  __shared__ __attribute__((aligned(1024))) char lds[2 * TILE::kStageBytes];
  Found f;
  if (!find_tile<kThreads>(g.offset, g.n, g.slots, g.first + blockIdx.x, g.col_tiles, TILE::kRows, &f)) return;
  using IA = typename TILE::template A<true>;
  using IB = typename TILE::template B<B_KC>;
  const int64_t n0 = tile_start(f.col, TILE::kCols, g.cols);
  const T* w = static_cast<const T*>(g.w) + f.expert * g.w_expert;
  Staged<IA, kInOrder, TINY> a;
  a.init_rows(g.a, g.a_stride, g.source, g.div, g.limit, f.begin, f.end);
  Staged<IB, kInOrder, TINY> b;
  if constexpr (B_KC) b.init_rows(w, g.w_stride, nullptr, Divisor{}, 0, n0, g.cols);
  else b.init_columns(w, g.w_stride, nullptr, n0, g.cols, 0);
  typename TILE::Sums acc;
  clear(acc);
  sum_staged<TILE, IA, IB, false>(lds, a, b, Table{}, g.depth, acc);
  store_tile(acc, f.begin + TILE::wave_row(), f.end, n0 + TILE::wave_col(), g.cols, g.source, g.div, g.limit,
             static_cast<T*>(g.c), g.cols);
}

// LIST: which operand's rows are found through source (0: neither, 1: A, 2: B)
enum Load { kDirect, kStaged, kTiny };
template <class TILE, int LIST, Load LOAD, bool BOTH>
__global__ __launch_bounds__(kThreads, 2) void weight_tiles_kernel(WeightArgs g) {
  using T = typename TILE::T;
  __shared__ __attribute__((aligned(1024))) char lds[(LOAD == kDirect ? 3 : 2) * TILE::kStageBytes];
  __shared__ int32_t rows[LIST != 0 ? kTable : 1];
  __shared__ uint32_t there[LIST != 0 ? kTable / 32 : 1];
  int e;
  int64_t m0, n0;
  if (!find_weight_tile(g, g.first + blockIdx.x, &e, &m0, &n0)) return;
  int64_t begin, end;
  places(g.offset, e, g.slots, &begin, &end);
  T* c = static_cast<T*>(g.c) + e * g.m * g.cols;
  const char *from_a = static_cast<const char*>(g.a), *from_b = static_cast<const char*>(g.b);
  int64_t m_tiles = g.m_tiles, col_tiles = g.col_tiles;
  if constexpr (BOTH) {
    const bool rows_twice = g.stacked == 1;
    int64_t& at = rows_twice ? m0 : n0;
    (rows_twice ? m_tiles : col_tiles) = g.one;
    if (at >= g.one) {
      at -= g.one;
      (rows_twice ? from_a : from_b) += g.apart;
      c = static_cast<T*>(g.c_up) + e * g.m * g.cols;
    }
  }
  // An expert without places: zeros as one run, not in tiles, whose rows begin and end inside cache lines (31 experts of 2950 x 2919,
  // 534 MB, three of them with one place: 108 us, in tiles 182)
  if (begin == end) {
    store_zeros<kThreads>(c, g.m * g.cols, m0 * col_tiles + n0, m_tiles * col_tiles);
    return;
  }
  m0 = LOAD == kDirect ? m0 * TILE::kRows : tile_start(m0, TILE::kRows, g.m);
  n0 = LOAD == kDirect ? n0 * TILE::kCols : tile_start(n0, TILE::kCols, g.cols);
  using IA = typename TILE::template A<false>;
  using IB = typename TILE::template B<false>;
  constexpr Order kOrderA = LIST == 0 ? kInOrder : LIST == 1 ? kListed : kInOrderWhereListed;
  constexpr Order kOrderB = LIST == 0 ? kInOrder : LIST == 2 ? kListed : kInOrderWhereListed;
  std::conditional_t<LOAD == kDirect, Direct<IA, kOrderA>, Staged<IA, kOrderA, LOAD == kTiny>> a;
  a.init_columns(from_a, g.a_stride, rows, m0, g.m, begin);
  std::conditional_t<LOAD == kDirect, Direct<IB, kOrderB>, Staged<IB, kOrderB, LOAD == kTiny>> b;
  b.init_columns(from_b, g.b_stride, rows, n0, g.cols, begin);
  typename TILE::Sums acc;
  clear(acc);
  const Table table{rows, there, LIST == 0 ? nullptr : (LIST == 1 ? g.a_source : g.b_source) + begin, g.div,
                    LIST == 1 ? g.a_limit : g.b_limit};
  if constexpr (LOAD == kDirect) sum_direct<TILE, IA, IB, LIST != 0>(lds, a, b, table, end - begin, acc);
  else sum_staged<TILE, IA, IB, LIST != 0>(lds, a, b, table, end - begin, acc);
  store_tile(acc, m0 + TILE::wave_row(), g.m, n0 + TILE::wave_col(), g.cols, nullptr, Divisor{}, 0, c, g.cols);
}

template <class TILE, bool TINY>
int rows_tile(RowsArgs g, bool k_contiguous, hipStream_t stream) {
  g.col_tiles = (g.cols + TILE::kCols - 1) / TILE::kCols;
  return in_launches<kThreads>(g, rows_blocks(g, TILE::kRows), [&](const RowsArgs& part, dim3 grid) {
    if (k_contiguous) hipLaunchKernelGGL((rows_tiles_kernel<TILE, true, TINY>), grid, dim3(kThreads), 0, stream, part);
    else hipLaunchKernelGGL((rows_tiles_kernel<TILE, false, TINY>), grid, dim3(kThreads), 0, stream, part);
  });
}

template <class TILE, Load LOAD, bool BOTH>
int weight_tile_of(const WeightArgs& g, int64_t blocks, hipStream_t stream) {
  return in_launches<kThreads>(g, blocks, [&](const WeightArgs& part, dim3 grid) {
    const dim3 block(kThreads);
    if (part.a_source != nullptr) hipLaunchKernelGGL((weight_tiles_kernel<TILE, 1, LOAD, BOTH>), grid, block, 0, stream, part);
    else if (part.b_source != nullptr) hipLaunchKernelGGL((weight_tiles_kernel<TILE, 2, LOAD, BOTH>), grid, block, 0, stream, part);
    else hipLaunchKernelGGL((weight_tiles_kernel<TILE, 0, LOAD, BOTH>), grid, block, 0, stream, part);
  });
}
template <class TILE, Load LOAD>
int weight_tile(WeightArgs g, hipStream_t stream) {
  if (g.c_up == nullptr) {
    const int64_t blocks = split_tiles(&g, TILE::kRows, TILE::kCols);
    return weight_tile_of<TILE, LOAD, false>(g, blocks, stream);
  }
  WeightArgs all = g;
  const int64_t m_tiles = (g.m + TILE::kRows - 1) / TILE::kRows, col_tiles = (g.cols + TILE::kCols - 1) / TILE::kCols;
  g.one = g.stacked == 1 ? m_tiles : col_tiles;
  all.m = m_tiles * TILE::kRows * (g.stacked == 1 ? 2 : 1), all.cols = col_tiles * TILE::kCols * (g.stacked == 1 ? 1 : 2);
  const int64_t blocks = split_tiles(&all, TILE::kRows, TILE::kCols);
  g.m_tiles = all.m_tiles, g.col_tiles = all.col_tiles, g.die_m = all.die_m, g.die_cols = all.die_cols;
  return weight_tile_of<TILE, LOAD, true>(g, blocks, stream);
}
template <class T>
int rows_type(const RowsArgs& g, bool k_contiguous, TileKind kind, hipStream_t stream) {
  // rows shorter than 16 bytes
  if (g.depth < 16 / int(sizeof(T)) || (!k_contiguous && g.cols < 16 / int(sizeof(T))))
    return rows_tile<Small<T>, true>(g, k_contiguous, stream);
  if constexpr (sizeof(T) == 2)
    if (kind == kMiddle) return rows_tile<Middle<T, 128>, false>(g, k_contiguous, stream);
  return rows_tile<Small<T>, false>(g, k_contiguous, stream);
}
template <class T>
int weight_type(const WeightArgs& g, TileKind kind, hipStream_t stream) {
  if (g.m < 16 / int(sizeof(T)) || g.cols < 16 / int(sizeof(T))) return weight_tile<Small<T>, kTiny>(g, stream);
  if constexpr (sizeof(T) == 2) {
    if (kind == kWideDirect) return weight_tile<Wide<T>, kDirect>(g, stream);
    if (kind == kMiddle) return weight_tile<Middle<T, 64>, kStaged>(g, stream);
  }
  return weight_tile<Small<T>, kStaged>(g, stream);
}

}  // namespace

int launch_rows_tiles(int type, const RowsArgs& g, bool k_contiguous, TileKind kind, hipStream_t stream) {
  if (type == kF32) return rows_type<float>(g, k_contiguous, kind, stream);
  if (type == kBF16) return rows_type<bf16>(g, k_contiguous, kind, stream);
  if (type == kF16) return rows_type<f16>(g, k_contiguous, kind, stream);
  return -1;
}

int launch_weight_tiles(int type, const WeightArgs& g, TileKind kind, hipStream_t stream) {
  if (type == kF32) return weight_type<float>(g, kind, stream);
  if (type == kBF16) return weight_type<bf16>(g, kind, stream);
  if (type == kF16) return weight_type<f16>(g, kind, stream);
  return -1;
}

}  // namespace topk
