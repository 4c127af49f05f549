// The experts' feed-forward by workgroups of four wavefronts, 2 x 2: rows of any alignment and of few tiles.
//
// Of a pair of weights a tile holds as many columns of either: Middle, 128 x 128 sums, is 128 rows x 64 columns of both, 64 x 32 of
// both per wavefront; Small is 64 rows x 64 columns of both, 32 x 32 of both per wavefront.  Without a pair Middle is 128 x 128,
// Small 64 x 64.  Steps of 128 bytes of k pass through registers, two steps ahead, to two images.
//
// Two workgroups per compute unit: bound by reading operands again (some 40 bytes per ns and compute unit) and by whole rounds of
// tiles.  4001 x 2 places, 16 experts, 1001 -> 1515 float16: dx 134 us, 0.36 PFLOP/s; 3001 x 2, 12 experts, 1001 -> 2003, 8 bits: 50 us; 64 x
// 8, 128 experts, 2048 -> 768, gated 8 bits: 59 us, reading W at 6.7 TB/s (partly from the last cache); 1003 x 3, 10 experts, 515 -> 1001
// float32: 92 us, 67 TFLOP/s, matrix units busy 47 % (three workgroups per compute unit with steps of 64 bytes: 96).
#pragma once

#include "feed_forward.hpp"

namespace topk {
namespace {

// kBoth: two sums over k, one after the other.  float32 sums of four steps, 128 k, are added to the others' as a whole (as in
// expert_product_tiles.hip).  8-bit sums are exact.
template <class TILE, class IA, class IB, int SUMS, class LA, class LB>
__device__ __forceinline__ void sum_steps(char* lds, LA& a, LB& b, int64_t depth, int64_t ahead_a, int64_t ahead_b,
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
  const int once = int((depth + IA::kStepK - 1) / IA::kStepK), steps = SUMS * once;
  // k of a step, counted in its sum; steps behind the last are loaded as zeros
  const auto k_of = [&](int step) { return int64_t(SUMS == 2 && step >= once ? step - once : step) * IA::kStepK; };
  const auto load = [&](int set, int step) {
    const bool second = SUMS == 2 && step >= once;
    a.load(set, k_of(step), depth, second ? ahead_a : 0);
    b.load(set, k_of(step), depth, second ? ahead_b : 0);
  };
  load(0, 0);
  load(1, 1);
  for (int s = 0; s < steps; s += 2) {
#pragma unroll
    for (int set = 0; set < 2; ++set) {
      const int step = s + set;
      if (set == 1 && step >= steps) break;
      // (the image that is written was read two steps ago, and a barrier lies between)
      char* image = lds + set * TILE::kStageBytes;
      a.store(set, image, k_of(step), depth);
      b.store(set, image + IA::kBytes, k_of(step), depth);
      __syncthreads();
      load(set, step + 2);
      multiply<TILE, IA, IB>(image, acc, [](int, int) {});
    }
    if (kApart && (s & 2) != 0) add_part();
  }
  if constexpr (kApart) add_part();
}

template <class TILE, bool B_KC, bool TINY, Work WORK, class OUT>
__global__ __launch_bounds__(TILE::kThreads, 2) void feed_tiles_kernel(FeedArgs g) {
  using T = typename TILE::T;
  __shared__ __attribute__((aligned(1024))) char lds[2 * TILE::kStageBytes];
  Found f;
  if (!find_tile<TILE::kThreads>(g.offset, g.n, g.slots, g.first + blockIdx.x, g.col_tiles, TILE::kRows, &f)) return;
  using IA = typename TILE::template A<true>;
  using IB = typename TILE::template B<B_KC>;
  const int64_t n0 = tile_start(f.col, IB::kSpan, g.cols);
  const T* w = static_cast<const T*>(g.w) + f.expert * g.w_expert;
  const int64_t apart = is_pair(WORK) ? g.apart : 0;
  Staged<IA, kInOrder, TINY> a;
  a.init_rows(g.a, g.a_stride, WORK == kBoth ? nullptr : g.source, g.div, g.limit, f.begin, f.end);
  Staged<IB, kInOrder, TINY> b;
  if constexpr (B_KC) b.init_rows(w, g.w_stride, nullptr, Divisor{}, 0, n0, g.cols, apart);
  else b.init_columns(w, g.w_stride, nullptr, n0, g.cols, 0, apart);
  const auto rows = rows_of_tile<T, TILE::MI>(g, f.begin + TILE::wave_row(), f.end);
  typename TILE::Sums acc;
  clear(acc);
  constexpr int kSums = WORK == kBoth ? 2 : 1;
  sum_steps<TILE, IA, IB, kSums>(lds, a, b, g.depth, g.a_apart / int64_t(sizeof(T)), g.apart / int64_t(sizeof(T)), acc);
  finish_act<T, OUT, WORK>(acc, g, rows, f.expert, f.begin + TILE::wave_row(), f.end,
                           n0 + TILE::wave_col() / (is_pair(WORK) ? 2 : 1), g.cols);
}

template <class TILE, bool B_KC, bool TINY, Work WORK, class OUT>
int feed_tile(FeedArgs g, hipStream_t stream) {
  constexpr int kSpan = TILE::template B<B_KC>::kSpan;
  g.col_tiles = (g.cols + kSpan - 1) / kSpan;
  return in_launches<TILE::kThreads>(g, rows_blocks(g, TILE::kRows), [&](const FeedArgs& part, dim3 grid) {
    hipLaunchKernelGGL((feed_tiles_kernel<TILE, B_KC, TINY, WORK, OUT>), grid, dim3(TILE::kThreads), 0, stream, part);
  });
}

template <class T, bool B_KC, Work WORK, class OUT>
int feed_size(const FeedArgs& g, TileKind kind, hipStream_t stream) {
  constexpr bool kPair = is_pair(WORK);
  using Small = Tile<T, 64, kPair ? 128 : 64, 128, kPair>;
  // rows shorter than 16 bytes
  constexpr int kPart = 16 / int(sizeof(T));
  if (g.depth < kPart || (!B_KC && g.cols < kPart)) return feed_tile<Small, B_KC, true, WORK, OUT>(g, stream);
  if constexpr (sizeof(T) != 4)
    if (kind == kMiddle) return feed_tile<Tile<T, 128, 128, 128, kPair>, B_KC, false, WORK, OUT>(g, stream);
  return feed_tile<Small, B_KC, false, WORK, OUT>(g, stream);
}

template <class T>
int feed_work(const FeedArgs& g, bool k_contiguous, Work work, TileKind kind, hipStream_t stream) {
  if constexpr (sizeof(T) == 1) {
    if (!k_contiguous || (work != kPlain && work != kOut)) return -1;
    const auto to = [&](auto out) {
      using OUT = decltype(out);
      if (work == kPlain) return feed_size<T, true, kPlain, OUT>(g, kind, stream);
      return feed_size<T, true, kOut, OUT>(g, kind, stream);
    };
    if (g.out_type == kF32) return to(float{});
    if (g.out_type == kBF16) return to(bf16{});
    if (g.out_type == kF16) return to(f16{});
    return -1;
  } else {
    const auto as = [&](auto kc) {
      constexpr bool KC = decltype(kc)::value;
      if (work == kOut) return feed_size<T, KC, kOut, T>(g, kind, stream);
      if (work == kSlopes) return feed_size<T, KC, kSlopes, T>(g, kind, stream);
      if (work == kBoth) return feed_size<T, KC, kBoth, T>(g, kind, stream);
      return -1;
    };
    return k_contiguous ? as(std::true_type{}) : as(std::false_type{});
  }
}

}  // namespace
}  // namespace topk
