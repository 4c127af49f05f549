// The experts' feed-forward where every row is made of whole, aligned 16-byte parts: tiles of 256 x 256 sums (128 columns of either
// weight of a pair), operands loaded straight to LDS.
//
// A workgroup of four wavefronts, one per SIMD, holds the tile's sums in registers, 128 x 128 per wavefront: 8 fragments of 1 KB read
// from LDS feed 16 matrix instructions.  A step is 128 bytes of k (whole cache lines of rows that are contiguous in k), 32 KB of
// LDS for either operand: two stages of A, three of B, since weights come from HBM and have two steps to arrive.  The fragments of
// 32 bytes of k are read while those of the 32 before are multiplied, and loads are issued one by one between the instructions.
//
// Bound by the matrix instructions and the clock they leave where k is long (8192 rows, 8192 -> 4096, gated: bfloat16 830 to 954 us,
// 1.15 to 1.32 PFLOP/s; 8 bits 458 to 472 us, 2.33 to 2.40 POP/s), by 8 to 9 us of start and end per tile where it is not (8192 x 2 places, 32
// experts, 2048 -> 2048, gated: 310 to 327 us, 0.84 to 0.89 PFLOP/s, matrix units busy 42 %; slopes 364; dx 313; 8 bits 200, plain to 4096
// 207).  Steps of 64 bytes read half lines and measured slower; tiles that a workgroup takes one after the other spilled.
#pragma once

#include "feed_forward.hpp"

namespace topk {
namespace {

constexpr int kLargeThreads = 256;
constexpr int kLargeRows = 256, kLargeCols = 256;     // of a tile: rows of A, columns of the operands of B together
constexpr int kLargeStep = 128;                       // bytes of k
constexpr int kStagesA = 2, kStagesB = 3;
constexpr int kStageA = kLargeRows * kLargeStep, kStageB = kLargeCols * kLargeStep;
constexpr int kLargeBytes = kStagesA * kStageA + kStagesB * kStageB;

// The steps of one operand in the order in which they are loaded.  A sum starts at step `at` and goes around: where the rows'
// stride is a large power of two, a step of all rows lies in few memory channels, and tiles that start apart use different
// ones.  With two sums the steps of the second follow those of the first, `apart` bytes away.  Steps behind the last are loaded
// from the first's place; nothing reads them.
template <class LOAD, int SUMS, bool WHOLE>
struct Steps {
  using IMAGE = typename LOAD::Image;
  LOAD load;
  int at, left, once, steps;
  int64_t depth, apart;
  int64_t k0, offset, ahead;         // of the step that is loaded: k, bytes

  __device__ __forceinline__ void next() {
    const bool second = SUMS == 2 && at >= once;
    k0 = left > 0 ? int64_t(second ? at - once : at) * IMAGE::kStepK : 0;
    ahead = second && left > 0 ? apart : 0;
    offset = k0 * (IMAGE::kKC ? int64_t(sizeof(typename IMAGE::Type)) : load.stride) + ahead;
    at = at + 1 == steps ? 0 : at + 1;
    --left;
  }
  __device__ __forceinline__ void issue(int i, uint32_t to) const {
    if constexpr (WHOLE) {
      const int wave = __builtin_amdgcn_readfirstlane(int(threadIdx.x) / kWave);
      load_to_lds(load.p[i] + offset, to + (i * IMAGE::kThreads + wave * kWave) * 16);
    } else {
      load.issue_part(i, k0, depth, to, 0, ahead);
    }
  }
};

// A tile.  Of fewer than 256 rows only `high` blocks of 32 per wavefront are read and multiplied.  WHOLE: the rows of k are whole
// steps.
template <class T, bool B_KC, Work WORK, class OUT, bool WHOLE>
__global__ __launch_bounds__(kLargeThreads, 1) void feed_large_kernel(FeedArgs g) {
  __shared__ __attribute__((aligned(1024))) char lds[kLargeBytes];
  using IA = Image<T, true, kLargeRows, kLargeThreads, kLargeStep>;
  using IB = Image<T, B_KC, kLargeCols, kLargeThreads, kLargeStep, is_pair(WORK)>;
  constexpr int MI = kLargeRows / 2 / 32, NJ = kLargeCols / 2 / 32, kSums = WORK == kBoth ? 2 : 1;
  Found f;
  if (!find_group_tile<kLargeRows>(g, &f)) return;
  const int64_t n0 = f.col * IB::kSpan;
  const T* w = static_cast<const T*>(g.w) + f.expert * g.w_expert;
  Steps<Direct<IB, kInOrder>, kSums, WHOLE> b;
  const int64_t apart = is_pair(WORK) ? g.apart : 0;
  if constexpr (B_KC) b.load.init_rows(w, g.w_stride, nullptr, Divisor{}, 0, n0, g.cols, apart);
  else b.load.init_columns(w, g.w_stride, nullptr, n0, g.cols, 0, apart);
  Steps<Direct<IA, kInOrder>, kSums, WHOLE> a;
  const int once = int((g.depth + IA::kStepK - 1) / IA::kStepK), steps = kSums * once;
  a.once = b.once = once, a.steps = b.steps = a.left = b.left = steps, a.depth = b.depth = g.depth;
  a.at = b.at = int(f.col * steps / g.col_tiles), a.apart = g.a_apart, b.apart = g.apart;

  const uint32_t to_a = lds_address(lds), to_b = to_a + kStagesA * kStageA;
  const char* lds_b = lds + kStagesA * kStageA;
  const auto load_b = [&](int stage) {
    b.next();
#pragma unroll
    for (int i = 0; i < IB::kParts; ++i) b.issue(i, to_b + stage * kStageB);
  };
  const auto load_a = [&](int stage) {
    a.next();
#pragma unroll
    for (int i = 0; i < IA::kParts; ++i) a.issue(i, to_a + stage * kStageA);
  };
  const int wave = int(threadIdx.x) / kWave;
  const int high = int(f.end - f.begin + 63) / 64;
  const int wm = (wave & 1) * 32 * high, wn = (wave >> 1) * (kLargeCols / 2);
  const int64_t m0 = f.begin + wm, m_end = min(f.end, m0 + 32 * high);
  load_b(0);               // (before the rows of A are looked up)
  const auto rows = rows_of_tile<T, MI>(g, m0, m_end);
  a.load.init_rows(g.a, g.a_stride, WORK == kBoth ? nullptr : g.source, g.div, g.limit, f.begin, f.end);
  load_a(0);
  load_b(1);
  load_a(1);

  std::conditional_t<sizeof(T) == 1, i32x16, f32x16> acc[MI][NJ];
  clear(acc);
  wait_stage<IA::kParts + IB::kParts>();
  // the sum, for one number of blocks (branches between the instructions would cost the loop 40 %)
  const auto sum = [&](auto blocks) {
    constexpr int kHigh = decltype(blocks)::value, kReads = kHigh + NJ, kTurns = kHigh * NJ / 2;
    Fragment<T> fa[2][kHigh], fb[2][NJ];
    const auto read = [&](int i, const char* sa, const char* sb, int t) {
      if (i < NJ) fb[t & 1][i] = IB::read(sb, wn + 32 * i, t);
      else fa[t & 1][i - NJ] = IA::read(sa, wm + 32 * (i - NJ), t);
    };
    // the fragments t multiplied; between the instructions those of `other` are read, and COUNT loads are issued
    const auto multiply = [&](int t, const char* sa, const char* sb, int other, auto count, auto issue) {
      constexpr int kLoads = decltype(count)::value;
#pragma unroll
      for (int c = 0; c < kTurns; ++c) {
#pragma unroll
        for (int q = 2 * c; q < 2 * c + 2; ++q) {
          const int i = q / NJ, j = q % NJ;
          acc[i][j] = mma(0, fb[t & 1][j], fa[t & 1][i], acc[i][j]);
        }
#pragma unroll
        for (int i = c * kReads / kTurns; i < (c + 1) * kReads / kTurns; ++i) read(i, sa, sb, other);
#pragma unroll
        for (int i = c * kLoads / kTurns; i < (c + 1) * kLoads / kTurns; ++i) issue(i);
        __builtin_amdgcn_sched_barrier(0);
      }
    };
    const auto none = [](int) {};
    const std::integral_constant<int, 0> zero{};
    const std::integral_constant<int, IA::kParts * kHigh / MI> loads_a{};
    const std::integral_constant<int, IB::kParts> loads_b{};
#pragma unroll
    for (int i = 0; i < kReads; ++i) read(i, lds, lds_b, 0);
    int stage_a = 0, stage_b = 0;
    for (int step = 0; step < steps; ++step) {
      const char *sa = lds + stage_a * kStageA, *sb = lds_b + stage_b * kStageB;
      const int after_b = stage_b + 1 == kStagesB ? 0 : stage_b + 1, last_b = stage_b == 0 ? kStagesB - 1 : stage_b - 1;
      // (the stage of B before this one was done with before the last barrier)
      b.next();
      multiply(0, sa, sb, 1, loads_b, [&](int i) { b.issue(i, to_b + last_b * kStageB); });
      multiply(1, sa, sb, 2, zero, none);
      multiply(2, sa, sb, 3, zero, none);
      // everything of this step is in registers, and the next step is there
      wait_stage<IB::kParts>();
      a.next();
      multiply(3, lds + (stage_a ^ 1) * kStageA, lds_b + after_b * kStageB, 0, loads_a,
               [&](int i) { a.issue(i, to_a + stage_a * kStageA); });
      stage_a ^= 1, stage_b = after_b;
    }
  };
  if (high == 4) sum(std::integral_constant<int, 4>{});
  else if (high == 3) sum(std::integral_constant<int, 3>{});
  else if (high == 2) sum(std::integral_constant<int, 2>{});
  else sum(std::integral_constant<int, 1>{});
  wait_stage<0>();           // (no load may reach LDS that is another workgroup's by then)
  finish_act<T, OUT, WORK>(acc, g, rows, f.expert, m0, m_end, n0 + wn / (is_pair(WORK) ? 2 : 1), g.cols);
}

template <class T, bool B_KC, Work WORK, class OUT>
int feed_large(FeedArgs g, hipStream_t stream) {
  constexpr int kSpan = is_pair(WORK) ? kLargeCols / 2 : kLargeCols;
  g.col_tiles = (g.cols + kSpan - 1) / kSpan;
  return in_launches<kLargeThreads>(g, rows_blocks(g, kLargeRows), [&](const FeedArgs& part, dim3 grid) {
    const bool whole = part.depth * int64_t(sizeof(T)) % kLargeStep == 0;
    if (whole) hipLaunchKernelGGL((feed_large_kernel<T, B_KC, WORK, OUT, true>), grid, dim3(kLargeThreads), 0, stream, part);
    else hipLaunchKernelGGL((feed_large_kernel<T, B_KC, WORK, OUT, false>), grid, dim3(kLargeThreads), 0, stream, part);
  });
}

template <class T>
int large_work(const FeedArgs& g, bool k_contiguous, Work work, hipStream_t stream) {
  if constexpr (sizeof(T) == 1) {
    if (!k_contiguous || (work != kPlain && work != kOut)) return -1;
    const auto to = [&](auto out) {
      using OUT = decltype(out);
      if (work == kPlain) return feed_large<T, true, kPlain, OUT>(g, stream);
      return feed_large<T, true, kOut, OUT>(g, stream);
    };
    if (g.out_type == kF32) return to(float{});
    if (g.out_type == kBF16) return to(bf16{});
    if (g.out_type == kF16) return to(f16{});
    return -1;
  } else {
    const auto as = [&](auto kc) {
      constexpr bool KC = decltype(kc)::value;
      if (work == kOut) return feed_large<T, KC, kOut, T>(g, stream);
      if (work == kSlopes) return feed_large<T, KC, kSlopes, T>(g, stream);
      if (work == kBoth) return feed_large<T, KC, kBoth, T>(g, stream);
      return -1;
    };
    return k_contiguous ? as(std::true_type{}) : as(std::false_type{});
  }
}

}  // namespace
}  // namespace topk
