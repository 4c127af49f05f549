// Forward and dx of the experts' products (expert_product.hip) where every row is made of whole, aligned 16-byte parts: tiles
// of 256 x 256 outputs, operands loaded straight to LDS.
//
// A workgroup of eight wavefronts holds the tile's float32 sums in registers, 128 x 64 per wavefront: 12 fragments of 1 KB read
// from LDS feed 32 matrix instructions.  A step is 128 bytes of k (whole cache lines of rows that are contiguous in k), 64 KB
// of LDS for both operands, and lies in two halves: the fragments of a half are read while the other half is multiplied, and
// the loads of the step after the next are issued one by one between the second half's instructions (in a run before them
// they cost 8 % more).  The last tile of an expert's rows is one of 128 rows where it has no more.
//
// Bound by the distance between a step's loads and their use, not by LDS (no bank conflicts): at 8192 tokens x 2 to 32 experts of
// unequal shares, 2048 -> 4096, the matrix units are busy 43 % of the time and the wavefronts wait 40 % of theirs; bfloat16, forward
// 338 us, dx 336, 0.81 PFLOP/s with a seventh of the multiplied rows empty.  One expert of 8192 rows, 8192 -> 8192: 950 to 990 us, 1.11
// to 1.16 PFLOP/s.
#include "expert_tiles.hpp"

namespace topk {
namespace {

constexpr int kThreads = 512;
constexpr int kRows = 256, kCols = 256;    // of a tile (A, B)
constexpr int kStep = 128;                 // bytes of k
constexpr int kStageBytes = (kRows + kCols) * kStep;

// One tile of ROWS x kCols.  The sum starts at step `first` and goes around: where the rows' stride is a large power of two, a
// step of all rows lies in few memory channels, and tiles that start apart use different ones.
template <class T, int ROWS, bool B_KC>
__device__ __forceinline__ void rows_tile(const RowsArgs& g, const Found& f, char* lds) {
  using IA = Image<T, true, ROWS, kThreads, kStep>;
  using IB = Image<T, B_KC, kCols, kThreads, kStep>;
  const int64_t n0 = f.col * kCols;
  const T* w = static_cast<const T*>(g.w) + f.expert * g.w_expert;
  Direct<IA, kInOrder> a;
  a.init_rows(g.a, g.a_stride, g.source, g.div, g.limit, f.begin, f.end);
  Direct<IB, kInOrder> b;
  if constexpr (B_KC) b.init_rows(w, g.w_stride, nullptr, Divisor{}, 0, n0, g.cols);
  else b.init_columns(w, g.w_stride, nullptr, n0, g.cols, 0);

  const uint32_t lds0 = lds_address(lds);
  const int wave = int(threadIdx.x) / kWave;
  const int wm = (wave & 1) * (ROWS / 2), wn = (wave >> 1) * (kCols / 4);
  constexpr int MI = ROWS / 2 / 32, NJ = kCols / 4 / 32;
  f32x16 acc[MI][NJ];
  clear(acc);

  const int steps = int((g.depth + IA::kStepK - 1) / IA::kStepK);
  int at = int(f.col * steps / g.col_tiles);               // the next step to be loaded
  // k of the next step that is loaded; steps behind the last are loaded as zeros
  const auto next = [&](int step) {
    const int64_t k0 = int64_t(step < steps ? at : steps) * IA::kStepK;
    at = at + 1 == steps ? 0 : at + 1;
    return k0;
  };
  constexpr int kLoads = IA::kParts + IB::kParts;
  const auto issue = [&](int i, int64_t k0, int stage) {
    if (i < IA::kParts) a.issue_part(i, k0, g.depth, lds0 + stage * kStageBytes);
    else b.issue_part(i - IA::kParts, k0, g.depth, lds0 + stage * kStageBytes + kRows * kStep);
  };
  Fragment<T> fa[2][2][MI], fb[2][2][NJ];                  // of both halves of a step
  constexpr int kReads = 2 * (MI + NJ);
  const auto read = [&](int i, int stage, int half) {
    const char* la = lds + stage * kStageBytes;
    const int t = i / (MI + NJ), r = i % (MI + NJ);
    if (r < NJ) fb[half][t][r] = IB::read(la + kRows * kStep, wn + 32 * r, 2 * half + t);
    else fa[half][t][r - NJ] = IA::read(la, wm + 32 * (r - NJ), 2 * half + t);
  };
  // a half multiplied; between the instructions the fragments of another half are read, and a step is loaded
  constexpr int kTurns = MI * NJ;
  const auto multiply = [&](int half, int stage, int other, bool load, int64_t k0, int load_stage) {
#pragma unroll
    for (int c = 0; c < kTurns; ++c) {
#pragma unroll
      for (int q = 2 * c; q < 2 * c + 2; ++q) {
        const int t = q / (MI * NJ), i = q / NJ % MI, j = q % NJ;
        acc[i][j] = mma(0, fb[half][t][j], fa[half][t][i], acc[i][j]);
      }
#pragma unroll
      for (int i = c * kReads / kTurns; i < (c + 1) * kReads / kTurns; ++i) read(i, stage, other);
      if (load) {
#pragma unroll
        for (int i = c * kLoads / kTurns; i < (c + 1) * kLoads / kTurns; ++i) issue(i, k0, load_stage);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  int64_t k0 = next(0);
#pragma unroll
  for (int i = 0; i < kLoads; ++i) issue(i, k0, 0);
  wait_stage<0>();
  k0 = next(1);
#pragma unroll
  for (int i = 0; i < kLoads; ++i) issue(i, k0, 1);
#pragma unroll
  for (int i = 0; i < kReads; ++i) read(i, 0, 0);
  for (int step = 0; step < steps; ++step) {
    const int stage = step & 1;
    multiply(0, stage, 1, false, 0, 0);
    // everything of this step is in registers, and the next step is there
    wait_stage<0>();
    k0 = next(step + 2);
    multiply(1, stage ^ 1, 0, true, k0, stage);
  }
  wait_stage<0>();           // (no load may reach LDS that is another workgroup's by then)
  store_tile(acc, f.begin + wm, f.end, n0 + wn, g.cols, g.source, g.div, g.limit, static_cast<T*>(g.c), g.cols);
}

template <class T, bool B_KC>
__global__ __launch_bounds__(kThreads, 2) void rows_large_kernel(RowsArgs g) {
  __shared__ __attribute__((aligned(1024))) char lds[2 * kStageBytes];
  Found f;
  if (!find_tile<kThreads>(g.offset, g.n, g.slots, g.first + blockIdx.x, g.col_tiles, kRows, &f)) return;
  if (f.end - f.begin <= kRows / 2) rows_tile<T, kRows / 2, B_KC>(g, f, lds);
  else rows_tile<T, kRows, B_KC>(g, f, lds);
}

template <class T>
int rows_type(const RowsArgs& g, bool k_contiguous, hipStream_t stream) {
  return in_launches<kThreads>(g, rows_blocks(g, kRows), [&](const RowsArgs& part, dim3 grid) {
    if (k_contiguous) hipLaunchKernelGGL((rows_large_kernel<T, true>), grid, dim3(kThreads), 0, stream, part);
    else hipLaunchKernelGGL((rows_large_kernel<T, false>), grid, dim3(kThreads), 0, stream, part);
  });
}

}  // namespace

int launch_rows_large(int type, RowsArgs g, bool k_contiguous, hipStream_t stream) {
  g.col_tiles = (g.cols + kCols - 1) / kCols;
  if (type == kBF16) return rows_type<bf16>(g, k_contiguous, stream);
  if (type == kF16) return rows_type<f16>(g, k_contiguous, stream);
  return -1;
}

}  // namespace topk
