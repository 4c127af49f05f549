// The experts' feed-forward where larger tiles would leave compute units without work: 32 rows x 32 columns of either weight of a
// pair (64 without a pair) per workgroup, whose four wavefronts share k.  W contiguous in k, rows of any alignment.
//
// What bounds such calls is the time from a load to its use, times the steps of k: so every wavefront takes a quarter of the steps
// and has three of them on their way, straight to the registers that the matrix instructions read, without LDS or barriers.  The
// instructions of 16 x 16 outputs have 64 bytes of k of 16 rows at a time, so that a load reads 16 runs of 64 bytes (those of 32 x
// 32 outputs would read 32 runs of 32, and the first cache takes as long for each).  The wavefronts' sums meet in LDS.
//
// Gated, bfloat16: 32 x 8 places, 2048 -> 1024: 51 us, 5.3 TB/s of W, bound by HBM (64 rows per tile: 68); 1 x 32 12.2 us.
#pragma once

#include "feed_forward.hpp"

namespace topk {
namespace {

constexpr int kThinThreads = 256, kThinWaves = kThinThreads / kWave;
constexpr int kThinRows = 32, kThinStep = 128, kThinSets = 3;

// the last 16 - `skip` bytes of a part, zeros before them
template <class T>
__device__ __forceinline__ Fragment<T> behind_skip(const Fragment<T>& v, int skip) {
  typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
  u32x4 w = __builtin_bit_cast(u32x4, v);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int b = min(max(skip - 4 * i, 0), 4);
    w[i] = b == 4 ? 0u : w[i] & (~0u << (8 * b));
  }
  return __builtin_bit_cast(Fragment<T>, w);
}

// 16 x 16 outputs += 64 bytes of k: lane l holds the 16 bytes of k at (l / 16) * 16 of row l % 16 of either operand.  Outputs: lane l
// has column l % 16 (a row of the second operand) and rows 4 (l / 16) .. of the first.
__device__ __forceinline__ f32x4 mma16(int, bf16x8 a, bf16x8 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ f32x4 mma16(int, f16x8 a, f16x8 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ f32x4 mma16(int q, f32x4 a, f32x4 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x4f32(a[q], b[q], c, 0, 0, 0);
}
__device__ __forceinline__ i32x4 mma16(int, i32x4 a, i32x4 b, i32x4 c) {
  return __builtin_amdgcn_mfma_i32_16x16x64_i8(a, b, c, 0, 0, 0);
}

// kB: blocks of 16 columns of W, half of them of either weight of a pair
template <class T, class OUT, Work WORK, int kB>
__global__ __launch_bounds__(kThinThreads) void feed_thin_kernel(FeedArgs g) {
  constexpr int N = 16 / int(sizeof(T)), kParts = kThinStep / 64, kStepK = kThinStep / int(sizeof(T)), kPartK = 64 / int(sizeof(T));
  constexpr bool kPair = is_pair(WORK);
  constexpr int kA = 2, kSpan = 16 * kB / (kPair ? 2 : 1);      // blocks of 16 rows; columns of the output
  using Sum = std::conditional_t<sizeof(T) == 1, int, float>;
  __shared__ Sum lds[kThinWaves][16 * kB][kThinRows + 1];
  Found f;
  if (!find_group_tile<kThinRows>(g, &f)) return;
  const int lane = int(threadIdx.x) & (kWave - 1), l = lane & 15, quarter = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(int(threadIdx.x) / kWave);
  const int64_t n0 = f.col * kSpan;
  const T* w = static_cast<const T*>(g.w) + f.expert * g.w_expert;
  // (rows and columns behind the last are read from another one; they are not stored, or stored as zeros)
  const T *pa[kA], *pb[kB];
#pragma unroll
  for (int j = 0; j < kB; ++j) {
    const int64_t col = min(n0 + 16 * (kPair ? j % (kB / 2) : j) + l, g.cols - 1);
    const char* from = reinterpret_cast<const char*>(w + col * g.w_stride + quarter * N);
    pb[j] = reinterpret_cast<const T*>(kPair && j >= kB / 2 ? from + g.apart : from);
  }
#pragma unroll
  for (int i = 0; i < kA; ++i) {
    int64_t row = min(f.begin + 16 * i + l, f.end - 1);
    if (g.source != nullptr) row = min(int64_t(quotient(max(g.source[row], 0), g.div)), g.limit - 1);
    pa[i] = static_cast<const T*>(g.a) + row * g.a_stride + quarter * N;
  }

  const auto rows = rows_of_tile<T, 1>(g, f.begin, f.end);
  Fragment<T> va[kThinSets][kParts][kA], vb[kThinSets][kParts][kB];
  // (float32: sums of kThinSets steps, 96 k of the wavefront, are added to the others' as a whole, as in feed_tiles.hpp)
  constexpr bool kApart = sizeof(T) == 4;
  std::conditional_t<sizeof(T) == 1, i32x4, f32x4> sum[kA][kB] = {}, part[kA][kB] = {};
  auto& to = kApart ? part : sum;
  const auto add_part = [&]() {
#pragma unroll
    for (int i = 0; i < kA; ++i)
#pragma unroll
      for (int j = 0; j < kB; ++j) sum[i][j] += part[i][j], part[i][j] = {};
  };
  const auto load = [&](int set, int64_t k0) {
#pragma unroll
    for (int t = 0; t < kParts; ++t) {
#pragma unroll
      for (int i = 0; i < kA; ++i) va[set][t][i] = __builtin_bit_cast(Fragment<T>, (load_packed<T, N>(pa[i] + k0 + t * kPartK)));
#pragma unroll
      for (int j = 0; j < kB; ++j) vb[set][t][j] = __builtin_bit_cast(Fragment<T>, (load_packed<T, N>(pb[j] + k0 + t * kPartK)));
    }
  };
  const auto multiply = [&](int set) {
#pragma unroll
    for (int t = 0; t < kParts; ++t)
#pragma unroll
      for (int q = 0; q < kMma<T>; ++q)
#pragma unroll
        for (int i = 0; i < kA; ++i)
#pragma unroll
          for (int j = 0; j < kB; ++j) to[i][j] = mma16(q, vb[set][t][j], va[set][t][i], to[i][j]);
  };
  // whole steps: step wave + 4 i is the wavefront's i-th, and those behind its last are read from there (without branches, so that
  // the waits count the loads of later steps out)
  const int whole = int(g.depth / kStepK), mine = (whole - wave + kThinWaves - 1) / kThinWaves;
  if (mine > 0) {
    const auto k_of = [&](int i) { return int64_t(wave + min(i, mine - 1) * kThinWaves) * kStepK; };
#pragma unroll
    for (int s = 0; s < kThinSets; ++s) load(s, k_of(s));
    int i = 0;
    for (; i + kThinSets <= mine; i += kThinSets) {
#pragma unroll
      for (int s = 0; s < kThinSets; ++s) {
        multiply(s);
        load(s, k_of(i + kThinSets + s));
        __builtin_amdgcn_sched_barrier(0);
      }
      if constexpr (kApart) add_part();
    }
#pragma unroll
    for (int s = 0; s < kThinSets - 1; ++s)
      if (i + s < mine) multiply(s);
  }
  // the rest of the last step: a part that crosses the end is read from before it, and what it shares with the one before is zero
  // in both operands
  if (g.depth % kStepK != 0 && whole % kThinWaves == wave) {
#pragma unroll
    for (int t = 0; t < kParts; ++t) {
      const int64_t k = int64_t(whole) * kStepK + t * kPartK, mine_k = k + quarter * N;
      const int64_t over = min(max(mine_k + N - g.depth, int64_t(0)), mine_k);
      const int skip = int(min(over, int64_t(N))) * int(sizeof(T));
#pragma unroll
      for (int i = 0; i < kA; ++i)
        va[0][t][i] = behind_skip<T>(__builtin_bit_cast(Fragment<T>, (load_packed<T, N>(pa[i] + k - over))), skip);
#pragma unroll
      for (int j = 0; j < kB; ++j)
        vb[0][t][j] = behind_skip<T>(__builtin_bit_cast(Fragment<T>, (load_packed<T, N>(pb[j] + k - over))), skip);
    }
    multiply(0);
  }
  if constexpr (kApart) add_part();
#pragma unroll
  for (int i = 0; i < kA; ++i)
#pragma unroll
    for (int j = 0; j < kB; ++j)
#pragma unroll
      for (int r = 0; r < 4; ++r) lds[wave][16 * j + 4 * quarter + r][16 * i + l] = sum[i][j][r];
  __syncthreads();
  if (wave > 0) return;
  // (laid out as the instructions of 32 x 32 outputs leave them; columns of another block that is not there repeat this one's)
  constexpr int NJ = kPair || kB == 4 ? 2 : 1;
  std::conditional_t<sizeof(T) == 1, i32x16, f32x16> acc[1][NJ];
#pragma unroll
  for (int j = 0; j < NJ; ++j)
#pragma unroll
    for (int x = 0; x < 16; ++x) {
      const int col = (kPair ? kSpan : 32) * j + (x / 4 * 8 + 4 * (lane >> 5) + x % 4) % min(kSpan, 32);
      Sum v = lds[0][col][lane & 31];
#pragma unroll
      for (int o = 1; o < kThinWaves; ++o) v += lds[o][col][lane & 31];
      acc[0][j][x] = v;
    }
  finish_act<T, OUT, WORK>(acc, g, rows, f.expert, f.begin, f.end, n0, min(n0 + kSpan, g.cols));
}

template <class T, class OUT, Work WORK, int kB>
int feed_thin_cols(FeedArgs g, hipStream_t stream) {
  constexpr int kSpan = 16 * kB / (is_pair(WORK) ? 2 : 1);
  g.col_tiles = (g.cols + kSpan - 1) / kSpan;
  return in_launches<kThinThreads>(g, rows_blocks(g, kThinRows), [&](const FeedArgs& part, dim3 grid) {
    hipLaunchKernelGGL((feed_thin_kernel<T, OUT, WORK, kB>), grid, dim3(kThinThreads), 0, stream, part);
  });
}
template <class T, class OUT, Work WORK>
int feed_thin(const FeedArgs& g, bool narrow, hipStream_t stream) {
  return narrow ? feed_thin_cols<T, OUT, WORK, 2>(g, stream) : feed_thin_cols<T, OUT, WORK, 4>(g, stream);
}

template <class T>
int thin_work(const FeedArgs& g, Work work, bool narrow, hipStream_t stream) {
  if constexpr (sizeof(T) == 1) {
    const auto to = [&](auto out) {
      using OUT = decltype(out);
      return work == kPlain ? feed_thin<T, OUT, kPlain>(g, narrow, stream) : feed_thin<T, OUT, kOut>(g, narrow, stream);
    };
    if (work != kPlain && work != kOut) return -1;
    return g.out_type == kF32 ? to(float{}) : g.out_type == kBF16 ? to(bf16{}) : to(f16{});
  } else {
    if (work == kOut) return feed_thin<T, T, kOut>(g, narrow, stream);
    if (work == kSlopes) return feed_thin<T, T, kSlopes>(g, narrow, stream);
    return -1;
  }
}

}  // namespace
}  // namespace topk
