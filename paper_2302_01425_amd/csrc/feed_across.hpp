// The experts' feed-forward of few tiles where W has one row per k (dx of weights contiguous in k, and the forward pass of turned
// ones): 32 rows x 128 columns, or 64, of W per workgroup, whose four wavefronts share k as in feed_thin.hpp.
//
// Loads go straight to the registers that the matrix instructions read.  A lane takes CW neighbouring columns of every k of its
// half of a step, so that a load reads two rows of 32 CW columns; its i-th columns are those of the i-th instruction, which hence has
// every CW-th column.  In 16 bits the instruction wants eight k of a column in a lane: eight such loads, put together by register halves.
//
// Bound by the time from a load to its use where experts are few, by HBM where they are many: one expert of 1 to 64 places, 2048 -> 1024,
// gated, turned weights: float32 25 us (tiles of 64 rows through LDS 93), bfloat16 18 to 20 (24); 32 experts of 8, float32: 106 us, 5.1
// TB/s of W (165).  float32 sums in one chain per wavefront took 24 and 106 us, with errors (root mean
// square, of that of the sums, random terms) of 5.7e-7 at 4096 k and 1.13e-6 at 16384, where parts of 128 k have 2.1e-7 and 2.3e-7.
#pragma once

#include "feed_forward.hpp"

namespace topk {
namespace {

constexpr int kAcrossThreads = 256, kAcrossWaves = kAcrossThreads / kWave;
constexpr int kAcrossRows = 32;

template <class T, Work WORK, int CW>
__global__ __launch_bounds__(kAcrossThreads, 2) void feed_across_kernel(FeedArgs g) {
  constexpr bool kPair = is_pair(WORK);
  constexpr int N = 16 / int(sizeof(T)), kStepK = 2 * N, kAll = 32 * CW;       // k of a lane and of a step; columns of W
  constexpr int kSpan = kAll / (kPair ? 2 : 1), kSums = WORK == kBoth ? 2 : 1;
  constexpr int kSets = sizeof(T) == 2 ? 8 : 4;  // steps on their way (16 bits with four: 8 % slower, float32 with eight: 4 %)
  __shared__ float lds[kAcrossWaves][kAll][kAcrossRows + 1];
  Found f;
  if (!find_group_tile<kAcrossRows>(g, &f)) return;
  const int lane = int(threadIdx.x) & (kWave - 1), l = lane & 31, half = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(int(threadIdx.x) / kWave);
  // (the last tile of columns overlaps the one before it, and computes the same)
  const int64_t n0 = tile_start(f.col, kSpan, g.cols);
  const char* b = reinterpret_cast<const char*>(static_cast<const T*>(g.w) + f.expert * g.w_expert + n0 + l * CW % kSpan);
  if (kPair && l * CW >= kSpan) b += g.apart;
  // (rows behind the last are read from another one; they are not stored, or stored as zeros)
  int64_t row = min(f.begin + l, f.end - 1);
  if (WORK != kBoth && g.source != nullptr) row = min(int64_t(quotient(max(g.source[row], 0), g.div)), g.limit - 1);
  const char* a = reinterpret_cast<const char*>(static_cast<const T*>(g.a) + row * g.a_stride);
  const auto rows = rows_of_tile<T, 1>(g, f.begin, f.end);
  const int64_t stride = g.w_stride * int64_t(sizeof(T));

  Packed<T, N> va[kSets];
  Packed<T, CW> vb[kSets][N];
  // (float32: sums of 128 k of the wavefront are added to the others' as a whole, as in feed_tiles.hpp.  Such an addition between the
  // instructions of a step measured 10 % more, a loop of 128 k spilled.)
  constexpr bool kApart = sizeof(T) == 4;
  constexpr int kPartSteps = 128 / kStepK;
  f32x16 sum[1][CW], part[1][CW];
  f32x16(&to)[1][CW] = kApart ? part : sum;
  clear(sum);
  clear(part);
  const auto add_part = [&]() {
#pragma unroll
    for (int i = 0; i < CW; ++i) sum[0][i] += part[0][i];
    clear(part);
  };
  // N of k from `k` on, per half
  const auto load = [&](int set, int64_t k) {
    va[set] = load_packed<T, N>(reinterpret_cast<const T*>(a) + k);
    const char* from = b + k * stride;
#pragma unroll
    for (int e = 0; e < N; ++e) vb[set][e] = load_packed<T, CW>(reinterpret_cast<const T*>(from + e * stride));
  };
  const auto multiply = [&](int set) {
    const Fragment<T> fa = __builtin_bit_cast(Fragment<T>, va[set]);
#pragma unroll
    for (int i = 0; i < CW; ++i) {
      Fragment<T> fb;
#pragma unroll
      for (int e = 0; e < N; ++e) fb[e] = vb[set][e].v[i];
#pragma unroll
      for (int q = 0; q < kMma<T>; ++q) to[0][i] = mma(q, fb, fa, to[0][i]);
    }
  };
  const int64_t whole = g.depth / kStepK;
  const int mine = int((whole - wave + kAcrossWaves - 1) / kAcrossWaves);
#pragma unroll 1
  for (int s = 0; s < kSums; ++s) {
    // step wave + 4 i is the wavefront's i-th; those behind its last are read from there, as in feed_thin.hpp
    if (mine > 0) {
      const auto k_of = [&](int i) { return int64_t(wave + min(i, mine - 1) * kAcrossWaves) * kStepK + half * N; };
#pragma unroll
      for (int i = 0; i < kSets; ++i) load(i, k_of(i));
      int i = 0;
      for (; i + kSets <= mine; i += kSets) {
#pragma unroll
        for (int set = 0; set < kSets; ++set) {
          multiply(set);
          load(set, k_of(i + kSets + set));
          __builtin_amdgcn_sched_barrier(0);
        }
        if (kApart && (i + kSets) % kPartSteps == 0) add_part();
      }
#pragma unroll
      for (int set = 0; set < kSets - 1; ++set)
        if (i + set < mine) multiply(set);
    }
    // the rest of the last step: read from before the end, and what it shares with other steps is zero in both operands
    if (whole * kStepK < g.depth && whole % kAcrossWaves == wave) {
      const int64_t k = whole * kStepK + half * N, from = min(k, g.depth - N);
      const int skip = int(min(k - from, int64_t(N)));
      load(0, from);
#pragma unroll
      for (int e = 0; e < N; ++e) {
        va[0].v[e] = e < skip ? T(0.0f) : va[0].v[e];
#pragma unroll
        for (int i = 0; i < CW; ++i) vb[0][e].v[i] = e < skip ? T(0.0f) : vb[0][e].v[i];
      }
      multiply(0);
    }
    if constexpr (kApart) add_part();
    a += g.a_apart, b += g.apart;
  }
#pragma unroll
  for (int i = 0; i < CW; ++i)
#pragma unroll
    for (int x = 0; x < 16; ++x) lds[wave][CW * (x / 4 * 8 + 4 * half + x % 4) + i][l] = sum[0][i][x];
  __syncthreads();
  // 32 columns of the output per wavefront
  constexpr int NJ = kPair ? 2 : 1;
  if (wave * 32 >= kSpan) return;
  f32x16 acc[1][NJ];
#pragma unroll
  for (int j = 0; j < NJ; ++j)
#pragma unroll
    for (int x = 0; x < 16; ++x) {
      const int col = kSpan * j + 32 * wave + x / 4 * 8 + 4 * half + x % 4;
      float v = lds[0][col][l];
#pragma unroll
      for (int o = 1; o < kAcrossWaves; ++o) v += lds[o][col][l];
      acc[0][j][x] = v;
    }
  finish_act<T, T, WORK>(acc, g, rows, f.expert, f.begin, f.end, n0 + 32 * wave, g.cols);
}

template <class T, Work WORK, int CW>
int feed_across(FeedArgs g, hipStream_t stream) {
  constexpr int kSpan = 32 * CW / (is_pair(WORK) ? 2 : 1);
  if (g.cols < kSpan) return -1;
  g.col_tiles = (g.cols + kSpan - 1) / kSpan;
  return in_launches<kAcrossThreads>(g, rows_blocks(g, kAcrossRows), [&](const FeedArgs& part, dim3 grid) {
    hipLaunchKernelGGL((feed_across_kernel<T, WORK, CW>), grid, dim3(kAcrossThreads), 0, stream, part);
  });
}

template <class T>
int across_work(const FeedArgs& g, Work work, bool narrow, hipStream_t stream) {
  const auto of = [&](auto cw) {
    constexpr int CW = decltype(cw)::value;
    if (work == kOut) return feed_across<T, kOut, CW>(g, stream);
    if (work == kSlopes) return feed_across<T, kSlopes, CW>(g, stream);
    if (work == kBoth) return feed_across<T, kBoth, CW>(g, stream);
    return -1;
  };
  if constexpr (sizeof(T) == 4)
    if (!narrow) return of(std::integral_constant<int, 4>{});
  return of(std::integral_constant<int, 2>{});
}

}  // namespace
}  // namespace topk
