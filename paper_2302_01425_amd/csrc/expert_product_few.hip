// Forward and dx of the experts' products (expert_product.hip) for experts of few rows: one pass over W, which is all there is to
// read, by as many wavefronts as keep its loads on their way.
//
// A workgroup takes kRows rows of an expert and a few columns, its four wavefronts shares of k, and the sums meet by a butterfly
// that halves the values at every step, then in LDS.  No matrix instructions: they would multiply 32 rows of which kRows at most are
// there (for float32 that costs more than the loads), and no LDS images: a row of W is used by one workgroup.
//
// Bound by HBM and, for the smallest calls, by the launch and the search of the expert (5 us).  One token to two of 8 experts, W not in
// a cache, 2048 -> 4096: bfloat16 11.3 us, 3.0 TB/s, dx 12.9; float32 16.8 us, 4.0 TB/s, dx 28.1.
#include "expert_product.hpp"

namespace topk {
namespace {

constexpr int kThreads = 256, kWaves = kThreads / kWave;
constexpr int kRows = 4;
constexpr int kColsAlong = 4;        // W contiguous in k: columns of a workgroup, a lane holds 16 bytes of k of each
constexpr int kColsAcross = 32;      // W contiguous in n: columns of a workgroup, a lane holds 16 bytes of them for N k

// N values from p on as float, the first `skip` of them as zeros
template <class T, int N>
__device__ __forceinline__ void load_part(const T* p, int skip, float (&v)[N]) {
  const Packed<T, N> q = load_packed<T, N>(p);
#pragma unroll
  for (int i = 0; i < N; ++i) v[i] = i < skip ? 0.0f : to_f32(q.v[i]);
}

// Sums over the lanes that differ in the bits LAST .. 32 of their number: each of them ends up with COUNT / (64 / LAST) of the values,
// from the returned one on.
template <int COUNT, int LAST, int S = 32>
__device__ __forceinline__ int halve(float* v, int lane) {
  if constexpr (S < LAST) {
    return 0;
  } else {
    const bool upper = (lane & S) != 0;
#pragma unroll
    for (int i = 0; i < COUNT / 2; ++i) {
      const float keep = upper ? v[i + COUNT / 2] : v[i], send = upper ? v[i] : v[i + COUNT / 2];
      v[i] = keep + __shfl_xor(send, S, kWave);
    }
    return (upper ? COUNT / 2 : 0) + halve<COUNT / 2, LAST, S / 2>(v, lane);
  }
}

template <class T, bool KC>
__global__ __launch_bounds__(kThreads) void few_rows_kernel(RowsArgs g, int turns) {
  constexpr int N = 16 / int(sizeof(T));
  constexpr int kCols = KC ? kColsAlong : kColsAcross;
  __shared__ float sums[2][kWaves][kRows * kCols];
  Found f;
  if (!find_tile<kThreads>(g.offset, g.n, g.slots, g.first + blockIdx.x, g.col_tiles, kRows, &f)) return;
  const int lane = int(threadIdx.x) & (kWave - 1), wave = int(threadIdx.x) / kWave;
  const T* w = static_cast<const T*>(g.w) + f.expert * g.w_expert;
  // rows that are not there are read from another row, and not stored, or stored as zeros
  const T* x[kRows];
#pragma unroll
  for (int r = 0; r < kRows; ++r) {
    int64_t row = min(f.begin + r, f.end - 1);
    if (g.source != nullptr) row = min(int64_t(quotient(max(g.source[row], 0), g.div)), g.limit - 1);
    x[r] = static_cast<const T*>(g.a) + row * g.a_stride;
  }

  const auto finish = [&](int set, int64_t n0) {
    const int64_t row = f.begin + threadIdx.x / kCols, col = n0 + threadIdx.x % kCols;
    if (row >= f.end || col >= g.cols) return;
    float v = 0.0f;
#pragma unroll
    for (int i = 0; i < kWaves; ++i) v += sums[set][i][threadIdx.x];
    if (g.source != nullptr && !(g.source[row] >= 0 && quotient(g.source[row], g.div) < g.limit)) v = 0.0f;
    static_cast<T*>(g.c)[row * g.cols + col] = from_f32<T>(v);
  };

  if constexpr (KC) {
    constexpr int64_t kChunk = kWave * N;
    for (int turn = 0; turn < turns; ++turn) {
      const int64_t n0 = (f.col * turns + turn) * kCols;
      if (n0 >= g.cols) break;
      const T* p[kCols];
#pragma unroll
      for (int c = 0; c < kCols; ++c) p[c] = w + min(n0 + c, g.cols - 1) * g.w_stride;
      float acc[kCols * kRows] = {};
      const auto add = [&](const float (&a)[kCols][N], const float (&b)[kRows][N]) {
#pragma unroll
        for (int i = 0; i < N; ++i)
#pragma unroll
          for (int c = 0; c < kCols; ++c)
#pragma unroll
            for (int r = 0; r < kRows; ++r) acc[c * kRows + r] += a[c][i] * b[r][i];
      };
      int64_t k0 = wave * kChunk;
#pragma unroll 2
      for (; k0 + kChunk <= g.depth; k0 += kWaves * kChunk) {
        float a[kCols][N], b[kRows][N];
#pragma unroll
        for (int c = 0; c < kCols; ++c) load_part<T, N>(p[c] + k0 + lane * N, 0, a[c]);
#pragma unroll
        for (int r = 0; r < kRows; ++r) load_part<T, N>(x[r] + k0 + lane * N, 0, b[r]);
        add(a, b);
      }
      // (the part that crosses the end begins N before it; what it shares with the one before counts there)
      if (k0 + lane * N < g.depth) {
        const int64_t k = min(k0 + lane * N, g.depth - N);
        const int skip = int(k0 + lane * N - k);
        float a[kCols][N], b[kRows][N];
#pragma unroll
        for (int c = 0; c < kCols; ++c) load_part<T, N>(p[c] + k, skip, a[c]);
#pragma unroll
        for (int r = 0; r < kRows; ++r) load_part<T, N>(x[r] + k, skip, b[r]);
        add(a, b);
      }
      const int at = halve<kCols * kRows, 4>(acc, lane);
      acc[0] += __shfl_xor(acc[0], 2, kWave);
      acc[0] += __shfl_xor(acc[0], 1, kWave);
      if ((lane & 3) == 0) sums[turn & 1][wave][at % kRows * kCols + at / kRows] = acc[0];
      __syncthreads();               // (and the sums of the turn before are read)
      if (threadIdx.x < kRows * kCols) finish(turn & 1, n0);
    }
  } else {
    constexpr int kAcross = kCols / N, kDown = kWave / kAcross;      // lanes across the columns, and along k
    const int64_t n0 = min(f.col * kCols, g.cols - kCols);
    const T* p = w + n0 + lane % kAcross * N;
    const int64_t down = lane / kAcross * N;
    float acc[kRows * N] = {};
    constexpr int64_t kChunk = kDown * N;
    constexpr int kAtATime = sizeof(T) == 4 ? 4 : 1;       // (a part is N loads)
    int64_t k0 = wave * kChunk;
#pragma unroll kAtATime
    for (; k0 + kChunk <= g.depth; k0 += kWaves * kChunk) {
      float a[N][N], b[kRows][N];
#pragma unroll
      for (int i = 0; i < N; ++i) load_part<T, N>(p + (k0 + down + i) * g.w_stride, 0, a[i]);
#pragma unroll
      for (int r = 0; r < kRows; ++r) load_part<T, N>(x[r] + k0 + down, 0, b[r]);
#pragma unroll
      for (int i = 0; i < N; ++i)
#pragma unroll
        for (int r = 0; r < kRows; ++r)
#pragma unroll
          for (int q = 0; q < N; ++q) acc[r * N + q] += a[i][q] * b[r][i];
    }
    for (int i = 0; i < N; ++i) {
      const int64_t k = k0 + down + i;
      if (k >= g.depth) break;
      float a[N];
      load_part<T, N>(p + k * g.w_stride, 0, a);
#pragma unroll
      for (int r = 0; r < kRows; ++r) {
        const float b = to_f32(x[r][k]);
#pragma unroll
        for (int q = 0; q < N; ++q) acc[r * N + q] += a[q] * b;
      }
    }
    const int at = halve<kRows * N, kAcross>(acc, lane);
#pragma unroll
    for (int i = 0; i < kRows * N / kDown; ++i) {
      const int r = (at + i) / N, q = (at + i) % N;
      sums[0][wave][r * kCols + lane % kAcross * N + q] = acc[i];
    }
    __syncthreads();
    if (threadIdx.x < kRows * kCols) finish(0, n0);
  }
}
template <class T>
int few_type(RowsArgs g, bool k_contiguous, hipStream_t stream) {
  if (g.depth < 16 / int(sizeof(T)) || (!k_contiguous && g.cols < kColsAcross)) return -1;
  // W contiguous in k: several times the columns where some four workgroups per compute unit are left (2048 -> 4096, one place
  // each in two experts, bfloat16: one, two, four turns 15.5, 13.9, 12.1 us; 4096 -> 1024: 8.5, 10.2, 14.0)
  int64_t turns = 1;
  if (k_contiguous) {
    const int64_t all = (g.slots / kRows + min(int64_t(g.n), g.slots)) * ((g.cols + kColsAlong - 1) / kColsAlong);
    turns = max(int64_t(1), min(all / 1024, int64_t(4)));
  }
  const int64_t cols = k_contiguous ? kColsAlong * turns : kColsAcross;
  g.col_tiles = (g.cols + cols - 1) / cols;
  return in_launches<kThreads>(g, rows_blocks(g, kRows), [&](const RowsArgs& part, dim3 grid) {
    if (k_contiguous) hipLaunchKernelGGL((few_rows_kernel<T, true>), grid, dim3(kThreads), 0, stream, part, int(turns));
    else hipLaunchKernelGGL((few_rows_kernel<T, false>), grid, dim3(kThreads), 0, stream, part, int(turns));
  });
}

}  // namespace

int launch_rows_few(int type, const RowsArgs& g, bool k_contiguous, hipStream_t stream) {
  if (type == kF32) return few_type<float>(g, k_contiguous, stream);
  if (type == kBF16) return few_type<bf16>(g, k_contiguous, stream);
  if (type == kF16) return few_type<f16>(g, k_contiguous, stream);
  return -1;
}

}  // namespace topk
