// Rows as 8-bit integers: with a the largest magnitude of a row, scale = a / 127 and q = 127 x / a rounded to the nearest integer,
// ties to even, of the exact quotient.
//
// 127 x / a is taken in float32 as x (127 / a), off by less than 127 * 2^-23; within 2e-5 of a half it is divided in float64, whose
// quotient of two float32 numbers lies on the same side of every half as the exact one (two such numbers, 24 bits each, are
// either equal to it or off by at least 2^-33).  One branch for
// all elements of a part, with float64 for all of them, measured 15 % more.  x is read once, a row stays in the registers of one
// wavefront or workgroup; rows that do not fit are read twice.  8192 x 2048 bfloat16: 15.8 us, 3.2 TB/s; bound by some 15
// instructions per element, few rows by the launch.
#include "feed_forward.hpp"

namespace topk {
namespace {

constexpr int kThreads = 256;
constexpr int kHeld = 8;             // parts of 16 bytes of a row that a thread holds

__device__ __forceinline__ int8_t nearest(float x, float a, float r) {
  const float v = x * r, w = rintf(v);
  int q = int(w);
  if (__builtin_expect(!(fabsf(v - w) < 0.5f - 2e-5f), 0)) q = int(rint(127.0 * double(x) / double(a)));
  return int8_t(q);
}

// Of the 16 bytes of a row from element i on, which cross its end: those before it (h >= N).
template <class T, int N>
__device__ __forceinline__ int64_t part_start(int64_t i, int64_t h) {
  return min(i, h - N);
}

template <class T, int N>
__device__ __forceinline__ uint32_t largest(const Packed<T, N>& p) {
  uint32_t top = 0;
#pragma unroll
  for (int j = 0; j < N; ++j) top = max(top, __builtin_bit_cast(uint32_t, to_f32(p.v[j])) & 0x7fffffffu);
  return top;
}
template <class T, int N>
__device__ __forceinline__ void store_part(int8_t* q, const Packed<T, N>& p, float a, float r, bool finite) {
  Packed<int8_t, N> out;
#pragma unroll
  for (int j = 0; j < N; ++j) out.v[j] = finite && a > 0.0f ? nearest(to_f32(p.v[j]), a, r) : int8_t(0);
  store_packed<int8_t, N>(q, out);
}

// ALONG threads take a row: a wavefront, or the workgroup.
template <class T, int ALONG>
__global__ __launch_bounds__(kThreads) void quantise_kernel(QuantiseArgs g, int64_t first) {
  constexpr int N = 16 / int(sizeof(T));
  __shared__ uint32_t tops[kThreads / kWave];
  const int at = int(threadIdx.x) % ALONG;
  const int64_t row = first + int64_t(blockIdx.x) * (kThreads / ALONG) + threadIdx.x / ALONG;
  if (row >= g.m) return;              // (a whole wavefront; with ALONG 256 the workgroup)
  const T* x = static_cast<const T*>(g.x) + row * g.x_stride;
  int8_t* q = g.q + row * g.h;
  const int64_t parts = (g.h + N - 1) / N;
  const bool tiny = g.h < N;
  Packed<T, N> held[kHeld];
  uint32_t top = 0;
  if (tiny) {
    if (at < g.h) top = __builtin_bit_cast(uint32_t, to_f32(x[at])) & 0x7fffffffu;
  } else {
#pragma unroll
    for (int i = 0; i < kHeld; ++i) {
      const int64_t p = i * ALONG + at;
      if (p < parts) held[i] = load_packed<T, N>(x + part_start<T, N>(p * N, g.h));
      else held[i] = Packed<T, N>{};
    }
#pragma unroll
    for (int i = 0; i < kHeld; ++i) top = max(top, largest<T, N>(held[i]));
    for (int64_t p = int64_t(kHeld) * ALONG + at; p < parts; p += ALONG)
      top = max(top, largest<T, N>(load_packed<T, N>(x + part_start<T, N>(p * N, g.h))));
  }
  for (int off = kWave / 2; off > 0; off >>= 1) top = max(top, uint32_t(__shfl_xor(int(top), off, kWave)));
  if constexpr (ALONG > kWave) {
    if (threadIdx.x % kWave == 0) tops[threadIdx.x / kWave] = top;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kThreads / kWave; ++w) top = max(top, tops[w]);
  }
  // (the bits of magnitudes are in their order, infinity behind all numbers and NaN behind it)
  const bool finite = top < 0x7f800000u;
  const float a = __builtin_bit_cast(float, top);
  // where 127 / a is infinite every element is divided in float64
  const float r = a < 0x1p-118f ? __builtin_inff() : 127.0f / a;
  if (at == 0) g.scale[row] = finite ? a / 127.0f : __builtin_nanf("");
  if (tiny) {
    if (at < g.h) q[at] = finite && a > 0.0f ? nearest(to_f32(x[at]), a, r) : int8_t(0);
    return;
  }
#pragma unroll
  for (int i = 0; i < kHeld; ++i) {
    const int64_t p = i * ALONG + at;
    if (p < parts) store_part<T, N>(q + part_start<T, N>(p * N, g.h), held[i], a, r, finite);
  }
  for (int64_t p = int64_t(kHeld) * ALONG + at; p < parts; p += ALONG) {
    const int64_t i = part_start<T, N>(p * N, g.h);
    store_part<T, N>(q + i, load_packed<T, N>(x + i), a, r, finite);
  }
}

template <class T>
int quantise_type(const QuantiseArgs& g, hipStream_t stream) {
  constexpr int64_t kRowsOfLaunch = int64_t(1) << 22;
  // A wavefront or a workgroup per row (us, from a graph of calls): 1 x 512 bfloat16 2.7 / 2.8, 1024 x 512 3.4 / 4.4; 1 x 2048 4.3 / 2.8,
  // 1024 x 2048 6.6 / 4.9, 4096 x 2048 9.2 / 11.9; 1024 x 4096 10.6 / 6.3; float32 1 x 1024 3.0 / 2.4, 2048 x 1024 3.9 / 4.9
  constexpr int64_t kPart = kWave * (16 / int64_t(sizeof(T)));
  const bool wave = g.h <= kPart || (g.h <= kHeld * kPart && g.m > g.h);
  for (int64_t r = 0; r < g.m; r += kRowsOfLaunch) {
    const int64_t rows = min(g.m - r, kRowsOfLaunch);
    if (wave) {
      const dim3 grid(unsigned((rows + kThreads / kWave - 1) / (kThreads / kWave)));
      hipLaunchKernelGGL((quantise_kernel<T, kWave>), grid, dim3(kThreads), 0, stream, g, r);
    } else {
      hipLaunchKernelGGL((quantise_kernel<T, kThreads>), dim3(unsigned(rows)), dim3(kThreads), 0, stream, g, r);
    }
  }
  return 0;
}

}  // namespace

int launch_quantise(int type, const QuantiseArgs& g, hipStream_t stream) {
  if (type == kF32) return quantise_type<float>(g, stream);
  if (type == kBF16) return quantise_type<bf16>(g, stream);
  if (type == kF16) return quantise_type<f16>(g, stream);
  return -1;
}

}  // namespace topk
