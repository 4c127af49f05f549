// Rows as 8-bit integers: with a the largest magnitude of a row, scale = a / 127 and q = 127 x / a rounded to the nearest integer,
// ties to even, of the exact quotient.
//
// 127 x / a is taken in float32 as v = x (127 / a), off by less than 127 * 2^-23.  Where v is within 2e-5 of a half H, the sign of H a -
// 127 x decides: with t the float32 product 127 x and t + l the exact one, H a - t is at most 2^-13 a and a multiple of 2^-26 a, so that
// a fused operation gives it exactly, and subtracting l keeps the sign.  Of 16-bit
// values one in some 300 is such an element: half of the largest has the quotient 63.5.
// Rows whose largest magnitude is below 2^-100 or above 2^120, where such terms fall out of float32's range, are divided in float64.
//
// x is read once, a row stays in the registers of one wavefront or workgroup; rows that do not fit are read twice.  8192 x 4096
// float32 26.3 us, 6.4 TB/s (partly from the last cache); 8192 x 2048 bfloat16 15.6 us, 3.2 TB/s, bound by some 15 instructions per
// element; few rows by the launch.  One branch for a part of a row and its elements in float64 together measured 15 % more, float64
// in a loop over memory 40 % more.
#include "feed_forward.hpp"

namespace topk {
namespace {

constexpr int kThreads = 256;
constexpr int kHeld = 8;             // parts of 16 bytes of a row that a thread holds

__device__ __forceinline__ int8_t nearest(float x, float a, float r) {
  const float v = x * r;
  float w = rintf(v);
  if (__builtin_expect(fabsf(v - w) > 0.5f - 2e-5f, 0)) {
    const float side = v > w ? 1.0f : -1.0f, t = 127.0f * x, l = __builtin_fmaf(127.0f, x, -t);
    const float beyond = side * (l - __builtin_fmaf(w + 0.5f * side, a, -t));      // of 127 x behind the half
    const bool even = rintf(0.5f * w) == 0.5f * w;
    if (beyond > 0.0f || (beyond == 0.0f && !even)) w += side;
  }
  return int8_t(int(w));
}
__device__ __forceinline__ int8_t nearest_divided(float x, float a) { return int8_t(int(rint(127.0 * double(x) / double(a)))); }

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
__device__ __forceinline__ void store_part(int8_t* q, const Packed<T, N>& p, float a, float r) {
  Packed<int8_t, N> out;
#pragma unroll
  for (int j = 0; j < N; ++j) out.v[j] = nearest(to_f32(p.v[j]), a, r);
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
  if (at == 0) g.scale[row] = finite ? a / 127.0f : __builtin_nanf("");
  if (tiny || !finite || a < 0x1p-100f || a > 0x1p120f) {
#pragma unroll 1
    for (int64_t i = at; i < g.h; i += ALONG) q[i] = finite && a > 0.0f ? nearest_divided(to_f32(x[i]), a) : int8_t(0);
    return;
  }
  const float r = 127.0f / a;
#pragma unroll
  for (int i = 0; i < kHeld; ++i) {
    const int64_t p = i * ALONG + at;
    if (p < parts) store_part<T, N>(q + part_start<T, N>(p * N, g.h), held[i], a, r);
  }
#pragma unroll 1
  for (int64_t p = int64_t(kHeld) * ALONG + at; p < parts; p += ALONG) {
    const int64_t i = part_start<T, N>(p * N, g.h);
    store_part<T, N>(q + i, load_packed<T, N>(x + i), a, r);
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
