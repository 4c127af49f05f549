// The weighted sum of the experts' rows per token, and its gradient.
//   out[t] = sum_j val[t][j] y[slot[t][j]];   dy[slot[t][j]] = val[t][j] dout[t],  dval[t][j] = <dout[t], y[slot[t][j]]>
// Places outside [0, slots) are left out (dval 0).  Sums in float32, one rounding per output.  Bound by HBM: every row of y
// is read once (vjp: and a row of dy written), every row of out written (dout read) once.
#include "common.hpp"
#include "experts.hpp"

namespace topk {
namespace {

constexpr int kThreads = 256;

// N elements from column c, zeros behind the row's end
template <class T, int N>
__device__ __forceinline__ void load_part(const T* row, int64_t c, int64_t h, float (&v)[N]) {
  if (c + N <= h) {
    const Packed<T, N> q = load_packed<T, N>(row + c);
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = to_f32(q.v[i]);
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = c + i < h ? to_f32(row[c + i]) : 0.0f;
  }
}
template <class T, int N>
__device__ __forceinline__ void store_part(T* row, int64_t c, int64_t h, const float (&v)[N]) {
  if (c + N <= h) {
    Packed<T, N> q;
#pragma unroll
    for (int i = 0; i < N; ++i) q.v[i] = from_f32<T>(v[i]);
    store_packed<T, N>(row + c, q);
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (c + i < h) row[c + i] = from_f32<T>(v[i]);
  }
}

template <class T>
__global__ __launch_bounds__(kThreads) void combine_fwd_kernel(CombineArgs a, int64_t parts) {
  constexpr int N = 16 / sizeof(T);
  const int64_t i = int64_t(blockIdx.x) * kThreads + threadIdx.x;
  if (i >= a.rows * parts) return;
  const int64_t t = i / parts, c = (i - t * parts) * N;
  float sum[N];
#pragma unroll
  for (int q = 0; q < N; ++q) sum[q] = 0.0f;
  for (int64_t j = 0; j < a.k; ++j) {
    const int64_t s = a.slot[t * a.k + j];
    if (s < 0 || s >= a.slots) continue;
    const float w = a.val != nullptr ? a.val[t * a.k + j] : 1.0f;
    float v[N];
    load_part(static_cast<const T*>(a.y) + s * a.y_stride, c, a.h, v);
#pragma unroll
    for (int q = 0; q < N; ++q) sum[q] += w * v[q];
  }
  store_part(static_cast<T*>(a.out) + t * a.h, c, a.h, sum);
}

// one workgroup per token
template <class T>
__global__ __launch_bounds__(kThreads) void combine_vjp_kernel(CombineArgs a) {
  constexpr int N = 16 / sizeof(T);
  __shared__ float part[kThreads / kWave];
  const int64_t t = blockIdx.x;
  const T* tp = static_cast<const T*>(a.t) + t * a.t_stride;
  for (int64_t j = 0; j < a.k; ++j) {
    const int64_t s = a.slot[t * a.k + j];
    const bool there = s >= 0 && s < a.slots;
    const float w = a.val != nullptr ? a.val[t * a.k + j] : 1.0f;
    float dot = 0.0f;
    if (there) {
      for (int64_t c = int64_t(threadIdx.x) * N; c < a.h; c += kThreads * N) {
        float d[N], v[N];
        load_part(tp, c, a.h, d);
        if (a.dval != nullptr) {
          load_part(static_cast<const T*>(a.y) + s * a.y_stride, c, a.h, v);
#pragma unroll
          for (int q = 0; q < N; ++q) dot += d[q] * v[q];
        }
#pragma unroll
        for (int q = 0; q < N; ++q) v[q] = w * d[q];
        store_part(static_cast<T*>(a.dy) + s * a.h, c, a.h, v);
      }
    }
    if (a.dval == nullptr) continue;
    for (int off = kWave / 2; off >= 1; off >>= 1) dot += __shfl_xor(dot, off, kWave);
    if ((threadIdx.x & (kWave - 1)) == 0) part[threadIdx.x / kWave] = dot;
    __syncthreads();
    if (threadIdx.x == 0) {
      float all = 0.0f;
      for (int q = 0; q < kThreads / kWave; ++q) all += part[q];
      a.dval[t * a.k + j] = all;
    }
    __syncthreads();
  }
}

template <class T>
int fwd_type(const CombineArgs& a, hipStream_t stream) {
  const int64_t parts = (a.h * int64_t(sizeof(T)) + 15) / 16;
  const int64_t blocks = (a.rows * parts + kThreads - 1) / kThreads;
  if (blocks >= (int64_t(1) << 31)) return -1;
  hipLaunchKernelGGL(combine_fwd_kernel<T>, dim3(unsigned(blocks)), dim3(kThreads), 0, stream, a, parts);
  return 0;
}
template <class T>
int vjp_type(const CombineArgs& a, hipStream_t stream) {
  hipLaunchKernelGGL(combine_vjp_kernel<T>, dim3(unsigned(a.rows)), dim3(kThreads), 0, stream, a);
  return 0;
}

}  // namespace

int launch_combine_fwd(int type, const CombineArgs& a, hipStream_t stream) {
  if (type == kF32) return fwd_type<float>(a, stream);
  if (type == kBF16) return fwd_type<bf16>(a, stream);
  if (type == kF16) return fwd_type<f16>(a, stream);
  return -1;
}

int launch_combine_vjp(int type, const CombineArgs& a, hipStream_t stream) {
  if (type == kF32) return vjp_type<float>(a, stream);
  if (type == kBF16) return vjp_type<bf16>(a, stream);
  if (type == kF16) return vjp_type<f16>(a, stream);
  return -1;
}

}  // namespace topk
