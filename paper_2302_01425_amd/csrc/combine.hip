// The weighted sum of the experts' rows per token, and its gradient.
//   out[t] = sum_j val[t][j] y[slot[t][j]];   dy[slot[t][j]] = val[t][j] dout[t],  dval[t][j] = <dout[t], y[slot[t][j]]>
// Places outside [0, slots) are left out (dval 0).  Sums in float32, one rounding per output.  Bound by HBM: every row of y
// is read once (vjp: and a row of dy written), every row of out written (dout read) once.  16384 x 2 rows of 2048 bfloat16: 41 us,
// 4.9 TB/s; gradient of 8191 x 8 rows of 1001 float16: 74 us, 3.8 TB/s (a row of an odd number of elements begins inside a line).
#include "common.hpp"
#include "experts.hpp"

namespace topk {
namespace {

constexpr int kThreads = 256;

// A row is cut into parts of 16 bytes, N elements; the last part of a row that is no multiple of N begins N before the end, and
// the elements it shares with the part before are computed (and stored) twice.  So every access is one of 16 bytes.  (With a
// branch to single elements the compiler took the vector loads apart as well: 39 us in the place of 30.)  Rows shorter than N
// elements: SHORT, one lane, element by element.
template <class T, int N, bool SHORT>
__device__ __forceinline__ void load_part(const T* p, int64_t h, float (&v)[N]) {
  if constexpr (SHORT) {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = i < h ? to_f32(p[i]) : 0.0f;
  } else {
    const Packed<T, N> q = load_packed<T, N>(p);
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = to_f32(q.v[i]);
  }
}
template <class T, int N, bool SHORT>
__device__ __forceinline__ void store_part(T* p, int64_t h, const float (&v)[N]) {
  if constexpr (SHORT) {
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (i < h) p[i] = from_f32<T>(v[i]);
  } else {
    Packed<T, N> q;
#pragma unroll
    for (int i = 0; i < N; ++i) q.v[i] = from_f32<T>(v[i]);
    store_packed<T, N>(p, q);
  }
}

// `lanes` lanes (a power of two) per token, of one workgroup: its parts are neighbours in memory; blockIdx.y: the
// slice of a row that is longer.  Two rows of y are on their way at a time (8192 x 8, 1024 columns of bfloat16: 32 us; four 36).
template <class T, bool SHORT>
__global__ __launch_bounds__(kThreads) void combine_fwd_kernel(CombineArgs a, int shift) {
  constexpr int N = 16 / sizeof(T);
  constexpr int kAhead = 2;
  const int lanes = 1 << shift;
  const int64_t t = (int64_t(blockIdx.x) * kThreads + threadIdx.x) >> shift;
  int64_t c = ((a.slice + blockIdx.y) * lanes + (threadIdx.x & (lanes - 1))) * N;
  if (t >= a.rows || c >= a.h) return;
  c = SHORT ? 0 : min(c, a.h - N);
  const T* yp = static_cast<const T*>(a.y) + c;
  float sum[N];
#pragma unroll
  for (int q = 0; q < N; ++q) sum[q] = 0.0f;
  for (int64_t j0 = 0; j0 < a.k; j0 += kAhead) {
    int64_t s[kAhead];
    float w[kAhead], v[kAhead][N];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      s[i] = -1;
      w[i] = 1.0f;
      if (j0 + i < a.k) {
        s[i] = a.slot[t * a.k + j0 + i];
        if (a.val != nullptr) w[i] = a.val[t * a.k + j0 + i];
      }
      if (s[i] >= a.slots) s[i] = -1;
    }
#pragma unroll
    for (int i = 0; i < kAhead; ++i)
      if (s[i] >= 0) load_part<T, N, SHORT>(yp + s[i] * a.y_stride, a.h, v[i]);
#pragma unroll
    for (int i = 0; i < kAhead; ++i)
      if (s[i] >= 0) {
#pragma unroll
        for (int q = 0; q < N; ++q) sum[q] += w[i] * v[i][q];
      }
  }
  store_part<T, N, SHORT>(static_cast<T*>(a.out) + t * a.h + c, a.h, sum);
}

// `lanes` lanes of a wavefront per pair (t, j): the pairs of a token lie side by side, so that its cotangent comes from the
// cache after the first.  Two parts of both rows are on their way at a time.
template <class T, bool SHORT>
__global__ __launch_bounds__(kThreads) void combine_vjp_kernel(CombineArgs a, int shift) {
  constexpr int N = 16 / sizeof(T);
  constexpr int kAhead = 2;
  const int lanes = 1 << shift;
  const int64_t pair = (int64_t(blockIdx.x) * kThreads + threadIdx.x) >> shift;
  if (pair >= a.rows * a.k) return;
  const int64_t t = pair / a.k;
  const int lane = int(threadIdx.x) & (lanes - 1);
  const int64_t s = a.slot[pair];
  const bool there = s >= 0 && s < a.slots;
  const float w = a.val != nullptr ? a.val[pair] : 1.0f;
  const T* tp = static_cast<const T*>(a.t) + t * a.t_stride;
  const T* yp = static_cast<const T*>(a.y) + s * a.y_stride;
  T* dp = static_cast<T*>(a.dy) + s * a.h;
  float dot = 0.0f;
  if (there) {
    const int64_t last = SHORT ? 0 : a.h - N;
    for (int64_t c0 = 0; c0 < a.h; c0 += int64_t(kAhead) * lanes * N) {
      float d[kAhead][N], v[kAhead][N];
#pragma unroll
      for (int i = 0; i < kAhead; ++i) {
        const int64_t c = min(c0 + int64_t(i * lanes + lane) * N, last);
        load_part<T, N, SHORT>(tp + c, a.h, d[i]);
        if (a.dval != nullptr) load_part<T, N, SHORT>(yp + c, a.h, v[i]);
      }
#pragma unroll
      for (int i = 0; i < kAhead; ++i) {
        const int64_t c = c0 + int64_t(i * lanes + lane) * N;
        if (c >= a.h) continue;
        const int64_t from = min(c, last);
        if (a.dval != nullptr) {
          float part = 0.0f;
#pragma unroll
          for (int q = 0; q < N; ++q) part += q >= c - from ? d[i][q] * v[i][q] : 0.0f;
          dot += part;
        }
#pragma unroll
        for (int q = 0; q < N; ++q) d[i][q] *= w;
        store_part<T, N, SHORT>(dp + from, a.h, d[i]);
      }
    }
  }
  if (a.dval == nullptr) return;
  for (int off = lanes / 2; off >= 1; off >>= 1) dot += __shfl_xor(dot, off, kWave);
  if (lane == 0) a.dval[pair] = dot;
}

// lanes of a row, as a power of two: as many as it has parts, up to 2^most
int lanes_shift(int64_t h, int size, int most) {
  int shift = 0;
  while (shift < most && (int64_t(16) << shift) < h * size) ++shift;
  return shift;
}

template <class T>
int fwd_type(const CombineArgs& a, hipStream_t stream) {
  const int shift = lanes_shift(a.h, sizeof(T), 8);
  const int64_t blocks = ((a.rows << shift) + kThreads - 1) / kThreads;
  if (!launchable(blocks * a.slices, kThreads) || a.slices > 65535) return -1;
  const dim3 grid = dim3(unsigned(blocks), unsigned(a.slices)), block(kThreads);
  if (a.h * int64_t(sizeof(T)) < 16) hipLaunchKernelGGL((combine_fwd_kernel<T, true>), grid, block, 0, stream, a, shift);
  else hipLaunchKernelGGL((combine_fwd_kernel<T, false>), grid, block, 0, stream, a, shift);
  return 0;
}
template <class T>
int vjp_type(const CombineArgs& a, hipStream_t stream) {
  const int shift = lanes_shift(a.h, sizeof(T), 6);
  const int64_t blocks = (((a.rows * a.k) << shift) + kThreads - 1) / kThreads;
  if (!launchable(blocks, kThreads)) return -1;
  const dim3 grid = dim3(unsigned(blocks)), block(kThreads);
  if (a.h * int64_t(sizeof(T)) < 16) hipLaunchKernelGGL((combine_vjp_kernel<T, true>), grid, block, 0, stream, a, shift);
  else hipLaunchKernelGGL((combine_vjp_kernel<T, false>), grid, block, 0, stream, a, shift);
  return 0;
}

}  // namespace

int64_t combine_slices(int type, int64_t h) {
  const int size = type == kF32 ? 4 : 2;
  const int64_t bytes = int64_t(16) << lanes_shift(h, size, 8);
  return (h * size + bytes - 1) / bytes;
}

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
