// The experts' products over ragged groups of rows.  With expert e's places [offset[e], offset[e + 1]):
//   forward   out[s] = W[e] x[r(s)]          (h -> ho)
//   dx        dx[s]  = W[e]^T dout[s]        (ho -> h)
//   dW        dW[e]  = sum_s dout[s] x[r(s)]^T, zeros for an expert without places
// r(s) = source[s] / k, or s where the rows are in expert order already.  All three are
//   C(m, n) = sum_k A(m, k) B(n, k)
// with A, B each either contiguous in k or contiguous in m / n, and a row of x found through `source`.  Matrix instructions
// with float32 sums, one rounding per output element.
#include "expert_product.hpp"

namespace topk {
namespace {

// One operand: element (row, k) at p[row * stride + k] (contiguous in k) or p[k * stride + row]; the index that `stride`
// belongs to goes through source / div where there is one, and is out where that is not in [0, limit).
template <class T>
struct Side {
  const T* p;
  int64_t stride;
  const int32_t* source;
  Divisor div;
  int64_t limit;
  __device__ __forceinline__ const T* at(int64_t i) const {        // null: out
    if (source != nullptr) {
      const int pair = source[i];
      if (pair < 0) return nullptr;
      i = quotient(pair, div);
    }
    return i < limit ? p + i * stride : nullptr;
  }
};

constexpr int kThreads = kProductThreads;
constexpr int kTile = 128;             // rows and columns of a workgroup's outputs
constexpr int kStep = 64;              // bytes of k per step
constexpr int kPitch = kStep + 16;     // bytes between rows in LDS

// 16 bytes per thread and turn of one operand's step (k0 .. k0 + 64 bytes), rows [r0, r0 + 128) up to `rows`, to LDS as
// [row][k]
template <class T, bool KC>
__device__ __forceinline__ void stage(const Side<T>& s, int64_t r0, int64_t rows, int64_t k0, int64_t kend, char* lds) {
  constexpr int N = 16 / sizeof(T);
  constexpr int kRow = KC ? kStep / 16 : kTile / N;      // 16-byte parts along the contiguous direction
#pragma unroll
  for (int i = 0; i < kTile * kStep / 16 / kThreads; ++i) {
    const int part = int(threadIdx.x) + i * kThreads;
    const int across = part / kRow, along = (part % kRow) * N;
    const int64_t outer = (KC ? r0 : k0) + across, inner = (KC ? k0 : r0) + along;
    const int64_t outer_end = KC ? rows : kend, inner_end = KC ? kend : rows;
    T v[N];
    const T* p = outer < outer_end ? s.at(outer) : nullptr;
    if (p != nullptr && inner + N <= inner_end) {
      const Packed<T, N> q = *reinterpret_cast<const Packed<T, N>*>(p + inner);
#pragma unroll
      for (int j = 0; j < N; ++j) v[j] = q.v[j];
    } else {
#pragma unroll
      for (int j = 0; j < N; ++j) v[j] = p != nullptr && inner + j < inner_end ? p[inner + j] : T(0.0f);
    }
    if constexpr (KC) {
      T* to = reinterpret_cast<T*>(lds + across * kPitch) + along;
#pragma unroll
      for (int j = 0; j < N; ++j) to[j] = v[j];
    } else {
#pragma unroll
      for (int j = 0; j < N; ++j) reinterpret_cast<T*>(lds + (along + j) * kPitch)[across] = v[j];
    }
  }
}

// C[m][n], m in [m0, m0 + 128) below m_end, n likewise, to c[m * c_stride + n]
template <class T, bool A_KC, bool B_KC>
__device__ __forceinline__ void tile_product(const Side<T>& a, const Side<T>& b, int64_t m0, int64_t m_end, int64_t n0,
                                             int64_t n_end, int64_t k_begin, int64_t k_end, T* c, int64_t c_stride) {
  __shared__ __attribute__((aligned(16))) char lds_a[kTile * kPitch];
  __shared__ __attribute__((aligned(16))) char lds_b[kTile * kPitch];
  constexpr int kStepK = kStep / sizeof(T);
  const int lane = int(threadIdx.x) & (kWave - 1), wave = int(threadIdx.x) / kWave;
  const int wm = (wave & 1) * 64, wn = (wave >> 1) * 64;
  f32x4 acc[4][4];
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  for (int64_t k0 = k_begin; k0 < k_end; k0 += kStepK) {
    stage<T, A_KC>(a, m0, m_end, k0, k_end, lds_a);
    stage<T, B_KC>(b, n0, n_end, k0, k_end, lds_b);
    __syncthreads();
    const int off = (lane & 15) * kPitch + (lane >> 4) * 16;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const Fragment<T> fa = *reinterpret_cast<const Fragment<T>*>(lds_a + (wm + 16 * i) * kPitch + off);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const Fragment<T> fb = *reinterpret_cast<const Fragment<T>*>(lds_b + (wn + 16 * j) * kPitch + off);
        acc[i][j] = mma(fb, fa, acc[i][j]);      // (n along the registers of a lane: stores of four neighbours)
      }
    }
    __syncthreads();
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int64_t m = m0 + wm + 16 * i + (lane & 15);
    if (m >= m_end) continue;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int64_t n = n0 + wn + 16 * j + (lane >> 4) * 4;
      T* to = c + m * c_stride + n;
      if (n + 4 <= n_end) {
        Packed<T, 4> q;
#pragma unroll
        for (int r = 0; r < 4; ++r) q.v[r] = from_f32<T>(acc[i][j][r]);
        *reinterpret_cast<Packed<T, 4>*>(to) = q;
      } else {
#pragma unroll
        for (int r = 0; r < 4; ++r)
          if (n + r < n_end) to[r] = from_f32<T>(acc[i][j][r]);
      }
    }
  }
}

template <class T, bool B_KC>
__global__ __launch_bounds__(kThreads) void rows_kernel(RowsArgs g) {
  Found f;
  if (!find_tile(g.offset, g.n, g.slots, blockIdx.x, g.col_tiles, kTile, &f)) return;
  const Side<T> a{static_cast<const T*>(g.a), g.a_stride, g.source, g.div, g.limit};
  const Side<T> b{static_cast<const T*>(g.w) + f.expert * g.w_expert, g.w_stride, nullptr, Divisor{}, INT64_MAX};
  tile_product<T, true, B_KC>(a, b, f.begin, f.end, f.col * kTile, g.cols, 0, g.depth,
                              static_cast<T*>(g.c), g.cols);
}

template <class T>
__global__ __launch_bounds__(kThreads) void weight_kernel(WeightArgs g) {
  const int64_t tile = die_order(blockIdx.x, g.n * g.m_tiles * g.col_tiles);
  if (tile < 0) return;
  const int64_t col = tile % g.col_tiles, rest = tile / g.col_tiles;
  const int e = int(rest / g.m_tiles);
  int64_t begin, end;
  places(g.offset, e, g.slots, &begin, &end);
  const Side<T> a{static_cast<const T*>(g.a), g.a_stride, g.a_source, g.div, g.a_limit};
  const Side<T> b{static_cast<const T*>(g.b), g.b_stride, g.b_source, g.div, g.b_limit};
  tile_product<T, false, false>(a, b, (rest % g.m_tiles) * kTile, g.m, col * kTile, g.cols, begin, end,
                                static_cast<T*>(g.c) + e * g.m * g.cols, g.cols);
}

int64_t tiles(int64_t v) { return (v + kTile - 1) / kTile; }

template <class T>
int rows_type(RowsArgs g, bool k_contiguous, hipStream_t stream) {
  g.col_tiles = tiles(g.cols);
  const int64_t most = g.slots / kTile + min(int64_t(g.n), g.slots);       // tiles of rows, at most
  const int64_t blocks = most * g.col_tiles + kDies - 1;                   // (the eight runs may end short)
  if (blocks >= (int64_t(1) << 31)) return -1;
  if (k_contiguous) hipLaunchKernelGGL((rows_kernel<T, true>), dim3(unsigned(blocks)), dim3(kThreads), 0, stream, g);
  else hipLaunchKernelGGL((rows_kernel<T, false>), dim3(unsigned(blocks)), dim3(kThreads), 0, stream, g);
  return 0;
}
int rows_any(int type, const RowsArgs& g, bool k_contiguous, hipStream_t stream) {
  if (rows_aligned(type, g, k_contiguous)) return launch_rows_tiles(type, g, k_contiguous, stream);
  if (type == kF32) return rows_type<float>(g, k_contiguous, stream);
  if (type == kBF16) return rows_type<bf16>(g, k_contiguous, stream);
  if (type == kF16) return rows_type<f16>(g, k_contiguous, stream);
  return -1;
}

template <class T>
int weight_type(WeightArgs g, hipStream_t stream) {
  g.m_tiles = tiles(g.m);
  g.col_tiles = tiles(g.cols);
  const int64_t blocks = g.n * g.m_tiles * g.col_tiles + kDies - 1;
  if (blocks >= (int64_t(1) << 31)) return -1;
  hipLaunchKernelGGL(weight_kernel<T>, dim3(unsigned(blocks)), dim3(kThreads), 0, stream, g);
  return 0;
}

}  // namespace

int launch_product_fwd(int type, const ProductArgs& p, hipStream_t stream) {
  RowsArgs g{p.x, p.x_stride, p.source, divisor(p.k), p.m, p.w, p.w_expert, p.w_in == 1 ? p.w_out : p.w_in, p.offset, p.slots, p.n,
             p.ho, p.h, 0, p.out};
  return rows_any(type, g, p.w_in == 1, stream);
}

int launch_product_dx(int type, const ProductArgs& p, hipStream_t stream) {
  RowsArgs g{p.t, p.t_stride, nullptr, Divisor{}, p.slots, p.w, p.w_expert, p.w_out == 1 ? p.w_in : p.w_out, p.offset, p.slots, p.n,
             p.h, p.ho, 0, p.dx};
  return rows_any(type, g, p.w_out == 1, stream);
}

int launch_product_dw(int type, const ProductArgs& p, hipStream_t stream) {
  // dW has the layout of w: its contiguous direction gives the columns
  WeightArgs g;
  if (p.w_in == 1)
    g = {p.t, p.x, p.t_stride, p.x_stride, nullptr, p.source, divisor(p.k), p.slots, p.m, p.offset, p.slots, p.n, p.ho, p.h, 0, 0, p.dw};
  else
    g = {p.x, p.t, p.x_stride, p.t_stride, p.source, nullptr, divisor(p.k), p.m, p.slots, p.offset, p.slots, p.n, p.h, p.ho, 0, 0, p.dw};
  if (weight_aligned(type, g)) return launch_weight_tiles(type, g, stream);
  if (type == kF32) return weight_type<float>(g, stream);
  if (type == kBF16) return weight_type<bf16>(g, stream);
  if (type == kF16) return weight_type<f16>(g, stream);
  return -1;
}

}  // namespace topk
