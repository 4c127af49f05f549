// The experts' feed-forward for experts of few rows, as in decoding: one pass over W, which is all there is to read, by as many
// wavefronts as keep its loads on their way.  W contiguous in k.
//
// Four rows of an expert and four columns of W (two of either weight of a pair) at a time: a lane has 16 bytes of k of each, and the
// 16 sums meet by a butterfly that halves the values at every step.  Rows of k of 4 KB and more are shared by the four wavefronts
// of a workgroup, whose sums meet in LDS; of shorter ones every wavefront takes columns of its own.  No matrix instructions: they
// would multiply 32 rows of which four at most are there.
//
// One token, 2 of 8 experts, gated 2048 -> 1024 bfloat16: 7.6 us on the GPU, 2.2 TB/s, bound by the chain of loads (offsets, rows, W) and
// the first read of the instructions; 4096 -> 4096: 27.8 us, 4.8 TB/s, bound by HBM; 8 bits 6.2 us.
#include "feed_forward.hpp"

namespace topk {
namespace {

constexpr int kFewThreads = 256, kFewWaves = kFewThreads / kWave;
constexpr int kFewRows = 4, kFewCols = 4;      // rows, and columns of W, that meet

template <class T>
struct SumOf {
  using type = float;
};
template <>
struct SumOf<int8_t> {
  using type = int;
};

// 16 bytes of W and of x per lane into the sums; of a part that crosses the end, and begins before it, the first `skip` elements
// are counted in another one
template <class T>
__device__ __forceinline__ void few_add(const T* const (&w)[kFewCols], const T* const (&x)[kFewRows], int64_t k, int skip,
                                        typename SumOf<T>::type (&acc)[kFewCols * kFewRows]) {
  constexpr int N = 16 / int(sizeof(T));
  Packed<T, N> a[kFewCols], b[kFewRows];
#pragma unroll
  for (int c = 0; c < kFewCols; ++c) a[c] = load_packed<T, N>(w[c] + k);
#pragma unroll
  for (int r = 0; r < kFewRows; ++r) b[r] = load_packed<T, N>(x[r] + k);
  if (skip > 0) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
#pragma unroll
      for (int c = 0; c < kFewCols; ++c) a[c].v[i] = i < skip ? T(0.0f) : a[c].v[i];
#pragma unroll
      for (int r = 0; r < kFewRows; ++r) b[r].v[i] = i < skip ? T(0.0f) : b[r].v[i];
    }
  }
  if constexpr (sizeof(T) == 1) {
#pragma unroll
    for (int c = 0; c < kFewCols; ++c) {
      const i32x4 u = __builtin_bit_cast(i32x4, a[c]);
#pragma unroll
      for (int r = 0; r < kFewRows; ++r) {
        const i32x4 v = __builtin_bit_cast(i32x4, b[r]);
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[c * kFewRows + r] = __builtin_amdgcn_sdot4(u[i], v[i], acc[c * kFewRows + r], false);
      }
    }
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
      for (int c = 0; c < kFewCols; ++c)
#pragma unroll
        for (int r = 0; r < kFewRows; ++r) acc[c * kFewRows + r] += to_f32(a[c].v[i]) * to_f32(b[r].v[i]);
  }
}

// Sums over the lanes that differ in the bits 4 .. 32 of their number: each of them ends up with one of the 16 values, the returned
// one, in v[0]; then over the last two bits.
template <int COUNT = kFewCols * kFewRows, int S = 32, class V>
__device__ __forceinline__ int few_halve(V* v, int lane) {
  if constexpr (S < 4) {
    v[0] += __shfl_xor(v[0], 2, kWave);
    v[0] += __shfl_xor(v[0], 1, kWave);
    return 0;
  } else {
    const bool upper = (lane & S) != 0;
#pragma unroll
    for (int i = 0; i < COUNT / 2; ++i) {
      const V keep = upper ? v[i + COUNT / 2] : v[i], send = upper ? v[i] : v[i + COUNT / 2];
      v[i] = keep + __shfl_xor(send, S, kWave);
    }
    return (upper ? COUNT / 2 : 0) + few_halve<COUNT / 2, S / 2>(v, lane);
  }
}

template <class T, class OUT, Work WORK, int ACT>
__device__ __forceinline__ void few_store(const FeedArgs& g, int64_t m, int64_t n, bool there, float t, float first,
                                          float second) {
  constexpr bool kFine = sizeof(OUT) == 4;
  OUT* c = static_cast<OUT*>(g.c) + m * g.c_stride + n;
  if constexpr (WORK == kPlain) {
    *c = from_f32<OUT>(there ? first : 0.0f);
  } else if constexpr (WORK == kOut) {
    if constexpr (sizeof(T) > 1) {
      if (g.pre != nullptr) {
        T* sums = static_cast<T*>(g.pre) + m * 2 * g.cols + n;
        sums[0] = from_f32<T>(there ? first : 0.0f);
        sums[g.cols] = from_f32<T>(there ? second : 0.0f);
      }
    }
    *c = from_f32<OUT>(there ? act_value<ACT, kFine>(first, nullptr) * second : 0.0f);
  } else {
    float slope;
    const float value = act_value<ACT, kFine>(first, &slope);
    c[0] = from_f32<OUT>(there ? t * second * slope : 0.0f);
    c[g.c_stride / 2] = from_f32<OUT>(there ? t * value : 0.0f);
  }
}

// what a wavefront's lanes wrote to LDS is there for its other lanes
__device__ __forceinline__ void meet() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// SHARED: the wavefronts of a workgroup share k.  A workgroup takes kFewCols `turns` columns of W (four times as many where its
// wavefronts have columns of their own).
template <class T, class OUT, Work WORK, bool SHARED>
__global__ __launch_bounds__(kFewThreads) void feed_few_kernel(FeedArgs g, int turns) {
  constexpr int N = 16 / int(sizeof(T)), kOf = is_pair(WORK) ? 2 : 1, kOuts = kFewCols / kOf;     // columns of the output
  using Sum = typename SumOf<T>::type;
  __shared__ Sum sums[SHARED ? 2 : kFewWaves][SHARED ? kFewWaves : 1][kFewRows * kFewCols];
  Found f;
  if (!find_group_tile<kFewRows>(g, &f)) return;
  const int lane = int(threadIdx.x) & (kWave - 1), wave = int(threadIdx.x) / kWave;
  const T* w = static_cast<const T*>(g.w) + f.expert * g.w_expert;
  // rows that are not there are read from another row, and not stored, or stored as zeros
  const T* x[kFewRows];
#pragma unroll
  for (int r = 0; r < kFewRows; ++r) {
    int64_t row = min(f.begin + r, f.end - 1);
    if (g.source != nullptr) row = min(int64_t(quotient(max(g.source[row], 0), g.div)), g.limit - 1);
    x[r] = static_cast<const T*>(g.a) + row * g.a_stride;
  }
  // what a thread needs for the output that it makes of the sums, looked up before them
  const int i = SHARED ? int(threadIdx.x) : lane, c = i % kOuts;
  const int64_t m = f.begin + i / kOuts;
  const bool mine = i < kFewRows * kOuts && m < f.end;
  bool there = mine;
  float scale = 0.0f;
  if (mine) {
    int64_t row = m;
    if (g.source != nullptr) {
      const int pair = g.source[m];
      row = quotient(max(pair, 0), g.div);
      there = pair >= 0 && row < g.limit;
    }
    if (sizeof(T) == 1 && there) scale = g.a_scale[row];
  }
  constexpr int64_t kChunk = kWave * N;
  const int64_t group = SHARED ? f.col : f.col * kFewWaves + wave;
  for (int turn = 0; turn < turns; ++turn) {
    const int64_t n0 = (group * turns + turn) * kOuts;
    if (n0 >= g.cols) break;               // (the same for all that share sums)
    const int64_t n = n0 + c;
    const bool store = mine && n < g.cols;
    float first_scale = 0.0f, second_scale = 0.0f, t = 0.0f;
    if (store && there) {
      if constexpr (sizeof(T) == 1) {
        first_scale = g.w_scale[f.expert * g.cols + n];
        if constexpr (kOf == 2) second_scale = g.u_scale[f.expert * g.cols + n];
      }
      if constexpr (WORK == kSlopes) t = to_f32(static_cast<const T*>(g.t)[m * g.t_stride + n]);
    }
    const T* p[kFewCols];
#pragma unroll
    for (int c = 0; c < kFewCols; ++c) {
      const char* from = reinterpret_cast<const char*>(w + min(n0 + c % kOuts, g.cols - 1) * g.w_stride);
      p[c] = reinterpret_cast<const T*>(c >= kOuts ? from + g.apart : from);
    }
    Sum acc[kFewCols * kFewRows] = {};
    constexpr int64_t kStride = (SHARED ? kFewWaves : 1) * kChunk;
    // (one copy of the instructions, which are read from memory by every launch: with two steps at a time and the last by itself a call
    // of one token, 2048 -> 1024, took 10.2 us in the place of 8.5)
#pragma unroll 1
    for (int64_t k = (SHARED ? wave * kChunk : 0) + lane * N; k < g.depth; k += kStride) {
      const int64_t from = min(k, g.depth - N);
      few_add<T>(p, x, from, int(k - from), acc);
    }
    const int at = few_halve(acc, lane);
    const int set = SHARED ? turn & 1 : wave;
    if ((lane & 3) == 0) sums[set][SHARED ? wave : 0][at] = acc[0];
    if constexpr (SHARED) __syncthreads();               // (and the sums of the turn before are read)
    else meet();
    if (store) {
      float v[2] = {0.0f, 0.0f};
#pragma unroll
      for (int o = 0; o < kOf; ++o) {
        Sum sum = 0;
#pragma unroll
        for (int q = 0; q < (SHARED ? kFewWaves : 1); ++q) sum += sums[set][q][(c + o * kOuts) * kFewRows + i / kOuts];
        v[o] = float(sum);
      }
      if constexpr (sizeof(T) == 1) {
        v[0] = scaled(v[0], row_scale(scale), first_scale);
        if constexpr (kOf == 2) v[1] = scaled(v[1], row_scale(scale), second_scale);
      }
      if constexpr (WORK == kPlain) few_store<T, OUT, WORK, 0>(g, m, n, there, t, v[0], v[1]);
      else if (g.act == kSilu) few_store<T, OUT, WORK, kSilu>(g, m, n, there, t, v[0], v[1]);
      else if (g.act == kGelu) few_store<T, OUT, WORK, kGelu>(g, m, n, there, t, v[0], v[1]);
      else if (g.act == kGeluTanh) few_store<T, OUT, WORK, kGeluTanh>(g, m, n, there, t, v[0], v[1]);
      else few_store<T, OUT, WORK, kRelu>(g, m, n, there, t, v[0], v[1]);
    }
    if constexpr (!SHARED) meet();
  }
}

template <class T, class OUT, Work WORK>
int few(FeedArgs g, hipStream_t stream) {
  constexpr int kOuts = kFewCols / (is_pair(WORK) ? 2 : 1);
  const bool shared = g.depth * int64_t(sizeof(T)) >= 4096;
  const int64_t wide = kOuts * (shared ? 1 : kFewWaves);         // columns of a workgroup and turn
  // several turns where some four workgroups per compute unit are left
  const int64_t all = (g.slots / kFewRows + min(int64_t(g.n), g.slots)) * ((g.cols + wide - 1) / wide);
  const int64_t turns = max(int64_t(1), min(all / 1024, int64_t(4)));
  g.col_tiles = (g.cols + wide * turns - 1) / (wide * turns);
  return in_launches<kFewThreads>(g, rows_blocks(g, kFewRows), [&](const FeedArgs& part, dim3 grid) {
    if (shared) hipLaunchKernelGGL((feed_few_kernel<T, OUT, WORK, true>), grid, dim3(kFewThreads), 0, stream, part, int(turns));
    else hipLaunchKernelGGL((feed_few_kernel<T, OUT, WORK, false>), grid, dim3(kFewThreads), 0, stream, part, int(turns));
  });
}

template <class T>
int few_work(const FeedArgs& g, Work work, hipStream_t stream) {
  if constexpr (sizeof(T) == 1) {
    const auto to = [&](auto out) {
      using OUT = decltype(out);
      return work == kPlain ? few<T, OUT, kPlain>(g, stream) : few<T, OUT, kOut>(g, stream);
    };
    if (work != kPlain && work != kOut) return -1;
    return g.out_type == kF32 ? to(float{}) : g.out_type == kBF16 ? to(bf16{}) : to(f16{});
  } else {
    if (work == kOut) return few<T, T, kOut>(g, stream);
    if (work == kSlopes) return few<T, T, kSlopes>(g, stream);
    return -1;
  }
}

}  // namespace

template <>
int launch_feed_few<float>(const FeedArgs& g, Work work, hipStream_t stream) {
  return few_work<float>(g, work, stream);
}
template <>
int launch_feed_few<bf16>(const FeedArgs& g, Work work, hipStream_t stream) {
  return few_work<bf16>(g, work, stream);
}
template <>
int launch_feed_few<f16>(const FeedArgs& g, Work work, hipStream_t stream) {
  return few_work<f16>(g, work, stream);
}
template <>
int launch_feed_few<int8_t>(const FeedArgs& g, Work work, hipStream_t stream) {
  return few_work<int8_t>(g, work, stream);
}

}  // namespace topk
