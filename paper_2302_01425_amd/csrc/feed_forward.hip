// The experts' feed-forward.  With expert e's places [offset[e], offset[e + 1]), r(s) = source[s] / k, or s where the rows are in
// expert order already:
//   forward   g = Wg[e] x[r(s)], u = Wu[e] x[r(s)], out[s] = act(g) u
//   slopes    dg[s] = t[s] u act'(g), du[s] = t[s] act(g)
//   dx        dx[s] = Wg[e]^T dg[s] + Wu[e]^T du[s], one sum over the k of both
//   dW        dWg[e] = sum_s dg[s] x[r(s)]^T, dWu[e] = sum_s du[s] x[r(s)]^T
// A pair of weights is one operand of twice the columns, of which 32 of either come in turn: a lane of the matrix instructions then
// holds g and u of the same outputs, and what is made of them needs no exchange.  The slopes lie in the caller's scratch, dg and
// du of a place side by side.  8-bit operands: int32 sums, exact, times the scales of row and column.  Here: which kernel takes
// a call.
#include "feed_forward.hpp"

namespace topk {
namespace {

int size_of(int type) { return type == kF32 ? 4 : 2; }
int64_t cut(int64_t v, int64_t size) { return (v + size - 1) / size; }

// Places per expert if they are spread evenly, and how many tiles of `rows` x `cols` outputs that makes.
int64_t even_share(int64_t slots, int n) { return slots > 0 ? cut(slots, min(int64_t(n), slots)) : 0; }
int64_t row_tiles(const FeedArgs& g, int64_t rows, int64_t cols) {
  return min(int64_t(g.n), g.slots) * cut(even_share(g.slots, g.n), rows) * cut(g.cols, cols);
}

// rows made of whole 16-byte parts that start at 16-byte boundaries
bool whole_parts(const void* p, int64_t stride, int64_t length, int size) {
  return reinterpret_cast<uintptr_t>(p) % 16 == 0 && stride * size % 16 == 0 && length * size % 16 == 0;
}

// Which kernel takes the rows (us, from a graph of calls with W from HBM; experts x places each, h -> f; gated bfloat16 where
// nothing else is said):
//   four rows at a time (few) / 32 rows of half the columns (narrow) / 32 rows (thin) / 64 rows (small): what bounds the first is
//     multiplications, of the others loads in flight per compute unit, then operands read again.
//     1 x 1 2048 -> 1024 6.0 / 9.4 / 13.9 / 25, 1 x 8 9.4 / 10.1 / 14.7 / 25, 1 x 32 20 / 12.2 / 16.9 / 25, 8 x 8 512 -> 512 7.4 / 6.0
//     / 7.4 / 10.2, 8 x 16 2048 -> 1024 66 / 20.6 / 20.1 / 32, 8 x 64 211 / 38 / 31 / 33, 32 x 8 137 / 59 / 51 / 68, 32 x 64 836 / -
//     / 104 / 69, 1 x 128 4096 -> 4096 299 / 70 / 54 / 57, 2 x 128 564 / 135 / 102 / 62.
//     Rows of W that do not begin at 16 bytes, 1001 -> 300: 8 x 4 7.8 / 14.4 / 21 / 19, 8 x 32 20 / 17.4 / 24 / 18.4, 32 x 4 15.4 /
//     33 / 36 / 23.
//     16 bits, 32 rows of all / 64 rows by tiles of 32 rows: 512, places 8 to 32 per expert 31 to 34 / 36 to 38, 64 30 / 30; 640, 64 places
//     42 / 32, 32 places 47 / 46; 768, 8 to 32 places 43 to 48 / 45; 1024, 16 60 / 67, 32 63 / 61.
//     float32: 1 x 1 2048 -> 1024 7.1 / 15.4 / 24 / 96, 1 x 32 17 / 21 / 30 / 95, 8 x 32 114 / 43 / 39 / 107, 32 x 32 426 / 155 / 138 /
//     170, 8 x 128 - / 137 / 114 / 109, 8 x 1 4096 -> 4096 182 / 210 / 212 / 319.  64 rows at a time are half empty where experts have 32
//     places or fewer, and take a whole round of 512 workgroups each time.  By tiles of 32 rows, narrow / thin / small: 768, 64 places
//     109 / 93 / 110, 128 102 / 86 / 105, 512 -> 1024 39 / 35 / 31; 832, 64 places 124 / 118 / 111; 896, 128 119 / 112 / 106; 1152, 64
//     158 / 146 / 164; 2048, 64 274 / 230 / 180; 1152, 32 places 177 / 166 / 260; 2048, 32 305 / 262 / 334; 4096, 32 619 / 528 / 667,
//     8 443 / 433 / 646.  Rows of W that begin anywhere, 8 x 128 1001 -> 300 (320 tiles) 27 / 35 / 54, 1001 -> 1001: 384, 8 places 35 / 38
//     / 60, 32 43 / 42 / 59; 512, 8 44 / 40 / 62, 32 58 / 46 / 63, 128 42 / 36 / 55; 768, 64 64 / 64 / 60; 1024, 64 84 / 74 / 63, 32 106
//     / 91 / 95; 2048, 32 193 / 171 / 185.
//     8 bits, plain: 1 x 8 2048 -> 1024 4.8 / 7.7 / 10.9 / 12.7, 1 x 64 10.2 / 9.3 / 12.7 / 12.1, 8 x 64 39 / 14.9 / 13.3 / 13.5, 32 x 8
//     24 / 21 / 20 / 16.5, 8 x 8 512 -> 512 6.4 / 5.2 / 6.8 / 6.7; gated: 1 x 8 5.5 / 8.4 / 11.1 / 14.9, 8 x 32 40 / 15.8 / 13.0 / 16.7,
//     32 x 8 46 / 40 / 35 / 26.
//   W with one row per k, 32 rows of half the columns / of all / 64 rows (us, turned weights; dx of kept sums with its slopes, tiles of 32
//     rows of all columns in brackets): float32 1 x 1 2048 -> 1024 25 / 40 / 93; 26 / 41 / 67, 8 x 32 (128) 41 / 47 / 103; 43 / 49 / 79,
//     8 x 64 (256) 67 / 48 / 104; 62 / 50 / 81, 32 x 8 (512) 121 / 106 / 166; 111 / 104 / 183, 32 x 64 (1024) 235 / 177 / 179; 227 / 178 /
//     203.  1024 -> 1024, 128 x 8 (2048; 1024) 224 / 206 / 333; 215 / 217 / 351, 128 x 32 298 / 238 / 341; 305 / 265 / 369, 64 x 64 236 / 178 /
//     184; 236 / 194 / 206, 16 x 256 205 / 160 / 165.  bfloat16 1 x 1 2048 -> 1024 18.3 / 32 / 24; 19.8 / 33 / 24, 8 x 1 (128) 28.7 / 49 / 33;
//     29.4 / 49 / 31, 8 x 64 43 / 50 / 36; 37 / 50 / 33, 8 x 32 1001 -> 301 15 / 22 / 18; 12.6 / 18 / 14.
//   whole parts, 128 x 128 / 256 x 256: 8 x 250 1000 -> 1500 (96 tiles) 33 / 37, 24 x 125 1024 -> 768 (144) 29 / 33, 5 x 1925 640 ->
//     1088 (360) 58 / 52, 32 x 512 2048 -> 2048 (1024) 427 / 310.
template <class T>
int launch_feed(const FeedArgs& g, bool k_contiguous, Work work, hipStream_t stream) {
  const int64_t share = even_share(g.slots, g.n), experts = min(int64_t(g.n), g.slots);
  constexpr int s = int(sizeof(T));
  const bool pair = is_pair(work);
  const int64_t most = (int64_t(1) << 31) - (1 << 10);     // workgroups
  // (limit 0: there is no row that could be read in the place of one that is out of range)
  if (k_contiguous && work != kBoth && g.limit > 0 && g.depth * s >= 16 && (g.slots / 4 + g.n) * cut(g.cols, 2) < most) {
    const bool aligned = reinterpret_cast<uintptr_t>(g.w) % 16 == 0 && g.w_stride * s % 16 == 0 && g.w_expert * s % 16 == 0 &&
                         (!pair || g.apart % 16 == 0);
    const int64_t fours = experts * cut(share, 4) * cut(g.cols, pair ? 2 : 4), multiplied = fours * 16 * g.depth;
    const int64_t tiles = experts * cut(share, 32) * cut(g.cols, pair ? 32 : 64);
    const bool few = s == 1 ? fours <= 1536 && multiplied <= (1 << 26)
                   : s == 2 ? multiplied <= (aligned ? 1 << 25 : 100000000)
                            : multiplied <= 100000000 || share <= 4;
    if (few) return launch_feed_few<T>(g, work, stream);
    if (tiles < (aligned ? 192 : s == 2 ? 96 : s == 4 ? 448 : 192)) return launch_feed_thin<T>(g, work, true, stream);
    const bool thin = s == 1 ? tiles < 300
                    : s == 2 ? tiles <= (share <= 16 ? 1024 : share <= 32 ? 768 : 512)
                             : tiles <= 768 || share <= 32;
    if ((aligned || s == 4) && thin) return launch_feed_thin<T>(g, work, false, stream);
  }
  if constexpr (s > 1) {
    const int64_t tiles = experts * cut(share, 32) * cut(g.cols, pair ? 64 : 128);
    const bool narrow = s == 2 || tiles <= 128;
    if (!k_contiguous && g.limit > 0 && g.depth * s >= 16 && g.cols >= (pair ? 64 : 128) / (narrow ? 2 : 1) &&
        (tiles <= (s == 4 ? 1024 : 128) || (s == 4 && share <= 32)) && (g.slots / 4 + g.n) * cut(g.cols, 2) < most)
      return launch_feed_across<T>(g, work, narrow, stream);
  }
  if constexpr (s < 4) {
    const bool whole = g.limit > 0 && whole_parts(g.a, g.a_stride, g.depth, s) &&
                       whole_parts(g.w, g.w_stride, k_contiguous ? g.depth : g.cols, s) && g.w_expert * s % 16 == 0 &&
                       g.apart % 16 == 0 && (g.slots / 256 + g.n) * cut(g.cols, pair ? 128 : 256) < most;
    if (whole && share >= 96 && row_tiles(g, 256, pair ? 128 : 256) >= 192)
      return launch_feed_large<T>(g, k_contiguous, work, stream);
  }
  const bool middle = share >= 96 && row_tiles(g, 128, pair ? 64 : 128) >= 200;
  return launch_feed_tiles<T>(g, k_contiguous, work, middle ? kMiddle : kSmall, stream);
}
int launch_type(int type, const FeedArgs& g, bool k_contiguous, Work work, hipStream_t stream) {
  if (type == kF32) return launch_feed<float>(g, k_contiguous, work, stream);
  if (type == kBF16) return launch_feed<bf16>(g, k_contiguous, work, stream);
  if (type == kF16) return launch_feed<f16>(g, k_contiguous, work, stream);
  return -1;
}

int64_t bytes_between(const void* a, const void* b) { return int64_t(uintptr_t(b)) - int64_t(uintptr_t(a)); }

FeedArgs projections(const GatedArgs& g) {
  const ProductArgs& p = g.p;
  FeedArgs f{};
  f.a = p.x, f.a_stride = p.x_stride, f.source = p.source, f.div = divisor(p.k), f.limit = p.m;
  f.w = p.w, f.w_expert = p.w_expert, f.w_stride = p.w_in == 1 ? p.w_out : p.w_in, f.apart = bytes_between(p.w, g.w_up);
  f.offset = p.offset, f.slots = p.slots, f.n = p.n, f.cols = p.ho, f.depth = p.h;
  f.act = g.act;
  return f;
}

// Slopes from the sums that the forward pass kept: 16 bytes of a place per thread.  Bound by HBM: 8002 places, f 1515 float16, gelu: 24
// us, 5.0 TB/s.
constexpr int kSlopeThreads = 256;
template <class T, int ACT>
__global__ __launch_bounds__(kSlopeThreads) void slopes_kernel(FeedArgs g, int64_t first) {
  constexpr int N = 16 / int(sizeof(T));
  const int64_t along = (g.cols + N - 1) / N, i = (first + blockIdx.x) * kSlopeThreads + threadIdx.x;
  const int64_t s = i / along;
  if (s >= g.slots || s >= g.offset[g.n]) return;
  const int64_t c = min(i % along * N, max(g.cols - N, int64_t(0)));
  bool there = true;
  if (g.source != nullptr) there = g.source[s] >= 0 && quotient(g.source[s], g.div) < g.limit;
  const T* sums = static_cast<const T*>(g.pre) + s * 2 * g.cols + c;
  const T* t = static_cast<const T*>(g.t) + s * g.t_stride + c;
  T* out = static_cast<T*>(g.c) + s * g.c_stride + c;
  const auto of = [&](float gv, float uv, float tv, T* dg, T* du) {
    float slope;
    const float value = act_value<ACT, sizeof(T) == 4>(gv, &slope);
    *dg = from_f32<T>(there ? tv * uv * slope : 0.0f);
    *du = from_f32<T>(there ? tv * value : 0.0f);
  };
  if (g.cols < N) {
    for (int j = 0; j < g.cols; ++j) {
      T a, b;
      of(to_f32(sums[j]), to_f32(sums[g.cols + j]), to_f32(t[j]), &a, &b);
      out[j] = a, out[g.c_stride / 2 + j] = b;
    }
    return;
  }
  const Packed<T, N> gv = load_packed<T, N>(sums), uv = load_packed<T, N>(sums + g.cols), tv = load_packed<T, N>(t);
  Packed<T, N> a, b;
#pragma unroll
  for (int j = 0; j < N; ++j) of(to_f32(gv.v[j]), to_f32(uv.v[j]), to_f32(tv.v[j]), &a.v[j], &b.v[j]);
  store_packed<T, N>(out, a);
  store_packed<T, N>(out + g.c_stride / 2, b);
}
template <class T, int ACT>
int slopes_act(const FeedArgs& g, hipStream_t stream) {
  constexpr int64_t kMost = (int64_t(1) << 31) / kSlopeThreads;
  const int64_t along = cut(g.cols, 16 / int64_t(sizeof(T))), blocks = cut(g.slots * along, kSlopeThreads);
  for (int64_t b = 0; b < blocks; b += kMost)
    hipLaunchKernelGGL((slopes_kernel<T, ACT>), dim3(unsigned(min(blocks - b, kMost))), dim3(kSlopeThreads), 0, stream, g, b);
  return 0;
}
template <class T>
int slopes_type(const FeedArgs& g, hipStream_t stream) {
  if (g.act == kSilu) return slopes_act<T, kSilu>(g, stream);
  if (g.act == kGelu) return slopes_act<T, kGelu>(g, stream);
  if (g.act == kGeluTanh) return slopes_act<T, kGeluTanh>(g, stream);
  return slopes_act<T, kRelu>(g, stream);
}

}  // namespace

int launch_slopes(int type, const FeedArgs& g, hipStream_t stream) {
  if (type == kF32) return slopes_type<float>(g, stream);
  if (type == kBF16) return slopes_type<bf16>(g, stream);
  if (type == kF16) return slopes_type<f16>(g, stream);
  return -1;
}

// two halves of whole 16-byte parts
int64_t slopes_stride(int type, int64_t f) { return 2 * cut(f, 16 / size_of(type)) * (16 / size_of(type)); }

int launch_gated_fwd(int type, const GatedArgs& g, hipStream_t stream) {
  FeedArgs f = projections(g);
  f.c = g.p.out, f.c_stride = g.p.ho, f.pre = g.pre;
  return launch_type(type, f, g.p.w_in == 1, kOut, stream);
}

int launch_gated_vjp(int type, const GatedArgs& g, hipStream_t stream) {
  const ProductArgs& p = g.p;
  const int64_t stride = slopes_stride(type, p.ho);
  if (p.slots > 0) {
    FeedArgs f = projections(g);
    f.c = g.scratch, f.c_stride = stride, f.t = p.t, f.t_stride = p.t_stride;
    int launched;
    if (g.kept != nullptr) {
      f.pre = const_cast<void*>(g.kept);       // (read only)
      launched = launch_slopes(type, f, stream);
    } else {
      launched = launch_type(type, f, p.w_in == 1, kSlopes, stream);
    }
    if (launched != 0) return launched;
    if (p.dx != nullptr) {
      FeedArgs b = projections(g);
      b.a = g.scratch, b.a_stride = stride, b.a_apart = stride / 2 * size_of(type);
      b.w_stride = p.w_out == 1 ? p.w_in : p.w_out;
      b.cols = p.h, b.depth = p.ho, b.c = p.dx, b.c_stride = p.h;
      launched = launch_type(type, b, p.w_out == 1, kBoth, stream);
      if (launched != 0) return launched;
    }
  }
  if (p.dw != nullptr) {
    // dW has the layout of w: its contiguous direction gives the columns
    const int64_t apart = stride / 2 * size_of(type);
    WeightArgs w;
    const bool x_first = p.w_in != 1;
    if (x_first)
      w = {p.x, g.scratch, p.x_stride, stride, p.source, nullptr, divisor(p.k), p.m, p.slots, p.offset, p.slots, p.n, 0, p.h, p.ho,
           nullptr};
    else
      w = {g.scratch, p.x, stride, p.x_stride, nullptr, p.source, divisor(p.k), p.slots, p.m, p.offset, p.slots, p.n, 0, p.ho, p.h,
           nullptr};
    const int s = size_of(type);
    const int64_t tiles = both_weights_tiles(w);
    const bool whole = s == 2 && p.m > 0 && whole_parts(w.a, w.a_stride, w.m, s) && whole_parts(w.b, w.b_stride, w.cols, s);
    // (one launch, of a few more workgroups than tiles; products of rows and strides in 32 bits)
    // (they cross between 1024 and 1536 places, times beside the kernel)
    if (whole && tiles >= 256 && tiles < (int64_t(1) << 22) && w.a_stride < (int64_t(1) << 31) && w.b_stride < (int64_t(1) << 31) &&
        even_share(p.slots, p.n) >= 1536)
      return launch_both_weights(type, w, x_first, apart, p.dw, g.dw_up, stream);
    ProductArgs q = p;
    q.t = g.scratch, q.t_stride = stride;
    return launch_product_dw(type, q, stream, apart, g.dw_up);
  }
  return 0;
}

int launch_eight(const EightArgs& e, hipStream_t stream) {
  FeedArgs f{};
  f.a = e.x, f.a_stride = e.x_stride, f.source = e.source, f.div = divisor(e.k), f.limit = e.m;
  f.w = e.w, f.w_expert = e.w_expert, f.w_stride = e.w_out;
  f.offset = e.offset, f.slots = e.slots, f.n = e.n, f.cols = e.f, f.depth = e.h;
  f.c = e.out, f.c_stride = e.f, f.act = e.act, f.out_type = e.out_type;
  f.a_scale = e.x_scale, f.w_scale = e.w_scale, f.u_scale = e.up_scale;
  if (e.w_up != nullptr) f.apart = bytes_between(e.w, e.w_up);
  return launch_feed<int8_t>(f, true, e.w_up != nullptr ? kOut : kPlain, stream);
}

}  // namespace topk
