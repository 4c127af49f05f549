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

template <class T>
int launch_feed(const FeedArgs& g, bool k_contiguous, Work work, hipStream_t stream) {
  const bool middle = even_share(g.slots, g.n) >= 128 && row_tiles(g, 128, is_pair(work) ? 64 : 128) >= 200;
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

// slopes from the sums that the forward pass kept: 16 bytes of a place per thread
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
    for (int i = 0; i < 2; ++i) {
      ProductArgs w = p;
      w.t = static_cast<const char*>(g.scratch) + (i == 0 ? 0 : stride / 2 * size_of(type));
      w.t_stride = stride;
      w.dw = i == 0 ? p.dw : g.dw_up;
      const int launched = launch_product_dw(type, w, stream);
      if (launched != 0) return launched;
    }
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
