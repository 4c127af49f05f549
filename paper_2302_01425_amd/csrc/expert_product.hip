// The experts' products over ragged groups of rows.  With expert e's places [offset[e], offset[e + 1]):
//   forward   out[s] = W[e] x[r(s)]          (h -> ho)
//   dx        dx[s]  = W[e]^T dout[s]        (ho -> h)
//   dW        dW[e]  = sum_s dout[s] x[r(s)]^T, zeros for an expert without places
// r(s) = source[s] / k, or s where the rows are in expert order already.  All three are
//   C(m, n) = sum_k A(m, k) B(n, k)
// with A, B each either contiguous in k or contiguous in m / n, and a row of x found through `source`.  Matrix instructions
// with float32 sums, one rounding per output element.  Here: which kernel takes a call.
#include "expert_product.hpp"

namespace topk {
namespace {

int size_of(int type) { return type == kF32 ? 4 : 2; }

// rows made of whole 16-byte parts that start at 16-byte boundaries
bool whole_parts(const void* p, int64_t stride, int64_t length, int size) {
  return reinterpret_cast<uintptr_t>(p) % 16 == 0 && stride * size % 16 == 0 && length * size % 16 == 0;
}

int64_t cut(int64_t v, int64_t size) { return (v + size - 1) / size; }

// Places per expert if they are spread evenly, and how many tiles of `rows` x `cols` outputs that makes.
int64_t even_share(int64_t slots, int n) { return slots > 0 ? cut(slots, min(int64_t(n), slots)) : 0; }
int64_t row_tiles(const RowsArgs& g, int64_t rows, int64_t cols) {
  return min(int64_t(g.n), g.slots) * cut(even_share(g.slots, g.n), rows) * cut(g.cols, cols);
}

// Which kernel takes the rows (bfloat16, us):
//   few rows, 64 x 64 / four rows at a time (each W on its first call; 1, 4, 16 tokens x 2 to 8 experts, 1 to 16 tokens x 4 to 64):
//     4096 -> 1024 38 / 9, 47 / 15, 47 / 25 (64 tokens: 47 / 41 with 8 places each), 2048 -> 4096 22 / 11, 30 / 32 (512 tiles), 2048 ->
//     1024 21 / 9, 27 / 19, 32 / 33 (8 tokens, 512 tiles); float32 112 / 11, 129 / 22, 130 / 34; 68 / 16, 96 / 43, 97 / 65; 59 / 11,
//     69 / 27, 131 / 71 (64 tokens, 4 places each, 210 / 126): there the matrix instructions of 32 rows take longer than the loads.
//   float32, 64 x 64 / 128 x 128: 16 experts of 64, 512 rows, 1024 -> 1024 49 / 88, 184 / 225; 4 of 4096, 1024 -> 2048 646 / 640.
//   whole parts, 64 x 64 / 256 x 256: 2048 -> 4096, 16 experts of 8, 64, 128, 256 rows on average 37 / 41, 60 / 68, 99 / 78,
//     170 / 116; 8 experts of 128 rows, 1024 -> 1024, 32 tiles of 256 x 256: 16 / 34; 16 of 250, 1000 -> 2008, 128 tiles 55 / 40.
//   others, 64 x 64 / 128 x 128: 64 experts of 32, 64, 256 rows, 1025 -> 2047 68 / 80, 109 / 113, 284 / 215; 16 of 250, 1001 ->
//     2005 62 / 58; 10 of 300, 515 -> 1001 (240 tiles) 20 / 18, 1001 -> 515 (150 tiles) 18 / 25; 8 of 2048, 2001 -> 3001 586 / 388.
int launch_rows(int type, const RowsArgs& g, bool k_contiguous, hipStream_t stream) {
  const int64_t share = even_share(g.slots, g.n);
  const int s = size_of(type);
  // (limit 0: there is no row that could be read in the place of one that is out of range)
  const bool few = (share <= 8 && cut(share, 4) * row_tiles(g, 64, 64) < 512) || (type == kF32 && share <= 4);
  if (few && g.limit > 0 && g.depth * s >= 16 && (k_contiguous || g.cols >= 32))
    return launch_rows_few(type, g, k_contiguous, stream);
  if (type == kF32) return launch_rows_tiles(type, g, k_contiguous, kSmall, stream);
  const bool whole = g.limit > 0 && whole_parts(g.a, g.a_stride, g.depth, s) &&
                     whole_parts(g.w, g.w_stride, k_contiguous ? g.depth : g.cols, s) && g.w_expert * s % 16 == 0;
  if (whole && share >= 96 && row_tiles(g, 256, 256) >= 96) return launch_rows_large(type, g, k_contiguous, stream);
  const bool middle = share >= 128 && row_tiles(g, 128, 128) >= 200;
  return launch_rows_tiles(type, g, k_contiguous, middle ? kMiddle : kSmall, stream);
}

}  // namespace

int launch_product_fwd(int type, const ProductArgs& p, hipStream_t stream) {
  RowsArgs g{p.x, p.x_stride, p.source, divisor(p.k), p.m, p.w, p.w_expert, p.w_in == 1 ? p.w_out : p.w_in, p.offset, p.slots,
             p.n, 0, p.ho, p.h, 0, p.out};
  return launch_rows(type, g, p.w_in == 1, stream);
}

int launch_product_dx(int type, const ProductArgs& p, hipStream_t stream) {
  RowsArgs g{p.t, p.t_stride, nullptr, Divisor{}, p.slots, p.w, p.w_expert, p.w_out == 1 ? p.w_in : p.w_out, p.offset, p.slots,
             p.n, 0, p.h, p.ho, 0, p.dx};
  return launch_rows(type, g, p.w_out == 1, stream);
}

int launch_product_dw(int type, const ProductArgs& p, hipStream_t stream, int64_t apart, void* dw_up) {
  // dW has the layout of w: its contiguous direction gives the columns
  WeightArgs g;
  if (p.w_in == 1)
    g = {p.t, p.x, p.t_stride, p.x_stride, nullptr, p.source, divisor(p.k), p.slots, p.m, p.offset, p.slots, p.n, 0, p.ho, p.h,
         p.dw};
  else
    g = {p.x, p.t, p.x_stride, p.t_stride, p.source, nullptr, divisor(p.k), p.m, p.slots, p.offset, p.slots, p.n, 0, p.h, p.ho,
         p.dw};
  g.stacked = p.w_in == 1 ? 1 : 2, g.apart = apart, g.c_up = dw_up;
  const int64_t arrays = dw_up != nullptr ? 2 : 1;
  const int s = size_of(type);
  const bool whole = whole_parts(g.a, g.a_stride, g.m, s) && whole_parts(g.b, g.b_stride, g.cols, s) &&
                     g.a_stride * s < (int64_t(1) << 32) && g.b_stride * s < (int64_t(1) << 32);   // (32-bit products of rows)
  // (bfloat16, us)  Whole parts, 64 x 64 / 128 x 256: 64 experts of 16, 64, 256 rows, 2048 x 1024 122 / 54, 159 / 74, 281 / 134; 8
  // of 128, 1024 x 1024, 256 tiles: 19 / 15.  Others, 64 x 64 / 128 x 128: 1025 x 2047, 64 experts of 32 rows 190 / 160, of 256
  // 374 / 271; 4 of 139 rows, 1501 x 1501, 576 tiles 20 / 19; 40 of 70, 777 x 333, 840 tiles 23 / 23; 10 of 300, 515 x 1001, 400
  // tiles 24 / 29.
  if (whole && apart % 16 == 0 && arrays * p.n * cut(g.m, 128) * cut(g.cols, 256) >= 256) return launch_weight_tiles(type, g, kWideDirect, stream);
  return launch_weight_tiles(type, g, arrays * p.n * cut(g.m, 128) * cut(g.cols, 128) >= 600 ? kMiddle : kSmall, stream);
}

}  // namespace topk
