// What the kernels of the experts' feed-forward share: the gated block (two projections of the same rows, the activation and the
// product), its gradients, and products in 8-bit integers.  Ragged rows, lists, tiles and operands as in expert_product.hpp.
#pragma once

#include "expert_tiles.hpp"

namespace topk {

enum ActCode : int { kSilu = 0, kGelu = 1, kGeluTanh = 2, kRelu = 3 };

// What becomes of the sums of a tile:
//   kPlain   8-bit operands: c = a_scale w_scale sum
//   kOut     of a pair of weights, g and u: c = act(g) u, and the sums themselves to `pre`
//   kSlopes  of a pair, with the cotangent t of act(g) u: t u act'(g) and t act(g), side by side in a row of c
//   kBoth    rows of such slopes times the pair, c = dg W + du W'
enum Work { kPlain, kOut, kSlopes, kBoth };
constexpr bool is_pair(Work w) { return w == kOut || w == kSlopes; }

struct FeedArgs : RowsArgs {
  int64_t apart;            // bytes from w to the second weights
  int64_t a_apart;          // kBoth: bytes from a's dg to its du
  int64_t c_stride;         // elements between rows of c; kSlopes: two halves
  int act, out_type;
  void* pre;                // kOut: [slots][2][cols] or null
  const void* t;            // kSlopes
  int64_t t_stride;
  const float *a_scale;     // 8-bit: of the rows of a
  const float *w_scale, *u_scale;      // [n][cols]
};

// ---- tiles ----------------------------------------------------------------------------------------------------------------
// As find_tile, with the tiles of rows of an expert in groups of kGroup, which meet all columns before the next: of the 32 tiles
// that a die works on at a time, 8 x 4 read 12 panels, 32 x 1 would read 33.  Every wavefront finds the tile by itself, 64 experts
// at a time.  (A die that takes an eighth of every expert's columns instead has the same work as the others, whatever the
// experts' shares, but reads all rows of x: 32 experts of 480 rows, 2048 -> 2048 x 2, 300 us against 245; of unequal shares, 512
// rows on average, 328 against 318.)
// Fewer than 2^31 workgroups, so that all numbers fit 32 bits.
constexpr uint32_t kGroup = 8;
template <int ROWS>
__device__ __forceinline__ bool find_group_tile(const FeedArgs& g, Found* f) {
  const int lane = int(threadIdx.x) & (kWave - 1);
  const uint32_t cols = uint32_t(g.col_tiles);
  const auto tiles_of = [&](int e, int64_t* begin, int64_t* end) {
    *begin = *end = 0;
    if (e < g.n) places(g.offset, e, g.slots, begin, end);
    return uint32_t((*end - *begin + ROWS - 1) / ROWS);
  };
  int64_t begin, end;
  uint32_t total = 0;
  for (int e = lane; e < g.n; e += kWave) total += tiles_of(e, &begin, &end);
  for (int off = kWave / 2; off > 0; off >>= 1) total += uint32_t(__shfl_xor(int(total), off, kWave));
  // (as dealt())
  const uint32_t block = g.first + blockIdx.x, run = min(max(total * cols / (8 * kDies), 1u), uint32_t(kRunMost));
  const uint32_t turn = block / kDies / run, pair = (turn * kDies + block % kDies) * run + (block / kDies - turn * run);
  uint32_t start = 0;
  for (int first = 0; first < g.n; first += kWave) {
    const uint32_t tiles = tiles_of(first + lane, &begin, &end);
    uint32_t scan = tiles;
    for (int off = 1; off < kWave; off <<= 1) {
      const uint32_t v = uint32_t(__shfl_up(int(scan), off, kWave));
      if (lane >= off) scan += v;
    }
    const uint32_t before = (start + scan - tiles) * cols;
    const unsigned long long here = __ballot(pair >= before && pair - before < tiles * cols);
    if (here != 0) {
      const int from = __ffsll(here) - 1;
      const auto of = [&](uint32_t v) { return uint32_t(__builtin_amdgcn_readlane(int(v), from)); };
      const uint32_t in = pair - of(before), group = in / (kGroup * cols), rest = in - group * kGroup * cols;
      const uint32_t high = min(of(tiles) - group * kGroup, kGroup), col = rest / high;
      const int64_t row = int64_t(of(uint32_t(begin))) + int64_t(group * kGroup + rest - col * high) * ROWS;
      *f = Found{first + from, row, min(row + ROWS, int64_t(of(uint32_t(end)))), int64_t(col)};
      return true;
    }
    start += uint32_t(__builtin_amdgcn_readlane(int(scan), kWave - 1));
  }
  return false;
}

// ---- activations --------------------------------------------------------------------------------------------------------
// exp(x): for outputs of 16 bits by the hardware's exp2, off by |x| 2^-24 and two steps more
template <bool FINE>
__device__ __forceinline__ float exp_of(float x) {
  if constexpr (FINE) return expf(x);
  else return __builtin_amdgcn_exp2f(x * 1.44269504f);
}
template <bool FINE>
__device__ __forceinline__ float inverse(float x) {
  if constexpr (FINE) return 1.0f / x;
  else return __builtin_amdgcn_rcpf(x);
}

// act(g) and act'(g).  Each comes from a form that keeps its digits where g is far below zero:
//   silu       g p, p = 1 / (1 + exp(-g));  p + g p (1 - p)
//   gelu       g F, F = P(N(0, 1) < g);  F + g exp(-g^2 / 2) / sqrt(2 pi).  F(-|g|) = exp(-g^2 / 2) q(t) t, t = 1 / (1 + 0.4 |g| /
//              sqrt 2), with q the polynomial of degree 10 through the Chebyshev nodes of t in (0, 1) of exp(x^2) erfc(x) / 2 t, x =
//              (1 / t - 1) / 0.4: off by 1.5e-8 of it with these coefficients, 3.4e-7 in float32.  g^2 is taken with the rounding it lost.
//   gelu_tanh  g (1 + tanh z) / 2 = g p(2 z), z = sqrt(2 / pi) (g + 0.044715 g^3)
//   relu       g where g > 0, slope 0 at 0
// NaN gives NaN (relu: and the slope 1).
template <int ACT, bool FINE>
__device__ __forceinline__ float act_value(float g, float* slope) {
  if constexpr (ACT == kSilu) {
    const float p = inverse<FINE>(1.0f + exp_of<FINE>(-g));
    if (slope != nullptr) *slope = p + g * p * (1.0f - p);
    return g * p;
  } else if constexpr (ACT == kGelu) {
    const float s = g * g;
    const float e = s < 208.0f ? exp_of<FINE>(-0.5f * s) * (1.0f - 0.5f * __builtin_fmaf(g, g, -s)) : 0.0f;
    const float t = inverse<FINE>(1.0f + 0.282842712f * fabsf(g));
    constexpr float kQ[11] = {0.112837916f, 0.112838158f, 0.10380036f, 0.085945286f, 0.0590475614f, 0.0435603211f,
                              -0.0268965838f, 0.0734016237f, -0.121520867f, 0.071920535f, -0.0149343143f};
    float q = kQ[10];
#pragma unroll
    for (int i = 9; i >= 0; --i) q = __builtin_fmaf(q, t, kQ[i]);
    const float tail = e * t * q;
    const float p = g < 0.0f ? tail : 1.0f - tail;
    if (slope != nullptr) *slope = __builtin_fmaf(g * e, 0.398942280f, p);
    return g * p;
  } else if constexpr (ACT == kGeluTanh) {
    const float b = g < -30.0f ? -30.0f : g > 30.0f ? 30.0f : g, b2 = b * b;      // (beyond, p is 0 or 1)
    const float z2 = 1.59576912f * b * __builtin_fmaf(0.044715f, b2, 1.0f);
    const float p = inverse<FINE>(1.0f + exp_of<FINE>(-z2));
    if (slope != nullptr) *slope = p + b * p * (1.0f - p) * 1.59576912f * __builtin_fmaf(0.134145f, b2, 1.0f);
    return g * p;
  } else {
    if (slope != nullptr) *slope = g <= 0.0f ? 0.0f : 1.0f;
    return g <= 0.0f ? 0.0f : g;
  }
}

// ---- outputs --------------------------------------------------------------------------------------------------------------
// A sum of 8-bit products with its scales, in an order in which nothing between leaves float32's range if the result does not: a row's
// scale comes first where its magnitude is below 1 (a whole number times it keeps its digits, and the channel's may be large), the channel's where
// it is not.  One of the two factors is 1.
struct RowScale {
  float first, last;
};
__device__ __forceinline__ RowScale row_scale(float scale) {
  const bool small = fabsf(scale) < 1.0f;
  return {small ? scale : 1.0f, small ? 1.0f : scale};
}
__device__ __forceinline__ float scaled(float sum, const RowScale& row, float channel) {
  return sum * row.first * channel * row.last;
}

template <class T>
__device__ __forceinline__ void load_four(const T* p, int64_t left, float (&v)[4]) {
  if (left >= 4) {
    const Packed<T, 4> q = load_packed<T, 4>(p);
#pragma unroll
    for (int r = 0; r < 4; ++r) v[r] = to_f32(q.v[r]);
  } else {
#pragma unroll
    for (int r = 0; r < 4; ++r) v[r] = r < left ? to_f32(p[r]) : 0.0f;
  }
}

// What a wavefront has to know of its rows, from m0 on (below m_end), when it has their sums.  Looked up before the sums: two loads,
// of which the second needs the first, would otherwise be waited for at the end of every tile.
template <int MI>
struct RowsOfTile {
  bool there[MI];          // the place has a row
  float scale[MI];         // 8-bit operands
};
template <class T, int MI>
__device__ __forceinline__ RowsOfTile<MI> rows_of_tile(const FeedArgs& g, int64_t m0, int64_t m_end) {
  RowsOfTile<MI> r;
#pragma unroll
  for (int i = 0; i < MI; ++i) {
    const int64_t m = m0 + 32 * i + (int(threadIdx.x) & 31);
    int64_t row = m;
    r.there[i] = m < m_end;
    if (r.there[i] && g.source != nullptr) {
      const int pair = g.source[m];
      row = quotient(max(pair, 0), g.div);
      r.there[i] = pair >= 0 && row < g.limit;
    }
    r.scale[i] = sizeof(T) == 1 && r.there[i] ? g.a_scale[row] : 0.0f;
  }
  return r;
}

// Sums of a wavefront, MI x NJ blocks of 32 x 32 from row m0 on (below m_end), to the outputs from column n0 on.  Rows whose place
// has no source are zeros, whatever their operands hold.  Columns from n_end on are left as they were.  T: type of the operands; OUT: of c.
template <class T, class OUT, Work WORK, int ACT, int MI, int NJ, class ACC>
__device__ __forceinline__ void finish_tile(const ACC (&acc)[MI][NJ], const FeedArgs& g, const RowsOfTile<MI>& rows, int expert,
                                            int64_t m0, int64_t m_end, int64_t n0, int64_t n_end) {
  constexpr bool kEight = sizeof(T) == 1, kFine = sizeof(OUT) == 4;
  constexpr int kOf = is_pair(WORK) ? 2 : 1;
  const int lane = int(threadIdx.x) & (kWave - 1);
  // (scales of all columns at once, as the cotangents below)
  float col_scale[kEight ? NJ : 1][4][4];
  if constexpr (kEight) {
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
      const int64_t mine = n0 + 32 * (j / kOf) + 4 * (lane >> 5);
      const float* from = (j % kOf == 0 ? g.w_scale : g.u_scale) + expert * g.cols;
#pragma unroll
      for (int q = 0; q < 4; ++q) load_four(from + mine + 8 * q, g.cols - mine - 8 * q, col_scale[j][q]);
    }
  }
#pragma unroll
  for (int j = 0; j < NJ; j += kOf) {
    const int64_t n = n0 + 32 * (j / kOf), mine = n + 4 * (lane >> 5);
    // cotangents of all blocks at once: the compiler would wait for each block's behind the stores of the one before
    Packed<T, 4> t[WORK == kSlopes ? MI : 1][4];
    if constexpr (WORK == kSlopes) {
      const bool whole = n + 32 <= g.cols;
#pragma unroll
      for (int i = 0; i < MI; ++i) {
        const T* row = static_cast<const T*>(g.t) + min(m0 + 32 * i + (lane & 31), m_end - 1) * g.t_stride;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const int64_t col = mine + 8 * q;
          if (whole) {
            t[i][q] = load_packed<T, 4>(row + col);
          } else {
#pragma unroll
            for (int r = 0; r < 4; ++r) t[i][q].v[r] = col + r < g.cols ? row[col + r] : T(0.0f);
          }
        }
      }
    }
#pragma unroll
    for (int i = 0; i < MI; ++i) {
      if (m0 + 32 * i >= m_end) break;
      const int64_t m = m0 + 32 * i + (lane & 31);
      const bool inside = m < m_end;
      OUT* row = static_cast<OUT*>(g.c) + m * g.c_stride;
      f32x16 first, second;
      const RowScale scale = row_scale(rows.scale[i]);
#pragma unroll
      for (int q = 0; q < 4; ++q) {
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int x = 4 * q + r;
          const auto of = [&](int at) {
            return kEight ? scaled(float(acc[i][at][x]), scale, col_scale[kEight ? at : 0][q][r]) : float(acc[i][at][x]);
          };
          first[x] = of(j);
          if constexpr (kOf == 2) second[x] = of(j + 1);
        }
      }
      if constexpr (kOf == 1) {
        store_block<OUT>(first, row, inside, rows.there[i], n, n_end);
      } else if constexpr (WORK == kOut) {
        if constexpr (!kEight) {
          if (g.pre != nullptr) {
            T* sums = static_cast<T*>(g.pre) + m * 2 * g.cols;
            store_block<T>(first, sums, inside, rows.there[i], n, n_end);
            store_block<T>(second, sums + g.cols, inside, rows.there[i], n, n_end);
          }
        }
#pragma unroll
        for (int x = 0; x < 16; ++x) first[x] = act_value<ACT, kFine>(first[x], nullptr) * second[x];
        store_block<OUT>(first, row, inside, rows.there[i], n, n_end);
      } else {
#pragma unroll
        for (int x = 0; x < 16; ++x) {
          float slope;
          const float tv = to_f32(t[i][x / 4].v[x % 4]), value = act_value<ACT, kFine>(first[x], &slope);
          first[x] = tv * second[x] * slope;
          second[x] = tv * value;
        }
        // (rounded to the operands' type, which the matrix instructions of the gradients take)
        store_block<OUT>(first, row, inside, rows.there[i], n, n_end);
        store_block<OUT>(second, row + g.c_stride / 2, inside, rows.there[i], n, n_end);
      }
    }
  }
}

template <class T, class OUT, Work WORK, int MI, int NJ, class ACC>
__device__ __forceinline__ void finish_act(const ACC (&acc)[MI][NJ], const FeedArgs& g, const RowsOfTile<MI>& rows, int expert,
                                           int64_t m0, int64_t m_end, int64_t n0, int64_t n_end) {
  if constexpr (!is_pair(WORK)) {
    finish_tile<T, OUT, WORK, 0>(acc, g, rows, expert, m0, m_end, n0, n_end);
  } else {
    if (g.act == kSilu) finish_tile<T, OUT, WORK, kSilu>(acc, g, rows, expert, m0, m_end, n0, n_end);
    else if (g.act == kGelu) finish_tile<T, OUT, WORK, kGelu>(acc, g, rows, expert, m0, m_end, n0, n_end);
    else if (g.act == kGeluTanh) finish_tile<T, OUT, WORK, kGeluTanh>(acc, g, rows, expert, m0, m_end, n0, n_end);
    else finish_tile<T, OUT, WORK, kRelu>(acc, g, rows, expert, m0, m_end, n0, n_end);
  }
}

// ---- launchers: which kernel takes a call is decided in feed_forward.hip -----------------------------------------------------
// tiles of feed_tiles.hpp: rows of any alignment.  float32 takes kSmall
template <class T>
int launch_feed_tiles(const FeedArgs& g, bool k_contiguous, Work work, TileKind kind, hipStream_t stream);
// tiles of feed_large.hpp: whole, aligned 16-byte parts, limit > 0; not float32
template <class T>
int launch_feed_large(const FeedArgs& g, bool k_contiguous, Work work, hipStream_t stream);

// feed_few.hip: few rows per expert, limit > 0, W contiguous in k, 16 bytes of it at least; not kBoth
template <class T>
int launch_feed_few(const FeedArgs& g, Work work, hipStream_t stream);

// feed_thin.hpp: few tiles, `narrow` for half as many columns each; otherwise as feed_few.hip
template <class T>
int launch_feed_thin(const FeedArgs& g, Work work, bool narrow, hipStream_t stream);

// feed_across.hpp: few tiles, W contiguous in n, limit > 0, 16 bytes of k and 128 columns (64 of a pair) at least, `narrow` half as
// many; not 8 bits
template <class T>
int launch_feed_across(const FeedArgs& g, Work work, bool narrow, hipStream_t stream);

// feed_weights.hip: both weights' gradients of whole, aligned 16-byte parts, not float32.  w: slopes (of the gate) and x, or x and
// slopes where x_first; few enough tiles for one launch, strides below 2^32 bytes
int64_t both_weights_tiles(const WeightArgs& g);
int launch_both_weights(int type, const WeightArgs& w, bool x_first, int64_t apart, void* c, void* c_up, hipStream_t stream);

// elementwise: slopes from the sums that the forward pass kept
int launch_slopes(int type, const FeedArgs& g, hipStream_t stream);

struct GatedArgs {
  ProductArgs p;             // w: gate, ho: f; out, dx; dw: gate
  const void* w_up;
  void *pre, *dw_up;
  const void* kept;          // pre of the forward pass or null
  int act;
  void* scratch;
};
int64_t slopes_stride(int type, int64_t f);      // elements between rows of slopes
int launch_gated_fwd(int type, const GatedArgs& g, hipStream_t stream);
int launch_gated_vjp(int type, const GatedArgs& g, hipStream_t stream);

struct EightArgs {
  const int8_t* x;
  int64_t x_stride, m;
  const float* x_scale;
  const int8_t *w, *w_up;    // w_up null: the plain product
  int64_t w_expert, w_out;
  const float *w_scale, *up_scale;
  const int32_t *offset, *source;
  int64_t k, slots;
  int n;
  int64_t h, f;
  int act, out_type;
  void* out;
};
int launch_eight(const EightArgs& g, hipStream_t stream);

struct QuantiseArgs {
  const void* x;
  int64_t x_stride, m, h;
  int8_t* q;
  float* scale;
};
int launch_quantise(int type, const QuantiseArgs& g, hipStream_t stream);

}  // namespace topk
