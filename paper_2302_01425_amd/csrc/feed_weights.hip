// Gradients of both weights of a gated block (feed_forward.hip) where every row is made of whole, aligned 16-byte parts: tiles of 256
// x 256 outputs, operands loaded straight to LDS as in feed_large.hpp.
//
// Four wavefronts hold 128 x 128 sums each.  A step is 32 places, whose rows of 512 bytes per operand are read transposed; four
// stages of 32 KB, so that a step's loads have three steps to arrive.  The gate's and the up projection's tiles are dealt as those of
// one array, every die an eighth of every expert's (split_tiles).  Slopes of a place without a row of x are zeros; its row of x,
// and what lies behind an expert's last place, is read as zeros.
//
// Two thirds of the operand bytes per output of tiles of 128 x 256 (expert_product_tiles.hip, both weights in one launch too), but nothing
// overlaps a tile's stores, so for experts of many places.  Slopes of kept sums and both weights, bfloat16, these / those, rows in expert
// order; found through source: 2048 x 2048, 32 experts of 512 places 484 / 432 us; 509 / 449, 16 of 1024 375 / 355; 395 / 388, 12 of 1280 330
// / 323; 347 / 348, 10 of 1536 315 / 310; 331 / 338, 8 of 2048 317 / 322; 335 / 350, 2 of 8192 271 / 295; 287 / 323.  1024 x 1024, 16 of 1024
// 103 / 101; 108 / 111, of 1536 144 / 150; 151 / 162.  4096 x 4096, one of 512 55 / 53; 58 / 58, of 1024 80 / 81; 87 / 92, of 2048 134 /
// 144; 145 / 161.  8192 x 4096 from 8192 places 877 / 1015; 963 / 1120.  The weights alone: 865 us, 1.27 PFLOP/s.
#include "feed_forward.hpp"

namespace topk {
namespace {

constexpr int kThreads = 256, kTile = 256, kStep = 64, kStages = 4, kStage = 2 * kTile * kStep;

struct BothWeightsArgs {
  WeightArgs w;              // a, b: slopes and x, or x and slopes; m, cols: those of one weight; tiles: of both together
  int64_t apart;             // bytes from dg to du
  void *c, *c_up;
  int32_t m_tiles, col_tiles;      // of one weight
};

// An operand with one row per k.  LISTED: rows of x behind an expert's places, looked up in `table`.
template <class IMAGE, bool LISTED>
struct Columns {
  using T = typename IMAGE::Type;
  static constexpr int kParts = IMAGE::kParts;
  const char* p[kParts];     // the parts' columns of the first place's row (LISTED: of row 0)
  int64_t stride, ahead;     // bytes; ahead: from the first step to the one that is loaded
  Table table;
  int64_t depth, k0;
  int32_t row[LISTED ? kParts : 1];

  __device__ __forceinline__ void init(const void* from, int64_t row_stride, int64_t first, int64_t end, int64_t begin, int64_t places) {
    stride = row_stride * int64_t(sizeof(T));
    depth = places;
    k0 = 0, ahead = 0;
    const char* base = static_cast<const char*>(from) + first * int64_t(sizeof(T));
#pragma unroll
    for (int i = 0; i < kParts; ++i) {
      p[i] = base + min(int64_t(IMAGE::part_of(i) * IMAGE::N), end - IMAGE::N - first) * int64_t(sizeof(T));
      if (!LISTED) p[i] += (begin + IMAGE::row_of(i)) * stride;
    }
  }
  __device__ __forceinline__ void next() {
    k0 += IMAGE::kStepK;
    ahead += IMAGE::kStepK * stride;
  }
  // LISTED: the rows of the step that is loaded
  __device__ __forceinline__ void fetch() {
    if constexpr (LISTED) {
      if ((k0 & (kTable - 1)) == 0) table.fill<kThreads>(k0, depth);
#pragma unroll
      for (int i = 0; i < kParts; ++i) row[i] = table.rows[(int(k0) + IMAGE::row_of(i)) & (kTable - 1)];
    }
  }
  // part i of the step; INSIDE: it does not cross the end
  template <bool INSIDE>
  __device__ __forceinline__ void issue(int i, uint32_t to) const {
    const int wave = __builtin_amdgcn_readfirstlane(int(threadIdx.x) / kWave);
    const char *from, *zeros = reinterpret_cast<const char*>(&zero_part);
    if constexpr (LISTED) {
      // (places behind the end have no row either)
      from = (row[i] >= 0 ? p[i] : zeros) + uint64_t(uint32_t(max(row[i], 0))) * uint32_t(stride);
    } else {
      from = p[i] + ahead;
      if constexpr (!INSIDE) from = k0 + IMAGE::row_of(i) < depth ? from : zeros;
    }
    load_to_lds(from, to + (i * kThreads + wave * kWave) * 16);
  }
};

// LIST: the operand that is x and has a source (0: neither, 1: A, 2: B).  X_FIRST: A is x
template <class T, int LIST, bool X_FIRST>
__global__ __launch_bounds__(kThreads, 1) void both_weights_kernel(BothWeightsArgs g) {
  __shared__ __attribute__((aligned(1024))) char lds[kStages * kStage];
  __shared__ int32_t rows[LIST != 0 ? kTable : 1];
  __shared__ uint32_t there[LIST != 0 ? kTable / 32 : 1];
  using I = Image<T, false, kTile, kThreads, kStep>;
  constexpr int MI = kTile / 2 / 32, NJ = MI, kReads = MI + NJ, kTurns = MI * NJ / 2, kLoads = 2 * I::kParts;
  int e;
  int64_t m, col;
  if (!find_weight_tile(g.w, g.w.first + blockIdx.x, &e, &m, &col)) return;
  const bool up = X_FIRST ? col >= g.col_tiles : m >= g.m_tiles;
  if (up && X_FIRST) col -= g.col_tiles;
  if (up && !X_FIRST) m -= g.m_tiles;
  int64_t begin, end;
  places(g.w.offset, e, g.w.slots, &begin, &end);
  T* c = static_cast<T*>(up ? g.c_up : g.c) + e * g.w.m * g.w.cols;
  if (begin == end) {
    store_zeros<kThreads>(c, g.w.m * g.w.cols, m * g.col_tiles + col, int64_t(g.m_tiles) * g.col_tiles);
    return;
  }
  const int64_t m0 = m * kTile, n0 = col * kTile;
  const char *pa = static_cast<const char*>(g.w.a), *pb = static_cast<const char*>(g.w.b);
  if (up) (X_FIRST ? pb : pa) += g.apart;
  Columns<I, LIST == 1> a;
  Columns<I, LIST == 2> b;
  a.init(pa, g.w.a_stride, m0, g.w.m, begin, end - begin);
  b.init(pb, g.w.b_stride, n0, g.w.cols, begin, end - begin);
  a.table = b.table = Table{rows, there, LIST == 0 ? nullptr : (LIST == 1 ? g.w.a_source : g.w.b_source) + begin, g.w.div,
                            LIST == 1 ? g.w.a_limit : g.w.b_limit};

  const uint32_t to = lds_address(lds);
  const int wave = int(threadIdx.x) / kWave;
  const int wm = (wave & 1) * (kTile / 2), wn = (wave >> 1) * (kTile / 2);
  const int steps = int((end - begin + I::kStepK - 1) / I::kStepK);
  const auto issue = [&](int i, int stage, auto inside) {
    constexpr bool kInside = decltype(inside)::value;
    if (i < I::kParts) a.template issue<kInside>(i, to + stage * kStage);
    else b.template issue<kInside>(i - I::kParts, to + stage * kStage + kTile * kStep);
  };
#pragma unroll
  for (int s = 0; s < kStages - 1; ++s) {
    a.fetch(), b.fetch();
#pragma unroll
    for (int i = 0; i < kLoads; ++i) issue(i, s, std::false_type{});
    a.next(), b.next();
  }
  f32x16 acc[MI][NJ];
  clear(acc);
  Fragment<T> fa[2][MI], fb[2][NJ];
  const auto read = [&](int i, int stage, int t) {
    const char* at = lds + stage * kStage;
    if (i < NJ) fb[t][i] = I::read(at + kTile * kStep, wn + 32 * i, t);
    else fa[t][i - NJ] = I::read(at, wm + 32 * (i - NJ), t);
  };
  // the fragments t multiplied; between the instructions those of `other` are read
  const auto multiply = [&](int t, int stage, int other, auto between) {
#pragma unroll
    for (int q = 0; q < kTurns; ++q) {
#pragma unroll
      for (int x = 2 * q; x < 2 * q + 2; ++x) acc[x / NJ][x % NJ] = mma(0, fb[t][x % NJ], fa[t][x / NJ], acc[x / NJ][x % NJ]);
#pragma unroll
      for (int i = q * kReads / kTurns; i < (q + 1) * kReads / kTurns; ++i) read(i, stage, other);
      between(q);
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  wait_stage<(kStages - 2) * kLoads>();
  a.fetch(), b.fetch();
#pragma unroll
  for (int i = 0; i < kLoads; ++i) issue(i, kStages - 1, std::false_type{});
  a.next(), b.next();
#pragma unroll
  for (int i = 0; i < kReads; ++i) read(i, 0, 0);
  int stage = 0;
  // a step, while the one four behind it is loaded (steps behind the last: zeros)
  const auto one = [&](auto inside) {
    const int after = stage + 1 == kStages ? 0 : stage + 1;
    multiply(0, stage, 1, [](int) {});
    a.fetch(), b.fetch();
    // everything of this step is in registers, and the next step is there
    wait_stage<(kStages - 2) * kLoads>();
    multiply(1, after, 0, [&](int q) {
#pragma unroll
      for (int i = q * kLoads / kTurns; i < (q + 1) * kLoads / kTurns; ++i) issue(i, stage, inside);
    });
    a.next(), b.next();
    stage = after;
  };
  const int whole = int((end - begin) / I::kStepK) - kStages;      // steps behind which a whole one is loaded
  int step = 0;
  for (; step < whole; ++step) one(std::true_type{});
  for (; step < steps; ++step) one(std::false_type{});
  wait_stage<0>();           // (no load may reach LDS that is another workgroup's by then)
  store_tile(acc, m0 + wm, g.w.m, n0 + wn, g.w.cols, nullptr, Divisor{}, 0, c, g.w.cols);
}

template <class T>
int both_weights(const BothWeightsArgs& g, int64_t blocks, bool x_first, hipStream_t stream) {
  const dim3 grid(static_cast<unsigned>(blocks)), block(kThreads);
  if (x_first) {
    if (g.w.a_source != nullptr) hipLaunchKernelGGL((both_weights_kernel<T, 1, true>), grid, block, 0, stream, g);
    else hipLaunchKernelGGL((both_weights_kernel<T, 0, true>), grid, block, 0, stream, g);
  } else {
    if (g.w.b_source != nullptr) hipLaunchKernelGGL((both_weights_kernel<T, 2, false>), grid, block, 0, stream, g);
    else hipLaunchKernelGGL((both_weights_kernel<T, 0, false>), grid, block, 0, stream, g);
  }
  return 0;
}

}  // namespace

int64_t both_weights_tiles(const WeightArgs& g) {
  return 2 * g.n * ((g.m + kTile - 1) / kTile) * ((g.cols + kTile - 1) / kTile);
}

int launch_both_weights(int type, const WeightArgs& w, bool x_first, int64_t apart, void* c, void* c_up, hipStream_t stream) {
  BothWeightsArgs g{};
  g.w = w;
  g.m_tiles = int32_t((w.m + kTile - 1) / kTile), g.col_tiles = int32_t((w.cols + kTile - 1) / kTile);
  WeightArgs stacked = w;              // tiles of both weights as those of one array
  stacked.m = int64_t(g.m_tiles) * kTile * (x_first ? 1 : 2), stacked.cols = int64_t(g.col_tiles) * kTile * (x_first ? 2 : 1);
  const int64_t blocks = split_tiles(&stacked, kTile, kTile);
  g.w.m_tiles = stacked.m_tiles, g.w.col_tiles = stacked.col_tiles, g.w.die_m = stacked.die_m, g.w.die_cols = stacked.die_cols;
  g.w.first = 0;
  g.apart = apart, g.c = c, g.c_up = c_up;
  if (type == kBF16) return both_weights<bf16>(g, blocks, x_first, stream);
  if (type == kF16) return both_weights<f16>(g, blocks, x_first, stream);
  return -1;
}

}  // namespace topk
