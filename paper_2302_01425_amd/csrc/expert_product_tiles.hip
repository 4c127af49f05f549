// The experts' products (expert_product.hip) where every row is made of whole, aligned 16-byte parts: tiles of 128 x 256
// outputs, operands brought from global memory to LDS by the load that goes there directly, two steps ahead.
//
// A workgroup of four wavefronts holds 128 x 256 float32 sums in registers, 64 x 128 per wavefront: 12 fragments of 1 KB read
// from LDS feed 32 matrix instructions of 16 cycles, 384 cycles of the LDS against 512 of the matrix unit.  A step is 64 bytes
// of k, 24 KB of LDS for both operands; three steps are 72 KB, so two workgroups share a compute unit and one computes while
// the other waits at its barrier.
//
// LDS images.  Operand contiguous in k: rows of four 16-byte parts, part p of row r at place p ^ 3 (r / 8 % 2): a quarter of
// a 16-byte read takes lanes 0..3, 12..15, 20..27 (then 4..11, 16..19, 28..31, and so on), which then meet 16 different bank
// groups; p ^ (r / 4 % 4) leaves conflicts of two.  Operand contiguous in m or n: rows of one k each.  16-bit types are read
// transposed (a quarter of a wavefront reads 4 rows of 16 elements and gets 4 k of one column per lane); blocks of 32 bytes are
// exchanged by k % 4 and k / 8 % 2, which the eight rows read at a time differ in.  float32 is read element by element; blocks
// of 64 bytes are exchanged by k / 4.
#include "expert_product.hpp"

namespace topk {
namespace {

constexpr int kThreads = kProductThreads;
constexpr int kRows = 128, kCols = 256;    // of a tile (A, B)
constexpr int kStep = 64;                  // bytes of k
constexpr int kStages = 3;
constexpr int kStageBytes = (kRows + kCols) * kStep;

__device__ uint4 zero_part;                // 16 bytes of zeros, read in the place of what is out of range

// 16 bytes per lane from `from` to LDS at `to` (the same for the wavefront) + 16 * lane.  Not waited for, and unknown to the
// compiler's own waits: wait_stage() counts these loads.
__device__ __forceinline__ void load_to_lds(const char* from, uint32_t to) {
  asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off" ::"v"(from), "s"(to) : "memory");
}

constexpr int kTable = 1024;               // places whose rows are looked up at a time (dW)

// One operand of a tile of R rows: where this thread's parts come from.  KC: contiguous in k.  LISTED (not KC): the row of a
// place is looked up in `table`, an LDS array.
template <class T, bool KC, int R, bool LISTED = false>
struct Loader {
  static constexpr int N = 16 / sizeof(T);               // elements per part
  static constexpr int kParts = R * kStep / 16 / kThreads;
  static constexpr int kStepK = kStep / int(sizeof(T));
  static constexpr int kAlong = KC ? kStep / 16 : R / N; // parts of a row of the LDS image
  const char* p[kParts];     // KC: the part at k = 0 of its row; LISTED: its column of row 0; else: the part of the next step
  int64_t stride;            // bytes between rows (not KC)
  const int32_t* table;

  // part i of this thread: row of the LDS image, and which part of that row of the operand lies there
  static __device__ __forceinline__ int row_of(int i) {
    return (i * kThreads + int(threadIdx.x)) / kAlong;
  }
  static __device__ __forceinline__ int part_of(int i) {
    const int c = (i * kThreads + int(threadIdx.x)) % kAlong, r = row_of(i);
    if constexpr (KC) return c ^ ((r >> 3) & 1) * 3;
    else if constexpr (sizeof(T) == 2) return c ^ (((r & 3) | ((r >> 3) & 1) << 2) << 1);
    else return c ^ (((r >> 2) & 3) << 2);
  }

  // Rows [first, end) of an operand contiguous in k, found through source where there is one.  Rows behind the last, and rows
  // whose place has none, are read from another row; their outputs are not stored, or stored as zeros.
  __device__ __forceinline__ void init_rows(const void* base, int64_t row_stride, const int32_t* source, const Divisor& d,
                                            int64_t limit, int64_t first, int64_t end) {
#pragma unroll
    for (int i = 0; i < kParts; ++i) {
      int64_t row = min(first + row_of(i), end - 1);
      if (source != nullptr) row = min(int64_t(quotient(max(source[row], 0), d)), limit - 1);
      p[i] = static_cast<const char*>(base) + row * row_stride * int64_t(sizeof(T)) + part_of(i) * 16;
    }
  }
  // Columns [first, end) of an operand with one row per k, from row k_begin on; columns behind the last as above.
  __device__ __forceinline__ void init_columns(const void* base, int64_t row_stride, const int32_t* rows, int64_t first,
                                               int64_t end, int64_t k_begin) {
    stride = row_stride * int64_t(sizeof(T));
    table = rows;
#pragma unroll
    for (int i = 0; i < kParts; ++i) {
      const int64_t at = min(first + part_of(i) * N, end - N);
      p[i] = static_cast<const char*>(base) + at * int64_t(sizeof(T));
      if (!LISTED) p[i] += (k_begin + row_of(i)) * stride;
    }
  }

  // the step from k0 on to LDS at `to`, zeros from k_end on.  Steps come in order.
  __device__ __forceinline__ void issue(int64_t k0, int64_t k_end, uint32_t to) {
    const int wave = __builtin_amdgcn_readfirstlane(int(threadIdx.x) / kWave);
    const char* zeros = reinterpret_cast<const char*>(&zero_part);
    const char* from[kParts];
    if constexpr (LISTED) {
#pragma unroll
      for (int i = 0; i < kParts; ++i) {
        const int row = table[(int(k0) + row_of(i)) & (kTable - 1)];
        from[i] = row >= 0 ? p[i] + uint64_t(uint32_t(row)) * uint32_t(stride) : zeros;
      }
    } else {
#pragma unroll
      for (int i = 0; i < kParts; ++i) from[i] = KC ? p[i] + k0 * int64_t(sizeof(T)) : p[i];
      if (k0 + kStepK > k_end) {
#pragma unroll
        for (int i = 0; i < kParts; ++i)
          if (k0 + (KC ? part_of(i) * N : row_of(i)) >= k_end) from[i] = zeros;
      }
      if constexpr (!KC) {
#pragma unroll
        for (int i = 0; i < kParts; ++i) p[i] += kStepK * stride;
      }
    }
#pragma unroll
    for (int i = 0; i < kParts; ++i) load_to_lds(from[i], to + (i * kThreads + wave * kWave) * 16);
  }

  // 16 bytes of k of row lane % 16 of the 16 rows from r0 (a multiple of 16)
  static __device__ __forceinline__ Fragment<T> read(const char* lds, int r0) {
    const int lane = int(threadIdx.x) & (kWave - 1), g = lane >> 4, l = lane & 15;
    if constexpr (KC) {
      return *reinterpret_cast<const Fragment<T>*>(lds + (r0 + l) * kStep + ((g ^ (l >> 3) * 3) << 4));
    } else if constexpr (sizeof(T) == 2) {
      typedef short s4 __attribute__((ext_vector_type(4)));
      typedef __attribute__((address_space(3))) s4* Lds4;
      const int f = (l >> 2) | (g & 1) << 2;
      const char* at = lds + (8 * g + (l >> 2)) * (R * 2) + (((r0 >> 4) ^ f) << 5) + (l & 3) * 8;
      union {
        s4 half[2];
        Fragment<T> whole;
      } u;
      u.half[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds4)at);
      u.half[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds4)(at + 4 * R * 2));
      return u.whole;
    } else {
      const char* at = lds + 4 * g * (R * 4) + (((r0 >> 4) ^ g) << 6) + l * 4;
      Fragment<T> v;
#pragma unroll
      for (int j = 0; j < 4; ++j) v[j] = *reinterpret_cast<const float*>(at + j * R * 4);
      return v;
    }
  }
};

// all loads to LDS but the last LEFT of this wavefront have arrived, all reads of LDS are done, and so for every wavefront
template <int LEFT>
__device__ __forceinline__ void wait_stage() {
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(LEFT) : "memory");
}

// Rows of places, filled kTable places at a time (dW).
struct Table {
  int32_t* rows;             // LDS, kTable of them
  const int32_t* source;
  Divisor div;
  int64_t limit;
  // places from k0 (a multiple of the table's size behind k_begin) on
  __device__ __forceinline__ void fill(int64_t k0, int64_t k_end) const {
    __syncthreads();
    for (int i = threadIdx.x; i < kTable; i += kThreads) {
      const int pair = k0 + i < k_end ? source[k0 + i] : -1;
      const int row = quotient(max(pair, 0), div);
      rows[(int(k0) + i) & (kTable - 1)] = pair >= 0 && row < limit ? row : -1;
    }
    __syncthreads();
  }
};

// C(m, n) of one tile: sums over k of [k_begin, k_end).  `source` of the rows of A (rows without one are stored as zeros).
template <class T, class LA, class LB, bool LISTED>
__device__ __forceinline__ void tile_product(LA& a, LB& b, const Table& table, int64_t m0, int64_t m_end, int64_t n0,
                                             int64_t n_end, int64_t k_begin, int64_t k_end, const int32_t* source,
                                             const Divisor& div, int64_t limit, T* c, int64_t c_stride) {
  constexpr int kLoads = LA::kParts + LB::kParts;
  __shared__ __attribute__((aligned(1024))) char lds[kStages * kStageBytes];
  const uint32_t lds0 = uint32_t(uintptr_t((__attribute__((address_space(3))) char*)lds));
  const int lane = int(threadIdx.x) & (kWave - 1), wave = int(threadIdx.x) / kWave;
  const int wm = (wave & 1) * (kRows / 2), wn = (wave >> 1) * (kCols / 2);
  constexpr int MI = kRows / 2 / 16, NJ = kCols / 2 / 16;
  f32x4 acc[MI][NJ];
#pragma unroll
  for (int i = 0; i < MI; ++i)
#pragma unroll
    for (int j = 0; j < NJ; ++j) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};

  if (k_begin < k_end) {
    // steps behind the last are loaded as zeros: the count of loads in flight stays the same
    const auto issue = [&](int64_t k, int stage) {
      if constexpr (LISTED) {
        if (((k - k_begin) & (kTable - 1)) == 0) table.fill(k, k_end);
      }
      a.issue(k, k_end, lds0 + stage * kStageBytes);
      b.issue(k, k_end, lds0 + stage * kStageBytes + kRows * kStep);
    };
    issue(k_begin, 0);
    issue(k_begin + LA::kStepK, 1);
    int stage = 0;
    for (int64_t k0 = k_begin; k0 < k_end; k0 += LA::kStepK) {
      wait_stage<kLoads>();
      issue(k0 + 2 * LA::kStepK, stage == 0 ? 2 : stage - 1);
      const char* la = lds + stage * kStageBytes;
      const char* lb = la + kRows * kStep;
      Fragment<T> fa[MI], fb[NJ];
#pragma unroll
      for (int i = 0; i < MI; ++i) fa[i] = LA::read(la, wm + 16 * i);
#pragma unroll
      for (int j = 0; j < NJ; ++j) fb[j] = LB::read(lb, wn + 16 * j);
#pragma unroll
      for (int j = 0; j < NJ; ++j)
#pragma unroll
        for (int i = 0; i < MI; ++i) acc[i][j] = mma(fb[j], fa[i], acc[i][j]);
      stage = stage == kStages - 1 ? 0 : stage + 1;
    }
    wait_stage<0>();         // (no load may reach LDS that is another workgroup's by then)
  }

  // lane l has row l % 16 of A and four neighbouring columns: n along the rows of the instruction's output
#pragma unroll
  for (int i = 0; i < MI; ++i) {
    const int64_t m = m0 + wm + 16 * i + (lane & 15);
    if (m >= m_end) continue;
    bool there = true;
    if (source != nullptr) there = source[m] >= 0 && quotient(source[m], div) < limit;
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
      const int64_t n = n0 + wn + 16 * j + (lane >> 4) * 4;
      if (n >= n_end) continue;                          // (columns come in whole 16-byte parts)
      Packed<T, 4> q;
#pragma unroll
      for (int r = 0; r < 4; ++r) q.v[r] = from_f32<T>(there ? acc[i][j][r] : 0.0f);
      *reinterpret_cast<Packed<T, 4>*>(c + m * c_stride + n) = q;
    }
  }
}

template <class T, bool B_KC>
__global__ __launch_bounds__(kThreads, 2) void rows_tiles_kernel(RowsArgs g) {
  Found f;
  if (!find_tile(g.offset, g.n, g.slots, blockIdx.x, g.col_tiles, kRows, &f)) return;
  const int64_t n0 = f.col * kCols;
  const T* w = static_cast<const T*>(g.w) + f.expert * g.w_expert;
  Loader<T, true, kRows> a;
  a.init_rows(g.a, g.a_stride, g.source, g.div, g.limit, f.begin, f.end);
  Loader<T, B_KC, kCols> b;
  if constexpr (B_KC) b.init_rows(w, g.w_stride, nullptr, Divisor{}, 0, n0, g.cols);
  else b.init_columns(w, g.w_stride, nullptr, n0, g.cols, 0);
  tile_product<T, Loader<T, true, kRows>, Loader<T, B_KC, kCols>, false>(a, b, Table{}, f.begin, f.end, n0, g.cols, 0, g.depth,
                                                                         g.source, g.div, g.limit, static_cast<T*>(g.c),
                                                                         g.cols);
}

// LIST: which operand's rows are found through source (0: neither, 1: A, 2: B)
template <class T, int LIST>
__global__ __launch_bounds__(kThreads, 2) void weight_tiles_kernel(WeightArgs g) {
  __shared__ int32_t rows[LIST != 0 ? kTable : 1];
  const int64_t tile = die_order(blockIdx.x, g.n * g.m_tiles * g.col_tiles);
  if (tile < 0) return;
  const int64_t col = tile % g.col_tiles, rest = tile / g.col_tiles;
  const int e = int(rest / g.m_tiles);
  int64_t begin, end;
  places(g.offset, e, g.slots, &begin, &end);
  const int64_t m0 = (rest % g.m_tiles) * kRows, n0 = col * kCols;
  using LA = Loader<T, false, kRows, LIST == 1>;
  using LB = Loader<T, false, kCols, LIST == 2>;
  LA a;
  a.init_columns(g.a, g.a_stride, rows, m0, g.m, begin);
  LB b;
  b.init_columns(g.b, g.b_stride, rows, n0, g.cols, begin);
  const Table table{rows, LIST == 1 ? g.a_source : g.b_source, g.div, LIST == 1 ? g.a_limit : g.b_limit};
  tile_product<T, LA, LB, LIST != 0>(a, b, table, m0, g.m, n0, g.cols, begin, end, nullptr, Divisor{}, 0,
                                     static_cast<T*>(g.c) + e * g.m * g.cols, g.cols);
}

template <class T>
int rows_type(const RowsArgs& g, bool k_contiguous, int64_t blocks, hipStream_t stream) {
  if (k_contiguous)
    hipLaunchKernelGGL((rows_tiles_kernel<T, true>), dim3(unsigned(blocks)), dim3(kThreads), 0, stream, g);
  else
    hipLaunchKernelGGL((rows_tiles_kernel<T, false>), dim3(unsigned(blocks)), dim3(kThreads), 0, stream, g);
  return 0;
}
template <class T>
int weight_type(const WeightArgs& g, int64_t blocks, hipStream_t stream) {
  const dim3 grid = dim3(unsigned(blocks)), block(kThreads);
  if (g.a_source != nullptr) hipLaunchKernelGGL((weight_tiles_kernel<T, 1>), grid, block, 0, stream, g);
  else if (g.b_source != nullptr) hipLaunchKernelGGL((weight_tiles_kernel<T, 2>), grid, block, 0, stream, g);
  else hipLaunchKernelGGL((weight_tiles_kernel<T, 0>), grid, block, 0, stream, g);
  return 0;
}

bool whole_parts(const void* p, int64_t stride, int64_t length, int size) {
  return reinterpret_cast<uintptr_t>(p) % 16 == 0 && stride * size % 16 == 0 && length * size % 16 == 0;
}
int size_of(int type) { return type == kF32 ? 4 : 2; }

}  // namespace

bool rows_aligned(int type, const RowsArgs& g, bool k_contiguous) {
  const int s = size_of(type);
  // (without a row of x every place would be read from nowhere)
  return g.limit > 0 && whole_parts(g.a, g.a_stride, g.depth, s) && whole_parts(g.w, g.w_stride, k_contiguous ? g.depth : g.cols, s) &&
         g.w_expert * s % 16 == 0 && whole_parts(g.c, g.cols, g.cols, s);
}

bool weight_aligned(int type, const WeightArgs& g) {
  const int s = size_of(type);
  return g.a_stride * s < (int64_t(1) << 32) && g.b_stride * s < (int64_t(1) << 32) &&       // (32-bit products of rows)
         whole_parts(g.a, g.a_stride, g.m, s) && whole_parts(g.b, g.b_stride, g.cols, s) && whole_parts(g.c, g.cols, g.cols, s);
}

int launch_rows_tiles(int type, RowsArgs g, bool k_contiguous, hipStream_t stream) {
  g.col_tiles = (g.cols + kCols - 1) / kCols;
  const int64_t blocks = (g.slots / kRows + min(int64_t(g.n), g.slots)) * g.col_tiles + kDies - 1;
  if (blocks >= (int64_t(1) << 31)) return -1;
  if (type == kF32) return rows_type<float>(g, k_contiguous, blocks, stream);
  if (type == kBF16) return rows_type<bf16>(g, k_contiguous, blocks, stream);
  if (type == kF16) return rows_type<f16>(g, k_contiguous, blocks, stream);
  return -1;
}

int launch_weight_tiles(int type, WeightArgs g, hipStream_t stream) {
  g.m_tiles = (g.m + kRows - 1) / kRows;
  g.col_tiles = (g.cols + kCols - 1) / kCols;
  const int64_t blocks = g.n * g.m_tiles * g.col_tiles + kDies - 1;
  if (blocks >= (int64_t(1) << 31)) return -1;
  if (type == kF32) return weight_type<float>(g, blocks, stream);
  if (type == kBF16) return weight_type<bf16>(g, blocks, stream);
  if (type == kF16) return weight_type<f16>(g, blocks, stream);
  return -1;
}

}  // namespace topk
