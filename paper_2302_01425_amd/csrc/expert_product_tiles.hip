// The experts' products (expert_product.hip) where every row is made of whole, aligned 16-byte parts: tiles of 128 x 256
// outputs, operands brought from global memory to LDS by the load that goes there directly, two steps ahead.
//
// A workgroup of four wavefronts holds 128 x 256 float32 sums in registers, 64 x 128 per wavefront: 12 fragments of 1 KB read
// from LDS feed 32 matrix instructions of 16 cycles, 384 cycles of the LDS against 512 of the matrix unit.  A step is 64 bytes
// of k, 24 KB of LDS for both operands; three steps are 72 KB, so two workgroups share a compute unit and one computes while
// the other waits at its barrier.
//
// LDS images.  Operand contiguous in k: rows of four 16-byte parts, part p of row r at place p ^ (r / 4 % 4): the 16 rows of a
// fragment then lie in 16 different bank groups.  Operand contiguous in m or n: rows of one k each.  16-bit types are read
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

// One operand of a tile of R rows: where this thread's parts come from.
template <class T, bool KC, int R>
struct Loader {
  static constexpr int N = 16 / sizeof(T);               // elements per part
  static constexpr int kParts = R * kStep / 16 / kThreads;
  static constexpr int kStepK = kStep / int(sizeof(T));
  static constexpr int kAlong = KC ? kStep / 16 : R / N; // parts of a row of the LDS image
  const char* p[kParts];     // KC: the part in its row (null: a row of zeros); else: its column in row 0 (null: out)
  int64_t stride;            // bytes between rows (not KC)
  const int32_t* source;
  Divisor div;
  int64_t limit;

  // part i of this thread: row of the LDS image, and which part of that row of the operand lies there
  static __device__ __forceinline__ int row_of(int i) {
    return (i * kThreads + int(threadIdx.x)) / kAlong;
  }
  static __device__ __forceinline__ int part_of(int i) {
    const int c = (i * kThreads + int(threadIdx.x)) % kAlong, r = row_of(i);
    if constexpr (KC) return c ^ ((r >> 2) & 3);
    else if constexpr (sizeof(T) == 2) return c ^ (((r & 3) | ((r >> 3) & 1) << 2) << 1);
    else return c ^ (((r >> 2) & 3) << 2);
  }

  // rows [first, end) of the operand, KC: found through source
  __device__ __forceinline__ void init(const void* base, int64_t stride_elements, const int32_t* src, const Divisor& d,
                                       int64_t lim, int64_t first, int64_t end) {
    stride = stride_elements * int64_t(sizeof(T));
    source = src;
    div = d;
    limit = lim;
    const char* b = static_cast<const char*>(base);
#pragma unroll
    for (int i = 0; i < kParts; ++i) {
      if constexpr (KC) {
        int64_t row = min(first + row_of(i), end - 1);   // (rows behind the last are computed and not stored)
        bool there = true;
        if (source != nullptr) {
          const int pair = source[row];
          row = quotient(max(pair, 0), div);
          there = pair >= 0;
        }
        p[i] = there && row < limit ? b + row * stride + part_of(i) * 16 : nullptr;
      } else {
        const int64_t at = first + part_of(i) * N;
        p[i] = at < end ? b + at * int64_t(sizeof(T)) : nullptr;
      }
    }
  }

  // the step k0 .. (k_end: of the operand) to LDS at `to`
  __device__ __forceinline__ void issue(int64_t k0, int64_t k_end, uint32_t to) const {
    const int wave = __builtin_amdgcn_readfirstlane(int(threadIdx.x) / kWave);
    const char* zeros = reinterpret_cast<const char*>(&zero_part);
#pragma unroll
    for (int i = 0; i < kParts; ++i) {
      const char* from;
      if constexpr (KC) {
        const bool in = k0 + part_of(i) * N < k_end;
        from = in && p[i] != nullptr ? p[i] + k0 * int64_t(sizeof(T)) : zeros;
      } else {
        const int64_t k = k0 + row_of(i);
        bool in = k < k_end && p[i] != nullptr;
        int64_t row = k;
        if (source != nullptr) {
          // a wavefront's part lies in few rows, whose places are read through the scalar cache: vector loads would wait for
          // the loads to LDS before them
          constexpr int kPer = kWave / kAlong > 0 ? kWave / kAlong : 1;      // rows of a wavefront's part
          const int64_t r0 = k0 + (i * kThreads + wave * kWave) / kAlong;
          typedef const __attribute__((address_space(4))) int32_t* Scalar;
          int pair = -1;
#pragma unroll
          for (int q = 0; q < kPer; ++q) {
            const int v = ((Scalar)(uintptr_t)source)[min(r0 + q, k_end - 1)];
            if (k == r0 + q) pair = v;
          }
          in = in && pair >= 0;
          row = quotient(max(pair, 0), div);
          in = in && row < limit;
        }
        from = in ? p[i] + row * stride : zeros;
      }
      load_to_lds(from, to + (i * kThreads + wave * kWave) * 16);
    }
  }

  // 16 bytes of k of row lane % 16 of the 16 rows from r0 (a multiple of 16)
  static __device__ __forceinline__ Fragment<T> read(const char* lds, int r0) {
    const int lane = int(threadIdx.x) & (kWave - 1), g = lane >> 4, l = lane & 15;
    if constexpr (KC) {
      return *reinterpret_cast<const Fragment<T>*>(lds + (r0 + l) * kStep + ((g ^ (l >> 2)) << 4));
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

template <class T, bool A_KC, bool B_KC>
__device__ __forceinline__ void tile_product(const Loader<T, A_KC, kRows>& a, const Loader<T, B_KC, kCols>& b, int64_t m0,
                                             int64_t m_end, int64_t n0, int64_t n_end, int64_t k_begin, int64_t k_end, T* c,
                                             int64_t c_stride) {
  using LA = Loader<T, A_KC, kRows>;
  using LB = Loader<T, B_KC, kCols>;
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
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
      const int64_t n = n0 + wn + 16 * j + (lane >> 4) * 4;
      if (n >= n_end) continue;                          // (columns come in whole 16-byte parts)
      Packed<T, 4> q;
#pragma unroll
      for (int r = 0; r < 4; ++r) q.v[r] = from_f32<T>(acc[i][j][r]);
      *reinterpret_cast<Packed<T, 4>*>(c + m * c_stride + n) = q;
    }
  }
}

template <class T, bool B_KC>
__global__ __launch_bounds__(kThreads, 2) void rows_tiles_kernel(RowsArgs g) {
  Found f;
  if (!find_tile(g.offset, g.n, g.slots, blockIdx.x, g.col_tiles, kRows, &f)) return;
  const int64_t n0 = f.col * kCols;
  Loader<T, true, kRows> a;
  a.init(g.a, g.a_stride, g.source, g.div, g.limit, f.begin, f.end);
  Loader<T, B_KC, kCols> b;
  b.init(static_cast<const T*>(g.w) + f.expert * g.w_expert, g.w_stride, nullptr, Divisor{}, INT64_MAX, n0, g.cols);
  tile_product<T, true, B_KC>(a, b, f.begin, f.end, n0, g.cols, 0, g.depth, static_cast<T*>(g.c), g.cols);
}

template <class T>
__global__ __launch_bounds__(kThreads, 2) void weight_tiles_kernel(WeightArgs g) {
  const int64_t tile = die_order(blockIdx.x, g.n * g.m_tiles * g.col_tiles);
  if (tile < 0) return;
  const int64_t col = tile % g.col_tiles, rest = tile / g.col_tiles;
  const int e = int(rest / g.m_tiles);
  int64_t begin, end;
  places(g.offset, e, g.slots, &begin, &end);
  const int64_t m0 = (rest % g.m_tiles) * kRows, n0 = col * kCols;
  Loader<T, false, kRows> a;
  a.init(g.a, g.a_stride, g.a_source, g.div, g.a_limit, m0, g.m);
  Loader<T, false, kCols> b;
  b.init(g.b, g.b_stride, g.b_source, g.div, g.b_limit, n0, g.cols);
  tile_product<T, false, false>(a, b, m0, g.m, n0, g.cols, begin, end, static_cast<T*>(g.c) + e * g.m * g.cols, g.cols);
}

template <class T>
int rows_type(const RowsArgs& g, bool k_contiguous, int64_t blocks, hipStream_t stream) {
  if (k_contiguous)
    hipLaunchKernelGGL((rows_tiles_kernel<T, true>), dim3(unsigned(blocks)), dim3(kThreads), 0, stream, g);
  else
    hipLaunchKernelGGL((rows_tiles_kernel<T, false>), dim3(unsigned(blocks)), dim3(kThreads), 0, stream, g);
  return 0;
}

bool whole_parts(const void* p, int64_t stride, int64_t length, int size) {
  return reinterpret_cast<uintptr_t>(p) % 16 == 0 && stride * size % 16 == 0 && length * size % 16 == 0;
}
int size_of(int type) { return type == kF32 ? 4 : 2; }

}  // namespace

bool rows_aligned(int type, const RowsArgs& g, bool k_contiguous) {
  const int s = size_of(type);
  return whole_parts(g.a, g.a_stride, g.depth, s) && whole_parts(g.w, g.w_stride, k_contiguous ? g.depth : g.cols, s) &&
         g.w_expert * s % 16 == 0 && whole_parts(g.c, g.cols, g.cols, s);
}

bool weight_aligned(int type, const WeightArgs& g) {
  const int s = size_of(type);
  return whole_parts(g.a, g.a_stride, g.m, s) && whole_parts(g.b, g.b_stride, g.cols, s) && whole_parts(g.c, g.cols, g.cols, s);
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
  if (type == kF32) hipLaunchKernelGGL(weight_tiles_kernel<float>, dim3(unsigned(blocks)), dim3(kThreads), 0, stream, g);
  else if (type == kBF16) hipLaunchKernelGGL(weight_tiles_kernel<bf16>, dim3(unsigned(blocks)), dim3(kThreads), 0, stream, g);
  else if (type == kF16) hipLaunchKernelGGL(weight_tiles_kernel<f16>, dim3(unsigned(blocks)), dim3(kThreads), 0, stream, g);
  else return -1;
  return 0;
}

}  // namespace topk
