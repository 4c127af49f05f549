// Tiles of the experts' products: the images that operands have in LDS, the two ways that fill them, and how fragments of the
// matrix instructions are read from them.
#pragma once

#include "expert_product.hpp"

namespace topk {

__device__ const uint4 zero_part = {0, 0, 0, 0};     // read in the place of what is out of range

// LDS image of one step (STEP bytes of k) of an operand's R rows, cut into 16-byte parts.
// KC, the operand is contiguous in k: an image row is a row of the operand.  Parts of a row change places, so that a quarter of
// a 16-byte read (lanes 0..3, 12..15, 20..27; then 4..11, 16..19, 28..31; and so on) meets 16 different bank groups: part p of
// row r lies at p ^ (r / 2 % 8) with rows of 128 bytes, at p ^ (r / 4 % 4) with rows of 64.
// Else an image row is one k of all R.  16-bit types are read transposed (a quarter of a wavefront reads 4 rows of 16 elements
// and gets 4 k of one column per lane); half a wavefront reads 64 bytes of four rows, so blocks of 64 bytes change places by
// k % 4 (rows of 128 bytes: by k / 2 % 2, odd and even ones lie in different banks anyway).  float32 is read element by
// element, 128 bytes of two rows that are four apart; blocks of 128 bytes change places by k / 4 % 2.
template <class T, bool KC, int R, int THREADS, int STEP>
struct Image {
  using Type = T;
  static constexpr bool kKC = KC;
  static constexpr int kThreads = THREADS;
  static constexpr int N = 16 / sizeof(T);               // elements per part
  static constexpr int kBytes = R * STEP;
  static constexpr int kParts = kBytes / 16 / THREADS;   // per thread
  static constexpr int kStepK = STEP / int(sizeof(T));
  static constexpr int kAlong = KC ? STEP / 16 : R / N;  // parts of an image row
  static_assert(R >= 64 && (STEP == 64 || STEP == 128), "exchanges stay inside a row");

  // what the number of a part in image row r is changed by
  static __device__ __forceinline__ int exchange(int r) {
    if constexpr (KC && STEP == 128) return (r >> 1) & 7;
    else if constexpr (KC) return (r >> 2) & 3;
    else if constexpr (sizeof(T) == 4) return ((r >> 2) & 1) << 3;
    else if constexpr (R == 64) return ((r >> 1) & 1) << 2;
    else return (r & 3) << 2;
  }
  // the thread's part i lies at 16 (i THREADS + thread); its image row, and which part of the operand's row it is
  static __device__ __forceinline__ int row_of(int i) { return (i * THREADS + int(threadIdx.x)) / kAlong; }
  static __device__ __forceinline__ int part_of(int i) {
    return (i * THREADS + int(threadIdx.x)) % kAlong ^ exchange(row_of(i));
  }

  // 16 bytes of k of row lane % 32 of the 32 rows from r0 (a multiple of 32): those of lane / 32 in the 32 bytes from 32 t on
  static __device__ __forceinline__ Fragment<T> read(const char* lds, int r0, int t) {
    const int lane = int(threadIdx.x) & (kWave - 1), h = lane >> 5, l = lane & 31;
    if constexpr (KC) {
      return *reinterpret_cast<const Fragment<T>*>(lds + (r0 + l) * STEP + (((2 * t + h) ^ exchange(l)) << 4));
    } else if constexpr (sizeof(T) == 2) {
      typedef short s4 __attribute__((ext_vector_type(4)));
      typedef __attribute__((address_space(3))) s4* Lds4;
      const int q = lane & 15, row = 16 * t + 8 * h + (q >> 2);          // (row + 4 has the same exchange)
      const int part = ((r0 >> 3) + ((lane >> 4) & 1) * 2 + ((q >> 1) & 1)) ^ exchange(row);
      const char* at = lds + row * (R * 2) + (part << 4) + (q & 1) * 8;
      union {
        s4 half[2];
        Fragment<T> whole;
      } u;
      u.half[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds4)at);
      u.half[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds4)(at + 4 * R * 2));
      return u.whole;
    } else {
      const int row = 8 * t + 4 * h;                                     // (the same exchange for four rows)
      const char* at = lds + row * (R * 4) + ((((r0 + l) >> 2) ^ exchange(row)) << 4) + (l & 3) * 4;
      Fragment<T> v;
#pragma unroll
      for (int j = 0; j < 4; ++j) v[j] = *reinterpret_cast<const float*>(at + j * R * 4);
      return v;
    }
  }
};

constexpr int kTable = 1024;               // places whose rows are looked up at a time (dW)

// Rows of x behind an expert's places, kTable places at a time (dW): -1 where there is none.
struct Table {
  int32_t* rows;             // LDS, kTable of them
  uint32_t* there;           // LDS, a bit each
  const int32_t* source;     // of the expert's first place
  Divisor div;
  int64_t limit;
  // places k0 (a multiple of the table's size) .. of the expert's `depth`
  template <int THREADS>
  __device__ __forceinline__ void fill(int64_t k0, int64_t depth) const {
    __syncthreads();
    for (int i = threadIdx.x; i < kTable; i += THREADS) {
      const int pair = k0 + i < depth ? source[k0 + i] : -1;
      const int row = quotient(max(pair, 0), div);
      const bool in = pair >= 0 && row < limit;
      rows[i] = in ? row : -1;
      const unsigned long long bits = __ballot(in);
      if ((i & 31) == 0) there[i >> 5] = uint32_t(bits >> (i & 32));
    }
    __syncthreads();
  }
  // bits of the places k0 (a multiple of 32) ..
  __device__ __forceinline__ uint32_t bits(int64_t k0) const { return there[(int(k0) & (kTable - 1)) >> 5]; }
};

// 16 bytes per lane from `from` to LDS at `to` (the same for the wavefront) + 16 * lane.  Not waited for, and unknown to the
// compiler's own waits: wait_stage() counts these loads.  (The hardware takes `to` from m0; one instruction has to lie between.)
__device__ __forceinline__ void load_to_lds(const char* from, uint32_t to) {
  asm volatile("s_nop 0\n\tglobal_load_lds_dwordx4 %0, off" ::"v"(from), "{m0}"(to) : "memory");
}
// all loads to LDS but the last LEFT of this wavefront have arrived, all its accesses of LDS are done, and so for every
// wavefront
template <int LEFT>
__device__ __forceinline__ void wait_stage() {
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(LEFT) : "memory");
}
__device__ __forceinline__ uint32_t lds_address(const char* p) {
  return uint32_t(uintptr_t((const __attribute__((address_space(3))) char*)p));
}

// Which row of an operand (not KC) belongs to a k: the k-th; the one that `table` lists; the k-th, but zeros where the table lists
// none (dW: a place without a row of x adds nothing, whatever its cotangent holds; 0 * infinity would be NaN).
enum Order { kInOrder, kListed, kInOrderWhereListed };

// An operand whose rows are made of whole, aligned parts, loaded to LDS without passing through registers.  k counts from the
// sum's first.
template <class IMAGE, Order ORDER>
struct Direct {
  using T = typename IMAGE::Type;
  static constexpr bool KC = IMAGE::kKC;
  const char* p[IMAGE::kParts];    // the part at k = 0 (kListed: its column of row 0)
  int64_t stride;                  // bytes between rows (not KC)
  const int32_t* table;

  // Rows [first, end) of an operand contiguous in k, found through source where there is one.  Rows behind the last, and rows
  // whose place has none, are read from another row; their outputs are not stored, or stored as zeros.
  __device__ __forceinline__ void init_rows(const void* base, int64_t row_stride, const int32_t* source, const Divisor& d,
                                            int64_t limit, int64_t first, int64_t end) {
#pragma unroll
    for (int i = 0; i < IMAGE::kParts; ++i) {
      int64_t row = min(first + IMAGE::row_of(i), end - 1);
      if (source != nullptr) row = min(int64_t(quotient(max(source[row], 0), d)), limit - 1);
      p[i] = static_cast<const char*>(base) + row * row_stride * int64_t(sizeof(T)) + IMAGE::part_of(i) * 16;
    }
  }
  // Columns [first, end) of an operand with one row per k, from row k_begin on; columns behind the last as above.
  __device__ __forceinline__ void init_columns(const void* base, int64_t row_stride, const int32_t* rows, int64_t first,
                                               int64_t end, int64_t k_begin) {
    stride = row_stride * int64_t(sizeof(T));
    table = rows;
#pragma unroll
    for (int i = 0; i < IMAGE::kParts; ++i) {
      const int64_t at = min(first + IMAGE::part_of(i) * IMAGE::N, end - IMAGE::N);
      p[i] = static_cast<const char*>(base) + at * int64_t(sizeof(T));
      if (ORDER != kListed) p[i] += (k_begin + IMAGE::row_of(i)) * stride;
    }
  }

  // part i of the step k0 .. to LDS at `to` (of the step's image), zeros from `depth` on; without branches.  `there`: the table's
  // bits of the step, read once (both gradients of 8192 tokens x 2, 32 experts, 2048 -> 4096: 745 us, 748 with a look into the
  // table for every part, 739 without either; with code of its own for steps that have such a place the sums left the registers)
  __device__ __forceinline__ void issue_part(int i, int64_t k0, int64_t depth, uint32_t to, uint32_t there = 0) const {
    const int wave = __builtin_amdgcn_readfirstlane(int(threadIdx.x) / kWave);
    const char* zeros = reinterpret_cast<const char*>(&zero_part);
    const char* from;
    if constexpr (ORDER == kListed) {
      const int row = table[(int(k0) + IMAGE::row_of(i)) & (kTable - 1)];
      // (the row is selected before the product: a product in one of two ways would be a branch)
      from = (row >= 0 ? p[i] : zeros) + uint64_t(uint32_t(max(row, 0))) * uint32_t(stride);
    } else if constexpr (ORDER == kInOrderWhereListed) {
      static_assert(IMAGE::kStepK == 32, "a word per step");
      from = (there >> IMAGE::row_of(i) & 1u) != 0 ? p[i] + k0 * stride : zeros;
    } else {
      from = p[i] + k0 * (KC ? int64_t(sizeof(T)) : stride);
      const int left = int(min(depth - k0, int64_t(IMAGE::kStepK)));
      from = (KC ? IMAGE::part_of(i) * IMAGE::N : IMAGE::row_of(i)) < left ? from : zeros;
    }
    load_to_lds(from, to + (i * IMAGE::kThreads + wave * kWave) * 16);
  }
};

// An operand of any alignment and width, loaded to one of two sets of registers and written to LDS two steps later.  Every load
// is one of 16 bytes, and every step has as many, so that the waits count exactly: a part that crosses the end of its row is
// read from N elements before the end and shifted into place when it is written.  TINY: rows shorter than that, element by
// element.
template <class IMAGE, Order ORDER, bool TINY>
struct Staged {
  using T = typename IMAGE::Type;
  static constexpr bool KC = IMAGE::kKC;
  static constexpr int N = IMAGE::N;
  const T* p[IMAGE::kParts];       // as in Direct; null (KC): a row of zeros
  int64_t stride;                  // elements
  const int32_t* table;
  int64_t edge;                    // not KC: columns from the tile's first to the operand's end
  Fragment<T> v[2][IMAGE::kParts];

  __device__ __forceinline__ void init_rows(const void* base, int64_t row_stride, const int32_t* source, const Divisor& d,
                                            int64_t limit, int64_t first, int64_t end) {
#pragma unroll
    for (int i = 0; i < IMAGE::kParts; ++i) {
      int64_t row = min(first + IMAGE::row_of(i), end - 1);
      bool there = true;
      if (source != nullptr) {
        const int pair = source[row];
        row = quotient(max(pair, 0), d);
        there = pair >= 0 && row < limit;
      }
      p[i] = there ? static_cast<const T*>(base) + row * row_stride + IMAGE::part_of(i) * N : nullptr;
    }
  }
  __device__ __forceinline__ void init_columns(const void* base, int64_t row_stride, const int32_t* rows, int64_t first,
                                               int64_t end, int64_t k_begin) {
    stride = row_stride;
    table = rows;
    edge = end - first;
#pragma unroll
    for (int i = 0; i < IMAGE::kParts; ++i) {
      // (columns behind the end are not stored)
      p[i] = static_cast<const T*>(base) + first + (TINY ? IMAGE::part_of(i) * N : min(int64_t(IMAGE::part_of(i) * N), edge - N));
      if (ORDER != kListed) p[i] += (k_begin + IMAGE::row_of(i)) * stride;
    }
  }

  // how far part i, read in step k0, lies before its place
  __device__ __forceinline__ int behind(int i, int64_t k0, int64_t depth) const {
    const int64_t over = (KC ? k0 : int64_t(0)) + IMAGE::part_of(i) * N + N - (KC ? depth : edge);
    return int(min(max(over, int64_t(0)), int64_t(N)));
  }
  // elements d .. of q, zeros behind them
  static __device__ __forceinline__ Fragment<T> shifted(const Fragment<T>& q, int d) {
    typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
    u32x4 w = __builtin_bit_cast(u32x4, q);
    const int bytes = d * int(sizeof(T));
    if (bytes & 8) w = u32x4{w[2], w[3], 0u, 0u};
    if (bytes & 4) w = u32x4{w[1], w[2], w[3], 0u};
    if (bytes & 2) w = u32x4{w[0] >> 16 | w[1] << 16, w[1] >> 16 | w[2] << 16, w[2] >> 16 | w[3] << 16, w[3] >> 16};
    return __builtin_bit_cast(Fragment<T>, w);
  }
  static __device__ __forceinline__ Fragment<T> whole(const T* from) {
    const Packed<T, N> q = load_packed<T, N>(from);
    return __builtin_bit_cast(Fragment<T>, q);
  }

  // the step k0 .. to the registers `set`, zeros from `depth` on
  __device__ __forceinline__ void load(int set, int64_t k0, int64_t depth) {
    const T* zeros = reinterpret_cast<const T*>(&zero_part);
#pragma unroll
    for (int i = 0; i < IMAGE::kParts; ++i) {
      const T* from;
      bool there;
      if constexpr (KC) {
        there = p[i] != nullptr;
        from = p[i] + k0;
      } else if constexpr (ORDER == kListed) {
        const int row = table[(int(k0) + IMAGE::row_of(i)) & (kTable - 1)];
        there = row >= 0;
        from = p[i] + row * stride;
      } else {
        if constexpr (ORDER == kInOrderWhereListed) there = table[(int(k0) + IMAGE::row_of(i)) & (kTable - 1)] >= 0;
        else there = k0 + IMAGE::row_of(i) < depth;
        from = p[i] + k0 * stride;
      }
      if constexpr (TINY) {
        const int64_t count = KC ? depth - (k0 + IMAGE::part_of(i) * N) : edge - IMAGE::part_of(i) * N;
#pragma unroll
        for (int j = 0; j < N; ++j) v[set][i][j] = there && j < count ? from[j] : T(0.0f);
      } else {
        if constexpr (KC) {
          const int d = behind(i, k0, depth);
          there = there && d < N;
          from -= d;
        }
        v[set][i] = whole(there ? from : zeros);
      }
    }
  }
  __device__ __forceinline__ void store(int set, char* to, int64_t k0, int64_t depth) const {
    const bool cross = !TINY && (KC ? k0 + IMAGE::kStepK > depth : edge < IMAGE::kAlong * N);
#pragma unroll
    for (int i = 0; i < IMAGE::kParts; ++i) {
      Fragment<T> q = v[set][i];
      if (cross) q = shifted(q, behind(i, k0, depth));
      *reinterpret_cast<Fragment<T>*>(to + (i * IMAGE::kThreads + int(threadIdx.x)) * 16) = q;
    }
  }
};

// N neighbouring columns from n on, those below n_end
template <class T, int N>
__device__ __forceinline__ void store_columns(T* row, int64_t n, int64_t n_end, const Packed<T, N>& v) {
  if (n + N <= n_end) {
    store_packed<T, N>(row + n, v);
  } else {
#pragma unroll
    for (int r = 0; r < N; ++r)
      if (n + r < n_end) row[n + r] = v.v[r];
  }
}

// Sums of a wavefront to C: MI x NJ blocks of 32 x 32 from (m0, n0) on, below (m_end, n_end); n runs along the rows of the
// instruction's output, so that a lane has four neighbouring columns at a time.  Of two such fours of 16-bit types, 8 columns
// apart, lane l takes the first with that of lane l + 32 behind it, lane l + 32 the second: 16 bytes each.  Rows whose place has
// no source are zeros.
template <class T, int MI, int NJ>
__device__ __forceinline__ void store_tile(const f32x16 (&acc)[MI][NJ], int64_t m0, int64_t m_end, int64_t n0, int64_t n_end,
                                           const int32_t* source, const Divisor& div, int64_t limit, T* c, int64_t c_stride) {
  const int lane = int(threadIdx.x) & (kWave - 1);
#pragma unroll
  for (int i = 0; i < MI; ++i) {
    const int64_t m = m0 + 32 * i + (lane & 31);
    bool there = m < m_end;
    if (there && source != nullptr) there = source[m] >= 0 && quotient(source[m], div) < limit;
    T* row = c + m * c_stride;
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
      Packed<T, 4> four[4];
#pragma unroll
      for (int q = 0; q < 4; ++q)
#pragma unroll
        for (int r = 0; r < 4; ++r) four[q].v[r] = from_f32<T>(there ? acc[i][j][4 * q + r] : 0.0f);
      const int64_t n = n0 + 32 * j;
      if constexpr (sizeof(T) == 2) {
        typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
#pragma unroll
        for (int q = 0; q < 4; q += 2) {
          const u32x2 a = __builtin_bit_cast(u32x2, four[q]), b = __builtin_bit_cast(u32x2, four[q + 1]);
          const auto x = __builtin_amdgcn_permlane32_swap(a[0], b[0], false, false);
          const auto y = __builtin_amdgcn_permlane32_swap(a[1], b[1], false, false);
          typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
          const u32x4 w = {x[0], y[0], x[1], y[1]};
          if (m < m_end) store_columns<T, 8>(row, n + 8 * (q + (lane >> 5)), n_end, __builtin_bit_cast(Packed<T, 8>, w));
        }
      } else {
#pragma unroll
        for (int q = 0; q < 4; ++q)
          if (m < m_end) store_columns<T, 4>(row, n + 8 * q + 4 * (lane >> 5), n_end, four[q]);
      }
    }
  }
}

// Zeros to share `part` of `parts` of the `count` elements at c, by a workgroup of THREADS.
template <int THREADS, class T>
__device__ __forceinline__ void store_zeros(T* c, int64_t count, int64_t part, int64_t parts) {
  constexpr int N = 16 / int(sizeof(T));
  const int64_t whole = count / N, end = whole * (part + 1) / parts;
  for (int64_t i = whole * part / parts + threadIdx.x; i < end; i += THREADS) store_packed<T, N>(c + i * N, Packed<T, N>{});
  if (part == 0 && threadIdx.x < count - whole * N) c[whole * N + threadIdx.x] = T(0.0f);
}

template <int MI, int NJ>
__device__ __forceinline__ void clear(f32x16 (&acc)[MI][NJ]) {
#pragma unroll
  for (int i = 0; i < MI; ++i)
#pragma unroll
    for (int j = 0; j < NJ; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.0f;
}

}  // namespace topk
