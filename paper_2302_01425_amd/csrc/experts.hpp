// Host-side launchers and shared device helpers of the operators behind a router: choosing experts (route.hip), places of
// the chosen pairs in expert order (expert_map.hip), the experts' products (expert_product.hip) and the weighted sum back
// per token (combine.hip).  Values come in float32, bfloat16 or float16; sums and statistics are float32 or wider.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace topk {

enum TypeCode : int { kF32 = 0, kBF16 = 1, kF16 = 2 };
enum ScoreCode : int { kSoftmax = 0, kSigmoid = 1 };

using bf16 = __bf16;
using f16 = _Float16;

constexpr int kExpertsMax = 1024;      // experts of a router: a row of scores fits one wavefront
constexpr int kChoicesMax = 64;        // choices per token

// A launch has fewer than 2^32 threads.
inline bool launchable(int64_t blocks, int threads) { return blocks < (int64_t(1) << 32) / threads; }

struct RouteArgs {
  const void* logits;
  int64_t stride;            // elements between rows
  const float* bias;         // [n] or null
  int64_t rows;
  int n, k, groups, keep, top;
  int score, renorm;
  float scale;
  int32_t* idx;
  float* val;
};
int launch_route_fwd(int type, const RouteArgs& a, hipStream_t stream);

struct RouteVjpArgs {
  const void* logits;
  int64_t stride;
  const int32_t* idx;
  const float* cotangent;
  int64_t rows;
  int n, k, score, renorm;
  float scale;
  void* grad;                // [rows][n]
};
int launch_route_vjp(int type, const RouteVjpArgs& a, hipStream_t stream);

struct MapArgs {
  const int32_t* idx;
  int64_t pairs;
  int n;
  int64_t capacity;          // pairs kept per expert
  int32_t *slot, *source, *offset, *load;
  int32_t* scratch;
};
int64_t map_chunks(int64_t pairs, int n);
inline int map_width(int n) { return (n + 3) / 4 * 4; }      // counts of a chunk in the scratch (16-byte rows)
int launch_expert_map(const MapArgs& a, hipStream_t stream);

// One product over the ragged groups.  Operand strides are in elements; w(e, o, i) = w[e * w_expert + o * w_out + i * w_in].
struct ProductArgs {
  const void* x;             // [m][h], or [slots][h] without source
  int64_t x_stride;
  int64_t m;                 // rows of x
  const void* w;
  int64_t w_expert, w_out, w_in;
  const int32_t* offset;     // [n + 1]
  const int32_t* source;     // [slots] or null
  int64_t k;                 // row of x behind place s: source[s] / k
  int64_t slots;
  int n;
  int64_t h, ho;
  const void* t;             // cotangent [slots][ho]
  int64_t t_stride;
  void *out, *dx, *dw;       // [slots][ho], [slots][h], layout of w
};
int launch_product_fwd(int type, const ProductArgs& a, hipStream_t stream);
int launch_product_dx(int type, const ProductArgs& a, hipStream_t stream);
// (with dw_up: also that of a second cotangent, `apart` bytes behind the first, in the same launch)
int launch_product_dw(int type, const ProductArgs& a, hipStream_t stream, int64_t apart = 0, void* dw_up = nullptr);

struct CombineArgs {
  const void* y;             // [slots][h]
  int64_t y_stride;
  const int32_t* slot;       // [rows][k]
  const float* val;          // [rows][k] or null (ones)
  const void* t;             // cotangent [rows][h]
  int64_t t_stride;
  int64_t rows, k, slots, h;
  int64_t slice, slices;     // forward: parts of a row, of a workgroup each, that a launch takes
  void* out;                 // [rows][h]
  void* dy;                  // [slots][h]
  float* dval;               // [rows][k]
};
int64_t combine_slices(int type, int64_t h);      // of a row
int launch_combine_fwd(int type, const CombineArgs& a, hipStream_t stream);
int launch_combine_vjp(int type, const CombineArgs& a, hipStream_t stream);

// ---- device helpers ---------------------------------------------------------------------------------------------------
template <class T>
__device__ __forceinline__ float to_f32(T v) {
  return float(v);
}
// rounding to nearest, ties to even, the one rounding of every output
template <class T>
__device__ __forceinline__ T from_f32(float v) {
  return T(v);
}

// N consecutive elements (a power of two, up to 16 bytes) at an address that is a multiple of their own size only, as one
// access: the hardware takes vector accesses at any byte address.  (As N elements the compiler splits them up again.)
template <int BYTES>
struct BitsOf;
template <>
struct BitsOf<4> {
  using type = uint32_t;
};
template <>
struct BitsOf<8> {
  typedef uint32_t type __attribute__((ext_vector_type(2)));
};
template <>
struct BitsOf<16> {
  typedef uint32_t type __attribute__((ext_vector_type(4)));
};
template <class T, int N>
struct Packed {
  T v[N];
};
template <class T, int N>
struct __attribute__((packed, aligned(sizeof(T) < 2 ? 1 : 2))) Loose {
  typename BitsOf<N * int(sizeof(T))>::type bits;
};
template <class T, int N>
__device__ __forceinline__ Packed<T, N> load_packed(const T* p) {
  // (global memory, which the compiler does not see through a choice of pointers)
  typedef const __attribute__((address_space(1))) Loose<T, N>* Global;
  return __builtin_bit_cast(Packed<T, N>, ((Global)(uintptr_t)p)->bits);
}
template <class T, int N>
__device__ __forceinline__ void store_packed(T* p, const Packed<T, N>& v) {
  reinterpret_cast<Loose<T, N>*>(p)->bits = __builtin_bit_cast(typename BitsOf<N * int(sizeof(T))>::type, v);
}

}  // namespace topk
