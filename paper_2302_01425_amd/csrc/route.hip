// Routing to experts.  Per row of logits l over n experts:
//   s = softmax(l) or 1 / (1 + exp(-l)),  c = s + bias (order of l itself where there is no bias),
//   the `keep` best of `groups` equal groups stay (score of a group: the sum of its `top` largest c),
//   idx = the k largest c in descending order, equal ones by ascending index, val = scale s[idx] (/ sum of the chosen s).
// A logit of -inf or NaN, or a bias of -inf or NaN, takes its expert out; where fewer than k are left, idx = -1, val = 0.
// Scores that are compared are float64: the choice jumps where two scores cross, and two float32 scores of 16384 x 256
// cross within their rounding a few times per call.  Logits are compared as they are.
#include <cmath>

#include "experts.hpp"
#include "wave.hpp"

namespace topk {
namespace {

constexpr int kThreads = 256;
constexpr float kNone = -INFINITY;

template <int GL, int LM = GL / 2>
__device__ __forceinline__ float group_max(float v) {
  if constexpr (LM == 0) return v;
  else return group_max<GL, LM / 2>(fmaxf(v, __uint_as_float(lane_xor<LM>(__float_as_uint(v)))));
}
template <int GL, int LM = GL / 2>
__device__ __forceinline__ double group_max(double v) {
  if constexpr (LM == 0) return v;
  else return group_max<GL, LM / 2>(fmax(v, lane_xor_f64<LM>(v)));
}
template <int GL, int LM = GL / 2>
__device__ __forceinline__ float group_sum_f32(float v) {
  if constexpr (LM == 0) return v;
  else return group_sum_f32<GL, LM / 2>(v + __uint_as_float(lane_xor<LM>(__float_as_uint(v))));
}

// exp(l - m) with m the largest l, infinite or not
__device__ __forceinline__ float exp_below(float l, float m) { return l == m ? 1.0f : expf(l - m); }
__device__ __forceinline__ double exp_below(double l, double m) { return l == m ? 1.0 : exp(l - m); }

// sigmoid(l) exp(-m) for m >= min(l, 0): with m the largest such of the chosen, sums of scores that are all tiny keep
// their relative accuracy
__device__ __forceinline__ float sigmoid_over(float l, float m) {
  return expf(fminf(l, 0.0f) - m) / (1.0f + expf(-fabsf(l)));
}

// GL lanes per row, E elements per lane.  Lanes are dealt to the groups first (`lanes` consecutive ones each, a power of
// two), so that a group's scores are reduced by a butterfly over its own lanes; a lane holds consecutive elements, so that
// the lowest lane and the lowest register hold the lowest index.
template <class T, int GL, int E, class KEY>
__global__ __launch_bounds__(kThreads) void route_fwd_kernel(RouteArgs a, int lanes) {
  const int64_t row = (int64_t(blockIdx.x) * kThreads + threadIdx.x) / GL;
  if (row >= a.rows) return;                                       // (whole row groups)
  const int lr = int(threadIdx.x) & (GL - 1);
  const int size = a.n / a.groups, g = lr / lanes, in = (lr & (lanes - 1)) * E;
  const int count = g < a.groups ? min(max(size - in, 0), E) : 0;  // elements of this lane
  const int base = g * size + in;
  const T* lp = static_cast<const T*>(a.logits) + row * a.stride + base;
  float l[E];
#pragma unroll
  for (int e = 0; e < E; ++e) {
    l[e] = e < count ? to_f32(lp[e]) : kNone;
    if (isnan(l[e])) l[e] = kNone;
  }
  float top = l[0];
#pragma unroll
  for (int e = 1; e < E; ++e) top = fmaxf(top, l[e]);
  top = group_max<GL>(top);

  // what is compared
  KEY key[E];
  if constexpr (sizeof(KEY) == 8) {
    double total = 1.0;
    if (a.score == kSoftmax) {
      double z = 0.0;
#pragma unroll
      for (int e = 0; e < E; ++e) {
        key[e] = l[e] == kNone ? 0.0 : exp_below(double(l[e]), double(top));
        z += key[e];
      }
      total = group_sum_f64<GL>(z);
    } else {
#pragma unroll
      for (int e = 0; e < E; ++e) key[e] = 1.0 / (1.0 + exp(-double(l[e])));
    }
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const float b = a.bias != nullptr && e < count ? a.bias[base + e] : 0.0f;
      const bool out = l[e] == kNone || !(b > kNone);
      key[e] = out ? -INFINITY : key[e] / total + double(b);
    }
  } else {
#pragma unroll
    for (int e = 0; e < E; ++e) key[e] = l[e];
  }

  if (a.groups > 1) {
    KEY first = -INFINITY, second = -INFINITY;
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const KEY v = key[e];
      second = fmax(second, fmin(first, v));
      first = fmax(first, v);
    }
    for (int off = 1; off < lanes; off <<= 1) {
      const KEY f = __shfl_xor(first, off, GL), s = __shfl_xor(second, off, GL);
      second = fmax(fmax(second, s), fmin(first, f));
      first = fmax(first, f);
    }
    const KEY score = a.top == 2 && second > KEY(-INFINITY) ? first + second : first;
    int rank = 0;
    for (int o = 0; o < a.groups; ++o) {
      const KEY other = __shfl(score, o * lanes, GL);
      rank += other > score || (other == score && o < g);
    }
    if (rank >= a.keep) {
#pragma unroll
      for (int e = 0; e < E; ++e) key[e] = -INFINITY;
    }
    if constexpr (sizeof(KEY) == 8) {
      if (a.bias == nullptr) {           // sums of scores chose the groups, the logits choose in them
#pragma unroll
        for (int e = 0; e < E; ++e)
          if (key[e] > -INFINITY) key[e] = double(l[e]);
      }
    }
  }

  // k times the largest of the row that is left
  int place[E];
#pragma unroll
  for (int e = 0; e < E; ++e) place[e] = -1;
  int found = 0;
  const int lane0 = int(threadIdx.x) & (kWave - 1) & ~(GL - 1);
  for (int j = 0; j < a.k; ++j) {
    KEY best = key[0];
    int at = 0;
#pragma unroll
    for (int e = 1; e < E; ++e)
      if (key[e] > best) {
        best = key[e];
        at = e;
      }
    const KEY m = group_max<GL>(best);
    if (!(m > KEY(-INFINITY))) continue;
    found = j + 1;
    const unsigned long long who = __ballot(best == m) >> lane0;
    if (lr == __ffsll(GL < 64 ? who & ((1ull << (GL & 63)) - 1ull) : who) - 1) {
#pragma unroll
      for (int e = 0; e < E; ++e)
        if (e == at) {
          place[e] = j;
          key[e] = -INFINITY;
        }
    }
  }

  // their weights
  float u[E], sum = 0.0f, factor;
  if (a.renorm) {
    float m = kNone;
#pragma unroll
    for (int e = 0; e < E; ++e)
      if (place[e] >= 0) m = fmaxf(m, a.score == kSoftmax ? l[e] : fminf(l[e], 0.0f));
    m = group_max<GL>(m);
#pragma unroll
    for (int e = 0; e < E; ++e) {
      u[e] = place[e] < 0 ? 0.0f : a.score == kSoftmax ? exp_below(l[e], m) : sigmoid_over(l[e], m);
      sum += u[e];
    }
    factor = a.scale / group_sum_f32<GL>(sum);
  } else if (a.score == kSoftmax) {
#pragma unroll
    for (int e = 0; e < E; ++e) {
      u[e] = l[e] == kNone ? 0.0f : exp_below(l[e], top);
      sum += u[e];
    }
    factor = a.scale / group_sum_f32<GL>(sum);
  } else {
#pragma unroll
    for (int e = 0; e < E; ++e) u[e] = sigmoid_over(l[e], 0.0f);
    factor = a.scale;
  }
#pragma unroll
  for (int e = 0; e < E; ++e)
    if (place[e] >= 0) {
      a.idx[row * a.k + place[e]] = base + e;
      a.val[row * a.k + place[e]] = u[e] * factor;
    }
  for (int j = found + lr; j < a.k; j += GL) {
    a.idx[row * a.k + j] = -1;
    a.val[row * a.k + j] = 0.0f;
  }
}

// Gradient in the logits of <val, cotangent>, val as above for the given idx (which carry no gradient).  With w the weights
// without `scale`, mean = sum_j w_j t_j:
//   softmax, renormalised   dl[idx_j] += scale w_j (t_j - mean)
//   softmax                 dl[idx_j] += scale w_j t_j,  dl -= scale s mean
//   sigmoid, renormalised   dl[idx_j] += scale w_j (1 - s_j) (t_j - mean)
//   sigmoid                 dl[idx_j] += scale s_j (1 - s_j) t_j
template <class T, int GL, int E>
__global__ __launch_bounds__(kThreads) void route_vjp_kernel(RouteVjpArgs a) {
  const int64_t row = (int64_t(blockIdx.x) * kThreads + threadIdx.x) / GL;
  if (row >= a.rows) return;
  const int lr = int(threadIdx.x) & (GL - 1);
  const int base = lr * E, count = min(max(a.n - base, 0), E);
  const T* lp = static_cast<const T*>(a.logits) + row * a.stride;
  const int32_t* ip = a.idx + row * a.k;
  const float* tp = a.cotangent + row * a.k;
  const bool whole = a.score == kSoftmax && !a.renorm;
  float s[E];
  float m = kNone, sum = 0.0f;
  if (whole) {
#pragma unroll
    for (int e = 0; e < E; ++e) {
      s[e] = e < count ? to_f32(lp[base + e]) : kNone;
      if (isnan(s[e])) s[e] = kNone;
      m = fmaxf(m, s[e]);
    }
    m = group_max<GL>(m);
#pragma unroll
    for (int e = 0; e < E; ++e) {
      s[e] = s[e] == kNone ? 0.0f : exp_below(s[e], m);
      sum += s[e];
    }
    sum = group_sum_f32<GL>(sum);
  } else {
#pragma unroll
    for (int e = 0; e < E; ++e) s[e] = 0.0f;
    if (a.renorm) {
      for (int j = 0; j < a.k; ++j) {
        const int i = ip[j];
        if (i < 0 || i >= a.n) continue;
        const float l = to_f32(lp[i]);
        if (!isnan(l)) m = fmaxf(m, a.score == kSoftmax ? l : fminf(l, 0.0f));
      }
    } else {
      m = 0.0f;
    }
  }
  // unnormalised weight of choice j (0: an empty place, or an expert that is out)
  const auto weight = [&](float l) -> float {
    if (!(l > kNone)) return 0.0f;
    return a.score == kSoftmax ? exp_below(l, m) : sigmoid_over(l, m);
  };
  float mean = 0.0f;
  if (whole || a.renorm) {
    float chosen = 0.0f;
    for (int j = 0; j < a.k; ++j) {
      const int i = ip[j];
      if (i < 0 || i >= a.n) continue;
      const float w = weight(to_f32(lp[i]));
      chosen += w;
      if (w > 0.0f) mean += w * tp[j];
    }
    if (!whole) sum = chosen;
  } else {
    sum = 1.0f;
  }
  const float inv = sum > 0.0f ? 1.0f / sum : 0.0f;
  mean *= inv;
  float d[E];
#pragma unroll
  for (int e = 0; e < E; ++e) d[e] = whole ? -s[e] * inv * mean : 0.0f;
  for (int j = 0; j < a.k; ++j) {
    const int i = ip[j];
    if (i < 0 || i >= a.n) continue;
    const float l = to_f32(lp[i]);
    const float w = weight(l) * inv;
    if (!(w > 0.0f)) continue;
    float v = w * (a.renorm ? tp[j] - mean : tp[j]);
    if (a.score == kSigmoid) v *= sigmoid_over(-l, 0.0f);
#pragma unroll
    for (int e = 0; e < E; ++e)
      if (base + e == i) d[e] += v;
  }
  T* gp = static_cast<T*>(a.grad) + row * a.n + base;
#pragma unroll
  for (int e = 0; e < E; ++e)
    if (e < count) gp[e] = from_f32<T>(a.scale * d[e]);
}

template <class T, int GL, int E>
void fwd(const RouteArgs& a, int lanes, bool f64, hipStream_t stream) {
  const dim3 grid(unsigned((a.rows * GL + kThreads - 1) / kThreads));
  if (f64) hipLaunchKernelGGL((route_fwd_kernel<T, GL, E, double>), grid, dim3(kThreads), 0, stream, a, lanes);
  else hipLaunchKernelGGL((route_fwd_kernel<T, GL, E, float>), grid, dim3(kThreads), 0, stream, a, lanes);
}

template <class T>
int fwd_type(const RouteArgs& a, hipStream_t stream) {
  // scores, not logits, are compared where a bias is added or scores of a group are
  const bool f64 = a.bias != nullptr || (a.groups > 1 && a.top == 2);
  int padded = 1;                        // groups, up to a power of two
  while (padded < a.groups) padded *= 2;
  const int size = a.n / a.groups;
  // the fewest lanes whose registers hold a row: the k rounds cost a reduction over the lanes each
  const auto fits = [&](int gl, int e) { return padded <= gl && size <= gl / padded * e; };
  if (fits(8, 4)) fwd<T, 8, 4>(a, 8 / padded, f64, stream);
  else if (fits(8, 8)) fwd<T, 8, 8>(a, 8 / padded, f64, stream);
  else if (fits(16, 8)) fwd<T, 16, 8>(a, 16 / padded, f64, stream);
  else if (fits(32, 8)) fwd<T, 32, 8>(a, 32 / padded, f64, stream);
  else if (fits(64, 8)) fwd<T, 64, 8>(a, 64 / padded, f64, stream);
  else if (fits(64, 16)) fwd<T, 64, 16>(a, 64 / padded, f64, stream);
  else if (fits(64, 32)) fwd<T, 64, 32>(a, 64 / padded, f64, stream);
  else return -1;
  return 0;
}

template <class T, int GL, int E>
void vjp(const RouteVjpArgs& a, hipStream_t stream) {
  const dim3 grid(unsigned((a.rows * GL + kThreads - 1) / kThreads));
  hipLaunchKernelGGL((route_vjp_kernel<T, GL, E>), grid, dim3(kThreads), 0, stream, a);
}

template <class T>
int vjp_type(const RouteVjpArgs& a, hipStream_t stream) {
  if (a.n <= 32) vjp<T, 8, 4>(a, stream);
  else if (a.n <= 64) vjp<T, 8, 8>(a, stream);
  else if (a.n <= 128) vjp<T, 16, 8>(a, stream);
  else if (a.n <= 256) vjp<T, 32, 8>(a, stream);
  else if (a.n <= 512) vjp<T, 64, 8>(a, stream);
  else if (a.n <= 1024) vjp<T, 64, 16>(a, stream);
  else return -1;
  return 0;
}

}  // namespace

int launch_route_fwd(int type, const RouteArgs& a, hipStream_t stream) {
  if (type == kF32) return fwd_type<float>(a, stream);
  if (type == kBF16) return fwd_type<bf16>(a, stream);
  if (type == kF16) return fwd_type<f16>(a, stream);
  return -1;
}

int launch_route_vjp(int type, const RouteVjpArgs& a, hipStream_t stream) {
  if (type == kF32) return vjp_type<float>(a, stream);
  if (type == kBF16) return vjp_type<bf16>(a, stream);
  if (type == kF16) return vjp_type<f16>(a, stream);
  return -1;
}

}  // namespace topk
