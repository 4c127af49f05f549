// Routing to experts.  Per row of logits l over n experts:
//   s = softmax(l) or 1 / (1 + exp(-l)),  c = s + bias (order of l itself where there is no bias),
//   the `keep` best of `groups` equal groups stay (score of a group: the sum of its `top` largest c),
//   idx = the k largest c in descending order, equal ones by ascending index, val = scale s[idx] (/ sum of the chosen s).
// A logit of -inf or NaN, or a bias of -inf or NaN, takes its expert out; where fewer than k are left, idx = -1, val = 0.
// Scores are compared as float64 would: the choice jumps where two scores cross, and two float32 scores of 16384 x 256
// cross within their rounding a few times per call.  Logits are compared as they are.
//
// A row lies in the registers of 8 to 64 lanes and is read once; k rounds take the largest each.  Bound by the launch below some
// 1000 rows (5 us a call), by instructions above: a round of 32 lanes x 8 elements is 87 of them.  16384 x 64 float32, softmax, k = 2:
// 4.4 us, 1.0 TB/s; 8192 x 256 bfloat16, sigmoid, bias, 8 groups, k = 8: 12.5 and 13.5 us a call (two draws of the inputs), 0.38 and
// 0.35 TB/s (16 lanes x 16 elements: 12 to 17 us, and 2 us more for few rows).
#include <cmath>

#include "experts.hpp"
#include "wave.hpp"

namespace topk {
namespace {

constexpr int kThreads = 256;
constexpr float kNone = -INFINITY;

__device__ __forceinline__ float max_of(float a, float b) { return __builtin_amdgcn_fmed3f(a, b, INFINITY); }   // (no NaN)
__device__ __forceinline__ double max_of(double a, double b) { return max_f64(a, b); }
template <int GL, int LM = GL / 2>
__device__ __forceinline__ float group_max(float v) {
  if constexpr (LM == 0) return v;
  else return group_max<GL, LM / 2>(max_of(v, __uint_as_float(lane_xor<LM>(__float_as_uint(v)))));
}
template <int GL, int LM = GL / 2>
__device__ __forceinline__ double group_max(double v) {
  if constexpr (LM == 0) return v;
  else return group_max<GL, LM / 2>(max_of(v, lane_xor_f64<LM>(v)));
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

// E consecutive elements as float, `fill` behind the first `count`
template <class T, int E>
__device__ __forceinline__ void load_row_part(const T* p, int count, float fill, float (&v)[E]) {
  if (count == E) {
    constexpr int N = E * sizeof(T) < 16 ? E : 16 / int(sizeof(T));
#pragma unroll
    for (int c = 0; c < E; c += N) {
      const Packed<T, N> q = load_packed<T, N>(p + c);
#pragma unroll
      for (int i = 0; i < N; ++i) v[c + i] = to_f32(q.v[i]);
    }
  } else {
#pragma unroll
    for (int e = 0; e < E; ++e) v[e] = e < count ? to_f32(p[e]) : fill;
  }
}
template <class T, int E>
__device__ __forceinline__ void store_row_part(T* p, int count, const float (&v)[E]) {
  if (count == E) {
    constexpr int N = E * sizeof(T) < 16 ? E : 16 / int(sizeof(T));
#pragma unroll
    for (int c = 0; c < E; c += N) {
      Packed<T, N> q;
#pragma unroll
      for (int i = 0; i < N; ++i) q.v[i] = from_f32<T>(v[c + i]);
      store_packed<T, N>(p + c, q);
    }
  } else {
#pragma unroll
    for (int e = 0; e < E; ++e)
      if (e < count) p[e] = from_f32<T>(v[e]);
  }
}

// What a lane knows of its row.  Lanes are dealt to the groups first (`lanes` consecutive ones each, a power of two), so that
// a group's scores are reduced by a butterfly over its own lanes; a lane holds consecutive elements, so that the lowest lane
// and the lowest register hold the lowest index.
template <int E>
struct Lane {
  float l[E];        // logits, -inf where there is none
  float b[E];        // bias
  float top;         // the row's largest logit
  int g, lanes, lr;
};

__device__ __forceinline__ float max3_of(float a, float b, float c) {
  float r;
  asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
  return r;
}
template <int E>
__device__ __forceinline__ float max_all(const float (&v)[E]) {
  float m = v[E - 1];                    // (E is even)
#pragma unroll
  for (int e = 0; e + 1 < E; e += 2) m = max3_of(m, v[e], v[e + 1]);
  return m;
}
template <int E>
__device__ __forceinline__ double max_all(const double (&v)[E]) {
  double m = v[0];
#pragma unroll
  for (int e = 1; e < E; ++e) m = max_of(m, v[e]);
  return m;
}

// A chosen element: score, bias, logit, index.
struct Record {
  float c, b, l;
  int i;
};
constexpr int kRecords = kChoicesMax + 2;

__device__ __forceinline__ double sigmoid_f64(float l) { return 1.0 / (1.0 + exp(-double(l))); }

// The first m records of a row in the order of their scores in float64, which take the place of c and b.  The records are few
// and nearly in order: one lane moves them.
template <int GL, int E>
__device__ __forceinline__ void settle(const RouteArgs& a, const Lane<E>& w, Record* line, int m) {
  double z = 0.0;
  if (a.score == kSoftmax) {
#pragma unroll
    for (int e = 0; e < E; ++e) z += w.l[e] == kNone ? 0.0 : exp_below(double(w.l[e]), double(w.top));
    z = 1.0 / group_sum_f64<GL>(z);
  }
  const auto score = [](const Record& r) {
    double d;
    __builtin_memcpy(&d, &r, sizeof(d));
    return d;
  };
  for (int j = w.lr; j < m; j += GL) {
    Record r = line[j];
    const double s = a.score == kSoftmax ? exp_below(double(r.l), double(w.top)) * z : sigmoid_f64(r.l);
    const double d = s + double(r.b);
    __builtin_memcpy(&r, &d, sizeof(d));
    line[j] = r;
  }
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  if (w.lr == 0) {
    for (int j = 1; j < m; ++j) {
      const Record r = line[j];
      const double d = score(r);
      int to = j;
      for (; to > 0; --to) {
        const Record q = line[to - 1];
        if (score(q) > d || (score(q) == d && q.i < r.i)) break;
        line[to] = q;
      }
      line[to] = r;
    }
  }
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
}

// The k largest and the two next to line[] (LDS, kRecords of the row), in order; returns how many of the k there are.  KEY
// float: `sure` says whether float64 would choose the same.  `base`: index of the lane's first element.
template <int GL, int E, class KEY>
__device__ __forceinline__ int choose(const RouteArgs& a, const Lane<E>& w, bool scored, int base, Record* line, bool* sure) {
  KEY key[E];
  float rel = 0.0f, err = 0.0f;          // a float32 score s is off by rel s + err at most
  if (scored) {
    if (a.score == kSoftmax) {
      KEY z = KEY(0);
#pragma unroll
      for (int e = 0; e < E; ++e) {
        key[e] = w.l[e] == kNone ? KEY(0) : exp_below(KEY(w.l[e]), KEY(w.top));
        z += key[e];
      }
      if constexpr (sizeof(KEY) == 8) z = group_sum_f64<GL>(z);
      else z = group_sum_f32<GL>(z);
      z = KEY(1) / z;
#pragma unroll
      for (int e = 0; e < E; ++e) key[e] *= z;
      // E + 6 roundings of the sum and ln n < 7 of its terms', 5 of exponential, quotient and product; and (top - l) s <= 1 / e
      // of the difference's
      rel = (E + 18) * 0x1p-24f;
      err = 0.5f * 0x1p-24f;
    } else {
#pragma unroll
      for (int e = 0; e < E; ++e) {
        if constexpr (sizeof(KEY) == 8) key[e] = sigmoid_f64(w.l[e]);
        else key[e] = 1.0f / (1.0f + expf(-w.l[e]));
      }
      // 2 of the exponential, 1 of the sum, 2 of the quotient
      rel = 5 * 0x1p-24f;
    }
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const bool out = w.l[e] == kNone || !(w.b[e] > kNone);
      key[e] = out ? KEY(-INFINITY) : key[e] + KEY(w.b[e]);
    }
  } else {
#pragma unroll
    for (int e = 0; e < E; ++e) key[e] = KEY(w.l[e]);
  }
  bool good = true;
  if (a.groups > 1) {
    KEY first = -INFINITY, second = -INFINITY;
#pragma unroll
    for (int e = 0; e < E; ++e) {
      second = max_of(second, fmin(first, key[e]));
      first = max_of(first, key[e]);
    }
    for (int off = 1; off < w.lanes; off <<= 1) {
      const KEY f = __shfl_xor(first, off, GL), s = __shfl_xor(second, off, GL);
      second = max_of(max_of(second, s), fmin(first, f));
      first = max_of(first, f);
    }
    const KEY score = a.top == 2 && second > KEY(-INFINITY) ? first + second : first;
    int rank = 0;
    for (int o = 0; o < a.groups; ++o) {
      const KEY other = __shfl(score, o * w.lanes, GL);
      rank += other > score || (other == score && o < w.g);
    }
    if (sizeof(KEY) == 4 && scored) {
      // A group's score is off by its scores' errors and by two roundings of each of the c it is the sum of, which may be far
      // larger than their sum (biases of both signs).  The groups are sure if no score that stays comes down to one that goes
      // when both move by that (twice the roundings leave room for those of this sum), and if float32 held all of them.
      const bool any = first > KEY(-INFINITY);
      const float size = any ? fabsf(float(first)) + (a.top == 2 && second > KEY(-INFINITY) ? fabsf(float(second)) : 0.0f) : 0.0f;
      const float off = 2.0f * (rel + err) + 0x1p-22f * (1.0f + size);
      const float in = rank < a.keep ? float(score) - off : INFINITY, out = rank < a.keep || w.g >= a.groups ? kNone : float(score) + off;
      const float low = -group_max<GL>(-in), high = group_max<GL>(out);
      good = (high == kNone || low > high) && size < 0x1p126f;
    }
    if (rank >= a.keep) {
#pragma unroll
      for (int e = 0; e < E; ++e) key[e] = -INFINITY;
    }
    if (scored && a.bias == nullptr) {     // sums of scores chose the groups, the logits choose in them
#pragma unroll
      for (int e = 0; e < E; ++e)
        if (key[e] > KEY(-INFINITY)) key[e] = KEY(w.l[e]);
    }
  }

  const bool check = sizeof(KEY) == 4 && scored && a.bias != nullptr;
  KEY score[E];
  int place[E];
#pragma unroll
  for (int e = 0; e < E; ++e) {
    score[e] = key[e];
    place[e] = -1;
  }
  int found = 0;
  const int lane0 = int(threadIdx.x) & (kWave - 1) & ~(GL - 1);
  const int rounds = check ? min(a.k + 2, a.n) : a.k;
  for (int j = 0; j < rounds; ++j) {
    const KEY best = max_all(key);
    const KEY m = group_max<GL>(best);
    const bool any = m > KEY(-INFINITY);
    const unsigned long long who = __ballot(best == m) >> lane0;
    bool mine = any && w.lr == __ffsll(GL < 64 ? who & ((1ull << (GL & 63)) - 1ull) : who) - 1;
    found += any;
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const bool hit = mine & (key[e] == m);
      place[e] = hit ? j : place[e];
      key[e] = hit ? KEY(-INFINITY) : key[e];
      mine = mine & !hit;
    }
  }
#pragma unroll
  for (int e = 0; e < E; ++e)
    if (place[e] >= 0) line[place[e]] = Record{float(score[e]), w.b[e], w.l[e], base + e};
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");           // (other lanes read the records)
  if constexpr (sizeof(KEY) == 4) {
    if (check) {
      // The first m records hold the k largest if a gap behind them is wider than the errors of any two scores (at most rel + err
      // each) and the roundings of the sums with their biases.
      const auto apart = [&](int j) {
        const float p = line[j].c, q = line[j + 1].c;
        return p - q > 2.0f * (rel + err) + 0x1p-22f * (1.0f + fabsf(p) + fabsf(q));
      };
      int m = found;
      if (found > a.k) {
        if (apart(a.k - 1)) m = a.k;
        else if (found == a.k + 1 || apart(a.k)) m = a.k + 1;
        else good = false;
      }
      // and are in order if neighbours are ties or further apart than their errors; else float64 puts them in order
      bool ordered = true;
      for (int j = w.lr; j + 1 < m; j += GL) {
        const Record p = line[j], q = line[j + 1];
        const bool tie = p.l == q.l && p.b == q.b;
        const float room = rel * (fabsf(p.c - p.b) + fabsf(q.c - q.b)) + 2.0f * err + 0x1p-22f * (1.0f + fabsf(p.c));
        if (!tie && !(p.c - q.c > room)) ordered = false;
      }
      const unsigned long long off = __ballot(!ordered) >> lane0;
      if (good && (GL < 64 ? off & ((1ull << (GL & 63)) - 1ull) : off) != 0ull) settle<GL, E>(a, w, line, m);
    }
  }
  if (sizeof(KEY) == 4 && scored) {
    const unsigned long long bad = __ballot(!good) >> lane0;
    good = (GL < 64 ? bad & ((1ull << (GL & 63)) - 1ull) : bad) == 0ull;
  }
  *sure = good;
  return min(found, a.k);
}

// GL lanes per row, E elements per lane
template <class T, int GL, int E>
__global__ __launch_bounds__(kThreads) void route_fwd_kernel(RouteArgs a, int lanes) {
  __shared__ __attribute__((aligned(16))) Record lines[kThreads / GL][kRecords];
  const int64_t row = (int64_t(blockIdx.x) * kThreads + threadIdx.x) / GL;
  if (row >= a.rows) return;                                       // (whole row groups; no barrier below)
  Lane<E> w;
  w.lr = int(threadIdx.x) & (GL - 1);
  w.lanes = lanes;
  w.g = w.lr / lanes;
  const int size = a.n / a.groups, in = (w.lr & (lanes - 1)) * E;
  const int count = w.g < a.groups ? min(max(size - in, 0), E) : 0;  // elements of this lane
  const int base = w.g * size + in;
  load_row_part<T, E>(static_cast<const T*>(a.logits) + row * a.stride + base, count, kNone, w.l);
  if (a.bias != nullptr) load_row_part<float, E>(a.bias + base, count, 0.0f, w.b);
#pragma unroll
  for (int e = 0; e < E; ++e) {
    if (a.bias == nullptr) w.b[e] = 0.0f;
    if (isnan(w.l[e])) w.l[e] = kNone;
  }
  w.top = group_max<GL>(max_all(w.l));

  // Scores, not logits, are compared where a bias is added or scores of a group are.  Float32 decides where its errors leave no
  // doubt; else float64 puts the few records in order (8192 x 256 with sigmoid scores, k = 8: about one row in a thousand), or all
  // the row, where it is not sure which they are.
  const bool scored = a.bias != nullptr || (a.groups > 1 && a.top == 2);
  bool sure;
  Record* line = lines[threadIdx.x / GL];
  int found = choose<GL, E, float>(a, w, scored, base, line, &sure);
  if (scored && !sure) found = choose<GL, E, double>(a, w, scored, base, line, &sure);

  // their weights: lane q takes the choices q, q + GL, ..
  float m = 0.0f, sum = 0.0f;
  if (a.renorm) {
    m = kNone;
    for (int j = w.lr; j < found; j += GL) m = max_of(m, a.score == kSoftmax ? line[j].l : fminf(line[j].l, 0.0f));
    m = group_max<GL>(m);
    for (int j = w.lr; j < found; j += GL) sum += a.score == kSoftmax ? exp_below(line[j].l, m) : sigmoid_over(line[j].l, m);
    sum = group_sum_f32<GL>(sum);
  } else if (a.score == kSoftmax) {
    m = w.top;
#pragma unroll
    for (int e = 0; e < E; ++e) sum += w.l[e] == kNone ? 0.0f : exp_below(w.l[e], m);
    sum = group_sum_f32<GL>(sum);
  } else {
    sum = 1.0f;
  }
  const float factor = a.scale / sum;
  for (int j = w.lr; j < a.k; j += GL) {
    const bool there = j < found;
    const float l = there ? line[j].l : 0.0f;
    const float u = a.score == kSoftmax ? exp_below(l, m) : sigmoid_over(l, m);
    a.idx[row * a.k + j] = there ? line[j].i : -1;
    a.val[row * a.k + j] = there ? u * factor : 0.0f;
  }
}

// Gradient in the logits of <val, cotangent>, val as above for the given idx (which carry no gradient).  With w the weights
// without `scale`, mean = sum_j w_j t_j:
//   softmax, renormalised   dl[idx_j] += scale w_j (t_j - mean)
//   softmax                 dl[idx_j] += scale w_j t_j,  dl -= scale s mean
//   sigmoid, renormalised   dl[idx_j] += scale w_j (1 - s_j) (t_j - mean)
//   sigmoid                 dl[idx_j] += scale s_j (1 - s_j) t_j
// Lane q of a row takes the choices q, q + GL, ..: their terms are then handed to the lanes that hold the entries.  Only
// softmax that is not renormalised reads the whole row.  All of the gradient is written: 32768 x 128 float32, k = 8: 12.6 us
// a call, 2.8 TB/s; the others 9.9 (softmax), 10.6 and 9.8 (sigmoid), 2.0 TB/s.
template <class T, int GL, int E>
__global__ __launch_bounds__(kThreads) void route_vjp_kernel(RouteVjpArgs a) {
  constexpr int J = kChoicesMax / GL;                              // choices of a lane, at most
  const int64_t row = (int64_t(blockIdx.x) * kThreads + threadIdx.x) / GL;
  if (row >= a.rows) return;
  const int lr = int(threadIdx.x) & (GL - 1);
  const int base = lr * E, count = min(max(a.n - base, 0), E);
  const T* lp = static_cast<const T*>(a.logits) + row * a.stride;
  const bool whole = a.score == kSoftmax && !a.renorm;
  int at[J];
  float l[J], t[J];
#pragma unroll
  for (int q = 0; q < J; ++q) {
    at[q] = -1;
    l[q] = kNone;
    t[q] = 0.0f;
    const int j = q * GL + lr;
    if (q * GL < a.k && j < a.k) {
      at[q] = a.idx[row * a.k + j];
      if (at[q] < 0 || at[q] >= a.n) at[q] = -1;
      if (at[q] >= 0) {
        l[q] = to_f32(lp[at[q]]);
        t[q] = a.cotangent[row * a.k + j];
      }
      if (!(l[q] > kNone)) {                                       // -inf, NaN: an expert that is out has weight 0
        l[q] = kNone;
        t[q] = 0.0f;
      }
    }
  }
  float s[E];
  float m = kNone;
  double sum = 0.0, mean = 0.0;
  if (whole) {
    load_row_part<T, E>(lp + base, count, kNone, s);
#pragma unroll
    for (int e = 0; e < E; ++e) {
      if (isnan(s[e])) s[e] = kNone;
      m = max_of(m, s[e]);
    }
    m = group_max<GL>(m);
#pragma unroll
    for (int e = 0; e < E; ++e) s[e] = s[e] == kNone ? 0.0f : exp_below(s[e], m);
#pragma unroll
    for (int e = 0; e < E; e += 4) sum += double((s[e] + s[e + 1]) + (s[e + 2] + s[e + 3]));
  } else if (a.renorm) {
#pragma unroll
    for (int q = 0; q < J; ++q) m = max_of(m, a.score == kSoftmax ? l[q] : fminf(l[q], 0.0f));
    m = group_max<GL>(m);
  } else {
    m = 0.0f;
  }
  float w[J];
#pragma unroll
  for (int q = 0; q < J; ++q) {
    w[q] = l[q] == kNone ? 0.0f : a.score == kSoftmax ? exp_below(l[q], m) : sigmoid_over(l[q], m);
    mean += double(w[q]) * double(t[q]);
    if (!whole) sum += double(w[q]);
  }
  if (whole || a.renorm) {
    sum = group_sum_f64<GL>(sum);
    mean = group_sum_f64<GL>(mean);
  } else {
    sum = 1.0;
  }
  const double inv = sum > 0.0 ? 1.0 / sum : 0.0;
  mean *= inv;
  const float less = float(-inv * mean);
  float d[E];
#pragma unroll
  for (int e = 0; e < E; ++e) d[e] = whole ? s[e] * less : 0.0f;
#pragma unroll
  for (int q = 0; q < J; ++q) {
    if (q * GL >= a.k) break;
    float v = float(double(w[q]) * inv * (a.renorm ? double(t[q]) - mean : double(t[q])));
    if (a.score == kSigmoid && l[q] > kNone) v *= sigmoid_over(-l[q], 0.0f);
    const int here = min(a.k - q * GL, GL);
    for (int j = 0; j < here; ++j) {
      const int i = __shfl(at[q], j, GL) - base;
      const float add = __shfl(v, j, GL);
#pragma unroll
      for (int e = 0; e < E; ++e) d[e] += i == e ? add : 0.0f;
    }
  }
#pragma unroll
  for (int e = 0; e < E; ++e) d[e] *= a.scale;
  store_row_part<T, E>(static_cast<T*>(a.grad) + row * a.n + base, count, d);
}

template <class T, int GL, int E>
void fwd(const RouteArgs& a, int padded, hipStream_t stream) {
  const dim3 grid(unsigned((a.rows * GL + kThreads - 1) / kThreads));
  hipLaunchKernelGGL((route_fwd_kernel<T, GL, E>), grid, dim3(kThreads), 0, stream, a, GL / padded);
}

template <class T>
int fwd_type(const RouteArgs& a, hipStream_t stream) {
  int padded = 1;                        // groups, up to a power of two
  while (padded < a.groups) padded *= 2;
  const int size = a.n / a.groups;
  // the fewest lanes whose registers hold a row: the k rounds cost a reduction over the lanes each
  const auto fits = [&](int gl, int e) { return padded <= gl && size <= gl / padded * e; };
  if (fits(8, 4)) fwd<T, 8, 4>(a, padded, stream);
  else if (fits(8, 8)) fwd<T, 8, 8>(a, padded, stream);
  else if (fits(16, 8)) fwd<T, 16, 8>(a, padded, stream);
  else if (fits(32, 8)) fwd<T, 32, 8>(a, padded, stream);
  else if (fits(64, 8)) fwd<T, 64, 8>(a, padded, stream);
  else if (fits(64, 16)) fwd<T, 64, 16>(a, padded, stream);
  else if (fits(64, 32)) fwd<T, 64, 32>(a, padded, stream);
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
