// C ABI of the operators behind a router: argument validation and dispatch.  See include/sparse_topk.h.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "../../include/sparse_topk.h"
#include "experts.hpp"

namespace {

constexpr int64_t kMost = int64_t(1) << 31;
constexpr int64_t kRowsOfLaunch = int64_t(1) << 25;      // routing: up to 64 threads each
constexpr int64_t kTokensOfLaunch = int64_t(1) << 23;    // weighted sums: up to 256, of each slice of a row
constexpr int64_t kSlicesOfLaunch = int64_t(1) << 15;    // (the second dimension of a grid has fewer than 2^16)
constexpr int64_t kPairsOfLaunch = int64_t(1) << 25;     // and their gradients: up to 64

int64_t size_of(int type) { return type == TOPK_TYPE_F32 ? 4 : 2; }
const void* ahead(const void* p, int64_t bytes) { return p == nullptr ? nullptr : static_cast<const char*>(p) + bytes; }
void* ahead(void* p, int64_t bytes) { return p == nullptr ? nullptr : static_cast<char*>(p) + bytes; }

bool known_type(int type) { return type >= TOPK_TYPE_F32 && type <= TOPK_TYPE_F16; }
bool known_score(int score) { return score == TOPK_SCORE_SOFTMAX || score == TOPK_SCORE_SIGMOID; }

// as in api.hip: an error that an earlier, unrelated call left is not this call's
void begin() { (void)hipGetLastError(); }
int finish(int launched) {
  if (launched != 0) return TOPK_ERR_INVALID;
  return hipGetLastError() == hipSuccess ? TOPK_OK : TOPK_ERR_LAUNCH;
}
hipStream_t as_stream(void* s) { return static_cast<hipStream_t>(s); }

int check_route(int type, int64_t stride, int64_t rows, int64_t n, int64_t k, int score, double scale) {
  if (rows < 0 || rows >= kMost || n < 1 || n > TOPK_EXPERTS_MAX || k < 1 || k > n || k > TOPK_CHOICES_MAX || stride < 0)
    return TOPK_ERR_INVALID;
  if (!known_type(type) || !known_score(score) || !std::isfinite(float(scale))) return TOPK_ERR_INVALID;
  return TOPK_OK;
}

int check_product(const topk::ProductArgs& p, int type) {
  if (!known_type(type) || p.n < 1 || p.n > TOPK_EXPERTS_MAX || p.h < 1 || p.ho < 1 || p.h >= kMost || p.ho >= kMost ||
      p.slots < 0 || p.slots >= kMost || p.m < 0 || p.m >= kMost || p.k < 1 || p.k >= kMost)
    return TOPK_ERR_INVALID;
  if (p.x_stride < 0 || p.t_stride < 0 || p.w_expert < 0 || p.w_out < 0 || p.w_in < 0) return TOPK_ERR_INVALID;
  if (p.w_out != 1 && p.w_in != 1) return TOPK_ERR_INVALID;
  if (p.offset == nullptr || (p.slots > 0 && p.source == nullptr && p.m < p.slots)) return p.offset == nullptr ? TOPK_ERR_NULL : TOPK_ERR_INVALID;
  return TOPK_OK;
}

int check_combine(const topk::CombineArgs& c, int type) {
  if (!known_type(type) || c.rows < 0 || c.rows >= kMost || c.k < 1 || c.k > kPairsOfLaunch || c.slots < 0 || c.slots >= kMost ||
      c.h < 1 || c.h >= kMost || c.y_stride < 0 || c.t_stride < 0)
    return TOPK_ERR_INVALID;
  return TOPK_OK;
}

}  // namespace

extern "C" {

int topk_route_fwd(const void* logits, int type, int64_t stride, const float* bias, int64_t rows, int64_t n, int64_t k,
                   int score, int64_t groups, int64_t keep_groups, int group_top, int renormalise, double scale,
                   int32_t* idx_out, float* val_out, void* stream) {
  const int rc = check_route(type, stride, rows, n, k, score, scale);
  if (rc != TOPK_OK) return rc;
  if (groups < 1 || groups > n || groups > TOPK_ROUTE_GROUPS_MAX || n % groups != 0 || keep_groups < 1 ||
      keep_groups > groups || (group_top != 1 && group_top != 2) || k > n / groups * keep_groups)
    return TOPK_ERR_INVALID;
  if (rows == 0) return TOPK_OK;
  if (logits == nullptr || idx_out == nullptr || val_out == nullptr) return TOPK_ERR_NULL;
  begin();
  int launched = 0;
  for (int64_t r = 0; r < rows && launched == 0; r += kRowsOfLaunch) {
    const topk::RouteArgs a{ahead(logits, r * stride * size_of(type)), stride, bias, std::min(rows - r, kRowsOfLaunch), int(n),
                            int(k), int(groups), int(keep_groups), group_top, score, renormalise != 0, float(scale),
                            idx_out + r * k, val_out + r * k};
    launched = topk::launch_route_fwd(type, a, as_stream(stream));
  }
  return finish(launched);
}

int topk_route_vjp(const void* logits, int type, int64_t stride, const int32_t* idx, const float* cotangent, int64_t rows,
                   int64_t n, int64_t k, int score, int renormalise, double scale, void* grad_out, void* stream) {
  const int rc = check_route(type, stride, rows, n, k, score, scale);
  if (rc != TOPK_OK) return rc;
  if (rows == 0) return TOPK_OK;
  if (logits == nullptr || idx == nullptr || cotangent == nullptr || grad_out == nullptr) return TOPK_ERR_NULL;
  begin();
  int launched = 0;
  for (int64_t r = 0; r < rows && launched == 0; r += kRowsOfLaunch) {
    const topk::RouteVjpArgs a{ahead(logits, r * stride * size_of(type)), stride, idx + r * k, cotangent + r * k,
                               std::min(rows - r, kRowsOfLaunch), int(n), int(k), score, renormalise != 0, float(scale),
                               ahead(grad_out, r * n * size_of(type))};
    launched = topk::launch_route_vjp(type, a, as_stream(stream));
  }
  return finish(launched);
}

size_t topk_expert_map_bytes(int64_t rows, int64_t k, int64_t n) {
  if (rows < 0 || k < 1 || n < 1 || n > TOPK_EXPERTS_MAX || rows > (kMost - 1) / k) return 0;
  const int64_t chunks = topk::map_chunks(rows * k, int(n));
  return chunks > 1 ? size_t(chunks) * size_t(topk::map_width(int(n))) * 4 : 0;
}

int topk_expert_map(const int32_t* idx, int64_t rows, int64_t k, int64_t n, int64_t capacity, int32_t* slot_out,
                    int32_t* source_out, int32_t* offset_out, int32_t* load_out, void* scratch, size_t scratch_bytes,
                    void* stream) {
  if (rows < 0 || k < 1 || n < 1 || n > TOPK_EXPERTS_MAX || rows > (kMost - 1) / k || capacity < 0) return TOPK_ERR_INVALID;
  if (offset_out == nullptr || load_out == nullptr) return TOPK_ERR_NULL;
  if (rows > 0 && (idx == nullptr || slot_out == nullptr || source_out == nullptr)) return TOPK_ERR_NULL;
  const size_t need = topk_expert_map_bytes(rows, k, n);
  if (need > 0 && (scratch == nullptr || scratch_bytes < need)) return TOPK_ERR_WORKSPACE;
  if (reinterpret_cast<uintptr_t>(scratch) % 16 != 0) return TOPK_ERR_INVALID;
  begin();
  const topk::MapArgs a{idx, rows * k, int(n), capacity > 0 ? capacity : kMost, slot_out, source_out, offset_out, load_out,
                        static_cast<int32_t*>(scratch)};
  return finish(topk::launch_expert_map(a, as_stream(stream)));
}

int topk_expert_product_fwd(const void* x, int64_t x_stride, int64_t m, const void* w, int64_t w_expert, int64_t w_out,
                            int64_t w_in, const int32_t* offset, const int32_t* source, int64_t k, int64_t slots, int64_t n,
                            int64_t h, int64_t ho, int type, void* out, void* stream) {
  topk::ProductArgs p{};
  p.x = x, p.x_stride = x_stride, p.m = m, p.w = w, p.w_expert = w_expert, p.w_out = w_out, p.w_in = w_in;
  p.offset = offset, p.source = source, p.k = k, p.slots = slots, p.n = int(n), p.h = h, p.ho = ho, p.out = out;
  if (n > TOPK_EXPERTS_MAX || n < 1) return TOPK_ERR_INVALID;
  const int rc = check_product(p, type);
  if (rc != TOPK_OK) return rc;
  if (slots == 0) return TOPK_OK;
  if ((x == nullptr && m > 0) || w == nullptr || out == nullptr) return TOPK_ERR_NULL;
  begin();
  return finish(topk::launch_product_fwd(type, p, as_stream(stream)));
}

int topk_expert_product_vjp(const void* x, int64_t x_stride, int64_t m, const void* w, int64_t w_expert, int64_t w_out,
                            int64_t w_in, const int32_t* offset, const int32_t* source, int64_t k, int64_t slots, int64_t n,
                            int64_t h, int64_t ho, int type, const void* cotangent, int64_t cotangent_stride, void* dx_out,
                            void* dw_out, void* stream) {
  topk::ProductArgs p{};
  p.x = x, p.x_stride = x_stride, p.m = m, p.w = w, p.w_expert = w_expert, p.w_out = w_out, p.w_in = w_in;
  p.offset = offset, p.source = source, p.k = k, p.slots = slots, p.n = int(n), p.h = h, p.ho = ho;
  p.t = cotangent, p.t_stride = cotangent_stride, p.dx = dx_out, p.dw = dw_out;
  if (n > TOPK_EXPERTS_MAX || n < 1) return TOPK_ERR_INVALID;
  const int rc = check_product(p, type);
  if (rc != TOPK_OK) return rc;
  if (dx_out == nullptr && dw_out == nullptr && slots > 0) return TOPK_ERR_NULL;
  if (slots > 0 && (cotangent == nullptr || (dw_out != nullptr && x == nullptr && m > 0) || (dx_out != nullptr && w == nullptr)))
    return TOPK_ERR_NULL;
  begin();
  int launched = 0;
  if (dx_out != nullptr && slots > 0) launched = topk::launch_product_dx(type, p, as_stream(stream));
  if (dw_out != nullptr && launched == 0) launched = topk::launch_product_dw(type, p, as_stream(stream));
  return finish(launched);
}

int topk_combine_fwd(const void* y, int64_t y_stride, const int32_t* slot, const float* val, int64_t rows, int64_t k,
                     int64_t slots, int64_t h, int type, void* out, void* stream) {
  const topk::CombineArgs c{y, y_stride, slot, val, nullptr, 0, rows, k, slots, h, 0, 0, out, nullptr, nullptr};
  const int rc = check_combine(c, type);
  if (rc != TOPK_OK) return rc;
  if (rows == 0) return TOPK_OK;
  if ((y == nullptr && slots > 0) || slot == nullptr || out == nullptr) return TOPK_ERR_NULL;
  begin();
  const int64_t slices = topk::combine_slices(type, h), across = std::min(slices, kSlicesOfLaunch);
  const int64_t tokens = kTokensOfLaunch / across;
  int launched = 0;
  for (int64_t s = 0; s < slices; s += across) {
    for (int64_t t = 0; t < rows && launched == 0; t += tokens) {
      topk::CombineArgs part = c;
      part.rows = std::min(rows - t, tokens);
      part.slot = slot + t * k;
      part.val = val == nullptr ? nullptr : val + t * k;
      part.out = ahead(out, t * h * size_of(type));
      part.slice = s;
      part.slices = std::min(slices - s, across);
      launched = topk::launch_combine_fwd(type, part, as_stream(stream));
    }
  }
  return finish(launched);
}

int topk_combine_vjp(const void* y, int64_t y_stride, const int32_t* slot, const float* val, const void* cotangent,
                     int64_t cotangent_stride, int64_t rows, int64_t k, int64_t slots, int64_t h, int type, void* dy_out,
                     float* dval_out, void* stream) {
  const topk::CombineArgs c{y, y_stride, slot, val, cotangent, cotangent_stride, rows, k, slots, h, 0, 0, nullptr, dy_out, dval_out};
  const int rc = check_combine(c, type);
  if (rc != TOPK_OK) return rc;
  if (rows == 0) return TOPK_OK;
  if (slot == nullptr || cotangent == nullptr || (slots > 0 && (dy_out == nullptr || (y == nullptr && dval_out != nullptr))))
    return TOPK_ERR_NULL;
  if (val != nullptr && dval_out == nullptr) return TOPK_ERR_NULL;
  begin();
  const int64_t tokens = kPairsOfLaunch / k;
  int launched = 0;
  for (int64_t t = 0; t < rows && launched == 0; t += tokens) {
    topk::CombineArgs part = c;
    part.rows = std::min(rows - t, tokens);
    part.slot = slot + t * k;
    part.val = val == nullptr ? nullptr : val + t * k;
    part.t = ahead(cotangent, t * cotangent_stride * size_of(type));
    part.dval = dval_out == nullptr ? nullptr : dval_out + t * k;
    launched = topk::launch_combine_vjp(type, part, as_stream(stream));
  }
  return finish(launched);
}

}  // extern "C"
