// C ABI of the experts' feed-forward: argument validation and dispatch.  See include/sparse_topk.h.
#include <hip/hip_runtime.h>

#include "../../include/sparse_topk.h"
#include "feed_forward.hpp"

namespace {

constexpr int64_t kMost = int64_t(1) << 31;

bool known_type(int type) { return type >= TOPK_TYPE_F32 && type <= TOPK_TYPE_F16; }
bool known_act(int act) { return act >= TOPK_ACT_SILU && act <= TOPK_ACT_RELU; }

// as in api.hip: an error that an earlier, unrelated call left is not this call's
void begin() { (void)hipGetLastError(); }
int finish(int launched) {
  if (launched != 0) return TOPK_ERR_INVALID;
  return hipGetLastError() == hipSuccess ? TOPK_OK : TOPK_ERR_LAUNCH;
}
hipStream_t as_stream(void* s) { return static_cast<hipStream_t>(s); }

// what the entry points share: shapes, the lists and the strides of rows and weights
int check_lists(int64_t m, int64_t k, int64_t slots, int64_t n, int64_t h, int64_t f, int64_t x_stride, int64_t w_expert,
                int64_t w_out, int64_t w_in, const int32_t* offset, const int32_t* source) {
  if (n < 1 || n > TOPK_EXPERTS_MAX || h < 1 || f < 1 || h >= kMost || f >= kMost || slots < 0 || slots >= kMost || m < 0 ||
      m >= kMost || k < 1 || k >= kMost || x_stride < 0 || w_expert < 0 || w_out < 0 || w_in < 0 || (w_out != 1 && w_in != 1))
    return TOPK_ERR_INVALID;
  if (offset == nullptr) return TOPK_ERR_NULL;
  if (slots > 0 && source == nullptr && m < slots) return TOPK_ERR_INVALID;
  return TOPK_OK;
}

topk::GatedArgs gated(const void* x, int64_t x_stride, int64_t m, const void* w_gate, const void* w_up, int64_t w_expert,
                      int64_t w_out, int64_t w_in, const int32_t* offset, const int32_t* source, int64_t k, int64_t slots,
                      int64_t n, int64_t h, int64_t f, int act) {
  topk::GatedArgs g{};
  topk::ProductArgs& p = g.p;
  p.x = x, p.x_stride = x_stride, p.m = m, p.w = w_gate, p.w_expert = w_expert, p.w_out = w_out, p.w_in = w_in;
  p.offset = offset, p.source = source, p.k = k, p.slots = slots, p.n = int(n), p.h = h, p.ho = f;
  g.w_up = w_up, g.act = act;
  return g;
}

int check_eight(const topk::EightArgs& e) {
  if (e.h > TOPK_I8_WIDTH_MAX || !known_type(e.out_type) || !known_act(e.act)) return TOPK_ERR_INVALID;
  if (e.slots == 0) return TOPK_OK;
  if ((e.m > 0 && (e.x == nullptr || e.x_scale == nullptr)) || e.w == nullptr || e.w_scale == nullptr || e.out == nullptr)
    return TOPK_ERR_NULL;
  return TOPK_OK;
}

}  // namespace

extern "C" {

int topk_expert_gated_fwd(const void* x, int64_t x_stride, int64_t m, const void* w_gate, const void* w_up, int64_t w_expert,
                          int64_t w_out, int64_t w_in, const int32_t* offset, const int32_t* source, int64_t k, int64_t slots,
                          int64_t n, int64_t h, int64_t f, int type, int act, void* out, void* pre_out, void* stream) {
  const int rc = check_lists(m, k, slots, n, h, f, x_stride, w_expert, w_out, w_in, offset, source);
  if (rc != TOPK_OK) return rc;
  if (!known_type(type) || !known_act(act)) return TOPK_ERR_INVALID;
  if (slots == 0) return TOPK_OK;
  if ((x == nullptr && m > 0) || w_gate == nullptr || w_up == nullptr || out == nullptr) return TOPK_ERR_NULL;
  topk::GatedArgs g = gated(x, x_stride, m, w_gate, w_up, w_expert, w_out, w_in, offset, source, k, slots, n, h, f, act);
  g.p.out = out, g.pre = pre_out;
  begin();
  return finish(topk::launch_gated_fwd(type, g, as_stream(stream)));
}

size_t topk_expert_gated_vjp_bytes(int64_t slots, int64_t f, int type) {
  if (slots < 0 || slots >= kMost || f < 1 || f >= kMost || !known_type(type)) return 0;
  size_t bytes;
  if (__builtin_mul_overflow(size_t(slots), size_t(topk::slopes_stride(type, f)) * (type == TOPK_TYPE_F32 ? 4 : 2), &bytes))
    return SIZE_MAX;
  return bytes;
}

int topk_expert_gated_vjp(const void* x, int64_t x_stride, int64_t m, const void* w_gate, const void* w_up, int64_t w_expert,
                          int64_t w_out, int64_t w_in, const int32_t* offset, const int32_t* source, int64_t k, int64_t slots,
                          int64_t n, int64_t h, int64_t f, int type, int act, const void* pre, const void* cotangent,
                          int64_t cotangent_stride, void* dx_out, void* dw_gate_out, void* dw_up_out, void* scratch,
                          size_t scratch_bytes, void* stream) {
  const int rc = check_lists(m, k, slots, n, h, f, x_stride, w_expert, w_out, w_in, offset, source);
  if (rc != TOPK_OK) return rc;
  if (!known_type(type) || !known_act(act) || cotangent_stride < 0) return TOPK_ERR_INVALID;
  if ((dw_gate_out == nullptr) != (dw_up_out == nullptr)) return TOPK_ERR_NULL;
  if (slots == 0 && dw_gate_out == nullptr) return TOPK_OK;
  if (slots > 0 && ((dx_out == nullptr && dw_gate_out == nullptr) || cotangent == nullptr || w_gate == nullptr ||
                    w_up == nullptr || (x == nullptr && m > 0)))
    return TOPK_ERR_NULL;
  const size_t need = topk_expert_gated_vjp_bytes(slots, f, type);
  if (need > 0 && (scratch == nullptr || scratch_bytes < need)) return TOPK_ERR_WORKSPACE;
  if (reinterpret_cast<uintptr_t>(scratch) % 16 != 0) return TOPK_ERR_INVALID;
  topk::GatedArgs g = gated(x, x_stride, m, w_gate, w_up, w_expert, w_out, w_in, offset, source, k, slots, n, h, f, act);
  g.p.t = cotangent, g.p.t_stride = cotangent_stride, g.p.dx = dx_out, g.p.dw = dw_gate_out, g.dw_up = dw_up_out;
  g.kept = pre, g.scratch = scratch;
  begin();
  return finish(topk::launch_gated_vjp(type, g, as_stream(stream)));
}

int topk_quantise_rows(const void* x, int64_t x_stride, int64_t m, int64_t h, int type, int8_t* q_out, float* scale_out,
                       void* stream) {
  if (m < 0 || m >= kMost || h < 1 || h >= kMost || x_stride < 0 || !known_type(type)) return TOPK_ERR_INVALID;
  if (m == 0) return TOPK_OK;
  if (x == nullptr || q_out == nullptr || scale_out == nullptr) return TOPK_ERR_NULL;
  begin();
  return finish(topk::launch_quantise(type, topk::QuantiseArgs{x, x_stride, m, h, q_out, scale_out}, as_stream(stream)));
}

int topk_expert_product_i8_fwd(const int8_t* x, int64_t x_stride, int64_t m, const float* x_scale, const int8_t* w,
                               int64_t w_expert, int64_t w_out, const float* w_scale, const int32_t* offset,
                               const int32_t* source, int64_t k, int64_t slots, int64_t n, int64_t h, int64_t ho, int out_type,
                               void* out, void* stream) {
  int rc = check_lists(m, k, slots, n, h, ho, x_stride, w_expert, w_out, 1, offset, source);
  if (rc != TOPK_OK) return rc;
  const topk::EightArgs e{x,      x_stride, m, x_scale, w,      nullptr, w_expert, w_out,         w_scale,  nullptr,
                          offset, source,   k, slots,   int(n), h,       ho,       TOPK_ACT_SILU, out_type, out};
  rc = check_eight(e);
  if (rc != TOPK_OK || slots == 0) return rc;
  begin();
  return finish(topk::launch_eight(e, as_stream(stream)));
}

int topk_expert_gated_i8_fwd(const int8_t* x, int64_t x_stride, int64_t m, const float* x_scale, const int8_t* w_gate,
                             const float* gate_scale, const int8_t* w_up, const float* up_scale, int64_t w_expert, int64_t w_out,
                             const int32_t* offset, const int32_t* source, int64_t k, int64_t slots, int64_t n, int64_t h,
                             int64_t f, int out_type, int act, void* out, void* stream) {
  int rc = check_lists(m, k, slots, n, h, f, x_stride, w_expert, w_out, 1, offset, source);
  if (rc != TOPK_OK) return rc;
  const topk::EightArgs e{x,      x_stride, m, x_scale, w_gate, w_up, w_expert, w_out, gate_scale, up_scale,
                          offset, source,   k, slots,   int(n), h,    f,        act,   out_type,   out};
  rc = check_eight(e);
  if (rc != TOPK_OK || slots == 0) return rc;
  if (w_up == nullptr || up_scale == nullptr) return TOPK_ERR_NULL;
  begin();
  return finish(topk::launch_eight(e, as_stream(stream)));
}

}  // extern "C"
