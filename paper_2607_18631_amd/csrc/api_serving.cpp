// C ABI of the operators around the layer: block-scaled formats and their expert MLP, the norm in front
// of a layer and its backward, the few-token layer.  Validation and dispatch only, as in api.cpp.
#include <hip/hip_runtime_api.h>

#include <cmath>

#include "../../include/moe.h"
#include "api_common.hpp"
#include "kernels.hpp"

namespace {

using namespace moe::abi;

int check_format(int format) {
  if (format != MOE_MX_E2M1 && format != MOE_MX_E4M3)
    return fail(MOE_ERR_UNSUPPORTED, "format (%d) is neither MOE_MX_E2M1 nor MOE_MX_E4M3", format);
  return MOE_OK;
}

int check_mx_sizes(int64_t rows, int32_t cols, int format) {
  if (rows < 0) return fail(MOE_ERR_INVALID_ARG, "rows (%lld) < 0", (long long)rows);
  if (cols <= 0) return fail(MOE_ERR_INVALID_ARG, "cols (%d) <= 0", cols);
  if (cols % 32) return fail(MOE_ERR_UNSUPPORTED, "cols (%d) %% 32 != 0 (blocks of 32 values share a scale)", cols);
  if (rows >= (int64_t(1) << 40) / cols)
    return fail(MOE_ERR_UNSUPPORTED, "rows * cols (%lld * %d) >= 2^40", (long long)rows, cols);
  return check_format(format);
}

moe::MxConvertProblem mx_problem(int64_t rows, int32_t cols, int format, const void* x, void* out, const void* elements,
                                 const void* scales) {
  moe::MxConvertProblem p{};
  p.x = static_cast<const moe::bf16_t*>(x);
  p.out = static_cast<moe::bf16_t*>(out);
  p.elements = static_cast<uint8_t*>(const_cast<void*>(elements));
  p.scales = static_cast<uint8_t*>(const_cast<void*>(scales));
  p.n = rows * cols;
  p.format = format;
  return p;
}

int check_norm_sizes(int64_t rows, int32_t d) {
  if (rows < 0) return fail(MOE_ERR_INVALID_ARG, "rows (%lld) < 0", (long long)rows);
  if (rows >= (int64_t(1) << 31)) return fail(MOE_ERR_UNSUPPORTED, "rows (%lld) >= 2^31", (long long)rows);
  if (d <= 0) return fail(MOE_ERR_INVALID_ARG, "d (%d) <= 0", d);
  if (d % 8) return fail(MOE_ERR_UNSUPPORTED, "d (%d) %% 8 != 0 (rows must be 16-byte bf16 vectors)", d);
  // column numbers are 32 bits wide, a workgroup's 32 columns of dgamma from the last whole 32 on included
  if (d > INT32_MAX - 31) return fail(MOE_ERR_UNSUPPORTED, "d (%d) > 2^31 - 32", d);
  return MOE_OK;
}

size_t norm_ws(int64_t rows, int32_t d) {
  return align_up((size_t)moe::add_norm_bwd_parts(rows, d) * (size_t)d * sizeof(float));
}

}  // namespace

extern "C" {

int moe_mx_quantize(int64_t rows, int32_t cols, int format, const void* x, void* elements, void* scales,
                    void* stream) {
  CHECK(check_mx_sizes(rows, cols, format));
  if (rows == 0) return ok();
  CHECK(check_ptr(x, 16, "x"));
  CHECK(check_ptr(elements, 16, "elements"));
  CHECK(check_ptr(scales, 16, "scales"));
  CHECK(hip_status(moe::launch_mx_quantize(mx_problem(rows, cols, format, x, nullptr, elements, scales),
                                           as_stream(stream)),
                   "block-scaled conversion launch"));
  return ok();
}

int moe_mx_dequantize(int64_t rows, int32_t cols, int format, const void* elements, const void* scales, void* x,
                      void* stream) {
  CHECK(check_mx_sizes(rows, cols, format));
  if (rows == 0) return ok();
  CHECK(check_ptr(elements, 16, "elements"));
  CHECK(check_ptr(scales, 16, "scales"));
  CHECK(check_ptr(x, 16, "x"));
  CHECK(hip_status(moe::launch_mx_dequantize(mx_problem(rows, cols, format, nullptr, x, elements, scales),
                                             as_stream(stream)),
                   "block-scaled conversion launch"));
  return ok();
}

int moe_mx_grouped_ffn(const moe_shape_t* shape, int format, const void* x_q, const void* x_scales,
                       const int32_t* offsets, const void* w13_q, const void* w13_scales, const void* w2_q,
                       const void* w2_scales, void* y_perm, void* ws, size_t ws_bytes, void* stream) {
  CHECK(check_shape(shape));
  CHECK(check_format(format));
  CHECK(check_mx_shape(shape));
  if (shape->E_local > moe::kMaxGroups)
    return fail(MOE_ERR_UNSUPPORTED, "E_local (%d) > %d", shape->E_local, moe::kMaxGroups);
  // 32-bit byte offsets into a tile's 256 rows and into a group's weights
  const int32_t widest = shape->d > shape->F ? shape->d : shape->F;
  if (widest >= moe::kMxRowValues) return fail(MOE_ERR_UNSUPPORTED, "d or F (%d) >= 2^20", widest);
  if ((int64_t)shape->d * shape->F >= moe::kMxGroupValues)
    return fail(MOE_ERR_UNSUPPORTED, "d * F (%lld) >= 2^31", (long long)shape->d * shape->F);
  if (shape->T == 0) return ok();
  CHECK(check_ptr(x_q, 16, "x_q"));
  CHECK(check_ptr(x_scales, 16, "x_scales"));
  CHECK(check_ptr(offsets, 4, "offsets"));
  CHECK(check_ptr(w13_q, 16, "w13_q"));
  CHECK(check_ptr(w13_scales, 16, "w13_scales"));
  CHECK(check_ptr(w2_q, 16, "w2_q"));
  CHECK(check_ptr(w2_scales, 16, "w2_scales"));
  CHECK(check_ptr(y_perm, 16, "y_perm"));
  const MxFfnLayout L = mx_ffn_layout(shape);
  CHECK(check_ws_bytes(L.total, ws, ws_bytes));
  moe::MxGemmProblem up{};
  up.X = static_cast<const uint8_t*>(x_q);
  up.X_scales = static_cast<const uint8_t*>(x_scales);
  up.offsets = offsets;
  up.groups = shape->E_local;
  up.max_rows = capacity(shape);
  up.seg_stride = shape->expert_capacity;
  up.W = static_cast<const uint8_t*>(w13_q);
  up.W_scales = static_cast<const uint8_t*>(w13_scales);
  up.N = shape->F;
  up.K = shape->d;
  up.format = format;
  up.swiglu = true;
  up.Yq = at<uint8_t>(ws, L.act);
  up.Y_scales = at<uint8_t>(ws, L.act_scales);
  CHECK(hip_status(moe::launch_mx_gemm(up, as_stream(stream)), "expert up-projection launch"));
  moe::MxGemmProblem dn = up;
  dn.X = up.Yq;
  dn.X_scales = up.Y_scales;
  dn.W = static_cast<const uint8_t*>(w2_q);
  dn.W_scales = static_cast<const uint8_t*>(w2_scales);
  dn.N = shape->d;
  dn.K = shape->F;
  dn.swiglu = false;
  dn.Y = static_cast<moe::bf16_t*>(y_perm);
  dn.Yq = nullptr;
  dn.Y_scales = nullptr;
  CHECK(hip_status(moe::launch_mx_gemm(dn, as_stream(stream)), "expert down-projection launch"));
  return ok();
}

int moe_add_rmsnorm(int64_t rows, int32_t d, float eps, const void* x, const void* residual, const void* gamma,
                    void* h, void* y, void* y_q, void* y_scales, float* rstd, void* stream) {
  CHECK(check_norm_sizes(rows, d));
  if (!std::isfinite(eps) || eps < 0.0f) return fail(MOE_ERR_INVALID_ARG, "eps (%g) is negative or not finite", (double)eps);
  if (y_q && d % 32) return fail(MOE_ERR_UNSUPPORTED, "d (%d) %% 32 != 0 (blocks of 32 values share a scale)", d);
  if (rows == 0) return ok();
  CHECK(check_ptr(x, 16, "x"));
  CHECK(check_ptr(gamma, 16, "gamma"));
  if (residual) {
    CHECK(check_ptr(residual, 16, "residual"));
    CHECK(check_ptr(h, 16, "h"));
  } else if (h) {
    return fail(MOE_ERR_INVALID_ARG, "h is given without a residual (h would be x)");
  }
  if (!y && !y_q) return fail(MOE_ERR_INVALID_ARG, "y and y_q are both NULL");
  if (y) CHECK(check_ptr(y, 16, "y"));
  if ((y_q != nullptr) != (y_scales != nullptr))
    return fail(MOE_ERR_INVALID_ARG, "y_q and y_scales go together: %s is NULL", y_q ? "y_scales" : "y_q");
  if (y_q) {
    CHECK(check_ptr(y_q, 16, "y_q"));
    CHECK(check_ptr(y_scales, 16, "y_scales"));
  }
  if (rstd) CHECK(check_ptr(rstd, 4, "rstd"));
  moe::AddNormProblem p{};
  p.x = static_cast<const moe::bf16_t*>(x);
  p.residual = static_cast<const moe::bf16_t*>(residual);
  p.gamma = static_cast<const moe::bf16_t*>(gamma);
  p.h = static_cast<moe::bf16_t*>(h);
  p.y = static_cast<moe::bf16_t*>(y);
  p.y_q = static_cast<uint8_t*>(y_q);
  p.y_scales = static_cast<uint8_t*>(y_scales);
  p.rstd = rstd;
  p.rows = rows;
  p.d = d;
  p.eps = eps;
  CHECK(hip_status(moe::launch_add_norm(p, as_stream(stream)), "norm launch"));
  return ok();
}

size_t moe_add_rmsnorm_workspace_size(int64_t rows, int32_t d) {
  if (check_norm_sizes(rows, d) != MOE_OK) return 0;
  return norm_ws(rows, d);
}

int moe_add_rmsnorm_backward(int64_t rows, int32_t d, const void* dy, const void* dh, const void* h,
                             const void* gamma, const float* rstd, void* dx, void* dgamma, void* ws,
                             size_t ws_bytes, void* stream) {
  CHECK(check_norm_sizes(rows, d));
  CHECK(check_ptr(gamma, 16, "gamma"));
  CHECK(check_ptr(dgamma, 16, "dgamma"));
  CHECK(check_ws_bytes(norm_ws(rows, d), ws, ws_bytes));
  if (rows > 0) {
    CHECK(check_ptr(dy, 16, "dy"));
    if (dh) CHECK(check_ptr(dh, 16, "dh"));
    CHECK(check_ptr(h, 16, "h"));
    CHECK(check_ptr(rstd, 4, "rstd"));
    CHECK(check_ptr(dx, 16, "dx"));
  }
  moe::AddNormBwdProblem p{};
  p.dy = static_cast<const moe::bf16_t*>(dy);
  p.dh = static_cast<const moe::bf16_t*>(dh);
  p.h = static_cast<const moe::bf16_t*>(h);
  p.gamma = static_cast<const moe::bf16_t*>(gamma);
  p.rstd = rstd;
  p.dx = static_cast<moe::bf16_t*>(dx);
  p.dgamma = static_cast<moe::bf16_t*>(dgamma);
  p.parts = static_cast<float*>(ws);
  p.rows = rows;
  p.d = d;
  CHECK(hip_status(moe::launch_add_norm_bwd(p, as_stream(stream)), "norm backward launch"));
  return ok();
}

int moe_layer_decode(const moe_shape_t* shape, const void* x, const void* w_router, const float* bias,
                     const void* w13, const void* w13_scales, const void* w2, const void* w2_scales,
                     const void* ws13, const void* ws13_scales, const void* ws2, const void* ws2_scales,
                     void* out, void* ws, size_t ws_bytes, void* stream) {
  CHECK(check_shape(shape));
  const moe_shape_t* s = shape;
  CHECK(check_decode_shape(s));
  if (s->E_local > moe::kMaxGroups) return fail(MOE_ERR_UNSUPPORTED, "E_local (%d) > %d", s->E_local, moe::kMaxGroups);
  if (bias && s->gate != MOE_GATE_SOFTMAX)
    return fail(MOE_ERR_UNSUPPORTED, "a router bias is only defined for softmax gating");
  const bool shared = s->F_shared > 0, mx = w13_scales != nullptr;
  if ((w2_scales != nullptr) != mx || (shared && ((ws13_scales != nullptr) != mx || (ws2_scales != nullptr) != mx)))
    return fail(MOE_ERR_INVALID_ARG, "scales are given for some of the weights and not for others");
  if (mx) {
    CHECK(check_mx_shape(s));
    if (s->F_shared % 32)
      return fail(MOE_ERR_UNSUPPORTED, "F_shared (%d) %% 32 != 0 (blocks of 32 values share a scale)", s->F_shared);
    // the scales of a workgroup's weight rows lie in LDS
    if (s->d > 16384 || s->F > 32768 || s->F_shared > 32768)
      return fail(MOE_ERR_UNSUPPORTED, "d (%d) > 16384, or F (%d) or F_shared (%d) > 32768, with 4-bit weights", s->d, s->F,
                  s->F_shared);
  }
  if (s->T == 0) return ok();
  CHECK(check_ptr(x, 16, "x"));
  CHECK(check_ptr(w_router, 16, "w_router"));
  if (bias) CHECK(check_ptr(bias, 4, "bias"));
  CHECK(check_ptr(w13, 16, "w13"));
  CHECK(check_ptr(w2, 16, "w2"));
  if (shared) {
    CHECK(check_ptr(ws13, 16, "ws13"));
    CHECK(check_ptr(ws2, 16, "ws2"));
  }
  if (mx) {
    CHECK(check_ptr(w13_scales, 16, "w13_scales"));
    CHECK(check_ptr(w2_scales, 16, "w2_scales"));
    if (shared) {
      CHECK(check_ptr(ws13_scales, 16, "ws13_scales"));
      CHECK(check_ptr(ws2_scales, 16, "ws2_scales"));
    }
  }
  CHECK(check_ptr(out, 16, "out"));
  const DecodeLayout L = decode_layout(s);
  CHECK(check_ws_bytes(L.total, ws, ws_bytes));
  moe::DecodeProblem p{};
  p.x = static_cast<const moe::bf16_t*>(x);
  p.w_router = static_cast<const moe::bf16_t*>(w_router);
  p.logits = at<float>(ws, L.logits);
  p.gate.logits = p.logits;
  p.gate.nsplit = moe::decode_logits_splits(s->E, s->d);
  p.gate.split_stride = s->T * (int64_t)s->E;
  p.gate.bias = bias;
  p.gate.T = s->T;
  p.gate.E = s->E;
  p.gate.top_k = s->top_k;
  p.gate.gate = s->gate;
  p.gate.n_group = s->n_group;
  p.gate.topk_group = s->topk_group;
  p.gate.renormalize = s->renormalize;
  p.gate.group_size = s->E / s->n_group;
  p.gate.routed_scale = s->routed_scale;
  p.gate.topk_idx = at<int32_t>(ws, L.topk_idx);
  p.gate.topk_w = at<float>(ws, L.topk_w);
  p.plan = at<moe::DecodePlan>(ws, L.plan);
  p.w13 = w13;
  p.w2 = w2;
  p.ws13 = ws13;
  p.ws2 = ws2;
  p.w13_scales = static_cast<const uint8_t*>(w13_scales);
  p.w2_scales = static_cast<const uint8_t*>(w2_scales);
  p.ws13_scales = static_cast<const uint8_t*>(ws13_scales);
  p.ws2_scales = static_cast<const uint8_t*>(ws2_scales);
  p.act = at<moe::bf16_t>(ws, L.act);
  p.act_shared = at<moe::bf16_t>(ws, L.act_shared);
  p.y = at<float>(ws, L.y);
  p.out = static_cast<moe::bf16_t*>(out);
  p.T = (int32_t)s->T;
  p.d = s->d;
  p.E = s->E;
  p.top_k = s->top_k;
  p.e_begin = s->e_begin;
  p.E_local = s->E_local;
  p.F = s->F;
  p.F_shared = s->F_shared;
  p.expert_capacity = s->expert_capacity;
  CHECK(hip_status(moe::launch_decode(p, as_stream(stream)), "few-token layer launch"));
  return ok();
}

}  // extern "C"
