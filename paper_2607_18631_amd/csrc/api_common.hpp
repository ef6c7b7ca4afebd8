// Host helpers shared by the C ABI's entry points: errors, argument checks, workspace layouts.
#pragma once
#include <hip/hip_runtime_api.h>
#include <stddef.h>
#include <stdint.h>

#include "../../include/moe.h"
#include "kernels.hpp"

namespace moe {
namespace abi {

// sets the thread's message and returns `status`
int fail(int status, const char* fmt, ...);
// clears the thread's message
int ok();

constexpr size_t kAlign = 256;
inline size_t align_up(size_t v) { return (v + kAlign - 1) / kAlign * kAlign; }

// rows of the expert-ordered buffers
int64_t capacity(const moe_shape_t* s);
int check_shape(const moe_shape_t* s);
int check_ptr(const void* p, size_t align, const char* name);
// a workspace of `need` bytes (0: none is needed)
int check_ws_bytes(size_t need, const void* ws, size_t ws_bytes);
int hip_status(hipError_t e, const char* what);

// the further limits of the block-scaled expert MLP and of the few-token layer
inline int check_mx_shape(const moe_shape_t* s) {
  if (s->d % 32) return fail(MOE_ERR_UNSUPPORTED, "d (%d) %% 32 != 0 (blocks of 32 values share a scale)", s->d);
  if (s->F % 32) return fail(MOE_ERR_UNSUPPORTED, "F (%d) %% 32 != 0 (blocks of 32 values share a scale)", s->F);
  return MOE_OK;
}
inline int check_decode_shape(const moe_shape_t* s) {
  if (s->T > MOE_DECODE_MAX_TOKENS)
    return fail(MOE_ERR_UNSUPPORTED, "T (%lld) > %d (MOE_DECODE_MAX_TOKENS)", (long long)s->T, MOE_DECODE_MAX_TOKENS);
  // 32-bit byte offsets into 16 weight rows and into the activations of every slot
  const int32_t widest = s->d > s->F ? (s->d > s->F_shared ? s->d : s->F_shared) : (s->F > s->F_shared ? s->F : s->F_shared);
  if (widest >= (1 << 20)) return fail(MOE_ERR_UNSUPPORTED, "d, F or F_shared (%d) >= 2^20", widest);
  // a launch has less than 2^32 threads: 256 for 64 features of each entry of the plan where there are so many, and for 32
  // of 16 tokens of the shared expert
  const int64_t features = s->d > s->F ? s->d : s->F, shared = s->F_shared > s->d ? s->F_shared : s->d;
  const int64_t blocks = decode_entries((int)s->T, s->top_k, s->E_local) * ((features + 63) / 64) +
                         (s->F_shared > 0 ? (s->T + 15) / 16 * ((shared + 31) / 32) : 0);
  if (blocks >= (int64_t(1) << 24))
    return fail(MOE_ERR_UNSUPPORTED, "d or F (%lld) makes 2^24 workgroups or more (%lld) of %d experts' rows",
                (long long)features, (long long)blocks, decode_entries((int)s->T, s->top_k, s->E_local));
  return MOE_OK;
}

// MOE_WS_MX_FFN: the activation's elements (room for 8-bit ones) and scales
struct MxFfnLayout {
  size_t act, act_scales, total;
};
inline MxFfnLayout mx_ffn_layout(const moe_shape_t* s) {
  MxFfnLayout L{};
  L.act_scales = align_up((size_t)capacity(s) * s->F);
  L.total = L.act_scales + align_up((size_t)capacity(s) * (s->F / 32));
  return L;
}

// MOE_WS_DECODE: the routing first, at the same offsets as in a MOE_WS_LAYER workspace
struct DecodeLayout {
  size_t topk_idx, topk_w, logits, plan, act, act_shared, y, total;
};
inline DecodeLayout decode_layout(const moe_shape_t* s) {
  DecodeLayout L{};
  const size_t T = (size_t)s->T, k = (size_t)s->top_k;
  size_t off = 0;
  auto take = [&](size_t bytes) {
    size_t o = off;
    off += align_up(bytes);
    return o;
  };
  L.topk_idx = take(T * k * 4);
  L.topk_w = take(T * k * 4);
  L.logits = take((size_t)decode_logits_splits(s->E, s->d) * T * s->E * sizeof(float));
  L.plan = take(sizeof(DecodePlan));
  L.act = take(T * k * (size_t)s->F * 2);
  L.act_shared = take(T * (size_t)s->F_shared * 2);
  L.y = take((T * k + (s->F_shared > 0 ? T : 0)) * (size_t)s->d * sizeof(float));
  L.total = off;
  return L;
}

inline hipStream_t as_stream(void* s) { return reinterpret_cast<hipStream_t>(s); }
template <class T>
inline T* at(void* base, size_t off) { return reinterpret_cast<T*>(static_cast<char*>(base) + off); }

#define CHECK(expr)          \
  do {                       \
    int _st = (expr);        \
    if (_st != MOE_OK) return _st; \
  } while (0)

}  // namespace abi
}  // namespace moe
