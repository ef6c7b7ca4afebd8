// Host-side checks of the operators around the layer, built with AddressSanitizer and
// UndefinedBehaviorSanitizer: valid calls over the stated limits, whose launches are recorded here
// and "fail", so that every call runs its whole setup.  Each problem is looked over for regions
// that leave the workspace, overlap, or are not aligned.  Prints one line per failed check and
// "ALL OK" when none failed.
#include <stdint.h>
#include <stdio.h>
#include <string.h>

#include <hip/hip_runtime_api.h>

#include "../../include/moe.h"
#include "../../paper_2607_18631_amd/csrc/kernels.hpp"

static int g_fail = 0, g_calls = 0;
static moe::MxGemmProblem g_gemm[2];
static moe::DecodeProblem g_decode;
static moe::AddNormBwdProblem g_norm_bwd;
static hipError_t g_result = hipSuccess;

namespace moe {
hipError_t launch_mx_quantize(const MxConvertProblem&, hipStream_t) { return ++g_calls, g_result; }
hipError_t launch_mx_dequantize(const MxConvertProblem&, hipStream_t) { return ++g_calls, g_result; }
hipError_t launch_mx_gemm(const MxGemmProblem& p, hipStream_t) { return g_gemm[g_calls++ & 1] = p, g_result; }
hipError_t launch_add_norm(const AddNormProblem&, hipStream_t) { return ++g_calls, g_result; }
hipError_t launch_add_norm_bwd(const AddNormBwdProblem& p, hipStream_t) { return ++g_calls, g_norm_bwd = p, g_result; }
hipError_t launch_decode(const DecodeProblem& p, hipStream_t) { return ++g_calls, g_decode = p, g_result; }
}  // namespace moe

#define EXPECT(cond, ...)                         \
  do {                                            \
    if (!(cond)) {                                \
      ++g_fail;                                   \
      printf("FAIL line %d: ", __LINE__);         \
      printf(__VA_ARGS__);                        \
      printf(" [%s]\n", moe_last_error());        \
    }                                             \
  } while (0)

static char* const WS = reinterpret_cast<char*>(0x10000000);
static void* const FAKE = reinterpret_cast<void*>(0x100000);

struct Regions {
  const char* what;
  uint64_t at, total;
  void next(const void* p, uint64_t bytes, uint64_t align) {      // regions in the order of the layout
    const uint64_t a = (uint64_t)((const char*)p - WS);
    EXPECT(a % align == 0 && a >= at && a + bytes <= total, "%s: region %llu + %llu, before it %llu, total %llu", what,
           (unsigned long long)a, (unsigned long long)bytes, (unsigned long long)at, (unsigned long long)total);
    at = a + bytes;
  }
};

static moe_shape_t shape(int64_t T, int d, int E, int k, int F, int Fs, int cap = 0) {
  moe_shape_t s;
  memset(&s, 0, sizeof s);
  s.T = T; s.d = d; s.E = E; s.top_k = k; s.E_local = E; s.F = F; s.F_shared = Fs; s.expert_capacity = cap;
  s.n_group = 1; s.topk_group = 1; s.renormalize = 1; s.routed_scale = 1.0f;
  return s;
}

static void mlp(moe_shape_t s, int format) {
  const uint64_t total = moe_workspace_size(&s, MOE_WS_MX_FFN);
  EXPECT(total > 0, "workspace size");
  g_calls = 0;
  const int st = moe_mx_grouped_ffn(&s, format, FAKE, FAKE, (const int32_t*)FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, WS, total,
                                    nullptr);
  EXPECT(st == MOE_OK && g_calls == 2, "status %d, launches %d", st, g_calls);
  const uint64_t cap = (uint64_t)g_gemm[0].max_rows;
  Regions r{"mlp", 0, total};
  r.next(g_gemm[0].Yq, cap * s.F, 16);
  r.next(g_gemm[0].Y_scales, cap * (s.F / 32), 16);
  EXPECT(g_gemm[1].X == g_gemm[0].Yq && g_gemm[1].X_scales == g_gemm[0].Y_scales, "the activation is the next product's rows");
  EXPECT(g_gemm[1].N == s.d && g_gemm[1].K == s.F && g_gemm[0].N == s.F && g_gemm[0].K == s.d, "sizes");
  EXPECT(moe_mx_grouped_ffn(&s, format, FAKE, FAKE, (const int32_t*)FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, WS, total - 1,
                            nullptr) == MOE_ERR_WORKSPACE, "a byte less");
}

static void decode(moe_shape_t s, bool mx) {
  const uint64_t total = moe_workspace_size(&s, MOE_WS_DECODE);
  EXPECT(total > 0, "workspace size");
  g_calls = 0;
  void *sc = mx ? FAKE : nullptr, *sh = s.F_shared ? FAKE : nullptr, *shsc = s.F_shared ? sc : nullptr;
  const int st = moe_layer_decode(&s, FAKE, FAKE, (const float*)FAKE, FAKE, sc, FAKE, sc, sh, shsc, sh, shsc, FAKE, WS, total,
                                  nullptr);
  EXPECT(st == MOE_OK && g_calls == 1, "status %d, launches %d", st, g_calls);
  const moe::DecodeProblem& p = g_decode;
  const uint64_t slots = (uint64_t)s.T * s.top_k;
  // the regions in any order: none may reach into another
  struct { const void* at; uint64_t bytes; } all[] = {
      {p.gate.topk_idx, slots * 4}, {p.gate.topk_w, slots * 4},
      {p.logits, (uint64_t)moe::decode_logits_splits(s.E, s.d) * s.T * s.E * 4}, {p.plan, sizeof(moe::DecodePlan)},
      {p.act, slots * s.F * 2}, {p.act_shared, (uint64_t)s.T * s.F_shared * 2},
      {p.y, (slots + (s.F_shared ? s.T : 0)) * s.d * 4}};
  for (auto& a : all) {
    const uint64_t at = (uint64_t)((const char*)a.at - WS);
    EXPECT(at % 16 == 0 && at + a.bytes <= total, "a region at %llu of %llu bytes leaves %llu", (unsigned long long)at,
           (unsigned long long)a.bytes, (unsigned long long)total);
    for (auto& b : all) {
      const uint64_t bt = (uint64_t)((const char*)b.at - WS);
      EXPECT(&a == &b || !a.bytes || !b.bytes || at + a.bytes <= bt || bt + b.bytes <= at, "regions at %llu and %llu overlap",
             (unsigned long long)at, (unsigned long long)bt);
    }
  }
  // the plan has room for every slot, and for every block of 16 rows however the tokens choose
  EXPECT(slots <= sizeof(p.plan->slot) / sizeof(p.plan->slot[0]), "slots");
  EXPECT((uint64_t)moe::decode_entries((int)s.T, s.top_k, s.E_local) <= sizeof(p.plan->entry) / sizeof(p.plan->entry[0]),
         "entries");
}

int main() {
  for (int format = 0; format < 2; ++format) {
    mlp(shape(1, 32, 1, 1, 32, 0), format);
    mlp(shape(8192, 7168, 32, 1, 2048, 0), format);
    mlp(shape(1000000, 32, 1024, 16, 32, 0), format);
    mlp(shape(7, (1 << 20) - 32, 4, 2, 32, 0), format);
    mlp(shape(7, 32, 4, 2, (1 << 20) - 32, 0), format);
    mlp(shape(300, 64, 8, 2, 96, 0, 5), format);
  }
  const int T[] = {1, 2, 15, 16, 17, 63, 64};
  for (int t : T)
    for (int mx = 0; mx < 2; ++mx) {
      decode(shape(t, 32, 1, 1, 32, 0), mx);
      decode(shape(t, 7168, 384, 8, 2048, 2048), mx);
      decode(shape(t, 16384, 1024, 16, 32768, 32768), mx);
      decode(shape(t, 64, 24, 5, 96, 0, 3), mx);
      if (!mx) decode(shape(t, (1 << 20) - 8, 16, 2, (1 << 20) - 8, 8), false);
    }
  // more blocks of 16 rows than any way to choose needs
  for (int t = 1; t <= 64; ++t)
    for (int k = 1; k <= 16; ++k)
      for (int e = k; e <= 40; ++e) {
        // the most: a row for every expert as far as the slots go, then 16 more rows for each further block, of
        // which an expert has as many as the tokens allow (each token chooses it once)
        const int first = e < t * k ? e : t * k, more = (t * k - first) / 16, room = first * ((t - 1) / 16);
        const int blocks = first + (more < room ? more : room);
        EXPECT(blocks <= moe::decode_entries(t, k, e), "T %d, top_k %d, %d experts: %d blocks", t, k, e, blocks);
      }
  // norm
  const int64_t rows[] = {0, 1, 3, 255, 4096, 1 << 20, (int64_t(1) << 31) - 1};
  const int ds[] = {8, 32, 2048, 7168, 16384, 65536};
  for (int64_t n : rows)
    for (int d : ds) {
      const uint64_t total = moe_add_rmsnorm_workspace_size(n, d);
      EXPECT(moe_add_rmsnorm_backward(n, d, FAKE, FAKE, FAKE, FAKE, (const float*)FAKE, FAKE, FAKE, WS, total, nullptr) == MOE_OK,
             "norm backward %lld %d", (long long)n, d);
      EXPECT((uint64_t)moe::add_norm_bwd_parts(n, d) * d * 4 <= total && (char*)g_norm_bwd.parts == WS, "partial sums");
      EXPECT(moe_add_rmsnorm(n, d, 1e-6f, FAKE, FAKE, FAKE, FAKE, FAKE, d % 32 ? nullptr : FAKE, d % 32 ? nullptr : FAKE,
                             (float*)FAKE, nullptr) == MOE_OK, "norm %lld %d", (long long)n, d);
    }
  // a launch that fails is reported
  g_result = hipErrorNotSupported;
  moe_shape_t s = shape(8, 64, 8, 2, 96, 0);
  EXPECT(moe_mx_grouped_ffn(&s, 0, FAKE, FAKE, (const int32_t*)FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, WS, 1 << 30, nullptr) == MOE_ERR_HIP &&
             strstr(moe_last_error(), "stub launch"), "mlp launch failure");
  EXPECT(moe_mx_quantize(1, 32, 0, FAKE, FAKE, FAKE, nullptr) == MOE_ERR_HIP, "conversion launch failure");
  EXPECT(moe_mx_dequantize(1, 32, 0, FAKE, FAKE, FAKE, nullptr) == MOE_ERR_HIP, "conversion launch failure");
  if (!g_fail) printf("ALL OK\n");
  return g_fail != 0;
}
