// Gating and top-k: one wavefront per token (gate_device.hpp).
#include "common.hpp"
#include "gate_device.hpp"
#include "kernels.hpp"

namespace moe {
namespace {

constexpr int kMaxPerLane = 16;   // E <= 1024
constexpr int kWaves = 4;         // tokens per workgroup

template <int PL>
__global__ __launch_bounds__(64 * kWaves) void k_gate(GateProblem p) {
  __shared__ float s_key[kWaves][64 * PL];
  __shared__ float s_gscore[kWaves][64];
  const int w = threadIdx.x >> 6;
  const int64_t t = (int64_t)blockIdx.x * kWaves + w;
  if (t >= p.T) return;                                   // wave-uniform
  gate_token<PL>(p, t, s_key[w], s_gscore[w]);
}

template <int PL>
hipError_t launch_pl(const GateProblem& p, hipStream_t stream) {
  const unsigned blocks = (unsigned)((p.T + kWaves - 1) / kWaves);
  hipLaunchKernelGGL(k_gate<PL>, dim3(blocks), dim3(64 * kWaves), 0, stream, p);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_gate(const GateProblem& p, hipStream_t stream) {
  if (p.nsplit < 1) return hipErrorInvalidValue;
  const int pl = (p.E + 63) / 64;
  if (pl <= 1) return launch_pl<1>(p, stream);
  if (pl <= 2) return launch_pl<2>(p, stream);
  if (pl <= 4) return launch_pl<4>(p, stream);
  if (pl <= 8) return launch_pl<8>(p, stream);
  if (pl <= kMaxPerLane) return launch_pl<16>(p, stream);
  return hipErrorInvalidValue;
}

}  // namespace moe
