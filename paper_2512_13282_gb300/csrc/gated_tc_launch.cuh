// gated_tc_launch.cuh -- launch of one instantiation of the gated feed-forward
// block's tensor-core kernel (included by the instantiation translation units).
#pragma once
#include "gated_tc.cuh"

namespace gb300 {

template <int BN, bool PAIR, bool KM, bool BWD>
cudaError_t launch_gated_kernel(const GatedMaps &m, const GatedTcParams &p, int grid, cudaStream_t st) {
  using Cfg = GatedCfg<BN, PAIR, BWD>;
  auto kern = gated_tc_kernel<BN, PAIR, KM, BWD>;
  static std::atomic<uint64_t> allowed{0};
  const cudaError_t e = allow_shared_memory((const void *)kern, Cfg::kSmemBytes, allowed);
  if (e != cudaSuccess) return e;
  return launch_ex(kern, dim3((unsigned)grid), dim3(Cfg::kThreads), Cfg::kSmemBytes, st, PAIR ? 2 : 1, m.a, m.b[0],
                   m.b[1], p);
}

}  // namespace gb300
