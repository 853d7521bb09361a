// gated_tc_fwd.cu -- the forward instantiations of the gated feed-forward
// block's tensor-core kernel.
#include "gated_tc_launch.cuh"

namespace gb300 {

cudaError_t launch_gated_tc_fwd(const GatedTile &tile, bool km, const GatedMaps &m, const GatedTcParams &p, int grid,
                                cudaStream_t st) {
  if (tile.pair)
    return km ? launch_gated_kernel<256, true, true, false>(m, p, grid, st)
              : launch_gated_kernel<256, true, false, false>(m, p, grid, st);
  return km ? launch_gated_kernel<128, false, true, false>(m, p, grid, st)
            : launch_gated_kernel<128, false, false, false>(m, p, grid, st);
}

}  // namespace gb300
