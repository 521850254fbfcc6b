// The attention kernel with a window (k_attend_tiles.cuh) for head_dim 128.
#include "k_attend_tiles.cuh"

namespace bkv {

cudaError_t launch_attend_window_128(const AtPlan& p, const CUtensorMap& qmap, const CUtensorMap& kmap,
                                    const CUtensorMap& vmap, const AtSinkMaps<true>& sink, const AtKernelArgs& a,
                                    cudaStream_t st) {
  return launch_attend_tiles_d<128, true>(p, qmap, kmap, vmap, sink, a, st);
}

}  // namespace bkv
