// The attention kernel (k_attend_tiles.cuh) for head_dim 128.
#include "k_attend_tiles.cuh"

namespace bkv {

cudaError_t launch_attend_tiles_128(const AtPlan& p, const CUtensorMap& qmap, const CUtensorMap& kmap,
                                   const CUtensorMap& vmap, const AtKernelArgs& a, cudaStream_t st) {
  return launch_attend_tiles_d<128, false>(p, qmap, kmap, vmap, {}, a, st);
}

}  // namespace bkv
