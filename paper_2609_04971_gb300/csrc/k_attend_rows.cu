// The attention kernel for many query rows (k_attend_rows.cuh).
#include "k_attend_rows.cuh"

namespace bkv {

cudaError_t launch_attend_rows(int d, const AtPlan& p, const CUtensorMap& qmap, const CUtensorMap& kmap,
                               const CUtensorMap& vmap, const AtKernelArgs& a, cudaStream_t st) {
  const RestMap<false> none;
  return d == 128 ? launch<128, false>(p, qmap, kmap, vmap, none, a, st)
                  : launch<64, false>(p, qmap, kmap, vmap, none, a, st);
}

}  // namespace bkv
