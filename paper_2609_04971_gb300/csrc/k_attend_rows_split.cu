// The attention kernel for many query rows (k_attend_rows.cuh) over fp16 numbers, the keys in two terms: 4-bit caches
// that were unpacked for it.
#include "k_attend_rows.cuh"

namespace bkv {

cudaError_t launch_attend_rows_split(int d, const AtPlan& p, const CUtensorMap& qmap, const CUtensorMap& kmap,
                                     const CUtensorMap& restmap, const CUtensorMap& vmap, const AtKernelArgs& a,
                                     cudaStream_t st) {
  const RestMap<true> rest{restmap};
  return d == 128 ? launch<128, false>(p, qmap, kmap, vmap, rest, a, st)
                  : launch<64, false>(p, qmap, kmap, vmap, rest, a, st);
}

}  // namespace bkv
