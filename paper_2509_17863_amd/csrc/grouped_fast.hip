// Grouped products on large tiles (grouped_pp.h): forward, both gradients, and the forward
// in 8-bit integers.
#include "grouped_pp.h"

namespace eaas {

template <int DIR, bool I8>
hipError_t launch_grouped_pp(const GroupedParams& p, long long tiles, hipStream_t stream) {
  return launch_pp<DIR, I8, kPlain>(p, tiles, stream);
}

template hipError_t launch_grouped_pp<kForward, false>(const GroupedParams&, long long, hipStream_t);
template hipError_t launch_grouped_pp<kForward, true>(const GroupedParams&, long long, hipStream_t);
template hipError_t launch_grouped_pp<kGradRows, false>(const GroupedParams&, long long, hipStream_t);
template hipError_t launch_grouped_pp<kGradWeights, false>(const GroupedParams&, long long, hipStream_t);

}  // namespace eaas
