// The grouped products with an epilogue on large tiles (grouped_pp.h).
#include "grouped_pp.h"

namespace eaas {

hipError_t launch_grouped_swiglu_pp(const GroupedParams& p, long long tiles, hipStream_t stream) {
  return launch_pp<kForward, false, kSwiglu>(p, tiles, stream);
}

hipError_t launch_grouped_swiglu_grad_pp(const GroupedParams& p, long long tiles,
                                         hipStream_t stream) {
  return launch_pp<kGradRows, false, kSwigluGrad>(p, tiles, stream);
}

}  // namespace eaas
