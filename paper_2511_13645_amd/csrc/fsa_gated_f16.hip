// The gated feed-forward block on fp16.
#define FSA_GATED_KIND 2
#include "fsa_gated_kernels.hip.h"

namespace fsa {
hipError_t gated_forward_f16(const GatedArgs& a, hipStream_t stream) { return forward(a, stream); }
hipError_t gated_backward_f16(const GatedArgs& a, hipStream_t stream) { return backward(a, stream); }
}  // namespace fsa
