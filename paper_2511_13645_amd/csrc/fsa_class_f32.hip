// Class losses on fp32 tables.
#define FSA_CLASS_KIND 0
#include "fsa_class_kernels.hip.h"

namespace fsa {
hipError_t class_forward_f32(const ClassArgs& a, hipStream_t stream) { return forward(a, stream); }
hipError_t class_gradient_f32(const ClassArgs& a, hipStream_t stream) { return gradient(a, stream); }
}  // namespace fsa
