// The launches of the block's kernel files, as the C ABI calls them.
#pragma once

#include <hip/hip_runtime.h>

#include "fsa_block.h"

namespace fsa {

hipError_t norm_forward(const NormArgs&, hipStream_t);
hipError_t norm_backward(const NormArgs&, hipStream_t);

hipError_t gated_forward_f32(const GatedArgs&, hipStream_t);
hipError_t gated_forward_bf16(const GatedArgs&, hipStream_t);
hipError_t gated_forward_f16(const GatedArgs&, hipStream_t);
hipError_t gated_backward_f32(const GatedArgs&, hipStream_t);
hipError_t gated_backward_bf16(const GatedArgs&, hipStream_t);
hipError_t gated_backward_f16(const GatedArgs&, hipStream_t);

hipError_t orthogonalize(const OrthoArgs&, hipStream_t);

}  // namespace fsa
