// The chunked attention kernels' launchers, one translation unit a type.
#pragma once

#include "sequence.hpp"

namespace mmbev {

hipError_t launch_attention_f32(const AttnArgs& a, bool state_only, hipStream_t st);
hipError_t launch_attention_grad_f32(const AttnGradArgs& a, hipStream_t st);
hipError_t launch_attention_f16(const AttnArgs& a, bool state_only, hipStream_t st);
hipError_t launch_attention_grad_f16(const AttnGradArgs& a, hipStream_t st);
hipError_t launch_attention_bf16(const AttnArgs& a, bool state_only, hipStream_t st);
hipError_t launch_attention_grad_bf16(const AttnGradArgs& a, hipStream_t st);

}  // namespace mmbev
