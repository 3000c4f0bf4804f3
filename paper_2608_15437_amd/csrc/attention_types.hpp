// The chunked attention kernels' launchers, one translation unit a type.
#pragma once

#include "sequence.hpp"

namespace mmbev {

hipError_t launch_attention_states_f32(const AttnPair& p, hipStream_t st);
hipError_t launch_attention_f32(const AttnArgs& a, hipStream_t st);
hipError_t launch_attention_backward_f32(const AttnArgs& a, const AttnGradArgs& b, hipStream_t st);
hipError_t launch_attention_states_f16(const AttnPair& p, hipStream_t st);
hipError_t launch_attention_f16(const AttnArgs& a, hipStream_t st);
hipError_t launch_attention_backward_f16(const AttnArgs& a, const AttnGradArgs& b, hipStream_t st);
hipError_t launch_attention_states_bf16(const AttnPair& p, hipStream_t st);
hipError_t launch_attention_bf16(const AttnArgs& a, hipStream_t st);
hipError_t launch_attention_backward_bf16(const AttnArgs& a, const AttnGradArgs& b, hipStream_t st);

}  // namespace mmbev
