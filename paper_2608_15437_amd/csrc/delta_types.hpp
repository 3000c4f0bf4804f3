// The gated delta rule's chunked kernels' launchers, one translation unit a
// type.
#pragma once

#include "sequence.hpp"

namespace mmbev {

// mode: DeltaMode
hipError_t launch_delta_walk_f32(const DeltaArgs& a, int mode, hipStream_t st);
hipError_t launch_delta_grad_f32(const DeltaGradArgs& a, hipStream_t st);
hipError_t launch_delta_walk_f16(const DeltaArgs& a, int mode, hipStream_t st);
hipError_t launch_delta_grad_f16(const DeltaGradArgs& a, hipStream_t st);
hipError_t launch_delta_walk_bf16(const DeltaArgs& a, int mode, hipStream_t st);
hipError_t launch_delta_grad_bf16(const DeltaGradArgs& a, hipStream_t st);

}  // namespace mmbev
