// The gated delta rule's chunked kernels of fp32 rows.
#include "delta.hpp"
#include "delta_types.hpp"

namespace mmbev {

hipError_t launch_delta_walk_f32(const DeltaArgs& a, int mode, hipStream_t st) { return delta_walk<float>(a, mode, st); }

hipError_t launch_delta_grad_f32(const DeltaGradArgs& a, hipStream_t st) { return grad_of<float>(a, st); }

}  // namespace mmbev
