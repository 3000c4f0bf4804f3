// The gated delta rule's chunked kernels of fp16 rows.
#include "delta.hpp"
#include "delta_types.hpp"

namespace mmbev {

hipError_t launch_delta_walk_f16(const DeltaArgs& a, int mode, hipStream_t st) { return delta_walk<f16>(a, mode, st); }

hipError_t launch_delta_grad_f16(const DeltaGradArgs& a, hipStream_t st) { return grad_of<f16>(a, st); }

}  // namespace mmbev
