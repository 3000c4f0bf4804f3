// The gated delta rule's chunked kernels of bf16 rows.
#include "delta.hpp"
#include "delta_types.hpp"

namespace mmbev {

hipError_t launch_delta_walk_bf16(const DeltaArgs& a, int mode, hipStream_t st) { return delta_walk<bf16>(a, mode, st); }

hipError_t launch_delta_grad_bf16(const DeltaGradArgs& a, hipStream_t st) { return grad_of<bf16>(a, st); }

}  // namespace mmbev
