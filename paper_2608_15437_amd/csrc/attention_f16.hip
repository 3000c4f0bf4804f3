// The chunked attention kernels of f16 rows.
#include "attention.hpp"
#include "attention_types.hpp"

namespace mmbev {

hipError_t launch_attention_f16(const AttnArgs& a, bool state_only, hipStream_t st) { return walk_of<f16>(a, state_only, st); }

hipError_t launch_attention_grad_f16(const AttnGradArgs& a, hipStream_t st) { return grad_of<f16>(a, st); }

}  // namespace mmbev
