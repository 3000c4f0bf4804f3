// The chunked attention kernels of f32 rows.
#include "attention.hpp"
#include "attention_types.hpp"

namespace mmbev {

hipError_t launch_attention_f32(const AttnArgs& a, bool state_only, hipStream_t st) { return walk_of<float>(a, state_only, st); }

hipError_t launch_attention_grad_f32(const AttnGradArgs& a, hipStream_t st) { return grad_of<float>(a, st); }

}  // namespace mmbev
