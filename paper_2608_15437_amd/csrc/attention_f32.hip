// The chunked attention kernels of f32 rows.
#include "attention.hpp"
#include "attention_types.hpp"

namespace mmbev {

hipError_t launch_attention_states_f32(const AttnPair& p, hipStream_t st) { return states_of<float>(p, st); }

hipError_t launch_attention_f32(const AttnArgs& a, hipStream_t st) { return walk_of<float>(a, st); }

hipError_t launch_attention_backward_f32(const AttnArgs& a, const AttnGradArgs& b, hipStream_t st) { return backward_of<float>(a, b, st); }

}  // namespace mmbev
