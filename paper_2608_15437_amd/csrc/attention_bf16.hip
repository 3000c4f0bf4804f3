// The chunked attention kernels of bf16 rows.
#include "attention.hpp"
#include "attention_types.hpp"

namespace mmbev {

hipError_t launch_attention_states_bf16(const AttnPair& p, hipStream_t st) { return states_of<bf16>(p, st); }

hipError_t launch_attention_bf16(const AttnArgs& a, hipStream_t st) { return walk_of<bf16>(a, st); }

hipError_t launch_attention_backward_bf16(const AttnArgs& a, const AttnGradArgs& b, hipStream_t st) { return backward_of<bf16>(a, b, st); }

}  // namespace mmbev
