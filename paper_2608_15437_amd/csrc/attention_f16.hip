// The chunked attention kernels of f16 rows.
#include "attention.hpp"
#include "attention_types.hpp"

namespace mmbev {

hipError_t launch_attention_states_f16(const AttnPair& p, hipStream_t st) { return states_of<f16>(p, st); }

hipError_t launch_attention_f16(const AttnArgs& a, hipStream_t st) { return walk_of<f16>(a, st); }

hipError_t launch_attention_backward_f16(const AttnArgs& a, const AttnGradArgs& b, hipStream_t st) { return backward_of<f16>(a, b, st); }

}  // namespace mmbev
