// The chunked attention kernels of f32 rows.
#include "attention.hpp"
#include "attention_types.hpp"

namespace mmbev {

hipError_t launch_attention_f32(const AttnArgs& a, bool state_only, hipStream_t st) {
  return attention_of<float>(a, state_only, st);
}

}  // namespace mmbev
