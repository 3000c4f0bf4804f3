// The chunked attention kernels of f16 rows.
#include "attention.hpp"
#include "attention_types.hpp"

namespace mmbev {

hipError_t launch_attention_f16(const AttnArgs& a, bool state_only, hipStream_t st) {
  return attention_of<f16>(a, state_only, st);
}

}  // namespace mmbev
