// The chunked attention kernels of bf16 rows.
#include "attention.hpp"
#include "attention_types.hpp"

namespace mmbev {

hipError_t launch_attention_bf16(const AttnArgs& a, bool state_only, hipStream_t st) {
  return attention_of<bf16>(a, state_only, st);
}

}  // namespace mmbev
