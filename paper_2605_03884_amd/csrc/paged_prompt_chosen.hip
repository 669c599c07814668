// paged_prompt_chosen.hip — attention of many new tokens over the pages chosen for each.
#include "paged_prompt.h"

namespace qkv {

hipError_t launch_paged_prompt_chosen(const PagedPromptArgs& a, uint32_t head_dim, bool bf16, hipStream_t stream) {
  return bf16 ? launch_prompt_type<BFloat, true>(a, head_dim, stream) : launch_prompt_type<Half, true>(a, head_dim, stream);
}

}  // namespace qkv
