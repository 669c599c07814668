// paged_prompt.hip — attention of many new tokens over all their pages.
#include "paged_prompt.h"

namespace qkv {

hipError_t launch_paged_prompt(const PagedPromptArgs& a, uint32_t head_dim, bool bf16, hipStream_t stream) {
  return bf16 ? launch_prompt_type<BFloat, false>(a, head_dim, stream) : launch_prompt_type<Half, false>(a, head_dim, stream);
}

}  // namespace qkv
