// Whole prompts of head_dim 256: one wave a SIMD, its accumulators in the 256 registers that only matrix instructions reach (with the flags of
// cf_attn_prompt.hip 357 us for 2 x 333 tokens over 20333 keys, like this 296).
#include "cf_attn_prompt.h"

namespace cf {
namespace attn {

hipError_t launch_prompt256(const PromptArgs &a, hipStream_t s) { return a.h.dtype == BF16 ? prompt_dim<BF16, 256>(a, s) : prompt_dim<F16, 256>(a, s); }

}  // namespace attn
}  // namespace cf
