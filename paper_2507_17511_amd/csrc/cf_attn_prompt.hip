// Whole prompts of head_dim 64 and 128: two waves a SIMD, of 256 vector registers each.  Compiled with the results of matrix instructions
// in these (build.py): scores need not be moved before they are used.  16384 x 24 heads of zeros 2270 -> 2100 us, 4096 x 24 heads 218 -> 207.
#include "cf_attn_prompt.h"

namespace cf {
namespace attn {

hipError_t launch_prompt256(const PromptArgs &a, hipStream_t s);

hipError_t launch_prompt(const PromptArgs &a, hipStream_t s)
{
    if (a.h.head_dim == 256) return launch_prompt256(a, s);
    if (a.h.dtype == BF16) return a.h.head_dim == 64 ? prompt_dim<BF16, 64>(a, s) : prompt_dim<BF16, 128>(a, s);
    return a.h.head_dim == 64 ? prompt_dim<F16, 64>(a, s) : prompt_dim<F16, 128>(a, s);
}

}  // namespace attn
}  // namespace cf
