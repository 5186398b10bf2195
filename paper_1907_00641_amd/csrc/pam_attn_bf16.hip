// Differential attention (gfx950) of bf16 activations.
#include "pam_attn_kernels.h"

namespace pam {

hipError_t attn_fwd_bf16(const AttnArgs &a, bool wide, bool few, hipStream_t s)
{
    return attn_fwd<bf16>(a, wide, few, s);
}
hipError_t attn_bwd_bf16(const AttnArgs &a, bool wide, hipStream_t s) { return attn_bwd<bf16>(a, wide, s); }

}  // namespace pam
