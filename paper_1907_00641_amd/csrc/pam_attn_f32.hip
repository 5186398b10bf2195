// Differential attention (gfx950) of f32 activations.
#include "pam_attn_kernels.h"

namespace pam {

hipError_t attn_fwd_f32(const AttnArgs &a, bool wide, bool few, hipStream_t s)
{
    return attn_fwd<float>(a, wide, few, s);
}
hipError_t attn_bwd_f32(const AttnArgs &a, bool wide, hipStream_t s) { return attn_bwd<float>(a, wide, s); }

}  // namespace pam
