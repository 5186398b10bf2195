// Differential attention (gfx950) of f16 activations.
#include "pam_attn_kernels.h"

namespace pam {

hipError_t attn_fwd_f16(const AttnArgs &a, bool wide, bool few, hipStream_t s)
{
    return attn_fwd<f16>(a, wide, few, s);
}
hipError_t attn_bwd_f16(const AttnArgs &a, bool wide, hipStream_t s) { return attn_bwd<f16>(a, wide, s); }

}  // namespace pam
