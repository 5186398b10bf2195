// Attention over packed sequences (gfx950) of f16 activations.
#include "pam_packed_kernels.h"

namespace pam {

hipError_t packed_fwd_f16(const PackedArgs &a, hipStream_t s) { return packed_fwd<f16>(a, s); }
hipError_t packed_bwd_f16(const PackedArgs &a, hipStream_t s) { return packed_bwd<f16>(a, s); }

}  // namespace pam
