// Attention over packed sequences (gfx950) of f32 activations.
#include "pam_packed_kernels.h"

namespace pam {

hipError_t packed_fwd_f32(const PackedArgs &a, hipStream_t s) { return packed_fwd<float>(a, s); }
hipError_t packed_bwd_f32(const PackedArgs &a, hipStream_t s) { return packed_bwd<float>(a, s); }

}  // namespace pam
