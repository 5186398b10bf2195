// Attention over packed sequences (gfx950) of bf16 activations.
#include "pam_packed_kernels.h"

namespace pam {

hipError_t packed_fwd_bf16(const PackedArgs &a, hipStream_t s) { return packed_fwd<bf16>(a, s); }
hipError_t packed_bwd_bf16(const PackedArgs &a, hipStream_t s) { return packed_bwd<bf16>(a, s); }

}  // namespace pam
