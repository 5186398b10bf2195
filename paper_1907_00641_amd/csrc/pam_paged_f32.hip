// Attention over a paged cache (gfx950) for f32 queries.
#include "pam_paged_kernels.h"

namespace pam {

hipError_t paged_f32(const PagedArgs &a, int store, bool wide, hipStream_t s) { return paged_type<float>(a, store, wide, s); }

}  // namespace pam
