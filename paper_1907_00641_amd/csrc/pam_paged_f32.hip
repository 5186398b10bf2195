// Attention over a paged cache (gfx950) for f32 queries.
#include "pam_paged_kernels.h"

namespace pam {

hipError_t paged_f32(const PagedArgs &a, int store, int piece, hipStream_t s)
{
    return paged_type<float>(a, store, piece, s);
}

}  // namespace pam
