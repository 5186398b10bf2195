// Attention over a paged cache (gfx950) for f16 queries.
#include "pam_paged_kernels.h"

namespace pam {

hipError_t paged_f16(const PagedArgs &a, int store, int piece, hipStream_t s)
{
    return paged_type<f16>(a, store, piece, s);
}

}  // namespace pam
