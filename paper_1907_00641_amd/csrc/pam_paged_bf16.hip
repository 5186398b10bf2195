// Attention over a paged cache (gfx950) for bf16 queries.
#include "pam_paged_kernels.h"

namespace pam {

hipError_t paged_bf16(const PagedArgs &a, int store, int piece, hipStream_t s)
{
    return paged_type<bf16>(a, store, piece, s);
}

}  // namespace pam
