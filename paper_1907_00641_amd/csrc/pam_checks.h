// What the C entry points of the attention operators check their arguments with:
// refusals with a text, the memory that an array spans, overlaps.
#pragma once

#include <math.h>
#include <stdint.h>

#include <algorithm>
#include <initializer_list>

#include "pam_internal.h"

#define REQUIRE(cond, text)                                                                       \
    do {                                                                                          \
        if (!(cond))                                                                              \
            return abi_fail(PAM_ERR_INVALID_ARGUMENT, text);                                      \
    } while (0)

#define LAUNCH(call, what)                                                                        \
    do {                                                                                          \
        pam_status_t st_ = abi_sticky_error();                                                    \
        if (st_ != PAM_OK)                                                                        \
            return st_;                                                                           \
        hipError_t e_ = (call);                                                                   \
        if (e_ != hipSuccess)                                                                     \
            return abi_hip_fail(e_, what);                                                        \
    } while (0)

namespace pam {

inline bool known_type(int32_t t) { return t == PAM_F32 || t == PAM_F16 || t == PAM_BF16; }
inline int64_t bytes_of(int32_t t) { return t == PAM_F32 ? 4 : 2; }

// bytes that an array of `n` axes spans, from its lowest to past its highest
// element; false if that does not fit 62 bits
struct Span {
    const char *from, *to;
};
inline bool span_of(const void *p, int32_t dtype, const int64_t *len, const int64_t *stride, int n, int64_t last, Span *s)
{
    __int128 lo = 0, hi = last;
    for (int i = 0; i < n; ++i) {
        if (len[i] <= 0) {
            *s = {(const char *)p, (const char *)p};
            return true;
        }
        const __int128 far = (__int128)(len[i] - 1) * stride[i];
        (far < 0 ? lo : hi) += far;
    }
    const __int128 most = (__int128)1 << 59;
    if (lo < -most || hi > most)
        return false;
    const int64_t e = bytes_of(dtype);
    *s = {(const char *)p + (int64_t)lo * e, (const char *)p + (int64_t)hi * e};
    return true;
}
inline Span bytes_at(const void *p, int64_t n) { return {(const char *)p, (const char *)p + (p ? n : 0)}; }
inline bool meet(const Span &a, const Span &b)
{
    return a.from < a.to && b.from < b.to && a.from < b.to && b.from < a.to;
}
inline bool meet_any(const Span &a, std::initializer_list<Span> with)
{
    for (const Span &b : with)
        if (meet(a, b))
            return true;
    return false;
}

}  // namespace pam
