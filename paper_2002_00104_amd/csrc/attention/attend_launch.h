// The kernels of one pair of types: its own source, so that the pairs compile beside each other.
#pragma once

#include "attend_few.h"
#include "attend_many.h"

namespace pwlq_attention {

template <typename T, typename C> void attend_launch(const Attend &a, int D, int rows, unsigned grid, hipStream_t stream)
{
    // plain scores have the scale as a factor of products that may be masked by then: it must leave a normal number
    const bool tiny = fabsf(a.scale) < 0x1p-100f;
    // tiles of 128 rows multiply three quarters of the channels where the others are none
#define PWLQ_ATTEND_AS(DP, SCORES)                                                                                             \
    do {                                                                                                                       \
        if (rows == 16) k_attend_few<T, C, DP, 1, SCORES><<<grid, 256, 0, stream>>>(a);                                        \
        else if (DP == 256 || rows == 128) {                                                                                   \
            if (DP != 64 && a.c.D <= DP * 3 / 4) k_attend_many<T, C, DP, DP == 64 ? DP : DP * 3 / 4, SCORES><<<grid, 256, 0, stream>>>(a); \
            else k_attend_many<T, C, DP, DP, SCORES><<<grid, 256, 0, stream>>>(a);                                             \
        } else if constexpr (DP != 256) k_attend_few<T, C, DP, 2, SCORES><<<grid, 256, 0, stream>>>(a);                        \
    } while (0)
#define PWLQ_ATTEND(DP)                                       \
    do {                                                      \
        if (a.cap > 0.0f) PWLQ_ATTEND_AS(DP, kCapped);        \
        else if (a.slopes || tiny) PWLQ_ATTEND_AS(DP, kSloped); \
        else PWLQ_ATTEND_AS(DP, kPlain);                      \
    } while (0)
    if (D == 64) PWLQ_ATTEND(64);
    else if (D == 128) PWLQ_ATTEND(128);
    else PWLQ_ATTEND(256);
#undef PWLQ_ATTEND
#undef PWLQ_ATTEND_AS
}

} // namespace pwlq_attention
