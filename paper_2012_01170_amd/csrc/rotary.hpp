// What the rotations by positions share: which pairs a lane has, and a pair's turn.
//
// A token's lanes have one vector of pairs each (of the pairs themselves, or of their first
// and of their second halves), and further lanes one of channels past the last pair.
#pragma once

#include "seq.hpp"

namespace sbc {

// Pairs of a lane: one vector of them, or of each of their halves
template <typename T, bool kInterleaved> constexpr int kPairs = kInterleaved ? kVec<T> / 2 : kVec<T>;

// Cosine and sine of position * freq.  The angle is taken in revolutions in float64, where
// the product of two float32 is exact and 1 / 2 pi costs 2^-53 of it, and reduced before
// sine and cosine in float32: angles of 1e6 (timestamps) are as good as small ones.
__device__ __forceinline__ void turn_of(double position, float freq, float &c, float &s) {
    double rev = position * (double)freq * 0.15915494309189533577;
    rev -= rint(rev);
    sincospif((float)(2.0 * rev), &s, &c);
}

// Lanes that a token takes
inline int64_t rotary_units(sbc_dtype dtype, bool interleaved, int64_t pairs, int64_t d) {
    const int V = dtype == SBC_F32 ? 4 : 8;
    const int N = interleaved ? V / 2 : V;  // (kPairs)
    return (pairs + N - 1) / N + (d - 2 * pairs + V - 1) / V;
}

// A plan's pairs, and those of its axes so far
inline sbc_status check_rotary(const sbc_rotary_plan *plan, int32_t d, int64_t *pairs,
                               int32_t (&upto)[SBC_MAX_AXES]) {
    if (plan->n_axes < 1 || plan->n_axes > SBC_MAX_AXES)
        return fail(SBC_ERR_INVALID_ARG, "n_axes must be 1 .. SBC_MAX_AXES");
    *pairs = 0;
    for (int x = 0; x < plan->n_axes; ++x) {
        if (plan->sections[x] < 0) return fail(SBC_ERR_INVALID_ARG, "a section is negative");
        *pairs += plan->sections[x];
        upto[x] = (int32_t)(*pairs <= d ? *pairs : d);
    }
    if (*pairs < 1 || 2 * *pairs > d)
        return fail(SBC_ERR_INVALID_ARG, "the sections must sum to 1 .. d / 2 pairs");
    if (plan->position_stride < plan->n_axes)
        return fail(SBC_ERR_INVALID_ARG, "position_stride is smaller than n_axes");
    return SBC_OK;
}

}  // namespace sbc
