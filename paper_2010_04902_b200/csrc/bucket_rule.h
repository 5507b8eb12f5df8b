// Distances at which the logarithmic buckets of a relative position bias begin (host only).
#pragma once

#include <math.h>
#include <stdint.h>

namespace bz {

// Of nb buckets the first e = nb / 2 hold a distance each; bucket e + t, t = 0 .. nb - e - 1, begins at the smallest whole
// n >= e * (distance / e)^(t / (nb - e)), which is starts[t].  The products below are off by less than 128 * 3 * 2^-53 = 5e-14
// of their value, and no bound of any nb <= 256 and distance <= 2048 that is not a whole number lies closer than 2e-11 of its
// value above one: what lies within 1e-12 above a whole number is that number.
inline void bucket_starts(int nb, int distance, uint16_t* starts) {
    const int e = nb / 2, steps = nb - e;
    const double ratio = pow(static_cast<double>(distance) / e, 1.0 / steps);
    double x = e;
    starts[0] = static_cast<uint16_t>(e);
    for (int t = 1; t < steps; ++t) starts[t] = static_cast<uint16_t>(ceil((x *= ratio) * (1.0 - 1e-12)));
}

}  // namespace bz
