// The rate of dropout as a whole number of 65536ths (host).
#pragma once

#include <math.h>
#include <stdint.h>

namespace bz {

// false: not a rate
inline bool drop_threshold(double rate, uint32_t* least) {
    if (!(rate >= 0.0 && rate < 1.0)) return false;
    const double t = nearbyint(rate * 65536.0);   // ties to even
    *least = static_cast<uint32_t>(t);
    return t < 65536.0;
}
inline float drop_scale(uint32_t least) { return static_cast<float>(65536.0 / (65536.0 - least)); }

}  // namespace bz
