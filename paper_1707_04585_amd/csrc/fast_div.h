// Division of an index by a number that the host knows: one 64-bit product and a shift.  With p = 31 + ceil(log2 d) and
// m = ceil(2^p / d), which is below 2^32, the quotient is (e * m) >> p for every 0 <= e < 2^31: m * d - 2^p < d <= 2^(p - 31),
// so that e * m / 2^p exceeds e / d by less than 2^31 * 2^(p - 31) / (2^p * d) = 1 / d.
#pragma once

#include <cstdint>

#if defined(__HIPCC__)
#include <hip/hip_runtime.h>
#define RVN_HOST_DEVICE __host__ __device__ __forceinline__
#else
#define RVN_HOST_DEVICE inline
#endif

namespace rvn {

struct FastDiv {
    uint32_t m, d;
    int p;
};

inline FastDiv fast_div(int d) {
    int up = 0;
    while (((int64_t)1 << up) < d) ++up;
    const int p = 31 + up;
    return FastDiv{(uint32_t)((((uint64_t)1 << p) + (uint64_t)d - 1) / (uint64_t)d), (uint32_t)d, p};
}

RVN_HOST_DEVICE int quotient(int e, const FastDiv &f) { return (int)(((uint64_t)(uint32_t)e * f.m) >> f.p); }

}  // namespace rvn
