// Division by a number that the host knows, as a multiplication and a shift.  Plain C++, for the host, the kernels and a test.
#pragma once
#include <stdint.h>

#if defined(__HIP__)
#define DHSA_BOTH __host__ __device__ __forceinline__
#else
#define DHSA_BOTH inline
#endif

namespace dhsa {

// With l = ceil(log2 d) and mul = floor(2^(31 + l) / d) + 1 < 2^32, mul d - 2^(31 + l) is in 1 .. d <= 2^l, so x mul / 2^(31 + l) is
// above x / d by less than 1 / d for x < 2^31.  1 <= d <= 2^30.
inline void set_divisor(uint32_t d, uint32_t *mul, int *shift) {
    int l = 0;
    while (((uint64_t)1 << l) < d) ++l;
    *mul = (uint32_t)((((uint64_t)1 << (31 + l)) / d) + 1);
    *shift = 31 + l;
}
DHSA_BOTH int divided(int x, uint32_t mul, int shift) { return (int)(((uint64_t)(uint32_t)x * mul) >> shift); }      // x >= 0

}  // namespace dhsa
