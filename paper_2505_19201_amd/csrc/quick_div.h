// Divisions by numbers that are the same for a whole launch.
#pragma once
#include <hip/hip_runtime.h>
#include <cstdint>

namespace dream {

// x / d for x * d below 2^32 by one multiplication (a division is some 20 instructions): magic_of(d), 0 for d = 1
inline uint32_t magic_of(uint32_t d) { return d == 1 ? 0u : (uint32_t)(((1ull << 32) + d - 1) / d); }
__device__ __forceinline__ uint32_t quick_div(uint32_t x, uint32_t magic) { return magic ? __umulhi(x, magic) : x; }

}  // namespace dream
