// Stands in place of csrc/lds_load.hpp on the CPU (test infrastructure; see
// main.cpp): the descriptor's range check, and a load that lands at once.
#pragma once

#include <hip/hip_runtime.h>

namespace cliff {

constexpr uint32_t NOWHERE = 0x80000000u;

inline void load_to_lds(const void* from, uint32_t offset, char* to)
{
    to += 16 * emulate::lane_id();
    if ((uint64_t)offset + 16 > 0x7fffffffu) memset(to, 0, 16);
    else memcpy(to, static_cast<const char*>(from) + offset, 16);
}
inline void wait_direct() {}

}  // namespace cliff
