// Stands in place of csrc/lds_load.hpp on the CPU (test infrastructure; see
// main.cpp): the descriptor's range check, and a load that lands at once or, the
// other extreme, when the thread waits for it.
#pragma once

#include <hip/hip_runtime.h>

namespace cliff {

constexpr uint32_t NOWHERE = 0x80000000u;

inline void load_to_lds(const void* from, uint32_t offset, char* to)
{
    const bool outside = (uint64_t)offset + 16 > 0x7fffffffu;
    emulate::load(outside ? nullptr : static_cast<const char*>(from) + offset, to + 16 * emulate::lane_id());
}
inline void wait_direct() { emulate::wait_loads(); }

}  // namespace cliff
