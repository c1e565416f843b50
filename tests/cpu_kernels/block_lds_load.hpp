// Stands in place of csrc/lds_load.hpp on the CPU (test infrastructure; see
// block_main.cpp), lds_load.hpp with what the 8-bit products use beside it: the
// descriptor's range check, a load that lands at once or, the other extreme, when the
// thread waits for it, and a barrier.
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
inline void barrier_alone() { emulate::meet_workgroup(); }
template <int N>
void wait_direct_but()
{
    emulate::wait_loads_but(N);
}

}  // namespace cliff
