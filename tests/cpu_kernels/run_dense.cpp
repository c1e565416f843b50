// dense.hip on the CPU, and its dynamic LDS (test infrastructure; see main.cpp).
#include "dense.hip"

namespace cliff {
namespace {
thread_local u4 smem4[160 * 1024 / 16];
emulate::DynamicLds lds(smem4, sizeof smem4);
}  // namespace
}  // namespace cliff
