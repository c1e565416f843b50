// dense_int8.hip on the CPU, and its dynamic LDS (test infrastructure; see
// block_main.cpp).
#include "dense_int8.hip"

namespace cliff {
namespace {
thread_local u4 smem4[160 * 1024 / 16];
emulate::DynamicLds lds(smem4, sizeof smem4);
}  // namespace
}  // namespace cliff
