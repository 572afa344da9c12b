// How a list is shared among the threads of a workgroup.  Plain C++, the same on the device and in a host test.
#pragma once

#include <cstdint>

namespace craft {

// Neighbouring items of each of THREADS threads, so that all n are taken.  n may be any number of requests that a call
// takes, up to 2^31 - 1: rounding it up passes 32 bits with a sign, not without.
template <uint32_t THREADS> constexpr int32_t share_of(int32_t n) { return (int32_t)(((uint32_t)n + (THREADS - 1)) / THREADS); }

}  // namespace craft
