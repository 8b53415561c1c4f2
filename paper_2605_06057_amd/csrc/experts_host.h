// Checks that the 8-bit-integer product and the tokens' way to their experts share (host side).
#pragma once
#include "host_common.h"
#include "lcma_experts_params.h"

namespace lcma {

constexpr int64_t kRowLimit = (int64_t)1 << 31;   // rows, columns and slots are counted in 32 bits on the device
constexpr int64_t kPitchLimit = (int64_t)1 << 29; // leading dimensions: 2^31 rows of 2^29 elements of 4 bytes are 2^62 bytes

constexpr int64_t kGridLimit = (int64_t)1 << 32;  // threads of a launch along a dimension

// the kernels of the product by number (lcma_experts_params.h), named by the rows and columns of their tiles
constexpr const char *kI8KernelNames[kI8Kernels] = {"16x16", "32x32", "64x64", "64x128", "128x128", "128x256", "256x256"};
int tuning_i8_kernel(); // csrc/api.cc; -1: choose

// whether two ranges of bytes have one in common
inline bool touch(const void *a, int64_t a_bytes, const void *b, int64_t b_bytes) {
    return a && b && a_bytes > 0 && b_bytes > 0 && (uintptr_t)a < (uintptr_t)b + (uint64_t)b_bytes && (uintptr_t)b < (uintptr_t)a + (uint64_t)a_bytes;
}

} // namespace lcma
