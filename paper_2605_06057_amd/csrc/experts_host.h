// Checks that the calls in 8 and 4 bits, the experts' products and the tokens' way to their experts share (host side).
#pragma once
#include "host_common.h"
#include "lcma_experts_params.h"

namespace lcma {

constexpr int64_t kRowLimit = (int64_t)1 << 31;   // rows, columns and slots are counted in 32 bits on the device
constexpr int64_t kPitchLimit = (int64_t)1 << 29; // leading dimensions: 2^31 rows of 2^29 elements of 4 bytes are 2^62 bytes

constexpr int64_t kMatrixLimit = (int64_t)1 << 44; // elements of an expert's matrix: 1024 of them are 2^56 bytes at most

constexpr int64_t kGridLimit = (int64_t)1 << 32;  // threads of a launch along a dimension

// Kernels with a work-group of up to 512 threads for each tile: whether one launch holds them all, whether several do (the device counts tiles in 32 bits), and what fills one: tiles of an eighth of them.
inline bool one_launch(int64_t tiles) { return (tiles + 8) * 512 < kGridLimit / 2; }
inline bool several_launches(int64_t tiles) { return tiles < kRowLimit - 1024; }
constexpr int64_t kLaunchEighth = kGridLimit / 2 / 512 / 8 - 2;

// the kernels of the product by number (lcma_experts_params.h), named by the rows and columns of their tiles
constexpr const char *kI8KernelNames[kI8Kernels] = {"16x16", "32x32", "64x64", "64x128", "128x128", "128x256", "256x256"};
int tuning_i8_kernel(); // csrc/api.cc; -1: choose
// of the experts' products: those that take any sizes and alignments, and those for whole 16 bytes; of the product with 4-bit weights
constexpr const char *kExpKernelNames[kExpKernels] = {"any64x64", "any128x128", "any32x32", "16x16", "32x32", "64x64", "64x128", "128x256", "256x256"};
int tuning_experts_kernel();
constexpr const char *kI4KernelNames[kI4Kernels] = {"16x16", "16x32", "16x64", "64x64"};
int tuning_i4_kernel();

// whether two ranges of bytes have one in common
inline bool touch(const void *a, int64_t a_bytes, const void *b, int64_t b_bytes) {
    return a && b && a_bytes > 0 && b_bytes > 0 && (uintptr_t)a < (uintptr_t)b + (uint64_t)b_bytes && (uintptr_t)b < (uintptr_t)a + (uint64_t)a_bytes;
}

} // namespace lcma
