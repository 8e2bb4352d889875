// Microscaled 4-bit floating point: elements E2M1 (0, 0.5, 1, 1.5, 2, 3, 4, 6 and their negatives) in blocks of 32 along a row, each
// with a power of two held as its exponent and a bias of 127 (OCP Microscaling Formats specification, 2023).
//
// A row of C elements has ceil(C / 32) blocks: 16 bytes of codes each, element i in the low half of byte i / 2 for even i, in the high half
// for odd i, and one byte for the power; 255 stands for NaN.
#pragma once

#include "rows.cuh"

namespace emc2 {

constexpr int kMxBlock = 32;
constexpr int kMaxMxChannels = 8192;
inline int mx4_blocks(int channels) { return (channels + kMxBlock - 1) / kMxBlock; }

#ifdef __CUDACC__

// 2^(byte - 127), NaN for 255.
__device__ __forceinline__ float mx_power(uint32_t byte) {
    return __uint_as_float(byte == 255u ? 0x7FC00000u : byte == 0u ? 0x00400000u : byte << 23);
}

#endif

}  // namespace emc2
