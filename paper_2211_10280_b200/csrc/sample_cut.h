// How many blocks share a row in the draw of the next token: plain host arithmetic.
#pragma once
#include <stdint.h>

namespace tensair {

constexpr uint32_t kMostRowBlocks = 16;

// Blocks enough for the device, as long as a slice is worth the cluster's barriers; a power of two, `most` (what the device holds a cluster of) at most.
// us, 1, 2, 4, 8, 16 blocks to a row, each with 10 for the launch: 256 rows of 100,000, 0.9 of the mass: 108, 170, 212; first 50: 65, 109; 64 rows of
// 10,000: 25, 28, 32, 47, 83; 16 rows of 100,000: 194, 112, 74, 53, 55; one row of 100,000: 69, 46, 29, 28, 24
inline uint32_t row_blocks(uint32_t n, uint32_t V, uint32_t sms, uint32_t most) {
    uint32_t cluster = 1;
    while (cluster * 2 <= most && (uint64_t)n * cluster < sms && V > cluster * 8000) cluster *= 2;
    return cluster;
}

}  // namespace tensair
