// How a launch of the recurrence cuts its work: plain host arithmetic.
#pragma once
#include <stdint.h>

namespace tensair {
namespace recurrence {

constexpr int kThreads = 256;
constexpr int kSteps = 8;                // of a thread
constexpr uint32_t kClusters[] = {1, 2, 4, 8, 12, 16};
constexpr int kSizes = sizeof(kClusters) / sizeof(kClusters[0]);
constexpr uint32_t kMostCluster = 16;
constexpr uint32_t kClusterChannels = 64;      // of a block that is part of a cluster, at most

// A block covers `units` pieces of channels (of all sequences, one after the other) and kThreads / units stretches of kSteps steps at a time.
struct Plan {
    uint32_t units;        // power of two
    uint32_t cluster, turns;
    uint32_t groups;       // of `units` pieces
    uint32_t grid;
};

// Cuts T steps of `total` pieces of e channels so that the blocks that the device holds at once (`room`: clusters of each size; 0: it holds none of that
// size, which is left out) come out even: the fewest turns of the busiest one, a group of channels
// counting half a turn more, and turns in clusters by what their exchange takes.  us, stretches x cluster: gradient of 64 sequences of 1,024 of
// 512, bf16: 16 x 1 97, 16 x 2 89, 16 x 4 92, 32 x 1 110, 32 x 2 107, 32 x 8 206; forward, 64 padded of 1,021 of 300, fp32: 72, 68, 67, 68, 69, 151; one
// of 65,536 of 512, bf16: 32 x 4 198, 32 x 8 137, 32 x 12 103, 32 x 16 121.  (Measured when a factor had one form; a twentieth more since.)
inline Plan cut(uint32_t T, uint32_t total, uint32_t e, const uint32_t (&room)[kSizes]) {
    Plan best = {};
    uint64_t least = ~0ull;
    uint32_t most = 1;      // stretches enough for the sequence, 32 at most
    while (most < 32 && most * kSteps < T) most *= 2;
    for (uint32_t stretches = most; stretches && stretches >= most / 2; stretches /= 2) {
        Plan c = {};
        c.units = kThreads / stretches;
        c.groups = (total + c.units - 1) / c.units;
        static constexpr uint32_t kTurn[kSizes] = {8, 9, 10, 11, 11, 12};
        for (int i = 0; i < kSizes; ++i) {
            c.cluster = kClusters[i];
            const uint64_t span = (uint64_t)c.cluster * stretches * kSteps, turns = (T + span - 1) / span;
            const uint64_t held = i == 0 && !room[i] ? 1 : room[i];      // single blocks always go
            if (held) {
                const uint64_t rounds = (c.groups + held - 1) / held;
                const uint64_t cost = rounds * (2 * turns + 1) * kTurn[i];
                if (cost < least) {
                    least = cost;
                    c.turns = (uint32_t)turns;
                    c.grid = (uint32_t)(c.groups < held ? c.groups : held) * c.cluster;
                    best = c;
                }
            }
            if (turns == 1 || c.units * e > kClusterChannels) break;
        }
    }
    return best;
}

// The lanes of a thread's warp that belong to the last `channels` (a power of two from 16 on) threads of a block, as that thread does.
#ifdef __CUDACC__
__device__
#endif
inline uint32_t last_lanes(uint32_t channels, uint32_t thread) { return channels >= 32 ? 0xFFFFFFFFu : 0xFFFFu << (thread & 16); }

}  // namespace recurrence
}  // namespace tensair
