// Device pieces of the token sorts: reading ids, sums over a block, ranking by a digit.
#pragma once
#include "operators.h"

namespace tensair {

constexpr int kSortBlock = 1024;
constexpr int kSortBlockWarps = kSortBlock / 32;
constexpr int kMaxDigitBits = 10;

__device__ __forceinline__ uint32_t token_key(const TokenIds& t, uint32_t i) {
    const int64_t id = t.wide ? reinterpret_cast<const int64_t*>(t.ids)[i] : reinterpret_cast<const int32_t*>(t.ids)[i];
    if (t.is_token(id)) return (uint32_t)id;
    t.report(id);
    return t.V;
}

// Exclusive sum of `x` over the block's threads in thread order; *total (optional) receives the sum of all.
__device__ __forceinline__ uint32_t block_exclusive(uint32_t x, uint32_t* warp_sums, uint32_t* total) {
    const uint32_t lane = threadIdx.x & 31, wid = threadIdx.x >> 5;
    uint32_t incl = x;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const uint32_t u = __shfl_up_sync(0xFFFFFFFFu, incl, o);
        if (lane >= (uint32_t)o) incl += u;
    }
    if (lane == 31) warp_sums[wid] = incl;
    __syncthreads();
    const uint32_t mine = lane < (blockDim.x >> 5) ? warp_sums[lane] : 0;
    const uint32_t before = __reduce_add_sync(0xFFFFFFFFu, lane < wid ? mine : 0);
    if (total) *total = __reduce_add_sync(0xFFFFFFFFu, mine);
    __syncthreads();
    return before + incl - x;
}

// Rank of the thread's item among the block's items of its digit, in item order.  counts: [warp][digit] in shared memory, 16 bits
// each.  publish(x, totals) is called once for every pair of digits (2x, 2x + 1) with the block's two totals, 16 bits each.
//
// Within a warp the lanes of a digit find each other by one ballot per bit (the match instruction gains nothing: it takes longer
// the more digits a warp's items have, and the slowest block counts).
template <typename F>
__device__ __forceinline__ uint32_t block_rank(uint32_t digit, uint32_t digit_bits, uint32_t* counts, F&& publish) {
    const uint32_t lane = threadIdx.x & 31, wid = threadIdx.x >> 5, pairs = 1u << digit_bits >> 1;
    for (uint32_t x = threadIdx.x; x < kSortBlockWarps * pairs; x += kSortBlock) counts[x] = 0;
    uint32_t peers = 0xFFFFFFFFu;
#pragma unroll
    for (int bit = 0; bit < kMaxDigitBits; ++bit)
        if (bit < (int)digit_bits) {
            const bool one = (digit & 1u << bit) != 0;
            peers &= __ballot_sync(0xFFFFFFFFu, one) ^ (one ? 0u : 0xFFFFFFFFu);
        }
    const uint32_t rank = __popc(peers & ((1u << lane) - 1));
    uint16_t* mine = reinterpret_cast<uint16_t*>(counts) + wid * 2 * pairs;
    __syncthreads();
    if (rank == 0) mine[digit] = (uint16_t)__popc(peers);
    __syncthreads();
    if (threadIdx.x < pairs) {       // exclusive sum over the warps, two digits at once
        uint32_t run = 0;
#pragma unroll 16
        for (int w = 0; w < kSortBlockWarps; ++w) {
            const uint32_t c = counts[w * pairs + threadIdx.x];
            counts[w * pairs + threadIdx.x] = run;
            run += c;
        }
        publish(threadIdx.x, run);
    }
    __syncthreads();
    return rank + mine[digit];
}

}  // namespace tensair
