// The positions of a batch sorted by token (stable), with the segments of equal tokens: what the embedding gradient
// sums by.  Positions that hold no token (padding, ids outside [0,V)) sort behind all others, as key V.
//
// Up to 2^17 positions the whole sort is one launch of one thread-block cluster.  A batch of that size is a
// megabyte at most, so it stays in the cluster's shared memory: every pass ranks its items in registers, exchanges the
// digit totals through distributed shared memory and scatters the items straight into the shared memory of the block
// that owns their place.  What bounds it is latency (a handful of cluster barriers and shared-memory round trips
// per pass), so the digits are as wide as the counters allow: ten bits, two passes up to V = 2^20 - 1.
// Larger batches go through the library's multi-launch radix sort.
#include <cooperative_groups.h>

#include <atomic>

#include "kernels.h"
#include "operators.h"

namespace cg = cooperative_groups;

namespace tensair {

namespace {

constexpr int kSortBlock = 1024;
constexpr int kSortBlockWarps = kSortBlock / 32;
constexpr int kMaxDigitBits = 10;
constexpr uint32_t kMaxCluster = 8;                            // the portable cluster size
constexpr uint32_t kOneLaunch = kMaxCluster * kSortBlock * 16;  // 131,072 positions

__device__ __forceinline__ uint32_t token_key(const TokenIds& t, uint32_t i) {
    const int64_t id = t.wide ? reinterpret_cast<const int64_t*>(t.ids)[i] : reinterpret_cast<const int32_t*>(t.ids)[i];
    if (id == t.padding) return t.V;
    if ((uint64_t)id < t.V) return (uint32_t)id;
    if (t.err) atomicOr(t.err, kErrBadToken);
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
    uint32_t scan = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const uint32_t u = __shfl_up_sync(0xFFFFFFFFu, scan, o);
        if (lane >= (uint32_t)o) scan += u;
    }
    if (total) *total = __shfl_sync(0xFFFFFFFFu, scan, 31);
    const uint32_t before = __shfl_sync(0xFFFFFFFFu, scan - mine, wid);
    __syncthreads();
    return before + incl - x;
}

struct ClusterShared {
    uint32_t warp_sums[kSortBlockWarps];
    uint32_t heads[kMaxCluster], valid[kMaxCluster];   // of every block of the cluster, written by that block
    uint32_t digit_base[1 << kMaxDigitBits];
};

template <int kItems>
constexpr size_t cluster_shared_bytes() {
    return sizeof(ClusterShared) + (size_t)kSortBlock * kItems * 8                // items
           + (size_t)kSortBlockWarps * (1 << kMaxDigitBits) * 2                   // counters per warp
           + (size_t)kMaxCluster * (1 << kMaxDigitBits) * 2;                      // digit totals of every block
}

template <int kItems>
__global__ void __launch_bounds__(kSortBlock, 1)
k_cluster_sort(TokenIds t, SortedTokens s, uint32_t key_bits, uint32_t digit_bits) {
    cg::cluster_group cluster = cg::this_cluster();
    const uint32_t rank = cluster.block_rank(), blocks = cluster.num_blocks();
    extern __shared__ __align__(16) uint8_t raw[];
    ClusterShared& sh = *reinterpret_cast<ClusterShared*>(raw);
    uint2* items = reinterpret_cast<uint2*>(raw + sizeof(ClusterShared));         // (key, position)
    uint16_t* counts = reinterpret_cast<uint16_t*>(items + kSortBlock * kItems);  // [warp][digit]
    uint16_t* totals = counts + (kSortBlockWarps << kMaxDigitBits);               // [block][digit]
    constexpr uint32_t kPerBlock = kSortBlock * kItems;
    const uint32_t lane = threadIdx.x & 31, wid = threadIdx.x >> 5;
    const uint32_t first = rank * kPerBlock;          // first position of this block
    const uint32_t bins = 1u << digit_bits, mask = bins - 1;
    const uint32_t my = wid * 32 * kItems + lane;     // a warp owns 32 * kItems consecutive items
    const uint32_t lower = (1u << lane) - 1;
    uint2 item[kItems];
    uint32_t place[kItems];
#pragma unroll
    for (int r = 0; r < kItems; ++r) {
        const uint32_t i = first + my + r * 32;
        // places past the batch sort behind everything, in order
        item[r] = make_uint2(i < t.n ? token_key(t, i) : 0xFFFFFFFFu, i);
    }
    for (uint32_t shift = 0; shift < key_bits; shift += digit_bits) {
        for (uint32_t x = threadIdx.x; x < kSortBlockWarps * bins / 2; x += kSortBlock)
            reinterpret_cast<uint32_t*>(counts)[x] = 0;
        __syncthreads();
        uint16_t* mine = counts + wid * bins;
#pragma unroll
        for (int r = 0; r < kItems; ++r) {
            const uint32_t digit = (item[r].x >> shift) & mask;
            const uint32_t peers = __match_any_sync(0xFFFFFFFFu, digit);
            const uint32_t before = mine[digit];
            __syncwarp();
            place[r] = before + __popc(peers & lower);
            if ((peers & lower) == 0) mine[digit] = (uint16_t)(before + __popc(peers));
            __syncwarp();
        }
        __syncthreads();
        // per digit: exclusive sum over the warps, and the block's total to every block of the cluster
        for (uint32_t digit = threadIdx.x; digit < bins; digit += kSortBlock) {
            uint32_t run = 0;
#pragma unroll 8
            for (int w = 0; w < kSortBlockWarps; ++w) {
                const uint32_t c = counts[w * bins + digit];
                counts[w * bins + digit] = (uint16_t)run;
                run += c;
            }
            for (uint32_t b = 0; b < blocks; ++b) cluster.map_shared_rank(totals, b)[rank * bins + digit] = (uint16_t)run;
        }
        cluster.sync();   // every block's totals are here, and every item of the previous pass is in registers
        uint32_t sum = 0, before = 0;
        if (threadIdx.x < bins)
            for (uint32_t b = 0; b < blocks; ++b) {
                const uint32_t c = totals[b * bins + threadIdx.x];
                if (b < rank) before += c;
                sum += c;
            }
        const uint32_t digit_start = block_exclusive(sum, sh.warp_sums, nullptr);
        if (threadIdx.x < bins) sh.digit_base[threadIdx.x] = digit_start + before;
        __syncthreads();
#pragma unroll
        for (int r = 0; r < kItems; ++r) {
            const uint32_t digit = (item[r].x >> shift) & mask;
            const uint32_t to = sh.digit_base[digit] + mine[digit] + place[r];
            cluster.map_shared_rank(items, to / kPerBlock)[to % kPerBlock] = item[r];
        }
        cluster.sync();
        if (shift + digit_bits < key_bits) {
#pragma unroll
            for (int r = 0; r < kItems; ++r) item[r] = items[my + r * 32];
        }
    }
    // this block now holds sorted positions [first, first + kPerBlock): mark the first position of every token
    uint32_t head_bits = 0, n_valid = 0, n_heads = 0;
#pragma unroll
    for (int r = 0; r < kItems; ++r) {
        const uint32_t at = my + r * 32;
        item[r] = items[at];
        uint32_t previous = 0xFFFFFFFFu;
        if (at) previous = items[at - 1].x;
        else if (rank) previous = cluster.map_shared_rank(items, rank - 1)[kPerBlock - 1].x;
        const bool valid = item[r].x < t.V;
        const bool head = valid && item[r].x != previous;
        const uint32_t heads = __ballot_sync(0xFFFFFFFFu, head);
        n_valid += __popc(__ballot_sync(0xFFFFFFFFu, valid));
        place[r] = n_heads + __popc(heads & lower);   // heads of this warp before the item
        n_heads += __popc(heads);
        head_bits |= (uint32_t)head << r;
    }
    uint32_t block_heads, block_valid;
    uint32_t before = block_exclusive(lane == 0 ? n_heads : 0, sh.warp_sums, &block_heads);
    before = __shfl_sync(0xFFFFFFFFu, before, 0);
    block_exclusive(lane == 0 ? n_valid : 0, sh.warp_sums, &block_valid);
    if (threadIdx.x < blocks) {
        cluster.map_shared_rank(sh.heads, threadIdx.x)[rank] = block_heads;
        cluster.map_shared_rank(sh.valid, threadIdx.x)[rank] = block_valid;
    }
    cluster.sync();       // no block reads another one's shared memory after this
    uint32_t all_heads = 0, all_valid = 0;
    for (uint32_t b = 0; b < blocks; ++b) {
        if (b < rank) before += sh.heads[b];
        all_heads += sh.heads[b];
        all_valid += sh.valid[b];
    }
#pragma unroll
    for (int r = 0; r < kItems; ++r) {
        const uint32_t i = first + my + r * 32;
        if (i < t.n) {
            const uint32_t h = before + place[r];
            s.key[i] = item[r].x;
            s.pos[i] = item[r].y;
            if (head_bits >> r & 1) s.seg_start[h] = i;
            if ((i & (s.span - 1)) == 0) s.span_rank[i / s.span] = h;
        }
    }
    if (rank == 0 && threadIdx.x == 0) {
        s.info[0] = all_valid;
        s.info[1] = all_heads;
        s.info[2] = s.info[3] = 0;
        s.seg_start[all_heads] = all_valid;
    }
}

template <int kItems>
cudaError_t cluster_sort(cudaStream_t stream, const TokenIds& t, const SortedTokens& s, uint32_t blocks) {
    constexpr size_t shared = cluster_shared_bytes<kItems>();
    static std::atomic<uint64_t> ready{0};     // devices on which the kernel may use that much shared memory
    static_assert(kMaxDevices <= 64, "one bit per device");
    int device = 0;
    cudaError_t e = cudaGetDevice(&device);
    if (e != cudaSuccess) return e;
    if (device >= kMaxDevices || !(ready.load(std::memory_order_relaxed) >> device & 1)) {
        e = cudaFuncSetAttribute(k_cluster_sort<kItems>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)shared);
        if (e != cudaSuccess) return e;
        if (device < kMaxDevices) ready.fetch_or(1ull << device, std::memory_order_relaxed);
    }
    uint32_t key_bits = 1;
    while (key_bits < 32 && t.V >> key_bits) ++key_bits;
    const uint32_t passes = (key_bits + kMaxDigitBits - 1) / kMaxDigitBits;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = blocks;
    cfg.blockDim = kSortBlock;
    cfg.dynamicSmemBytes = shared;
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = blocks;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, k_cluster_sort<kItems>, t, s, key_bits, (key_bits + passes - 1) / passes);
}

// ---- larger batches
constexpr int kTileThreads = 256;
constexpr uint32_t kTileItems = 4096;

__global__ void __launch_bounds__(kTileThreads) k_token_items(TokenIds t, item_t* __restrict__ items) {
    const uint32_t i = blockIdx.x * kTileThreads + threadIdx.x;
    if (i < t.n) items[i] = make_item(token_key(t, i), i);
}

__device__ __forceinline__ bool begins_token(const item_t* items, uint32_t i, uint32_t V) {
    const uint32_t key = item_key(items[i]);
    return key < V && (i == 0 || item_key(items[i - 1]) != key);
}

__global__ void __launch_bounds__(kTileThreads)
k_count_tokens(const item_t* __restrict__ items, uint32_t n, uint32_t V, uint32_t* __restrict__ tile_counts) {
    uint32_t c = 0;
    for (uint32_t x = threadIdx.x; x < kTileItems; x += kTileThreads) {
        const uint64_t i = (uint64_t)blockIdx.x * kTileItems + x;
        if (i < n) c += begins_token(items, (uint32_t)i, V);
    }
    __shared__ uint32_t warp_sums[kTileThreads / 32];
    uint32_t total;
    block_exclusive(c, warp_sums, &total);
    if (threadIdx.x == 0) tile_counts[blockIdx.x] = total;
}

__global__ void __launch_bounds__(kTileThreads)
k_write_tokens(const item_t* __restrict__ items, uint32_t n, uint32_t V, const uint32_t* __restrict__ tile_counts,
               SortedTokens s) {
    __shared__ uint32_t warp_sums[kTileThreads / 32];
    uint32_t c = 0, run;
    for (uint32_t x = threadIdx.x; x < blockIdx.x; x += kTileThreads) c += tile_counts[x];
    block_exclusive(c, warp_sums, &run);
    for (uint32_t x = 0; x < kTileItems; x += kTileThreads) {
        const uint64_t i64 = (uint64_t)blockIdx.x * kTileItems + x + threadIdx.x;
        const uint32_t i = (uint32_t)i64;
        const bool in = i64 < n;
        const bool head = in && begins_token(items, i, V);
        uint32_t heads;
        const uint32_t h = run + block_exclusive(head, warp_sums, &heads);
        if (in) {
            const uint32_t key = item_key(items[i]);
            s.key[i] = key;
            s.pos[i] = item_payload(items[i]);
            if (head) s.seg_start[h] = i;
            if ((i & (s.span - 1)) == 0) s.span_rank[i / s.span] = h;
            if (i + 1 == n || (key < V && item_key(items[i + 1]) >= V)) {    // the last valid position, or the batch's end
                if (key < V) {
                    s.info[0] = i + 1;
                    s.info[1] = h + head;
                    s.seg_start[h + head] = i + 1;
                } else if (item_key(items[0]) >= V) {
                    s.info[0] = s.info[1] = 0;
                    s.seg_start[0] = 0;
                }
            }
            if (i == 0) s.info[2] = s.info[3] = 0;
        }
        run += heads;
    }
}

}  // namespace

bool sorts_in_one_launch(uint32_t n) { return n <= kOneLaunch; }

cudaError_t launch_token_sort(cudaStream_t stream, const TokenIds& t, const SortedTokens& s, const SortScratch& w) {
    if (sorts_in_one_launch(t.n)) {
        // as many items per thread as needed for eight blocks, as few blocks as hold four per thread: fewer blocks mean
        // cheaper cluster barriers, more items per thread a longer ranking loop
        if (t.n <= kSortBlock) return cluster_sort<1>(stream, t, s, 1);
        uint32_t blocks = 1;
        while (blocks < kMaxCluster && blocks * kSortBlock * 4 < t.n) blocks *= 2;
        if (t.n <= blocks * kSortBlock * 4) return cluster_sort<4>(stream, t, s, blocks);
        if (t.n <= blocks * kSortBlock * 8) return cluster_sort<8>(stream, t, s, blocks);
        return cluster_sort<16>(stream, t, s, blocks);
    }
    uint64_t launches = 0;
    Launcher L{stream, &launches, 0, nullptr};
    L.lim.err = s.info;    // only read by the checked build's scatter, whose positions are below n by construction
    uint32_t key_bits = 1;
    while (key_bits < 32 && t.V >> key_bits) ++key_bits;
    k_token_items<<<(t.n + kTileThreads - 1) / kTileThreads, kTileThreads, 0, stream>>>(t, w.a);
    item_t* sorted = nullptr;
    const cudaError_t e = launch_sort(L, w.a, w.b, t.n, key_bits, w.hist, &sorted);
    if (e != cudaSuccess) return e;
    const uint32_t tiles = (t.n + kTileItems - 1) / kTileItems;
    k_count_tokens<<<tiles, kTileThreads, 0, stream>>>(sorted, t.n, t.V, w.tile_counts);
    k_write_tokens<<<tiles, kTileThreads, 0, stream>>>(sorted, t.n, t.V, w.tile_counts, s);
    return cudaGetLastError();
}

}  // namespace tensair
