// The positions of a batch sorted by token (stable), with the segments of equal tokens: what the embedding gradient
// sums by.  Positions that hold no token (padding, ids outside [0,V)) sort behind all others, as key V.
//
// Up to 2^17 positions the whole sort is one launch of one thread-block cluster.  A batch of that size is a
// megabyte at most, so it stays in the cluster's shared memory: every pass ranks its items in registers, exchanges the
// digit totals through distributed shared memory and writes the items, put in digit order first, into the shared memory
// of the block that owns their place.  What bounds it is latency: issue slots of the ranking (which fall with the number
// of blocks) and a few barriers per pass, so a batch is spread over as many blocks as a cluster may have, and the digits are
// as wide as the counters allow: ten bits, two passes up to V = 2^20 - 1.
// Larger batches go through the library's multi-launch radix sort.
#include <cooperative_groups.h>

#include <atomic>
#include <utility>

#include "kernels.h"
#include "operators.h"

namespace cg = cooperative_groups;

namespace tensair {

namespace {

constexpr int kSortBlock = 1024;
constexpr int kSortBlockWarps = kSortBlock / 32;
constexpr int kMaxDigitBits = 10;
constexpr uint32_t kMaxCluster = 16;                           // needs leave of the device; 8 always works
constexpr uint32_t kPortableCluster = 8;
constexpr int kMaxItems = 8;                                   // per thread

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
    const uint32_t before = __reduce_add_sync(0xFFFFFFFFu, lane < wid ? mine : 0);
    if (total) *total = __reduce_add_sync(0xFFFFFFFFu, mine);
    __syncthreads();
    return before + incl - x;
}

// Part `part` of `parts` of the rows set to zero by the calling block.
__device__ void clear_part(const ClearRows& c, uint64_t part, uint64_t parts) {
    const uint4 zero = make_uint4(0, 0, 0, 0);
    const bool whole = c.stride == c.width;            // one stretch of memory, taken as one row
    const uint64_t rows = whole ? 1 : c.rows, width = whole ? c.rows * c.width : c.width;
    const uint64_t per_row = whole ? parts : 1;        // parts that share a row
    for (uint64_t row = part / per_row; row < rows; row += whole ? rows : parts) {
        uint8_t* data = c.data + row * c.stride;
        uint64_t head = (16 - (uintptr_t)data % 16) % 16;
        if (head > width) head = width;
        const uint64_t vecs = (width - head) / 16, each = (vecs + per_row - 1) / per_row;
        const uint64_t from = part % per_row * each, to = from + each < vecs ? from + each : vecs;
        uint4* at = reinterpret_cast<uint4*>(data + head);
        for (uint64_t x = from + threadIdx.x; x < to; x += blockDim.x) at[x] = zero;
        if (part % per_row == 0) {                     // the ends, in 16-bit steps: no element is narrower
            const uint64_t tail = head + vecs * 16;
            if (threadIdx.x * 2 < head) *reinterpret_cast<uint16_t*>(data + threadIdx.x * 2) = 0;
            if (tail + threadIdx.x * 2 < width) *reinterpret_cast<uint16_t*>(data + tail + threadIdx.x * 2) = 0;
        }
    }
}

struct ClusterShared {
    uint32_t warp_sums[kSortBlockWarps];
    uint32_t heads[kMaxCluster], valid[kMaxCluster];   // of every block of the cluster, written by that block
    uint32_t digit_base[1 << kMaxDigitBits];
};

constexpr size_t larger(size_t a, size_t b) { return a > b ? a : b; }
template <int kItems>
constexpr size_t cluster_shared_bytes(size_t bins, size_t blocks) {
    return sizeof(ClusterShared) + (size_t)kSortBlock * kItems * 8                          // items
           + larger(kSortBlockWarps * bins * 2, (size_t)kSortBlock * kItems * 8)            // counters per warp, then staging
           + blocks * bins * 2;                                                             // digit totals of every block
}
static_assert(cluster_shared_bytes<kMaxItems>(1 << kMaxDigitBits, kMaxCluster) <= 227 * 1024, "fits a block's shared memory");

template <int kItems>
__global__ void __launch_bounds__(kSortBlock, 1)
k_cluster_sort(TokenIds t, SortedTokens s, uint32_t key_bits, uint32_t digit_bits, ClearRows clear) {
    cg::cluster_group cluster = cg::this_cluster();
    let_next_launch_begin();
    const uint32_t rank = cluster.block_rank(), blocks = cluster.num_blocks();
    if (blockIdx.x >= blocks) {     // the first cluster sorts; the others clear beside it
        clear_part(clear, blockIdx.x - blocks, gridDim.x - blocks);
        return;
    }
    extern __shared__ __align__(16) uint8_t raw[];
    constexpr uint32_t kPerBlock = kSortBlock * kItems;
    const uint32_t bins = 1u << digit_bits, mask = bins - 1;
    ClusterShared& sh = *reinterpret_cast<ClusterShared*>(raw);
    uint2* items = reinterpret_cast<uint2*>(raw + sizeof(ClusterShared));         // (key, position)
    uint2* staged = items + kPerBlock;                                            // the block's items in digit order
    uint32_t* counts = reinterpret_cast<uint32_t*>(staged);                       // [warp][digit], 16 bits each; then staged
    uint16_t* totals = reinterpret_cast<uint16_t*>(raw + sizeof(ClusterShared) + kPerBlock * 8 +
                                                   max(kSortBlockWarps * bins * 2, kPerBlock * 8));   // [block][digit]
    const uint32_t lane = threadIdx.x & 31, wid = threadIdx.x >> 5;
    const uint32_t first = rank * kPerBlock;          // first position of this block
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
        for (uint32_t x = threadIdx.x; x < kSortBlockWarps * bins / 2; x += kSortBlock) counts[x] = 0;
        __syncthreads();
        uint16_t* mine = reinterpret_cast<uint16_t*>(counts) + wid * bins;
        // Rank of an item among the warp's items of its digit, in item order.  The lanes of a digit find each other by one
        // ballot per bit; the first of them moves the warp's counter on, with a plain store (an atomic add on shared memory, which
        // would spare the two barriers, took twice as long).  The rounds follow each other in order.
        constexpr int kGroup = kItems < 4 ? kItems : 4;
#pragma unroll
        for (int r0 = 0; r0 < kItems; r0 += kGroup) {
            uint32_t peers[kGroup];
#pragma unroll
            for (int r = 0; r < kGroup; ++r) peers[r] = 0xFFFFFFFFu;
#pragma unroll
            for (int bit = 0; bit < kMaxDigitBits; ++bit)
                if (bit < (int)digit_bits)
#pragma unroll
                    for (int r = 0; r < kGroup; ++r) {
                        const bool one = (item[r0 + r].x >> shift & 1u << bit) != 0;
                        peers[r] &= __ballot_sync(0xFFFFFFFFu, one) ^ (one ? 0u : 0xFFFFFFFFu);
                    }
#pragma unroll
            for (int r = 0; r < kGroup; ++r) {
                const uint32_t digit = item[r0 + r].x >> shift & mask;
                const uint32_t before = mine[digit];
                place[r0 + r] = before + __popc(peers[r] & lower);
                __syncwarp();
                if ((peers[r] & lower) == 0) mine[digit] = (uint16_t)(before + __popc(peers[r]));
                __syncwarp();
            }
        }
        __syncthreads();
        // per pair of digits: exclusive sum over the warps, and the block's totals to every block of the cluster
        if (threadIdx.x < bins / 2) {
            uint32_t run = 0;     // two 16-bit sums; a block has at most 2^13 items
#pragma unroll 8
            for (int w = 0; w < kSortBlockWarps; ++w) {
                const uint32_t c = counts[w * (bins / 2) + threadIdx.x];
                counts[w * (bins / 2) + threadIdx.x] = run;
                run += c;
            }
            for (uint32_t b = 0; b < blocks; ++b)
                reinterpret_cast<uint32_t*>(cluster.map_shared_rank(totals, b))[rank * (bins / 2) + threadIdx.x] = run;
        }
        auto arrived = cluster.barrier_arrive();
        __syncthreads();
        // the block's own items in digit order, where the counters were
        const uint32_t own = threadIdx.x < bins ? totals[rank * bins + threadIdx.x] : 0;
        const uint32_t own_start = block_exclusive(own, sh.warp_sums, nullptr);
#pragma unroll
        for (int r = 0; r < kItems; ++r) {
            const uint32_t digit = item[r].x >> shift & mask;
            place[r] += mine[digit];
        }
        if (threadIdx.x < bins) sh.digit_base[threadIdx.x] = own_start;
        __syncthreads();
#pragma unroll
        for (int r = 0; r < kItems; ++r) staged[sh.digit_base[item[r].x >> shift & mask] + place[r]] = item[r];
        cluster.barrier_wait(std::move(arrived));   // every block's totals are here, and every block has read its items
        uint32_t sum = 0, before = 0;
        if (threadIdx.x < bins)
            for (uint32_t b = 0; b < blocks; ++b) {
                const uint32_t c = totals[b * bins + threadIdx.x];
                if (b < rank) before += c;
                sum += c;
            }
        const uint32_t digit_start = block_exclusive(sum, sh.warp_sums, nullptr);
        if (threadIdx.x < bins) sh.digit_base[threadIdx.x] = digit_start + before - own_start;   // from staged place to final place
        __syncthreads();
#pragma unroll
        for (int r = 0; r < kItems; ++r) {
            const uint32_t at = r * kSortBlock + threadIdx.x;
            const uint2 it = staged[at];
            const uint32_t to = sh.digit_base[it.x >> shift & mask] + at;
            cluster.map_shared_rank(items, to / kPerBlock)[to % kPerBlock] = it;
        }
        cluster.sync();
#pragma unroll
        for (int r = 0; r < kItems; ++r) item[r] = items[my + r * 32];
    }
    // this block now holds sorted positions [first, first + kPerBlock): mark the first position of every token
    uint32_t previous = 0xFFFFFFFFu;                   // of the warp's first item
    if (lane == 0) {
        if (my) previous = items[my - 1].x;
        else if (rank) previous = cluster.map_shared_rank(items, rank - 1)[kPerBlock - 1].x;
    }
    uint32_t head_bits = 0, n_valid = 0, n_heads = 0;
#pragma unroll
    for (int r = 0; r < kItems; ++r) {
        const uint32_t left = __shfl_up_sync(0xFFFFFFFFu, item[r].x, 1);
        const bool valid = item[r].x < t.V;
        const bool head = valid && item[r].x != (lane ? left : previous);
        previous = __shfl_sync(0xFFFFFFFFu, item[r].x, 31);
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
            if (i % kSpan == 0) s.span_rank[i / kSpan] = h;
        }
    }
    if (rank == 0 && threadIdx.x == 0) {
        s.info[0] = all_valid;
        s.info[1] = all_heads;
        s.info[2] = 0;
        s.seg_start[all_heads] = all_valid;
    }
}

// Blocks that clear: one per 64 KB, at most four per multiprocessor (they are handed out as others end), in whole clusters.
uint32_t clear_blocks(const ClearRows& c, int sms, uint32_t cluster) {
    if (!c.rows) return 0;
    const uint64_t want = (c.rows * c.width + 65535) / 65536, most = (uint64_t)sms * 4;
    return (uint32_t)(((want < most ? want : most) + cluster - 1) / cluster * cluster);
}

__global__ void __launch_bounds__(kSortBlock) k_clear(ClearRows c) { clear_part(c, blockIdx.x, gridDim.x); }

template <int kItems>
cudaLaunchConfig_t cluster_launch(cudaStream_t stream, uint32_t blocks, uint32_t digit_bits, cudaLaunchAttribute* attr) {
    attr->id = cudaLaunchAttributeClusterDimension;
    attr->val.clusterDim.x = blocks;
    attr->val.clusterDim.y = attr->val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = blocks;
    cfg.blockDim = kSortBlock;
    cfg.dynamicSmemBytes = cluster_shared_bytes<kItems>((size_t)1 << digit_bits, blocks);
    cfg.stream = stream;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cfg;
}

// What k_cluster_sort<kItems> needs set on a device before its first launch there; returns the largest cluster it may have.
template <int kItems>
cudaError_t prepare_cluster(int device, uint32_t* most) {
    static std::atomic<uint32_t> known[kMaxDevices];
    *most = device < kMaxDevices ? known[device].load(std::memory_order_relaxed) : 0;
    if (*most) return cudaSuccess;
    cudaError_t e = cudaFuncSetAttribute(k_cluster_sort<kItems>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                         (int)cluster_shared_bytes<kItems>(1 << kMaxDigitBits, kMaxCluster));
    if (e != cudaSuccess) return e;
    *most = kPortableCluster;
    if (cudaFuncSetAttribute(k_cluster_sort<kItems>, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) == cudaSuccess) {
        cudaLaunchAttribute attr[1];
        const cudaLaunchConfig_t cfg = cluster_launch<kItems>(nullptr, kMaxCluster, kMaxDigitBits, attr);
        int clusters = 0;
        if (cudaOccupancyMaxActiveClusters(&clusters, k_cluster_sort<kItems>, &cfg) == cudaSuccess && clusters > 0) *most = kMaxCluster;
    }
    cudaGetLastError();       // a refusal of the larger cluster is no error
    if (device < kMaxDevices) known[device].store(*most, std::memory_order_relaxed);
    return cudaSuccess;
}

template <int kItems>
cudaError_t cluster_sort(cudaStream_t stream, const TokenIds& t, const SortedTokens& s, uint32_t key_bits, int device,
                         const ClearRows& clear, int sms, bool* done) {
    uint32_t most;
    const cudaError_t e = prepare_cluster<kItems>(device, &most);
    if (e != cudaSuccess) return e;
    uint32_t blocks = 1;
    while (blocks < most && blocks * kSortBlock * kItems < t.n) blocks *= 2;
    if (blocks * kSortBlock * kItems < t.n) return cudaSuccess;
    *done = true;
    const uint32_t passes = (key_bits + kMaxDigitBits - 1) / kMaxDigitBits, digit_bits = (key_bits + passes - 1) / passes;
    cudaLaunchAttribute attr[1];
    cudaLaunchConfig_t cfg = cluster_launch<kItems>(stream, blocks, digit_bits, attr);
    cfg.gridDim.x += clear_blocks(clear, sms, blocks);
    return cudaLaunchKernelEx(&cfg, k_cluster_sort<kItems>, t, s, key_bits, digit_bits, clear);
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
            if (i % kSpan == 0) s.span_rank[i / kSpan] = h;
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
            if (i == 0) s.info[2] = 0;
        }
        run += heads;
    }
}

}  // namespace

bool sorts_in_one_launch(uint32_t n) { return n <= kPortableCluster * kSortBlock * kMaxItems; }

cudaError_t launch_clear(cudaStream_t stream, const ClearRows& c, int sms) {
    k_clear<<<clear_blocks(c, sms, 1), kSortBlock, 0, stream>>>(c);
    return cudaGetLastError();
}

cudaError_t launch_token_sort(cudaStream_t stream, const TokenIds& t, const SortedTokens& s, const SortScratch& w,
                              const ClearRows& c, int sms) {
    uint32_t key_bits = 1;
    while (key_bits < 32 && t.V >> key_bits) ++key_bits;
    int device = 0;
    cudaError_t e = cudaGetDevice(&device);
    if (e != cudaSuccess) return e;
    bool done = false;         // with the fewest items per thread that a cluster can hold the batch with
    if (t.n <= kMaxCluster * kSortBlock) e = cluster_sort<1>(stream, t, s, key_bits, device, c, sms, &done);
    if (e == cudaSuccess && !done && t.n <= kMaxCluster * kSortBlock * 2) e = cluster_sort<2>(stream, t, s, key_bits, device, c, sms, &done);
    if (e == cudaSuccess && !done && t.n <= kMaxCluster * kSortBlock * 4) e = cluster_sort<4>(stream, t, s, key_bits, device, c, sms, &done);
    if (e == cudaSuccess && !done && t.n <= kMaxCluster * kSortBlock * 8) e = cluster_sort<8>(stream, t, s, key_bits, device, c, sms, &done);
    if (e != cudaSuccess || done) return e;
    if (c.rows) {
        e = launch_clear(stream, c, sms);
        if (e != cudaSuccess) return e;
    }
    uint64_t launches = 0;
    Launcher L{stream, &launches, 0, nullptr};
    L.lim.err = s.info;    // only read by the checked build's scatter, whose positions are below n by construction
    k_token_items<<<(t.n + kTileThreads - 1) / kTileThreads, kTileThreads, 0, stream>>>(t, w.a);
    item_t* sorted = nullptr;
    e = launch_sort(L, w.a, w.b, t.n, key_bits, w.hist, &sorted);
    if (e != cudaSuccess) return e;
    const uint32_t tiles = (t.n + kTileItems - 1) / kTileItems;
    k_count_tokens<<<tiles, kTileThreads, 0, stream>>>(sorted, t.n, t.V, w.tile_counts);
    k_write_tokens<<<tiles, kTileThreads, 0, stream>>>(sorted, t.n, t.V, w.tile_counts, s);
    return cudaGetLastError();
}

}  // namespace tensair
