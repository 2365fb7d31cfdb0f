// The positions of a batch sorted by token (stable), with the segments of equal tokens: what the embedding gradient
// sums by.  Positions that hold no token (padding, ids outside [0,V)) sort behind all others, as key V.
//
// A radix sort with one item per thread in blocks of 1,024, so that ranking (some 50 integer instructions per item and pass,
// which is what a block's time goes into) is spread over as many multiprocessors as there are items for.  Digits are
// as wide as the counters allow: ten bits, two passes up to V = 2^20 - 1.
//   up to 2^14 positions   one launch of one thread-block cluster.  The items stay in the cluster's shared memory; every pass
//                          exchanges the digit totals through distributed shared memory and writes the items straight into
//                          the shared memory of the block that owns their place.  Bound by the latency of its barriers:
//                          2,048 tokens 8.8 us, 4,096 9.3 us, 16,384 12.5 us (V = 100,000).
//   up to 2^17             two launches per pass, rank and scatter, and one that lists the tokens; items and totals go through
//                          the level-2 cache, and every block adds up the totals it needs itself.  Each launch begins
//                          while the one before it runs.  32,768 tokens 17.7 us, 65,536 22.2 us, 131,072 31.8 us (V = 1 M); in one
//                          cluster, with 4 items per thread, 65,536 took 27 us; 16,384 took 14 us this way.
//   beyond                 the library's multi-launch radix sort (262,144 tokens 78 us), whose totals are scanned by a launch of their
//                          own.
#include <cooperative_groups.h>

#include <atomic>
#include <utility>

#include "kernels.h"
#include "operators.h"
#include "token_sort.cuh"

namespace cg = cooperative_groups;

namespace tensair {

namespace {

constexpr uint32_t kMaxCluster = 16;                           // needs leave of the device; 8 always works
constexpr uint32_t kPortableCluster = 8;
constexpr uint32_t kMaxTiles = kTiledSort / kSortBlock;        // blocks of the sort in several launches

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

__device__ __forceinline__ uint32_t most_tokens(uint32_t n, uint32_t V) { return n < V ? n : V; }   // distinct ones; seg_start has one place more

struct ClusterShared {
    uint32_t warp_sums[kSortBlockWarps];
    uint32_t heads[kMaxCluster], valid[kMaxCluster];   // of every block of the cluster, written by that block
    uint32_t digit_base[1 << kMaxDigitBits];
    uint2 items[kSortBlock];                           // (key, position)
};
constexpr size_t counts_bytes(size_t bins) { return kSortBlockWarps * bins * 2; }
constexpr size_t cluster_shared_bytes(size_t bins, size_t blocks) {
    return sizeof(ClusterShared) + counts_bytes(bins) + blocks * bins * 2;     // ..., digit totals of every block
}

__global__ void __launch_bounds__(kSortBlock, 1)
k_cluster_sort(TokenIds t, SortedTokens s, uint32_t key_bits, uint32_t digit_bits) {
    cg::cluster_group cluster = cg::this_cluster();
    let_next_launch_begin();
    // Another block's shared memory may be written only once that block is known to have started: every block says so here, and
    // all wait for it behind the read of the ids, before the first pass's totals go out.
    auto started = cluster.barrier_arrive();
    const uint32_t rank = cluster.block_rank(), blocks = cluster.num_blocks();
    extern __shared__ __align__(16) uint8_t raw[];
    const uint32_t bins = 1u << digit_bits, mask = bins - 1, tid = threadIdx.x;
    ClusterShared& sh = *reinterpret_cast<ClusterShared*>(raw);
    uint32_t* counts = reinterpret_cast<uint32_t*>(raw + sizeof(ClusterShared));
    uint16_t* totals = reinterpret_cast<uint16_t*>(counts) + kSortBlockWarps * bins;   // [block][digit]
    const uint32_t at = rank * kSortBlock + tid;
    // places past the batch sort behind everything, in order
    uint2 item = make_uint2(at < t.n ? token_key(t, at) : 0xFFFFFFFFu, at);
    cluster.barrier_wait(std::move(started));
    for (uint32_t shift = 0; shift < key_bits; shift += digit_bits) {
        const uint32_t digit = item.x >> shift & mask;
        const uint32_t place = block_rank(digit, digit_bits, counts, [&](uint32_t x, uint32_t two) {
            for (uint32_t b = 0; b < blocks; ++b) reinterpret_cast<uint32_t*>(cluster.map_shared_rank(totals, b))[rank * (bins / 2) + x] = two;
        });
        cluster.sync();   // every block's totals are here, and every block has read its items
        uint32_t sum = 0, before = 0;
        if (tid < bins)
            for (uint32_t b = 0; b < blocks; ++b) {
                const uint32_t c = totals[b * bins + tid];
                if (b < rank) before += c;
                sum += c;
            }
        const uint32_t digit_start = block_exclusive(sum, sh.warp_sums, nullptr);
        if (tid < bins) sh.digit_base[tid] = digit_start + before;
        __syncthreads();
        const uint32_t to = sh.digit_base[digit] + place;
        if (in_bounds(t.err, to, blocks * kSortBlock)) cluster.map_shared_rank(sh.items, to / kSortBlock)[to % kSortBlock] = item;
        cluster.sync();
        item = sh.items[tid];
    }
    // the thread now holds sorted position `at`: mark the first position of every token
    uint32_t previous = 0xFFFFFFFFu;
    if (tid) previous = sh.items[tid - 1].x;
    else if (rank) previous = cluster.map_shared_rank(sh.items, rank - 1)[kSortBlock - 1].x;
    const bool valid = item.x < t.V, head = valid && item.x != previous;
    uint32_t block_heads;
    uint32_t before = block_exclusive(head, sh.warp_sums, &block_heads);
    const uint32_t block_valid = __syncthreads_count(valid);
    if (tid < blocks) {
        cluster.map_shared_rank(sh.heads, tid)[rank] = block_heads;
        cluster.map_shared_rank(sh.valid, tid)[rank] = block_valid;
    }
    cluster.sync();       // no block reads another one's shared memory after this
    uint32_t all_heads = 0, all_valid = 0;
    for (uint32_t b = 0; b < blocks; ++b) {
        if (b < rank) before += sh.heads[b];
        all_heads += sh.heads[b];
        all_valid += sh.valid[b];
    }
    const uint32_t most = most_tokens(t.n, t.V);
    if (at < t.n) {
        s.key[at] = item.x;
        s.pos[at] = item.y;
        if (head && in_bounds(t.err, before, most)) s.seg_start[before] = at;
        if (at % kSpan == 0) s.span_rank[at / kSpan] = before;
    }
    if (at == 0) {
        s.info[0] = all_valid;
        s.info[1] = all_heads;
        s.info[2] = s.info[3] = 0;
        if (in_bounds(t.err, all_heads, most + 1)) s.seg_start[all_heads] = all_valid;
    }
    after_previous_launch();     // the launch that clears the table, if there is one, has run beside this one and ends with it
}

// ---- in several launches.  Each takes a share of the rows to clear: its blocks past the tiles clear beside the others.
struct ClearShare {
    ClearRows rows;
    uint32_t share, shares;
    __device__ __forceinline__ void run(uint32_t tiles) const {
        const uint64_t blocks = gridDim.x - tiles;
        clear_part(rows, share * blocks + blockIdx.x - tiles, shares * blocks);
    }
};

// What these kernels read was written while they were already waiting, so their parameters are not marked const __restrict__: that
// would allow the compiler reads that count on memory which no one changes while the kernel runs.  Each lets its successor begin
// only behind its own wait: no launch is ever more than one ahead of the one that runs.
//
// A tile is the 1,024 items of a block; hist: [tile][digit], 16 bits each.
// Ranks the tile's items of a pass by digit: place[i] is the rank among the tile's items of its digit.
template <bool kFirst>
__global__ void __launch_bounds__(kSortBlock)
k_tile_rank(TokenIds t, const uint2* items, uint2* out, uint16_t* place, uint32_t* hist, uint32_t shift, uint32_t digit_bits,
            uint32_t tiles, ClearShare clear) {
    extern __shared__ __align__(16) uint32_t counts[];
    if (!kFirst) after_previous_launch();
    let_next_launch_begin();
    if (blockIdx.x >= tiles) return clear.run(tiles);
    const uint32_t at = blockIdx.x * kSortBlock + threadIdx.x, pairs = 1u << digit_bits >> 1;
    uint32_t key = 0xFFFFFFFFu;
    if (at < t.n) {
        key = kFirst ? token_key(t, at) : items[at].x;
        if (kFirst) out[at] = make_uint2(key, at);
    }
    const uint32_t rank = block_rank(key >> shift & (2 * pairs - 1), digit_bits, counts,
                                     [&](uint32_t x, uint32_t two) { hist[blockIdx.x * pairs + x] = two; });
    if (at < t.n) place[at] = (uint16_t)rank;
}

// Moves the items to where the pass has them; the last pass writes keys and positions apart.
template <bool kLast>
__global__ void __launch_bounds__(kSortBlock)
k_tile_scatter(uint32_t n, const uint2* items, uint2* out, const uint16_t* place, const uint16_t* hist, uint32_t shift,
               uint32_t digit_bits, uint32_t tiles, SortedTokens s, ClearShare clear) {
    __shared__ uint32_t base[1 << kMaxDigitBits], warp_sums[kSortBlockWarps];
    const uint32_t tid = threadIdx.x, at = blockIdx.x * kSortBlock + tid, bins = 1u << digit_bits;
    after_previous_launch();
    let_next_launch_begin();
    if (blockIdx.x >= tiles) return clear.run(tiles);
    uint2 item = make_uint2(0, 0);
    uint32_t rank = 0;
    if (at < n) {
        item = items[at];
        rank = place[at];
    }
    uint32_t all = 0, before = 0;      // items of the digit in all tiles, and in the tiles before this one
    if (tid < bins) {
#pragma unroll 16
        for (uint32_t x = 0; x < tiles; ++x) {
            const uint32_t c = hist[x * bins + tid];
            if (x < blockIdx.x) before += c;
            all += c;
        }
    }
    const uint32_t start = block_exclusive(all, warp_sums, nullptr);
    if (tid < bins) base[tid] = start + before;
    __syncthreads();
    if (at >= n) return;
    const uint32_t to = base[item.x >> shift & (bins - 1)] + rank;     // below n: the places past the batch come last
    if (!in_bounds(s.err, to, n)) return;
    if (kLast) {
        s.key[to] = item.x;
        s.pos[to] = item.y;
    } else out[to] = item;
}

// Lists the tokens of the sorted positions.  A block counts the tokens that begin before it from the keys themselves.
__global__ void __launch_bounds__(kSortBlock)
k_list_tokens(uint32_t n, uint32_t V, uint32_t tiles, SortedTokens s, ClearShare clear) {
    __shared__ uint32_t warp_sums[kSortBlockWarps];
    const uint32_t tid = threadIdx.x, first = blockIdx.x * kSortBlock, at = first + tid;
    after_previous_launch();
    let_next_launch_begin();
    if (blockIdx.x >= tiles) return clear.run(tiles);
    uint32_t c = 0;
    const uint4* keys = reinterpret_cast<const uint4*>(s.key);
#pragma unroll 8
    for (uint32_t x = tid; x < first / 4; x += kSortBlock) {
        const uint4 k = keys[x];
        const uint32_t left = x ? s.key[4 * x - 1] : 0xFFFFFFFFu;
        c += (k.x < V && k.x != left) + (k.y < V && k.y != k.x) + (k.z < V && k.z != k.y) + (k.w < V && k.w != k.z);
    }
    uint32_t run, heads;
    block_exclusive(c, warp_sums, &run);
    const uint32_t key = at < n ? s.key[at] : 0xFFFFFFFFu;
    const bool head = key < V && (at == 0 || s.key[at - 1] != key);
    const uint32_t h = run + block_exclusive(head, warp_sums, &heads);
    if (at >= n || !in_bounds(s.err, h + head, most_tokens(n, V) + 1)) return;
    if (head) s.seg_start[h] = at;
    if (at % kSpan == 0) s.span_rank[at / kSpan] = h;
    const bool ends = at + 1 == n || s.key[at + 1] >= V;
    if (key < V && ends) {             // the last position with a token
        s.info[0] = at + 1;
        s.info[1] = h + head;
        s.seg_start[h + head] = at + 1;
    }
    if (at == 0) {
        s.info[2] = s.info[3] = 0;
        if (key >= V) s.info[0] = s.info[1] = s.seg_start[0] = 0;
    }
}

// One block per multiprocessor: all start at once, so the launch that follows can run beside them.  102 MB take 18.5 us, 5.5 TB/s, alone
// (a memset 16.6), 26 with the sort of 16,384 tokens beside them.
constexpr int kClearThreads = 512;
__global__ void __launch_bounds__(kClearThreads) k_clear(ClearRows c) {
    let_next_launch_begin();
    clear_part(c, blockIdx.x, gridDim.x);
}

cudaLaunchConfig_t cluster_launch(cudaStream_t stream, uint32_t blocks, uint32_t digit_bits, cudaLaunchAttribute* attr) {
    attr->id = cudaLaunchAttributeClusterDimension;
    attr->val.clusterDim.x = blocks;
    attr->val.clusterDim.y = attr->val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = blocks;
    cfg.blockDim = kSortBlock;
    cfg.dynamicSmemBytes = cluster_shared_bytes((size_t)1 << digit_bits, blocks);
    cfg.stream = stream;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cfg;
}

// What the kernels need set on a device before their first launch there; *most: the largest cluster it may have.
cudaError_t prepare_device(uint32_t* most) {
    static std::atomic<uint32_t> known[kMaxDevices];
    int device = 0;
    cudaError_t e = cudaGetDevice(&device);
    if (e != cudaSuccess) return e;
    *most = device < kMaxDevices ? known[device].load(std::memory_order_relaxed) : 0;
    if (*most) return cudaSuccess;
    const int counts = (int)counts_bytes(1 << kMaxDigitBits);
    e = cudaFuncSetAttribute(k_cluster_sort, cudaFuncAttributeMaxDynamicSharedMemorySize,
                             (int)cluster_shared_bytes(1 << kMaxDigitBits, kMaxCluster));
    if (e == cudaSuccess) e = cudaFuncSetAttribute(k_tile_rank<true>, cudaFuncAttributeMaxDynamicSharedMemorySize, counts);
    if (e == cudaSuccess) e = cudaFuncSetAttribute(k_tile_rank<false>, cudaFuncAttributeMaxDynamicSharedMemorySize, counts);
    if (e != cudaSuccess) return e;
    *most = kPortableCluster;
    if (cudaFuncSetAttribute(k_cluster_sort, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) == cudaSuccess) {
        cudaLaunchAttribute attr[1];
        const cudaLaunchConfig_t cfg = cluster_launch(nullptr, kMaxCluster, kMaxDigitBits, attr);
        int clusters = 0;
        if (cudaOccupancyMaxActiveClusters(&clusters, k_cluster_sort, &cfg) == cudaSuccess && clusters > 0) *most = kMaxCluster;
    }
    cudaGetLastError();       // a refusal of the larger cluster is no error
    if (device < kMaxDevices) known[device].store(*most, std::memory_order_relaxed);
    return cudaSuccess;
}

cudaError_t sort_in_tiles(cudaStream_t stream, const TokenIds& t, const SortedTokens& s, const SortScratch& w, uint32_t key_bits,
                          uint32_t digit_bits, const ClearRows& clear, int sms) {
    const uint32_t tiles = (t.n + kSortBlock - 1) / kSortBlock;
    const size_t counts = counts_bytes((size_t)1 << digit_bits);
    uint2* from = reinterpret_cast<uint2*>(w.a);
    uint2* to = reinterpret_cast<uint2*>(w.b);
    uint16_t* place = reinterpret_cast<uint16_t*>(w.tile_counts);
    const uint32_t passes = (key_bits + digit_bits - 1) / digit_bits;
    ClearShare share{clear, 0, 2 * passes + 1};
    const uint32_t grid = tiles + (clear.rows ? (uint32_t)sms : 0u);
    for (uint32_t shift = 0; shift < key_bits; shift += digit_bits) {
        cudaError_t e;
        if (shift == 0) {
            k_tile_rank<true><<<grid, kSortBlock, counts, stream>>>(t, nullptr, from, place, w.hist, shift, digit_bits, tiles, share);
            e = cudaGetLastError();
        } else {
            e = launch_early(k_tile_rank<false>, grid, kSortBlock, counts, stream, t, (const uint2*)from, to, place, w.hist, shift,
                             digit_bits, tiles, share);
        }
        ++share.share;
        if (e != cudaSuccess) return e;
        auto scatter = shift + digit_bits < key_bits ? k_tile_scatter<false> : k_tile_scatter<true>;
        e = launch_early(scatter, grid, kSortBlock, 0, stream, t.n, (const uint2*)from, to, (const uint16_t*)place,
                         (const uint16_t*)w.hist, shift, digit_bits, tiles, s, share);
        ++share.share;
        if (e != cudaSuccess) return e;
        std::swap(from, to);
    }
    return launch_early(k_list_tokens, grid, kSortBlock, 0, stream, t.n, t.V, tiles, s, share);
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
        if (in && in_bounds(s.err, h + head, most_tokens(n, V) + 1)) {
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
            if (i == 0) s.info[2] = s.info[3] = 0;
        }
        run += heads;
    }
}

}  // namespace

SortScratchBytes sort_scratch_bytes(uint32_t n) {
    SortScratchBytes b = {0, 0, 0};
    if (n <= kPortableCluster * kSortBlock) return b;
    b.items = (size_t)n * 8;
    if (n <= kMaxTiles * kSortBlock) {
        b.hist = ((size_t)n + kSortBlock - 1) / kSortBlock * (2 << kMaxDigitBits);
        b.tile_counts = (size_t)n * 2;
    } else {
        b.hist = (size_t)sort_hist_words(n) * 4;
        b.tile_counts = ((size_t)n + kTileItems - 1) / kTileItems * 4;
    }
    return b;
}

cudaError_t launch_clear(cudaStream_t stream, const ClearRows& c, int sms) {
    k_clear<<<sms, kClearThreads, 0, stream>>>(c);
    return cudaGetLastError();
}

cudaError_t launch_token_sort(cudaStream_t stream, const TokenIds& t, const SortedTokens& s, const SortScratch& w,
                              const ClearRows& c, int sms) {
    uint32_t key_bits = 1, most = 0;
    while (key_bits < 32 && t.V >> key_bits) ++key_bits;
    const uint32_t passes = (key_bits + kMaxDigitBits - 1) / kMaxDigitBits, digit_bits = (key_bits + passes - 1) / passes;
    cudaError_t e = prepare_device(&most);
    if (e != cudaSuccess) return e;
    if (t.n <= most * kSortBlock) {
        uint32_t blocks = 1;
        while (blocks * kSortBlock < t.n) blocks *= 2;
        cudaLaunchAttribute attr[2];
        cudaLaunchConfig_t cfg = cluster_launch(stream, blocks, digit_bits, attr);
        if (c.rows) {          // beside the launch that clears
            e = launch_clear(stream, c, sms);
            if (e != cudaSuccess) return e;
            attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
            attr[1].val.programmaticStreamSerializationAllowed = 1;
            cfg.numAttrs = 2;
        }
        return cudaLaunchKernelEx(&cfg, k_cluster_sort, t, s, key_bits, digit_bits);
    }
    if (t.n <= kMaxTiles * kSortBlock) return sort_in_tiles(stream, t, s, w, key_bits, digit_bits, c, sms);
    if (c.rows) {
        e = launch_clear(stream, c, sms);
        if (e != cudaSuccess) return e;
    }
    uint64_t launches = 0;
    Launcher L{stream, &launches, 0, nullptr};
    L.lim.err = s.err;     // of the checked build's scatter
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
