// The sums by token of short batches, up to 1,024 positions, in one launch: what a long batch takes three launches for (sort,
// sums, joining) is bound by their latencies when there is little to add up.  Every block sorts the whole batch in its shared
// memory and then adds up its own few columns for all tokens: the sort is repeated, but beside itself, and nothing has to be
// exchanged.
//
// Up to 256 positions a block has 256 threads, and a position's place is the number of positions before it, counted by comparing it
// with all others; beyond, a block of 1,024 threads runs the radix sort's passes.  A token with more than 16 positions is added up
// in pieces by several threads, which leave their sums in shared memory to be joined in order.
//
// Bound by latency.  Added to the table, d = 1,024: 1 token 4.2 us, 128 tokens 6 to 8 us, 256 10.3 us, 512 11 us, 1,024 12.4 us; the
// launches for long batches take 14.4 us for 129 tokens and 16.4 us for 512 to 1,024.
#include <atomic>
#include <cstddef>

#include "embedding.cuh"
#include "token_sort.cuh"

namespace tensair {

namespace {

constexpr uint32_t kFewTokens = 256;
constexpr uint32_t kShortVecs = 4;     // most vectors of columns of a block

// kThreads positions at most.
template <int kThreads>
struct ShortShared {
    uint2 items[kThreads];             // (token, position), in sorted order
    uint32_t pos[kThreads];
    uint32_t warp_sums[32];
    uint32_t digit_base[kThreads == 1024 ? 1 << kMaxDigitBits : 1];
    alignas(16) uint2 parts[kThreads]; // (first | rows << 11 | slot << 17 | piece << 31, token's rank)
    uint16_t large[kThreads / 17 + 1]; // parts that are the first piece of a token
    uint32_t n_large;
};
static_assert(offsetof(ShortShared<kFewTokens>, parts) % 16 == 0, "the keys that are compared lie there first, four to a read");
static_assert(offsetof(ShortShared<1024>, digit_base) % 8 == 0, "totals are written two at a time");
// After it: counters of the radix sort (kThreads 1,024), then the sums of the pieces: [slot][columns of the block].
template <int kThreads>
constexpr uint32_t kMaxPieces = kThreads / 16 + kThreads / 17 + 1;

template <SumKind kKind, typename TG, typename TO, typename C, int kThreads>
__global__ void __launch_bounds__(kThreads)
k_short_sums(const __grid_constant__ SumArgs a, TokenIds t, uint32_t all_vecs, uint32_t slab_vecs, uint32_t key_bits, uint32_t digit_bits) {
    constexpr int E = C::E;
    extern __shared__ __align__(16) uint8_t raw[];
    ShortShared<kThreads>& sh = *reinterpret_cast<ShortShared<kThreads>*>(raw);
    uint8_t* rest = raw + (sizeof(ShortShared<kThreads>) + 15) / 16 * 16;
    const uint32_t tid = threadIdx.x, n = t.n;
    const uint32_t vec0 = blockIdx.x * slab_vecs, vecs = all_vecs - vec0 < slab_vecs ? all_vecs - vec0 : slab_vecs;
    if (tid == 0) sh.n_large = 0;
    // ---- sort: thread i ends with sorted position i
    uint2 item = make_uint2(tid < n ? token_key(t, tid) : 0xFFFFFFFFu, tid);
    if constexpr (kThreads == 1024) {
        const uint32_t bins = 1u << digit_bits, mask = bins - 1;
        uint32_t* counts = reinterpret_cast<uint32_t*>(rest);
        for (uint32_t shift = 0; shift < key_bits; shift += digit_bits) {
            const uint32_t digit = item.x >> shift & mask;
            const uint32_t place = block_rank(digit, digit_bits, counts, [&](uint32_t x, uint32_t two) {
                reinterpret_cast<uint2*>(sh.digit_base)[x] = make_uint2(two & 0xFFFFu, two >> 16);
            });
            const uint32_t total = tid < bins ? sh.digit_base[tid] : 0;
            const uint32_t start = block_exclusive(total, sh.warp_sums, nullptr);
            if (tid < bins) sh.digit_base[tid] = start;
            __syncthreads();
            const uint32_t to = sh.digit_base[digit] + place;
            if (in_bounds(t.err, to, kThreads)) sh.items[to] = item;
            __syncthreads();
            item = sh.items[tid];
        }
    } else {
        uint32_t* keys = reinterpret_cast<uint32_t*>(sh.parts);
        keys[tid] = item.x;
        __syncthreads();
        uint32_t place = 0;
        const uint4* four = reinterpret_cast<const uint4*>(keys);
#pragma unroll 8
        for (uint32_t x = 0; 4 * x < n; ++x) {
            const uint4 k = four[x];
            place += (k.x < item.x || (k.x == item.x && 4 * x < tid)) + (k.y < item.x || (k.y == item.x && 4 * x + 1 < tid)) +
                     (k.z < item.x || (k.z == item.x && 4 * x + 2 < tid)) + (k.w < item.x || (k.w == item.x && 4 * x + 3 < tid));
        }
        const uint32_t to = tid < n ? place : tid;     // places past the batch stay where they are
        if (in_bounds(t.err, to, kThreads)) sh.items[to] = item;
        __syncthreads();
        item = sh.items[tid];
    }
    // ---- the tokens and their parts
    sh.pos[tid] = tid >= n || in_bounds(t.err, item.y, n) ? item.y : 0;
    const bool valid = item.x < t.V;
    const bool head = valid && (tid == 0 || sh.items[tid - 1].x != item.x);
    uint32_t tokens;
    const uint32_t rank = block_exclusive(head, sh.warp_sums, &tokens) + head - 1;
    const uint32_t n_valid = __syncthreads_count(valid);
    uint16_t* starts = reinterpret_cast<uint16_t*>(rest);       // the counters are done with
    if (head) starts[rank] = (uint16_t)tid;
    if (tid == 0) starts[tokens] = (uint16_t)n_valid;
    __syncthreads();
    uint32_t start = 0, len = 0;
    if (valid) {
        start = starts[rank];
        len = starts[rank + 1] - start;
    }
    const bool piece = len > kWindow && (tid - start) % kWindow == 0, part = valid && (piece || (head && len <= kWindow));
    uint32_t n_parts, pieces;
    const uint32_t index = block_exclusive(part, sh.warp_sums, &n_parts);
    const uint32_t slot = block_exclusive(piece, sh.warp_sums, &pieces);
    if (part) {
        const uint32_t left = start + len - tid, rows = left < kWindow ? left : kWindow;
        sh.parts[index] = make_uint2(tid | rows << 11 | slot << 17 | (uint32_t)piece << 31, rank);
        if (piece && head) sh.large[atomicAdd(&sh.n_large, 1u)] = (uint16_t)index;      // the list's order changes no sum
    }
    float* sums = reinterpret_cast<float*>(rest + (size_t)(kThreads + 2) * 2 / 16 * 16 + 16);
    __syncthreads();
    // ---- their rows
    after_previous_launch();      // the launch that clears the table, if there is one
    float grad_scale = 1.0f;
    if (kKind == kSumAdamw && !adamw_grad_scale(a.adamw, &grad_scale)) return;
    if (kKind == kSumRows && blockIdx.x == 0 && tid == 0) *a.out_count = tokens;
    for (uint32_t w = tid; w < n_parts * vecs; w += kThreads) {
        const uint32_t q = w / vecs, vec = w - q * vecs, col = (vec0 + vec) * E;
        const uint2 p = sh.parts[q];
        const uint32_t first = p.x & 0x7FF, rows = p.x >> 11 & 0x3F, key = sh.items[first].x;
        if (!in_bounds(t.err, first + rows, n + 1) || !in_bounds(t.err, key, t.V)) continue;
        Finish<kKind, TO, C> row;
        if (!(p.x >> 31)) row.fetch(a, key, col);
        float sum[E];
        add_rows<kKind, C>((const TG*)a.grad.data + col, a.grad.stride, sh.pos + first, rows, a.d - col, sum);
        if (!(p.x >> 31)) row.put(a, grad_scale, key, p.y, col, sum);
        else if (in_bounds(t.err, p.x >> 17 & 0x3FFF, kMaxPieces<kThreads>))
            store_pack<float, E>(sums + ((p.x >> 17 & 0x3FFF) * slab_vecs + vec) * E, sum);
    }
    if (!pieces) return;
    __syncthreads();
    for (uint32_t w = tid; w < sh.n_large * vecs; w += kThreads) {
        const uint32_t q = w / vecs, vec = w - q * vecs, col = (vec0 + vec) * E;
        const uint2 p = sh.parts[sh.large[q]];
        const uint32_t first = p.x & 0x7FF, key = sh.items[first].x;
        const uint32_t slot0 = p.x >> 17 & 0x3FFF, count = (starts[p.y + 1] - first + kWindow - 1) / kWindow;
        if (!in_bounds(t.err, slot0 + count, kMaxPieces<kThreads> + 1) || !in_bounds(t.err, key, t.V)) continue;
        Finish<kKind, TO, C> row;
        row.fetch(a, key, col);
        float sum[E];
#pragma unroll
        for (int e = 0; e < E; ++e) sum[e] = 0.0f;
        for (uint32_t x = 0; x < count; ++x) {
            const Pack<float, E> y = load_pack<float, E>(sums + ((slot0 + x) * slab_vecs + vec) * E);
#pragma unroll
            for (int e = 0; e < E; ++e) sum[e] += y.v[e];
        }
        row.put(a, grad_scale, key, p.y, col, sum);
    }
}

template <SumKind kKind, typename TG, typename TO, typename C, int kThreads>
cudaError_t launch_short(cudaStream_t stream, const SumArgs& a, const TokenIds& t, uint32_t sms) {
    uint32_t key_bits = 1;
    while (key_bits < 32 && t.V >> key_bits) ++key_bits;
    const uint32_t passes = (key_bits + kMaxDigitBits - 1) / kMaxDigitBits, digit_bits = (key_bits + passes - 1) / passes;
    const uint32_t vecs = (a.d + C::E - 1) / C::E;
    const size_t starts = (size_t)(kThreads + 2) * 2 / 16 * 16 + 16, sums = (size_t)kMaxPieces<kThreads> * kShortVecs * C::E * 4;
    const size_t counters = kThreads == 1024 ? (size_t)kSortBlockWarps * 2 << digit_bits : 0;
    const size_t shared = (sizeof(ShortShared<kThreads>) + 15) / 16 * 16 + (starts + sums > counters ? starts + sums : counters);
    auto kernel = k_short_sums<kKind, TG, TO, C, kThreads>;
    if (shared > 48 * 1024) {
        static std::atomic<uint64_t> allowed{0};
        int device = 0;
        cudaError_t e = cudaGetDevice(&device);
        if (e == cudaSuccess && (device >= 64 || !(allowed.load(std::memory_order_relaxed) >> device & 1))) {
            e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, 128 * 1024);
            if (e == cudaSuccess && device < 64) allowed.fetch_or(1ull << device, std::memory_order_relaxed);
        }
        if (e != cudaSuccess) return e;
    }
    // one vector to a block while there are multiprocessors for that: the blocks sort beside one another anyway
    uint32_t slab_vecs = (vecs + sms - 1) / sms;
    if (slab_vecs > kShortVecs) slab_vecs = kShortVecs;
    const uint32_t blocks = (vecs + slab_vecs - 1) / slab_vecs;
    if (kKind == kSumTable && !a.accumulate) return launch_early(kernel, blocks, kThreads, shared, stream, a, t, vecs, slab_vecs, key_bits, digit_bits);
    kernel<<<blocks, kThreads, shared, stream>>>(a, t, vecs, slab_vecs, key_bits, digit_bits);
    return cudaGetLastError();
}

}  // namespace

bool is_short(uint32_t n) { return n <= 1024; }

cudaError_t launch_short_sums(cudaStream_t stream, SumKind kind, const SumArgs& a, const TokenIds& t, int sms) {
    return with_sum(kind, a, [&](auto k, auto tg, auto to, auto c) {
        using TG = decltype(tg);
        using TO = decltype(to);
        using C = decltype(c);
        if (t.n <= kFewTokens) return launch_short<decltype(k)::value, TG, TO, C, kFewTokens>(stream, a, t, sms);
        return launch_short<decltype(k)::value, TG, TO, C, 1024>(stream, a, t, sms);
    });
}

}  // namespace tensair
