// Embedding lookup with scaling, and the sums by token that its gradient and the AdamW step of the touched rows are
// made of (for batches of more than 1,024 positions; embedding_short.cu has the others).
//
// Sums.  The batch's positions are sorted by token (token_sort.cu).  A block takes 64 sorted positions (and a slab of the
// columns), lists the tokens that begin there in shared memory, and each of its threads then works through (token,
// vector of columns) pairs: it adds up the token's gradient rows in fp32, in sorted order, and puts the finished row where
// it belongs: the gradient table, the message, or through the AdamW update.  A token with more than 16 positions is added
// up in pieces, one partial row per window of 16, and a second launch joins those in window order: no thread has more than
// 16 rows to add, whatever the tokens' frequencies are, and no sum depends on timing.
//
// What bounds it, 65,536 tokens of a Zipf vocabulary of 1 M, d = 300: scattered rows of 1,200 bytes.  Rows (fp32): 24 us for
// 112 MB, 4.7 TB/s.  AdamW (bf16 gradients, fp32 table and moments): 47 us for 237 MB, 5.0 TB/s; the reads and writes of those rows
// alone, in a kernel that does nothing else, take 45 us.  Shared memory is kept small because the reads in flight live in the
// level-1 cache beside it (40 KB per block: +14 us).  A short batch is bound by the latency of the launches: 4,096 tokens of
// 128 floats take 18 us in all, of which the sort takes 9.
#include "embedding.cuh"

namespace tensair {

namespace {

// ------------------------------------------------------------------ lookup
constexpr int kLookupThreads = 128;
constexpr int kLookupUnroll = 3;     // see below

// out[i] = scale * table[ids[i]]; a thread moves kLookupUnroll vectors of E elements, a block's width apart, whatever rows
// they belong to, so no lane is idle for any width.  First all their ids, then all their rows, then all stores.
// Bound by memory and the latency of its two reads in a row: 65,536 rows of 300 floats out of 1 M take 22.6 us, 5.0 TB/s (0.76
// of the measured copy rate; rows of 1,200 bytes in no order do not reach it); 65,536 rows of 255 bf16 23 us; one token
// 2.5 us, a launch.  Two, four, eight vectors a thread: 24.6, 22.6, 28 us, and 22.5, 24.7, 35 us for the odd rows; blocks of 256 and 512
// threads are slower (24, 25 us).
template <typename TT, typename TO, typename C>
__global__ void __launch_bounds__(kLookupThreads)
k_lookup(TokenIds t, uint32_t row0, const TT* __restrict__ table, uint64_t table_stride, TO* __restrict__ out,
         uint64_t out_stride, FastDiv vecs, uint32_t d, uint32_t total, float scale) {
    constexpr int E = C::E;
    const uint32_t base = blockIdx.x * (kLookupThreads * kLookupUnroll) + threadIdx.x;
    const TT* from[kLookupUnroll];
    Pack<TT, E> x[kLookupUnroll];
#pragma unroll
    for (int u = 0; u < kLookupUnroll; ++u) {
        const uint32_t w = base + u * kLookupThreads;
        from[u] = nullptr;
        if (w < total) {
            const uint32_t r = vecs.div(w), col = (w - r * vecs.divisor) * E;
            const int64_t id = t.wide ? __ldg(reinterpret_cast<const long long*>(t.ids) + row0 + r)
                                      : __ldg(reinterpret_cast<const int32_t*>(t.ids) + row0 + r);
            if (t.is_token(id)) from[u] = table + (uint64_t)id * table_stride + col;
            else t.report(id);
        }
    }
#pragma unroll
    for (int u = 0; u < kLookupUnroll; ++u) {
        const uint32_t w = base + u * kLookupThreads;
        if (from[u]) x[u] = load_columns<C>(from[u], d - (w - vecs.div(w) * vecs.divisor) * E);
    }
#pragma unroll
    for (int u = 0; u < kLookupUnroll; ++u) {
        const uint32_t w = base + u * kLookupThreads;
        if (w >= total) break;
        const uint32_t r = vecs.div(w), col = (w - r * vecs.divisor) * E;
        float y[E];
#pragma unroll
        for (int e = 0; e < E; ++e) y[e] = from[u] ? to_float(x[u].v[e]) * scale : 0.0f;
        store_columns<C>(out + (uint64_t)(row0 + r) * out_stride + col, y, d - col);
    }
}

constexpr uint32_t kMaxItems = 0x7FFFFFFFu;   // vectors per launch, so that their numbers stay below 2^31

}  // namespace

cudaError_t launch_lookup(cudaStream_t stream, const TokenIds& t, const RowsView& table, const RowsView& out, uint32_t d,
                          float scale) {
    uint32_t e = vector_of(table, d, widest(table, out));
    e = vector_of(out, d, e);
    const FastDiv vecs(pieces_of(d, e));
    const uint32_t most = kMaxItems / vecs.divisor;     // rows of one launch
    for (uint32_t row0 = 0; row0 < t.n; row0 += most) {
        const uint32_t total = (t.n - row0 < most ? t.n - row0 : most) * vecs.divisor;
        const uint32_t grid = (uint32_t)(((uint64_t)total + kLookupThreads * kLookupUnroll - 1) / (kLookupThreads * kLookupUnroll));
        const cudaError_t err = with_type(table.type, [&](auto tt) {
            return with_type(out.type, [&](auto to) {
                return with_columns(e, [&](auto c) {
                    using TT = decltype(tt);
                    using TO = decltype(to);
                    k_lookup<TT, TO, decltype(c)><<<grid, kLookupThreads, 0, stream>>>(
                        t, row0, (const TT*)table.data, table.stride, (TO*)out.data, out.stride, vecs, d, total, scale);
                    return cudaGetLastError();
                });
            });
        });
        if (err != cudaSuccess) return err;
    }
    return cudaSuccess;
}

namespace {

// ------------------------------------------------------------------ sums by token
constexpr int kSumThreads = 256;
constexpr uint32_t kMaxParts = kSpan;  // every part begins at a position of its own
enum SumPart : uint32_t { kWholeToken, kPiece0, kPiece1 };   // pieces: see SumArgs::partials
constexpr uint32_t kSumBlocks = 4;   // blocks per multiprocessor aimed at
constexpr uint32_t kFewPieces = 8;     // after the first
constexpr int kJoinThreads = 256;
constexpr int kJoinWarps = kJoinThreads / 32;

template <SumKind kKind, typename TG, typename TO, typename C>
__global__ void __launch_bounds__(kSumThreads)
k_token_sums(const __grid_constant__ SumArgs a, uint32_t all_vecs, uint32_t slab_vecs) {
    constexpr int E = C::E;
    // What the block adds up, in order: (first position | rows << 8 | SumPart << 16 | piece's window << 24, token, rank).
    // No large shared arrays: the reads in flight need the level-1 cache, which shares its memory with them.
    __shared__ __align__(16) uint4 parts[kMaxParts];
    __shared__ uint32_t pos[kSpan + kWindow], head_masks[kSpan / 32], part_masks[kSpan / 32];
    const uint32_t tid = threadIdx.x, begin = blockIdx.x * kSpan;
    const uint32_t vec0 = blockIdx.y * slab_vecs;
    const uint32_t vecs = all_vecs - vec0 < slab_vecs ? all_vecs - vec0 : slab_vecs;
    after_previous_launch();
    let_next_launch_begin();
    float grad_scale = 1.0f;
    if (kKind == kSumAdamw && !adamw_grad_scale(a.adamw, &grad_scale)) return;
    const uint32_t n_valid = a.s.info[0];
    if (kKind == kSumRows && begin == 0 && vec0 == 0 && tid == 0) *a.out_count = a.s.info[1];
    if (begin >= n_valid || !in_bounds(a.s.err, n_valid, a.n + 1)) return;
    const uint32_t before = a.s.span_rank[blockIdx.x];           // tokens that begin before the span
    if (tid < kSpan + kWindow && begin + tid < n_valid) {
        const uint32_t p = a.s.pos[begin + tid];
        pos[tid] = in_bounds(a.s.err, p, a.n) ? p : 0;
    }
    const uint32_t at = begin + tid;
    const bool mine = tid < kSpan && at < n_valid;               // this thread has a position of the span
    uint32_t key = 0;
    bool head = false;
    if (tid < kSpan) {
        if (mine) {
            key = a.s.key[at];
            head = at == 0 || a.s.key[at - 1] != key;
        }
        const uint32_t heads = __ballot_sync(0xFFFFFFFFu, head);
        if (tid % 32 == 0) head_masks[tid / 32] = heads;
    }
    __syncthreads();
    // A token with up to kWindow positions is one part, in the span it begins in.  A larger one has a part, a piece, in
    // every window of kWindow positions that it reaches into.
    bool part = false;
    uint32_t first = tid, rows = 0, kind = kWholeToken, rank = 0;
    if (tid < kSpan) {
        if (mine) {
            const unsigned long long heads = (unsigned long long)head_masks[1] << 32 | head_masks[0];
            rank = before + __popcll(heads & (~0ull >> (63 - tid))) - 1;
        }
        if (mine && in_bounds(a.s.err, rank, a.n < a.V ? a.n : a.V) && in_bounds(a.s.err, key, a.V)) {
            const uint32_t start = a.s.seg_start[rank], end = a.s.seg_start[rank + 1];
            const bool large = end - start > kWindow;
            part = head || (large && tid % kWindow == 0);
            rows = end - at;
            if (large) {
                const uint32_t stop = kWindow - tid % kWindow;
                if (rows > stop) rows = stop;
                kind = head ? kPiece1 : kPiece0;
                if (head && blockIdx.y == 0) {
                    // many pieces: the list from its front; few: from its end.  The order in it changes no sum.
                    const uint32_t from = at / kWindow, to = (end - 1) / kWindow;
                    const bool many = to - from > kFewPieces;
                    const uint32_t slot = atomicAdd(a.s.info + (many ? 3 : 2), 1u);
                    if (in_bounds(a.s.err, slot, a.n / (kWindow + 1)))
                        a.large[many ? slot : a.n / (kWindow + 1) - 1 - slot] = make_uint4(from, rank, to, key);
                }
            }
        }
        const uint32_t mask = __ballot_sync(0xFFFFFFFFu, part);
        if (tid % 32 == 0) part_masks[tid / 32] = mask;
    }
    __syncthreads();
    const unsigned long long part_mask = (unsigned long long)part_masks[1] << 32 | part_masks[0];
    const uint32_t n_parts = __popcll(part_mask);
    if (part) parts[__popcll(part_mask & ((1ull << tid) - 1))] = make_uint4(first | rows << 8 | kind << 16 | (tid / kWindow) << 24, key, rank, 0);
    __syncthreads();
    // A thread takes every kSumThreads-th (part, vector) pair.
    const uint32_t step_q = kSumThreads / vecs, step_vec = kSumThreads - step_q * vecs;
    uint32_t q = tid / vecs, vec = tid - q * vecs;
    for (; q < n_parts; q += step_q, vec += step_vec) {
        if (vec >= vecs) {
            vec -= vecs;
            if (++q >= n_parts) break;
        }
        const uint4 p = parts[q];
        const uint32_t from = p.x & 0xFF, count = p.x >> 8 & 0xFF, what = p.x >> 16 & 0xFF;
        if (!in_bounds(a.s.err, from + count, kSpan + kWindow + 1)) continue;
        const uint32_t col = (vec0 + vec) * E;
        const TG* grad = (const TG*)a.grad.data + col;
        Finish<kKind, TO, C> row;
        if (what == kWholeToken) row.fetch(a, p.y, col);
        float sum[E];
        add_rows<kKind, C>(grad, a.grad.stride, pos + from, count, a.d - col, sum);
        if (what == kWholeToken) row.put(a, grad_scale, p.y, p.z, col, sum);
        else {
            const uint64_t slot = ((uint64_t)blockIdx.x * (kSpan / kWindow) + (p.x >> 24)) * 2 + (what == kPiece1);
            store_pack<float, E>(a.partials + slot * a.partial_stride + col, sum);
        }
    }
}

// Joins the pieces of the tokens with more than kWindow positions: slot 1 of the window a token begins in, then slot 0 of the
// windows that follow.  A token with few pieces takes a warp for each 32 vectors of columns, one with many takes a block, whose
// warps each add a stretch of the pieces.  7 us at the sizes above (300 such tokens, the largest with 300 pieces), mostly
// latency.  Joining them in the launch above instead, by the block that finishes last, made short batches slower (18 -> 23 us).
template <SumKind kKind, typename TO, typename C>
__global__ void __launch_bounds__(kJoinThreads)
k_join_pieces(const __grid_constant__ SumArgs a, uint32_t slabs) {
    constexpr int E = C::E;
    __shared__ float join[kJoinWarps][32 * E + 1];
    after_previous_launch();
    float grad_scale = 1.0f;
    if (kKind == kSumAdamw && !adamw_grad_scale(a.adamw, &grad_scale)) return;
    const uint32_t lane = threadIdx.x & 31, wid = threadIdx.x >> 5;
    const uint64_t few = ((uint64_t)a.s.info[2] * slabs + kJoinWarps - 1) / kJoinWarps, many = (uint64_t)a.s.info[3] * slabs;
    const uint64_t step = (uint64_t)2 * a.partial_stride;
    for (uint64_t w = blockIdx.x; w < many + few; w += gridDim.x) {
        const bool shared = w < many;      // the block's warps share a token
        const uint64_t item = shared ? w : (w - many) * kJoinWarps + wid;
        const uint32_t q = (uint32_t)(item / slabs);
        bool in = (shared || q < a.s.info[2]) && in_bounds(a.s.err, q, a.n / (kWindow + 1));
        uint4 c = make_uint4(0, 0, 0, 0);
        if (in) {
            c = a.large[shared ? q : a.n / (kWindow + 1) - 1 - q];
            in = in_bounds(a.s.err, c.z, (a.n + kWindow - 1) / kWindow) && in_bounds(a.s.err, c.x, c.z + 1) && in_bounds(a.s.err, c.w, a.V) &&
                 in_bounds(a.s.err, c.y, a.n < a.V ? a.n : a.V);
        }
        const uint32_t col = ((uint32_t)(item - (uint64_t)q * slabs) * 32 + lane) * E;
        const uint32_t rest = c.z - c.x;   // pieces after the first
        const uint32_t share = shared ? (rest + kJoinWarps - 1) / kJoinWarps : rest;
        const uint32_t from = shared ? wid * share : 0, to = from + share < rest ? from + share : rest;
        const bool first = in && col < a.d && (!shared || wid == 0);
        Finish<kKind, TO, C> row;
        float sum[E];
#pragma unroll
        for (int e = 0; e < E; ++e) sum[e] = 0.0f;
        if (in && col < a.d) {
            const float* at = a.partials + (uint64_t)c.x * step + col;
            if (first) {
                row.fetch(a, c.w, col);
                const Pack<float, E> head = load_pack<float, E>(at + a.partial_stride);
#pragma unroll
                for (int e = 0; e < E; ++e) sum[e] = head.v[e];
            }
            at += (uint64_t)(from + 1) * step;
#pragma unroll 8
            for (uint32_t s = from; s < to; ++s, at += step) {
                const Pack<float, E> x = load_pack<float, E>(at);
#pragma unroll
                for (int e = 0; e < E; ++e) sum[e] += x.v[e];
            }
        }
        if (shared) {
#pragma unroll
            for (int e = 0; e < E; ++e) join[wid][lane * E + e] = sum[e];
            __syncthreads();
            if (first)
                for (int x = 1; x < kJoinWarps; ++x)
#pragma unroll
                    for (int e = 0; e < E; ++e) sum[e] += join[x][lane * E + e];
            __syncthreads();
        }
        if (first) row.put(a, grad_scale, c.w, c.y, col, sum);
    }
}

}  // namespace

template <SumKind kKind, typename TG, typename TO, typename C>
static cudaError_t launch_sums(cudaStream_t stream, const SumArgs& a, int sms) {
    const uint32_t spans = (a.n + kSpan - 1) / kSpan, vecs = (a.d + C::E - 1) / C::E;
    // enough blocks to go round, as long as a block's slab keeps a few vectors
    uint32_t slabs = (uint32_t)sms * kSumBlocks / spans + 1;
    const uint32_t most = (vecs + 15) / 16;
    if (slabs > most) slabs = most;
    if (slabs < vecs / 65536 + 1) slabs = vecs / 65536 + 1;
    const uint32_t slab_vecs = (vecs + slabs - 1) / slabs;
    slabs = (vecs + slab_vecs - 1) / slab_vecs;
    const cudaError_t e = launch_early(k_token_sums<kKind, TG, TO, C>, dim3(spans, slabs), kSumThreads, 0, stream, a, vecs, slab_vecs);
    if (e != cudaSuccess || a.n <= kWindow) return e;
    const uint32_t join_slabs = (vecs + 31) / 32;
    uint64_t blocks = (uint64_t)(a.n / (kWindow + 1)) * join_slabs;
    if (blocks > (uint64_t)sms * 4) blocks = (uint64_t)sms * 4;
    return launch_early(k_join_pieces<kKind, TO, C>, dim3((uint32_t)blocks), kJoinThreads, 0, stream, a, join_slabs);
}

cudaError_t launch_token_sums(cudaStream_t stream, SumKind kind, const SumArgs& a, int sms) {
    return with_sum(kind, a, [&](auto k, auto tg, auto to, auto c) {
        return launch_sums<decltype(k)::value, decltype(tg), decltype(to), decltype(c)>(stream, a, sms);
    });
}

}  // namespace tensair
