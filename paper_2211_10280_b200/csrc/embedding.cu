// Embedding lookup with scaling, and the sums by token that its gradient and the AdamW step of the touched rows are
// made of.
//
// Sums.  The batch's positions are sorted by token (token_sort.cu).  The sorted positions are cut into spans of equal
// length; one thread takes one span and one vector of columns, walks the span's gradient rows with several loads in
// flight and adds them up in fp32, in sorted order.  A token whose positions lie inside one span is finished there:
// its row goes straight to where it belongs (the gradient table, the message, or through the AdamW update).  A token
// that crosses spans leaves one partial row per span, and a second launch adds those up in span order.  Every thread
// has the same number of rows to read whatever the tokens' frequencies are, and no sum depends on timing.
#include "adamw.cuh"
#include "operators.h"

namespace tensair {

namespace {

// ------------------------------------------------------------------ lookup
constexpr int kLookupThreads = 256;
constexpr int kLookupUnroll = 4;

// out[i] = scale * table[ids[i]]; a thread moves kLookupUnroll vectors of E elements, a block's width apart.
template <typename TT, typename TO, int E>
__global__ void __launch_bounds__(kLookupThreads)
k_lookup(TokenIds t, uint32_t row0, const TT* __restrict__ table, uint64_t table_stride, TO* __restrict__ out,
         uint64_t out_stride, FastDiv vecs, uint32_t total, float scale) {
    const uint32_t base = blockIdx.x * (kLookupThreads * kLookupUnroll) + threadIdx.x;
    Pack<TT, E> x[kLookupUnroll];
    uint32_t row[kLookupUnroll], col[kLookupUnroll];
    bool held[kLookupUnroll];
#pragma unroll
    for (int u = 0; u < kLookupUnroll; ++u) {
        const uint32_t w = base + u * kLookupThreads;
        const uint32_t r = w < total ? vecs.div(w) : 0;
        col[u] = (w - r * vecs.divisor) * E;
        row[u] = row0 + r;
        held[u] = false;
        if (w < total) {
            const int64_t id = t.wide ? __ldg(reinterpret_cast<const long long*>(t.ids) + row[u])
                                      : __ldg(reinterpret_cast<const int32_t*>(t.ids) + row[u]);
            held[u] = id != t.padding && (uint64_t)id < t.V;
            if (held[u]) x[u] = load_pack<TT, E>(table + (uint64_t)id * table_stride + col[u]);
            else if (id != t.padding && t.err) atomicOr(t.err, kErrBadToken);
        }
    }
#pragma unroll
    for (int u = 0; u < kLookupUnroll; ++u) {
        if (base + u * kLookupThreads >= total) break;
        float y[E];
#pragma unroll
        for (int e = 0; e < E; ++e) y[e] = held[u] ? to_float(x[u].v[e]) * scale : 0.0f;
        store_pack<TO, E>(out + (uint64_t)row[u] * out_stride + col[u], y);
    }
}

// Widest vector, in elements, that rows of d elements can be moved by (at most `limit`): every row begins on a multiple
// of it, or of 16 bytes where it is wider than that.
uint32_t vector_of(const RowsView& r, uint32_t d, uint32_t limit) {
    uint32_t e = limit;
    for (; e > 1; e /= 2) {
        const uint32_t bytes = e * type_bytes(r.type) > 16 ? 16 : e * type_bytes(r.type);
        if (d % e == 0 && r.stride * type_bytes(r.type) % bytes == 0 && (uintptr_t)r.data % bytes == 0) break;
    }
    return e;
}
// 16 bytes of the narrower of two types
uint32_t widest(const RowsView& a, const RowsView& b) {
    return 16 / (type_bytes(a.type) < type_bytes(b.type) ? type_bytes(a.type) : type_bytes(b.type));
}

// Calls f with a value of the element type as its argument.
template <typename F>
cudaError_t with_type(uint32_t type, F&& f) {
    switch (type) {
        case 0: return f(float());
        case 1: return f(__nv_bfloat16());
        default: return f(__half());
    }
}
template <int E> struct Width { static constexpr int value = E; };
template <typename F>
cudaError_t with_width(uint32_t e, F&& f) {
    switch (e) {
        case 8: return f(Width<8>());
        case 4: return f(Width<4>());
        case 2: return f(Width<2>());
        default: return f(Width<1>());
    }
}

constexpr uint32_t kMaxItems = 0x7FFFFFFFu;   // vectors per launch, so that their numbers stay below 2^31

}  // namespace

cudaError_t launch_lookup(cudaStream_t stream, const TokenIds& t, const RowsView& table, const RowsView& out, uint32_t d,
                          float scale) {
    uint32_t e = vector_of(table, d, widest(table, out));
    e = vector_of(out, d, e);
    const FastDiv vecs(d / e);
    const uint32_t most = kMaxItems / vecs.divisor;     // rows of one launch
    for (uint32_t row0 = 0; row0 < t.n; row0 += most) {
        const uint32_t total = (t.n - row0 < most ? t.n - row0 : most) * vecs.divisor;
        const uint32_t grid = (uint32_t)(((uint64_t)total + kLookupThreads * kLookupUnroll - 1) / (kLookupThreads * kLookupUnroll));
        const cudaError_t err = with_type(table.type, [&](auto tt) {
            return with_type(out.type, [&](auto to) {
                return with_width(e, [&](auto w) {
                    using TT = decltype(tt);
                    using TO = decltype(to);
                    k_lookup<TT, TO, decltype(w)::value><<<grid, kLookupThreads, 0, stream>>>(
                        t, row0, (const TT*)table.data, table.stride, (TO*)out.data, out.stride, vecs, total, scale);
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
constexpr int kCrossThreads = 512;
constexpr int kCrossWarps = kCrossThreads / 32;
constexpr uint32_t kLongCrossing = 16; // a segment over more spans than this is added up by a whole block

// What becomes of the finished sum of a token, E columns from `col` on.  fetch() reads what it is joined with, so that
// several tokens' reads are in flight before the first is needed; put() joins and stores.
template <SumKind kKind, typename TO, int E>
struct Finish {
    Pack<TO, E> old;
    Pack<float, E> m0, v0;

    __device__ __forceinline__ void fetch(const SumArgs& a, uint32_t key, uint32_t col) {
        if (kKind == kSumRows || (kKind == kSumTable && !a.accumulate)) return;
        old = load_pack<TO, E>((const TO*)a.out.data + (uint64_t)key * a.out.stride + col);
        if (kKind == kSumAdamw) {
            m0 = load_pack<float, E>(a.m + (uint64_t)key * a.m_stride + col);
            v0 = load_pack<float, E>(a.v + (uint64_t)key * a.v_stride + col);
        }
    }
    __device__ __forceinline__ void put(const SumArgs& a, float grad_scale, uint32_t key, uint32_t rank, uint32_t col,
                                        const float (&sum)[E]) {
        float y[E];
#pragma unroll
        for (int e = 0; e < E; ++e) y[e] = sum[e] * a.scale;
        TO* out = (TO*)a.out.data + (uint64_t)(kKind == kSumRows ? rank : key) * a.out.stride + col;
        if (kKind == kSumTable) {
            if (a.accumulate)
#pragma unroll
                for (int e = 0; e < E; ++e) y[e] += to_float(old.v[e]);
        } else if (kKind == kSumRows) {
            if (col == 0) a.out_ids[rank] = key;
        } else {
            float m[E], v[E];
#pragma unroll
            for (int e = 0; e < E; ++e) {
                m[e] = m0.v[e];
                v[e] = v0.v[e];
                y[e] = adamw_update(to_float(old.v[e]), y[e] * grad_scale, m[e], v[e], a.adamw, a.adamw.step_size, a.adamw.keep);
            }
            store_pack<float, E>(a.m + (uint64_t)key * a.m_stride + col, m);
            store_pack<float, E>(a.v + (uint64_t)key * a.v_stride + col, v);
        }
        store_pack<TO, E>(out, y);
    }
};


template <SumKind kKind, typename TG, typename TO, int E>
__global__ void __launch_bounds__(kSumThreads)
k_segment_sums(const __grid_constant__ SumArgs a, uint32_t span0, uint32_t total, FastDiv vecs) {
    constexpr int kBatch = kKind == kSumRows ? 8 : 4;   // gradient vectors in flight; fewer where finished rows bring reads of their own
    let_next_launch_begin();
    const uint32_t w = blockIdx.x * kSumThreads + threadIdx.x;
    const uint32_t q = vecs.div(w);
    const uint32_t span = span0 + q, col = (w - q * vecs.divisor) * E;
    const uint32_t begin = span * a.s.span;
    const TG* grad = (const TG*)a.grad.data + col;
    after_previous_launch();
    float grad_scale = 1.0f;
    if (kKind == kSumAdamw && !adamw_grad_scale(a.adamw, &grad_scale)) return;
    const uint32_t n_valid = a.s.info[0];
    if (kKind == kSumRows && span0 == 0 && w == 0) *a.out_count = a.s.info[1];
    if (w >= total || begin >= n_valid) return;
    const uint32_t end = begin + a.s.span < n_valid ? begin + a.s.span : n_valid;
    uint32_t k[kBatch + 1];
    k[0] = a.s.key[begin];
    bool whole = begin == 0 || a.s.key[begin - 1] != k[0];       // the current token begins in this span
    uint32_t rank = a.s.span_rank[span] - (whole ? 0u : 1u);
    float* partial = a.partials + (uint64_t)span * 2 * a.partial_stride + col;
    float sum[E];
#pragma unroll
    for (int e = 0; e < E; ++e) sum[e] = 0.0f;
    bool ended = true;
    for (uint32_t i = begin; i < end; i += kBatch) {
        Pack<TG, E> x[kBatch];
        Finish<kKind, TO, E> row[kBatch];
        bool ends[kBatch];
#pragma unroll
        for (int j = 0; j < kBatch; ++j)
            if (i + j < end) {
                k[j + 1] = i + j + 1 < n_valid ? a.s.key[i + j + 1] : 0xFFFFFFFFu;
                x[j] = load_pack<TG, E>(grad + (uint64_t)a.s.pos[i + j] * a.grad.stride);
            }
        bool here = whole;
#pragma unroll
        for (int j = 0; j < kBatch; ++j) {
            ends[j] = i + j < end && k[j + 1] != k[j];
            if (ends[j] && here) row[j].fetch(a, k[j], col);
            here |= ends[j];
        }
#pragma unroll
        for (int j = 0; j < kBatch; ++j)
            if (i + j < end) {
#pragma unroll
                for (int e = 0; e < E; ++e) sum[e] += to_float(x[j].v[e]);
                if (ends[j]) {
                    if (whole) row[j].put(a, grad_scale, k[j], rank, col, sum);
                    else store_pack<float, E>(partial, sum);     // the end of a token from an earlier span
                    ++rank;
                    whole = true;
#pragma unroll
                    for (int e = 0; e < E; ++e) sum[e] = 0.0f;
                }
                ended = ends[j];
                k[0] = k[j + 1];
            }
    }
    if (ended) return;
    // the token goes on in the next span; k[0] is its id
    store_pack<float, E>(partial + (whole ? a.partial_stride : 0u), sum);
    if (whole && col == 0) {
        const uint32_t last = (a.s.seg_start[rank + 1] - 1) / a.s.span;
        const bool large = last - span > kLongCrossing;
        const uint32_t at = atomicAdd(a.s.info + (large ? 3 : 2), 1u);   // the list's order changes no sum
        a.crossing[(large ? (a.n + a.s.span - 1) / a.s.span : 0u) + at] = make_uint4(span, rank, last, k[0]);
    }
}

// Adds up the partial rows of the tokens that cross spans: the tail of the span they begin in, then the heads of the
// spans that follow.  Short ones take one thread per vector of columns; long ones a block per 32 vectors, whose
// warps each add a stretch of the spans and join them in order.
template <SumKind kKind, typename TO, int E>
__global__ void __launch_bounds__(kCrossThreads)
k_crossing_sums(const __grid_constant__ SumArgs a, FastDiv vecs, uint32_t slabs) {
    __shared__ float join[kCrossWarps][32 * E + 1];
    after_previous_launch();
    float grad_scale = 1.0f;
    if (kKind == kSumAdamw && !adamw_grad_scale(a.adamw, &grad_scale)) return;
    const uint64_t n_short = a.s.info[2], n_long = a.s.info[3];
    const uint64_t step = (uint64_t)2 * a.partial_stride;
    for (uint64_t w = (uint64_t)blockIdx.x * kCrossThreads + threadIdx.x; w < n_short * vecs.divisor;
         w += (uint64_t)gridDim.x * kCrossThreads) {
        const uint32_t q = (uint32_t)(w / vecs.divisor);
        const uint4 c = a.crossing[q];
        const uint32_t col = (uint32_t)(w - (uint64_t)q * vecs.divisor) * E;
        Finish<kKind, TO, E> row;
        row.fetch(a, c.w, col);
        const float* at = a.partials + (uint64_t)c.x * step + col;
        const Pack<float, E> tail = load_pack<float, E>(at + a.partial_stride);
        float sum[E];
#pragma unroll
        for (int e = 0; e < E; ++e) sum[e] = tail.v[e];
#pragma unroll 4
        for (uint32_t s = c.x + 1; s <= c.z; ++s) {
            at += step;
            const Pack<float, E> x = load_pack<float, E>(at);
#pragma unroll
            for (int e = 0; e < E; ++e) sum[e] += x.v[e];
        }
        row.put(a, grad_scale, c.w, c.y, col, sum);
    }
    const uint32_t spans = (a.n + a.s.span - 1) / a.s.span;
    const uint32_t lane = threadIdx.x & 31, wid = threadIdx.x >> 5;
    for (uint64_t w = blockIdx.x; w < n_long * slabs; w += gridDim.x) {
        const uint32_t q = (uint32_t)(w / slabs);
        const uint4 c = a.crossing[spans + q];
        const uint32_t col = ((uint32_t)(w - (uint64_t)q * slabs) * 32 + lane) * E;
        const uint32_t heads = c.z - c.x;              // partial rows after the first
        const uint32_t share = (heads + kCrossWarps - 1) / kCrossWarps;
        const uint32_t from = wid * share, to = from + share < heads ? from + share : heads;
        Finish<kKind, TO, E> row;
        float sum[E];
#pragma unroll
        for (int e = 0; e < E; ++e) sum[e] = 0.0f;
        if (col < a.d) {
            const float* at = a.partials + (uint64_t)c.x * step + col;
            if (wid == 0) {
                row.fetch(a, c.w, col);
                const Pack<float, E> tail = load_pack<float, E>(at + a.partial_stride);
#pragma unroll
                for (int e = 0; e < E; ++e) sum[e] = tail.v[e];
            }
            at += (uint64_t)(from + 1) * step;
#pragma unroll 8
            for (uint32_t s = from; s < to; ++s, at += step) {
                const Pack<float, E> x = load_pack<float, E>(at);
#pragma unroll
                for (int e = 0; e < E; ++e) sum[e] += x.v[e];
            }
        }
#pragma unroll
        for (int e = 0; e < E; ++e) join[wid][lane * E + e] = sum[e];
        __syncthreads();
        if (wid == 0 && col < a.d) {
            for (int x = 1; x < kCrossWarps; ++x)
#pragma unroll
                for (int e = 0; e < E; ++e) sum[e] += join[x][lane * E + e];
            row.put(a, grad_scale, c.w, c.y, col, sum);
        }
        __syncthreads();
    }
}

}  // namespace

// Sorted positions per span.
constexpr uint32_t kLongBatch = 8192;
uint32_t span_length(uint32_t n, uint32_t) { return n >= kLongBatch ? 16 : 8; }
uint32_t longest_with_shorter_spans(uint32_t n, uint32_t) { return n >= kLongBatch ? kLongBatch - 1 : 0; }

template <SumKind kKind, typename TG, typename TO, int E>
static cudaError_t launch_sums(cudaStream_t stream, const SumArgs& a) {
    const uint32_t spans = (a.n + a.s.span - 1) / a.s.span;
    const FastDiv vecs(a.d / E);
    const uint32_t most = kMaxItems / vecs.divisor;
    for (uint32_t span0 = 0; span0 < spans; span0 += most) {
        const uint32_t total = (spans - span0 < most ? spans - span0 : most) * vecs.divisor;
        const cudaError_t e = launch_early(k_segment_sums<kKind, TG, TO, E>, (total + kSumThreads - 1) / kSumThreads, kSumThreads,
                                           stream, a, span0, total, vecs);
        if (e != cudaSuccess) return e;
    }
    if (spans > 1) {
        const uint32_t slabs = (vecs.divisor + 31) / 32;
        uint64_t blocks = ((uint64_t)spans * vecs.divisor + kCrossThreads - 1) / kCrossThreads;
        if (blocks > 592) blocks = 592;
        return launch_early(k_crossing_sums<kKind, TO, E>, (uint32_t)blocks, kCrossThreads, stream, a, vecs, slabs);
    }
    return cudaSuccess;
}

cudaError_t launch_segment_sums(cudaStream_t stream, SumKind kind, const SumArgs& a) {
    uint32_t e = vector_of(a.grad, a.d, widest(a.grad, a.out));
    e = vector_of(a.out, a.d, e);
    if (kind == kSumAdamw) {
        e = vector_of(RowsView{a.m, a.m_stride, 0}, a.d, e);
        e = vector_of(RowsView{a.v, a.v_stride, 0}, a.d, e);
    }
    return with_type(a.grad.type, [&](auto tg) {
        return with_type(a.out.type, [&](auto to) {
            return with_width(e, [&](auto w) {
                using TG = decltype(tg);
                using TO = decltype(to);
                constexpr int E = decltype(w)::value;
                if (kind == kSumAdamw) return launch_sums<kSumAdamw, TG, TO, E>(stream, a);
                if (kind == kSumTable) return launch_sums<kSumTable, TG, TO, E>(stream, a);
                if constexpr (sizeof(TO) == 4) return launch_sums<kSumRows, TG, TO, E>(stream, a);
                else return cudaErrorInvalidValue;
            });
        });
    });
}

}  // namespace tensair
