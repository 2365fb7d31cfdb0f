// A gated linear recurrence, channel by channel:
//
//     f_t = sigmoid(gate_t),  h_t = f_t h_{t-1} + (1 - f_t) v_t
//
// and its gradient, with e the gradient of the state after the last step and dh_t the incoming one:
//
//     D_t = dh_t + e_{t+1},  e_t = f_t D_t,  dv_t = (1 - f_t) D_t,  dgate_t = f_t (1 - f_t) (h_{t-1} - v_t) D_t
//
// Both are first-order linear recurrences x <- (1 - r) x + b.  Steps compose: (r, b) then (r', b') is (r + r' - r r', (1 - r') b + b').  A thread takes
// 8 steps of a few channels and holds them in registers; the threads of a block cover more steps one after the other, the blocks of
// a cluster still more, and a block goes on with its cluster's next stretch until the sequence ends.  Every level passes on the
// composition of what it holds, gets the state that it begins with, and only then makes its outputs: the inputs are read once.
// Compositions are joined in step order, so no result depends on timing.
//
// The gradient needs h_{t-1} again: the forward call leaves the state before every eighth step in fp32 (half a byte per element),
// and a thread of the backward call replays its own 8 steps from there.
#include <cooperative_groups.h>

#include "columns.cuh"
#include "layers.h"

namespace tensair {

namespace {

namespace cg = cooperative_groups;

constexpr int kThreads = 256;
constexpr int kSteps = kMark;            // of a thread
constexpr uint32_t kMostCluster = 16;

// r = 1 - f = sigmoid(-gate) and e = exp(gate).  What is kept of f is r: f x = x - r x in one fused step has the relative accuracy of
// r, so a gate near 1 remembers for as long as it should (1 - 6e-8 would be the f next to 1) and a gate of -inf forgets all.
__device__ __forceinline__ float complement(float gate, float& e) {
    e = expf(gate);
    return __fdividef(1.0f, 1.0f + e);
}
__device__ __forceinline__ float decay(float rest, float x) { return fmaf(-rest, x, x); }
// The complement of a product of two factors, from theirs.  (The product itself, rounded near 1 step after step, drifts: 20,000 steps
// of 1 - 8e-7 were off by 6e-5.)
__device__ __forceinline__ float join_rest(float a, float b) { return fmaf(b, 1.0f - a, a); }

// What the threads of a block pass one another: for each of its channels, the compositions of its stretches of steps.
// [stretch][channel]; kThreads * E of each.
template <int E>
struct Joint {
    float r[kThreads * E], b[kThreads * E];
    float carry[kThreads * E], start[kThreads * E];
    float2 ranks[2][kMostCluster][64];       // the cluster's compositions, of two turns (channels of a block that is part of a cluster: 64 at most)
};

// The state that every stretch of the block begins with, from the stretches' compositions (kBack: from the last one to the first).
// On return `joint.r, b` hold the composition of what comes before each stretch inside the block, joint.start the state the block
// begins with, and joint.carry the state after the cluster's whole turn.
template <bool kBack, int E>
__device__ __forceinline__ void join_block(Joint<E>& joint, uint32_t channels, uint32_t stretches, uint32_t cluster, uint32_t rank, uint32_t turn) {
    __syncthreads();
    for (uint32_t c = threadIdx.x; c < channels; c += kThreads) {
        float rest = 0.0f, b = 0.0f;
#pragma unroll 4
        for (uint32_t s = 0; s < stretches; ++s) {
            const uint32_t at = (kBack ? stretches - 1 - s : s) * channels + c;
            const float r = joint.r[at], add = joint.b[at];
            joint.r[at] = rest;
            joint.b[at] = b;
            b = decay(r, b) + add;
            rest = join_rest(rest, r);
        }
        if (cluster == 1) {
            const float carry = joint.carry[c];
            joint.start[c] = carry;
            joint.carry[c] = decay(rest, carry) + b;
        } else {
            cg::cluster_group all = cg::this_cluster();
            for (uint32_t r = 0; r < cluster; ++r)
                *all.map_shared_rank(&joint.ranks[turn & 1][rank][c], r) = make_float2(rest, b);
        }
    }
    if (cluster > 1) {
        cg::this_cluster().sync();
        for (uint32_t c = threadIdx.x; c < channels; c += kThreads) {
            float carry = joint.carry[c], start = 0.0f;
            for (uint32_t q = 0; q < cluster; ++q) {
                const uint32_t r = kBack ? cluster - 1 - q : q;
                if (r == rank) start = carry;
                const float2 x = joint.ranks[turn & 1][r][c];
                carry = decay(x.x, carry) + x.y;
            }
            joint.start[c] = start;
            joint.carry[c] = carry;
        }
    }
    __syncthreads();
}

// How a launch cuts its work: a block covers `units` pieces of channels (of all sequences, one after the other) and kThreads /
// units stretches of kSteps steps.
struct Cut {
    FastDiv vecs;          // pieces of channels of a sequence
    uint32_t total;        // of all sequences
    uint32_t units;        // power of two
    uint32_t cluster;
    uint32_t turns;
};

template <typename T, typename C>
__global__ void __launch_bounds__(kThreads)
k_recurrence(const __grid_constant__ RecurrenceArgs a, const __grid_constant__ Cut cut) {
    constexpr int E = C::E;
    __shared__ Joint<E> joint;
    const uint32_t u = threadIdx.x & (cut.units - 1), stretch = threadIdx.x / cut.units, stretches = kThreads / cut.units;
    const uint32_t rank = blockIdx.x % cut.cluster, unit = blockIdx.x / cut.cluster * cut.units + u;
    const uint32_t channels = cut.units * E;
    const bool mine = unit < cut.total;
    const uint32_t s = mine ? cut.vecs.div(unit) : 0, col = mine ? (unit - s * cut.vecs.divisor) * E : 0, left = a.d - col;
    uint32_t length = mine ? a.T : 0;
    if (mine && a.lengths) {
        const int32_t n = a.lengths[s];
        length = n < 0 ? 0 : (uint32_t)n < a.T ? (uint32_t)n : a.T;
    }
    const T* gate = (const T*)a.gate.data + s * a.gate.batch + col;
    const T* value = (const T*)a.value.data + s * a.value.batch + col;
    T* out = (T*)a.out.data + s * a.out.batch + col;
    const uint64_t row = (uint64_t)s * a.d + col;
    if (stretch == 0) {
        Pack<float, E> first = {};
#pragma unroll
        for (int e = 0; e < E; ++e) joint.carry[u * E + e] = mine && a.state && (!C::kRagged || e < (int)left) ? a.state[row + e] : 0.0f;
    }
    if (cut.cluster > 1) cg::this_cluster().sync();      // no block writes into another's memory before that one has started
    const uint32_t marks = (a.T + kMark - 1) / kMark;
    for (uint32_t turn = 0; turn < cut.turns; ++turn) {
        const uint64_t t64 = ((uint64_t)(turn * cut.cluster + rank) * stretches + stretch) * kSteps;
        const uint32_t t0 = t64 < a.T ? (uint32_t)t64 : a.T;
        Pack<T, E> rg[kSteps] = {}, rv[kSteps] = {};
#pragma unroll
        for (int l = 0; l < kSteps; ++l)
            if (t0 + l < length) {
                rg[l] = load_columns<C>(gate + (t0 + l) * a.gate.step, left);
                rv[l] = load_columns<C>(value + (t0 + l) * a.value.step, left);
            }
        // the stretch's composition: h <- (1 - r) h + b
        float rest[kSteps][E], r[E], b[E];
#pragma unroll
        for (int e = 0; e < E; ++e) r[e] = b[e] = 0.0f;
#pragma unroll
        for (int l = 0; l < kSteps; ++l)
#pragma unroll
            for (int e = 0; e < E; ++e) {
                float exp_gate;
                rest[l][e] = t0 + l < length ? complement(to_float(rg[l].v[e]), exp_gate) : 0.0f;     // padding: h stays
                r[e] = join_rest(r[e], rest[l][e]);
                b[e] = fmaf(rest[l][e], to_float(rv[l].v[e]), decay(rest[l][e], b[e]));
            }
#pragma unroll
        for (int e = 0; e < E; ++e) {
            joint.r[stretch * channels + u * E + e] = r[e];
            joint.b[stretch * channels + u * E + e] = b[e];
        }
        join_block<false, E>(joint, channels, stretches, cut.cluster, rank, turn);
        float h[E];
#pragma unroll
        for (int e = 0; e < E; ++e)
            h[e] = decay(joint.r[stretch * channels + u * E + e], joint.start[u * E + e]) + joint.b[stretch * channels + u * E + e];
        __syncthreads();
        if (!mine || t0 >= a.T) continue;
        if (a.marks) store_columns<C>(a.marks + ((uint64_t)s * marks + t0 / kMark) * a.d + col, h, left);
#pragma unroll
        for (int l = 0; l < kSteps; ++l) {
            if (t0 + l >= a.T) break;
            float y[E];
#pragma unroll
            for (int e = 0; e < E; ++e) {
                h[e] = fmaf(rest[l][e], to_float(rv[l].v[e]), decay(rest[l][e], h[e]));
                y[e] = t0 + l < length ? h[e] : 0.0f;
            }
            store_columns<C>(out + (t0 + l) * a.out.step, y, left);
        }
    }
    if (a.last && mine && rank == 0 && stretch == 0)
#pragma unroll
        for (int e = 0; e < E; ++e)
            if (!C::kRagged || e < (int)left) a.last[row + e] = joint.carry[u * E + e];
}

template <typename T, typename C>
__global__ void __launch_bounds__(kThreads)
k_recurrence_gradient(const __grid_constant__ RecurrenceArgs a, const __grid_constant__ Cut cut) {
    constexpr int E = C::E;
    __shared__ Joint<E> joint;
    const uint32_t u = threadIdx.x & (cut.units - 1), stretch = threadIdx.x / cut.units, stretches = kThreads / cut.units;
    const uint32_t rank = blockIdx.x % cut.cluster, unit = blockIdx.x / cut.cluster * cut.units + u;
    const uint32_t channels = cut.units * E;
    const bool mine = unit < cut.total;
    const uint32_t s = mine ? cut.vecs.div(unit) : 0, col = mine ? (unit - s * cut.vecs.divisor) * E : 0, left = a.d - col;
    uint32_t length = mine ? a.T : 0;
    if (mine && a.lengths) {
        const int32_t n = a.lengths[s];
        length = n < 0 ? 0 : (uint32_t)n < a.T ? (uint32_t)n : a.T;
    }
    const T* gate = (const T*)a.gate.data + s * a.gate.batch + col;
    const T* value = (const T*)a.value.data + s * a.value.batch + col;
    const T* grad = (const T*)a.out.data + s * a.out.batch + col;
    T* dgate = (T*)a.dgate.data + s * a.dgate.batch + col;
    T* dvalue = (T*)a.dvalue.data + s * a.dvalue.batch + col;
    const uint64_t row = (uint64_t)s * a.d + col;
    if (stretch == 0) {
#pragma unroll
        for (int e = 0; e < E; ++e) joint.carry[u * E + e] = mine && a.state && (!C::kRagged || e < (int)left) ? a.state[row + e] : 0.0f;
    }
    if (cut.cluster > 1) cg::this_cluster().sync();
    const uint32_t marks = (a.T + kMark - 1) / kMark;
    for (uint32_t turn = cut.turns; turn-- > 0;) {
        const uint64_t t64 = ((uint64_t)(turn * cut.cluster + rank) * stretches + stretch) * kSteps;
        const uint32_t t0 = t64 < a.T ? (uint32_t)t64 : a.T;
        Pack<T, E> rg[kSteps] = {}, rv[kSteps] = {}, rd[kSteps] = {};
        Pack<float, E> mark = {};
        if (t0 < length) mark = load_columns<C>(a.marks + ((uint64_t)s * marks + t0 / kMark) * a.d + col, left);
#pragma unroll
        for (int l = 0; l < kSteps; ++l)
            if (t0 + l < length) {
                rg[l] = load_columns<C>(gate + (t0 + l) * a.gate.step, left);
                rv[l] = load_columns<C>(value + (t0 + l) * a.value.step, left);
                rd[l] = load_columns<C>(grad + (t0 + l) * a.out.step, left);
            }
        // r = 1 - f and f r (h_{t-1} - v_t) of every step, h from the mark on
        float rest[kSteps][E], slope[kSteps][E], h[E], r[E], b[E];
#pragma unroll
        for (int e = 0; e < E; ++e) h[e] = mark.v[e], r[e] = b[e] = 0.0f;
#pragma unroll
        for (int l = 0; l < kSteps; ++l)
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const float g = to_float(rg[l].v[e]), v = to_float(rv[l].v[e]);
                float exp_gate;
                const float now = complement(g, exp_gate), f = g < 0.0f ? exp_gate * now : 1.0f - now;
                rest[l][e] = t0 + l < length ? now : 0.0f;
                slope[l][e] = t0 + l < length ? f * now * (h[e] - v) : 0.0f;
                h[e] = fmaf(now, v, decay(now, h[e]));
            }
#pragma unroll
        for (int l = kSteps - 1; l >= 0; --l)
#pragma unroll
            for (int e = 0; e < E; ++e) {
                r[e] = join_rest(r[e], rest[l][e]);
                b[e] = decay(rest[l][e], b[e] + to_float(rd[l].v[e]));      // padding: the gradient passes, none is added
            }
#pragma unroll
        for (int e = 0; e < E; ++e) {
            joint.r[stretch * channels + u * E + e] = r[e];
            joint.b[stretch * channels + u * E + e] = b[e];
        }
        join_block<true, E>(joint, channels, stretches, cut.cluster, rank, turn);
#pragma unroll
        for (int e = 0; e < E; ++e)
            b[e] = decay(joint.r[stretch * channels + u * E + e], joint.start[u * E + e]) + joint.b[stretch * channels + u * E + e];
        __syncthreads();
        if (!mine || t0 >= a.T) continue;
#pragma unroll
        for (int l = kSteps - 1; l >= 0; --l) {
            if (t0 + l >= a.T) continue;
            float dg[E], dv[E];
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const float D = to_float(rd[l].v[e]) + b[e];
                b[e] = decay(rest[l][e], D);
                dg[e] = slope[l][e] * D;
                dv[e] = rest[l][e] * D;
            }
            store_columns<C>(dgate + (t0 + l) * a.dgate.step, dg, left);
            store_columns<C>(dvalue + (t0 + l) * a.dvalue.step, dv, left);
        }
    }
    if (a.last && mine && rank == 0 && stretch == 0)
#pragma unroll
        for (int e = 0; e < E; ++e)
            if (!C::kRagged || e < (int)left) a.last[row + e] = joint.carry[u * E + e];
}

// One step, for serving: a thread per piece of channels.
template <typename T, typename C>
__global__ void __launch_bounds__(128)
k_recurrence_step(const __grid_constant__ RecurrenceArgs a, const __grid_constant__ FastDiv vecs, uint32_t total) {
    constexpr int E = C::E;
    const uint32_t unit = blockIdx.x * 128 + threadIdx.x;
    if (unit >= total) return;
    const uint32_t s = vecs.div(unit), col = (unit - s * vecs.divisor) * E, left = a.d - col;
    const Pack<T, E> g = load_columns<C>((const T*)a.gate.data + s * a.gate.batch + col, left);
    const Pack<T, E> v = load_columns<C>((const T*)a.value.data + s * a.value.batch + col, left);
    const uint64_t row = (uint64_t)s * a.d + col;
    Pack<float, E> old = {};
    if (a.state) old = load_columns<C>(a.state + row, left);
    float h[E];
#pragma unroll
    for (int e = 0; e < E; ++e) {
        float exp_gate;
        const float rest = complement(to_float(g.v[e]), exp_gate);
        h[e] = fmaf(rest, to_float(v.v[e]), decay(rest, old.v[e]));
    }
    store_columns<C>(a.last + row, h, left);
    store_columns<C>((T*)a.out.data + s * a.out.batch + col, h, left);
}

// Widest piece, of at most `e` columns, that all rows of a view begin on a multiple of.
uint32_t piece_of(const StepsView& v, uint32_t type, uint32_t T, uint32_t B, uint32_t e) {
    const uint32_t b = type_bytes(type);
    for (; e > 1; e /= 2)
        if ((uintptr_t)v.data % (e * b) == 0 && (T < 2 || v.step % e == 0) && (B < 2 || v.batch % e == 0)) break;
    return e;
}
uint32_t piece_of(const float* p, uint32_t e) {
    while (e > 1 && (uintptr_t)p % (e * 4)) e /= 2;
    return e;
}

// Calls f(columns): pieces of 8 bytes, or of as many columns one by one.
template <typename T, int E, typename F>
cudaError_t with_pieces(const RecurrenceArgs& a, bool back, F&& f) {
    uint32_t e = a.d % E ? 1 : E;
    e = piece_of(a.gate, a.type, a.T, a.B, e);
    e = piece_of(a.value, a.type, a.T, a.B, e);
    e = piece_of(a.out, a.type, a.T, a.B, e);
    if (back) {
        e = piece_of(a.dgate, a.type, a.T, a.B, e);
        e = piece_of(a.dvalue, a.type, a.T, a.B, e);
    }
    e = piece_of(a.marks, e);
    e = piece_of(a.state, e);
    e = piece_of(a.last, e);
    return e == E ? f(Columns<E, false>()) : f(Columns<E, true>());
}

Cut cut_of(const RecurrenceArgs& a, uint32_t e, int sms) {
    Cut c;
    c.vecs = FastDiv((a.d + e - 1) / e);
    c.total = a.B * c.vecs.divisor;
    // stretches enough for the sequence, 32 at most
    uint32_t stretches = 1;
    while (stretches < 32 && stretches * kSteps < a.T) stretches *= 2;
    c.units = kThreads / stretches;
    c.cluster = 1;
    const uint64_t blocks = (c.total + c.units - 1) / c.units;
    while (c.cluster < kMostCluster && blocks * c.cluster < (uint64_t)sms * 2 && (uint64_t)c.cluster * stretches * kSteps < a.T && c.units * e <= 64) c.cluster *= 2;
    const uint64_t span = (uint64_t)c.cluster * stretches * kSteps;
    c.turns = (uint32_t)((a.T + span - 1) / span);
    return c;
}

template <typename K>
cudaError_t launch_cut(cudaStream_t stream, K kernel, const RecurrenceArgs& a, const Cut& c) {
    const uint64_t blocks = (uint64_t)((c.total + c.units - 1) / c.units) * c.cluster;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((uint32_t)blocks);
    cfg.blockDim = dim3(kThreads);
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim = {c.cluster, 1, 1};
    if (c.cluster > 1) {
        cfg.attrs = attr;
        cfg.numAttrs = 1;
        if (c.cluster > 8) {
            const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
            if (e != cudaSuccess) return e;
        }
    }
    return cudaLaunchKernelEx(&cfg, kernel, a, c);
}

}  // namespace

cudaError_t launch_recurrence(cudaStream_t stream, const RecurrenceArgs& a, int sms) {
    return with_type(a.type, [&](auto t) {
        using T = decltype(t);
        constexpr int E = 8 / sizeof(T);
        return with_pieces<T, E>(a, false, [&](auto c) {
            return launch_cut(stream, k_recurrence<T, decltype(c)>, a, cut_of(a, E, sms));
        });
    });
}

cudaError_t launch_recurrence_gradient(cudaStream_t stream, const RecurrenceArgs& a, int sms) {
    return with_type(a.type, [&](auto t) {
        using T = decltype(t);
        return with_pieces<T, 2>(a, true, [&](auto c) {
            return launch_cut(stream, k_recurrence_gradient<T, decltype(c)>, a, cut_of(a, 2, sms));
        });
    });
}

cudaError_t launch_recurrence_step(cudaStream_t stream, const RecurrenceArgs& a) {
    return with_type(a.type, [&](auto t) {
        using T = decltype(t);
        constexpr int E = 8 / sizeof(T);
        return with_pieces<T, E>(a, false, [&](auto c) {
            using C = decltype(c);
            const FastDiv vecs((a.d + E - 1) / E);
            const uint32_t total = a.B * vecs.divisor;
            k_recurrence_step<T, C><<<(total + 127) / 128, 128, 0, stream>>>(a, vecs, total);
            return cudaGetLastError();
        });
    });
}

}  // namespace tensair
