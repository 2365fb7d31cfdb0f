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
// a cluster still more, and a block goes on with its cluster's next stretch until the sequence ends, and then with other channels.  Every
// level passes on the composition of what it holds, gets the state that it begins with, and only then makes its outputs: the inputs are
// read once.  Compositions are joined in step order, so no result depends on timing.
//
// The gradient needs h_{t-1} again: the forward call leaves the state before every eighth step in fp32 (half a byte per element),
// and a thread of the backward call replays its own 8 steps from there.
//
// Kept of a gate is n = f - 1 = -sigmoid(-gate), not f: x + n x in one fused step has the relative accuracy of n, so a gate near 1
// remembers for as long as it should (1 - 6e-8 would be the f next to 1) and a gate of minus infinity forgets all.  Compositions keep
// f - 1 of their product for the same reason (the product itself, rounded near 1 step after step, drifts: 20,000 steps of 1 - 8e-7
// were off by 6e-5).  Two channels go through each instruction (packed fp32).
//
// The next stretch's inputs are on their way into shared memory (asynchronous copies, each thread its own) while this one's are worked on.
#include <cooperative_groups.h>

#include "columns.cuh"
#include "layers.h"
#include "packed.cuh"

namespace tensair {

namespace {

namespace cg = cooperative_groups;

constexpr int kThreads = 256;
constexpr int kSteps = kMark;            // of a thread
constexpr uint32_t kMostCluster = 16;
constexpr uint32_t kClusterChannels = 64;      // of a block that is part of a cluster, at most

__device__ __forceinline__ float exp2_approx(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float reciprocal_approx(float x) {
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float least_or_nan(float x, float y) {
    float z;
    asm("min.NaN.f32 %0, %1, %2;" : "=f"(z) : "f"(x), "f"(y));
    return z;
}
// exp(gate), at most 2^127.9 (whose 1 - f is zero all the same).  Gates of 16 bits: 2^x of the rounded product with log2(e), off by
// (1.5 |gate| + 2) 2^-24 of it; half a unit of the gate's own last place is 10^4 times as much.  Gates of 32 bits: expf.
template <typename T>
__device__ __forceinline__ Two exp_of(Two gate) {
    if constexpr (sizeof(T) == 2) {
        const float2 x = (gate * Two(1.44269504f)).floats();
        return Two(exp2_approx(least_or_nan(x.x, 127.9f)), exp2_approx(least_or_nan(x.y, 127.9f)));
    } else {
        const float2 x = gate.floats();
        return Two(expf(least_or_nan(x.x, 88.6f)), expf(least_or_nan(x.y, 88.6f)));
    }
}
// n = f - 1 from e = exp(gate): -1 / (1 + e)
__device__ __forceinline__ Two complement(Two e) {
    const float2 x = fma2(e, Two(-1.0f), Two(-1.0f)).floats();
    return Two(reciprocal_approx(x.x), reciprocal_approx(x.y));
}
__device__ __forceinline__ Two decay(Two n, Two x) { return fma2(n, x, x); }
__device__ __forceinline__ float decay(float n, float x) { return fmaf(n, x, x); }
// f - 1 of the product of two factors, from theirs.
__device__ __forceinline__ Two join_rest(Two a, Two b) { return fma2(b, a + Two(1.0f), a); }
__device__ __forceinline__ float join_rest(float a, float b) { return fmaf(b, a + 1.0f, a); }

// 8 bytes of raw elements as pairs of floats, and back.  kNegative: with their signs changed.
template <typename T, bool kNegative>
__device__ __forceinline__ void unpack(uint2 raw, Two (&x)[8 / sizeof(T) / 2]) {
    if constexpr (sizeof(T) == 4) {
        const uint32_t sign = kNegative ? 0x80000000u : 0;
        x[0] = Two(__uint_as_float(raw.x ^ sign), __uint_as_float(raw.y ^ sign));
    } else {
        const uint32_t sign = kNegative ? 0x80008000u : 0, words[2] = {raw.x ^ sign, raw.y ^ sign};
#pragma unroll
        for (int p = 0; p < 2; ++p) {
            if constexpr (std::is_same_v<T, __nv_bfloat16>) x[p] = Two(__uint_as_float(words[p] << 16), __uint_as_float(words[p] & 0xFFFF0000u));
            else {
                const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&words[p]));
                x[p] = Two(f.x, f.y);
            }
        }
    }
}
template <typename T>
__device__ __forceinline__ uint2 pack(const Two (&x)[8 / sizeof(T) / 2]) {
    if constexpr (sizeof(T) == 4) {
        const float2 f = x[0].floats();
        return make_uint2(__float_as_uint(f.x), __float_as_uint(f.y));
    } else {
        uint32_t words[2];
#pragma unroll
        for (int p = 0; p < 2; ++p) {
            const float2 f = x[p].floats();
            if constexpr (std::is_same_v<T, __nv_bfloat16>) {
                const __nv_bfloat162 y = __floats2bfloat162_rn(f.x, f.y);
                words[p] = *reinterpret_cast<const uint32_t*>(&y);
            } else {
                const __half2 y = __floats2half2_rn(f.x, f.y);
                words[p] = *reinterpret_cast<const uint32_t*>(&y);
            }
        }
        return make_uint2(words[0], words[1]);
    }
}
template <typename T, typename C>
__device__ __forceinline__ void store_raw(T* to, uint2 raw, uint32_t left) {
    if constexpr (!C::kRagged) *reinterpret_cast<uint2*>(to) = raw;
    else {
        const T* x = reinterpret_cast<const T*>(&raw);
#pragma unroll
        for (int e = 0; e < C::E; ++e)
            if (e < (int)left) to[e] = x[e];
    }
}
// Into shared memory: asynchronously, where the rows allow it.
template <typename T, typename C>
__device__ __forceinline__ void fetch(void* to, const T* from, uint32_t left) {
    if constexpr (!C::kRagged)
        asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"((uint32_t)__cvta_generic_to_shared(to)), "l"(from), "n"(sizeof(T) * C::E) : "memory");
    else *reinterpret_cast<Pack<T, C::E>*>(to) = load_columns<C>(from, left);
}
__device__ __forceinline__ void fetched() { asm volatile("cp.async.wait_all;" ::: "memory"); }
template <typename T>
__device__ __forceinline__ uint2 infinite() {      // gates that keep everything
    if constexpr (sizeof(T) == 4) return make_uint2(0x7F800000u, 0x7F800000u);
    else if constexpr (std::is_same_v<T, __half>) return make_uint2(0x7C007C00u, 0x7C007C00u);
    else return make_uint2(0x7F807F80u, 0x7F807F80u);
}

// Between the blocks of a cluster: values are sent straight into another block's memory, where a barrier counts their bytes.  (With the
// cluster's own barrier, which also waits for every store of the turn before, a turn of 16 blocks took 8.7 us instead of 3.)
__device__ __forceinline__ uint32_t shared_address(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void start_barrier(uint64_t* barrier) {
    asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" ::"r"(shared_address(barrier)) : "memory");
}
__device__ __forceinline__ void expect_bytes(uint64_t* barrier, uint32_t bytes) {
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(shared_address(barrier)), "r"(bytes) : "memory");
}
__device__ __forceinline__ void send(const float2* to, const uint64_t* barrier, uint32_t rank, float2 x) {
    uint32_t there, bar;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(there) : "r"(shared_address(to)), "r"(rank));
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(bar) : "r"(shared_address(barrier)), "r"(rank));
    asm volatile("st.async.weak.shared::cluster.mbarrier::complete_tx::bytes.v2.f32 [%0], {%1, %2}, [%3];" ::"r"(there), "f"(x.x), "f"(x.y), "r"(bar) : "memory");
}
// False: they did not come, after some 50 ms.
__device__ __forceinline__ bool wait_bytes(uint64_t* barrier, uint32_t parity) {
    for (int i = 0; i < 1 << 20; ++i) {
        uint32_t done;
        asm volatile("{\n.reg .pred p;\nmbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\nselp.u32 %0, 1, 0, p;\n}" : "=r"(done) : "r"(shared_address(barrier)), "r"(parity) : "memory");
        if (done) return true;
    }
    return false;
}

// What the threads of a block pass one another: for each of its channels, the compositions of its stretches of steps, in the order
// of the recurrence ([stretch][channel]).
template <int E>
struct Joint {
    alignas(16) float n[kThreads * E];
    alignas(16) float b[kThreads * E];
    float carry[kThreads * E], start[kThreads * E];
    float2 parts[kThreads];
    float2 ranks[2][kMostCluster][kClusterChannels];       // the cluster's compositions, of two turns
    uint64_t arrived[2];                                   // barriers that count the bytes of those
};

// How a launch cuts its work: a block covers `units` pieces of channels (of all sequences, one after the other) and kThreads /
// units stretches of kSteps steps at a time.
struct Cut {
    FastDiv vecs;          // pieces of channels of a sequence
    uint32_t total;        // of all sequences
    uint32_t units;        // power of two
    uint32_t cluster, turns;
    uint32_t groups;       // of `units` pieces
};

// The state that every stretch of the block begins with, from the stretches' compositions.  `place`: of the block in its cluster, in the order
// of the recurrence.  On return joint.n, b hold the composition of what comes before each stretch inside the block, joint.start the state the block
// begins with, and joint.carry the state after the cluster's whole turn.
template <int E>
__device__ __forceinline__ void join_block(Joint<E>& joint, const Cut& cut, uint32_t stretches, uint32_t place, uint32_t turn) {
    const uint32_t odd = turn & 1;
    const uint32_t channels = cut.units * E, parts = channels < kThreads ? kThreads / channels : 1, each = stretches / parts;
    __syncthreads();
    // a channel's stretches are cut into parts of E (or are one part, where there are few)
    for (uint32_t i = threadIdx.x; i < channels * parts; i += kThreads) {
        const uint32_t c = i & (channels - 1), from = i / channels * each;
        float n = 0.0f, b = 0.0f;
#pragma unroll 4
        for (uint32_t s = from; s < from + each; ++s) {
            const float then = joint.n[s * channels + c];
            b = decay(then, b) + joint.b[s * channels + c];
            n = join_rest(n, then);
        }
        if (parts > 1) joint.parts[i] = make_float2(n, b);
    }
    if (parts > 1) __syncthreads();
    for (uint32_t i = threadIdx.x; i < channels * parts; i += kThreads) {
        const uint32_t c = i & (channels - 1), part = i / channels;
        float n = 0.0f, b = 0.0f;
#pragma unroll 4
        for (uint32_t q = 0; q < part; ++q) {
            const float2 x = joint.parts[q * channels + c];
            b = decay(x.x, b) + x.y;
            n = join_rest(n, x.x);
        }
#pragma unroll 4
        for (uint32_t s = part * each; s < (part + 1) * each; ++s) {
            const float then = joint.n[s * channels + c], add = joint.b[s * channels + c];
            joint.n[s * channels + c] = n;
            joint.b[s * channels + c] = b;
            b = decay(then, b) + add;
            n = join_rest(n, then);
        }
        if (part + 1 < parts) continue;
        if (cut.cluster == 1) {
            const float carry = joint.carry[c];
            joint.start[c] = carry;
            joint.carry[c] = decay(n, carry) + b;
        } else {
#pragma unroll 4
            for (uint32_t r = 0; r < cut.cluster; ++r) send(&joint.ranks[odd][place][c], &joint.arrived[odd], r, make_float2(n, b));
        }
    }
    if (cut.cluster > 1) {
        // What is written over has been read: who sent for the turn before had read this turn's predecessor but one.
        if (threadIdx.x == 0) expect_bytes(&joint.arrived[odd], cut.cluster * channels * 8);
        if (threadIdx.x < channels) {
            const uint32_t c = threadIdx.x;
            float carry = joint.carry[c], start = 0.0f;
            if (!wait_bytes(&joint.arrived[odd], turn >> 1 & 1)) carry = NAN;      // all that follows is NaN, and ends
#pragma unroll 4
            for (uint32_t q = 0; q < cut.cluster; ++q) {
                if (q == place) start = carry;
                const float2 x = joint.ranks[odd][q][c];
                carry = decay(x.x, carry) + x.y;
            }
            joint.start[c] = start;
            joint.carry[c] = carry;
        }
    }
    __syncthreads();
}

// A thread's place in a group of channels.
struct Piece {
    uint32_t s, col, left, length;      // sequence, first channel, channels from there on, steps that count
    bool mine;
};
template <int E>
__device__ __forceinline__ Piece piece_of(const RecurrenceArgs& a, const Cut& cut, uint32_t group) {
    Piece p;
    const uint32_t unit = group * cut.units + (threadIdx.x & (cut.units - 1));
    p.mine = group < cut.groups && unit < cut.total;
    p.s = p.mine ? cut.vecs.div(unit) : 0;
    p.col = p.mine ? (unit - p.s * cut.vecs.divisor) * E : 0;
    p.left = a.d - p.col;
    p.length = p.mine ? a.T : 0;
    if (p.mine && a.lengths) {
        const int32_t n = a.lengths[p.s];
        p.length = n < 0 ? 0 : (uint32_t)n < a.T ? (uint32_t)n : a.T;
    }
    return p;
}
// The first of the thread's steps in a turn.
__device__ __forceinline__ uint32_t first_step(const RecurrenceArgs& a, const Cut& cut, uint32_t turn, uint32_t rank) {
    const uint64_t t = ((uint64_t)(turn * cut.cluster + rank) * (kThreads / cut.units) + threadIdx.x / cut.units) * kSteps;
    return t < a.T ? (uint32_t)t : a.T;
}

// kBack: the gradient, from the last step to the first.  The data of a thread's steps in shared memory: [gate, value, (gradient)][step][thread].
template <typename T, typename C, bool kBack>
__global__ void __launch_bounds__(kThreads, 2)
k_recurrence(const __grid_constant__ RecurrenceArgs a, const __grid_constant__ Cut cut) {
    constexpr int E = C::E, P = E / 2, kRows = (kBack ? 3 : 2) * kSteps;
    extern __shared__ __align__(16) unsigned char memory[];
    Joint<E>& joint = *reinterpret_cast<Joint<E>*>(memory);
    uint2* rows = reinterpret_cast<uint2*>(memory + (sizeof(Joint<E>) + 15) / 16 * 16) + threadIdx.x;
    float* mark = reinterpret_cast<float*>(memory + (sizeof(Joint<E>) + 15) / 16 * 16 + kRows * kThreads * 8) + threadIdx.x * E;
    const uint32_t u = threadIdx.x & (cut.units - 1), stretch = threadIdx.x / cut.units, stretches = kThreads / cut.units;
    const uint32_t channels = cut.units * E, rank = blockIdx.x % cut.cluster;
    const uint32_t at = (kBack ? stretches - 1 - stretch : stretch) * channels + u * E;      // in joint.n and b
    const uint32_t marks = (a.T + kMark - 1) / kMark;

    // asks for a turn's data
    auto ask = [&](const Piece& p, uint32_t turn) {
        const uint32_t t0 = first_step(a, cut, turn, rank);
        const uint32_t live = t0 < p.length ? p.length - t0 : 0;
        const T* gate = (const T*)a.gate.data + p.s * a.gate.batch + t0 * a.gate.step + p.col;
        const T* value = (const T*)a.value.data + p.s * a.value.batch + t0 * a.value.step + p.col;
        const T* grad = kBack ? (const T*)a.out.data + p.s * a.out.batch + t0 * a.out.step + p.col : nullptr;
        if (live >= kSteps) {
#pragma unroll
            for (int l = 0; l < kSteps; ++l, gate += a.gate.step, value += a.value.step, grad += kBack ? a.out.step : 0) {
                fetch<T, C>(rows + l * kThreads, gate, p.left);
                fetch<T, C>(rows + (kSteps + l) * kThreads, value, p.left);
                if (kBack) fetch<T, C>(rows + (2 * kSteps + l) * kThreads, grad, p.left);
            }
        } else
#pragma unroll 1
        for (int l = 0; l < kSteps; ++l) {
            if (l < live) {
                fetch<T, C>(rows + l * kThreads, gate + l * a.gate.step, p.left);
                fetch<T, C>(rows + (kSteps + l) * kThreads, value + l * a.value.step, p.left);
                if (kBack) fetch<T, C>(rows + (2 * kSteps + l) * kThreads, grad + l * a.out.step, p.left);
            } else {
                rows[l * kThreads] = infinite<T>();
                rows[(kSteps + l) * kThreads] = make_uint2(0, 0);
                if (kBack) rows[(2 * kSteps + l) * kThreads] = make_uint2(0, 0);
            }
        }
        if (kBack) {
            const float* from = a.marks + ((uint64_t)p.s * marks + t0 / kMark) * a.d + p.col;
            if (live) fetch<float, C>(mark, from, p.left);
            else
#pragma unroll
                for (int e = 0; e < E; ++e) mark[e] = 0.0f;
        }
    };
    // the state that a group begins with, by the threads of the first stretch
    auto first_state = [&](const Piece& p) {
        Pack<float, E> x = {};
        if (stretch == 0 && p.mine && a.state) x = load_columns<Columns<E, true>>(a.state + (uint64_t)p.s * a.d + p.col, p.left);
        return x;
    };

    uint32_t group = blockIdx.x / cut.cluster;
    const uint32_t clusters = gridDim.x / cut.cluster;
    Piece piece = piece_of<E>(a, cut, group);
    Pack<float, E> first = first_state(piece);
    ask(piece, kBack ? cut.turns - 1 : 0);
    if (cut.cluster > 1) {
        if (threadIdx.x == 0) {
            start_barrier(&joint.arrived[0]);
            start_barrier(&joint.arrived[1]);
            asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        }
        cg::this_cluster().sync();      // no block writes into another's memory before that one has started
    }
    for (uint32_t done = 0, count = 0; group < cut.groups; ++count) {
        const uint32_t turn = kBack ? cut.turns - 1 - done : done;
        const Piece now = piece;
        if (done == 0 && stretch == 0) {
#pragma unroll
            for (int e = 0; e < E; ++e) joint.carry[u * E + e] = first.v[e];
        }
        fetched();
        Two n[kSteps][P], slope[kBack ? kSteps : 1][P], all_n[P], all_b[P];
        uint2 other[kSteps];      // values; backward: gradients
#pragma unroll
        for (int p = 0; p < P; ++p) all_n[p] = all_b[p] = Two(0.0f);
        if constexpr (!kBack) {
#pragma unroll
            for (int l = 0; l < kSteps; ++l) {
                Two gate[P], v[P];
                unpack<T, false>(rows[l * kThreads], gate);
                other[l] = rows[(kSteps + l) * kThreads];
                unpack<T, true>(other[l], v);
#pragma unroll
                for (int p = 0; p < P; ++p) {
                    n[l][p] = complement(exp_of<T>(gate[p]));
                    all_n[p] = join_rest(all_n[p], n[l][p]);
                    all_b[p] = fma2(n[l][p], v[p], decay(n[l][p], all_b[p]));
                }
            }
        } else {
            Two h[P];
#pragma unroll
            for (int p = 0; p < P; ++p) h[p] = Two(mark[2 * p], mark[2 * p + 1]);
#pragma unroll
            for (int l = 0; l < kSteps; ++l) {
                Two gate[P], v[P];
                unpack<T, false>(rows[l * kThreads], gate);
                unpack<T, true>(rows[(kSteps + l) * kThreads], v);
#pragma unroll
                for (int p = 0; p < P; ++p) {
                    const Two e = exp_of<T>(gate[p]);
                    n[l][p] = complement(e);
                    slope[l][p] = (e * n[l][p]) * n[l][p] * (h[p] + v[p]);      // (-f) (-(1 - f)) (h - v)
                    h[p] = fma2(n[l][p], v[p], decay(n[l][p], h[p]));
                }
                other[l] = rows[(2 * kSteps + l) * kThreads];
            }
#pragma unroll
            for (int l = kSteps - 1; l >= 0; --l) {
                Two dh[P];
                unpack<T, false>(other[l], dh);
#pragma unroll
                for (int p = 0; p < P; ++p) {
                    all_n[p] = join_rest(all_n[p], n[l][p]);
                    all_b[p] = decay(n[l][p], all_b[p] + dh[p]);      // padding: the gradient passes, none is added
                }
            }
        }
        // the next turn's data, of this group or of the next
        if (++done == cut.turns) {
            done = 0;
            group += clusters;
            piece = piece_of<E>(a, cut, group);
            first = first_state(piece);
        }
        if (group < cut.groups) ask(piece, kBack ? cut.turns - 1 - done : done);
#pragma unroll
        for (int p = 0; p < P; ++p) {
            *reinterpret_cast<float2*>(&joint.n[at + 2 * p]) = all_n[p].floats();
            *reinterpret_cast<float2*>(&joint.b[at + 2 * p]) = all_b[p].floats();
        }
        join_block<E>(joint, cut, stretches, kBack ? cut.cluster - 1 - rank : rank, count);
        Two x[P];      // the state before the thread's steps; backward: its gradient behind them
#pragma unroll
        for (int p = 0; p < P; ++p) {
            const float2 then_n = *reinterpret_cast<const float2*>(&joint.n[at + 2 * p]), then_b = *reinterpret_cast<const float2*>(&joint.b[at + 2 * p]);
            x[p] = decay(Two(then_n.x, then_n.y), Two(joint.start[u * E + 2 * p], joint.start[u * E + 2 * p + 1])) + Two(then_b.x, then_b.y);
        }
        __syncthreads();
        const uint32_t t0 = first_step(a, cut, turn, rank);
        if (now.mine && t0 < a.T) {
            if constexpr (!kBack) {
                T* out = (T*)a.out.data + now.s * a.out.batch + t0 * a.out.step + now.col;
                if (a.marks) {
                    float y[E];
#pragma unroll
                    for (int p = 0; p < P; ++p) {
                        const float2 f = x[p].floats();
                        y[2 * p] = f.x;
                        y[2 * p + 1] = f.y;
                    }
                    store_columns<C>(a.marks + ((uint64_t)now.s * marks + t0 / kMark) * a.d + now.col, y, now.left);
                }
                const bool whole = t0 + kSteps <= now.length;
#pragma unroll
                for (int l = 0; l < kSteps; ++l, out += a.out.step) {
                    Two v[P];
                    unpack<T, true>(other[l], v);
#pragma unroll
                    for (int p = 0; p < P; ++p) x[p] = fma2(n[l][p], v[p], decay(n[l][p], x[p]));
                    uint2 raw = pack<T>(x);
                    if (!whole) {
                        if (t0 + l >= a.T) break;
                        if (t0 + l >= now.length) raw = make_uint2(0, 0);
                    }
                    store_raw<T, C>(out, raw, now.left);
                }
            } else {
                T* dgate = (T*)a.dgate.data + now.s * a.dgate.batch + t0 * a.dgate.step + now.col;
                T* dvalue = (T*)a.dvalue.data + now.s * a.dvalue.batch + t0 * a.dvalue.step + now.col;
                const bool whole = t0 + kSteps <= now.length;
#pragma unroll
                for (int l = kSteps - 1; l >= 0; --l) {
                    Two dh[P], dg[P], dv[P];
                    unpack<T, false>(other[l], dh);
#pragma unroll
                    for (int p = 0; p < P; ++p) {
                        const Two D = dh[p] + x[p];
                        x[p] = decay(n[l][p], D);
                        dg[p] = slope[l][p] * D;
                        dv[p] = n[l][p] * D;      // the sign is changed below
                    }
                    uint2 g = pack<T>(dg), v = pack<T>(dv);
                    constexpr uint32_t sign = sizeof(T) == 4 ? 0x80000000u : 0x80008000u;
                    v.x ^= sign;
                    v.y ^= sign;
                    if (!whole) {
                        if (t0 + l >= a.T) continue;
                        if (t0 + l >= now.length) g = v = make_uint2(0, 0);
                    }
                    store_raw<T, C>(dgate + l * a.dgate.step, g, now.left);
                    store_raw<T, C>(dvalue + l * a.dvalue.step, v, now.left);
                }
            }
        }
        // after a group's last turn: joint.carry is written again behind the next barrier
        if (done == 0 && a.last && now.mine && rank == 0 && stretch == 0)
#pragma unroll
            for (int e = 0; e < E; ++e)
                if (!C::kRagged || e < (int)now.left) a.last[(uint64_t)now.s * a.d + now.col + e] = joint.carry[u * E + e];
    }
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
    const Pack<float, E> old = load_columns<C>(a.state + row, left);
    float h[E];
#pragma unroll
    for (int e = 0; e < E; e += 2) {
        const float2 n = complement(exp_of<T>(Two(to_float(g.v[e]), to_float(g.v[e + 1])))).floats();
        h[e] = fmaf(n.x, -to_float(v.v[e]), decay(n.x, old.v[e]));
        h[e + 1] = fmaf(n.y, -to_float(v.v[e + 1]), decay(n.y, old.v[e + 1]));
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
template <int E, typename F>
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

// Cuts the work so that the blocks that the device holds at once, two to a multiprocessor, come out even: the fewest turns of the busiest one,
// where a turn of a cluster counts an eighth more for its barrier.
Cut cut_of(const RecurrenceArgs& a, uint32_t e, int sms) {
    Cut c;
    c.vecs = FastDiv((a.d + e - 1) / e);
    c.total = a.B * c.vecs.divisor;
    // stretches enough for the sequence, 32 at most
    uint32_t stretches = 1;
    while (stretches < 32 && stretches * kSteps < a.T) stretches *= 2;
    c.units = kThreads / stretches;
    c.groups = (c.total + c.units - 1) / c.units;
    c.cluster = 1;
    uint64_t least = ~0ull;
    for (uint32_t cluster = 1; cluster <= kMostCluster; cluster *= 2) {
        const uint64_t span = (uint64_t)cluster * stretches * kSteps, turns = (a.T + span - 1) / span;
        const uint64_t room = (uint64_t)sms * 2 / cluster, rounds = (c.groups + room - 1) / room;
        const uint64_t cost = turns * rounds * (cluster > 1 ? 9 : 8);
        if (cost < least) {
            least = cost;
            c.cluster = cluster;
            c.turns = (uint32_t)turns;
        }
        if (turns == 1 || c.units * e > kClusterChannels) break;
    }
    return c;
}

template <typename T, typename C, bool kBack>
cudaError_t launch_cut(cudaStream_t stream, const RecurrenceArgs& a, int sms) {
    const Cut c = cut_of(a, C::E, sms);
    auto* kernel = k_recurrence<T, C, kBack>;
    constexpr size_t shared = (sizeof(Joint<C::E>) + 15) / 16 * 16 + (kBack ? 3 : 2) * kSteps * kThreads * 8 + (kBack ? kThreads * C::E * 4 : 0);
    static_assert(2 * (shared + 1024) <= 227 * 1024, "two blocks to a multiprocessor");
    cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)shared);
    if (e == cudaSuccess && c.cluster > 8) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
    if (e != cudaSuccess) return e;
    uint32_t clusters = (uint32_t)sms * 2 / c.cluster;
    if (clusters > c.groups) clusters = c.groups;
    if (!clusters) clusters = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(clusters * c.cluster);
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = shared;
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim = {c.cluster, 1, 1};
    cfg.attrs = attr;
    cfg.numAttrs = c.cluster > 1 ? 1 : 0;
    return cudaLaunchKernelEx(&cfg, kernel, a, c);
}

}  // namespace

cudaError_t launch_recurrence(cudaStream_t stream, const RecurrenceArgs& a, int sms) {
    return with_type(a.type, [&](auto t) {
        using T = decltype(t);
        return with_pieces<8 / sizeof(T)>(a, false, [&](auto c) { return launch_cut<T, decltype(c), false>(stream, a, sms); });
    });
}

cudaError_t launch_recurrence_gradient(cudaStream_t stream, const RecurrenceArgs& a, int sms) {
    return with_type(a.type, [&](auto t) {
        using T = decltype(t);
        return with_pieces<8 / sizeof(T)>(a, true, [&](auto c) { return launch_cut<T, decltype(c), true>(stream, a, sms); });
    });
}

cudaError_t launch_recurrence_step(cudaStream_t stream, const RecurrenceArgs& a) {
    return with_type(a.type, [&](auto t) {
        using T = decltype(t);
        constexpr int E = 8 / sizeof(T);
        return with_pieces<E>(a, false, [&](auto c) {
            using C = decltype(c);
            const FastDiv vecs((a.d + E - 1) / E);
            const uint32_t total = a.B * vecs.divisor;
            k_recurrence_step<T, C><<<(total + 127) / 128, 128, 0, stream>>>(a, vecs, total);
            return cudaGetLastError();
        });
    });
}

}  // namespace tensair
