// A gated linear recurrence, channel by channel:
//
//     f_t = sigmoid(gate_t),  h_t = f_t h_{t-1} + (1 - f_t) v_t
//
// and its gradient, with e the gradient of the state after the last step and dh_t the incoming one:
//
//     D_t = dh_t + e_{t+1},  e_t = f_t D_t,  dv_t = (1 - f_t) D_t,  dgate_t = f_t (1 - f_t) (h_{t-1} - v_t) D_t
//
// Both are first-order linear recurrences x <- f x + b.  Steps compose: (f, b) then (f', b') is (f f', f' b + b').  A thread takes
// 8 steps of a few channels and holds them in registers; the threads of a block cover more steps one after the other, the blocks of
// a cluster still more, and a block goes on with its cluster's next stretch until the sequence ends, and then with other channels.  Every
// level passes on the composition of what it holds, gets the state that it begins with, and only then makes its outputs: the inputs are
// read once.  Compositions are joined in step order, so no result depends on timing.
//
// The gradient needs h_{t-1} again: the forward call leaves the state before every eighth step in fp32 (half a byte per element),
// and a thread of the backward call replays its own 8 steps from there.
//
// A factor f, of a step or of many, is kept as q: f - 1 (never positive) from f = 1/2 on, f itself below; the sign bit tells which.  So it keeps
// its relative accuracy at both ends.  A gate near 1 remembers for as long as it should (1 - 6e-8 would be the f next to 1; products of such an f, rounded
// step after step, drift: 20,000 steps of 1 - 8e-7 were off by 6e-5).  And what is left of a state that has been forgotten is right: with
// f - 1 alone a step of gate -17 was off by 44 %, 128 steps of gate 2 by 32 %.  (Three instructions an element forward, five
// backward: 64 sequences of 1,024 of 512 in bf16 63 us as before, their gradient 98 us for 93.)
//
// The next stretch's inputs are on their way into shared memory (asynchronous copies, each thread its own) while this one's are worked on.
//
// Bound by instructions and the barriers of a turn: 64 sequences of 1,024 of 512 in bf16 take 61 us forward (201 MB), 62 with marks (218 MB, 37
// instructions an element, issue slots 0.65 busy), and 97 us backward (352 MB, 54 instructions, 0.61); from 64 to 256 sequences 0.76 us a sequence
// forward, 4.2 TB/s.  One stream of 65,536 steps: 98 us, a chain of 22 turns of 12 blocks.  One step of 64 streams: 3 us, a launch.  Rows that
// begin between two pieces (301 channels of 16 bits) are read one by one and not ahead of their turn: 64 sequences of 1,021 take 105 us and 183.
#include <cooperative_groups.h>

#include <atomic>
#include <type_traits>

#include "columns.cuh"
#include "kernels.h"
#include "layers.h"
#include "recurrence_cut.h"

namespace tensair {

namespace {

namespace cg = cooperative_groups;

using namespace recurrence;
static_assert(kSteps == kMark, "a thread's steps begin with a mark");

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
// e = exp(gate).  Gates of 16 bits: 2^x of the rounded product with log2(e), off by (1.5 |gate| + 2) 2^-24 of it, which is a choice: it is as if the
// gate were off by that, and half a unit of the gate's own last place is at least 9,000 (bf16) or 1,100 (fp16) times as much for gates of 1 and
// more, 160 or 20 times for one of 0.01.  (f and 1 - f, whichever is smaller: at most 1.4 times that off, of all gates of 16 bits.)
// Gates of 32 bits: expf; f and 1 - f at most 4.3 2^-24 off.
template <typename T>
__device__ __forceinline__ float exp_of(float gate) {
    if constexpr (sizeof(T) == 2) return exp2_approx(gate * 1.44269504f);
    else return expf(gate);
}
// f - 1 from e = exp(gate): -1 / (1 + e).  The quotient is off by a unit in the last place of 32 bits at most, and zero below 2^-126.
__device__ __forceinline__ float complement(float e) { return reciprocal_approx(-1.0f - e); }
// q of a factor: f - 1 or, where the sign bit is not set, f.
__device__ __forceinline__ bool near_one(float q) { return __float_as_int(q) < 0; }
constexpr float kOne = -0.0f;      // the factor 1
// f x
__device__ __forceinline__ float decay(float q, float x) { return fmaf(q, x, near_one(q) ? x : 0.0f); }
// (1 - f) x
__device__ __forceinline__ float share(float q, float x) { return fmaf(-q, x, near_one(q) ? 0.0f : x); }
// f x + (1 - f) v: x + n (x - v), or v + f (x - v)
__device__ __forceinline__ float advance(float q, float x, float v) { return fmaf(q, x, fmaf(-q, v, near_one(q) ? x : v)); }
// Factors one after the other: their product p, and that less one, n = sum of (f - 1) * (the product before), whose terms have one sign.  p's
// rounding errors are few (a stretch's, a block's), and n goes on where p is near 1: nothing drifts.
struct Product {
    float p = 1.0f, n = kOne;
    __device__ __forceinline__ void join(float f, float rest) {
        n = fmaf(rest, p, n);
        p *= f;
    }
    __device__ __forceinline__ float q() const { return p <= 0.5f ? p : n; }
};
// A composition: what is there already comes before what is joined to it.
struct Joined {
    Product product;
    float b = 0.0f;
    __device__ __forceinline__ void join(float q, float add) {
        const float f = near_one(q) ? q + 1.0f : q;
        product.join(f, q);      // (n is not used behind a factor of 1/2 or less)
        b = fmaf(f, b, add);
    }
};

// 8 bytes of raw elements as floats, and back.
template <typename T>
__device__ __forceinline__ void unpack(uint2 raw, float (&x)[8 / sizeof(T)]) {
    const uint32_t words[2] = {raw.x, raw.y};
#pragma unroll
    for (int p = 0; p < 2; ++p) {
        if constexpr (sizeof(T) == 4) x[p] = __uint_as_float(words[p]);
        else if constexpr (std::is_same_v<T, __nv_bfloat16>) {
            x[2 * p] = __uint_as_float(words[p] << 16);
            x[2 * p + 1] = __uint_as_float(words[p] & 0xFFFF0000u);
        } else {
            const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&words[p]));
            x[2 * p] = f.x;
            x[2 * p + 1] = f.y;
        }
    }
}
template <typename T>
__device__ __forceinline__ uint2 pack(const float (&x)[8 / sizeof(T)]) {
    uint32_t words[2];
#pragma unroll
    for (int p = 0; p < 2; ++p) {
        if constexpr (sizeof(T) == 4) words[p] = __float_as_uint(x[p]);
        else if constexpr (std::is_same_v<T, __nv_bfloat16>) {
            const __nv_bfloat162 y = __floats2bfloat162_rn(x[2 * p], x[2 * p + 1]);
            words[p] = *reinterpret_cast<const uint32_t*>(&y);
        } else {
            const __half2 y = __floats2half2_rn(x[2 * p], x[2 * p + 1]);
            words[p] = *reinterpret_cast<const uint32_t*>(&y);
        }
    }
    return make_uint2(words[0], words[1]);
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

// Between the blocks of a cluster: compositions are stored straight from registers into the others' shared memory, where a barrier counts
// their bytes.  (us of a turn of 16 blocks, two to a multiprocessor: 3.5; with the cluster's own barrier, which also waits for every store of the turn
// before, 4.4; by one copy to a block out of shared memory, behind the fence that needs, 4.1.)
__device__ __forceinline__ uint32_t shared_address(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void start_barrier(uint64_t* barrier) {
    asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" ::"r"(shared_address(barrier)) : "memory");
}
__device__ __forceinline__ void expect_bytes(uint64_t* barrier, uint32_t bytes) {
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(shared_address(barrier)), "r"(bytes) : "memory");
}
__device__ __forceinline__ void send(const float2* to, const uint64_t* barrier, uint32_t rank, float4 x) {
    uint32_t there, bar;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(there) : "r"(shared_address(to)), "r"(rank));
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(bar) : "r"(shared_address(barrier)), "r"(rank));
    asm volatile("st.async.weak.shared::cluster.mbarrier::complete_tx::bytes.v4.f32 [%0], {%1, %2, %3, %4}, [%5];"
                 ::"r"(there), "f"(x.x), "f"(x.y), "f"(x.z), "f"(x.w), "r"(bar) : "memory");
}
// False: they did not come, however often it was asked.
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
    alignas(16) float n[2][kThreads * E];      // of two turns
    alignas(16) float b[2][kThreads * E];
    float carry[kThreads * E], start[kThreads * E];
    float2 parts[kThreads];
    alignas(16) float2 ranks[2][kMostCluster][kClusterChannels];       // the cluster's compositions, of two turns
    uint64_t arrived[2];                                   // barriers that count the bytes of those
};

struct Cut : Plan {
    FastDiv vecs;          // pieces of channels of a sequence
    uint32_t total;        // of all sequences
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
        Joined all;
#pragma unroll 4
        for (uint32_t s = from; s < from + each; ++s) all.join(joint.n[odd][s * channels + c], joint.b[odd][s * channels + c]);
        if (parts > 1) joint.parts[i] = make_float2(all.product.q(), all.b);
    }
    if (parts > 1) __syncthreads();
    for (uint32_t i = threadIdx.x; i < channels * parts; i += kThreads) {
        const uint32_t c = i & (channels - 1), part = i / channels;
        Joined all;
#pragma unroll 4
        for (uint32_t q = 0; q < part; ++q) {
            const float2 x = joint.parts[q * channels + c];
            all.join(x.x, x.y);
        }
#pragma unroll 4
        for (uint32_t s = part * each; s < (part + 1) * each; ++s) {
            const float then = joint.n[odd][s * channels + c], add = joint.b[odd][s * channels + c];
            joint.n[odd][s * channels + c] = all.product.q();
            joint.b[odd][s * channels + c] = all.b;
            all.join(then, add);
        }
        const float n = all.product.q(), b = all.b;
        if (part + 1 < parts) continue;
        if (cut.cluster == 1) {
            const float carry = joint.carry[c];
            joint.start[c] = carry;
            joint.carry[c] = decay(n, carry) + b;
        } else {
            // Two neighbours send both their channels, each to half of the blocks.  What is written over has been read: who sends this turn's
            // compositions has those of the turn before, and they were sent by who had read the ones before them.
            const uint32_t lanes = last_lanes(channels, threadIdx.x);      // at most 64 channels: their last parts are those of the last threads
            const float other_n = __shfl_xor_sync(lanes, n, 1), other_b = __shfl_xor_sync(lanes, b, 1);
            const bool second = c & 1;
            const float4 both = second ? make_float4(other_n, other_b, n, b) : make_float4(n, b, other_n, other_b);
#pragma unroll 4
            for (uint32_t r = second ? cut.cluster / 2 : 0; r < (second ? cut.cluster : cut.cluster / 2); ++r)
                send(&joint.ranks[odd][place][c & ~1u], &joint.arrived[odd], r, both);
        }
    }
    if (cut.cluster > 1) {
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
    constexpr int E = C::E, kRows = (kBack ? 3 : 2) * kSteps;
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
        } else if (kBack || live)      // the forward call does not look at steps of padding alone
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
        // forward: the product of the factors up to a step, and what the steps up to it add; backward: a step's factor, and f (h - v)
        float by[kSteps][E], with[kSteps][E], all_b[E];
        uint2 grads[kBack ? kSteps : 1];
        Product all[E];
#pragma unroll
        for (int e = 0; e < E; ++e) all_b[e] = 0.0f;
        const uint32_t t0 = first_step(a, cut, turn, rank);
        // nothing but padding: the state stays  (forwards 65 us become 56, a padded batch; backwards the same made unpadded ones 8 us slower)
        if (!kBack && t0 >= now.length) {
#pragma unroll
            for (int l = 0; l < kSteps; ++l) {
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    by[l][e] = 1.0f;
                    with[l][e] = 0.0f;
                }
            }
        } else {
            float h[E];
            if constexpr (kBack) {
#pragma unroll
                for (int e = 0; e < E; ++e) h[e] = mark[e];
            }
#pragma unroll
            for (int l = 0; l < kSteps; ++l) {
                float gate[E], v[E], dh[E];
                unpack<T>(rows[l * kThreads], gate);
                unpack<T>(rows[(kSteps + l) * kThreads], v);
                if constexpr (kBack) {
                    grads[l] = rows[(2 * kSteps + l) * kThreads];
                    unpack<T>(grads[l], dh);
                }
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    const float exp_gate = exp_of<T>(gate[e]), rest = complement(exp_gate), small = exp_gate * -rest;
                    const bool near = !(gate[e] < 0.0f);
                    const float f = near ? 1.0f + rest : small;
                    all[e].join(f, rest);
                    if constexpr (!kBack) {
                        all_b[e] = fmaf(f, all_b[e], -rest * v[e]);
                        by[l][e] = all[e].p;
                        with[l][e] = all_b[e];
                    } else {
                        all_b[e] = fmaf(all[e].p, dh[e], all_b[e]);      // padding: the gradient passes, none is added
                        by[l][e] = near ? rest : small;
                        with[l][e] = f * (h[e] - v[e]);
                        h[e] = fmaf(f, h[e], -rest * v[e]);
                    }
                }
            }
        }
        float all_n[E];
#pragma unroll
        for (int e = 0; e < E; ++e) all_n[e] = all[e].q();
        // the next turn's data, of this group or of the next
        if (++done == cut.turns) {
            done = 0;
            group += clusters;
            piece = piece_of<E>(a, cut, group);
            first = first_state(piece);
        }
        if (group < cut.groups) ask(piece, kBack ? cut.turns - 1 - done : done);
        store_pack<float, E>(&joint.n[count & 1][at], all_n);
        store_pack<float, E>(&joint.b[count & 1][at], all_b);
        join_block<E>(joint, cut, stretches, kBack ? cut.cluster - 1 - rank : rank, count);
        float x[E];      // the state before the thread's steps; backward: its gradient behind them
        {
            const Pack<float, E> then_n = load_pack<float, E>(&joint.n[count & 1][at]), then_b = load_pack<float, E>(&joint.b[count & 1][at]);
#pragma unroll
            for (int e = 0; e < E; ++e) x[e] = decay(then_n.v[e], joint.start[u * E + e]) + then_b.v[e];
        }
        if (now.mine && t0 < a.T) {
            if constexpr (!kBack) {
                T* out = (T*)a.out.data + now.s * a.out.batch + t0 * a.out.step + now.col;
                if (a.marks) store_columns<C>(a.marks + ((uint64_t)now.s * marks + t0 / kMark) * a.d + now.col, x, now.left);
                const bool whole = t0 + kSteps <= now.length;
#pragma unroll
                for (int l = 0; l < kSteps; ++l, out += a.out.step) {
                    float h[E];
#pragma unroll
                    for (int e = 0; e < E; ++e) h[e] = fmaf(by[l][e], x[e], with[l][e]);
                    uint2 raw = pack<T>(h);
                    if (!whole) {
                        if (t0 + l >= a.T) break;
                        if (t0 + l >= now.length) raw = make_uint2(0, 0);
                    }
                    store_raw<T, C>(out, raw, now.left);
                }
            } else {
                T* dgate = (T*)a.dgate.data + now.s * a.dgate.batch + (t0 + kSteps - 1) * a.dgate.step + now.col;
                T* dvalue = (T*)a.dvalue.data + now.s * a.dvalue.batch + (t0 + kSteps - 1) * a.dvalue.step + now.col;
                const bool whole = t0 + kSteps <= now.length;
#pragma unroll
                for (int l = kSteps - 1; l >= 0; --l, dgate -= a.dgate.step, dvalue -= a.dvalue.step) {
                    float dh[E], dg[E], dv[E];
                    unpack<T>(grads[l], dh);
#pragma unroll
                    for (int e = 0; e < E; ++e) {
                        const float D = dh[e] + x[e];
                        x[e] = decay(by[l][e], D);
                        dv[e] = share(by[l][e], D);
                        dg[e] = with[l][e] * dv[e];
                    }
                    uint2 g = pack<T>(dg), v = pack<T>(dv);
                    if (!whole) {
                        if (t0 + l >= a.T) continue;
                        if (t0 + l >= now.length) g = v = make_uint2(0, 0);
                    }
                    store_raw<T, C>(dgate, g, now.left);
                    store_raw<T, C>(dvalue, v, now.left);
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
    for (int e = 0; e < E; ++e) {
        const float gate = to_float(g.v[e]), exp_gate = exp_of<T>(gate), rest = complement(exp_gate);
        h[e] = advance(gate < 0.0f ? exp_gate * -rest : rest, old.v[e], to_float(v.v[e]));
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

// How many clusters of each size the device holds at once, two blocks to a multiprocessor: asked for once.  (148 multiprocessors hold 71 of 4, 33 of 8,
// 14 of 16; one more than that waits until another has ended.  A part of a device may hold none of the large ones.)
template <typename T, typename C, bool kBack>
cudaError_t rooms(size_t shared, int sms, uint32_t (&room)[kSizes]) {
    auto* kernel = k_recurrence<T, C, kBack>;
    static std::atomic<int> known[kMaxDevices][kSizes];      // one more than the answer; 0: not asked for yet
    int device = 0;
    cudaError_t e = cudaGetDevice(&device);
    if (e != cudaSuccess) return e;
    for (int i = 0; i < kSizes; ++i) {
        int n = device < kMaxDevices ? known[device][i].load(std::memory_order_relaxed) - 1 : -1;
        if (n < 0) {
            e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)shared);
            if (e != cudaSuccess) return e;
            cudaLaunchConfig_t cfg = {};
            cfg.gridDim = dim3(kClusters[i] * sms);
            cfg.blockDim = dim3(kThreads);
            cfg.dynamicSmemBytes = shared;
            cudaLaunchAttribute attr[1];
            attr[0].id = cudaLaunchAttributeClusterDimension;
            attr[0].val.clusterDim = {kClusters[i], 1, 1};
            cfg.attrs = attr;
            cfg.numAttrs = 1;
            e = cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
            if (e == cudaSuccess || kClusters[i] <= 8) e = cudaOccupancyMaxActiveClusters(&n, kernel, &cfg);
            if (e != cudaSuccess) {
                if (i == 0) return e;
                cudaGetLastError();      // a refusal of a cluster is no error
                n = 0;
            }
            if (device < kMaxDevices) known[device][i].store(n + 1, std::memory_order_relaxed);
        }
        room[i] = n;
    }
    return cudaSuccess;
}

template <typename T, typename C, bool kBack>
cudaError_t launch_cut(cudaStream_t stream, const RecurrenceArgs& a, int sms) {
    auto* kernel = k_recurrence<T, C, kBack>;
    constexpr size_t shared = (sizeof(Joint<C::E>) + 15) / 16 * 16 + (kBack ? 3 : 2) * kSteps * kThreads * 8 + (kBack ? kThreads * C::E * 4 : 0);
    static_assert(2 * (shared + 1024) <= 227 * 1024, "two blocks to a multiprocessor");
    uint32_t room[kSizes];
    const cudaError_t e = rooms<T, C, kBack>(shared, sms, room);
    if (e != cudaSuccess) return e;
    Cut c;
    c.vecs = FastDiv((a.d + C::E - 1) / C::E);
    c.total = a.B * c.vecs.divisor;
    static_cast<Plan&>(c) = cut(a.T, c.total, C::E, room);
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(c.grid);
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
