// The draw of the next token from rows of logits and given random numbers.
//
// A row's tokens are ordered by (logit descending, id ascending).  Kept are: the first k; of those the tokens with less than
// p times the mass of those before them; of those the ones whose logit is at least temperature * ln(min_p) below the largest.  All three keep
// a front of the order, so the kept tokens are the logits above a border and the first few, by id, of those on it.  The token
// is the lowest id whose running kept weight, ids ascending, exceeds u times the whole.
//
// Nothing is sorted.  The border is found by counting logits (or adding up their weights) into 1,024 buckets, first of equal width below
// the largest logit, then of ever narrower ranges of the bits of the bucket that holds the border, until that holds one value.
// A weight is exp((logit - largest) / temperature), in 64 bits, rounded to a multiple of 2^-bits: sums of weights are whole numbers, exact in
// any order, so the draw does not depend on how a row is cut or on timing, and shared-memory atomics may add them up.
//
// Few of a row's tokens are near the border, though.  One pass counts all logits (and adds up their weights, where a share of the mass is
// asked for); the counts bound the masses, and say from which logit on the border must lie.  Those tokens, in order of their ids, are
// taken out into the shared memory of one block, which finds border and token among them.
//
// A block has a row to itself in large batches; in small ones a cluster of blocks shares it.  Bound by instructions (256 rows of 100,000 bf16
// logits, 0.9 of the mass: 100 to 108 us, of which the pass with the weights takes a third, 34 instructions a logit; reading alone would be 8) and, for
// single rows, by the latency of some 25 steps with a barrier each (one row of 100,000: 22 us).
#include <cooperative_groups.h>

#include <atomic>
#include <cstddef>
#include <type_traits>

#include "columns.cuh"
#include "kernels.h"
#include "layers.h"
#include "sample_cut.h"

namespace tensair {

namespace {

namespace cg = cooperative_groups;

constexpr int kThreads = 512;
constexpr int kWarps = kThreads / 32;
constexpr uint32_t kMostCluster = kMostRowBlocks;
constexpr uint32_t kBuckets = 1024;          // two to a thread
constexpr float kPerLogit = 48.0f;           // buckets of the first turn
typedef unsigned long long mass_t;

// Keys order as logits do, 16-bit logits in 16 bits; NaN counts as minus infinity, minus zero as zero.
template <typename T>
struct Keys {
    static constexpr int kBits = sizeof(T) * 8;
    static constexpr uint32_t kSign = 1u << (kBits - 1), kAll = kSign | (kSign - 1);
    static __device__ __forceinline__ uint32_t bits_of(T x) {
        if constexpr (sizeof(T) == 4) return __float_as_uint(x);
        else return *reinterpret_cast<const unsigned short*>(&x);
    }
    static __device__ __forceinline__ uint32_t of(T x) {
        const uint32_t b = bits_of(x);
        const uint32_t k = b & kSign ? (b == kSign ? kSign : ~b & kAll) : b | kSign;
        return to_float(x) == to_float(x) ? k : nothing();
    }
    static __device__ __forceinline__ float logit(uint32_t key) {
        const uint32_t b = key & kSign ? key & ~kSign : ~key & kAll;
        if constexpr (sizeof(T) == 4) return __uint_as_float(b);
        else {
            const unsigned short h = (unsigned short)b;
            return to_float(*reinterpret_cast<const T*>(&h));
        }
    }
    // of minus infinity, the lowest key
    static __device__ __forceinline__ uint32_t nothing() { return ~bits_of(from_float<T>(-INFINITY)) & kAll; }
};

// (ln 2 / 32)^k / k!: in constant memory, from where the multiply-adds take them as operands (as literals they cost two moves each, for
// every logit: 30 instructions a logit more in the kernel's first form).
__constant__ double kSeries[6] = {1.0, 0.02166084939249829, 0.00023459619820224677, 1.6938509724371819e-06,
                                    9.172562701824643e-09, 3.9737099845494154e-11};
constexpr double kLog2e = 1.44269504088896340736;

// Weights relative to that of the largest logit.  Logits up to `least` have none.
struct Weights {
    double largest, step;            // 32 log2(e) / temperature
    const double* roots;             // 2^(j/32), j < 32
    double magic;                    // 2^(52 - bits)
    float top, least;
    bool alone;                      // only the largest logit has weight: it is infinite, or the next smaller number is too far below
    uint32_t bits;

    __device__ __forceinline__ double gap(float x) const { return x == top ? 0.0 : (double)x - largest; }
    __device__ void set(float largest_logit, float temperature, double log2e_32_by_temperature, uint32_t weight_bits, const double* table) {
        top = largest_logit;
        largest = (double)top;
        step = log2e_32_by_temperature;
        roots = table;
        bits = weight_bits;
        magic = __longlong_as_double((long long)(1023 + 52 - (int)bits) << 52);
        const double none = -32.0 * (bits + 2);
        least = (float)(largest - (double)temperature * ((bits + 2) / kLog2e));
        if (!(least < top)) least = top;
        // the next number further down, a few times at most: the first one below has rounded to here
        while (gap(least) * step > none && least != -INFINITY) least = __uint_as_float(least > 0.0f ? __float_as_uint(least) - 1 : least < 0.0f ? __float_as_uint(least) + 1 : 0x80000001u);
        alone = !(gap(least) * step > -32000.0);
    }
    // As raw bits: the sum of n of them less n times none() is the sum of the weights, as whole numbers.
    // exp by table and polynomial (after Tang, ACM TOMS 15, 1989): 2^(s/32) = 2^(n/32) 2^((s-n)/32) with |s - n| <= 1/2, the
    // latter by its series up to the fifth power (what is left out is below 2.3e-15 of it).
    // fall: how many 32nds of an octave it is below the largest (rounded).
    template <bool kAlone>
    __device__ __forceinline__ mass_t raw(float x, int& fall) const {
        if (kAlone) {
            fall = x == top ? 0 : kBuckets;
            return (mass_t)__double_as_longlong((x == top ? 1.0 : 0.0) + magic);
        }
        const double g = (double)fmaxf(x, least) - largest;
        const double shifted = fma(g, step, 0x1.8p52);
        const int n = (int)__double_as_longlong(shifted);
        fall = -n;
        const double r = fma(g, step, 0x1.8p52 - shifted);
        double y = kSeries[5];
        y = fma(y, r, kSeries[4]);
        y = fma(y, r, kSeries[3]);
        y = fma(y, r, kSeries[2]);
        y = fma(y, r, kSeries[1]);
        y = fma(y, r, 1.0) * roots[n & 31];
        y = __hiloint2double(__double2hiint(y) + ((n >> 5) << 20), __double2loint(y));
        return (mass_t)__double_as_longlong(y + magic);
    }
    template <bool kAlone>
    __device__ __forceinline__ mass_t raw(float x) const {
        int fall;
        return raw<kAlone>(x, fall);
    }
    __device__ __forceinline__ mass_t none() const { return (mass_t)__double_as_longlong(magic); }
    __device__ __forceinline__ mass_t of(float x) const { return (alone ? raw<true>(x) : raw<false>(x)) - none(); }
};

// The tokens kept: keys above `key`, and the first `ties` ids of those that have it (kAllTies: all).
constexpr uint32_t kAllTies = 0xFFFFFFFFu;
struct Border {
    uint32_t key, ties;
    __device__ __forceinline__ bool operator<(const Border& o) const { return key > o.key || (key == o.key && ties < o.ties); }   // keeps less
};

// Tokens that are taken out of a row, at most.  0.9 of the mass of 100,000 logits (normal, 3.1 wide): 3,100 tokens, in one row of twelve more
// than 4,096, for which the search through the whole row would take three times as long and the others wait.  Rows of which more is kept go that way
// still.  bf16 logits 3.1 wide, 0.95 of the mass at temperatures 1 (7,300 of 100,000 tokens, about the list's length) and 1.3 (23,000), and 0.9 at 0.8
// (500) beside them: 256 rows of 100,000 217, 247 and 100 us; 24 of 500,000 146, 171 and 76; one of 100,000 47, 63 and 42.
constexpr uint32_t kList = 8192;
struct Shared {
    // logits (of any type) and ids of tokens that are taken out
    alignas(16) unsigned char listed[kList * 4];
    alignas(16) uint32_t ids[kList];
    // of two turns; a mass is high 2^32 + low.  Read two at a time.
    alignas(16) uint32_t count[2][kBuckets];
    alignas(16) uint32_t low[2][kBuckets];
    alignas(16) uint32_t high[2][kBuckets];
    double roots[32];
    // what each block of the cluster tells the others
    mass_t mass[kMostCluster];
    uint32_t largest[kMostCluster], first[kMostCluster], ties[kMostCluster], tokens[kMostCluster];
    mass_t warp_mass[kWarps];
    uint32_t warp_count[kWarps];
    // the bucket that holds the border
    mass_t mass_before;
    uint32_t bucket, count_before, count_in;
    uint32_t edge[2];
};
constexpr uint32_t kShort = 4096;            // rows whose border is looked for among all their tokens
constexpr uint32_t kSharedBytes = (sizeof(Shared) + 15) / 16 * 16;

// A row's slice, cut into kWarps runs of `steps` accesses of a warp.
template <typename T>
struct Slice {
    static constexpr int E = 16 / sizeof(T);
    const T* logits;           // in shared or in device memory
    uint32_t begin, length;    // in the row
    uint32_t steps;
    bool whole;                // accesses of 16 bytes
    __device__ __forceinline__ uint32_t place(uint32_t run, uint32_t step) const { return ((run * steps + step) * 32 + (threadIdx.x & 31)) * E; }
    __device__ __forceinline__ uint32_t place(uint32_t step) const { return place(threadIdx.x / 32, step); }
    // E logits from `at` on; behind the slice: minus infinity
    __device__ __forceinline__ Pack<T, E> load(uint32_t at) const {
        if (whole && at + E <= length) return load_pack<T, E>(logits + at);
        Pack<T, E> x;
#pragma unroll
        for (int e = 0; e < E; ++e) x.v[e] = at + e < length ? logits[at + e] : from_float<T>(-INFINITY);
        return x;
    }
    // One bit for each logit from `from` on.
    static __device__ __forceinline__ uint32_t from_on(const Pack<T, E>& x, T from) {
        uint32_t mask = 0;
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int e = 0; e < E; ++e) mask |= (x.v[e] >= from ? 1u : 0u) << e;
        } else {
            // two comparisons in one; of four results' bytes a bit each
            using Two = std::conditional_t<std::is_same_v<T, __half>, __half2, __nv_bfloat162>;
            const Two* two = reinterpret_cast<const Two*>(x.v);
            Two edge;
            edge.x = edge.y = from;
#pragma unroll
            for (int e = 0; e < E; e += 4) {
                const uint32_t bytes = __byte_perm(__hge2_mask(two[e / 2], edge), __hge2_mask(two[e / 2 + 1], edge), 0x6420);
                mask |= ((bytes & 0x08040201u) * 0x01010101u >> 24) << e;
            }
        }
        return mask;
    }
    // f(place, logits) for the accesses of the thread.  (Several read before the first is used: no faster for 32-bit logits, and a fifth slower
    // for 16-bit ones, for want of registers.)
    template <typename F>
    __device__ __forceinline__ void accesses(F&& f) const {
        for (uint32_t s = 0; s < steps; ++s) {
            const uint32_t at = place(s);
            if (at - (threadIdx.x & 31) * E >= length) break;      // the same for a warp
            f(at, load(at));
        }
    }
    template <typename F>
    __device__ __forceinline__ void each(F&& f) const {
        accesses([&](uint32_t, const Pack<T, E>& x) {
#pragma unroll
            for (int e = 0; e < E; ++e) f(x.v[e]);
        });
    }
};

__device__ __forceinline__ uint32_t warp_max(uint32_t x) { return __reduce_max_sync(0xFFFFFFFFu, x); }
__device__ __forceinline__ mass_t warp_sum(mass_t x) {
#pragma unroll
    for (int o = 16; o; o /= 2) x += __shfl_xor_sync(0xFFFFFFFFu, x, o);
    return x;
}

struct Team {                  // the cluster
    uint32_t size, rank;
    __device__ __forceinline__ void sync() const {
        if (size > 1) cg::this_cluster().sync();
        else __syncthreads();
    }
    // No block writes into another's memory before that one has started: it says so first thing, and asks before it writes.
    __device__ __forceinline__ void started() const {
        if (size > 1) asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");
    }
    __device__ __forceinline__ void all_started() const {
        if (size > 1) asm volatile("barrier.cluster.wait.aligned;" ::: "memory");
    }
    template <typename T>
    __device__ __forceinline__ T* of(T* p, uint32_t r) const { return size > 1 ? cg::this_cluster().map_shared_rank(p, r) : p; }
};

// The bucket, of equal width in logits below the largest.
__device__ __forceinline__ uint32_t linear_bucket(float x, float largest) {
    const float gap = fminf((largest - x) * kPerLogit, (float)(kBuckets - 1));      // NaN: the last one
    return x == largest ? 0 : (uint32_t)gap;
}

// The largest key up to `top` whose linear bucket is at least b (there is one for any b < kBuckets), by one warp.
template <typename T>
__device__ __forceinline__ uint32_t key_at(uint32_t b, uint32_t top, float largest) {
    uint32_t lo = Keys<T>::nothing(), hi = top;      // buckets fall as keys rise
    const uint32_t lane = threadIdx.x & 31;
    while (lo < hi) {      // 32 probes between lo, which has it, and hi
        const uint32_t step = (hi - lo + 31) / 32, probe = lo + (lane + 1) * step;
        const bool has = probe <= hi && linear_bucket(Keys<T>::logit(probe), largest) >= b;
        const uint32_t n = __popc(__ballot_sync(0xFFFFFFFFu, has));
        lo += n * step;
        const uint32_t end = lo + step - 1;      // the next probe does not have it, or lies behind hi
        if (end < hi) hi = end;
    }
    return lo;
}

// What every thread of the cluster has added up.
__device__ __forceinline__ mass_t team_sum(Shared& sh, const Team& team, mass_t x) {
    const uint32_t lane = threadIdx.x & 31, warp = threadIdx.x / 32;
    x = warp_sum(x);
    __syncthreads();
    if (lane == 0) sh.warp_mass[warp] = x;
    __syncthreads();
    if (warp == 0) {
        x = warp_sum(lane < kWarps ? sh.warp_mass[lane] : 0);
        if (lane < team.size) *team.of(&sh.mass[team.rank], lane) = x;
    }
    team.sync();
    x = 0;
    for (uint32_t r = 0; r < team.size; ++r) x += sh.mass[r];
    return x;
}

// The thread's two buckets, added up over the cluster, and what is in the buckets before them; `whole`: what is in all.
template <bool kByMass>
struct Pair {
    uint32_t count[2], before;
    mass_t mass[2], mass_before, whole;
    __device__ __forceinline__ Pair(Shared& sh, const Team& team, uint32_t which) : count{0, 0}, before(0), mass{0, 0}, mass_before(0), whole(0) {
        const uint32_t tid = threadIdx.x, lane = tid & 31, warp = tid / 32;
#pragma unroll 4
        for (uint32_t i = 0; i < team.size; ++i) {
            const uint32_t r = (team.rank + i) & (team.size - 1);      // each its own first: no block is read by all others at once
            const uint2 c = *(const uint2*)team.of(&sh.count[which][tid * 2], r);
            count[0] += c.x;
            count[1] += c.y;
            if (kByMass) {
                const uint2 l = *(const uint2*)team.of(&sh.low[which][tid * 2], r), h = *(const uint2*)team.of(&sh.high[which][tid * 2], r);
                mass[0] += (mass_t)h.x << 32 | l.x;
                mass[1] += (mass_t)h.y << 32 | l.y;
            }
        }
        uint32_t upto = count[0] + count[1];
        mass_t mass_upto = mass[0] + mass[1];
#pragma unroll
        for (int o = 1; o < 32; o *= 2) {
            const uint32_t c = __shfl_up_sync(0xFFFFFFFFu, upto, o);
            const mass_t m = kByMass ? __shfl_up_sync(0xFFFFFFFFu, mass_upto, o) : 0;
            if (lane >= (uint32_t)o) {
                upto += c;
                mass_upto += m;
            }
        }
        if (lane == 31) {
            sh.warp_count[warp] = upto;
            if (kByMass) sh.warp_mass[warp] = mass_upto;
        }
        // the other turn's buckets are read by nobody any more
        for (uint32_t b = tid; b < kBuckets; b += kThreads) sh.count[which ^ 1][b] = sh.low[which ^ 1][b] = sh.high[which ^ 1][b] = 0;
        __syncthreads();
        before = upto - count[0] - count[1];
        mass_before = mass_upto - mass[0] - mass[1];
        for (int w = 0; w < kWarps; ++w) {
            if (w < (int)warp) {
                before += sh.warp_count[w];
                if (kByMass) mass_before += sh.warp_mass[w];
            }
            if (kByMass) whole += sh.warp_mass[w];
        }
    }
};

// The place that the random number u has in the kept weight.
__device__ __forceinline__ mass_t target_of(float u, mass_t total) {
    const mass_t target = u > 0.0f ? u < 1.0f ? (mass_t)((double)u * (double)total) : total - 1 : 0;
    return target < total ? target : total - 1;
}
__device__ __forceinline__ float logprob_of(const Weights& weights, float logit, float temperature, mass_t total) {
    return (float)(weights.gap(logit) / (double)temperature - log((double)total * exp2(-(double)weights.bits)));
}

// A front of the order that the border is in: the logits from `from` on, `tokens` of them.
struct Front {
    float from;
    uint32_t tokens;
    mass_t whole;      // weight of all tokens; by mass alone
};
// By rank: the buckets up to the one with the k-th token.  By mass: the counts in the buckets bound the masses there, from below and
// from above, which gives a bucket that the border cannot be behind.
template <bool kByMass, typename T>
__device__ Front find_front(Shared& sh, const Slice<T>& slice, const Team& team, const Weights& weights, uint32_t top, uint32_t& turn, uint32_t k, double share) {
    const uint32_t tid = threadIdx.x, lane = tid & 31, warp = tid / 32, which = turn & 1;
    const float largest = weights.top;
    ++turn;
    mass_t sum = 0;
    uint32_t n = 0;
    if (kByMass && !weights.alone)
        slice.each([&](T x) {
            int fall;
            sum += weights.template raw<false>(to_float(x), fall);
            atomicAdd(&sh.count[which][fall < (int)kBuckets ? fall : kBuckets - 1], 1);
            ++n;
        });
    else if (!kByMass)
        slice.each([&](T x) { atomicAdd(&sh.count[which][linear_bucket(to_float(x), largest)], 1); });
    else return Front{-INFINITY, kList + 1, 0};      // few have weight, and who knows how many: the search among all finds them
    Front front{-INFINITY, kList + 1, 0};
    if (kByMass) front.whole = team_sum(sh, team, sum - n * weights.none());
    else team.sync();
    const Pair<false> mine(sh, team, which);
    const uint32_t upto[2] = {mine.before + mine.count[0], mine.before + mine.count[0] + mine.count[1]};
    bool reached[2];
    if (kByMass) {
        // a token of bucket b weighs between 2^(-(b + 1/2) / 32) and 2^(-(b - 1/2) / 32)
        const float once = exp2f(-1.0f / 32.0f), w = exp2f((0.5f - (float)(tid * 2)) / 32.0f);
        float low[2], high[2];
        high[0] = (float)mine.count[0] * w;
        low[0] = high[0] * once;
        high[1] = (float)mine.count[1] * (w * once);
        low[1] = tid * 2 + 1 < kBuckets - 1 ? high[1] * once : 0.0f;
        high[1] += high[0];
        low[1] += low[0];
        float low_upto = low[1], high_upto = high[1];
#pragma unroll
        for (int o = 1; o < 32; o *= 2) {
            const float x = __shfl_up_sync(0xFFFFFFFFu, low_upto, o), y = __shfl_up_sync(0xFFFFFFFFu, high_upto, o);
            if (lane >= (uint32_t)o) {
                low_upto += x;
                high_upto += y;
            }
        }
        __syncthreads();
        if (lane == 31) {
            sh.warp_count[warp] = __float_as_uint(low_upto);
            sh.warp_mass[warp] = __float_as_uint(high_upto);
        }
        __syncthreads();
        float low_before = low_upto - low[1], high_before = high_upto - high[1], high_all = 0.0f;
        for (uint32_t v = 0; v < kWarps; ++v) {
            const float h = __uint_as_float((uint32_t)sh.warp_mass[v]);
            if (v < warp) {
                low_before += __uint_as_float(sh.warp_count[v]);
                high_before += h;
            }
            high_all += h;
        }
        // an eighth of a percent, and 2^-16 of all that was added, for what is rounded
        const double scale = exp2(-(double)weights.bits);
        const float target = (float)(share * (double)front.whole * scale) * 1.00125f, rest = (float)((1.0 - share) * (double)front.whole * scale);
#pragma unroll
        for (int i = 0; i < 2; ++i)
            reached[i] = upto[i] > 0 &&
                         (low_before + low[i] >= target || (high_all - (high_before + high[i])) * 1.00125f + high_all * 0x1p-16f <= rest);
    } else {
#pragma unroll
        for (int i = 0; i < 2; ++i) reached[i] = upto[i] >= k;
    }
    // the first bucket that reaches it
    if (tid == 0) sh.bucket = kBuckets;
    __syncthreads();
    if (reached[0] || reached[1]) atomicMin(&sh.bucket, tid * 2 + (reached[0] ? 0 : 1));
    __syncthreads();
    const uint32_t bucket = sh.bucket;
    if (bucket / 2 == tid) sh.count_in = upto[bucket & 1];
    __syncthreads();
    if (bucket < kBuckets - 1) {
        // below every logit of the bucket, by what the arithmetic there and here may have rounded
        const float width = kByMass ? (float)(1.0 / weights.step) : 1.0f / kPerLogit;
        const float edge = largest - ((float)bucket + (kByMass ? 0.5f : 1.0f)) * width * (1.0f + 0x1p-20f);
        front.from = fmaxf(edge - fabsf(edge) * 0x1p-21f - fabsf(largest) * 0x1p-22f, -3.4028234e38f);
        front.tokens = sh.count_in;
    }
    return front;
}

enum Taken { kTooMany, kByOther, kHere };
// Takes the logits from `from` on out of the row, in order of their ids, into the cluster's first block, which goes on alone: its list is a
// slice like any other.
template <typename T>
__device__ Taken take_out(Shared& sh, Slice<T>& slice, Team& team, T from) {
    constexpr int E = Slice<T>::E;
    const uint32_t tid = threadIdx.x, lane = tid & 31, warp = tid / 32;
    // What goes of an access is kept as a byte for the second pass, as long as there is room: where the sums of masses are otherwise, which are not
    // in use yet (and are set to zero again below).
    unsigned char* bytes = reinterpret_cast<unsigned char*>(sh.low);
    static_assert(offsetof(Shared, high) == offsetof(Shared, low) + sizeof(Shared::low), "one behind the other");
    const bool kept = slice.steps * kThreads <= sizeof(sh.low) + sizeof(sh.high);
    auto clear = [&] {
        if (kept)
            for (uint32_t b = tid; b < kBuckets; b += kThreads) sh.low[0][b] = sh.low[1][b] = sh.high[0][b] = sh.high[1][b] = 0;
        __syncthreads();
    };
    uint32_t here = 0;
    for (uint32_t s = 0; s < slice.steps; ++s) {
        const uint32_t place = slice.place(s);
        if (place - lane * E >= slice.length) break;
        const uint32_t mine = slice.from_on(slice.load(place), from);
        if (kept) bytes[s * kThreads + tid] = (unsigned char)mine;
        here += __popc(mine);
    }
    here = __reduce_add_sync(0xFFFFFFFFu, here);
    __syncthreads();
    if (lane == 0) sh.warp_count[warp] = here;
    __syncthreads();
    uint32_t at = 0, count = 0;
    for (uint32_t w = 0; w < kWarps; ++w) {
        const uint32_t n = sh.warp_count[w];
        if (w < warp) at += n;
        count += n;
    }
    if (tid < team.size) *team.of(&sh.tokens[team.rank], tid) = count;
    team.sync();
    count = 0;
    for (uint32_t r = 0; r < team.size; ++r) {
        const uint32_t n = sh.tokens[r];
        if (r < team.rank) at += n;
        count += n;
    }
    if (count > kList) {
        clear();
        return kTooMany;
    }
    T* logits = team.of((T*)sh.listed, 0);
    uint32_t* ids = team.of(&sh.ids[0], 0);
    if (here)
        for (uint32_t s = 0; s < slice.steps; ++s) {
            const uint32_t place = slice.place(s);
            if (place - lane * E >= slice.length) break;
            uint32_t mine = kept ? bytes[s * kThreads + tid] : slice.from_on(slice.load(place), from);
            if (!__any_sync(0xFFFFFFFFu, mine)) continue;
            const uint32_t own = __popc(mine);
            uint32_t upto = own;
#pragma unroll
            for (int o = 1; o < 32; o *= 2) {
                const uint32_t c = __shfl_up_sync(0xFFFFFFFFu, upto, o);
                if (lane >= (uint32_t)o) upto += c;
            }
            // few lanes have any, and few of them more than one
            for (uint32_t to = at + upto - own; mine; mine &= mine - 1, ++to) {
                const uint32_t id = place + __ffs(mine) - 1;
                if (!in_bounds(nullptr, to, kList)) break;
                logits[to] = slice.logits[id];
                ids[to] = slice.begin + id;
            }
            at += __shfl_sync(0xFFFFFFFFu, upto, 31);
        }
    team.sync();      // all is there
    if (team.rank != 0) return kByOther;
    clear();
    team = Team{1, 0};
    slice.logits = (const T*)sh.listed;
    slice.begin = 0;
    slice.length = count;
    slice.steps = (count + kWarps * 32 * E - 1) / (kWarps * 32 * E);
    slice.whole = true;
    return kHere;
}

// The border by rank (k tokens are kept) or by mass (tokens are kept as long as the mass before them is below share * the whole).
// `limit`: tokens beyond it do not count; `whole`: the weight of all others, 0: of what there is here.  `lowest`: the key that no logit here
// is below; minus infinity's: the first turn has buckets of equal width.  Buckets are numbered from the largest logit down.
template <bool kByMass, typename T>
__device__ Border find_border(Shared& sh, const Slice<T>& slice, const Team& team, const Weights& weights, uint32_t top, uint32_t& turn, uint32_t k,
                              double share, mass_t whole, const Border& limit, uint32_t lowest) {
    using K = Keys<T>;
    const uint32_t tid = threadIdx.x, lane = tid & 31, warp = tid / 32;
    const float largest = weights.top;
    uint32_t lo = lowest, hi = top, shift = 0, count_before = 0, count_in = 0;
    mass_t mass_before = 0;
    double target = share * (double)whole;
    bool whole_known = whole != 0;
    const float limit_logit = K::logit(limit.key);
    const bool ties_too = limit.ties == kAllTies;
    bool linear = lowest == K::nothing();
    while ((hi - lo) >> shift >= kBuckets) ++shift;
    // ranges of 32 bits shrink by 10 bits a turn: five turns at most
    for (int turns = 0; turns < 6; ++turns, linear = false) {
        const uint32_t which = turn & 1;
        ++turn;
        auto add = [&](float x, uint32_t b, uint32_t times) {
            if (!in_bounds(nullptr, b, kBuckets)) return;
            if (kByMass) {
                const mass_t m = weights.of(x) * times;
                if (!m) return;
                const uint32_t low = (uint32_t)m, old = atomicAdd(&sh.low[which][b], low);
                const uint32_t carry = old + low < old;
                if ((uint32_t)(m >> 32) + carry) atomicAdd(&sh.high[which][b], (uint32_t)(m >> 32) + carry);
            }
            atomicAdd(&sh.count[which][b], times);
        };
        if (linear) {
            if (kByMass) {
                slice.each([&](T x) {
                    const float f = to_float(x);
                    if (f > limit_logit || (ties_too && f == limit_logit)) add(f, linear_bucket(f, largest), 1);
                });
                if (!ties_too && limit.ties && team.rank == 0 && tid == 0) add(limit_logit, linear_bucket(limit_logit, largest), limit.ties);
            } else {
                slice.each([&](T x) { add(0.0f, linear_bucket(to_float(x), largest), 1); });
            }
        } else {
            const float low = K::logit(lo), high = K::logit(hi);
            slice.each([&](T x) {
                const float f = to_float(x);
                if (f >= low && f <= high) {
                    if (kByMass && !(f > limit_logit || (ties_too && f == limit_logit))) return;
                    add(f, (hi - K::of(x)) >> shift, 1);
                } else if (!kByMass && lo == K::nothing() && f != f) add(0.0f, (hi - lo) >> shift, 1);
            });
            if (kByMass && !ties_too && limit.ties && team.rank == 0 && tid == 0 && limit.key >= lo && limit.key <= hi)
                add(limit_logit, (hi - limit.key) >> shift, limit.ties);
        }
        team.sync();
        if (tid == 0) sh.bucket = kBuckets;
        // every block adds up the cluster's buckets and looks for the border: two buckets to a thread
        const Pair<kByMass> mine(sh, team, which);
        if (kByMass && !whole_known) {
            target = share * (double)mine.whole;
            whole_known = true;
        }
        uint32_t count_base = count_before + mine.before;
        mass_t mass_base = mass_before + mine.mass_before;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const uint32_t c = count_base + mine.count[i];
            const mass_t m = mass_base + mine.mass[i];
            // the first bucket that reaches the border
            const bool before = kByMass ? count_base > 0 && (double)mass_base >= target : count_base >= k;
            const bool reached = kByMass ? c > 0 && (double)m >= target : c >= k;
            if (reached && !before) {
                sh.bucket = tid * 2 + i;
                sh.count_before = count_base;
                sh.mass_before = mass_base;
                sh.count_in = mine.count[i];
            }
            count_base = c;
            mass_base = m;
        }
        __syncthreads();
        const uint32_t bucket = sh.bucket;
        if (bucket == kBuckets) return Border{K::nothing(), kAllTies};      // the border is behind all that is here
        count_before = sh.count_before;
        mass_before = sh.mass_before;
        count_in = sh.count_in;
        if (linear) {
            if (warp < 2 && bucket + warp < kBuckets) {
                const uint32_t key = key_at<T>(bucket + warp, top, largest);
                if (lane == 0) sh.edge[warp] = key;
            }
            __syncthreads();
            hi = sh.edge[0];
            lo = bucket + 1 < kBuckets ? sh.edge[1] + 1 : K::nothing();
        } else {
            hi -= bucket << shift;
            const uint32_t width = (1u << shift) - 1;
            if (hi - lo > width) lo = hi - width;
        }
        if (kByMass ? count_in == 1 : k - count_before == count_in) return Border{lo, kAllTies};     // all of the bucket
        if (lo == hi) break;
        shift = 0;
        while ((hi - lo) >> shift >= kBuckets) ++shift;
    }
    if (!kByMass) return Border{lo, k - count_before};
    // the ties of one key: as many as begin below the target
    const mass_t each = weights.of(K::logit(lo));
    uint32_t ties = 1;
    if (each) {
        const double want = (target - (double)mass_before) / (double)each;
        ties = want > 1.0 ? want < (double)count_in ? (uint32_t)want : count_in : 1;
        while (ties > 1 && (double)(mass_before + (mass_t)(ties - 1) * each) >= target) --ties;
        while (ties < count_in && (double)(mass_before + (mass_t)ties * each) < target) ++ties;
    }
    return Border{lo, ties};
}

template <typename T>
__global__ void __launch_bounds__(kThreads, 2)
k_sample(const __grid_constant__ SampleArgs a, uint32_t cluster, uint32_t steps, bool staged, bool whole) {
    constexpr int E = Slice<T>::E;
    using K = Keys<T>;
    extern __shared__ __align__(16) unsigned char memory[];
    Shared& sh = *reinterpret_cast<Shared*>(memory);
    unsigned char* stage = memory + kSharedBytes;
    const uint32_t tid = threadIdx.x, lane = tid & 31, warp = tid / 32;
    Team team{cluster, blockIdx.x % cluster};
    team.started();
    const uint32_t row = blockIdx.x / cluster;
    const uint32_t slice_length = kWarps * steps * 32 * E;
    const T* logits = (const T*)a.logits.data + (uint64_t)row * a.logits.stride;
    Slice<T> slice;
    slice.begin = team.rank * slice_length;
    slice.length = slice.begin < a.V ? (a.V - slice.begin < slice_length ? a.V - slice.begin : slice_length) : 0;
    slice.steps = steps;
    slice.whole = whole;
    slice.logits = logits + (slice.length ? slice.begin : 0);
    for (uint32_t b = tid; b < kBuckets; b += kThreads)
        for (int w = 0; w < 2; ++w) sh.count[w][b] = sh.low[w][b] = sh.high[w][b] = 0;
    if (tid < 32) sh.roots[tid] = exp2(tid / 32.0);
    const float given = a.temperature.of(row), temperature = given < 1e30f ? given : given >= 1e30f ? 1e30f : 0.0f;      // NaN: the largest logit
    const double step = 32.0 * kLog2e / (double)temperature;
    // the slice, into shared memory, and its largest logit
    float largest = -INFINITY;
    slice.accesses([&](uint32_t at, const Pack<T, E>& x) {
        if (staged) *(Pack<T, E>*)((T*)stage + at) = x;
#pragma unroll
        for (int e = 0; e < E; ++e) largest = fmaxf(largest, to_float(x.v[e]));      // of NaN and a number: the number
    });
    if (staged) {
        slice.logits = (const T*)stage;
        slice.whole = true;
    }
    // as keys from here on: minus zero and zero are one
    uint32_t top = warp_max(K::of(from_float<T>(largest)));
    if (lane == 0) sh.warp_count[warp] = top;
    __syncthreads();
    team.all_started();
    if (warp == 0) {
        top = warp_max(lane < kWarps ? sh.warp_count[lane] : 0);
        if (lane < team.size) *team.of(&sh.largest[team.rank], lane) = top;
    }
    team.sync();
    top = K::nothing();
    for (uint32_t r = 0; r < team.size; ++r) top = top > sh.largest[r] ? top : sh.largest[r];
    largest = K::logit(top);
    if (top == K::nothing()) {      // there is no token to draw
        if (team.rank == 0 && tid == 0) {
            a.token[row] = -1;
            if (a.logprob) a.logprob[row] = -INFINITY;
        }
        return;
    }
    if (!(temperature > 0.0f)) {      // the largest logit, its lowest id
        uint32_t first = 0xFFFFFFFFu;
        slice.accesses([&](uint32_t at, const Pack<T, E>& x) {
#pragma unroll
            for (int e = E - 1; e >= 0; --e)
                if (to_float(x.v[e]) == largest && slice.begin + at + e < first) first = slice.begin + at + e;
        });
        first = __reduce_min_sync(0xFFFFFFFFu, first);
        if (lane == 0) sh.warp_count[warp] = first;
        __syncthreads();
        if (warp == 0) {
            first = __reduce_min_sync(0xFFFFFFFFu, lane < kWarps ? sh.warp_count[lane] : 0xFFFFFFFFu);
            if (lane == 0) *team.of(&sh.first[team.rank], 0) = first;
        }
        team.sync();
        if (team.rank == 0 && tid == 0) {
            for (uint32_t r = 0; r < team.size; ++r) first = first < sh.first[r] ? first : sh.first[r];
            a.token[row] = first;
            if (a.logprob) a.logprob[row] = 0.0f;
        }
        return;
    }
    Weights weights;
    weights.set(largest, temperature, step, a.bits, sh.roots);
    uint32_t turn = 0;
    Border border{K::nothing(), kAllTies};
    const int32_t first_k = a.top_k.of(row);
    const uint32_t k = first_k > 0 && (uint32_t)first_k < a.V ? (uint32_t)first_k : 0;
    const float p = a.top_p.of(row), min_p = a.min_p.of(row), u = a.uniform[row];
    if (min_p > 0.0f) {
        // the smallest logit that is close enough to the largest
        const double least = min_p < 1.0f ? (double)temperature * log((double)min_p) : 0.0;
        auto close = [&](uint32_t x) { return x == top || weights.gap(K::logit(x)) >= least; };
        uint32_t key = K::of(from_float<T>((float)((double)largest + least)));
        if (key > top) key = top;
        while (key > K::nothing() && close(key - 1)) --key;
        while (!close(key)) ++key;
        border.key = key;
    }
    bool taken_out = false;
    if (k || p < 1.0f) {
        mass_t whole = 0;
        uint32_t lowest = K::nothing();
        if (a.V > kShort) {
            const Front front = k ? find_front<false>(sh, slice, team, weights, top, turn, k, 0.0)
                                  : find_front<true>(sh, slice, team, weights, top, turn, 0, (double)p);
            whole = front.whole;
            if (front.tokens <= kList) {
                T from = from_float<T>(front.from);
                if (to_float(from) > front.from) from = from_float<T>(K::logit(K::of(from) - 1));      // rounded up
                const Taken taken = take_out(sh, slice, team, from);
                if (taken == kByOther) return;
                if (taken == kHere) {
                    taken_out = true;
                    lowest = K::of(from);
                }
            }
        }
        Border b{K::nothing(), kAllTies};
        if (k) b = find_border<false>(sh, slice, team, weights, top, turn, k, 0.0, 0, b, lowest);
        if (b < border) border = b;
        if (p < 1.0f) {
            b = find_border<true>(sh, slice, team, weights, top, turn, 0, (double)p, whole, b, lowest);
            if (b < border) border = b;
        }
    }
    // kept weights in order of ids: of each warp's run, of the blocks, of the row
    const float edge = K::logit(border.key);
    mass_t mass = 0;
    uint32_t ties = 0, n = 0;
    if (edge == -INFINITY && !weights.alone)      // all of them
        slice.each([&](T x) {
            mass += weights.template raw<false>(to_float(x));
            ++n;
        });
    else
        slice.each([&](T x) {
            const float f = to_float(x);
            if (f > edge) mass += weights.of(f);
            ties += f == edge;
        });
    mass = warp_sum(mass - n * weights.none());
    ties = __reduce_add_sync(0xFFFFFFFFu, ties);
    __syncthreads();      // the arrays were read by the search
    if (lane == 0) {
        sh.warp_mass[warp] = mass;
        sh.warp_count[warp] = ties;
    }
    __syncthreads();
    if (warp == 0) {
        const mass_t m = warp_sum(lane < kWarps ? sh.warp_mass[lane] : 0);
        const uint32_t t = __reduce_add_sync(0xFFFFFFFFu, lane < kWarps ? sh.warp_count[lane] : 0);
        if (lane < team.size) {
            *team.of(&sh.mass[team.rank], lane) = m;
            *team.of(&sh.ties[team.rank], lane) = t;
        }
    }
    team.sync();
    const mass_t each = weights.of(edge);
    // with `seen` ties before it, a run with `here` ties has so many that are kept
    auto kept_ties = [&](uint32_t seen, uint32_t here) { return seen >= border.ties ? 0u : border.ties - seen < here ? border.ties - seen : here; };
    mass_t total = 0, before = 0;
    uint32_t seen = 0, seen_before = 0;
    for (uint32_t r = 0; r < team.size; ++r) {
        if (r == team.rank) {
            before = total;
            seen_before = seen;
        }
        total += sh.mass[r] + kept_ties(seen, sh.ties[r]) * each;
        seen += sh.ties[r];
    }
    const mass_t target = target_of(u, total);
    // the warp's run that has the token: all threads find the same
    bool here = false;
    uint32_t run = 0;
    for (uint32_t w = 0; w < kWarps; ++w) {
        const mass_t m = sh.warp_mass[w] + kept_ties(seen_before, sh.warp_count[w]) * each;
        if (target >= before && target < before + m) {
            here = true;
            run = w;
            break;
        }
        before += m;
        seen_before += sh.warp_count[w];
    }
    if (!here) return;
    // the access of that run that has it: an access to a warp, kWarps at a time
    for (uint32_t s0 = 0; s0 < slice.steps; s0 += kWarps) {
        const uint32_t at = slice.place(run, s0 + warp);
        const Pack<T, E> x = s0 + warp < slice.steps ? slice.load(at) : slice.load(slice.length);
        mass_t m[E], sum = 0;
        uint32_t equal = 0;
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const float f = to_float(x.v[e]);
            m[e] = f > edge ? weights.of(f) : 0;
            equal += f == edge;
            sum += m[e];
        }
        const mass_t all = warp_sum(sum);
        const uint32_t all_equal = __reduce_add_sync(0xFFFFFFFFu, equal);
        __syncthreads();
        if (lane == 0) {
            sh.warp_mass[warp] = all;
            sh.warp_count[warp] = all_equal;
        }
        __syncthreads();
        bool mine = false, found = false;
        for (uint32_t w = 0; w < kWarps && !found; ++w) {
            const mass_t k = sh.warp_mass[w] + kept_ties(seen_before, sh.warp_count[w]) * each;
            found = target < before + k;
            mine = found && w == warp;
            if (!found) {
                before += k;
                seen_before += sh.warp_count[w];
            }
        }
        if (!found) continue;
        if (!mine) return;
        // of that access, the lane and the logit
        uint32_t upto = equal;
#pragma unroll
        for (int o = 1; o < 32; o *= 2) {
            const uint32_t c = __shfl_up_sync(0xFFFFFFFFu, upto, o);
            if (lane >= (uint32_t)o) upto += c;
        }
        uint32_t tie = seen_before + upto - equal;
#pragma unroll
        for (int e = 0; e < E; ++e)
            if (to_float(x.v[e]) == edge) {
                if (tie < border.ties) {
                    m[e] = each;
                    sum += each;
                }
                ++tie;
            }
        mass_t running = sum;
#pragma unroll
        for (int o = 1; o < 32; o *= 2) {
            const mass_t c = __shfl_up_sync(0xFFFFFFFFu, running, o);
            if (lane >= (uint32_t)o) running += c;
        }
        mass_t from = before + running - sum;
        if (target >= from && target < from + sum) {
            int place = -1;
            float logit = 0.0f;
#pragma unroll
            for (int e = 0; e < E; ++e) {
                from += m[e];
                if (place < 0 && target < from) {
                    place = e;
                    logit = to_float(x.v[e]);
                }
            }
            a.token[row] = taken_out ? sh.ids[at + place] : slice.begin + at + place;
            if (a.logprob) a.logprob[row] = logprob_of(weights, logit, temperature, total);
        }
        return;
    }
}

// Shared memory for a slice, at most: of a block that has a multiprocessor to itself, and of one that shares it with another.  (Large batches read
// their rows again out of the level-2 cache: as fast.)
constexpr uint32_t kStage = 226 * 1024 - kSharedBytes, kStageShared = 112 * 1024 - kSharedBytes;

cudaLaunchConfig_t launch_of(uint32_t rows, uint32_t cluster, uint32_t shared, cudaStream_t stream, cudaLaunchAttribute* attr) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(rows * cluster);
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = shared;
    cfg.stream = stream;
    attr->id = cudaLaunchAttributeClusterDimension;
    attr->val.clusterDim = {cluster, 1, 1};
    cfg.attrs = attr;
    cfg.numAttrs = cluster > 1 ? 1 : 0;
    return cfg;
}

// The kernel's attributes, and the largest cluster that the device holds (with the most shared memory that a block takes): once for each device.
template <typename T>
cudaError_t prepare(void (*kernel)(SampleArgs, uint32_t, uint32_t, bool, bool), int sms, uint32_t* most) {
    static std::atomic<uint32_t> known[kMaxDevices];      // 0: not asked for yet
    int device = 0;
    cudaError_t e = cudaGetDevice(&device);
    if (e != cudaSuccess) return e;
    *most = device < kMaxDevices ? known[device].load(std::memory_order_relaxed) : 0;
    if (*most) return cudaSuccess;
    e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSharedBytes + kStage);
    if (e != cudaSuccess) return e;
    *most = cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) == cudaSuccess ? kMostCluster : 8;
    for (; *most > 1; *most /= 2) {
        cudaLaunchAttribute attr[1];
        const cudaLaunchConfig_t cfg = launch_of((uint32_t)sms, *most, kSharedBytes + kStage, nullptr, attr);
        int clusters = 0;
        if (cudaOccupancyMaxActiveClusters(&clusters, kernel, &cfg) == cudaSuccess && clusters > 0) break;
    }
    cudaGetLastError();      // a refusal of a larger cluster is no error
    if (device < kMaxDevices) known[device].store(*most, std::memory_order_relaxed);
    return cudaSuccess;
}

}  // namespace

cudaError_t launch_sample(cudaStream_t stream, const SampleArgs& a, int sms) {
    return with_type(a.logits.type, [&](auto t) {
        using T = decltype(t);
        constexpr uint32_t E = Slice<T>::E, unit = kWarps * 32 * E;      // tokens of one access of a block
        auto* kernel = k_sample<T>;
        uint32_t most = 0;
        const cudaError_t e = prepare<T>(kernel, sms, &most);
        if (e != cudaSuccess) return e;
        const uint32_t cluster = row_blocks(a.n, a.V, sms, most);
        const uint32_t steps = (uint32_t)(((uint64_t)a.V + (uint64_t)cluster * unit - 1) / ((uint64_t)cluster * unit));
        const uint64_t bytes = (uint64_t)steps * unit * sizeof(T);
        const bool staged = bytes <= ((uint64_t)a.n * cluster <= (uint64_t)sms ? kStage : kStageShared);
        const bool whole = (uintptr_t)a.logits.data % 16 == 0 && (a.n < 2 || a.logits.stride % E == 0);
        cudaLaunchAttribute attr[1];
        const cudaLaunchConfig_t cfg = launch_of(a.n, cluster, kSharedBytes + (staged ? (uint32_t)bytes : 0), stream, attr);
        return cudaLaunchKernelEx(&cfg, kernel, a, cluster, steps, staged, whole);
    });
}

}  // namespace tensair
