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
// A cluster of blocks shares a row, each with a slice of it in its shared memory: the logits are read from memory once, whatever is
// asked for.  (Slices that do not fit are read again, out of the level-2 cache.)
#include <cooperative_groups.h>

#include "columns.cuh"
#include "layers.h"

namespace tensair {

namespace {

namespace cg = cooperative_groups;

constexpr int kThreads = 512;
constexpr int kWarps = kThreads / 32;
constexpr uint32_t kMostCluster = 16;
constexpr uint32_t kBuckets = 1024;          // two to a thread
constexpr float kPerLogit = 48.0f;           // buckets of the first turn
constexpr uint32_t kNothing = 0x007FFFFFu;   // the key of minus infinity
typedef unsigned long long mass_t;

// Keys order as logits do; NaN counts as minus infinity, minus zero as zero.
__device__ __forceinline__ uint32_t key_of(float x) {
    const uint32_t b = __float_as_uint(x + 0.0f);
    const uint32_t k = b & 0x80000000u ? ~b : b | 0x80000000u;
    return x != x ? kNothing : k;
}
__device__ __forceinline__ float logit_of(uint32_t key) {
    return __uint_as_float(key & 0x80000000u ? key & 0x7FFFFFFFu : ~key);
}

// Weights relative to that of the largest logit.
struct Weights {
    double largest, per_logit;       // log2(e) / temperature
    const double* roots;             // 2^(j/16), j < 16
    double magic;                    // 2^(52 - bits)
    uint32_t largest_key;
    // exp by table and polynomial (after Tang, ACM TOMS 15, 1989): 2^z = 2^(n/16) 2^r with |r| <= 1/32, the
    // latter by its series up to r^6 (what is left out is below 5e-16 of it)
    __device__ __forceinline__ mass_t of(uint32_t key) const {
        if (key == largest_key) return (mass_t)(__double_as_longlong(1.0 + magic) - __double_as_longlong(magic));
        const double z = ((double)logit_of(key) - largest) * per_logit;
        if (!(z > -64.0)) return 0;      // rounds to nothing: bits is at most 46
        const double shifted = z * 16.0 + 0x1.8p52;
        const int n = (int)__double_as_longlong(shifted);
        const double r = fma(shifted - 0x1.8p52, -0.0625, z) * 0.69314718055994530942;
        double y = 1.0 / 720.0;
        y = fma(y, r, 1.0 / 120.0);
        y = fma(y, r, 1.0 / 24.0);
        y = fma(y, r, 1.0 / 6.0);
        y = fma(y, r, 0.5);
        y = fma(y, r, 1.0);
        y = fma(y, r, 1.0) * roots[n & 15];
        y = __longlong_as_double(__double_as_longlong(y) + ((long long)(n >> 4) << 52));
        return (mass_t)(__double_as_longlong(y + magic) - __double_as_longlong(magic));
    }
};

// The tokens kept: keys above `key`, and the first `ties` ids of those that have it.
struct Border {
    uint32_t key, ties;
    __device__ __forceinline__ bool operator<(const Border& o) const { return key > o.key || (key == o.key && ties < o.ties); }   // keeps less
};

struct Shared {
    uint32_t count[2][kBuckets], low[2][kBuckets], high[2][kBuckets];    // of two turns; a mass is high 2^32 + low
    double roots[16];
    // what each block of the cluster tells the others
    uint32_t largest[kMostCluster], first[kMostCluster], ties[kMostCluster];
    mass_t mass[kMostCluster];
    mass_t warp_mass[kWarps];
    uint32_t warp_count[kWarps];
    // the bucket that holds the border
    mass_t mass_before;
    uint32_t bucket, count_before, count_in;
    uint32_t edge[2];
};

// A row's slice, cut into kWarps runs of `steps` accesses of a warp.
template <typename T>
struct Slice {
    static constexpr int E = 16 / sizeof(T);
    const T* logits;           // in shared or in device memory
    uint32_t begin, length;    // in the row
    uint32_t steps;
    bool whole;                // accesses of 16 bytes
    __device__ __forceinline__ uint32_t place(uint32_t step) const {
        return ((threadIdx.x / 32 * steps + step) * 32 + (threadIdx.x & 31)) * E;
    }
    // E keys from `at` on; behind the slice: minus infinity
    __device__ __forceinline__ void keys(uint32_t at, uint32_t (&key)[E]) const {
        if (whole && at + E <= length) {
            const Pack<T, E> x = load_pack<T, E>(logits + at);
#pragma unroll
            for (int e = 0; e < E; ++e) key[e] = key_of(to_float(x.v[e]));
        } else {
#pragma unroll
            for (int e = 0; e < E; ++e) key[e] = at + e < length ? key_of(to_float(logits[at + e])) : kNothing;
        }
    }
    template <typename F>
    __device__ __forceinline__ void each(F&& f) const {
        for (uint32_t s = 0; s < steps; ++s) {
            const uint32_t at = place(s);
            if (at - (threadIdx.x & 31) * E >= length) break;
            uint32_t key[E];
            keys(at, key);
#pragma unroll
            for (int e = 0; e < E; ++e) f(key[e]);
        }
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
    template <typename T>
    __device__ __forceinline__ T* of(T* p, uint32_t r) const { return size > 1 ? cg::this_cluster().map_shared_rank(p, r) : p; }
};

// The bucket, of equal width in logits below the largest.
__device__ __forceinline__ uint32_t linear_bucket(uint32_t key, uint32_t largest_key, float largest) {
    if (key == largest_key) return 0;
    const float gap = (largest - logit_of(key)) * kPerLogit;
    return gap < (float)(kBuckets - 1) ? (uint32_t)gap : kBuckets - 1;
}

// The largest key in [kNothing, largest_key] whose linear bucket is at least b (0: there is none), by one warp.
__device__ __forceinline__ uint32_t key_at(uint32_t b, uint32_t largest_key, float largest) {
    uint32_t lo = kNothing, hi = largest_key;      // buckets fall as keys rise
    const uint32_t lane = threadIdx.x & 31;
    if (linear_bucket(lo, largest_key, largest) < b) return 0;
    while (lo < hi) {      // 32 probes between lo, which has it, and hi
        const uint32_t step = (hi - lo + 31) / 32, probe = lo + (lane + 1) * step;
        const bool has = probe <= hi && probe >= lo && linear_bucket(probe, largest_key, largest) >= b;
        const uint32_t n = __popc(__ballot_sync(0xFFFFFFFFu, has));
        const uint32_t next = lo + n * step;
        const uint32_t end = next + step - 1;      // the next probe does not have it, or lies behind hi
        lo = next;
        if (end < hi) hi = end;
    }
    return lo;
}

// The border by rank (k tokens are kept) or by mass (tokens are kept as long as the mass before them is below share * the whole).
// `limit`: tokens beyond it do not count.  Buckets are numbered from the largest logit down.
template <bool kByMass, typename T>
__device__ Border find_border(Shared& sh, const Slice<T>& slice, const Team& team, const Weights& weights, uint32_t& turn, uint32_t k, double share,
                              const Border& limit) {
    const float largest = logit_of(weights.largest_key);
    const uint32_t tid = threadIdx.x, lane = tid & 31, warp = tid / 32;
    uint32_t lo = 0, hi = 0xFFFFFFFFu, shift = 0, count_before = 0, count_in = 0;
    mass_t mass_before = 0;
    double target = 0.0;
    bool linear = true;
    // ranges of 32 bits shrink by 10 bits a turn: five turns at most
    for (int turns = 0; turns < 6; ++turns, linear = false) {
        const uint32_t which = turn & 1;
        ++turn;
        auto add = [&](uint32_t key, uint32_t times) {
            if (key < lo || key > hi) return;
            const uint32_t b = linear ? linear_bucket(key, weights.largest_key, largest) : (hi - key) >> shift;
            if (kByMass) {
                const mass_t m = weights.of(key) * times;
                if (!m) return;
                const uint32_t low = (uint32_t)m, old = atomicAdd(&sh.low[which][b], low);
                const uint32_t carry = old + low < old;
                if ((uint32_t)(m >> 32) + carry) atomicAdd(&sh.high[which][b], (uint32_t)(m >> 32) + carry);
            }
            atomicAdd(&sh.count[which][b], times);
        };
        slice.each([&](uint32_t key) {
            if (!kByMass || key > limit.key) add(key, 1);
        });
        if (kByMass && limit.ties && team.rank == 0 && tid == 0) add(limit.key, limit.ties);
        team.sync();
        // every block adds up the cluster's buckets and looks for the border: two buckets to a thread
        uint32_t count[2] = {0, 0};
        mass_t mass[2] = {0, 0};
        for (uint32_t r = 0; r < team.size; ++r) {
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
            sh.warp_mass[warp] = mass_upto;
        }
        // the other turn's buckets are read by nobody any more
        for (uint32_t b = tid; b < kBuckets; b += kThreads) sh.count[which ^ 1][b] = sh.low[which ^ 1][b] = sh.high[which ^ 1][b] = 0;
        __syncthreads();
        uint32_t count_base = count_before;
        mass_t mass_base = mass_before, whole = mass_before;
        for (int w = 0; w < kWarps; ++w) {
            if (w < (int)warp) {
                count_base += sh.warp_count[w];
                mass_base += sh.warp_mass[w];
            }
            whole += sh.warp_mass[w];
        }
        if (kByMass && linear) target = share * (double)whole;
        count_base += upto - count[0] - count[1];
        mass_base += mass_upto - mass[0] - mass[1];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const uint32_t c = count_base + count[i];
            const mass_t m = mass_base + mass[i];
            // the first bucket that reaches the border
            const bool before = kByMass ? count_base > 0 && (double)mass_base >= target : count_base >= k;
            const bool reached = kByMass ? c > 0 && (double)m >= target : c >= k;
            if (reached && !before) {
                sh.bucket = tid * 2 + i;
                sh.count_before = count_base;
                sh.mass_before = mass_base;
                sh.count_in = count[i];
            }
            count_base = c;
            mass_base = m;
        }
        __syncthreads();
        const uint32_t bucket = sh.bucket;
        count_before = sh.count_before;
        mass_before = sh.mass_before;
        count_in = sh.count_in;
        if (linear) {
            if (warp < 2) {
                const uint32_t key = key_at(bucket + warp, weights.largest_key, largest);
                if (lane == 0) sh.edge[warp] = key;
            }
            __syncthreads();
            hi = sh.edge[0];
            lo = bucket + 1 < kBuckets ? sh.edge[1] + 1 : kNothing;
        } else {
            hi -= bucket << shift;
            const uint32_t width = (1u << shift) - 1;
            if (hi - lo > width) lo = hi - width;
        }
        if (kByMass ? count_in == 1 : k - count_before == count_in) return Border{lo - 1, 0};     // all of the bucket
        if (lo == hi) break;
        shift = 0;
        while ((hi - lo) >> shift >= kBuckets) ++shift;
    }
    if (!kByMass) return Border{lo, k - count_before};
    // the ties of one key: as many as begin below the target
    const mass_t each = weights.of(lo);
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
__global__ void __launch_bounds__(kThreads)
k_sample(const __grid_constant__ SampleArgs a, uint32_t cluster, uint32_t steps, bool staged, bool whole) {
    constexpr int E = Slice<T>::E;
    extern __shared__ __align__(16) unsigned char stage[];
    __shared__ Shared sh;
    const uint32_t tid = threadIdx.x, lane = tid & 31, warp = tid / 32;
    const Team team{cluster, blockIdx.x % cluster};
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
    if (tid < 16) sh.roots[tid] = exp2(tid / 16.0);
    // the slice, into shared memory, and its largest key
    uint32_t top = kNothing;
    for (uint32_t s = 0; s < steps; ++s) {
        const uint32_t at = slice.place(s);
        if (at - lane * E >= slice.length) break;
        uint32_t key[E];
        if (staged) {
            T* to = (T*)stage + at;
            Pack<T, E> x;
            if (whole && at + E <= slice.length) x = load_pack<T, E>(slice.logits + at);
            else
#pragma unroll
                for (int e = 0; e < E; ++e) x.v[e] = at + e < slice.length ? slice.logits[at + e] : from_float<T>(-INFINITY);
            *(Pack<T, E>*)to = x;
#pragma unroll
            for (int e = 0; e < E; ++e) key[e] = key_of(to_float(x.v[e]));
        } else slice.keys(at, key);
#pragma unroll
        for (int e = 0; e < E; ++e) top = top > key[e] ? top : key[e];
    }
    if (staged) {
        slice.logits = (const T*)stage;
        slice.whole = true;
    }
    top = warp_max(top);
    if (lane == 0) sh.warp_count[warp] = top;
    team.sync();          // no block writes into another's memory before that one has started
    if (warp == 0) {
        top = warp_max(lane < kWarps ? sh.warp_count[lane] : 0);
        if (lane < team.size) *team.of(&sh.largest[team.rank], lane) = top;
    }
    team.sync();
    top = kNothing;
    for (uint32_t r = 0; r < team.size; ++r) top = top > sh.largest[r] ? top : sh.largest[r];
    const float temperature = a.temperature.of(row);
    if (top == kNothing) {      // there is no token to draw
        if (team.rank == 0 && tid == 0) {
            a.token[row] = -1;
            if (a.logprob) a.logprob[row] = -INFINITY;
        }
        return;
    }
    if (!(temperature > 0.0f)) {      // the largest logit, its lowest id
        uint32_t first = 0xFFFFFFFFu;
        for (uint32_t s = 0; s < steps; ++s) {
            const uint32_t at = slice.place(s);
            if (at - lane * E >= slice.length) break;
            uint32_t key[E];
            slice.keys(at, key);
#pragma unroll
            for (int e = E - 1; e >= 0; --e)
                if (key[e] == top && slice.begin + at + e < first) first = slice.begin + at + e;
        }
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
    weights.largest = logit_of(top);
    weights.largest_key = top;
    weights.per_logit = 1.44269504088896340736 / (double)temperature;
    weights.roots = sh.roots;
    weights.magic = __longlong_as_double((long long)(1023 + 52 - (int)a.bits) << 52);
    uint32_t turn = 0;
    Border border{0, 0};
    const int32_t k = a.top_k.of(row);
    if (k > 0 && (uint32_t)k < a.V) border = find_border<false>(sh, slice, team, weights, turn, (uint32_t)k, 0.0, border);
    const float p = a.top_p.of(row);
    if (p < 1.0f) {
        const Border b = find_border<true>(sh, slice, team, weights, turn, 0, (double)p, border);
        if (b < border) border = b;
    }
    const float min_p = a.min_p.of(row);
    if (min_p > 0.0f) {
        // the smallest logit that is close enough to the largest
        const double least = min_p < 1.0f ? (double)temperature * log((double)min_p) : 0.0;
        uint32_t key = key_of((float)(weights.largest + least));
        if (key > top) key = top;
        auto close = [&](uint32_t x) { return x == top || (double)logit_of(x) - weights.largest >= least; };
        while (key > kNothing && close(key - 1)) --key;
        while (!close(key)) ++key;
        const Border b{key - 1, 0};
        if (b < border) border = b;
    }
    // kept weights in order of ids: of each warp's run, of the blocks, of the row
    mass_t mass = 0;
    uint32_t ties = 0;
    slice.each([&](uint32_t key) {
        if (key > border.key) mass += weights.of(key);
        ties += key == border.key;
    });
    mass = warp_sum(mass);
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
    const mass_t each = border.ties ? weights.of(border.key) : 0;
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
    const float u = a.uniform[row];
    mass_t target = u > 0.0f ? u < 1.0f ? (mass_t)((double)u * (double)total) : total - 1 : 0;
    if (target >= total) target = total - 1;
    for (uint32_t w = 0; w < warp; ++w) {
        before += sh.warp_mass[w] + kept_ties(seen_before, sh.warp_count[w]) * each;
        seen_before += sh.warp_count[w];
    }
    const mass_t mine = sh.warp_mass[warp] + kept_ties(seen_before, sh.warp_count[warp]) * each;
    if (target < before || target >= before + mine) return;
    // the warp that has the token goes through its run
    for (uint32_t s = 0; s < steps; ++s) {
        const uint32_t at = slice.place(s);
        uint32_t key[E], here = 0;
        slice.keys(at, key);
#pragma unroll
        for (int e = 0; e < E; ++e) here += key[e] == border.key;
        uint32_t upto = here;
#pragma unroll
        for (int o = 1; o < 32; o *= 2) {
            const uint32_t c = __shfl_up_sync(0xFFFFFFFFu, upto, o);
            if (lane >= (uint32_t)o) upto += c;
        }
        uint32_t tie = seen_before + upto - here;
        mass_t m[E], sum = 0;
#pragma unroll
        for (int e = 0; e < E; ++e) {
            m[e] = key[e] > border.key ? weights.of(key[e]) : key[e] == border.key && tie < border.ties ? each : 0;
            tie += key[e] == border.key;
            sum += m[e];
        }
        mass_t running = sum;
#pragma unroll
        for (int o = 1; o < 32; o *= 2) {
            const mass_t c = __shfl_up_sync(0xFFFFFFFFu, running, o);
            if (lane >= (uint32_t)o) running += c;
        }
        mass_t from = before + running - sum;
        if (target >= from && target < from + sum) {
            int found = -1;
#pragma unroll
            for (int e = 0; e < E; ++e) {
                from += m[e];
                if (found < 0 && target < from) found = e;
            }
            a.token[row] = slice.begin + at + found;
            if (a.logprob) {
                const double gap = key[found] == top ? 0.0 : (double)logit_of(key[found]) - weights.largest;
                a.logprob[row] = (float)(gap / (double)temperature - log((double)total * exp2(-(double)a.bits)));
            }
        }
        before += __shfl_sync(0xFFFFFFFFu, running, 31);
        seen_before += __shfl_sync(0xFFFFFFFFu, upto, 31);
        if (target < before) return;
    }
}

constexpr uint32_t kStage = 160 * 1024;      // of shared memory for a slice, at most

}  // namespace

cudaError_t launch_sample(cudaStream_t stream, const SampleArgs& a, int sms) {
    return with_type(a.logits.type, [&](auto t) {
        using T = decltype(t);
        constexpr uint32_t E = Slice<T>::E, unit = kWarps * 32 * E;      // tokens of one access of a block
        // blocks enough for the device, and for a slice to fit
        uint32_t cluster = 1;
        while (cluster < kMostCluster && cluster * unit < a.V &&
               ((uint64_t)a.n * cluster < (uint64_t)sms * 2 || (uint64_t)a.V * sizeof(T) > (uint64_t)cluster * 56 * 1024)) cluster *= 2;
        const uint32_t steps = (uint32_t)(((uint64_t)a.V + (uint64_t)cluster * unit - 1) / ((uint64_t)cluster * unit));
        const uint64_t bytes = (uint64_t)steps * unit * sizeof(T);
        const bool staged = bytes <= kStage;
        const bool whole = (uintptr_t)a.logits.data % 16 == 0 && (a.n < 2 || a.logits.stride % E == 0);
        auto* kernel = k_sample<T>;
        cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kStage);
        if (e == cudaSuccess && cluster > 8) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
        if (e != cudaSuccess) return e;
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3(a.n * cluster);
        cfg.blockDim = dim3(kThreads);
        cfg.dynamicSmemBytes = staged ? bytes : 0;
        cfg.stream = stream;
        cudaLaunchAttribute attr[1];
        attr[0].id = cudaLaunchAttributeClusterDimension;
        attr[0].val.clusterDim = {cluster, 1, 1};
        cfg.attrs = attr;
        cfg.numAttrs = cluster > 1 ? 1 : 0;
        return cudaLaunchKernelEx(&cfg, kernel, a, cluster, steps, staged, whole);
    });
}

}  // namespace tensair
