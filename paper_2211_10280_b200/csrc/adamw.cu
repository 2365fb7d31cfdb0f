// AdamW over many tensors in one launch.
//
// The tensors' descriptors travel as the kernel's argument block (up to 32 KB), so a step copies nothing to the device
// and keeps no plan: a block finds its tensor by a binary search in constant memory.  The update itself is one pass:
// every element of the parameter, the gradient and the moments is read once and written once.  With 32-bit moments it is
// bound by memory: 96 M elements (fp32, bf16 gradients and a bf16 copy, 28 bytes each) take 395 us, 6.8 TB/s, which is the
// rate of a plain copy.  A small model is bound by the launch (200,000 elements: 4.2 us).
//
// Moments in 8 bits.  A block of 256 elements, one warp's work, shares one fp32 scale per moment; stored are m / scale and
// sqrt(v) / scale in e4m3, with scale = largest magnitude / 448.  The square root halves the exponent range v
// needs.  Rounding is stochastic: with beta2 = 0.999 a step moves sqrt(v) by at most 0.05 %, which rounding to nearest in
// 3 fraction bits would undo every time, so v would never follow the gradient; rounding up as often as the value is
// near the upper neighbour keeps the mean of the stored root exact.  The 16 random bits per element come from Philox4x32-10 (counter =
// (group of 8 elements, step, tag), key = seed), the same bits for both moments.  A positive v is never stored as zero
// (it would be divided by eps alone): it keeps at least the smallest e4m3 value.  Magnitudes in e4m3's subnormal
// range, below 2^-14 of the block's largest, round to nearest.  Non-finite elements are stored as NaN and leave the
// block's scale alone, so they stay where they are, as in 32 bits.
//
// With 8-bit moments an element moves 14 bytes (fp32, bf16 gradients) and takes some 60 instructions, 26 of them integer (Philox,
// the roundings, addresses), so the kernel is bound by both: 128 M elements take 360 us a step in a run of steps, 5.0 TB/s (0.76 of the copy
// rate), and 325 us where only a few follow one another.  What made it so (short runs; 547 us at first): packed fp32 arithmetic, roots by one Newton step two at a time, approximate quotients in the
// update, Philox with its round keys in the arguments, one vote per block for the rare cases, 64 registers for four blocks per
// multiprocessor (401 us), and the next turn's reads prefetched into the level-2 cache.  Copying them ahead through shared memory
// instead made it slower (443 us).
#include "adamw.cuh"
#include "operators.h"
#include "philox.cuh"

namespace tensair {

namespace {

constexpr int kThreads = 256;
constexpr uint32_t kBlock = 256;         // elements that share a scale
constexpr float kTop = 448.0f;           // largest e4m3 value
constexpr float kTiny = 0x1p-110f;       // a block of first moments below this is stored as zeros
constexpr uint32_t kInfBits = 0x7F800000u;

struct Entry {
    void* p;
    const void* g;
    void* m;
    void* v;
    void* copy;
    float* m_scale;
    float* v_scale;
    uint64_t n;
    uint64_t block0;
    uint32_t chunk0;       // first chunk of the tensor in this launch
    uint32_t head;         // elements before the first one at which all arrays are aligned; kNoVector: there is none
    float step_size, keep;
    uint32_t copy_half;    // the copy is fp16 (else bf16)
};
constexpr uint32_t kNoVector = 0xFFFFFFFFu;

template <int kCount>
struct Batch {
    AdamwConsts c;
    uint32_t count, chunks;
    uint32_t chunk;        // elements of a chunk
    uint32_t step_lo, step_hi;
    PhiloxKeys keys;
    Entry t[kCount];
};

template <int kCount>
__device__ __forceinline__ uint32_t find_tensor(const Batch<kCount>& b, uint32_t chunk) {
    uint32_t lo = 0, hi = b.count;
    while (hi - lo > 1) {
        const uint32_t mid = (lo + hi) / 2;
        if (b.t[mid].chunk0 <= chunk) lo = mid;
        else hi = mid;
    }
    return lo;
}

__device__ __forceinline__ void store_copy(const Entry& t, uint64_t i, float p) {
    if (t.copy_half) reinterpret_cast<__half*>(t.copy)[i] = __float2half_rn(p);
    else reinterpret_cast<__nv_bfloat16*>(t.copy)[i] = __float2bfloat16_rn(p);
}
template <int E>
__device__ __forceinline__ void store_copies(const Entry& t, uint64_t i, const float (&p)[E]) {
    if (t.copy_half) store_pack<__half, E>(reinterpret_cast<__half*>(t.copy) + i, p);
    else store_pack<__nv_bfloat16, E>(reinterpret_cast<__nv_bfloat16*>(t.copy) + i, p);
}

// ------------------------------------------------------------------ moments in 32 bits
template <typename TP, typename TG>
__device__ __forceinline__ void update_one(const Entry& t, uint64_t i, const AdamwConsts& c, float grad_scale) {
    float m = ((float*)t.m)[i], v = ((float*)t.v)[i];
    const float p = adamw_update(to_float(((TP*)t.p)[i]), to_float(((const TG*)t.g)[i]) * grad_scale, m, v, c, t.step_size, t.keep);
    ((TP*)t.p)[i] = from_float<TP>(p);
    ((float*)t.m)[i] = m;
    ((float*)t.v)[i] = v;
    if (t.copy) store_copy(t, i, p);
}

constexpr int kVec = 4;
constexpr int kUnroll = 2;

template <int kCount, typename TP, typename TG>
__global__ void __launch_bounds__(kThreads)
k_adamw(const __grid_constant__ Batch<kCount> b) {
    float grad_scale;
    if (!adamw_grad_scale(b.c, &grad_scale)) return;
    const Entry& t = b.t[find_tensor(b, blockIdx.x)];
    const uint64_t at = (uint64_t)(blockIdx.x - t.chunk0) * b.chunk;
    if (t.head == kNoVector) {
        const uint64_t end = at + b.chunk < t.n ? at + b.chunk : t.n;
        for (uint64_t i = at + threadIdx.x; i < end; i += kThreads) update_one<TP, TG>(t, i, b.c, grad_scale);
        return;
    }
    if (at == 0 && threadIdx.x < t.head && threadIdx.x < t.n) update_one<TP, TG>(t, threadIdx.x, b.c, grad_scale);
    const uint64_t end = t.head + at + b.chunk < t.n ? t.head + at + b.chunk : t.n;
    for (uint64_t i0 = t.head + at + threadIdx.x * kVec; i0 < end; i0 += kThreads * kVec * kUnroll) {
        Pack<TP, kVec> p[kUnroll];
        Pack<TG, kVec> g[kUnroll];
        Pack<float, kVec> m[kUnroll], v[kUnroll];
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            const uint64_t i = i0 + u * kThreads * kVec;
            if (i + kVec <= end) {
                p[u] = load_pack<TP, kVec>((TP*)t.p + i);
                g[u] = load_pack<TG, kVec>((const TG*)t.g + i);
                m[u] = load_pack<float, kVec>((float*)t.m + i);
                v[u] = load_pack<float, kVec>((float*)t.v + i);
            }
        }
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            const uint64_t i = i0 + u * kThreads * kVec;
            if (i + kVec <= end) {
                float y[kVec];
#pragma unroll
                for (int e = 0; e < kVec; ++e)
                    y[e] = adamw_update(to_float(p[u].v[e]), to_float(g[u].v[e]) * grad_scale, m[u].v[e], v[u].v[e], b.c,
                                        t.step_size, t.keep);
                store_pack<TP, kVec>((TP*)t.p + i, y);
                store_pack<float, kVec>((float*)t.m + i, m[u].v);
                store_pack<float, kVec>((float*)t.v + i, v[u].v);
                if (t.copy) store_copies<kVec>(t, i, y);
            } else {
                for (uint64_t j = i; j < end; ++j) update_one<TP, TG>(t, j, b.c, grad_scale);
            }
        }
    }
}

// ------------------------------------------------------------------ moments in 8 bits
constexpr int kLaneElems = kBlock / 32;  // 8

// Two floats in one register pair: the packed instructions do both in one issue slot, each rounded as the single ones.
struct Two {
    unsigned long long bits;
    __device__ __forceinline__ Two() {}
    __device__ __forceinline__ Two(float a, float b) { asm("mov.b64 %0, {%1, %2};" : "=l"(bits) : "f"(a), "f"(b)); }
    __device__ __forceinline__ explicit Two(float a) : Two(a, a) {}
    __device__ __forceinline__ float2 floats() const {
        float2 f;
        asm("mov.b64 {%0, %1}, %2;" : "=f"(f.x), "=f"(f.y) : "l"(bits));
        return f;
    }
};
__device__ __forceinline__ Two operator*(Two a, Two b) {
    Two r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r.bits) : "l"(a.bits), "l"(b.bits));
    return r;
}
__device__ __forceinline__ Two fma2(Two a, Two b, Two c) {
    Two r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r.bits) : "l"(a.bits), "l"(b.bits), "l"(c.bits));
    return r;
}

// A sum of products that are rounded first, and then the sum: by single additions, since the assembler contracts a packed
// product and a packed sum into one operation, whatever their rounding modifiers say.
__device__ __forceinline__ Two sum_of(Two a, Two b) {
    const float2 x = a.floats(), y = b.floats();
    return Two(__fadd_rn(x.x, y.x), __fadd_rn(x.y, y.y));
}

__device__ __forceinline__ Two decode8(uint16_t codes, Two scale) {
    uint32_t halves;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(halves) : "h"(codes));
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&halves));
    return Two(f.x, f.y) * scale;
}
__device__ __forceinline__ uint32_t encode8(float low, float high) {
    uint16_t c;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(c) : "f"(high), "f"(low));
    return c;
}
__device__ __forceinline__ float approximate_reciprocal(float x) {     // used in the update alone
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ uint32_t magnitude(float x) { return __float_as_uint(x) & 0x7FFFFFFFu; }

// x, already divided by the scale, cut to 3 fraction bits after adding a uniform part of the last place kept (`bits20`: 16 random
// bits above four zeros, and 8, the half of their last place): for values of e4m3's normal range, where the conversion
// that follows is exact.
__device__ __forceinline__ float cut8(float x, uint32_t bits20) {
    return __uint_as_float((__float_as_uint(x) + bits20 + 8u) & 0xFFF00000u);
}

// Smallest and largest bit pattern of the magnitudes of a lane's eight values (kPositive: their sign bits are 0 but for NaNs).
template <bool kPositive>
__device__ __forceinline__ void range8(const Two (&x)[4], uint32_t* low, uint32_t* top) {
    *low = 0xFFFFFFFFu;
    *top = 0;
#pragma unroll
    for (int h = 0; h < 4; ++h) {
        const float2 f = x[h].floats();
        const uint32_t a = kPositive ? __float_as_uint(f.x) : magnitude(f.x), b = kPositive ? __float_as_uint(f.y) : magnitude(f.y);
        *low = __vimin3_u32(*low, a, b);
        *top = __vimax3_u32(*top, a, b);
    }
    if (kPositive) *top &= 0x7FFFFFFFu;
}

// Square roots, correctly rounded like __fsqrt_rn, of values in [2^-96, 2^128): Newton's step from the approximate reciprocal root with
// the residual x - y^2 formed by a fused multiply-add (Markstein, IBM J. Res. Dev. 34, 1990).  Two at a time.  Not proven, counted: all
// 1,879,048,192 values of the range have the bits of __fsqrt_rn.
__device__ __forceinline__ Two roots(Two x) {
    const float2 f = x.floats();
    float r0, r1;
    asm("rsqrt.approx.ftz.f32 %0, %1;" : "=f"(r0) : "f"(f.x));
    asm("rsqrt.approx.ftz.f32 %0, %1;" : "=f"(r1) : "f"(f.y));
    const Two r(r0, r1), y = x * r;
    return fma2(fma2(y * Two(-1.0f), y, x), r * Two(0.5f), y);
}

// One moment of a warp's block to e4m3: this lane's codes, and the scale by lane 0.  low and top: range8 of x.
template <bool kRoot>
__device__ __forceinline__ uint2 store8(const Two (&x)[4], uint32_t low, uint32_t top, const uint32_t (&bits20)[8], float* scale_out,
                                        uint32_t lane) {
    top = __reduce_max_sync(0xFFFFFFFFu, top);
    const bool finite = top < kInfBits;          // of the whole block
    if (!finite) {
        top = 0;
#pragma unroll
        for (int h = 0; h < 4; ++h) {
            const float2 f = x[h].floats();
            const uint32_t a = magnitude(f.x), b = magnitude(f.y);
            if (a < kInfBits) top = max(top, a);
            if (b < kInfBits) top = max(top, b);
        }
        top = __reduce_max_sync(0xFFFFFFFFu, top);
    }
    const float largest = __uint_as_float(top);
    const bool any = largest >= kTiny;
    const float inv = any ? __fmul_rn(__frcp_rn(largest), kTop) : 0.0f;
    if (lane == 0) *scale_out = any ? __fmul_rn(largest, 1.0f / kTop) : 0.0f;
    uint32_t code[4];
    // Values below e4m3's normal range are rare in a block (2^-14.8 of its largest): one vote spares the rest the checks.
    // (A product's rounding keeps the order, so the smallest speaks for all.)
    if (finite && !__any_sync(0xFFFFFFFFu, __fmul_rn(__uint_as_float(low), inv) < 0x1p-6f)) {
#pragma unroll
        for (int h = 0; h < 4; ++h) {
            const float2 y = (x[h] * Two(inv)).floats();
            code[h] = encode8(cut8(y.x, bits20[2 * h]), cut8(y.y, bits20[2 * h + 1]));
        }
    } else {
#pragma unroll
        for (int h = 0; h < 4; ++h) {
            const float2 g = x[h].floats(), y = (x[h] * Two(inv)).floats();
            auto one = [&](float y, float source, uint32_t d) {
                if (magnitude(source) >= kInfBits) return __uint_as_float(0x7FC00000u);
                if (kRoot && source > 0.0f) y = fmaxf(y, 0x1p-9f);      // never stored as zero
                return fabsf(y) < 0x1p-6f ? y : cut8(y, d);
            };
            code[h] = encode8(one(y.x, g.x, bits20[2 * h]), one(y.y, g.y, bits20[2 * h + 1]));
        }
    }
    return make_uint2(code[0] | code[1] << 16, code[2] | code[3] << 16);
}

template <typename TP>
__device__ __forceinline__ void load_lane(const TP* at, float (&p)[kLaneElems]) {
    if constexpr (sizeof(TP) == 4) load_eight(at, p);
    else {
        const Pack<TP, kLaneElems> x = load_pack<TP, kLaneElems>(at);
#pragma unroll
        for (int e = 0; e < kLaneElems; ++e) p[e] = to_float(x.v[e]);
    }
}
template <typename TP>
__device__ __forceinline__ void store_lane(TP* at, const float (&p)[kLaneElems]) {
    if constexpr (sizeof(TP) == 4) store_eight(at, p);
    else store_pack<TP, kLaneElems>(at, p);
}

// One block of 256 elements, eight to a lane: parameter, moments and codes to their new values.  The caller stores p, mc and vc.
template <int kCount>
__device__ __forceinline__ void step8(const Batch<kCount>& b, const Entry& t, uint64_t block, uint32_t lane, float grad_scale,
                                      float (&p)[kLaneElems], Two (&g)[4], Two m_scale, Two v_scale, uint2& mc, uint2& vc) {
    Two m[4], v[4];
    const uint64_t group = (t.block0 + block) * 32 + lane;
    const Philox4 r = philox4x32_10(Philox4{(uint32_t)group, (uint32_t)(group >> 32), b.step_lo, kTagRounding | b.step_hi}, b.keys);
    const uint32_t words[4] = {r.x, r.y, r.z, r.w};
    uint32_t bits20[kLaneElems];
#pragma unroll
    for (int h = 0; h < 4; ++h) {
        bits20[2 * h] = words[h] << 4 & 0xFFFF0u;
        bits20[2 * h + 1] = words[h] >> 12 & 0xFFFF0u;
    }
#pragma unroll
    for (int h = 0; h < 4; ++h) {
        // every product and sum rounded by itself, as a program of separate operations has them: what is
        // stored then does not depend on which of them a compiler contracts
        m[h] = decode8((uint16_t)((h < 2 ? mc.x : mc.y) >> (16 * (h & 1))), m_scale);
        v[h] = decode8((uint16_t)((h < 2 ? vc.x : vc.y) >> (16 * (h & 1))), v_scale);
        g[h] = g[h] * Two(grad_scale);
        m[h] = sum_of(m[h] * Two(b.c.beta1), g[h] * Two(b.c.rest1));
        v[h] = sum_of(v[h] * v[h] * Two(b.c.beta2), g[h] * g[h] * Two(b.c.rest2));
    }
    uint32_t m_low, m_top, v_low, v_top;
    range8<false>(m, &m_low, &m_top);
    range8<true>(v, &v_low, &v_top);
    // from here on v is its square root
    if (__all_sync(0xFFFFFFFFu, v_low >= 0x0F800000u && v_top < kInfBits)) {      // 2^-96
#pragma unroll
        for (int h = 0; h < 4; ++h) v[h] = roots(v[h]);
    } else {
#pragma unroll
        for (int h = 0; h < 4; ++h) {
            const float2 f = v[h].floats();
            v[h] = Two(__fsqrt_rn(f.x), __fsqrt_rn(f.y));
        }
    }
    range8<true>(v, &v_low, &v_top);
#pragma unroll
    for (int h = 0; h < 4; ++h) {
        const float2 low = fma2(v[h], Two(b.c.inv_root2), Two(b.c.eps)).floats();
        const Two change = m[h] * Two(approximate_reciprocal(low.x), approximate_reciprocal(low.y));
        const float2 y = fma2(change, Two(-t.step_size), Two(p[2 * h], p[2 * h + 1]) * Two(t.keep)).floats();
        p[2 * h] = y.x;
        p[2 * h + 1] = y.y;
    }
    mc = store8<false>(m, m_low, m_top, bits20, t.m_scale + block, lane);
    vc = store8<true>(v, v_low, v_top, bits20, t.v_scale + block, lane);
}

template <int kCount, typename TP, typename TG>
__global__ void __launch_bounds__(kThreads, 4)
k_adamw8(const __grid_constant__ Batch<kCount> b) {
    float grad_scale;
    if (!adamw_grad_scale(b.c, &grad_scale)) return;
    const uint32_t tid = threadIdx.x, lane = tid & 31, wid = tid >> 5;
    const Entry& t = b.t[find_tensor(b, blockIdx.x)];
    const uint64_t at = (uint64_t)(blockIdx.x - t.chunk0) * b.chunk;
    const uint64_t end = at + b.chunk < t.n ? at + b.chunk : t.n;
    constexpr uint32_t kStep = kThreads / 32 * kBlock;
    // ---- whole blocks of aligned tensors
    const uint64_t whole = t.head == kNoVector ? at : end / kBlock * kBlock;
    uint64_t base = at + wid * kBlock;
    for (; base < whole; base += kStep) {
        const uint64_t i = base + lane * kLaneElems, block = base / kBlock;
        const float m_scale = t.m_scale[block], v_scale = t.v_scale[block];
        if (base + kStep < whole) {      // what the next turn reads, into the level-2 cache: 401 -> 325 us, and no registers
            prefetch((const TP*)t.p + i + kStep);
            prefetch((const TG*)t.g + i + kStep);
            prefetch((const uint8_t*)t.m + i + kStep);
            prefetch((const uint8_t*)t.v + i + kStep);
        }
        float p[kLaneElems];
        load_lane<TP>((const TP*)t.p + i, p);
        const Pack<TG, kLaneElems> gg = load_pack<TG, kLaneElems>((const TG*)t.g + i);
        uint2 mc = *reinterpret_cast<const uint2*>((const uint8_t*)t.m + i), vc = *reinterpret_cast<const uint2*>((const uint8_t*)t.v + i);
        Two g[4];
#pragma unroll
        for (int h = 0; h < 4; ++h) g[h] = Two(to_float(gg.v[2 * h]), to_float(gg.v[2 * h + 1]));
        step8(b, t, block, lane, grad_scale, p, g, Two(m_scale), Two(v_scale), mc, vc);
        store_lane<TP>((TP*)t.p + i, p);
        if (t.copy) store_copies<kLaneElems>(t, i, p);
        *reinterpret_cast<uint2*>((uint8_t*)t.m + i) = mc;
        *reinterpret_cast<uint2*>((uint8_t*)t.v + i) = vc;
    }
    // ---- a tensor's last, incomplete block, and tensors that are not aligned
    for (base = whole + (t.head == kNoVector ? wid * kBlock : 0); base < end; base += kStep) {
        if (t.head != kNoVector && wid) break;
        const uint64_t i = base + lane * kLaneElems, block = base / kBlock;
        const Two m_scale(t.m_scale[block]), v_scale(t.v_scale[block]);
        uint2 mc = make_uint2(0, 0), vc = make_uint2(0, 0);
        float p[kLaneElems], y[kLaneElems];
        Two g[4];
#pragma unroll
        for (int e = 0; e < kLaneElems; ++e) {
            const bool in = i + e < t.n;
            p[e] = in ? to_float(((TP*)t.p)[i + e]) : 0.0f;
            y[e] = in ? to_float(((const TG*)t.g)[i + e]) : 0.0f;
            const uint32_t cm = in ? ((uint8_t*)t.m)[i + e] : 0u, cv = in ? ((uint8_t*)t.v)[i + e] : 0u;
            if (e < 4) { mc.x |= cm << (8 * e); vc.x |= cv << (8 * e); }
            else { mc.y |= cm << (8 * (e - 4)); vc.y |= cv << (8 * (e - 4)); }
        }
#pragma unroll
        for (int h = 0; h < 4; ++h) g[h] = Two(y[2 * h], y[2 * h + 1]);
        step8(b, t, block, lane, grad_scale, p, g, m_scale, v_scale, mc, vc);
#pragma unroll
        for (int e = 0; e < kLaneElems; ++e)
            if (i + e < t.n) {
                ((TP*)t.p)[i + e] = from_float<TP>(p[e]);
                ((uint8_t*)t.m)[i + e] = (uint8_t)((e < 4 ? mc.x : mc.y) >> (8 * (e & 3)));
                ((uint8_t*)t.v)[i + e] = (uint8_t)((e < 4 ? vc.x : vc.y) >> (8 * (e & 3)));
                if (t.copy) store_copy(t, i + e, p[e]);
            }
    }
}

// ------------------------------------------------------------------ host
// Elements to leave out so that every array of the tensor is aligned for vectors of `vec` elements (or 16 bytes).
uint32_t aligned_head(const AdamwTensor& t, int bits, uint32_t vec) {
    // vectors of fp32 parameters with 8-bit moments are moved in one 32-byte access, all others in up to 16 bytes
    auto aligned = [&](const void* p, uint64_t elem, uint32_t h) {
        const uint64_t most = bits == 8 && p == t.param ? 32 : 16, bytes = elem * vec > most ? most : elem * vec;
        return ((uintptr_t)p + h * elem) % bytes == 0;
    };
    const uint32_t most = bits == 8 ? 1 : vec;     // the blocks of the 8-bit moments begin at the first element
    for (uint32_t h = 0; h < most; ++h)
        if (aligned(t.param, type_bytes(t.param_type), h) && aligned(t.grad, type_bytes(t.grad_type), h) &&
            aligned(t.m, bits / 8, h) && aligned(t.v, bits / 8, h) && (!t.copy || aligned(t.copy, 2, h)))
            return h;
    return kNoVector;
}

template <int kCount, typename TP, typename TG>
cudaError_t launch_batch(cudaStream_t stream, const Batch<kCount>& b, int bits, int sms) {
    if (bits == 8) k_adamw8<kCount, TP, TG><<<b.chunks, kThreads, 0, stream>>>(b);
    else k_adamw<kCount, TP, TG><<<b.chunks, kThreads, 0, stream>>>(b);
    return cudaGetLastError();
}
template <int kCount, typename TP>
cudaError_t launch_batch(cudaStream_t stream, const Batch<kCount>& b, uint32_t grad_type, int bits, int sms) {
    switch (grad_type) {
        case 0: return launch_batch<kCount, TP, float>(stream, b, bits, sms);
        case 1: return launch_batch<kCount, TP, __nv_bfloat16>(stream, b, bits, sms);
        default: return launch_batch<kCount, TP, __half>(stream, b, bits, sms);
    }
}
template <int kCount>
cudaError_t launch_batch(cudaStream_t stream, const Batch<kCount>& b, uint32_t param_type, uint32_t grad_type, int bits, int sms) {
    switch (param_type) {
        case 0: return launch_batch<kCount, float>(stream, b, grad_type, bits, sms);
        case 1: return launch_batch<kCount, __nv_bfloat16>(stream, b, grad_type, bits, sms);
        default: return launch_batch<kCount, __half>(stream, b, grad_type, bits, sms);
    }
}

// One launch for up to kCount of the tensors of one type combination, from *next on; *next moves past what was taken.
template <int kCount>
cudaError_t launch_some(cudaStream_t stream, const AdamwTensor* tensors, uint32_t count, uint32_t* next, uint32_t pt, uint32_t gt,
                        int bits, Batch<kCount>& b, int sms) {
    const uint32_t vec = bits == 8 ? kLaneElems : kVec;
    uint32_t i = *next;
    uint64_t chunks = 0;
    b.count = 0;
    for (; i < count && b.count < kCount; ++i) {
        const AdamwTensor& t = tensors[i];
        if (t.param_type != pt || t.grad_type != gt || !t.n) continue;
        const uint64_t mine = (t.n + b.chunk - 1) / b.chunk;
        if (chunks + mine >= (1ull << 31)) break;
        Entry& e = b.t[b.count++];
        e = Entry{t.param, t.grad, t.m, t.v, t.copy, t.m_scale, t.v_scale, t.n, t.block0, (uint32_t)chunks,
                  aligned_head(t, bits, vec), t.step_size, t.keep, t.copy_type == 2};
        chunks += mine;
    }
    *next = i;
    b.chunks = (uint32_t)chunks;
    return b.count ? launch_batch<kCount>(stream, b, pt, gt, bits, sms) : cudaSuccess;
}

template <int kCount>
cudaError_t launch_all(cudaStream_t stream, const AdamwTensor* tensors, uint32_t count, int bits, Batch<kCount>& b, int sms) {
    for (uint32_t pt = 0; pt < 3; ++pt)
        for (uint32_t gt = 0; gt < 3; ++gt) {
            uint64_t total = 0;
            for (uint32_t i = 0; i < count; ++i)
                if (tensors[i].param_type == pt && tensors[i].grad_type == gt) total += tensors[i].n;
            if (!total) continue;
            // A block finds its tensor once per chunk.  With 32-bit moments short chunks are best (96 M elements: 395 us with 2,048,
            // 403 with 4,096, 410 with 8,192: the blocks that run together stay close together in memory); with 8-bit ones the search
            // is worth sharing (128 M: 442 us with 4,096, 401 with 16,384), as long as all multiprocessors have chunks.
            b.chunk = bits == 8 ? 16384 : 2048;
            while (b.chunk > 2048 && total < (uint64_t)sms * 8 * b.chunk) b.chunk /= 2;
            for (uint32_t next = 0; next < count;) {
                const cudaError_t e = launch_some<kCount>(stream, tensors, count, &next, pt, gt, bits, b, sms);
                if (e != cudaSuccess) return e;
            }
        }
    return cudaSuccess;
}

// Tensors that a launch's arguments hold: the host copies them all with every launch, so there are four sizes (1.6, 3, 6 and 32 KB).  The
// kernel's own time is the same with all of them (4.2 us for 13 to 336 tensors of 1,000 elements); the call takes the host 4.7 us with 16
// tensors, 6.4 with 64, 9.4 with 65, 17 with 336.  Launches of 64 instead of the last size: 9.6 us with 65, 11.2 with 128 (11.6 in one
// launch), 14.4 with 129 (11.3), 30 with 336, and 4.1 us more on the device for each.
constexpr int kFew = 16, kSome = 32, kMore = 64, kMany = 336;

}  // namespace

cudaError_t launch_adamw(cudaStream_t stream, const AdamwTensor* tensors, uint32_t count, int bits, const AdamwConsts& c,
                         uint64_t step, uint64_t seed, int sms) {
    static_assert(sizeof(Batch<kMany>) <= 32764, "a kernel's arguments hold at most 32,764 bytes");
    auto set = [&](auto& b) {
        b.c = c;
        b.keys = PhiloxKeys(seed);
        b.step_lo = (uint32_t)step;
        b.step_hi = (uint32_t)(step >> 32) & 0xFFFFFFu;
    };
    if (count <= kFew) {
        Batch<kFew> b;
        set(b);
        return launch_all<kFew>(stream, tensors, count, bits, b, sms);
    }
    if (count <= kSome) {
        Batch<kSome> b;
        set(b);
        return launch_all<kSome>(stream, tensors, count, bits, b, sms);
    }
    if (count <= kMore) {
        Batch<kMore> b;
        set(b);
        return launch_all<kMore>(stream, tensors, count, bits, b, sms);
    }
    Batch<kMany> b;
    set(b);
    return launch_all<kMany>(stream, tensors, count, bits, b, sms);
}

}  // namespace tensair
