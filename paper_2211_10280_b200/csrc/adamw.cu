// AdamW over many tensors in one launch.
//
// The tensors' descriptors travel as the kernel's argument block (up to 32 KB), so a step copies nothing to the device
// and keeps no plan: a block finds its tensor by a binary search in constant memory.  The update itself is one pass:
// every element of the parameter, the gradient and the moments is read once and written once.  It is bound by memory.
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
    uint32_t key0, key1, step_lo, step_hi;
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
    for (uint32_t chunk = blockIdx.x; chunk < b.chunks; chunk += gridDim.x) {
        const Entry& t = b.t[find_tensor(b, chunk)];
        const uint64_t at = (uint64_t)(chunk - t.chunk0) * b.chunk;
        if (t.head == kNoVector) {
            const uint64_t end = at + b.chunk < t.n ? at + b.chunk : t.n;
            for (uint64_t i = at + threadIdx.x; i < end; i += kThreads) update_one<TP, TG>(t, i, b.c, grad_scale);
            continue;
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
}

// ------------------------------------------------------------------ moments in 8 bits
constexpr int kLaneElems = kBlock / 32;  // 8

__device__ __forceinline__ void decode8(uint2 codes, float scale, float (&x)[kLaneElems]) {
#pragma unroll
    for (int h = 0; h < 4; ++h) {
        const uint16_t two = (uint16_t)((h < 2 ? codes.x : codes.y) >> (16 * (h & 1)));
        uint32_t halves;
        asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(halves) : "h"(two));
        const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&halves));
        x[2 * h] = f.x * scale;
        x[2 * h + 1] = f.y * scale;
    }
}

// |x| / scale to e4m3, the sign taken from x; bits16: 16 random bits in the low half.
// Values of e4m3's normal range are cut to 3 fraction bits after adding a uniform part of the last place.
__device__ __forceinline__ float round8(float x, float inv_scale, uint32_t bits16, bool keep_positive) {
    float size = fabsf(x) * inv_scale;
    if (keep_positive && x > 0.0f) size = fmaxf(size, 0x1p-9f);
    const float near = __uint_as_float((__float_as_uint(size) + (bits16 << 4) + 8u) & 0xFFF00000u);
    const float y = size < 0x1p-6f ? size : near;
    return __uint_as_float(__float_as_uint(y) | (__float_as_uint(x) & 0x80000000u));
}

__device__ __forceinline__ uint2 encode8(const float (&y)[kLaneElems]) {
    uint32_t two[4];
#pragma unroll
    for (int h = 0; h < 4; ++h) {
        uint16_t c;
        asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(c) : "f"(y[2 * h + 1]), "f"(y[2 * h]));
        two[h] = c;
    }
    return make_uint2(two[0] | two[1] << 16, two[2] | two[3] << 16);
}

// Stores one moment of a warp's block: the scale (lane 0) and this lane's codes.
__device__ __forceinline__ uint2 store8(const float (&x)[kLaneElems], const uint32_t (&words)[4], bool keep_positive, float* scale_out,
                                        uint32_t lane) {
    uint32_t top = 0;
#pragma unroll
    for (int e = 0; e < kLaneElems; ++e) top = max(top, __float_as_uint(x[e]) & 0x7FFFFFFFu);
    top = __reduce_max_sync(0xFFFFFFFFu, top);
    const bool finite = top < kInfBits;      // of the whole block
    if (!finite) {
        top = 0;
#pragma unroll
        for (int e = 0; e < kLaneElems; ++e) {
            const uint32_t bits = __float_as_uint(x[e]) & 0x7FFFFFFFu;
            if (bits < kInfBits) top = max(top, bits);
        }
        top = __reduce_max_sync(0xFFFFFFFFu, top);
    }
    const float largest = __uint_as_float(top);
    const bool any = largest >= kTiny;
    const float inv = any ? __fmul_rn(__frcp_rn(largest), kTop) : 0.0f;
    if (lane == 0) *scale_out = any ? __fmul_rn(largest, 1.0f / kTop) : 0.0f;
    float y[kLaneElems];
#pragma unroll
    for (int e = 0; e < kLaneElems; ++e)
        y[e] = round8(x[e], inv, e & 1 ? words[e >> 1] >> 16 : words[e >> 1] & 0xFFFFu, keep_positive);
    if (!finite) {
#pragma unroll
        for (int e = 0; e < kLaneElems; ++e)
            if ((__float_as_uint(x[e]) & 0x7FFFFFFFu) >= kInfBits) y[e] = __uint_as_float(0x7FC00000u);
    }
    return encode8(y);
}

template <int kCount, typename TP, typename TG>
__global__ void __launch_bounds__(kThreads)
k_adamw8(const __grid_constant__ Batch<kCount> b) {
    float grad_scale;
    if (!adamw_grad_scale(b.c, &grad_scale)) return;
    const uint32_t lane = threadIdx.x & 31, wid = threadIdx.x >> 5;
    for (uint32_t chunk = blockIdx.x; chunk < b.chunks; chunk += gridDim.x) {
        const Entry& t = b.t[find_tensor(b, chunk)];
        const uint64_t at = (uint64_t)(chunk - t.chunk0) * b.chunk;
        const uint64_t end = at + b.chunk < t.n ? at + b.chunk : t.n;
        for (uint64_t base = at + wid * kBlock; base < end; base += kThreads / 32 * kBlock) {
            const uint64_t i = base + lane * kLaneElems, block = base / kBlock;
            const bool vector = t.head != kNoVector && i + kLaneElems <= t.n;
            float p[kLaneElems], g[kLaneElems], m[kLaneElems], v[kLaneElems];
            const float m_scale = t.m_scale[block], v_scale = t.v_scale[block];
            uint2 mc = make_uint2(0, 0), vc = make_uint2(0, 0);
            if (vector) {
                const Pack<TP, kLaneElems> pp = load_pack<TP, kLaneElems>((TP*)t.p + i);
                const Pack<TG, kLaneElems> gg = load_pack<TG, kLaneElems>((const TG*)t.g + i);
                mc = *reinterpret_cast<const uint2*>((uint8_t*)t.m + i);
                vc = *reinterpret_cast<const uint2*>((uint8_t*)t.v + i);
#pragma unroll
                for (int e = 0; e < kLaneElems; ++e) {
                    p[e] = to_float(pp.v[e]);
                    g[e] = to_float(gg.v[e]) * grad_scale;
                }
            } else {
#pragma unroll
                for (int e = 0; e < kLaneElems; ++e) {
                    const bool in = i + e < t.n;
                    p[e] = in ? to_float(((TP*)t.p)[i + e]) : 0.0f;
                    g[e] = in ? to_float(((const TG*)t.g)[i + e]) * grad_scale : 0.0f;
                    const uint32_t cm = in ? ((uint8_t*)t.m)[i + e] : 0u, cv = in ? ((uint8_t*)t.v)[i + e] : 0u;
                    if (e < 4) { mc.x |= cm << (8 * e); vc.x |= cv << (8 * e); }
                    else { mc.y |= cm << (8 * (e - 4)); vc.y |= cv << (8 * (e - 4)); }
                }
            }
            decode8(mc, m_scale, m);
            decode8(vc, v_scale, v);
#pragma unroll
            for (int e = 0; e < kLaneElems; ++e) {
                // every product and sum rounded by itself, as a program of separate operations has them: what is
                // stored then does not depend on which of them a compiler contracts
                m[e] = __fadd_rn(__fmul_rn(m[e], b.c.beta1), __fmul_rn(g[e], b.c.rest1));
                v[e] = __fadd_rn(__fmul_rn(__fmul_rn(v[e], v[e]), b.c.beta2), __fmul_rn(__fmul_rn(g[e], g[e]), b.c.rest2));
                v[e] = __fsqrt_rn(v[e]);     // from here on the square root
                p[e] = fmaf(p[e], t.keep, -t.step_size * (m[e] / fmaf(v[e], b.c.inv_root2, b.c.eps)));
            }
            const uint64_t group = (t.block0 + block) * 32 + lane;
            const Philox4 r = philox4x32_10(Philox4{(uint32_t)group, (uint32_t)(group >> 32), b.step_lo, kTagRounding | b.step_hi},
                                            b.key0, b.key1);
            const uint32_t words[4] = {r.x, r.y, r.z, r.w};
            mc = store8(m, words, false, t.m_scale + block, lane);
            vc = store8(v, words, true, t.v_scale + block, lane);
            if (vector) {
                store_pack<TP, kLaneElems>((TP*)t.p + i, p);
                *reinterpret_cast<uint2*>((uint8_t*)t.m + i) = mc;
                *reinterpret_cast<uint2*>((uint8_t*)t.v + i) = vc;
                if (t.copy) store_copies<kLaneElems>(t, i, p);
            } else {
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
    }
}

// ------------------------------------------------------------------ host
// Elements to leave out so that every array of the tensor is aligned for vectors of `vec` elements (or 16 bytes).
uint32_t aligned_head(const AdamwTensor& t, int bits, uint32_t vec) {
    auto aligned = [vec](const void* p, uint64_t elem, uint32_t h) {
        const uint64_t bytes = elem * vec > 16 ? 16 : elem * vec;
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
    const uint32_t grid = b.chunks < (uint32_t)sms * 16 ? b.chunks : (uint32_t)sms * 16;
    if (bits == 8) k_adamw8<kCount, TP, TG><<<grid, kThreads, 0, stream>>>(b);
    else k_adamw<kCount, TP, TG><<<grid, kThreads, 0, stream>>>(b);
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
            b.chunk = total >= (uint64_t)sms * 8 * 4096 ? 4096 : 2048;
            for (uint32_t next = 0; next < count;) {
                const cudaError_t e = launch_some<kCount>(stream, tensors, count, &next, pt, gt, bits, b, sms);
                if (e != cudaSuccess) return e;
            }
        }
    return cudaSuccess;
}

constexpr int kFew = 16, kMany = 340;

}  // namespace

cudaError_t launch_adamw(cudaStream_t stream, const AdamwTensor* tensors, uint32_t count, int bits, const AdamwConsts& c,
                         uint64_t step, uint64_t seed, int sms) {
    static_assert(sizeof(Batch<kMany>) <= 32764, "a kernel's arguments hold at most 32,764 bytes");
    auto set = [&](auto& b) {
        b.c = c;
        b.key0 = (uint32_t)seed;
        b.key1 = (uint32_t)(seed >> 32);
        b.step_lo = (uint32_t)step;
        b.step_hi = (uint32_t)(step >> 32) & 0xFFFFFFu;
    };
    if (count <= kFew) {
        Batch<kFew> b;
        set(b);
        return launch_all<kFew>(stream, tensors, count, bits, b, sms);
    }
    Batch<kMany> b;
    set(b);
    return launch_all<kMany>(stream, tensors, count, bits, b, sms);
}

}  // namespace tensair
