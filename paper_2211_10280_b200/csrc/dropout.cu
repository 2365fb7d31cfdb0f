// Dropout whose mask is never stored: element e is kept where word e % 4 of Philox4x32-10 of counter (e / 4, call) reaches
// p 2^32, so the backward pass draws the same mask again.  y = kept ? x / (1 - p) : 0, plus a residual if there is one.
//
// Bound by the generator beside memory: ten rounds with two wide products each for four elements, 30 instructions an element in all (0.63 of
// the issue slots).  33.5 M bf16 elements with a residual 48 us, 4.2 TB/s; 16.8 M fp32 without 27 us, 5.0 TB/s.
#include "columns.cuh"
#include "layers.h"
#include "philox.cuh"

namespace tensair {

namespace {

constexpr int kThreads = 256;

// A thread takes one vector, or two of 32-bit elements, a block's width apart, whose words are drawn while both are on their way.  (bf16 with a
// residual, 33.5 M elements: one vector 49 us, two 60 us, for want of threads; fp32 without, 16.8 M: 31 and 27 us.)
template <typename T>
constexpr int kVectors = sizeof(T) == 4 ? 2 : 1;
template <typename T, typename C, bool kResidual>
__global__ void __launch_bounds__(kThreads, sizeof(T) == 4 ? 5 : 7)
k_dropout(const __grid_constant__ DropoutArgs a, const __grid_constant__ PhiloxKeys keys) {
    constexpr int E = C::E;
    using Piece = Columns<E, true>;      // the last vector, or one of a tensor that begins between two vectors
    const uint64_t v0 = (uint64_t)blockIdx.x * (kThreads * kVectors<T>) + threadIdx.x;
    Pack<T, E> x[kVectors<T>], r[kVectors<T>];
    uint32_t left[kVectors<T>];
#pragma unroll
    for (int i = 0; i < kVectors<T>; ++i) {
        const uint64_t at = (v0 + i * kThreads) * E;
        left[i] = at >= a.n ? 0 : a.n - at < E ? (uint32_t)(a.n - at) : E;
        if (!C::kRagged && left[i] == E) {
            x[i] = load_pack<T, E>((const T*)a.x + at);
            if (kResidual) r[i] = load_pack<T, E>((const T*)a.residual + at);
        } else if (left[i]) {
            x[i] = load_columns<Piece>((const T*)a.x + at, left[i]);
            if (kResidual) r[i] = load_columns<Piece>((const T*)a.residual + at, left[i]);
        }
    }
    const uint64_t call = a.call + (a.call_at ? *a.call_at : 0);
#pragma unroll
    for (int i = 0; i < kVectors<T>; ++i) {
        if (!left[i]) return;
        const uint64_t at = (v0 + i * kThreads) * E;
        float y[E];
#pragma unroll
        for (int q = 0; q < E / 4; ++q) {
            const uint64_t group = at / 4 + q;
            const Philox4 w = philox4x32_10(Philox4{(uint32_t)group, (uint32_t)(group >> 32), (uint32_t)call,
                                                    kTagDropout | ((uint32_t)(call >> 32) & 0xFFFFFFu)}, keys);
            const uint32_t word[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                y[q * 4 + e] = word[e] >= a.least && !a.none ? to_float(x[i].v[q * 4 + e]) * a.scale : 0.0f;
                if (kResidual) y[q * 4 + e] += to_float(r[i].v[q * 4 + e]);
            }
        }
        if (!C::kRagged && left[i] == E) store_pack<T, E>((T*)a.out + at, y);
        else store_columns<Piece>((T*)a.out + at, y, left[i]);
    }
}

}  // namespace

cudaError_t launch_dropout(cudaStream_t stream, const DropoutArgs& a) {
    const uintptr_t places = (uintptr_t)a.x | (uintptr_t)a.out | (uintptr_t)a.residual;
    const PhiloxKeys keys(a.seed);
    return with_type(a.type, [&](auto t) {
        using T = decltype(t);
        constexpr int E = 16 / sizeof(T);
        auto launch = [&](auto c, auto residual) {
            using C = decltype(c);
            const uint64_t vecs = (a.n + C::E - 1) / C::E;
            k_dropout<T, C, decltype(residual)::value><<<(uint32_t)((vecs + kThreads * kVectors<T> - 1) / (kThreads * kVectors<T>)), kThreads, 0, stream>>>(a, keys);
            return cudaGetLastError();
        };
        auto with_residual = [&](auto c) {
            return a.residual ? launch(c, std::true_type()) : launch(c, std::false_type());
        };
        return places % 16 == 0 ? with_residual(Columns<E, false>()) : with_residual(Columns<4, true>());
    });
}

}  // namespace tensair
