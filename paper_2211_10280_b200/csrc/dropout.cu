// Dropout whose mask is never stored: element e is kept where word e % 4 of Philox4x32-10 of counter (e / 4, call) reaches
// p 2^32, so the backward pass draws the same mask again.  y = kept ? x / (1 - p) : 0, plus a residual if there is one.
#include "columns.cuh"
#include "layers.h"
#include "philox.cuh"

namespace tensair {

namespace {

constexpr int kThreads = 256;

template <typename T, typename C, bool kResidual>
__global__ void __launch_bounds__(kThreads)
k_dropout(const __grid_constant__ DropoutArgs a, const __grid_constant__ PhiloxKeys keys, uint64_t vecs) {
    constexpr int E = C::E;
    const uint64_t v = (uint64_t)blockIdx.x * kThreads + threadIdx.x;
    if (v >= vecs) return;
    const uint64_t call = a.call + (a.call_at ? *a.call_at : 0);
    const uint64_t at = v * E;
    const uint32_t left = a.n - at < E ? (uint32_t)(a.n - at) : E;
    const bool whole = !C::kRagged && left == E;
    using Piece = Columns<E, true>;      // the last vector, or one of a tensor that begins between two vectors
    const T* px = (const T*)a.x + at;
    const Pack<T, E> x = whole ? load_pack<T, E>(px) : load_columns<Piece>(px, left);
    Pack<T, E> r;
    if (kResidual) r = whole ? load_pack<T, E>((const T*)a.residual + at) : load_columns<Piece>((const T*)a.residual + at, left);
    float y[E];
#pragma unroll
    for (int q = 0; q < E / 4; ++q) {
        const uint64_t group = at / 4 + q;
        const Philox4 w = philox4x32_10(Philox4{(uint32_t)group, (uint32_t)(group >> 32), (uint32_t)call,
                                                kTagDropout | ((uint32_t)(call >> 32) & 0xFFFFFFu)}, keys);
        const uint32_t word[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            y[q * 4 + e] = word[e] >= a.least && !a.none ? to_float(x.v[q * 4 + e]) * a.scale : 0.0f;
            if (kResidual) y[q * 4 + e] += to_float(r.v[q * 4 + e]);
        }
    }
    if (whole) store_pack<T, E>((T*)a.out + at, y);
    else store_columns<Piece>((T*)a.out + at, y, left);
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
            k_dropout<T, C, decltype(residual)::value><<<(uint32_t)((vecs + kThreads - 1) / kThreads), kThreads, 0, stream>>>(a, keys, vecs);
            return cudaGetLastError();
        };
        auto with_residual = [&](auto c) {
            return a.residual ? launch(c, std::true_type()) : launch(c, std::false_type());
        };
        return places % 16 == 0 ? with_residual(Columns<E, false>()) : with_residual(Columns<4, true>());
    });
}

}  // namespace tensair
