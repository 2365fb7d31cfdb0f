// What the launches that add up gradient rows by token share: how a finished row is put where it belongs, how a token's rows are
// added up, and the choice of a kernel by types and widths.
#pragma once
#include "adamw.cuh"
#include "columns.cuh"
#include "operators.h"

namespace tensair {

template <int kCount> struct Rows { static constexpr int value = kCount; };

// What becomes of the finished sum of a token, E columns from `col` on.  fetch() reads what it is joined with, so that
// several tokens' reads are in flight before the first is needed; put() joins and stores.
template <SumKind kKind, typename TO, typename C>
struct Finish {
    static constexpr int E = C::E;
    Pack<TO, E> old;
    Pack<float, E> m0, v0;

    __device__ __forceinline__ void fetch(const SumArgs& a, uint32_t key, uint32_t col) {
        if (kKind == kSumRows || (kKind == kSumTable && !a.accumulate)) return;
        old = load_columns<C>((const TO*)a.out.data + (uint64_t)key * a.out.stride + col, a.d - col);
        if (kKind == kSumAdamw) {
            m0 = load_columns<C>(a.m + (uint64_t)key * a.m_stride + col, a.d - col);
            v0 = load_columns<C>(a.v + (uint64_t)key * a.v_stride + col, a.d - col);
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
            store_columns<C>(a.m + (uint64_t)key * a.m_stride + col, m, a.d - col);
            store_columns<C>(a.v + (uint64_t)key * a.v_stride + col, v, a.d - col);
        }
        store_columns<C>(out, y, a.d - col);
    }
};


// Adds up `count` gradient rows, E columns of them, `left` of which are inside the rows: row i is the batch's position pos[i].
// Whole batches first, then what is left in halves: no access is guarded, and few are waited for alone (guarded batches of four
// took 47 us where this takes 43: whole table in bf16, 16,384 tokens of 512).
template <SumKind kKind, typename C, typename TG>
__device__ __forceinline__ void add_rows(const TG* grad, uint32_t stride, const uint32_t* pos, uint32_t count, uint32_t left, float (&sum)[C::E]) {
    constexpr int E = C::E;
#pragma unroll
    for (int e = 0; e < E; ++e) sum[e] = 0.0f;
    auto add = [&](uint32_t i, auto batch) {
        constexpr int kRows = decltype(batch)::value;
        Pack<TG, E> x[kRows];
#pragma unroll
        for (int j = 0; j < kRows; ++j) x[j] = load_columns<C>(grad + (uint64_t)pos[i + j] * stride, left);
#pragma unroll
        for (int j = 0; j < kRows; ++j)
#pragma unroll
            for (int e = 0; e < E; ++e) sum[e] += to_float(x[j].v[e]);
    };
    constexpr int kWhole = kKind == kSumAdamw ? 8 : 4;
    uint32_t i = 0;
    for (; i + kWhole <= count; i += kWhole) add(i, Rows<kWhole>());
    if (kWhole > 4 && i + 4 <= count) { add(i, Rows<4>()); i += 4; }
    if (i + 2 <= count) { add(i, Rows<2>()); i += 2; }
    if (i < count) add(i, Rows<1>());
}

template <SumKind kKind> struct Kind { static constexpr SumKind value = kKind; };
// Calls f(kind, gradient type, output type, columns) for what `a` asks for.
template <typename F>
cudaError_t with_sum(SumKind kind, const SumArgs& a, F&& f) {
    uint32_t e = vector_of(a.grad, a.d, widest(a.grad, a.out));
    e = vector_of(a.out, a.d, e);
    if (kind == kSumAdamw) {
        e = vector_of(RowsView{a.m, a.m_stride, 0}, a.d, e);
        e = vector_of(RowsView{a.v, a.v_stride, 0}, a.d, e);
    }
    return with_type(a.grad.type, [&](auto tg) {
        return with_type(a.out.type, [&](auto to) {
            return with_columns(e, [&](auto c) {
                if (kind == kSumAdamw) return f(Kind<kSumAdamw>(), tg, to, c);
                if (kind == kSumTable) return f(Kind<kSumTable>(), tg, to, c);
                if constexpr (sizeof(to) == 4) return f(Kind<kSumRows>(), tg, to, c);
                else return cudaErrorInvalidValue;
            });
        });
    });
}

}  // namespace tensair
