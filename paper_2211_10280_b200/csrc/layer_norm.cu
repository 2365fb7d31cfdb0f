// Layer norm of rows and its gradient.
//
//     y = (x - mean) rstd w + b           mean, rstd = 1 / sqrt(variance + eps) of the row
//     c = (x - mean) rstd, g = dy w:      dx = rstd (g - mean(g) - c mean(g c)),  dw = sum over rows of dy c,  db = of dy
//
// A row is read once: it stays in the registers of the threads that share it (8 lanes, a warp, or a block for wide rows), and the
// variance is taken about the mean, in a second pass over those registers.  Rows that do not fit (beyond 16,384 columns of 16 bits)
// are read again, out of the level-2 cache.  The sums over rows (dw, db) stay in the registers of a grid that goes round
// the rows; each block leaves one partial row, and a second launch adds those up in block order: no sum depends on timing.
//
// Bound by the latency of the rows' reads.  65,536 rows of 512 in bf16: forward 35 us (134 MB, 3.8 TB/s; blocks for five to a
// multiprocessor; six spill, 41 us), backward 48 us (201 MB, 4.2 TB/s) and 6 for the second launch.  The backward pass has 16 warps to
// a multiprocessor, whose registers hold weight and sums of 16 columns to a lane; the next rows are prefetched into the level-2
// cache (52 us against 54).  Held in registers instead they left room for half the warps (74 us).  One row: 4.4 us, a launch.
// Rows that fit into no block: 1,024 of 20,000 in bf16 43 us forward; the gradient 281, of which 231 are the sums over rows, by columns of
// 2 or 4 bytes to a thread, from a grid that reads its inputs once more.
//
// The sums over rows are held in 32 bits: a thread adds up n / 9,472 to n / 296 rows, by their width (n / 1,024 of the widest); the blocks' partial
// rows are joined by sums of up to 10 and of 32 of those.
#include "columns.cuh"
#include "layers.h"

namespace tensair {

namespace {

constexpr int kThreads = 256;            // of blocks whose rows belong to warps or parts of them
constexpr int kMostThreads = 512;        // of a block that shares a row
constexpr int kWideThreads = 1024;       // of blocks for rows that do not fit into one

// `E` values of a parameter vector from column `col` on.
template <typename C>
__device__ __forceinline__ void load_param(const void* p, uint32_t type, uint32_t col, uint32_t left, float (&out)[C::E]) {
    auto take = [&](auto zero) {
        using T = decltype(zero);
        const Pack<T, C::E> x = load_columns<C>((const T*)p + col, left);
#pragma unroll
        for (int e = 0; e < C::E; ++e) out[e] = to_float(x.v[e]);
    };
    if (type == 0) take(float());
    else if (type == 1) take(__nv_bfloat16());
    else take(__half());
}

// Sums of two values over the threads that share a row: 8 or 32 lanes, or (kGroup 0) the block; every thread gets them.
template <int kGroup>
struct RowSum {
    float2* shared;      // [2][32], kGroup 0 alone
    uint32_t turn = 0;
    __device__ __forceinline__ float2 operator()(float2 x) {
        constexpr int kLanes = kGroup ? kGroup : 32;
#pragma unroll
        for (int o = kLanes / 2; o; o /= 2) {
            x.x += __shfl_xor_sync(0xFFFFFFFFu, x.x, o);
            x.y += __shfl_xor_sync(0xFFFFFFFFu, x.y, o);
        }
        if constexpr (kGroup == 0) {
            float2* at = shared + (turn ^= 32);
            const uint32_t warps = blockDim.x / 32, lane = threadIdx.x & 31;
            if (lane == 0) at[threadIdx.x / 32] = x;
            __syncthreads();      // two turns' places: the next turn's writes do not meet this one's reads
            x = lane < warps ? at[lane] : make_float2(0.0f, 0.0f);
#pragma unroll
            for (int o = 16; o; o /= 2) {
                x.x += __shfl_xor_sync(0xFFFFFFFFu, x.x, o);
                x.y += __shfl_xor_sync(0xFFFFFFFFu, x.y, o);
            }
        }
        return x;
    }
    __device__ __forceinline__ float operator()(float x) {
        return operator()(make_float2(x, 0.0f)).x;
    }
};
template <>
__device__ __forceinline__ float RowSum<32>::operator()(float x) {
#pragma unroll
    for (int o = 16; o; o /= 2) x += __shfl_xor_sync(0xFFFFFFFFu, x, o);
    return x;
}
template <>
__device__ __forceinline__ float RowSum<8>::operator()(float x) {
#pragma unroll
    for (int o = 4; o; o /= 2) x += __shfl_xor_sync(0xFFFFFFFFu, x, o);
    return x;
}

// Where a thread stands: which of its group, and which group of the block (a block of kGroup 0 is one group).
template <int kGroup>
struct Place {
    uint32_t lane, group, groups, width;
    __device__ Place() {
        if constexpr (kGroup == 0) {
            lane = threadIdx.x; group = 0; groups = 1; width = blockDim.x;
        } else {
            lane = threadIdx.x % kGroup; group = threadIdx.x / kGroup; groups = kThreads / kGroup; width = kGroup;
        }
    }
};

// ------------------------------------------------------------------ forward
// K vectors of a row to a thread.
template <typename TX, typename TY, typename C, int kGroup, int K>
__global__ void __launch_bounds__(kGroup ? kThreads : kMostThreads, K < 4 ? kGroup ? 5 : 3 : kGroup ? 3 : 1)
k_norm(const __grid_constant__ NormArgs a, uint32_t vecs) {
    constexpr int E = C::E;
    __shared__ float2 shared[kGroup ? 1 : 64];
    const Place<kGroup> at;
    RowSum<kGroup> row_sum{shared};
    const uint32_t row = blockIdx.x * at.groups + at.group;
    const bool in = row < a.n;
    const TX* x = (const TX*)a.x.data + (uint64_t)(in ? row : 0) * a.x.stride;
    Pack<TX, E> raw[K];
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const uint32_t v = at.lane + k * at.width;
        if (in && v < vecs) raw[k] = load_columns<C>(x + v * E, a.d - v * E);
    }
    float c[K][E], sum = 0.0f;
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const bool mine = in && at.lane + k * at.width < vecs;
#pragma unroll
        for (int e = 0; e < E; ++e) {
            c[k][e] = mine ? to_float(raw[k].v[e]) : 0.0f;      // columns behind a ragged row are zeros
            sum += c[k][e];
        }
    }
    const float mean = row_sum(sum) / (float)a.d;
    float square = 0.0f;
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const uint32_t v = at.lane + k * at.width;
#pragma unroll
        for (int e = 0; e < E; ++e) {
            c[k][e] -= mean;
            if (v < vecs && (!C::kRagged || v * E + e < a.d)) square += c[k][e] * c[k][e];
        }
    }
    const float rstd = 1.0f / sqrtf(row_sum(square) / (float)a.d + a.eps);
    if (!in) return;
    if (at.lane == 0 && a.mean) {
        a.mean[row] = mean;
        a.rstd[row] = rstd;
    }
    TY* y = (TY*)a.y.data + (uint64_t)row * a.y.stride;
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const uint32_t v = at.lane + k * at.width, col = v * E;
        if (v >= vecs) break;
        float w[E], b[E];
        load_param<C>(a.weight, a.param_type, col, a.d - col, w);
        if (a.bias) load_param<C>(a.bias, a.param_type, col, a.d - col, b);
#pragma unroll
        for (int e = 0; e < E; ++e) {
            w[e] *= c[k][e] * rstd;
            if (a.bias) w[e] += b[e];
        }
        store_columns<C>(y + col, w, a.d - col);
    }
}

// Rows that do not fit into a block's registers: three passes, the later ones out of the level-2 cache.
template <typename TX, typename TY, typename C>
__global__ void __launch_bounds__(kWideThreads)
k_norm_wide(const __grid_constant__ NormArgs a, uint32_t vecs) {
    constexpr int E = C::E;
    __shared__ float2 shared[64];
    RowSum<0> row_sum{shared};
    const uint32_t row = blockIdx.x;
    const TX* x = (const TX*)a.x.data + (uint64_t)row * a.x.stride;
    float sum = 0.0f, square = 0.0f;
    for (uint32_t v = threadIdx.x; v < vecs; v += kWideThreads) {
        const Pack<TX, E> raw = load_columns<C>(x + v * E, a.d - v * E);
#pragma unroll
        for (int e = 0; e < E; ++e) sum += to_float(raw.v[e]);
    }
    const float mean = row_sum(sum) / (float)a.d;
    for (uint32_t v = threadIdx.x; v < vecs; v += kWideThreads) {
        const Pack<TX, E> raw = load_columns<C>(x + v * E, a.d - v * E);
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const float c = to_float(raw.v[e]) - mean;
            if (!C::kRagged || v * E + e < a.d) square += c * c;
        }
    }
    const float rstd = 1.0f / sqrtf(row_sum(square) / (float)a.d + a.eps);
    if (threadIdx.x == 0 && a.mean) {
        a.mean[row] = mean;
        a.rstd[row] = rstd;
    }
    TY* y = (TY*)a.y.data + (uint64_t)row * a.y.stride;
    for (uint32_t v = threadIdx.x; v < vecs; v += kWideThreads) {
        const uint32_t col = v * E;
        const Pack<TX, E> raw = load_columns<C>(x + col, a.d - col);
        float w[E], b[E];
        load_param<C>(a.weight, a.param_type, col, a.d - col, w);
        if (a.bias) load_param<C>(a.bias, a.param_type, col, a.d - col, b);
#pragma unroll
        for (int e = 0; e < E; ++e) {
            w[e] *= (to_float(raw.v[e]) - mean) * rstd;
            if (a.bias) w[e] += b[e];
        }
        store_columns<C>(y + col, w, a.d - col);
    }
}

// ------------------------------------------------------------------ backward
// The grid goes round the rows; a thread keeps the weight and the sums for its columns.
template <typename TX, typename TY, typename C, int kGroup, int K>
__global__ void __launch_bounds__(kGroup ? kThreads : kMostThreads)
k_norm_gradient(const __grid_constant__ NormArgs a, uint32_t vecs) {
    constexpr int E = C::E;
    __shared__ float2 shared[kGroup ? 1 : 64];
    __shared__ float join[kGroup ? kThreads * E : 1];
    const Place<kGroup> at;
    RowSum<kGroup> row_sum{shared};
    float w[K][E], dw[K][E], db[K][E];
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const uint32_t v = at.lane + k * at.width;
#pragma unroll
        for (int e = 0; e < E; ++e) w[k][e] = dw[k][e] = db[k][e] = 0.0f;
        if (v < vecs) load_param<C>(a.weight, a.param_type, v * E, a.d - v * E, w[k]);
    }
    const uint32_t step = gridDim.x * at.groups;
    // every group makes the same number of turns, so that all lanes of a warp (all warps of a block) take part in its sums
    const uint32_t turns = (a.n + step - 1) / step;
    uint64_t row = blockIdx.x * at.groups + at.group;
    for (uint32_t turn = 0; turn < turns; ++turn, row += step) {
        const bool in = row < a.n;
        const TX* x = (const TX*)a.x.data + (in ? row : 0) * a.x.stride;
        const TY* dy = (const TY*)a.y.data + (in ? row : 0) * a.y.stride;
        Pack<TX, E> rx[K];
        Pack<TY, E> rg[K];
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const uint32_t v = at.lane + k * at.width;
            if (in && v < vecs) {
                rx[k] = load_columns<C>(x + v * E, a.d - v * E);
                rg[k] = load_columns<C>(dy + v * E, a.d - v * E);
            }
        }
        const float mean = in ? a.mean[row] : 0.0f, rstd = in ? a.rstd[row] : 0.0f;
        if (row + step < a.n) {      // the next row, into the level-2 cache
            const TX* next_x = x + (uint64_t)step * a.x.stride;
            const TY* next_dy = dy + (uint64_t)step * a.y.stride;
#pragma unroll
            for (int k = 0; k < K; ++k) {
                const uint32_t v = at.lane + k * at.width;
                if (v < vecs) {
                    prefetch(next_x + v * E);
                    prefetch(next_dy + v * E);
                }
            }
        }
        float2 sum = make_float2(0.0f, 0.0f);
#pragma unroll
        for (int k = 0; k < K; ++k) {
            if (in && at.lane + k * at.width < vecs) {
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    const float c = (to_float(rx[k].v[e]) - mean) * rstd, g = to_float(rg[k].v[e]);
                    dw[k][e] += g * c;       // columns behind a ragged row: g is zero
                    db[k][e] += g;
                    sum.x += g * w[k][e];
                    sum.y += g * w[k][e] * c;
                }
            }
        }
        sum = row_sum(sum);
        sum.x /= (float)a.d;
        sum.y /= (float)a.d;
        if (!in) continue;
        TX* dx = (TX*)a.dx.data + row * a.dx.stride;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const uint32_t v = at.lane + k * at.width;
            if (v >= vecs) break;
            float out[E];
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const float c = (to_float(rx[k].v[e]) - mean) * rstd, g = to_float(rg[k].v[e]);
                out[e] = rstd * (g * w[k][e] - sum.x - c * sum.y);
            }
            store_columns<C>(dx + v * E, out, a.d - v * E);
        }
    }
    if (!a.partials) return;
    // the block's groups joined, in their order
    float* part = a.partials + (uint64_t)blockIdx.x * 2 * a.partial_stride;
#pragma unroll
    for (int k = 0; k < K; ++k) {
#pragma unroll
        for (int which = 0; which < 2; ++which) {
            const uint32_t v = at.lane + k * at.width;
            float sum[E];
#pragma unroll
            for (int e = 0; e < E; ++e) sum[e] = which ? db[k][e] : dw[k][e];
            if constexpr (kGroup != 0) {
                // [E][threads]: neighbours write to neighbouring banks
                __syncthreads();
#pragma unroll
                for (int e = 0; e < E; ++e) join[e * kThreads + threadIdx.x] = sum[e];
                __syncthreads();
                if (at.group == 0)
                    for (uint32_t g = 1; g < at.groups; ++g)
#pragma unroll
                        for (int e = 0; e < E; ++e) sum[e] += join[e * kThreads + g * kGroup + at.lane];
            }
            if (at.group == 0 && v < vecs) store_pack<float, E>(part + which * a.partial_stride + v * E, sum);
        }
    }
}

template <typename TX, typename TY, typename C>
__global__ void __launch_bounds__(kWideThreads)
k_norm_gradient_wide(const __grid_constant__ NormArgs a, uint32_t vecs) {
    constexpr int E = C::E;
    __shared__ float2 shared[64];
    RowSum<0> row_sum{shared};
    const uint32_t row = blockIdx.x;
    const TX* x = (const TX*)a.x.data + (uint64_t)row * a.x.stride;
    const TY* dy = (const TY*)a.y.data + (uint64_t)row * a.y.stride;
    TX* dx = (TX*)a.dx.data + (uint64_t)row * a.dx.stride;
    const float mean = a.mean[row], rstd = a.rstd[row];
    float2 sum = make_float2(0.0f, 0.0f);
    for (uint32_t v = threadIdx.x; v < vecs; v += kWideThreads) {
        const uint32_t col = v * E;
        const Pack<TX, E> rx = load_columns<C>(x + col, a.d - col);
        const Pack<TY, E> rg = load_columns<C>(dy + col, a.d - col);
        float w[E];
        load_param<C>(a.weight, a.param_type, col, a.d - col, w);
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const float c = (to_float(rx.v[e]) - mean) * rstd, g = to_float(rg.v[e]) * w[e];
            if (!C::kRagged || col + e < a.d) {
                sum.x += g;
                sum.y += g * c;
            }
        }
    }
    sum = row_sum(sum);
    sum.x /= (float)a.d;
    sum.y /= (float)a.d;
    for (uint32_t v = threadIdx.x; v < vecs; v += kWideThreads) {
        const uint32_t col = v * E;
        const Pack<TX, E> rx = load_columns<C>(x + col, a.d - col);
        const Pack<TY, E> rg = load_columns<C>(dy + col, a.d - col);
        float w[E];
        load_param<C>(a.weight, a.param_type, col, a.d - col, w);
#pragma unroll
        for (int e = 0; e < E; ++e) w[e] = rstd * (to_float(rg.v[e]) * w[e] - sum.x - (to_float(rx.v[e]) - mean) * rstd * sum.y);
        store_columns<C>(dx + col, w, a.d - col);
    }
}

// The sums over rows for wide rows: a thread takes a column, a block 32 of them and every gridDim.y-th row.
template <typename TX, typename TY>
__global__ void __launch_bounds__(kWideThreads)
k_norm_columns(const __grid_constant__ NormArgs a) {
    __shared__ float join[2][32][33];
    const uint32_t lane = threadIdx.x % 32, part = threadIdx.x / 32, col = blockIdx.x * 32 + lane;
    float dw = 0.0f, db = 0.0f;
    if (col < a.d)
        for (uint64_t row = blockIdx.y * 32 + part; row < a.n; row += gridDim.y * 32) {
            const float g = to_float(((const TY*)a.y.data)[row * a.y.stride + col]);
            dw += g * (to_float(((const TX*)a.x.data)[row * a.x.stride + col]) - a.mean[row]) * a.rstd[row];
            db += g;
        }
    join[0][part][lane] = dw;
    join[1][part][lane] = db;
    __syncthreads();
    if (part < 2 && col < a.d) {
        float sum = 0.0f;
        for (int r = 0; r < 32; ++r) sum += join[part][r][lane];
        a.partials[((uint64_t)blockIdx.y * 2 + part) * a.partial_stride + col] = sum;
    }
}

// Adds up the blocks' partial rows: 32 columns to a block, every 32nd partial row to a warp.
__global__ void __launch_bounds__(kWideThreads)
k_norm_join(const __grid_constant__ NormArgs a, uint32_t count) {
    __shared__ float join[32][33];
    after_previous_launch();
    const uint32_t lane = threadIdx.x % 32, part = threadIdx.x / 32, col = blockIdx.x * 32 + lane, which = blockIdx.y;
    float sum = 0.0f;
    if (col < a.d) {
        const float* at = a.partials + which * a.partial_stride + col;
#pragma unroll 4
        for (uint32_t r = part; r < count; r += 32) sum += at[(uint64_t)r * 2 * a.partial_stride];
    }
    join[part][lane] = sum;
    __syncthreads();
    void* out = which ? a.dbias : a.dweight;
    if (part != 0 || col >= a.d || !out) return;
    for (int r = 1; r < 32; ++r) sum += join[r][lane];
    if (a.param_type == 0) ((float*)out)[col] = sum;
    else if (a.param_type == 1) ((__nv_bfloat16*)out)[col] = from_float<__nv_bfloat16>(sum);
    else ((__half*)out)[col] = from_float<__half>(sum);
}

// ------------------------------------------------------------------ launches
template <int kGroup, int kVectors> struct Shape2 {
    static constexpr int group = kGroup, k = kVectors;
};
// Calls f(shape) for rows of `vecs` vectors; false: they do not fit.
template <typename F>
bool with_shape(uint32_t vecs, F&& f) {
    if (vecs <= 8) f(Shape2<8, 1>());
    else if (vecs <= 32) f(Shape2<32, 1>());
    else if (vecs <= 64) f(Shape2<32, 2>());
    else if (vecs <= 128) f(Shape2<32, 4>());
    else if (vecs <= kMostThreads * 2) f(Shape2<0, 2>());
    else if (vecs <= kMostThreads * 4) f(Shape2<0, 4>());
    else return false;
    return true;
}
uint32_t threads_of(int group, int k, uint32_t vecs) {
    if (group) return kThreads;
    const uint32_t t = (vecs + k - 1) / k;
    return (t + 31) / 32 * 32;
}

template <typename F>
cudaError_t with_norm_types(uint32_t x, uint32_t y, F&& f) {
    if (x == 0 && y == 0) return f(float(), float());
    if (x == 0 && y == 1) return f(float(), __nv_bfloat16());
    if (x == 0 && y == 2) return f(float(), __half());
    if (x == 1 && y == 1) return f(__nv_bfloat16(), __nv_bfloat16());
    if (x == 2 && y == 2) return f(__half(), __half());
    return cudaErrorInvalidValue;
}
// 16-bit rows: 8, 4 or single columns at once; fp32 rows: 4 or single ones.
template <bool kEight, typename F>
cudaError_t with_norm_columns(uint32_t e, F&& f) {
    if constexpr (kEight)
        if (e == 8) return f(Columns<8, false>());
    if (e >= 4) return f(Columns<4, false>());
    return f(Columns<4, true>());
}
uint32_t columns_of(const NormArgs& a) {
    const uint32_t most = a.y.type == 0 ? 4 : 8;
    uint32_t e = vector_of(a.x, a.d, most);
    e = vector_of(a.y, a.d, e);
    if (a.dx.data) e = vector_of(a.dx, a.d, e);
    e = vector_of(RowsView{const_cast<void*>(a.weight), a.d, a.param_type}, a.d, e);
    if (a.bias) e = vector_of(RowsView{const_cast<void*>(a.bias), a.d, a.param_type}, a.d, e);
    return e;
}

}  // namespace

cudaError_t launch_norm(cudaStream_t stream, const NormArgs& a) {
    return with_norm_types(a.x.type, a.y.type, [&](auto tx, auto ty) {
        using TX = decltype(tx);
        using TY = decltype(ty);
        return with_norm_columns<sizeof(TY) == 2>(columns_of(a), [&](auto c) {
            using C = decltype(c);
            const uint32_t vecs = (a.d + C::E - 1) / C::E;
            const bool fits = with_shape(vecs, [&](auto shape) {
                using S = decltype(shape);
                const uint32_t threads = threads_of(S::group, S::k, vecs), rows = S::group ? kThreads / S::group : 1;
                k_norm<TX, TY, C, S::group, S::k><<<(a.n + rows - 1) / rows, threads, 0, stream>>>(a, vecs);
            });
            if (!fits) k_norm_wide<TX, TY, C><<<a.n, kWideThreads, 0, stream>>>(a, vecs);
            return cudaGetLastError();
        });
    });
}

// Blocks of the backward launch, whatever the device: the order of the sums hangs on it.
static constexpr uint32_t kNormBlocks = 148 * 2, kWideParts = 32;
uint32_t norm_partials(uint32_t n, uint32_t d) {
    // the widest any of the ways takes for rows of d columns
    const uint32_t most = d <= kMostThreads * 4 * 8 ? kNormBlocks : kWideParts;
    return n < most ? n : most;
}

cudaError_t launch_norm_gradient(cudaStream_t stream, const NormArgs& a) {
    uint32_t parts = 0;
    const cudaError_t err = with_norm_types(a.x.type, a.y.type, [&](auto tx, auto ty) {
        using TX = decltype(tx);
        using TY = decltype(ty);
        return with_norm_columns<sizeof(TY) == 2>(columns_of(a), [&](auto c) {
            using C = decltype(c);
            const uint32_t vecs = (a.d + C::E - 1) / C::E;
            const bool fits = with_shape(vecs, [&](auto shape) {
                using S = decltype(shape);
                const uint32_t threads = threads_of(S::group, S::k, vecs), rows = S::group ? kThreads / S::group : 1;
                parts = (a.n + rows - 1) / rows;
                if (parts > kNormBlocks) parts = kNormBlocks;
                k_norm_gradient<TX, TY, C, S::group, S::k><<<parts, threads, 0, stream>>>(a, vecs);
            });
            if (!fits) {
                if (a.partials) {      // first: dx may be written over the incoming gradient
                    parts = a.n < kWideParts ? a.n : kWideParts;
                    k_norm_columns<TX, TY><<<dim3((a.d + 31) / 32, parts), kWideThreads, 0, stream>>>(a);
                }
                k_norm_gradient_wide<TX, TY, C><<<a.n, kWideThreads, 0, stream>>>(a, vecs);
            }
            return cudaGetLastError();
        });
    });
    if (err != cudaSuccess || !a.partials) return err;
    return launch_early(k_norm_join, dim3((a.d + 31) / 32, 2), kWideThreads, 0, stream, a, parts);
}

}  // namespace tensair
