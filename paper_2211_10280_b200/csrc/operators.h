// Shared pieces of the language-model operators (embedding lookup, its gradient, AdamW): argument blocks, element
// types, and the host-side launchers.  These calls have no context: they work on caller-owned tensors, on the
// caller's stream, and count no launches of a context.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <utility>

#include "common.cuh"

namespace tensair {

constexpr int64_t kNoPadding = INT64_MIN;
// How the token ids of a batch are read.
struct TokenIds {
    const void* ids;
    int64_t padding;      // an id equal to this stands for "no token"; kNoPadding: none does
    uint32_t* err;        // nullable: receives kErrBadToken (checked build: and kErrBounds)
    uint32_t n, V;
    bool wide;            // 64-bit ids

    __device__ __forceinline__ bool is_token(int64_t id) const { return (uint64_t)id < V && id != padding; }
    // for an id that is no token
    __device__ __forceinline__ void report(int64_t id) const {
        if (err && (id != padding || padding == kNoPadding)) atomicOr(err, kErrBadToken);
    }
};

// ---- element types: everything is computed in fp32 and rounded to nearest once, when it is stored
__device__ __forceinline__ float to_float(float x) { return x; }
__device__ __forceinline__ float to_float(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ float to_float(__half x) { return __half2float(x); }
template <typename T> __device__ __forceinline__ T from_float(float x);
template <> __device__ __forceinline__ float from_float<float>(float x) { return x; }
template <> __device__ __forceinline__ __nv_bfloat16 from_float<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }
template <> __device__ __forceinline__ __half from_float<__half>(float x) { return __float2half_rn(x); }

// E consecutive elements, aligned for one access of up to 16 bytes (wider packs are two of them).
template <typename T, int E>
struct alignas(sizeof(T) * E > 16 ? 16 : sizeof(T) * E) Pack {
    T v[E];
};
template <typename T, int E>
__device__ __forceinline__ Pack<T, E> load_pack(const T* p) { return *reinterpret_cast<const Pack<T, E>*>(p); }
template <typename T, int E>
__device__ __forceinline__ void store_pack(T* p, const float (&x)[E]) {
    Pack<T, E> out;
#pragma unroll
    for (int e = 0; e < E; ++e) out.v[e] = from_float<T>(x[e]);
    *reinterpret_cast<Pack<T, E>*>(p) = out;
}

// How rows are cut into the pieces that a thread moves at once: E columns in one access (or two of 16 bytes), where every row
// begins on a multiple of it; or, for rows of odd widths or places, four columns in an access each, `left` of which are inside
// the row.  Four to a thread all the same: what it does per piece is worth more than the accesses, whose cache lines its
// neighbours share.
template <int kColumns, bool kIsRagged>
struct Columns {
    static constexpr int E = kColumns;
    static constexpr bool kRagged = kIsRagged;
};
template <typename C, typename T>
__device__ __forceinline__ Pack<T, C::E> load_columns(const T* p, uint32_t left) {
    if constexpr (!C::kRagged) return load_pack<T, C::E>(p);
    else {
        Pack<T, C::E> x;
#pragma unroll
        for (int e = 0; e < C::E; ++e) x.v[e] = e < (int)left ? p[e] : from_float<T>(0.0f);
        return x;
    }
}
template <typename C, typename T>
__device__ __forceinline__ void store_columns(T* p, const float (&x)[C::E], uint32_t left) {
    if constexpr (!C::kRagged) store_pack<T, C::E>(p, x);
    else {
#pragma unroll
        for (int e = 0; e < C::E; ++e)
            if (e < (int)left) p[e] = from_float<T>(x[e]);
    }
}

// Asks for a line to be brought into the level-2 cache.
__device__ __forceinline__ void prefetch(const void* p) { asm volatile("prefetch.global.L2 [%0];" ::"l"(p)); }

// Eight floats in one 32-byte access (sm_100 has them), where the address is a multiple of 32.
__device__ __forceinline__ void load_eight(const float* p, float (&x)[8]) {
    asm volatile("ld.global.v8.f32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=f"(x[0]), "=f"(x[1]), "=f"(x[2]), "=f"(x[3]), "=f"(x[4]), "=f"(x[5]), "=f"(x[6]), "=f"(x[7]) : "l"(p));
}
__device__ __forceinline__ void store_eight(float* p, const float (&x)[8]) {
    asm volatile("st.global.v8.f32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
                 ::"l"(p), "f"(x[0]), "f"(x[1]), "f"(x[2]), "f"(x[3]), "f"(x[4]), "f"(x[5]), "f"(x[6]), "f"(x[7]) : "memory");
}

// x / divisor for 32-bit x by one multiplication with a reciprocal rounded up (Granlund & Montgomery 1994):
// exact for x < 2^31 and any divisor >= 1.
struct FastDiv {
    uint32_t divisor, mul, shift;
    explicit FastDiv(uint32_t d = 1) : divisor(d) {
        shift = 0;
        while (shift < 31 && (1ull << shift) < d) ++shift;
        mul = (uint32_t)(((1ull << 32) * ((1ull << shift) - d)) / d + 1);
    }
    __device__ __forceinline__ uint32_t div(uint32_t x) const { return (__umulhi(x, mul) + x) >> shift; }
};

// The constants of one AdamW step (see adamw.cuh for the formulas).
struct AdamwConsts {
    float beta1, rest1;        // beta1, 1 - beta1
    float beta2, rest2;
    float eps;
    float inv_root2;           // 1 / sqrt(1 - beta2^t)
    float step_size;           // lr / (1 - beta1^t)
    float keep;                // 1 - lr * weight_decay
    const float* grad_scale;   // device, nullable
};

// ---- token_sort.cu
// A batch's positions sorted by token, stable, with the tokens' segments.
struct SortedTokens {
    uint32_t* key;         // [n] token of each sorted position; V from n_valid on
    uint32_t* pos;         // [n] the batch position it came from
    uint32_t* seg_start;   // [min(n, V) + 1] first sorted position of each distinct token, then n_valid
    uint32_t* span_rank;   // [spans] distinct tokens that begin before the span
    uint32_t* info;        // [0] n_valid, [1] distinct tokens, [2], [3] set to zero: entries of SumArgs::large
    uint32_t* err;         // nullable: the caller's error word (checked build)
};
constexpr uint32_t kSpan = 64;         // sorted positions
// Sorted positions; a token with more is added up in pieces.  Whole table bf16 (16,384 tokens of 512), rows, AdamW rows (65,536 of 300):
// 43, 60, 87 us with 16; 45, 66, 92 with 8; 47, 61, 85 with 32; 54, 66, 86 with 64.
constexpr uint32_t kWindow = 16;
struct SortScratch {
    item_t* a;
    item_t* b;
    uint32_t* hist;
    uint32_t* tile_counts;
};
// Rows to set to zero, in bytes; rows 0: none.
struct ClearRows {
    uint8_t* data;
    uint64_t stride, width, rows;
};
struct SortScratchBytes {
    size_t items, hist, tile_counts;   // of a and b each, and of the other two
};
SortScratchBytes sort_scratch_bytes(uint32_t n);
constexpr uint32_t kTiledSort = 1 << 17;   // the longest batch whose scratch is that of the sort in tiles
// Also clears `c`, beside the sort.
cudaError_t launch_token_sort(cudaStream_t stream, const TokenIds& t, const SortedTokens& s, const SortScratch& w,
                              const ClearRows& c, int sms);
cudaError_t launch_clear(cudaStream_t stream, const ClearRows& c, int sms);

// ---- embedding.cu
struct RowsView {          // rows of d elements, `stride` elements apart
    void* data;
    uint32_t stride;       // below 2^31: a row's offset is one 32 x 32 -> 64-bit product
    uint32_t type;
};
enum SumKind { kSumTable, kSumRows, kSumAdamw };
struct SumArgs {
    SortedTokens s;
    RowsView grad;         // [n] gradient rows
    uint32_t n, V, d;
    float scale;
    float* partials;       // [windows][2][partial_stride]: the pieces of tokens with more than kWindow positions: of one that
                           // began in an earlier window, of one that begins in this window
    uint32_t partial_stride;
    uint4* large;          // [n / (kWindow + 1)] those tokens: (window, rank, last window, token), the ones with many pieces
                           // from the front, the others from the end
    // where a finished row goes
    RowsView out;          // kSumTable: row `token`; kSumRows: row `rank`; kSumAdamw: the table of parameters
    int accumulate;        // kSumTable: add to what is there
    uint32_t* out_ids;     // kSumRows
    uint32_t* out_count;   // kSumRows
    float* m;
    float* v;
    uint32_t m_stride, v_stride;
    AdamwConsts adamw;
};
cudaError_t launch_lookup(cudaStream_t stream, const TokenIds& t, const RowsView& table, const RowsView& out, uint32_t d,
                          float scale);
// embedding_short.cu: sort and sums of a batch of up to 1,024 positions in one launch, without a workspace; for kSumTable without
// accumulate the launch before it on the stream has to be launch_clear.
bool is_short(uint32_t n);
cudaError_t launch_short_sums(cudaStream_t stream, SumKind kind, const SumArgs& a, const TokenIds& t, int sms);
cudaError_t launch_token_sums(cudaStream_t stream, SumKind kind, const SumArgs& a, int sms);
// A launch that may begin while the launch before it on the stream is still running: its blocks wait in
// after_previous_launch() before they touch what that one writes, and let their own successor begin only after that (the sort in a
// cluster lets it begin at once: no launch before it writes what it or its successor reads).  What the launch before writes is read through plain pointers (no const __restrict__, no __ldg): reads of memory that is taken to stay
// unchanged for the whole kernel are not ordered by the wait.
template <typename... Params, typename... Args>
cudaError_t launch_early(void (*kernel)(Params...), dim3 grid, uint32_t block, size_t shared, cudaStream_t stream, Args&&... args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = block;
    cfg.dynamicSmemBytes = shared;
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, std::forward<Args>(args)...);
}
__device__ __forceinline__ void after_previous_launch() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void let_next_launch_begin() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }

// ---- adamw.cu
struct AdamwTensor {
    void* param;
    const void* grad;
    void* m;
    void* v;
    float* m_scale;        // 8-bit moments
    float* v_scale;
    void* copy;            // nullable
    uint64_t n;
    uint64_t block0;       // 8-bit moments: blocks of the tensors before it
    float step_size, keep;
    uint32_t param_type, grad_type, copy_type;
};
cudaError_t launch_adamw(cudaStream_t stream, const AdamwTensor* tensors, uint32_t count, int bits, const AdamwConsts& c,
                         uint64_t step, uint64_t seed, int sms);

inline uint32_t type_bytes(uint32_t type) { return type == 0 ? 4 : 2; }

}  // namespace tensair
