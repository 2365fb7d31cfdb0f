// Shared pieces of the operators of a recurrent language model (layer norm, dropout, gated linear recurrence, sampling): argument
// blocks and the host-side launchers.
#pragma once
#include "operators.h"

namespace tensair {

// ---- layer_norm.cu
struct NormArgs {
    RowsView x;            // [n]
    RowsView y;            // [n] what the forward call writes; the incoming gradient of the backward call
    RowsView dx;           // [n] backward
    const void* weight;    // [d] of param_type
    const void* bias;      // nullable
    float* mean;           // [n] forward: nullable, written; backward: read
    float* rstd;
    void* dweight;         // backward: [d] of param_type, nullable
    void* dbias;
    float* partials;       // backward: [norm_partials(n, d)][2][partial_stride], the blocks' sums for weight and bias
    uint32_t partial_stride, param_type, n, d;
    float eps;
};
cudaError_t launch_norm(cudaStream_t stream, const NormArgs& a);
uint32_t norm_partials(uint32_t n, uint32_t d);
cudaError_t launch_norm_gradient(cudaStream_t stream, const NormArgs& a);

// ---- dropout.cu
struct DropoutArgs {
    const void* x;
    const void* residual;          // nullable
    void* out;
    uint64_t n;
    uint64_t seed, call;
    const uint64_t* call_at;       // nullable: device, added to `call`
    float scale;                   // of what is kept
    uint32_t least;                // smallest word that keeps its element
    uint32_t type;
    bool none;                     // nothing is kept
};
cudaError_t launch_dropout(cudaStream_t stream, const DropoutArgs& a);

// ---- recurrence.cu
struct StepsView {                 // [B][T] rows of d elements
    void* data;
    uint64_t batch, step;          // elements between sequences and between steps
};
constexpr uint32_t kMark = 8;      // steps between the marks
struct RecurrenceArgs {
    StepsView gate, value;
    StepsView out;                 // forward: h; backward: the incoming gradient
    StepsView dgate, dvalue;       // backward
    const float* state;            // [B][d], nullable: forward: the states before the first step; backward: the gradient of the last
    float* last;                   // [B][d], nullable: forward: the states after the last step; backward: the gradient of the first
    float* marks;                  // [B][ceil(T / kMark)][d], forward: nullable, written; backward: read
    const int32_t* lengths;        // [B], nullable
    uint32_t B, T, d, type;
};
cudaError_t launch_recurrence(cudaStream_t stream, const RecurrenceArgs& a, int sms);
cudaError_t launch_recurrence_gradient(cudaStream_t stream, const RecurrenceArgs& a, int sms);
// One step: `state` is read and `last` (which may be the same) written.
cudaError_t launch_recurrence_step(cudaStream_t stream, const RecurrenceArgs& a);

// ---- sample.cu
// A setting of the draw: one value for all rows, or one for each row.
template <typename T>
struct Setting {
    const T* rows;
    T all;
    __device__ __forceinline__ T of(uint32_t row) const { return rows ? rows[row] : all; }
};
struct SampleArgs {
    RowsView logits;               // [n]
    const float* uniform;          // [n]
    int64_t* token;                // [n]
    float* logprob;                // [n], nullable
    Setting<float> temperature, top_p, min_p;
    Setting<int32_t> top_k;
    uint32_t n, V, bits;           // a weight is a multiple of 2^-bits
};
cudaError_t launch_sample(cudaStream_t stream, const SampleArgs& a, int sms);

}  // namespace tensair
