// C entry points of the operators of a recurrent language model: argument checks and launches.
#include "layers.h"

#include <cmath>

#include "context.h"
#include "operator_checks.h"

using namespace tensair;

namespace {

constexpr uint64_t kMaxRows = 1ull << 30, kMaxStep = 1ull << 40;

int check_norm(const tensair_norm* h, const tensair_rows* x, const tensair_rows* y, const char* y_bad) {
    TENSAIR_REQUIRE(h, "norm: NULL");
    TENSAIR_REQUIRE(h->n <= kMaxRows, "norm: n must be at most 2^30");
    TENSAIR_REQUIRE(std::isfinite(h->eps) && h->eps >= 0, "norm: eps must be finite and not negative");
    TENSAIR_REQUIRE(is_float_type(h->param_type), "norm: param_type");
    const uintptr_t b = type_bytes(h->param_type);
    TENSAIR_REQUIRE(h->weight && (uintptr_t)h->weight % b == 0 && (uintptr_t)h->bias % b == 0, "norm: weight is NULL, or weight or bias not aligned to their type");
    TENSAIR_REQUIRE((h->mean == nullptr) == (h->rstd == nullptr) && (uintptr_t)h->mean % 4 == 0 && (uintptr_t)h->rstd % 4 == 0,
                    "norm: mean and rstd go together, aligned to 4 bytes");
    TENSAIR_REQUIRE(x && x->d >= 1 && x->d <= kMaxWidth, "x: NULL, or d not in 1 .. 2^20");
    int rc = check_rows(x, x->d, h->n == 0, "x: NULL", "x: type, stride or alignment");
    if (rc == TENSAIR_OK) rc = check_rows(y, x->d, h->n == 0, y_bad, y_bad);
    if (rc != TENSAIR_OK) return rc;
    TENSAIR_REQUIRE(y->type == x->type || x->type == TENSAIR_FLOAT32, "types: rows of 16 bits are normed to their own type");
    return TENSAIR_OK;
}

uint32_t norm_stride(uint32_t d) { return (uint32_t)round_up(d, 8); }

bool fits(const tensair_steps& s, const tensair_sequences& q, bool written) {
    const uint64_t b = type_bytes(q.type);
    if (!s.data || (uintptr_t)s.data % b || s.batch >= kMaxStep || s.step >= kMaxStep) return false;
    // rows that are written lie apart
    return !written || ((q.T < 2 || s.step >= q.d) && (q.B < 2 || s.batch >= q.d));
}
int check_sequences(const tensair_sequences* q) {
    TENSAIR_REQUIRE(q, "seq: NULL");
    TENSAIR_REQUIRE(q->d >= 1 && q->d <= kMaxWidth, "seq: d must be 1 .. 2^20");
    TENSAIR_REQUIRE(is_float_type(q->type), "seq: type");
    TENSAIR_REQUIRE(q->B <= kMaxRows && q->T <= kMaxRows && q->B * ((q->d + 1) / 2) <= kMaxRows, "seq: B, T or B * d too large");
    TENSAIR_REQUIRE((uintptr_t)q->lengths % 4 == 0, "seq: lengths are not aligned");
    if (q->B && q->T) TENSAIR_REQUIRE(fits(q->gate, *q, false) && fits(q->value, *q, false), "seq: gate or value: NULL, alignment or strides");
    return TENSAIR_OK;
}
StepsView view_of(const tensair_steps& s) { return StepsView{s.data, s.batch, s.step}; }
RecurrenceArgs args_of(const tensair_sequences& q) {
    RecurrenceArgs a = {};
    a.gate = view_of(q.gate);
    a.value = view_of(q.value);
    a.lengths = q.lengths;
    a.B = (uint32_t)q.B;
    a.T = (uint32_t)q.T;
    a.d = q.d;
    a.type = q.type;
    return a;
}
// No steps: `to` (nullable) is `from`, or zeros.
int pass_on(const tensair_sequences& q, const float* from, float* to, void* stream) {
    const size_t bytes = (size_t)q.B * q.d * 4;
    if (!to || !bytes || from == to) return TENSAIR_OK;
    return launched(from ? cudaMemcpyAsync(to, from, bytes, cudaMemcpyDeviceToDevice, (cudaStream_t)stream)
                         : cudaMemsetAsync(to, 0, bytes, (cudaStream_t)stream));
}

}  // namespace

extern "C" {

int tensair_layer_norm(const tensair_norm* norm, const tensair_rows* x, const tensair_rows* out, void* stream) {
    const int rc = check_norm(norm, x, out, "out: NULL, type, width, stride or alignment");
    if (rc != TENSAIR_OK || !norm->n) return rc;
    NormArgs a = {};
    a.x = view_of(*x);
    a.y = view_of(*out);
    a.weight = norm->weight;
    a.bias = norm->bias;
    a.mean = norm->mean;
    a.rstd = norm->rstd;
    a.param_type = norm->param_type;
    a.n = (uint32_t)norm->n;
    a.d = x->d;
    a.eps = norm->eps;
    return launched(launch_norm((cudaStream_t)stream, a));
}

int tensair_norm_workspace_bytes(uint64_t n, uint32_t d, uint64_t* bytes) {
    TENSAIR_REQUIRE(bytes, "bytes: NULL");
    TENSAIR_REQUIRE(n <= kMaxRows && d >= 1 && d <= kMaxWidth, "n or d out of range");
    *bytes = (uint64_t)norm_partials((uint32_t)n, d) * 2 * norm_stride(d) * 4;
    return TENSAIR_OK;
}

int tensair_layer_norm_gradient(const tensair_norm* norm, const tensair_rows* grad, const tensair_rows* x, const tensair_rows* dx,
                                void* dweight, void* dbias, void* workspace, uint64_t workspace_bytes, void* stream) {
    int rc = check_norm(norm, x, grad, "grad: NULL, type, width, stride or alignment");
    if (rc == TENSAIR_OK) rc = check_rows(dx, x->d, norm->n == 0, "dx: NULL", "dx: type, width, stride or alignment");
    if (rc != TENSAIR_OK) return rc;
    TENSAIR_REQUIRE(dx->type == x->type, "dx: must be of x's type");
    TENSAIR_REQUIRE(!norm->n || norm->mean, "norm: mean and rstd are NULL");
    const uint64_t b = type_bytes(norm->param_type);
    TENSAIR_REQUIRE((uintptr_t)dweight % b == 0 && (uintptr_t)dbias % b == 0, "dweight or dbias: not aligned to their type");
    const bool sums = dweight || dbias;
    const uint32_t d = x->d;
    if (!norm->n) {
        for (void* p : {dweight, dbias})
            if (p) {
                const cudaError_t e = cudaMemsetAsync(p, 0, (size_t)d * b, (cudaStream_t)stream);
                if (e != cudaSuccess) return launched(e);
            }
        return TENSAIR_OK;
    }
    if (sums) {
        TENSAIR_REQUIRE(workspace && (uintptr_t)workspace % 256 == 0, "workspace: NULL or not aligned to 256 bytes");
        if (workspace_bytes < (uint64_t)norm_partials((uint32_t)norm->n, d) * 2 * norm_stride(d) * 4)
            return refuse(TENSAIR_ENOMEM, "workspace: smaller than tensair_norm_workspace_bytes says");
    }
    NormArgs a = {};
    a.x = view_of(*x);
    a.y = view_of(*grad);
    a.dx = view_of(*dx);
    a.weight = norm->weight;
    a.mean = norm->mean;
    a.rstd = norm->rstd;
    a.dweight = dweight;
    a.dbias = dbias;
    a.partials = sums ? (float*)workspace : nullptr;
    a.partial_stride = norm_stride(d);
    a.param_type = norm->param_type;
    a.n = (uint32_t)norm->n;
    a.d = d;
    a.eps = norm->eps;
    return launched(launch_norm_gradient((cudaStream_t)stream, a));
}

int tensair_dropout(const tensair_dropout_call* h, void* stream) {
    TENSAIR_REQUIRE(h, "dropout: NULL");
    TENSAIR_REQUIRE(is_float_type(h->type), "dropout: type");
    TENSAIR_REQUIRE(h->n < (1ull << 40), "dropout: n must be below 2^40");
    TENSAIR_REQUIRE(h->p >= 0 && h->p <= 1, "dropout: p must be 0 .. 1");
    TENSAIR_REQUIRE(h->call < (1ull << 56), "dropout: call must be below 2^56");
    TENSAIR_REQUIRE((uintptr_t)h->call_at % 8 == 0, "dropout: call_at is not aligned");
    const uintptr_t b = type_bytes(h->type);
    TENSAIR_REQUIRE((!h->n || (h->x && h->out)) && (uintptr_t)h->x % b == 0 && (uintptr_t)h->out % b == 0 && (uintptr_t)h->residual % b == 0,
                    "dropout: x or out is NULL, or a pointer not aligned to its type");
    if (!h->n) return TENSAIR_OK;
    if (!h->call_at) {
        cudaStreamCaptureStatus status = cudaStreamCaptureStatusNone;
        const cudaError_t e = cudaStreamIsCapturing((cudaStream_t)stream, &status);
        if (e != cudaSuccess) return launched(e);
        TENSAIR_REQUIRE(status == cudaStreamCaptureStatusNone, "a dropout without call_at cannot be captured: replays would repeat its mask");
    }
    DropoutArgs a = {};
    a.x = h->x;
    a.residual = h->residual;
    a.out = h->out;
    a.n = h->n;
    a.seed = h->seed;
    a.call = h->call;
    a.call_at = h->call_at;
    const double least = std::floor(h->p * 4294967296.0);
    a.none = least >= 4294967296.0;
    a.least = a.none ? 0xFFFFFFFFu : (uint32_t)least;
    a.scale = a.none ? 0.0f : (float)(1 / (1 - h->p));
    a.type = h->type;
    return launched(launch_dropout((cudaStream_t)stream, a));
}

int tensair_recurrence(const tensair_sequences* seq, const float* state, const tensair_steps* out, float* last, float* marks, void* stream) {
    const int rc = check_sequences(seq);
    if (rc != TENSAIR_OK) return rc;
    TENSAIR_REQUIRE((uintptr_t)state % 4 == 0 && (uintptr_t)last % 4 == 0 && (uintptr_t)marks % 4 == 0, "state, last or marks: not aligned");
    if (!seq->B || !seq->T) return pass_on(*seq, state, last, stream);
    TENSAIR_REQUIRE(out && fits(*out, *seq, true), "out: NULL, alignment or strides");
    const int sms = multiprocessors();
    if (!sms) return refuse(TENSAIR_ECUDA, "no CUDA device is current");
    RecurrenceArgs a = args_of(*seq);
    a.out = view_of(*out);
    a.state = state;
    a.last = last;
    a.marks = marks;
    return launched(launch_recurrence((cudaStream_t)stream, a, sms));
}

int tensair_recurrence_gradient(const tensair_sequences* seq, const tensair_steps* grad, const float* grad_last, const float* marks,
                                const tensair_steps* dgate, const tensair_steps* dvalue, float* dstate, void* stream) {
    const int rc = check_sequences(seq);
    if (rc != TENSAIR_OK) return rc;
    TENSAIR_REQUIRE((uintptr_t)grad_last % 4 == 0 && (uintptr_t)dstate % 4 == 0 && (uintptr_t)marks % 4 == 0, "grad_last, dstate or marks: not aligned");
    TENSAIR_REQUIRE(!dstate || grad_last != dstate, "dstate: may not be grad_last");
    if (!seq->B || !seq->T) return pass_on(*seq, grad_last, dstate, stream);
    TENSAIR_REQUIRE(grad && fits(*grad, *seq, false), "grad: NULL, alignment or strides");
    TENSAIR_REQUIRE(dgate && fits(*dgate, *seq, true) && dvalue && fits(*dvalue, *seq, true), "dgate or dvalue: NULL, alignment or strides");
    TENSAIR_REQUIRE(marks, "marks: NULL");
    const int sms = multiprocessors();
    if (!sms) return refuse(TENSAIR_ECUDA, "no CUDA device is current");
    RecurrenceArgs a = args_of(*seq);
    a.out = view_of(*grad);
    a.dgate = view_of(*dgate);
    a.dvalue = view_of(*dvalue);
    a.state = grad_last;
    a.last = dstate;
    a.marks = const_cast<float*>(marks);
    return launched(launch_recurrence_gradient((cudaStream_t)stream, a, sms));
}

int tensair_recurrence_step(const tensair_sequences* seq, float* state, const tensair_steps* out, void* stream) {
    const int rc = check_sequences(seq);
    if (rc != TENSAIR_OK) return rc;
    TENSAIR_REQUIRE(seq->T == 1 && !seq->lengths, "seq: one step, without lengths");
    if (!seq->B) return TENSAIR_OK;
    TENSAIR_REQUIRE(state && (uintptr_t)state % 4 == 0, "state: NULL or not aligned");
    TENSAIR_REQUIRE(out && fits(*out, *seq, true), "out: NULL, alignment or strides");
    RecurrenceArgs a = args_of(*seq);
    a.out = view_of(*out);
    a.state = state;
    a.last = state;
    return launched(launch_recurrence_step((cudaStream_t)stream, a));
}

int tensair_sample(const tensair_draw* h, const tensair_rows* logits, void* stream) {
    TENSAIR_REQUIRE(h, "draw: NULL");
    TENSAIR_REQUIRE(h->n <= (1ull << 24), "draw: n must be at most 2^24");
    TENSAIR_REQUIRE(logits && logits->d >= 1 && logits->d <= kMaxWidth, "logits: NULL, or d not in 1 .. 2^20");
    const int rc = check_rows(logits, logits->d, h->n == 0, "logits: NULL", "logits: type, stride or alignment");
    if (rc != TENSAIR_OK) return rc;
    TENSAIR_REQUIRE(h->temperatures || std::isfinite(h->temperature), "draw: temperature must be finite");
    TENSAIR_REQUIRE(h->top_ps || !std::isnan(h->top_p), "draw: top_p is NaN");
    TENSAIR_REQUIRE(h->min_ps || !std::isnan(h->min_p), "draw: min_p is NaN");
    TENSAIR_REQUIRE((!h->n || (h->uniform && h->token)) && (uintptr_t)h->uniform % 4 == 0 && (uintptr_t)h->token % 8 == 0 && (uintptr_t)h->logprob % 4 == 0,
                    "draw: uniform or token is NULL, or a pointer not aligned to its type");
    TENSAIR_REQUIRE(((uintptr_t)h->temperatures | (uintptr_t)h->top_ps | (uintptr_t)h->min_ps | (uintptr_t)h->top_ks) % 4 == 0,
                    "draw: a setting is not aligned to its type");
    if (!h->n) return TENSAIR_OK;
    const int sms = multiprocessors();
    if (!sms) return refuse(TENSAIR_ECUDA, "no CUDA device is current");
    SampleArgs a = {};
    a.logits = tensair::view_of(*logits);
    a.uniform = h->uniform;
    a.token = h->token;
    a.logprob = h->logprob;
    a.temperature = {h->temperatures, h->temperature};
    a.top_p = {h->top_ps, h->top_p};
    a.min_p = {h->min_ps, h->min_p};
    a.top_k = {h->top_ks, h->top_k};
    a.n = (uint32_t)h->n;
    a.V = logits->d;
    uint32_t bits = 0;
    while ((a.V - 1) >> bits) ++bits;
    a.bits = 62 - bits < 46 ? 62 - bits : 46;
    return launched(launch_sample((cudaStream_t)stream, a, sms));
}

}  // extern "C"
