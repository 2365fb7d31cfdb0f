// C entry points of the language-model operators: argument checks, workspace layout, launches.
#include "../../include/tensair.h"

#include <algorithm>
#include <atomic>
#include <cmath>
#include <cstdio>
#include <vector>

#include "context.h"
#include "operator_checks.h"
#include "operators.h"

using namespace tensair;

namespace {

constexpr uint64_t kMaxTokens = 1ull << 30, kMaxVocabulary = 1ull << 30;

// What the last refused or failed operator call of this thread said (these calls have no context to keep it in).
// A fixed array: setting it can neither allocate nor throw.
thread_local char last_refusal[160] = "";

int check_tokens(const tensair_tokens* t) {
    TENSAIR_REQUIRE(t, "tokens: NULL");
    TENSAIR_REQUIRE(t->V >= 1 && t->V <= kMaxVocabulary, "tokens: V must be 1 .. 2^30");
    TENSAIR_REQUIRE(t->n <= kMaxTokens, "tokens: n must be at most 2^30");
    TENSAIR_REQUIRE(t->type == TENSAIR_INT32 || t->type == TENSAIR_INT64, "tokens: ids must be TENSAIR_INT32 or TENSAIR_INT64");
    TENSAIR_REQUIRE(!t->n || t->ids, "tokens: ids are NULL");
    TENSAIR_REQUIRE((uintptr_t)t->ids % (t->type == TENSAIR_INT64 ? 8 : 4) == 0, "tokens: ids are not aligned to their type");
    TENSAIR_REQUIRE((uintptr_t)t->error % 4 == 0, "tokens: the error word is not aligned");
    return TENSAIR_OK;
}

}  // namespace

namespace tensair {

int refuse(int code, const char* why) {
    std::snprintf(last_refusal, sizeof(last_refusal), "%s", why);
    return code;
}
int launched(cudaError_t e) {
    if (e == cudaSuccess) return TENSAIR_OK;
    return refuse(TENSAIR_ECUDA, cudaGetErrorString(e));
}

int check_rows(const tensair_rows* r, uint32_t d, bool empty, const char* null, const char* bad) {
    TENSAIR_REQUIRE(r && (empty || r->data), null);
    TENSAIR_REQUIRE(is_float_type(r->type) && r->d == d && (empty || (r->stride >= d && r->stride <= kMaxStride)) &&
                    (uintptr_t)r->data % type_bytes(r->type) == 0, bad);
    return TENSAIR_OK;
}

int multiprocessors() {
    static std::atomic<int> known[kMaxDevices];
    int device = 0;
    if (cudaGetDevice(&device) != cudaSuccess) return 0;
    int sms = device < kMaxDevices ? known[device].load(std::memory_order_relaxed) : 0;
    if (!sms) {
        if (cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, device) != cudaSuccess) return 0;
        if (device < kMaxDevices) known[device].store(sms, std::memory_order_relaxed);
    }
    return sms;
}

}  // namespace tensair

namespace {

TokenIds tokens_of(const tensair_tokens& t) {
    return TokenIds{t.ids, t.padding_id, t.error, (uint32_t)t.n, (uint32_t)t.V, t.type == TENSAIR_INT64};
}

// The workspace of the gradient calls for a batch of n tokens.
struct Layout {
    uint64_t key, pos, seg_start, span_rank, info, large, partials, items_a, items_b, hist, tile_counts, total;
    uint32_t partial_stride;
};
Layout layout_of(uint32_t n, uint32_t V, uint32_t d) {
    Layout l;
    const uint64_t windows = ((uint64_t)n + kWindow - 1) / kWindow;
    l.partial_stride = (uint32_t)round_up(d, 4);
    uint64_t off = 0;
    auto take = [&off](uint64_t bytes) { const uint64_t at = off; off = round_up(off + bytes, 256); return at; };
    l.info = take(16);
    l.key = take((uint64_t)n * 4);
    l.pos = take((uint64_t)n * 4);
    l.seg_start = take(((uint64_t)(n < V ? n : V) + 1) * 4);
    l.span_rank = take(((uint64_t)n + kSpan - 1) / kSpan * 4);
    l.large = take((uint64_t)(n / (kWindow + 1)) * sizeof(uint4));
    l.partials = take(windows * 2 * l.partial_stride * 4);
    // the sort's needs change with the length class: a workspace takes the largest of what shorter batches need
    SortScratchBytes s = sort_scratch_bytes(n);
    const SortScratchBytes shorter = sort_scratch_bytes(n < kTiledSort ? n : kTiledSort);
    s.hist = std::max(s.hist, shorter.hist);
    s.tile_counts = std::max(s.tile_counts, shorter.tile_counts);
    l.items_a = take(s.items);
    l.items_b = take(s.items);
    l.hist = take(s.hist);
    l.tile_counts = take(s.tile_counts);
    l.total = off;
    return l;
}

// The part all gradient calls share: checks, workspace, sort, sums.
int gradient_call(const tensair_tokens* tokens, const tensair_rows* grad, float scale, void* workspace, uint64_t bytes,
                  void* stream, SumKind kind, SumArgs& a, uint32_t d, const ClearRows& clear = ClearRows{}) {
    TENSAIR_REQUIRE(std::isfinite(scale), "scale is not finite");
    const int rc = check_rows(grad, d, tokens->n == 0, "grad: NULL", "grad: type, width, stride or alignment");
    if (rc != TENSAIR_OK) return rc;
    const uint32_t n = (uint32_t)tokens->n, V = (uint32_t)tokens->V;
    const Layout l = layout_of(n, V, d);
    if (n) {
        TENSAIR_REQUIRE(workspace && (uintptr_t)workspace % 256 == 0, "workspace: NULL or not aligned to 256 bytes");
        if (bytes < l.total) return refuse(TENSAIR_ENOMEM, "workspace: smaller than tensair_embedding_workspace_bytes says");
    }
    const int sms = multiprocessors();
    if (!sms) return refuse(TENSAIR_ECUDA, "no CUDA device is current");
    if (!n) return clear.rows ? launched(launch_clear((cudaStream_t)stream, clear, sms)) : TENSAIR_OK;
    a.grad = view_of(*grad);
    a.n = n;
    a.V = V;
    a.d = d;
    a.scale = scale;
    if (is_short(n)) {
        cudaError_t e = clear.rows ? launch_clear((cudaStream_t)stream, clear, sms) : cudaSuccess;
        if (e == cudaSuccess) e = launch_short_sums((cudaStream_t)stream, kind, a, tokens_of(*tokens), sms);
        return launched(e);
    }
    uint8_t* w = (uint8_t*)workspace;
    a.s = SortedTokens{(uint32_t*)(w + l.key), (uint32_t*)(w + l.pos), (uint32_t*)(w + l.seg_start),
                       (uint32_t*)(w + l.span_rank), (uint32_t*)(w + l.info), tokens->error};
    a.partials = (float*)(w + l.partials);
    a.partial_stride = l.partial_stride;
    a.large = (uint4*)(w + l.large);
    const SortScratch scratch{(item_t*)(w + l.items_a), (item_t*)(w + l.items_b), (uint32_t*)(w + l.hist),
                              (uint32_t*)(w + l.tile_counts)};
    cudaError_t e = launch_token_sort((cudaStream_t)stream, tokens_of(*tokens), a.s, scratch, clear, sms);
    if (e == cudaSuccess) e = launch_token_sums((cudaStream_t)stream, kind, a, sms);
    return launched(e);
}

int check_adamw(const tensair_adamw* h) {
    TENSAIR_REQUIRE(h, "adamw: NULL");
    TENSAIR_REQUIRE(std::isfinite(h->lr) && h->lr >= 0, "adamw: lr must be finite and not negative");
    TENSAIR_REQUIRE(h->beta1 >= 0 && h->beta1 < 1 && h->beta2 >= 0 && h->beta2 < 1, "adamw: beta1 and beta2 must be in [0,1)");
    TENSAIR_REQUIRE(std::isfinite(h->eps) && h->eps >= 0, "adamw: eps must be finite and not negative");
    TENSAIR_REQUIRE(std::isfinite(h->weight_decay) && h->weight_decay >= 0, "adamw: weight_decay must be finite and not negative");
    TENSAIR_REQUIRE(h->step >= 1 && h->step < (1ull << 56), "adamw: step counts from 1");
    TENSAIR_REQUIRE((uintptr_t)h->grad_scale % 4 == 0, "adamw: grad_scale is not aligned");
    return TENSAIR_OK;
}

AdamwConsts consts_of(const tensair_adamw& h) {
    AdamwConsts c;
    c.beta1 = (float)h.beta1;
    c.rest1 = (float)(1 - h.beta1);
    c.beta2 = (float)h.beta2;
    c.rest2 = (float)(1 - h.beta2);
    c.eps = (float)h.eps;
    c.inv_root2 = (float)(1 / std::sqrt(1 - std::pow(h.beta2, (double)h.step)));
    c.step_size = (float)(h.lr / (1 - std::pow(h.beta1, (double)h.step)));
    c.keep = (float)(1 - h.lr * h.weight_decay);
    c.grad_scale = h.grad_scale;
    return c;
}

}  // namespace

namespace tensair {
const char* operator_error() { return last_refusal; }
}  // namespace tensair

extern "C" {

int tensair_embedding_lookup(const tensair_tokens* tokens, const tensair_rows* table, const tensair_rows* out, float scale,
                             void* stream) {
    int rc = check_tokens(tokens);
    if (rc != TENSAIR_OK) return rc;
    TENSAIR_REQUIRE(table && table->d >= 1 && table->d <= kMaxWidth, "table: NULL, or d not in 1 .. 2^20");
    rc = check_rows(table, table->d, false, "table: NULL", "table: type, stride or alignment");
    if (rc == TENSAIR_OK) rc = check_rows(out, table->d, tokens->n == 0, "out: NULL", "out: type, width, stride or alignment");
    if (rc != TENSAIR_OK) return rc;
    if (!tokens->n) return TENSAIR_OK;
    return launched(launch_lookup((cudaStream_t)stream, tokens_of(*tokens), view_of(*table), view_of(*out), table->d, scale));
}

int tensair_embedding_workspace_bytes(uint64_t n, uint64_t V, uint32_t d, uint64_t* bytes) {
    TENSAIR_REQUIRE(bytes, "bytes: NULL");
    TENSAIR_REQUIRE(n <= kMaxTokens && V >= 1 && V <= kMaxVocabulary && d >= 1 && d <= kMaxWidth, "n, V or d out of range");
    *bytes = layout_of((uint32_t)n, (uint32_t)V, d).total;
    return TENSAIR_OK;
}

int tensair_embedding_gradient(const tensair_tokens* tokens, const tensair_rows* grad, const tensair_rows* out, float scale,
                               int accumulate, void* workspace, uint64_t workspace_bytes, void* stream) {
    int rc = check_tokens(tokens);
    if (rc != TENSAIR_OK) return rc;
    TENSAIR_REQUIRE(out && out->d >= 1 && out->d <= kMaxWidth, "out: NULL, or d not in 1 .. 2^20");
    rc = check_rows(out, out->d, false, "out: NULL", "out: type, stride or alignment");
    if (rc != TENSAIR_OK) return rc;
    SumArgs a = {};
    a.out = view_of(*out);
    a.accumulate = accumulate != 0;
    const uint64_t b = type_bytes(out->type);
    const ClearRows clear{(uint8_t*)out->data, out->stride * b, out->d * b, accumulate ? 0 : tokens->V};
    return gradient_call(tokens, grad, scale, workspace, workspace_bytes, stream, kSumTable, a, out->d, clear);
}

int tensair_embedding_gradient_rows(const tensair_tokens* tokens, const tensair_rows* grad, float scale, uint32_t* row_ids,
                                    const tensair_rows* rows, uint32_t* count, void* workspace, uint64_t workspace_bytes,
                                    void* stream) {
    int rc = check_tokens(tokens);
    if (rc != TENSAIR_OK) return rc;
    TENSAIR_REQUIRE(rows && rows->d >= 1 && rows->d <= kMaxWidth, "rows: NULL, or d not in 1 .. 2^20");
    rc = check_rows(rows, rows->d, tokens->n == 0, "rows: NULL", "rows: type, stride or alignment");
    if (rc != TENSAIR_OK) return rc;
    TENSAIR_REQUIRE(rows->type == TENSAIR_FLOAT32, "rows: must be TENSAIR_FLOAT32");
    TENSAIR_REQUIRE(count && (uintptr_t)count % 4 == 0, "count: NULL or not aligned");
    TENSAIR_REQUIRE((!tokens->n || row_ids) && (uintptr_t)row_ids % 4 == 0, "row_ids: NULL or not aligned");
    SumArgs a = {};
    a.out = view_of(*rows);
    a.out_ids = row_ids;
    a.out_count = count;
    if (!tokens->n) return launched(cudaMemsetAsync(count, 0, 4, (cudaStream_t)stream));
    return gradient_call(tokens, grad, scale, workspace, workspace_bytes, stream, kSumRows, a, rows->d);
}

int tensair_embedding_adamw(const tensair_tokens* tokens, const tensair_rows* grad, float scale, const tensair_rows* table,
                            const tensair_rows* m, const tensair_rows* v, const tensair_adamw* adamw, void* workspace,
                            uint64_t workspace_bytes, void* stream) {
    int rc = check_tokens(tokens);
    if (rc == TENSAIR_OK) rc = check_adamw(adamw);
    if (rc != TENSAIR_OK) return rc;
    TENSAIR_REQUIRE(table && table->d >= 1 && table->d <= kMaxWidth, "table: NULL, or d not in 1 .. 2^20");
    rc = check_rows(table, table->d, false, "table: NULL", "table: type, stride or alignment");
    if (rc == TENSAIR_OK) rc = check_rows(m, table->d, false, "m: NULL", "m: type, width, stride or alignment");
    if (rc == TENSAIR_OK) rc = check_rows(v, table->d, false, "v: NULL", "v: type, width, stride or alignment");
    if (rc != TENSAIR_OK) return rc;
    TENSAIR_REQUIRE(m->type == TENSAIR_FLOAT32 && v->type == TENSAIR_FLOAT32, "m and v must be TENSAIR_FLOAT32");
    SumArgs a = {};
    a.out = view_of(*table);
    a.m = (float*)m->data;
    a.v = (float*)v->data;
    a.m_stride = (uint32_t)m->stride;
    a.v_stride = (uint32_t)v->stride;
    a.adamw = consts_of(*adamw);
    return gradient_call(tokens, grad, scale, workspace, workspace_bytes, stream, kSumAdamw, a, table->d);
}

int tensair_adamw_step(const tensair_adamw_tensor* tensors, uint64_t count, uint32_t state_bits, const tensair_adamw* adamw,
                       void* stream) {
    const int rc = check_adamw(adamw);
    if (rc != TENSAIR_OK) return rc;
    TENSAIR_REQUIRE(state_bits == 32 || state_bits == 8, "state_bits must be 32 or 8");
    TENSAIR_REQUIRE(!count || tensors, "tensors: NULL");
    TENSAIR_REQUIRE(count < (1ull << 31), "tensors: too many");
    const AdamwConsts c = consts_of(*adamw);
    try {
        std::vector<AdamwTensor> list;
        list.reserve(count);
        uint64_t block0 = 0;
        for (uint64_t i = 0; i < count; ++i) {
            const tensair_adamw_tensor& t = tensors[i];
            TENSAIR_REQUIRE(t.n < (1ull << 40), "tensors: n must be below 2^40");
            const uint64_t place = block0;
            block0 += (t.n + 255) / 256;
            if (t.skip) continue;
            TENSAIR_REQUIRE(is_float_type(t.param_type) && is_float_type(t.grad_type), "tensors: param_type or grad_type");
            TENSAIR_REQUIRE(!t.copy || t.copy_type == TENSAIR_BFLOAT16 || t.copy_type == TENSAIR_FLOAT16,
                            "tensors: a copy must be TENSAIR_BFLOAT16 or TENSAIR_FLOAT16");
            TENSAIR_REQUIRE(std::isfinite(t.lr_factor) && t.lr_factor >= 0 && std::isfinite(t.decay_factor) && t.decay_factor >= 0,
                            "tensors: lr_factor and decay_factor must be finite and not negative");
            if (!t.n) continue;
            TENSAIR_REQUIRE(t.param && t.grad && t.m && t.v, "tensors: param, grad, m or v is NULL");
            TENSAIR_REQUIRE(state_bits == 32 || (t.m_scale && t.v_scale), "tensors: 8-bit moments need m_scale and v_scale");
            TENSAIR_REQUIRE((uintptr_t)t.param % type_bytes(t.param_type) == 0 && (uintptr_t)t.grad % type_bytes(t.grad_type) == 0 &&
                            (state_bits == 8 || ((uintptr_t)t.m % 4 == 0 && (uintptr_t)t.v % 4 == 0)) &&
                            (uintptr_t)t.m_scale % 4 == 0 && (uintptr_t)t.v_scale % 4 == 0 && (uintptr_t)t.copy % 2 == 0,
                            "tensors: a pointer is not aligned to its type");
            list.push_back(AdamwTensor{t.param, t.grad, t.m, t.v, t.m_scale, t.v_scale, t.copy, t.n, place,
                                       (float)(c.step_size * t.lr_factor),
                                       (float)(1 - adamw->lr * t.lr_factor * adamw->weight_decay * t.decay_factor),
                                       t.param_type, t.grad_type, t.copy_type});
        }
        if (list.empty()) return TENSAIR_OK;
        if (state_bits == 8) {
            cudaStreamCaptureStatus status = cudaStreamCaptureStatusNone;
            const cudaError_t e = cudaStreamIsCapturing((cudaStream_t)stream, &status);
            if (e != cudaSuccess) return launched(e);
            TENSAIR_REQUIRE(status == cudaStreamCaptureStatusNone,
                            "a step with 8-bit moments cannot be captured: replays would repeat its random bits");
        }
        const int sms = multiprocessors();
        if (!sms) return refuse(TENSAIR_ECUDA, "no CUDA device is current");
        return launched(launch_adamw((cudaStream_t)stream, list.data(), (uint32_t)list.size(), (int)state_bits, c, adamw->step,
                                     adamw->seed, sms));
    } catch (...) {      // the list could not be had
        return refuse(TENSAIR_ENOMEM, "out of host memory");
    }
}

}  // extern "C"
