// gem_ops.cpp -- the C ABI of the worker's operators: handles and argument
// checks.  Kernels live in gem_logits.hip and gem_scan.hip.
#include <hip/hip_runtime.h>

#include <cmath>
#include <new>

#include "gem_ops.hpp"

struct gem_ops_handle {
    hipStream_t stream = nullptr;
    void* memory = nullptr;
    gemk::OpsDevice dev{};
};

namespace {

#define OPS_HIP(expr)                                                 \
    do {                                                              \
        const hipError_t e_ = (expr);                                 \
        if (e_ != hipSuccess) {                                       \
            gemk::note_hip_error("gem_ops.cpp", #expr, e_, __LINE__); \
            return GEM_EHIP;                                          \
        }                                                             \
    } while (0)

// Most rows of logits (a launch of a block a row stays within the 2^32 threads of a
// dispatch), and the largest row stride in elements: products of these, of
// GEM_TOKENS_MAX and of elements' sizes stay within 63 bits.
constexpr int64_t kRowsMax = int64_t{1} << 22;
constexpr int64_t kStrideMax = int64_t{1} << 28;

bool aligned(const void* p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }

size_t element(int32_t dtype) { return dtype == GEM_BF16 ? 2 : 4; }

// A row stride as given (0: `width`); false if out of range.
bool row_stride(int64_t given, int64_t width, int64_t* out)
{
    *out = given ? given : width;
    return *out >= width && *out <= kStrideMax;
}

int check_logits(const gem_logits* z, gemk::LogitArgs* l)
{
    if (!z) return GEM_EINVAL;
    if (z->dtype != GEM_F32 && z->dtype != GEM_BF16) return GEM_EDTYPE;
    if (z->rows < 0 || z->rows > kRowsMax || z->vocab < 1 || z->vocab > GEM_VOCAB_MAX)
        return GEM_EINVAL;
    if (!std::isfinite(z->temperature) || !(z->temperature > 0.0f)) return GEM_EINVAL;
    const double scale = 1.4426950408889634074 / static_cast<double>(z->temperature);
    const double inv_t = 1.0 / static_cast<double>(z->temperature);
    l->scale = static_cast<float>(scale);
    l->inv_t = static_cast<float>(inv_t);
    // A temperature whose reciprocal leaves binary32 has no scores.
    if (!std::isfinite(l->scale) || !std::isnormal(l->inv_t)) return GEM_EINVAL;
    if (!row_stride(z->stride, z->vocab, &l->stride)) return GEM_EINVAL;
    if (z->rows > 0 && !z->data) return GEM_EINVAL;
    if (!aligned(z->data, element(z->dtype))) return GEM_EALIGN;
    l->z = z->data;
    l->rows = z->rows;
    l->vocab = z->vocab;
    return GEM_OK;
}

int check_scan(const gem_scan* s, gem_scan* out)
{
    if (!s) return GEM_EINVAL;
    if (s->dtype != GEM_F32 && s->dtype != GEM_BF16) return GEM_EDTYPE;
    if (s->tokens < 0 || s->tokens > GEM_TOKENS_MAX || s->channels < 1 || s->sequences < 1)
        return GEM_EINVAL;
    *out = *s;
    if (!row_stride(s->x_stride, s->channels, &out->x_stride)) return GEM_EINVAL;
    if (!row_stride(s->gate_stride, s->channels, &out->gate_stride)) return GEM_EINVAL;
    if (!s->offsets && s->tokens % s->sequences != 0) return GEM_EINVAL;
    // A launch's threads, 32 a row, are counted in 32 bits (arrays of more rows would not fit
    // any device).
    if (gemk::scan_rows(s->tokens, s->channels) >= int64_t{1} << 27) return GEM_EINVAL;
    if (s->tokens > 0 && (!s->x || !s->gate)) return GEM_EINVAL;
    if (!aligned(s->x, element(s->dtype)) || !aligned(s->gate, element(s->dtype)) ||
        !aligned(s->offsets, 8) || !aligned(s->h0, 4))
        return GEM_EALIGN;
    return GEM_OK;
}

// One token a sequence needs no scratch.
bool single_tokens(const gem_scan& s) { return !s.offsets && s.tokens == s.sequences; }

}  // namespace

extern "C" {

int gem_ops_create(int64_t scratch_bytes, void* stream, gem_ops_t** out)
{
    if (!out || scratch_bytes < 0) return GEM_EINVAL;
    *out = nullptr;
    gem_ops_handle* o = new (std::nothrow) gem_ops_handle();
    if (!o) return GEM_ENOMEM;
    o->stream = static_cast<hipStream_t>(stream);
    const int rc = [&]() -> int {
        int device = 0;
        OPS_HIP(hipGetDevice(&device));
        OPS_HIP(hipDeviceGetAttribute(&o->dev.cus, hipDeviceAttributeMultiprocessorCount, device));
        if (scratch_bytes > INT64_MAX - gemk::kFixedScratch) return GEM_ENOMEM;
        const size_t bytes = static_cast<size_t>(scratch_bytes + gemk::kFixedScratch);
        const hipError_t e = hipMalloc(&o->memory, bytes);
        if (e != hipSuccess) {
            gemk::note_hip_error("gem_ops.cpp", "hipMalloc", e, __LINE__);
            (void)hipGetLastError();
            o->memory = nullptr;
            return GEM_ENOMEM;
        }
        char* base = static_cast<char*>(o->memory);
        o->dev.scratch = base;
        o->dev.scan = base + gemk::kFixedScratch;
        o->dev.scan_bytes = scratch_bytes;
        return GEM_OK;
    }();
    if (rc != GEM_OK) {
        (void)gem_ops_destroy(o);
        return rc;
    }
    *out = o;
    return GEM_OK;
}

int gem_ops_destroy(gem_ops_t* ops)
{
    if (!ops) return GEM_EINVAL;
    if (ops->memory) {
        (void)hipStreamSynchronize(ops->stream);
        (void)hipFree(ops->memory);
    }
    delete ops;
    return GEM_OK;
}

int gem_token_scores(gem_ops_t* ops, const gem_logits* z, const int32_t* tokens, int32_t n_tokens,
                     int32_t top_k, const gem_scores* out)
{
    if (!ops || !out) return GEM_EINVAL;
    gemk::ScoreArgs a{};
    const int rc = check_logits(z, &a.l);
    if (rc != GEM_OK) return rc;
    if (n_tokens < 0 || n_tokens > GEM_VOCAB_MAX || top_k < 0 || top_k > GEM_TOP_MAX) return GEM_EINVAL;
    if (n_tokens > 0 && !tokens && z->rows > 0) return GEM_EINVAL;
    if (!aligned(tokens, 4) || !aligned(out->logprob, 4) || !aligned(out->entropy, 4) ||
        !aligned(out->lse, 4) || !aligned(out->top_ids, 4) || !aligned(out->top_logprob, 4))
        return GEM_EALIGN;
    a.tokens = tokens;
    a.n_tokens = out->logprob ? n_tokens : 0;
    a.top_k = out->top_ids || out->top_logprob ? top_k : 0;
    a.out = *out;
    if (a.l.rows == 0) return GEM_OK;
    OPS_HIP(gemk::launch_scores(a, z->dtype == GEM_BF16, ops->dev, ops->stream));
    return GEM_OK;
}

static int distill(gem_ops_t* ops, const gem_logits* z, const gem_teacher* t, const float* weight,
                   float* loss, void* grad, int64_t grad_stride)
{
    gemk::DistillArgs a{};
    const int rc = check_logits(z, &a.l);
    if (rc != GEM_OK) return rc;
    if (!t || t->k < 1 || t->k > GEM_TOP_MAX || (t->tail != 0 && t->tail != 1)) return GEM_EINVAL;
    if (z->rows > 0 && (!t->ids || !t->logprob)) return GEM_EINVAL;
    if (!row_stride(grad_stride, z->vocab, &a.grad_stride)) return GEM_EINVAL;
    if (grad == z->data && grad && a.grad_stride != a.l.stride) return GEM_EINVAL;
    if (!aligned(t->ids, 4) || !aligned(t->logprob, 4) || !aligned(weight, 4) || !aligned(loss, 4) ||
        !aligned(grad, element(z->dtype)))
        return GEM_EALIGN;
    a.ids = t->ids;
    a.lp = t->logprob;
    a.k = t->k;
    a.tail = t->tail;
    a.weight = weight;
    a.loss = loss;
    a.grad = grad;
    if (a.l.rows == 0) return GEM_OK;
    OPS_HIP(gemk::launch_distill(a, z->dtype == GEM_BF16, ops->dev, ops->stream));
    return GEM_OK;
}

int gem_distill_loss(gem_ops_t* ops, const gem_logits* z, const gem_teacher* teacher,
                     const float* weight, float* loss)
{
    if (!ops || !z || (!loss && z->rows > 0)) return GEM_EINVAL;
    return distill(ops, z, teacher, weight, loss, nullptr, 0);
}

int gem_distill_grad(gem_ops_t* ops, const gem_logits* z, const gem_teacher* teacher,
                     const float* weight, float* loss, void* grad, int64_t grad_stride)
{
    if (!ops || !z || (!grad && z->rows > 0)) return GEM_EINVAL;
    return distill(ops, z, teacher, weight, loss, grad, grad_stride);
}

int gem_scan_scratch(int64_t tokens, int32_t channels, int64_t* bytes)
{
    if (!bytes || tokens < 0 || tokens > GEM_TOKENS_MAX || channels < 1) return GEM_EINVAL;
    *bytes = gemk::scan_scratch_bytes(tokens, channels);
    return GEM_OK;
}

int gem_scan_state_rows(int64_t tokens, int64_t* rows)
{
    if (!rows || tokens < 0 || tokens > GEM_TOKENS_MAX) return GEM_EINVAL;
    *rows = (tokens + gemk::kStateTokens - 1) / gemk::kStateTokens;
    return GEM_OK;
}

int gem_scan_forward(gem_ops_t* ops, const gem_scan* s, void* y, int64_t y_stride, float* h_last,
                     float* states)
{
    if (!ops) return GEM_EINVAL;
    gemk::ScanArgs a{};
    const int rc = check_scan(s, &a.s);
    if (rc != GEM_OK) return rc;
    if (s->tokens > 0 && !y) return GEM_EINVAL;
    if (!row_stride(y_stride, s->channels, &a.y_stride)) return GEM_EINVAL;
    if (!aligned(y, element(s->dtype)) || !aligned(h_last, 4) || !aligned(states, 4)) return GEM_EALIGN;
    a.y = y;
    a.h_last = h_last;
    a.states = states;
    if (gemk::scan_bytes(s->tokens, s->channels) > ops->dev.scan_bytes && !single_tokens(*s))
        return GEM_ESCRATCH;
    OPS_HIP(gemk::launch_scan_forward(a, s->dtype == GEM_BF16, ops->dev, ops->stream));
    return GEM_OK;
}

int gem_scan_backward(gem_ops_t* ops, const gem_scan* s, const float* states, const void* dy,
                      int64_t dy_stride, const float* dh_last, void* dx, int64_t dx_stride,
                      void* dgate, int64_t dgate_stride, float* dh0)
{
    if (!ops) return GEM_EINVAL;
    gemk::ScanBackArgs a{};
    const int rc = check_scan(s, &a.s);
    if (rc != GEM_OK) return rc;
    if (s->tokens > 0 && (!states || !dy || !dx || !dgate)) return GEM_EINVAL;
    if (!row_stride(dy_stride, s->channels, &a.dy_stride)) return GEM_EINVAL;
    if (!row_stride(dx_stride, s->channels, &a.dx_stride)) return GEM_EINVAL;
    if (!row_stride(dgate_stride, s->channels, &a.dgate_stride)) return GEM_EINVAL;
    if (!aligned(states, 4) || !aligned(dy, element(s->dtype)) || !aligned(dh_last, 4) ||
        !aligned(dx, element(s->dtype)) || !aligned(dgate, element(s->dtype)) || !aligned(dh0, 4))
        return GEM_EALIGN;
    a.states = states;
    a.dy = dy;
    a.dh_last = dh_last;
    a.dx = dx;
    a.dgate = dgate;
    a.dh0 = dh0;
    if (gemk::scan_bytes(s->tokens, s->channels) > ops->dev.scan_bytes) return GEM_ESCRATCH;
    OPS_HIP(gemk::launch_scan_backward(a, s->dtype == GEM_BF16, ops->dev, ops->stream));
    return GEM_OK;
}

}  // extern "C"
