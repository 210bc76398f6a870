// Host side of what closes a policy update: the draw from given numbers, the gradient of the objective, the optimiser's step.
#include <algorithm>
#include <cmath>
#include <memory>
#include <new>

#include "host_checks.h"

using namespace spiral;

// ---------------------------------------------------------------------------------------------
// draw
// ---------------------------------------------------------------------------------------------
extern "C" size_t spiral_sample_uniform_workspace_bytes(int B, int V) {
    if (B < 1 || B > SPIRAL_MAX_BATCH || V < 1) return 0;
    return draw_workspace_bytes(B, V);
}

extern "C" int spiral_sample_uniform(const void* dev_logits, int logits_dtype, long long row_stride, int B, int V,
                                     const float* host_temperature, const int32_t* host_top_k, const float* host_top_p,
                                     const float* host_min_p, const float* dev_uniform, void* dev_workspace, size_t workspace_bytes,
                                     int32_t* dev_out_tokens, float* dev_out_logp, void* stream) {
    if (!dev_logits || !dev_uniform || !dev_out_tokens) return fail(SPIRAL_ERR_INVALID_ARG, "sample_uniform: null logits, numbers or output");
    if (B < 1 || B > SPIRAL_MAX_BATCH || V < 1) return fail(SPIRAL_ERR_INVALID_ARG, "sample_uniform: bad B=%d or V=%d", B, V);
    const int size = dtype_size(logits_dtype);
    if (!size) return fail(SPIRAL_ERR_INVALID_ARG, "sample_uniform: unknown logits type %d", logits_dtype);
    if (row_stride < V) return fail(SPIRAL_ERR_INVALID_ARG, "sample_uniform: row stride %lld is less than V=%d", row_stride, V);
    if (!aligned(dev_logits, size) || !aligned(dev_uniform, 4) || !aligned(dev_out_tokens, 4) || !aligned(dev_out_logp, 4))
        return fail(SPIRAL_ERR_INVALID_ARG, "sample_uniform: misaligned buffer");
    if (!dev_workspace || !aligned(dev_workspace, 256)) return fail(SPIRAL_ERR_INVALID_ARG, "sample_uniform: workspace is null or not 256-byte aligned");
    const size_t need = draw_workspace_bytes(B, V);
    if (workspace_bytes < need) return fail(SPIRAL_ERR_INVALID_ARG, "sample_uniform: workspace of %zu bytes, %zu needed", workspace_bytes, need);
    for (int i = 0; i < B; ++i) {
        if (host_temperature && (!(host_temperature[i] >= 0.f) || !std::isfinite(host_temperature[i])))
            return fail(SPIRAL_ERR_INVALID_ARG, "sample_uniform: temperature of row %d must be finite and >= 0", i);
        if (host_top_p && !(host_top_p[i] > 0.f && host_top_p[i] <= 1.f))
            return fail(SPIRAL_ERR_INVALID_ARG, "sample_uniform: top_p of row %d must be in (0, 1] (1 disables)", i);
        if (host_min_p && !(host_min_p[i] >= 0.f && host_min_p[i] <= 1.f))
            return fail(SPIRAL_ERR_INVALID_ARG, "sample_uniform: min_p of row %d must be in [0, 1] (0 disables)", i);
    }
    const size_t per_row = (size_t)B * 4;
    const Span spans[] = {span_of(dev_logits, matrix_bytes(B, row_stride, V, size), false), span_of(dev_uniform, per_row, false),
                          span_of(dev_out_tokens, per_row, true), span_of(dev_out_logp, per_row, true), span_of(dev_workspace, need, true)};
    if (any_overlap(spans, 5)) return fail(SPIRAL_ERR_INVALID_ARG, "sample_uniform: a buffer that is written overlaps another");
    DrawArgs a = {};
    a.logits = dev_logits; a.row_stride = row_stride; a.B = B; a.V = V;
    a.uniform = dev_uniform; a.tokens = dev_out_tokens; a.logp = dev_out_logp;
    return done(launch_draw(a, logits_dtype, host_temperature, host_top_k, host_top_p, host_min_p, dev_workspace, (hipStream_t)stream), "sample_uniform");
}

// ---------------------------------------------------------------------------------------------
// policy gradient
// ---------------------------------------------------------------------------------------------
extern "C" size_t spiral_policy_gradient_workspace_bytes(long long n_rows, int V) {
    if (n_rows < 1 || n_rows > 0x7FFFFFFFll || V < 1) return 0;
    return policy_grad_workspace_bytes(n_rows, V);
}

extern "C" int spiral_policy_gradient(const void* dev_logits, int dtype, long long row_stride, long long n_rows, int V,
                                      const int32_t* dev_targets, const float* dev_logp_old, const float* dev_advantage,
                                      const int32_t* dev_mask, float temperature, float clip_eps, float scale, float* dev_logp,
                                      void* dev_grad, long long grad_stride, void* dev_workspace, size_t workspace_bytes, void* stream) {
    if (!dev_logits || !dev_targets || !dev_advantage || !dev_logp || !dev_grad) return fail(SPIRAL_ERR_INVALID_ARG, "policy_gradient: null pointer");
    if (n_rows < 1 || n_rows > 0x7FFFFFFFll || V < 1) return fail(SPIRAL_ERR_INVALID_ARG, "policy_gradient: bad n_rows=%lld or V=%d", n_rows, V);
    const int size = dtype_size(dtype);
    if (!size) return fail(SPIRAL_ERR_INVALID_ARG, "policy_gradient: unknown type %d", dtype);
    if (row_stride < V || grad_stride < V) return fail(SPIRAL_ERR_INVALID_ARG, "policy_gradient: a row stride is less than V=%d", V);
    if (!aligned(dev_logits, size) || !aligned(dev_grad, size) || !aligned(dev_targets, 4) || !aligned(dev_logp_old, 4) ||
        !aligned(dev_advantage, 4) || !aligned(dev_mask, 4) || !aligned(dev_logp, 4))
        return fail(SPIRAL_ERR_INVALID_ARG, "policy_gradient: misaligned buffer");
    if (!(temperature >= 1e-30f) || !std::isfinite(temperature)) return fail(SPIRAL_ERR_INVALID_ARG, "policy_gradient: temperature must be finite and at least 1e-30");
    if (!(clip_eps >= 0.f) || !std::isfinite(clip_eps) || !std::isfinite(scale)) return fail(SPIRAL_ERR_INVALID_ARG, "policy_gradient: bad clip parameter or scale");
    const size_t in_bytes = matrix_bytes(n_rows, row_stride, V, size), out_bytes = matrix_bytes(n_rows, grad_stride, V, size), per_row = (size_t)n_rows * 4;
    const bool in_place = dev_grad == dev_logits && row_stride == grad_stride;
    const Span matrices[] = {span_of(dev_logits, in_bytes, false), span_of(dev_grad, out_bytes, true)};
    if (!in_place && any_overlap(matrices, 2)) return fail(SPIRAL_ERR_INVALID_ARG, "policy_gradient: the gradient overlaps the logits without being in place");
    const size_t need = policy_grad_workspace_bytes(n_rows, V);
    if (!dev_workspace || !aligned(dev_workspace, 256)) return fail(SPIRAL_ERR_INVALID_ARG, "policy_gradient: workspace is null or not 256-byte aligned");
    if (workspace_bytes < need) return fail(SPIRAL_ERR_INVALID_ARG, "policy_gradient: workspace of %zu bytes, %zu needed", workspace_bytes, need);
    const Span spans[] = {span_of(in_place ? nullptr : dev_logits, in_bytes, false), span_of(dev_grad, out_bytes, true), span_of(dev_targets, per_row, false),
                          span_of(dev_logp_old, per_row, false), span_of(dev_advantage, per_row, false), span_of(dev_mask, per_row, false),
                          span_of(dev_logp, per_row, true), span_of(dev_workspace, need, true)};
    if (any_overlap(spans, 8)) return fail(SPIRAL_ERR_INVALID_ARG, "policy_gradient: a buffer that is written overlaps another");
    GradArgs a = {};
    a.logits = dev_logits; a.row_stride = row_stride; a.grad = dev_grad; a.grad_stride = grad_stride;
    a.n_rows = n_rows; a.V = V;
    a.targets = dev_targets; a.logp_old = dev_logp_old; a.advantage = dev_advantage; a.mask = dev_mask;
    a.inv_t = 1.f / temperature; a.clip_eps = clip_eps; a.unit = (double)scale / temperature; a.logp = dev_logp;
    return done(launch_policy_grad(a, dtype, dev_workspace, (hipStream_t)stream), "policy_gradient");
}

// ---------------------------------------------------------------------------------------------
// AdamW
// ---------------------------------------------------------------------------------------------
struct spiral_adamw {
    int n = 0, steps = 0;
    long long chunks = 0;
    std::unique_ptr<AdamwRec[]> table;      // what the device holds a copy of
    std::unique_ptr<Span[]> written;        // [n_written], in order and apart from each other: what a step writes
    size_t n_written = 0;
    char* mem = nullptr;
};

static size_t adamw_table_bytes(int n) { return ((size_t)n * sizeof(AdamwRec) + 255) & ~(size_t)255; }
static int adamw_upload(const spiral_adamw* o, void* stream, const char* who) {
    static_assert(sizeof(AdamwRec) % 4 == 0, "uploaded as 32-bit words");
    for (int t = 0; t < o->n; t += 1024) {                       // sizes of launch_upload are ints
        const int m = std::min(1024, o->n - t);
        const hipError_t e = launch_upload((int32_t*)(o->mem + (size_t)t * sizeof(AdamwRec)), (const int32_t*)&o->table[t], (int)(m * sizeof(AdamwRec) / 4),
                                           (hipStream_t)stream);
        if (e != hipSuccess) return done(e, who);
    }
    return SPIRAL_OK;
}

extern "C" size_t spiral_adamw_bytes(int n_tensors) {
    return n_tensors < 1 ? 0 : adamw_table_bytes(n_tensors) + kAdamwParts * sizeof(double);
}

extern "C" int spiral_adamw_create(const spiral_adamw_tensor* host_tensors, int n_tensors, void* dev_mem, size_t bytes, void* stream,
                                   spiral_adamw** out) {
    if (!out) return fail(SPIRAL_ERR_INVALID_ARG, "adamw_create: null out");
    *out = nullptr;
    if (!host_tensors || n_tensors < 1) return fail(SPIRAL_ERR_INVALID_ARG, "adamw_create: no tensors");
    if (!dev_mem || !aligned(dev_mem, 256) || bytes < spiral_adamw_bytes(n_tensors))
        return fail(SPIRAL_ERR_INVALID_ARG, "adamw_create: memory is null, not 256-byte aligned or less than %zu bytes", spiral_adamw_bytes(n_tensors));
    std::unique_ptr<spiral_adamw> o(new (std::nothrow) spiral_adamw());
    const size_t most = (size_t)n_tensors * 7 + 1;
    std::unique_ptr<Span[]> spans(new (std::nothrow) Span[most]);
    if (o) o->table.reset(new (std::nothrow) AdamwRec[n_tensors]);
    if (!o || !o->table || !spans) return fail(SPIRAL_ERR_INVALID_ARG, "adamw_create: out of host memory");
    size_t n_spans = 0;
    auto span = [&](const void* p, long long n, int size, bool written) {
        if (p) spans[n_spans++] = {(uintptr_t)p, (uintptr_t)p + (uintptr_t)n * size, written};
    };
    span(dev_mem, (long long)spiral_adamw_bytes(n_tensors), 1, true);
    long long elements = 0, chunks = 0;
    for (int t = 0; t < n_tensors; ++t) {
        const spiral_adamw_tensor& x = host_tensors[t];
        const int ps = dtype_size(x.param_dtype), gs = dtype_size(x.grad_dtype);
        const bool codes = x.state_dtype == SPIRAL_DTYPE_E4M3;
        if (!ps || !gs || !(codes || x.state_dtype == SPIRAL_DTYPE_FP32)) return fail(SPIRAL_ERR_INVALID_ARG, "adamw_create: tensor %d: unknown type", t);
        if (x.n < 1 || x.n > (1ll << 48)) return fail(SPIRAL_ERR_INVALID_ARG, "adamw_create: tensor %d: %lld elements", t, x.n);
        if (!x.dev_param || !x.dev_grad || !x.dev_m || !x.dev_v) return fail(SPIRAL_ERR_INVALID_ARG, "adamw_create: tensor %d: null pointer", t);
        if (x.dev_master && x.param_dtype == SPIRAL_DTYPE_FP32) return fail(SPIRAL_ERR_INVALID_ARG, "adamw_create: tensor %d: an fp32 parameter has no master", t);
        if (codes != (x.dev_m_scale != nullptr) || codes != (x.dev_v_scale != nullptr))
            return fail(SPIRAL_ERR_INVALID_ARG, "adamw_create: tensor %d: scales go with 8-bit states", t);
        if (x.decay != 0 && x.decay != 1) return fail(SPIRAL_ERR_INVALID_ARG, "adamw_create: tensor %d: decay is 0 or 1", t);
        const int ss = codes ? 1 : 4;
        if (!aligned(x.dev_param, ps) || !aligned(x.dev_grad, gs) || !aligned(x.dev_master, 4) || !aligned(x.dev_m, ss) || !aligned(x.dev_v, ss) ||
            !aligned(x.dev_m_scale, 4) || !aligned(x.dev_v_scale, 4))
            return fail(SPIRAL_ERR_INVALID_ARG, "adamw_create: tensor %d: misaligned pointer", t);
        const long long blocks = (x.n + kAdamwBlock - 1) / kAdamwBlock;
        span(x.dev_param, x.n, ps, true);
        span(x.dev_grad, x.n, gs, false);
        span(x.dev_master, x.n, 4, true);
        span(x.dev_m, x.n, ss, true);
        span(x.dev_v, x.n, ss, true);
        span(x.dev_m_scale, blocks, 4, true);
        span(x.dev_v_scale, blocks, 4, true);
        o->table[t] = {x.dev_param, x.dev_grad, x.dev_master, x.dev_m, x.dev_v, x.dev_m_scale, x.dev_v_scale, x.n, 0,
                       x.param_dtype, x.grad_dtype, x.state_dtype, x.decay};
        elements += x.n;
    }
    std::sort(spans.get(), spans.get() + n_spans, [](const Span& a, const Span& b) { return a.lo < b.lo; });
    uintptr_t end = 0, written_end = 0;                          // of all spans so far, and of those that are written
    for (size_t i = 0; i < n_spans; ++i) {
        if (spans[i].lo < (spans[i].written ? end : written_end)) return fail(SPIRAL_ERR_INVALID_ARG, "adamw_create: a buffer that is written overlaps another");
        end = std::max(end, spans[i].hi);
        if (spans[i].written) written_end = std::max(written_end, spans[i].hi);
    }
    for (size_t i = 0; i < n_spans; ++i)
        if (spans[i].written) spans[o->n_written++] = spans[i];
    o->written = std::move(spans);
    o->n = n_tensors;
    o->steps = adamw_steps(elements);
    for (int t = 0; t < n_tensors; ++t) {
        o->table[t].first_chunk = chunks;
        chunks += adamw_chunks(o->table[t].n, o->steps);
    }
    o->chunks = chunks;
    o->mem = (char*)dev_mem;
    const int rc = adamw_upload(o.get(), stream, "adamw_create");
    if (rc) return rc;
    *out = o.release();
    return SPIRAL_OK;
}

// whether a step writes any of these bytes
static bool overwritten(const spiral_adamw* o, const void* p, uintptr_t bytes) {
    const uintptr_t lo = (uintptr_t)p;
    const Span* end = o->written.get() + o->n_written;
    const Span* next = std::upper_bound((const Span*)o->written.get(), end, lo, [](uintptr_t v, const Span& s) { return v < s.hi; });      // the first that ends behind lo
    return next != end && next->lo < lo + bytes;
}

static int check_grads(const spiral_adamw* o, const void* const* host_dev_grads, const char* who) {
    if (!o) return fail(SPIRAL_ERR_NOT_LOADED, "%s: null object", who);
    if (!host_dev_grads) return fail(SPIRAL_ERR_INVALID_ARG, "%s: null array", who);
    for (int t = 0; t < o->n; ++t) {
        if (!host_dev_grads[t] || !aligned(host_dev_grads[t], dtype_size(o->table[t].grad_dtype)))
            return fail(SPIRAL_ERR_INVALID_ARG, "%s: gradient %d is null or misaligned", who, t);
        if (overwritten(o, host_dev_grads[t], (uintptr_t)o->table[t].n * dtype_size(o->table[t].grad_dtype)))
            return fail(SPIRAL_ERR_INVALID_ARG, "%s: gradient %d overlaps a buffer that is written", who, t);
    }
    return SPIRAL_OK;
}

extern "C" int spiral_adamw_check_grads(const spiral_adamw* o, const void* const* host_dev_grads, int n) {
    if (!o) return fail(SPIRAL_ERR_NOT_LOADED, "adamw_check_grads: null object");
    if (n != o->n) return fail(SPIRAL_ERR_INVALID_ARG, "adamw_check_grads: %d gradients for %d tensors", n, o->n);
    return check_grads(o, host_dev_grads, "adamw_check_grads");
}

extern "C" int spiral_adamw_set_grads(spiral_adamw* o, const void* const* host_dev_grads, void* stream) {
    const int rc = check_grads(o, host_dev_grads, "adamw_set_grads");
    if (rc) return rc;
    for (int t = 0; t < o->n; ++t) o->table[t].grad = host_dev_grads[t];
    return adamw_upload(o, stream, "adamw_set_grads");
}

extern "C" int spiral_adamw_step(spiral_adamw* o, double lr, double beta1, double beta2, double eps, double weight_decay, int step,
                                 float grad_scale, float max_norm, float* dev_norm, void* stream) {
    if (!o) return fail(SPIRAL_ERR_NOT_LOADED, "adamw_step: null object");
    if (!(lr >= 0.0) || !std::isfinite(lr) || !(weight_decay >= 0.0) || !std::isfinite(weight_decay))
        return fail(SPIRAL_ERR_INVALID_ARG, "adamw_step: lr and weight_decay must be finite and >= 0");
    if (!(beta1 >= 0.0 && beta1 < 1.0) || !(beta2 >= 0.0 && beta2 < 1.0)) return fail(SPIRAL_ERR_INVALID_ARG, "adamw_step: betas must be in [0, 1)");
    if (!(eps >= 1e-30) || !(eps <= 1e30)) return fail(SPIRAL_ERR_INVALID_ARG, "adamw_step: eps must be in [1e-30, 1e30]");
    if (!(max_norm >= 0.f) || !std::isfinite(max_norm) || !std::isfinite(grad_scale)) return fail(SPIRAL_ERR_INVALID_ARG, "adamw_step: bad max_norm or grad_scale");
    if (step < 1) return fail(SPIRAL_ERR_INVALID_ARG, "adamw_step: steps are counted from 1");
    const float decay = (float)(lr * weight_decay), step_size = (float)(lr / (1.0 - std::pow(beta1, step)));
    if (!std::isfinite(decay) || !std::isfinite(step_size)) return fail(SPIRAL_ERR_INVALID_ARG, "adamw_step: lr * weight_decay or lr / (1 - beta1^step) passes 32 bits");
    if (!aligned(dev_norm, 4)) return fail(SPIRAL_ERR_INVALID_ARG, "adamw_step: misaligned norm");
    if (dev_norm) {                                  // also none of the gradients, which other workgroups still read when it is written
        bool meets = overwritten(o, dev_norm, 4);
        for (int t = 0; t < o->n && !meets; ++t) {
            const uintptr_t lo = (uintptr_t)o->table[t].grad, hi = lo + (uintptr_t)o->table[t].n * dtype_size(o->table[t].grad_dtype);
            meets = (uintptr_t)dev_norm < hi && lo < (uintptr_t)dev_norm + 4;
        }
        if (meets) return fail(SPIRAL_ERR_INVALID_ARG, "adamw_step: the norm overlaps a buffer of the table");
    }
    AdamwArgs a = {};
    a.table = (const AdamwRec*)o->mem;
    a.n_tensors = o->n;
    a.chunks = o->chunks;
    a.part = (double*)(o->mem + adamw_table_bytes(o->n));
    a.norm = dev_norm;
    a.beta1 = (float)beta1; a.rest1 = (float)(1.0 - beta1);
    a.beta2 = (float)beta2; a.rest2 = (float)(1.0 - beta2);
    a.eps = (float)eps;
    a.decay = decay;
    a.step_size = step_size;
    a.root_scale = (float)(1.0 / std::sqrt(1.0 - std::pow(beta2, step)));
    a.grad_scale = grad_scale;
    a.max_norm = max_norm;
    return done(launch_adamw(a, o->steps, (hipStream_t)stream), "adamw_step");
}

extern "C" void spiral_adamw_free(spiral_adamw* o) { delete o; }
