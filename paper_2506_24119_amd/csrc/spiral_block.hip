// Host side of the learner's operators between a decoder block's matrix products: attention over packed sequences, addition with RMSNorm, norm and
// rotation of heads.
#include <algorithm>
#include <cmath>
#include <memory>
#include <new>

#include "host_checks.h"

using namespace spiral;

constexpr long long kMostRows = 0x7FFFFFFFll;

// ---------------------------------------------------------------------------------------------
// attention
// ---------------------------------------------------------------------------------------------
struct spiral_attention_plan {
    int n_q_heads = 0, n_kv_heads = 0, head_dim = 0, n_q_items = 0, n_k_items = 0, parts = 1;
    long long n_rows = 0;
    const int4 *q_items = nullptr, *k_items = nullptr;      // device
};

// Workgroups of a sequence: four units of 32 rows and a query head of the group, 128 tokens.
static long long q_blocks(int len, int group) { return (((long long)len + 31) / 32 * group + 3) / 4; }
static long long k_blocks(int len) { return ((long long)len + 127) / 128; }
// The gradients of k and v take a workgroup 128 tokens and one kv head.  Where those are few, and the first tokens' much longer than the last's, the group's heads
// are shared out (28 heads on 4, one sequence of 300 tokens: 112 -> 53 us forward and backward, of 4,000: 1,328 -> 577, of 16,001: 9.6 -> 7.8 ms), but for so few
// stages of 32 rows that the launch that joins the parts would take longer.
static int k_parts(long long items, int longest, int group, int n_kv_heads) {
    const long long wanted = 1024, least_stages = 12, wgs = items * n_kv_heads;
    if ((longest + 31) / 32 * (long long)group < least_stages) return 1;
    return (int)std::min<long long>(group, std::max<long long>(1, (wanted + wgs - 1) / wgs));
}

static size_t up256(size_t b) { return (b + 255) & ~(size_t)255; }

struct PlanSizes { long long rows = 0, q_items = 0, k_items = 0; };
static int check_plan(const int32_t* host_lens, int B, int hq, int hkv, int hd, PlanSizes* z, const char* who) {
    if (!host_lens || B < 1) return fail(SPIRAL_ERR_INVALID_ARG, "%s: no sequences", who);
    if (hd != 32 && hd != 64 && hd != 128) return fail(SPIRAL_ERR_SHAPE, "%s: head_dim %d is not 32, 64 or 128", who, hd);
    if (hkv < 1 || hq < 1 || hq % hkv || hq > 1024) return fail(SPIRAL_ERR_SHAPE, "%s: %d query heads on %d kv heads", who, hq, hkv);
    for (int i = 0; i < B; ++i) {
        if (host_lens[i] < 0) return fail(SPIRAL_ERR_INVALID_ARG, "%s: length %d of sequence %d", who, host_lens[i], i);
        z->rows += host_lens[i];
        z->q_items += q_blocks(host_lens[i], hq / hkv);
        z->k_items += k_blocks(host_lens[i]);
    }
    if (z->rows < 1 || z->rows > kMostRows) return fail(SPIRAL_ERR_INVALID_ARG, "%s: %lld rows", who, z->rows);
    if (z->q_items > (1 << 28)) return fail(SPIRAL_ERR_INVALID_ARG, "%s: %lld rows of groups of %d heads", who, z->rows, hq / hkv);
    return SPIRAL_OK;
}

extern "C" size_t spiral_attention_plan_bytes(const int32_t* host_lens, int B, int n_q_heads, int n_kv_heads, int head_dim) {
    PlanSizes z;
    if (check_plan(host_lens, B, n_q_heads, n_kv_heads, head_dim, &z, "attention_plan_bytes")) return 0;
    return up256((size_t)(z.q_items + z.k_items) * sizeof(int4));
}

extern "C" int spiral_attention_plan_create(const int32_t* host_lens, int B, int n_q_heads, int n_kv_heads, int head_dim, void* dev_mem, size_t bytes,
                                            void* stream, spiral_attention_plan** out) {
    if (!out) return fail(SPIRAL_ERR_INVALID_ARG, "attention_plan_create: null out");
    *out = nullptr;
    PlanSizes z;
    const int rc = check_plan(host_lens, B, n_q_heads, n_kv_heads, head_dim, &z, "attention_plan_create");
    if (rc) return rc;
    const size_t n_items = (size_t)(z.q_items + z.k_items), need = up256(n_items * sizeof(int4));
    if (!dev_mem || !aligned(dev_mem, 256) || bytes < need)
        return fail(SPIRAL_ERR_INVALID_ARG, "attention_plan_create: memory is null, not 256-byte aligned or less than %zu bytes", need);
    struct Seq { int row0, len; };
    std::unique_ptr<spiral_attention_plan> p(new (std::nothrow) spiral_attention_plan());
    std::unique_ptr<Seq[]> seqs(new (std::nothrow) Seq[B]);
    std::unique_ptr<int4[]> items(new (std::nothrow) int4[n_items]);
    if (!p || !seqs || !items) return fail(SPIRAL_ERR_INVALID_ARG, "attention_plan_create: out of host memory");
    int row = 0;
    for (int i = 0; i < B; ++i) { seqs[i] = {row, host_lens[i]}; row += host_lens[i]; }
    // Workgroups start in this order: those of rows with the most tokens before them and those of tokens with the most rows behind them first, whatever their sequence, so that the last to
    // start are short.  A sequence's blocks together instead, for the L2's sake: gradients of k and v 2.14 -> 2.22 ms (16 sequences of U[1024, 4096]), forward 36.5 -> 38.5 us (37 of
    // U[3, 999], 64 dimensions), 128 -> 130 (24 of U[256, 1024]), the rest the same.
    std::sort(seqs.get(), seqs.get() + B, [](const Seq& x, const Seq& y) { return x.len != y.len ? x.len > y.len : x.row0 < y.row0; });
    const int group = n_q_heads / n_kv_heads;
    int4* at = items.get();
    for (int i = 0; i < B; ++i)
        for (long long b = q_blocks(seqs[i].len, group) - 1; b >= 0; --b) *at++ = int4{seqs[i].row0, seqs[i].len, (int)b, 0};
    std::stable_sort(items.get(), at, [](const int4& x, const int4& y) { return x.z > y.z; });
    for (int i = 0; i < B; ++i)
        for (long long b = 0; b < k_blocks(seqs[i].len); ++b) *at++ = int4{seqs[i].row0, seqs[i].len, (int)b, 0};
    std::stable_sort(items.get() + z.q_items, at, [](const int4& x, const int4& y) { return x.y - 128ll * x.z > y.y - 128ll * y.z; });
    p->n_q_heads = n_q_heads; p->n_kv_heads = n_kv_heads; p->head_dim = head_dim;
    p->n_rows = z.rows; p->n_q_items = (int)z.q_items; p->n_k_items = (int)z.k_items;
    p->parts = k_parts(z.k_items, seqs[0].len, group, n_kv_heads);
    p->q_items = (const int4*)dev_mem; p->k_items = p->q_items + z.q_items;
    for (size_t t = 0; t < n_items; t += 1 << 20) {              // sizes of launch_upload are ints
        const hipError_t e = launch_upload((int32_t*)dev_mem + t * 4, (const int32_t*)(items.get() + t), (int)std::min<size_t>(1 << 20, n_items - t) * 4, (hipStream_t)stream);
        if (e != hipSuccess) return done(e, "attention_plan_create");
    }
    *out = p.release();
    return SPIRAL_OK;
}

extern "C" void spiral_attention_plan_free(spiral_attention_plan* plan) { delete plan; }

// pointer and stride of a matrix of the call
static bool matrix_ok(const void* p, long long stride, long long width) {
    return p && aligned(p, 16) && stride >= width && stride % 8 == 0 && stride <= (1ll << 22);
}
static PackArgs pack_args(const spiral_attention_plan* p, float scale) {
    PackArgs a = {};
    a.q_items = p->q_items; a.n_q_items = p->n_q_items; a.k_items = p->k_items; a.n_k_items = p->n_k_items; a.n_rows = p->n_rows;
    a.n_q_heads = p->n_q_heads; a.n_kv_heads = p->n_kv_heads; a.parts = p->parts;
    a.scale = scale; a.scale_log2e = (float)(scale * 1.4426950408889634);
    return a;
}
static bool scale_ok(float scale) { return scale >= 1e-30f && scale <= 1e30f; }

extern "C" int spiral_attention_forward(const spiral_attention_plan* plan, const void* dev_q, long long q_stride, const void* dev_k, long long k_stride,
                                        const void* dev_v, long long v_stride, int dtype, float scale, void* dev_out, long long out_stride, float* dev_lse,
                                        void* stream) {
    if (!plan) return fail(SPIRAL_ERR_NOT_LOADED, "attention_forward: null plan");
    if (dtype != SPIRAL_DTYPE_BF16 && dtype != SPIRAL_DTYPE_FP16) return fail(SPIRAL_ERR_INVALID_ARG, "attention_forward: unknown type %d", dtype);
    if (!scale_ok(scale)) return fail(SPIRAL_ERR_INVALID_ARG, "attention_forward: scale must be in [1e-30, 1e30]");
    const long long wq = (long long)plan->n_q_heads * plan->head_dim, wk = (long long)plan->n_kv_heads * plan->head_dim, n = plan->n_rows;
    if (!matrix_ok(dev_q, q_stride, wq) || !matrix_ok(dev_k, k_stride, wk) || !matrix_ok(dev_v, v_stride, wk) || !matrix_ok(dev_out, out_stride, wq) ||
        !dev_lse || !aligned(dev_lse, 4))
        return fail(SPIRAL_ERR_INVALID_ARG, "attention_forward: a matrix is null or misaligned, or its stride is less than a row, no multiple of 8 or above 2^22");
    const Rows rows[] = {rows_of(dev_q, q_stride, wq, n, 2, false), rows_of(dev_k, k_stride, wk, n, 2, false), rows_of(dev_v, v_stride, wk, n, 2, false),
                         rows_of(dev_out, out_stride, wq, n, 2, true), rows_of(dev_lse, 0, n * plan->n_q_heads, 1, 4, true)};
    if (any_meet(rows, 5)) return fail(SPIRAL_ERR_INVALID_ARG, "attention_forward: a buffer that is written overlaps another");
    PackArgs a = pack_args(plan, scale);
    a.q = dev_q; a.k = dev_k; a.v = dev_v; a.out = dev_out; a.lse = dev_lse;
    a.q_stride = q_stride; a.k_stride = k_stride; a.v_stride = v_stride; a.out_stride = out_stride;
    return done(launch_pack_forward(a, dtype, plan->head_dim, (hipStream_t)stream), "attention_forward");
}

extern "C" size_t spiral_attention_backward_workspace_bytes(const spiral_attention_plan* plan) {
    if (!plan) return 0;
    const size_t delta = up256((size_t)plan->n_rows * plan->n_q_heads * 4);
    return delta + (plan->parts > 1 ? up256((size_t)plan->parts * 2 * plan->n_rows * plan->n_kv_heads * plan->head_dim * 4) : 0);
}

extern "C" int spiral_attention_backward(const spiral_attention_plan* plan, const void* dev_q, long long q_stride, const void* dev_k, long long k_stride,
                                         const void* dev_v, long long v_stride, const void* dev_out, long long out_stride, const float* dev_lse,
                                         const void* dev_dout, long long dout_stride, int dtype, float scale, void* dev_dq, long long dq_stride,
                                         void* dev_dk, long long dk_stride, void* dev_dv, long long dv_stride, void* dev_workspace, size_t workspace_bytes,
                                         void* stream) {
    if (!plan) return fail(SPIRAL_ERR_NOT_LOADED, "attention_backward: null plan");
    if (dtype != SPIRAL_DTYPE_BF16 && dtype != SPIRAL_DTYPE_FP16) return fail(SPIRAL_ERR_INVALID_ARG, "attention_backward: unknown type %d", dtype);
    if (!scale_ok(scale)) return fail(SPIRAL_ERR_INVALID_ARG, "attention_backward: scale must be in [1e-30, 1e30]");
    const long long wq = (long long)plan->n_q_heads * plan->head_dim, wk = (long long)plan->n_kv_heads * plan->head_dim, n = plan->n_rows;
    if (!matrix_ok(dev_q, q_stride, wq) || !matrix_ok(dev_k, k_stride, wk) || !matrix_ok(dev_v, v_stride, wk) || !matrix_ok(dev_out, out_stride, wq) ||
        !matrix_ok(dev_dout, dout_stride, wq) || !matrix_ok(dev_dq, dq_stride, wq) || !matrix_ok(dev_dk, dk_stride, wk) || !matrix_ok(dev_dv, dv_stride, wk) ||
        !dev_lse || !aligned(dev_lse, 4))
        return fail(SPIRAL_ERR_INVALID_ARG, "attention_backward: a matrix is null or misaligned, or its stride is less than a row, no multiple of 8 or above 2^22");
    const size_t need = spiral_attention_backward_workspace_bytes(plan);
    if (!dev_workspace || !aligned(dev_workspace, 256)) return fail(SPIRAL_ERR_INVALID_ARG, "attention_backward: workspace is null or not 256-byte aligned");
    if (workspace_bytes < need) return fail(SPIRAL_ERR_INVALID_ARG, "attention_backward: workspace of %zu bytes, %zu needed", workspace_bytes, need);
    const Rows rows[] = {rows_of(dev_q, q_stride, wq, n, 2, false), rows_of(dev_k, k_stride, wk, n, 2, false), rows_of(dev_v, v_stride, wk, n, 2, false),
                         rows_of(dev_out, out_stride, wq, n, 2, false), rows_of(dev_dout, dout_stride, wq, n, 2, false),
                         rows_of(dev_lse, 0, n * plan->n_q_heads, 1, 4, false), rows_of(dev_dq, dq_stride, wq, n, 2, true),
                         rows_of(dev_dk, dk_stride, wk, n, 2, true), rows_of(dev_dv, dv_stride, wk, n, 2, true), rows_of(dev_workspace, 0, (long long)need, 1, 1, true)};
    if (any_meet(rows, 10)) return fail(SPIRAL_ERR_INVALID_ARG, "attention_backward: a buffer that is written overlaps another");
    PackArgs a = pack_args(plan, scale);
    a.q = dev_q; a.k = dev_k; a.v = dev_v; a.out_in = dev_out; a.lse = (float*)dev_lse; a.dout = dev_dout;
    a.dq = dev_dq; a.dk = dev_dk; a.dv = dev_dv; a.delta = (float*)dev_workspace;
    a.part = (float*)((char*)dev_workspace + up256((size_t)n * plan->n_q_heads * 4));
    a.q_stride = q_stride; a.k_stride = k_stride; a.v_stride = v_stride; a.out_stride = out_stride; a.dout_stride = dout_stride;
    a.dq_stride = dq_stride; a.dk_stride = dk_stride; a.dv_stride = dv_stride;
    return done(launch_pack_backward(a, dtype, plan->head_dim, (hipStream_t)stream), "attention_backward");
}

// ---------------------------------------------------------------------------------------------
// addition and RMSNorm
// ---------------------------------------------------------------------------------------------
static bool in_place(const void* a, long long a_stride, const void* b, long long b_stride) { return a == b && a_stride == b_stride; }
static bool norm_sizes_ok(long long n_rows, int d) { return n_rows >= 1 && n_rows <= kMostRows && d >= 1 && d <= (1 << 24); }
static bool eps_ok(float eps) { return eps >= 0.f && eps <= 1.f; }

extern "C" int spiral_add_rmsnorm(const void* dev_x, long long x_stride, const void* dev_residual, long long residual_stride, const float* dev_gain, int dtype,
                                  long long n_rows, int d, float eps, void* dev_out, int out_dtype, long long out_stride, float* dev_out_scale,
                                  void* dev_sum, long long sum_stride, float* dev_rstd, void* stream) {
    if (!dev_x || !dev_gain || !dev_out) return fail(SPIRAL_ERR_INVALID_ARG, "add_rmsnorm: null x, gain or output");
    if (!norm_sizes_ok(n_rows, d)) return fail(SPIRAL_ERR_INVALID_ARG, "add_rmsnorm: bad n_rows=%lld or d=%d", n_rows, d);
    const int size = dtype_size(dtype);
    const bool codes = out_dtype == SPIRAL_DTYPE_E4M3;
    if (!size || (!codes && out_dtype != dtype)) return fail(SPIRAL_ERR_INVALID_ARG, "add_rmsnorm: unknown type %d, or output %d of another", dtype, out_dtype);
    if (codes != (dev_out_scale != nullptr)) return fail(SPIRAL_ERR_INVALID_ARG, "add_rmsnorm: scales go with 8-bit outputs");
    if (x_stride < d || out_stride < d || (dev_residual && residual_stride < d) || (dev_sum && sum_stride < d))
        return fail(SPIRAL_ERR_INVALID_ARG, "add_rmsnorm: a row stride is less than d=%d", d);
    if (!aligned(dev_x, size) || !aligned(dev_residual, size) || !aligned(dev_sum, size) || !aligned(dev_out, codes ? 1 : size) || !aligned(dev_gain, 4) ||
        !aligned(dev_out_scale, 4) || !aligned(dev_rstd, 4))
        return fail(SPIRAL_ERR_INVALID_ARG, "add_rmsnorm: misaligned buffer");
    if (!eps_ok(eps)) return fail(SPIRAL_ERR_INVALID_ARG, "add_rmsnorm: eps must be in [0, 1]");
    const bool over_x = in_place(dev_sum, sum_stride, dev_x, x_stride), over_res = in_place(dev_sum, sum_stride, dev_residual, residual_stride);
    const Rows rows[] = {rows_of(over_x ? nullptr : dev_x, x_stride, d, n_rows, size, false),
                         rows_of(over_res ? nullptr : dev_residual, residual_stride, d, n_rows, size, false), rows_of(dev_gain, 0, d, 1, 4, false),
                         rows_of(dev_out, out_stride, d, n_rows, codes ? 1 : size, true), rows_of(dev_sum, sum_stride, d, n_rows, size, true),
                         rows_of(dev_out_scale, 0, n_rows, 1, 4, true), rows_of(dev_rstd, 0, n_rows, 1, 4, true)};
    if (any_meet(rows, 7)) return fail(SPIRAL_ERR_INVALID_ARG, "add_rmsnorm: a buffer that is written overlaps another");
    NormRowsArgs a = {};
    a.x = dev_x; a.x_stride = x_stride; a.residual = dev_residual; a.residual_stride = residual_stride; a.gain = dev_gain;
    a.n_rows = n_rows; a.d = d; a.eps = eps;
    a.out = dev_out; a.out_stride = out_stride; a.sum = dev_sum; a.sum_stride = sum_stride; a.out_scale = dev_out_scale; a.rstd = dev_rstd;
    return done(launch_add_norm_rows(a, dtype, (hipStream_t)stream), "add_rmsnorm");
}

extern "C" size_t spiral_add_rmsnorm_backward_workspace_bytes(long long n_rows, int d) {
    return norm_sizes_ok(n_rows, d) ? norm_grad_workspace_bytes(n_rows, d) : 0;
}

extern "C" int spiral_add_rmsnorm_backward(const void* dev_dout, long long dout_stride, const void* dev_sum, long long sum_stride, const float* dev_gain,
                                           const float* dev_rstd, const void* dev_dsum, long long dsum_stride, int dtype, long long n_rows, int d,
                                           void* dev_dx, long long dx_stride, float* dev_dgain, void* dev_workspace, size_t workspace_bytes, void* stream) {
    if (!dev_dout || !dev_sum || !dev_gain || !dev_rstd || !dev_dx) return fail(SPIRAL_ERR_INVALID_ARG, "add_rmsnorm_backward: null pointer");
    if (!norm_sizes_ok(n_rows, d)) return fail(SPIRAL_ERR_INVALID_ARG, "add_rmsnorm_backward: bad n_rows=%lld or d=%d", n_rows, d);
    const int size = dtype_size(dtype);
    if (!size) return fail(SPIRAL_ERR_INVALID_ARG, "add_rmsnorm_backward: unknown type %d", dtype);
    if (dout_stride < d || sum_stride < d || dx_stride < d || (dev_dsum && dsum_stride < d))
        return fail(SPIRAL_ERR_INVALID_ARG, "add_rmsnorm_backward: a row stride is less than d=%d", d);
    if (!aligned(dev_dout, size) || !aligned(dev_sum, size) || !aligned(dev_dsum, size) || !aligned(dev_dx, size) || !aligned(dev_gain, 4) ||
        !aligned(dev_rstd, 4) || !aligned(dev_dgain, 4))
        return fail(SPIRAL_ERR_INVALID_ARG, "add_rmsnorm_backward: misaligned buffer");
    const size_t need = dev_dgain ? norm_grad_workspace_bytes(n_rows, d) : 0;
    if (need && (!dev_workspace || !aligned(dev_workspace, 256))) return fail(SPIRAL_ERR_INVALID_ARG, "add_rmsnorm_backward: workspace is null or not 256-byte aligned");
    if (need && workspace_bytes < need) return fail(SPIRAL_ERR_INVALID_ARG, "add_rmsnorm_backward: workspace of %zu bytes, %zu needed", workspace_bytes, need);
    const bool over_dout = in_place(dev_dx, dx_stride, dev_dout, dout_stride), over_dsum = in_place(dev_dx, dx_stride, dev_dsum, dsum_stride);
    const Rows rows[] = {rows_of(over_dout ? nullptr : dev_dout, dout_stride, d, n_rows, size, false), rows_of(dev_sum, sum_stride, d, n_rows, size, false),
                         rows_of(over_dsum ? nullptr : dev_dsum, dsum_stride, d, n_rows, size, false), rows_of(dev_gain, 0, d, 1, 4, false),
                         rows_of(dev_rstd, 0, n_rows, 1, 4, false), rows_of(dev_dx, dx_stride, d, n_rows, size, true), rows_of(dev_dgain, 0, d, 1, 4, true),
                         rows_of(need ? dev_workspace : nullptr, 0, (long long)need, 1, 1, true)};
    if (any_meet(rows, 8)) return fail(SPIRAL_ERR_INVALID_ARG, "add_rmsnorm_backward: a buffer that is written overlaps another");
    NormGradArgs a = {};
    a.dout = dev_dout; a.dout_stride = dout_stride; a.sum = dev_sum; a.sum_stride = sum_stride; a.dsum = dev_dsum; a.dsum_stride = dsum_stride;
    a.gain = dev_gain; a.rstd = dev_rstd; a.n_rows = n_rows; a.d = d;
    a.dx = dev_dx; a.dx_stride = dx_stride; a.dgain = dev_dgain; a.part = need ? (float*)dev_workspace : nullptr;
    return done(launch_norm_grad(a, dtype, (hipStream_t)stream), "add_rmsnorm_backward");
}

// ---------------------------------------------------------------------------------------------
// norm and rotation of heads
// ---------------------------------------------------------------------------------------------
static int check_rope(int dtype, long long n_rows, int hq, int hkv, int hd, float eps, double theta, const int32_t* positions, const char* who) {
    if (!positions || !aligned(positions, 4)) return fail(SPIRAL_ERR_INVALID_ARG, "%s: positions are null or misaligned", who);
    if (n_rows < 1 || n_rows > kMostRows) return fail(SPIRAL_ERR_INVALID_ARG, "%s: bad n_rows=%lld", who, n_rows);
    if (hd != 32 && hd != 64 && hd != 128) return fail(SPIRAL_ERR_SHAPE, "%s: head_dim %d is not 32, 64 or 128", who, hd);
    if (hq < 1 || hkv < 1 || hq > 1024 || hkv > 1024) return fail(SPIRAL_ERR_SHAPE, "%s: %d query and %d kv heads", who, hq, hkv);
    if (!dtype_size(dtype)) return fail(SPIRAL_ERR_INVALID_ARG, "%s: unknown type %d", who, dtype);
    if (!eps_ok(eps)) return fail(SPIRAL_ERR_INVALID_ARG, "%s: eps must be in [0, 1]", who);
    if (!(theta >= 1.0 && theta <= 1e30)) return fail(SPIRAL_ERR_INVALID_ARG, "%s: theta must be in [1, 1e30]", who);
    return SPIRAL_OK;
}
static RopeFreq frequencies(double theta, int hd) {       // in turns a position
    RopeFreq f = {};
    const long double step = std::pow((long double)theta, -2.0L / hd);             // its powers are off by 2^-58, and take 0.5 us where a power each takes 1.2
    long double turns = 1.0L / 6.283185307179586476925286766559L;
    for (int c = 0; c < hd / 2; ++c, turns *= step) f.inv_freq[c] = (double)turns;
    return f;
}

extern "C" int spiral_norm_rope(const void* dev_q, long long q_stride, const void* dev_k, long long k_stride, const float* dev_gain_q, const float* dev_gain_k,
                                int dtype, long long n_rows, int n_q_heads, int n_kv_heads, int head_dim, float eps, double theta, const int32_t* dev_positions,
                                void* dev_out_q, long long out_q_stride, void* dev_out_k, long long out_k_stride, void* stream) {
    const int rc = check_rope(dtype, n_rows, n_q_heads, n_kv_heads, head_dim, eps, theta, dev_positions, "norm_rope");
    if (rc) return rc;
    if (!dev_q || !dev_k || !dev_out_q || !dev_out_k) return fail(SPIRAL_ERR_INVALID_ARG, "norm_rope: null heads or output");
    const int size = dtype_size(dtype);
    const long long wq = (long long)n_q_heads * head_dim, wk = (long long)n_kv_heads * head_dim;
    if (q_stride < wq || out_q_stride < wq || k_stride < wk || out_k_stride < wk) return fail(SPIRAL_ERR_INVALID_ARG, "norm_rope: a row stride is less than a row");
    if (!aligned(dev_q, size) || !aligned(dev_k, size) || !aligned(dev_out_q, size) || !aligned(dev_out_k, size) || !aligned(dev_gain_q, 4) || !aligned(dev_gain_k, 4))
        return fail(SPIRAL_ERR_INVALID_ARG, "norm_rope: misaligned buffer");
    const bool over_q = in_place(dev_q, q_stride, dev_out_q, out_q_stride), over_k = in_place(dev_k, k_stride, dev_out_k, out_k_stride);
    const Rows rows[] = {rows_of(over_q ? nullptr : dev_q, q_stride, wq, n_rows, size, false), rows_of(over_k ? nullptr : dev_k, k_stride, wk, n_rows, size, false),
                         rows_of(dev_gain_q, 0, head_dim, 1, 4, false), rows_of(dev_gain_k, 0, head_dim, 1, 4, false), rows_of(dev_positions, 0, n_rows, 1, 4, false),
                         rows_of(dev_out_q, out_q_stride, wq, n_rows, size, true), rows_of(dev_out_k, out_k_stride, wk, n_rows, size, true)};
    if (any_meet(rows, 7)) return fail(SPIRAL_ERR_INVALID_ARG, "norm_rope: a buffer that is written overlaps another");
    RopeArgs a = {};
    a.side[0] = {dev_q, nullptr, dev_out_q, q_stride, 0, out_q_stride, dev_gain_q, nullptr, n_q_heads};
    a.side[1] = {dev_k, nullptr, dev_out_k, k_stride, 0, out_k_stride, dev_gain_k, nullptr, n_kv_heads};
    a.n_rows = n_rows; a.positions = dev_positions; a.eps = eps;
    return done(launch_norm_rope(a, frequencies(theta, head_dim), dtype, head_dim, (hipStream_t)stream), "norm_rope");
}

extern "C" size_t spiral_norm_rope_backward_workspace_bytes(long long n_rows, int n_q_heads, int n_kv_heads, int head_dim) {
    if (n_rows < 1 || n_rows > kMostRows || n_q_heads < 1 || n_q_heads > 1024 || n_kv_heads < 1 || n_kv_heads > 1024 ||
        (head_dim != 32 && head_dim != 64 && head_dim != 128)) return 0;
    return norm_rope_grad_workspace_bytes(n_rows, head_dim);
}

extern "C" int spiral_norm_rope_backward(const void* dev_q, long long q_stride, const void* dev_k, long long k_stride, const void* dev_dout_q, long long dout_q_stride,
                                         const void* dev_dout_k, long long dout_k_stride, const float* dev_gain_q, const float* dev_gain_k, int dtype,
                                         long long n_rows, int n_q_heads, int n_kv_heads, int head_dim, float eps, double theta, const int32_t* dev_positions,
                                         void* dev_dq, long long dq_stride, void* dev_dk, long long dk_stride, float* dev_dgain_q, float* dev_dgain_k,
                                         void* dev_workspace, size_t workspace_bytes, void* stream) {
    const int rc = check_rope(dtype, n_rows, n_q_heads, n_kv_heads, head_dim, eps, theta, dev_positions, "norm_rope_backward");
    if (rc) return rc;
    if (!dev_dout_q || !dev_dout_k || !dev_dq || !dev_dk || (dev_gain_q && !dev_q) || (dev_gain_k && !dev_k))
        return fail(SPIRAL_ERR_INVALID_ARG, "norm_rope_backward: null pointer");
    if ((dev_dgain_q && !dev_gain_q) || (dev_dgain_k && !dev_gain_k)) return fail(SPIRAL_ERR_INVALID_ARG, "norm_rope_backward: a gradient of a gain that is not there");
    if (!dev_gain_q) dev_q = nullptr;                 // not read
    if (!dev_gain_k) dev_k = nullptr;
    const int size = dtype_size(dtype);
    const long long wq = (long long)n_q_heads * head_dim, wk = (long long)n_kv_heads * head_dim;
    if ((dev_q && q_stride < wq) || dout_q_stride < wq || dq_stride < wq || (dev_k && k_stride < wk) || dout_k_stride < wk || dk_stride < wk)
        return fail(SPIRAL_ERR_INVALID_ARG, "norm_rope_backward: a row stride is less than a row");
    if (!aligned(dev_q, size) || !aligned(dev_k, size) || !aligned(dev_dout_q, size) || !aligned(dev_dout_k, size) || !aligned(dev_dq, size) || !aligned(dev_dk, size) ||
        !aligned(dev_gain_q, 4) || !aligned(dev_gain_k, 4) || !aligned(dev_dgain_q, 4) || !aligned(dev_dgain_k, 4))
        return fail(SPIRAL_ERR_INVALID_ARG, "norm_rope_backward: misaligned buffer");
    const size_t need = dev_dgain_q || dev_dgain_k ? norm_rope_grad_workspace_bytes(n_rows, head_dim) : 0;
    if (need && (!dev_workspace || !aligned(dev_workspace, 256))) return fail(SPIRAL_ERR_INVALID_ARG, "norm_rope_backward: workspace is null or not 256-byte aligned");
    if (need && workspace_bytes < need) return fail(SPIRAL_ERR_INVALID_ARG, "norm_rope_backward: workspace of %zu bytes, %zu needed", workspace_bytes, need);
    const bool over_q = in_place(dev_dout_q, dout_q_stride, dev_dq, dq_stride), over_k = in_place(dev_dout_k, dout_k_stride, dev_dk, dk_stride);
    const Rows rows[] = {rows_of(dev_q, q_stride, wq, n_rows, size, false), rows_of(dev_k, k_stride, wk, n_rows, size, false),
                         rows_of(over_q ? nullptr : dev_dout_q, dout_q_stride, wq, n_rows, size, false), rows_of(over_k ? nullptr : dev_dout_k, dout_k_stride, wk, n_rows, size, false),
                         rows_of(dev_gain_q, 0, head_dim, 1, 4, false), rows_of(dev_gain_k, 0, head_dim, 1, 4, false), rows_of(dev_positions, 0, n_rows, 1, 4, false),
                         rows_of(dev_dq, dq_stride, wq, n_rows, size, true), rows_of(dev_dk, dk_stride, wk, n_rows, size, true),
                         rows_of(dev_dgain_q, 0, head_dim, 1, 4, true), rows_of(dev_dgain_k, 0, head_dim, 1, 4, true),
                         rows_of(need ? dev_workspace : nullptr, 0, (long long)need, 1, 1, true)};
    if (any_meet(rows, 12)) return fail(SPIRAL_ERR_INVALID_ARG, "norm_rope_backward: a buffer that is written overlaps another");
    RopeArgs a = {};
    a.side[0] = {dev_q, dev_dout_q, dev_dq, q_stride, dout_q_stride, dq_stride, dev_gain_q, dev_dgain_q, n_q_heads};
    a.side[1] = {dev_k, dev_dout_k, dev_dk, k_stride, dout_k_stride, dk_stride, dev_gain_k, dev_dgain_k, n_kv_heads};
    a.n_rows = n_rows; a.positions = dev_positions; a.eps = eps;
    a.part = need ? (float*)dev_workspace : nullptr;
    return done(launch_norm_rope_grad(a, frequencies(theta, head_dim), dtype, head_dim, (hipStream_t)stream), "norm_rope_backward");
}
