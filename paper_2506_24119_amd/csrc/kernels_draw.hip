// One token a row from given uniform numbers: the inverse of the running sum of the kept weights, in index order.
#include "spiral_internal.h"

namespace spiral {

namespace {

constexpr int kThreads = 1024;
constexpr int kWaves = kThreads / 64;

// larger float <=> larger key; -0 and +0 share a key
__device__ __forceinline__ uint32_t order_key(float z) {
    const uint32_t b = __float_as_uint(z + 0.0f);
    return (b & 0x80000000u) ? ~b : (b | 0x80000000u);
}

__device__ __forceinline__ float clean(float l) { return l == l ? l : -INFINITY; }      // an undefined logit is never drawn
template <class T> __device__ __forceinline__ float logit_at(const T* row, uint32_t v);
template <> __device__ __forceinline__ float logit_at(const float* row, uint32_t v) { return clean(row[v]); }
template <> __device__ __forceinline__ float logit_at(const __bf16* row, uint32_t v) { return clean((float)row[v]); }
template <> __device__ __forceinline__ float logit_at(const _Float16* row, uint32_t v) { return clean((float)row[v]); }

__device__ __forceinline__ uint64_t shfl_down_u64(uint64_t v, int d) {
    const uint32_t lo = __shfl_down((uint32_t)v, d, 64), hi = __shfl_down((uint32_t)(v >> 32), d, 64);
    return ((uint64_t)hi << 32) | lo;
}

// w = exp((l - m) / T) in 64 bits: the tokens follow from where u falls between sums of up to 10^5 of them, and an error of 1e-7 in those
// would draw another token once in a few dozen rows.  The largest logit, +inf too, weighs 1.
struct Weight {
    double m, inv_t;
    bool greedy;
    __device__ __forceinline__ double operator()(float l) const {
        if ((double)l == m) return 1.0;
        return greedy ? 0.0 : exp(((double)l - m) * inv_t);
    }
};

struct Select {
    uint32_t prefix;       // digits fixed so far (high bits)
    uint64_t remaining;    // how much (count or mass) must still be covered from the top of the current digit
};

// Among 256 bins, walking from bin 255 down, the one in which the running total first reaches `remaining`.  By one wave.
__device__ __forceinline__ void pick_digit(const uint64_t* hist, int shift, Select* sel, int lane) {
    uint64_t b[4], mine = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) { b[i] = hist[lane * 4 + i]; mine += b[i]; }
    uint64_t incl = mine;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const uint64_t o = shfl_down_u64(incl, d);
        if (lane + d < 64) incl += o;
    }
    uint64_t acc = incl - mine;
    const uint64_t need = sel->remaining;
    if (acc < need && need <= incl) {               // exactly one lane
#pragma unroll
        for (int i = 3; i >= 0; --i) {
            if (acc + b[i] >= need) { sel->prefix |= (uint32_t)(lane * 4 + i) << shift; sel->remaining = need - acc; break; }
            acc += b[i];
        }
    }
}

}  // namespace

// A row by a workgroup, in as many sweeps of it as the cuts need: one for the maximum, four digits of the k-th largest key, four of the
// key at which the mass reaches p, one for the sum of what is kept and a part of one for the token.
template <class T>
__global__ __launch_bounds__(kThreads) void draw_row_kernel(DrawArgs a, DrawRows rows) {
    __shared__ uint64_t hist[256];
    __shared__ Select sel;
    __shared__ double s_sum[kWaves];
    __shared__ float s_max[kWaves];
    const int r = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const T* row = (const T*)a.logits + (size_t)r * a.row_stride;
    const uint32_t V = a.V;

    float m = -INFINITY;
    for (uint32_t v = tid; v < V; v += kThreads) m = fmaxf(m, logit_at(row, v));
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor(m, o, 64));
    if (lane == 0) s_max[wave] = m;
    __syncthreads();
    for (int w = 0; w < kWaves; ++w) m = fmaxf(m, s_max[w]);
    if (m == -INFINITY) {                           // nothing can be drawn
        if (tid == 0) {
            a.tokens[r] = 0;
            if (a.logp) a.logp[r] = -INFINITY;
        }
        return;
    }
    const float temperature = rows.temperature[r];
    const bool greedy = temperature == 0.f;
    const Weight weight = {(double)m, greedy ? 0.0 : 1.0 / (double)temperature, greedy};
    const int top_k = greedy ? 0 : rows.top_k[r];
    const double top_p = greedy ? 1.0 : rows.top_p[r], min_p = greedy ? 0.0 : rows.min_p[r];
    uint32_t floor_key = 0;

    auto descend = [&](auto&& amount, auto&& total_known) {
        for (int shift = 24; shift >= 0; shift -= 8) {
            __syncthreads();
            if (tid < 256) hist[tid] = 0;
            __syncthreads();
            const uint32_t prefix = sel.prefix;
            for (uint32_t v = tid; v < V; v += kThreads) {
                const float l = logit_at(row, v);
                const uint32_t key = order_key(l);
                if (key >= floor_key && (shift == 24 || (key >> (shift + 8)) == (prefix >> (shift + 8)))) {
                    const uint64_t x = amount(l);
                    if (x) atomicAdd((unsigned long long*)&hist[key >> shift & 255u], (unsigned long long)x);
                }
            }
            __syncthreads();
            if (shift == 24) {
                if (tid == 0) total_known();
                __syncthreads();
            }
            if (wave == 0) pick_digit(hist, shift, &sel, lane);
        }
        __syncthreads();
        floor_key = sel.prefix > floor_key ? sel.prefix : floor_key;
        __syncthreads();
    };
    if (top_k > 0 && (uint32_t)top_k < V) {
        if (tid == 0) { sel.prefix = 0; sel.remaining = (uint64_t)top_k; }
        descend([](float) { return (uint64_t)1; }, [] {});
    }
    if (top_p < 1.0) {
        // integers add in any order: 2^-b of the largest weight, b as V of them leave room for
        const double unit = ldexp(1.0, 30 + __clz(V));
        if (tid == 0) { sel.prefix = 0; sel.remaining = 0; }
        descend([&](float l) { return (uint64_t)rint(weight(l) * unit); }, [&] {
            uint64_t z = 0;
            for (int i = 0; i < 256; ++i) z += hist[i];
            const uint64_t target = (uint64_t)ceil(top_p * (double)z);
            sel.remaining = target < 1 ? 1 : target > z ? z : target;
        });
    }

    auto kept = [&](float l) {
        if (order_key(l) < floor_key) return 0.0;
        const double w = weight(l);
        return w >= min_p ? w : 0.0;
    };
    // a wave has a run of neighbouring entries
    const uint32_t run = ((V + kWaves - 1) / kWaves + 63) & ~63u;
    const uint32_t lo = min((uint32_t)wave * run, V), hi = min(lo + run, V);
    double sum = 0.0;
    for (uint32_t v = lo + lane; v < hi; v += 64) sum += kept(logit_at(row, v));
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o, 64);
    if (lane == 0) s_sum[wave] = sum;
    __syncthreads();
    double total = 0.0;
    for (int w = 0; w < kWaves; ++w) total += s_sum[w];
    const float u = greedy ? 0.f : a.uniform[r];
    const double target = (double)fminf(fmaxf(u, 0.f), 0.99999994f) * total;      // fmaxf: a NaN counts as 0
    double before = 0.0;
    int mine = -1;
    for (int w = 0, done = 0; w < kWaves && !done; ++w) {
        if (s_sum[w] > 0.0) mine = w;               // rounding may leave none: then the last with anything in it
        if (before + s_sum[w] > target) done = 1;
        else if (w + 1 < kWaves) before += s_sum[w];
    }
    if (wave != mine) return;
    uint32_t token = 0;
    bool found = false;
    before = 0.0;
    for (int w = 0; w < mine; ++w) before += s_sum[w];
    for (uint32_t v0 = lo; v0 < hi && !found; v0 += 64) {
        const uint32_t v = v0 + lane;
        const double w = v < hi ? kept(logit_at(row, v)) : 0.0;
        double c = w;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const double o = __shfl_up(c, d, 64);
            if (lane >= d) c += o;
        }
        const uint64_t over = __builtin_amdgcn_ballot_w64(w > 0.0 && before + c > target), any = __builtin_amdgcn_ballot_w64(w > 0.0);
        if (over) { token = v0 + __builtin_ctzll(over); found = true; }
        else if (any) token = v0 + 63 - __builtin_clzll(any);
        before += __shfl(c, 63, 64);
    }
    if (lane == 0) {
        a.tokens[r] = (int32_t)token;
        if (a.logp) a.logp[r] = greedy ? 0.f : (float)(log(weight(logit_at(row, token))) - log(total));
    }
}

size_t draw_workspace_bytes(int, int) { return 256; }

hipError_t launch_draw(const DrawArgs& a, int dtype, const float* temperature, const int32_t* top_k, const float* top_p, const float* min_p,
                       void*, hipStream_t s) {
    const size_t size = dtype == SPIRAL_DTYPE_FP32 ? 4 : 2;
    for (int off = 0; off < a.B; off += kDrawRows) {
        DrawRows rows;
        const int n = a.B - off < kDrawRows ? a.B - off : kDrawRows;
        for (int i = 0; i < n; ++i) {
            rows.temperature[i] = temperature ? temperature[off + i] : 1.f;
            rows.top_k[i] = top_k ? top_k[off + i] : 0;
            rows.top_p[i] = top_p ? top_p[off + i] : 1.f;
            rows.min_p[i] = min_p ? min_p[off + i] : 0.f;
        }
        DrawArgs g = a;
        g.B = n;
        g.logits = (const char*)a.logits + (size_t)off * a.row_stride * size;
        g.uniform = a.uniform + off;
        g.tokens = a.tokens + off;
        g.logp = a.logp ? a.logp + off : nullptr;
        if (dtype == SPIRAL_DTYPE_FP32) hipLaunchKernelGGL(draw_row_kernel<float>, dim3(n), dim3(kThreads), 0, s, g, rows);
        else if (dtype == SPIRAL_DTYPE_BF16) hipLaunchKernelGGL(draw_row_kernel<__bf16>, dim3(n), dim3(kThreads), 0, s, g, rows);
        else hipLaunchKernelGGL(draw_row_kernel<_Float16>, dim3(n), dim3(kThreads), 0, s, g, rows);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace spiral
