// Log-probabilities of given tokens and the gradient of the policy objective in the logits.
//
// The slope of a row's gradient needs only the row itself (ratio, clip and advantage are its own), so one kernel does what a forward and a backward pass do:
// max and sum in one sweep, slope * (softmax - 1{target}) in a second.  Bound by memory: each logit once from HBM, each gradient once to it.  The second
// sweep reads what the first left in the last-level cache (512 rows of 304 KB at a time, of its 256 MB), but for what the threads have kept in
// registers.  4,096 rows of 151,936 bf16 logits, a third of them masked: 411 us by the clock, 5.1 TB/s of the 2.08 GB that have to be moved (425 in a trace; a copy of 4 GiB: 4.8); two
// sweeps of single elements by 256 threads took 1,574.  1,500 rows of as many fp32: 366 us, 5.0 TB/s.
//
// Exponentials are the hardware's exp2 of (l - m) (log2 e / T), the factor rounded once: off by up to 4 |z| + 4 of 2^-24, a little more than expf of (l - m) / T
// would be.  1 / T is rounded before it multiplies; scale / T is held in 64 bits.
#include "spiral_internal.h"

namespace spiral {

namespace {

constexpr float kLog2e = 1.4426950408889634f;
// When a row is cut into slices, and into how many: see policy_grad_slices.
constexpr int kSplitRows = 96, kSplitFrom = 16384, kSplitVecs = 1024, kSplitWgs = 1024;

// 16 bytes of a row, aligned to an element only: the wide loads take any address
template <class T> struct RowVec;
template <> struct RowVec<float> {
    static constexpr int N = 4, U = 4;               // elements; vectors whose loads are in flight together and that share a maximum
    typedef float type __attribute__((ext_vector_type(4), aligned(4)));
};
template <> struct RowVec<__bf16> {
    static constexpr int N = 8, U = 2;
    typedef __bf16 type __attribute__((ext_vector_type(8), aligned(2)));
};
template <> struct RowVec<_Float16> {
    static constexpr int N = 8, U = 2;
    typedef _Float16 type __attribute__((ext_vector_type(8), aligned(2)));
};

// The largest logit so far and the sum of exp2((l - m) c) over them: the softmax's pair, in one sweep.  An undefined logit stays in the sum,
// -inf adds nothing, also before there is any other.
struct Pair {
    float m = -INFINITY, s = 0.f;
    __device__ __forceinline__ void join(float om, float os, float c) {
        const float mm = fmaxf(m, om);
        if (mm == -INFINITY) { s += os; return; }              // 0 + 0, or undefined
        s = (m == mm ? s : s * exp2f((m - mm) * c)) + (om == mm ? os : os * exp2f((om - mm) * c));
        m = mm;
    }
};

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// d(-scale J)/d logit_v = slope (p_v - 1{v = target}),  slope = scale mask A r [r A <= clip(r) A] / T, or without the ratio: scale mask A / T
__device__ __forceinline__ float policy_slope(const GradArgs& a, long long row, float logp) {
    const float A = a.advantage[row];
    float d = logp == logp ? A : NAN;
    if (a.logp_old && A != 0.f) {                      // no advantage, no slope: not that of an infinite ratio either
        const float r = expf(logp - a.logp_old[row]);
        const float rc = fminf(fmaxf(r, 1.f - a.clip_eps), 1.f + a.clip_eps);
        d = r * A <= rc * A ? r * A : r * A > rc * A ? 0.f : NAN;
    }
    return (float)((double)d * a.unit);                // scale / T may pass 32 bits where the slope does not, and nothing times it is nothing
}

// U vectors' maximum, then their sum under it; those beyond the end (`in` says which) may count for the maximum: they repeat one that is there
template <class T, class In>
__device__ __forceinline__ void add(Pair& p, const typename RowVec<T>::type (&x)[RowVec<T>::U], In in, float c) {
    constexpr int N = RowVec<T>::N, U = RowVec<T>::U;
    float m = p.m;
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
        for (int e = 0; e < N; ++e) m = fmaxf(m, (float)x[u][e]);
    const float ref = m == -INFINITY ? 0.f : m;       // nothing yet: -inf adds 0 then, an undefined logit stays
    float s = p.s != 0.f ? p.s * exp2_fast((p.m - ref) * c) : 0.f;
#pragma unroll
    for (int u = 0; u < U; ++u)
        if (in(u))
#pragma unroll
            for (int e = 0; e < N; ++e) s += exp2_fast(((float)x[u][e] - ref) * c);
    p.m = m; p.s = s;
}
__device__ __forceinline__ void add_one(Pair& p, float l, float c) { p.join(l, l == l ? l == -INFINITY ? 0.f : 1.f : NAN, c); }

// the pairs of a workgroup's threads as one, in every thread
template <int WAVES>
__device__ __forceinline__ Pair join_all(Pair p, float c) {
    __shared__ float s_m[WAVES], s_s[WAVES];
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) p.join(__shfl_xor(p.m, o, 64), __shfl_xor(p.s, o, 64), c);
    if ((threadIdx.x & 63) == 0) { s_m[threadIdx.x >> 6] = p.m; s_s[threadIdx.x >> 6] = p.s; }
    __syncthreads();
    p = {};
    for (int w = 0; w < WAVES; ++w) p.join(s_m[w], s_s[w], c);
    return p;
}

// What a row's gradient follows from.
struct RowGrad {
    float m, c, slope, f;                             // f = slope / sum
    uint32_t target;
    __device__ __forceinline__ float operator()(float l) const { return f * exp2_fast((l - m) * c); }
    // the last elements of a row, one a thread
    template <class T> __device__ __forceinline__ void one(T* row, float l, uint32_t v) const { row[v] = (T)(v == target ? (*this)(l) - slope : (*this)(l)); }
    template <class T> __device__ __forceinline__ void vec(T* row, const typename RowVec<T>::type& x, uint32_t v) const {
        constexpr int N = RowVec<T>::N;
        typename RowVec<T>::type g;
#pragma unroll
        for (int e = 0; e < N; ++e) g[e] = (T)(*this)((float)x[e]);
        if (target / N == v) {
#pragma unroll
            for (int e = 0; e < N; ++e)
                if (target % N == e) g[e] = (T)((*this)((float)x[e]) - slope);
        }
        __builtin_nontemporal_store(g, (typename RowVec<T>::type*)(row + (size_t)v * N));
    }
};
__device__ __forceinline__ RowGrad row_grad(const GradArgs& a, long long row, int target, float target_logit, Pair p, bool tells) {
    if (p.m == -INFINITY || p.m == INFINITY) p.s = NAN;          // a row without a distribution
    const float logp = (target_logit - p.m) * a.inv_t - logf(p.s);
    if (tells) a.logp[row] = logp;
    const float slope = policy_slope(a, row, logp);
    return {p.m, a.inv_t * kLog2e, slope, slope / p.s, (uint32_t)target};
}

__device__ __forceinline__ bool counts(const GradArgs& a, long long row, int target) { return target >= 0 && !(a.mask && a.mask[row] == 0); }

// zeros for the vectors [v0, v1) of a row and, `left` of them, for its last elements
template <class T, int THREADS>
__device__ __forceinline__ void clear(T* row, uint32_t v0, uint32_t v1, uint32_t n_vec, uint32_t left) {
    constexpr int N = RowVec<T>::N;
    typename RowVec<T>::type zero = 0;
    for (uint32_t v = v0 + threadIdx.x; v < v1; v += THREADS) __builtin_nontemporal_store(zero, (typename RowVec<T>::type*)(row + (size_t)v * N));
    if (threadIdx.x < left) row[n_vec * N + threadIdx.x] = (T)0.f;
}

}  // namespace

// A row by a workgroup, which reads it once for the sum and once more for the gradient, from the last-level cache then, but for the first HOLD vectors
// of each thread, which stay in registers.  EU: waves a SIMD.
template <class T, int THREADS, int HOLD, int EU>
__global__ __launch_bounds__(THREADS, EU) void policy_grad_kernel(GradArgs a) {
    typedef typename RowVec<T>::type V;
    constexpr int N = RowVec<T>::N, U = RowVec<T>::U;
    static_assert(HOLD % U == 0, "held vectors are added in groups");
    const long long row = blockIdx.x;
    const uint32_t tid = threadIdx.x;
    const T* lr = (const T*)a.logits + (size_t)row * a.row_stride;
    T* gr = (T*)a.grad + (size_t)row * a.grad_stride;
    const uint32_t n_vec = (uint32_t)a.V / N, left = (uint32_t)a.V % N;
    const int target = a.targets[row];
    if (!counts(a, row, target)) {
        clear<T, THREADS>(gr, 0, n_vec, n_vec, left);
        if (tid == 0) a.logp[row] = 0.f;
        return;
    }
    const float zt = target < a.V ? (float)lr[target] : NAN;       // read before an element of a gradient in place is written
    const float c = a.inv_t * kLog2e;
    const float last = tid < left ? (float)lr[n_vec * N + tid] : -INFINITY;
    const V* lv = (const V*)lr;
    Pair p;
    V held[HOLD / U][U];
    if (n_vec) {
#pragma unroll
        for (int h = 0; h < HOLD; ++h) held[h / U][h % U] = lv[min(tid + h * THREADS, n_vec - 1)];
#pragma unroll
        for (int h = 0; h < HOLD / U; ++h) add<T>(p, held[h], [&](int u) { return tid + (h * U + u) * THREADS < n_vec; }, c);
    }
    for (uint32_t v0 = tid + HOLD * THREADS; v0 < n_vec; v0 += THREADS * U) {
        V x[U];
#pragma unroll
        for (int u = 0; u < U; ++u) x[u] = lv[min(v0 + u * THREADS, n_vec - 1)];
        add<T>(p, x, [&](int u) { return v0 + u * THREADS < n_vec; }, c);
    }
    add_one(p, last, c);
    p = join_all<THREADS / 64>(p, c);
    const RowGrad g = row_grad(a, row, target, zt, p, tid == 0);
    for (uint32_t v0 = tid + HOLD * THREADS; v0 < n_vec; v0 += THREADS * U) {
        V x[U];
#pragma unroll
        for (int u = 0; u < U; ++u) x[u] = lv[min(v0 + u * THREADS, n_vec - 1)];
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (v0 + u * THREADS < n_vec) g.vec(gr, x[u], v0 + u * THREADS);
    }
#pragma unroll
    for (int h = 0; h < HOLD; ++h)
        if (tid + h * THREADS < n_vec) g.vec(gr, held[h / U][h % U], tid + h * THREADS);
    if (tid < left) g.one(gr, last, n_vec * N + tid);
}

// Few rows: slices of `per` vectors, a workgroup each, in two launches.  The first leaves every slice's pair and the target's logit (which a gradient in
// place overwrites) in the workspace.
constexpr int kSliceThreads = 256;
template <class T>
__global__ __launch_bounds__(kSliceThreads) void policy_pair_kernel(GradArgs a, uint32_t per, float2* pairs, float* target_logit) {
    typedef typename RowVec<T>::type V;
    constexpr int N = RowVec<T>::N, U = RowVec<T>::U;
    const long long row = blockIdx.y;
    const uint32_t tid = threadIdx.x;
    const T* lr = (const T*)a.logits + (size_t)row * a.row_stride;
    const uint32_t n_vec = (uint32_t)a.V / N, left = blockIdx.x + 1 == gridDim.x ? (uint32_t)a.V % N : 0;
    const uint32_t v1 = min((blockIdx.x + 1) * per, n_vec);
    const int target = a.targets[row];
    if (!counts(a, row, target)) return;
    const float c = a.inv_t * kLog2e;
    const V* lv = (const V*)lr;
    Pair p;
    for (uint32_t v0 = blockIdx.x * per + tid; v0 < v1; v0 += kSliceThreads * U) {
        V x[U];
#pragma unroll
        for (int u = 0; u < U; ++u) x[u] = lv[min(v0 + u * kSliceThreads, v1 - 1)];
        add<T>(p, x, [&](int u) { return v0 + u * kSliceThreads < v1; }, c);
    }
    if (tid < left) add_one(p, (float)lr[n_vec * N + tid], c);
    p = join_all<kSliceThreads / 64>(p, c);
    if (tid == 0) {
        pairs[(size_t)row * gridDim.x + blockIdx.x] = make_float2(p.m, p.s);
        if (blockIdx.x == 0) target_logit[row] = target < a.V ? (float)lr[target] : NAN;
    }
}

template <class T>
__global__ __launch_bounds__(kSliceThreads) void policy_slice_kernel(GradArgs a, uint32_t per, const float2* pairs, const float* target_logit) {
    typedef typename RowVec<T>::type V;
    constexpr int N = RowVec<T>::N, U = RowVec<T>::U;
    const long long row = blockIdx.y;
    const uint32_t tid = threadIdx.x;
    const T* lr = (const T*)a.logits + (size_t)row * a.row_stride;
    T* gr = (T*)a.grad + (size_t)row * a.grad_stride;
    const uint32_t n_vec = (uint32_t)a.V / N, left = blockIdx.x + 1 == gridDim.x ? (uint32_t)a.V % N : 0;
    const uint32_t vs = min(blockIdx.x * per, n_vec), v1 = min(vs + per, n_vec);
    const int target = a.targets[row];
    if (!counts(a, row, target)) {
        clear<T, kSliceThreads>(gr, vs, v1, n_vec, left);
        if (blockIdx.x == 0 && tid == 0) a.logp[row] = 0.f;
        return;
    }
    const float c = a.inv_t * kLog2e;
    const V* lv = (const V*)lr;
    V x[U];                                          // the first are on their way while the pairs are joined
    if (vs < v1)
#pragma unroll
        for (int u = 0; u < U; ++u) x[u] = lv[min(vs + tid + u * kSliceThreads, v1 - 1)];
    Pair p;
    for (uint32_t i = tid; i < gridDim.x; i += kSliceThreads) {
        const float2 e = pairs[(size_t)row * gridDim.x + i];
        p.join(e.x, e.y, c);
    }
    p = join_all<kSliceThreads / 64>(p, c);
    const RowGrad g = row_grad(a, row, target, target_logit[row], p, blockIdx.x == 0 && tid == 0);
    for (uint32_t v0 = vs + tid; v0 < v1;) {
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (v0 + u * kSliceThreads < v1) g.vec(gr, x[u], v0 + u * kSliceThreads);
        v0 += kSliceThreads * U;
        if (v0 < v1)
#pragma unroll
            for (int u = 0; u < U; ++u) x[u] = lv[min(v0 + u * kSliceThreads, v1 - 1)];
    }
    if (tid < left) g.one(gr, (float)lr[n_vec * N + tid], n_vec * N + tid);
}

// A workgroup takes 21 us for 304 KB, however few of them there are: up to 96 rows of 256 KB or more are cut, into slices of at least 16 KB, as many as give
// every compute unit four.  Rows of 151,936 logits, uncut and cut: bf16 one 21.5 and 9.6 us, 64 of them 22.1 and 14.7, 96 22.7 and 18.8, 128 24.5 and 25.3; fp32 one 22.0 and 9.2, 64
// 24.7 and 23.5, 80 26.0 and 29.3, 96 28.6 and 33.6 (a line of their own, at 64, would save those 80 to 96 rows an eighth).  Shorter rows are done before a second
// launch is made (50,000 fp32 logits: 12.1 us uncut, 14.8 cut).
int policy_grad_slices(long long n_rows, int V, int dtype) {
    const long long vecs = V / (dtype == SPIRAL_DTYPE_FP32 ? 4 : 8);
    if (n_rows > kSplitRows || vecs < kSplitFrom) return 1;
    const long long most = vecs / kSplitVecs, want = kSplitWgs / n_rows;
    return (int)(want < 2 ? 2 : want < most ? want : most);
}

static size_t pairs_bytes(long long n_rows, int slices) { return ((size_t)n_rows * slices * sizeof(float2) + 255) & ~(size_t)255; }
size_t policy_grad_workspace_bytes(long long n_rows, int V) {
    int most = 1;
    for (const int dtype : {SPIRAL_DTYPE_FP32, SPIRAL_DTYPE_BF16}) {
        const int slices = policy_grad_slices(n_rows, V, dtype);
        most = slices > most ? slices : most;
    }
    return most == 1 ? 256 : pairs_bytes(n_rows, most) + (((size_t)n_rows * sizeof(float) + 255) & ~(size_t)255);
}

template <class T>
static hipError_t launch_some(const GradArgs& a, int slices, void* workspace, hipStream_t s) {
    const uint32_t n_vec = (uint32_t)a.V / RowVec<T>::N;
    if (slices > 1) {
        const uint32_t per = (n_vec + slices - 1) / slices;
        float2* pairs = (float2*)workspace;
        float* target_logit = (float*)((char*)workspace + pairs_bytes(a.n_rows, slices));
        const dim3 grid(slices, (unsigned)a.n_rows);
        hipLaunchKernelGGL(policy_pair_kernel<T>, grid, dim3(kSliceThreads), 0, s, a, per, pairs, target_logit);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        hipLaunchKernelGGL(policy_slice_kernel<T>, grid, dim3(kSliceThreads), 0, s, a, per, pairs, target_logit);
        return hipGetLastError();
    }
    // As many threads as hold the whole row in 8 vectors each (3,000 rows of 8,000 bf16 logits 22 us; by 1,024 threads 64 to 100).  Longer rows of 16-bit logits
    // keep 8 as well, two workgroups a compute unit (4,096 x 151,936: 411 us; with none 436, all 19 in one workgroup 704); 32-bit ones keep 20 and have the compute
    // unit for themselves (1,500 x 151,936: 366 us; 8 and two workgroups 390, none 454).
    const dim3 grid((unsigned)a.n_rows);
    constexpr bool WIDE = sizeof(T) == 4;
    if (n_vec <= 256 * 8) hipLaunchKernelGGL((policy_grad_kernel<T, 256, 8, 8>), grid, dim3(256), 0, s, a);
    else if (n_vec <= 512 * 8) hipLaunchKernelGGL((policy_grad_kernel<T, 512, 8, 8>), grid, dim3(512), 0, s, a);
    else if (n_vec <= 1024 * 8 || !WIDE) hipLaunchKernelGGL((policy_grad_kernel<T, 1024, 8, 8>), grid, dim3(1024), 0, s, a);
    else hipLaunchKernelGGL((policy_grad_kernel<T, 1024, WIDE ? 20 : 8, WIDE ? 4 : 8>), grid, dim3(1024), 0, s, a);
    return hipGetLastError();
}

// A launch has at most 2^32 threads: 2^20 rows at a time.
template <class T>
static hipError_t launch_rows(const GradArgs& a, int slices, void* workspace, hipStream_t s) {
    constexpr long long MOST = 1ll << 20;
    for (long long r = 0; r < a.n_rows; r += MOST) {
        GradArgs g = a;
        g.n_rows = a.n_rows - r < MOST ? a.n_rows - r : MOST;
        g.logits = (const T*)a.logits + r * a.row_stride;
        g.grad = (T*)a.grad + r * a.grad_stride;
        g.targets += r;
        if (g.logp_old) g.logp_old += r;
        g.advantage += r;
        if (g.mask) g.mask += r;
        g.logp += r;
        const hipError_t e = launch_some<T>(g, slices, workspace, s);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

hipError_t launch_policy_grad(const GradArgs& a, int dtype, void* workspace, hipStream_t s) {
    const int slices = policy_grad_slices(a.n_rows, a.V, dtype);
    return dtype == SPIRAL_DTYPE_FP32 ? launch_rows<float>(a, slices, workspace, s) : dtype == SPIRAL_DTYPE_BF16 ? launch_rows<__bf16>(a, slices, workspace, s)
         : launch_rows<_Float16>(a, slices, workspace, s);
}

}  // namespace spiral
