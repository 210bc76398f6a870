// One AdamW step over many tensors: the global norm of the gradients, then the update.
#include "spiral_internal.h"

namespace spiral {

namespace {

constexpr int kThreads = 256;
constexpr int kPer = 8;                             // neighbouring elements of a thread; 32 threads have a block of 8-bit states
constexpr int kChunk = kThreads * kPer;
static_assert(kAdamwBlock == 32 * kPer, "a block is a half wave's");

__device__ __forceinline__ float load_as_f32(const void* p, int dtype, long long i) {
    if (dtype == SPIRAL_DTYPE_FP32) return ((const float*)p)[i];
    if (dtype == SPIRAL_DTYPE_BF16) return (float)((const __bf16*)p)[i];
    return (float)((const _Float16*)p)[i];
}
__device__ __forceinline__ void store_f32(void* p, int dtype, long long i, float v) {
    if (dtype == SPIRAL_DTYPE_FP32) ((float*)p)[i] = v;
    else if (dtype == SPIRAL_DTYPE_BF16) ((__bf16*)p)[i] = (__bf16)v;
    else ((_Float16*)p)[i] = (_Float16)v;
}

// the tensor that chunk `c` lies in: the last one whose first chunk is at most c
__device__ __forceinline__ int tensor_of(const AdamwRec* t, int n, long long c) {
    int lo = 0, hi = n - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (t[mid].first_chunk <= c) lo = mid;
        else hi = mid - 1;
    }
    return lo;
}

__device__ __forceinline__ double block_sum(double v, double* s) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
    if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = v;
    __syncthreads();
    v = 0.0;
    for (int w = 0; w < kThreads / 64; ++w) v += s[w];
    return v;
}

// e4m3 codes, nearest even
__device__ __forceinline__ float decode8(uint8_t c) { return __builtin_amdgcn_cvt_f32_fp8((int)c, 0); }
__device__ __forceinline__ uint8_t encode8(float v) { return (uint8_t)(__builtin_amdgcn_cvt_pk_fp8_f32(v, 0.f, 0, false) & 0xFF); }

// of a block whose largest magnitude is `most`: what its values are multiplied by to be encoded, and its codes to be decoded
__device__ __forceinline__ float code_factor(float most) { return most > kAdamwTiny ? kE4m3Max * (1.f / most) : 0.f; }
__device__ __forceinline__ float block_scale(float most) { return most > kAdamwTiny ? most * (1.f / kE4m3Max) : 0.f; }

__device__ __forceinline__ float half_wave_max(float v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor(v, o, 64));
    return v;
}

// Every operation of the moments is rounded by itself: an 8-bit code next to a border is then the one that any other evaluation in 32 bits comes to,
// and not, once in 10^5 elements, its neighbour, which moves the next step by a sixteenth.  (A fused multiply-add would be no faster: the kernel waits
// for memory.)
__device__ __forceinline__ void moments(const AdamwArgs& a, float g, float& m, float& v) {
#pragma clang fp contract(off)
    m = a.beta1 * m + a.rest1 * g;
    v = a.beta2 * v + a.rest2 * (g * g);
}

}  // namespace

// part[workgroup]: sum of squares of its chunks, in 64 bits (16-bit gradients of 1e20 square past 32); the order is fixed
__global__ __launch_bounds__(kThreads) void adamw_norm_kernel(AdamwArgs a) {
    __shared__ double s_sum[kThreads / 64];
    double sum = 0.0;
    const long long c0 = a.chunks * blockIdx.x / gridDim.x, c1 = a.chunks * (blockIdx.x + 1) / gridDim.x;
    int t = c0 < c1 ? tensor_of(a.table, a.n_tensors, c0) : 0;
    for (long long c = c0; c < c1; ++c) {
        while (t + 1 < a.n_tensors && a.table[t + 1].first_chunk <= c) ++t;
        const AdamwRec& r = a.table[t];
        const long long i0 = (c - r.first_chunk) * kChunk + threadIdx.x * kPer;
        for (int e = 0; e < kPer && i0 + e < r.n; ++e) {
            const double g = load_as_f32(r.grad, r.grad_dtype, i0 + e);
            sum = fma(g, g, sum);
        }
    }
    sum = block_sum(sum, s_sum);
    if (threadIdx.x == 0) a.part[blockIdx.x] = sum;
}

__global__ __launch_bounds__(kThreads) void adamw_step_kernel(AdamwArgs a) {
    __shared__ double s_sum[kThreads / 64];
    float clip = 1.f;
    if (a.n_part) {
        double sum = 0.0;
        for (int i = threadIdx.x; i < a.n_part; i += kThreads) sum += a.part[i];
        const float norm = (float)(sqrt(block_sum(sum, s_sum)) * fabs((double)a.grad_scale));
        if (a.norm && blockIdx.x == 0 && threadIdx.x == 0) *a.norm = norm;
        if (!(norm < INFINITY)) return;              // nothing is changed
        if (a.max_norm > 0.f && norm > a.max_norm) clip = a.max_norm / norm;
    }
    const long long c0 = a.chunks * blockIdx.x / gridDim.x, c1 = a.chunks * (blockIdx.x + 1) / gridDim.x;
    int t = c0 < c1 ? tensor_of(a.table, a.n_tensors, c0) : 0;
    for (long long c = c0; c < c1; ++c) {
        while (t + 1 < a.n_tensors && a.table[t + 1].first_chunk <= c) ++t;
        const AdamwRec& r = a.table[t];
        const long long i0 = (c - r.first_chunk) * kChunk + threadIdx.x * kPer;
        const int n = i0 < r.n ? (int)min((long long)kPer, r.n - i0) : 0;
        const bool codes = r.state_dtype == SPIRAL_DTYPE_E4M3;
        const long long blk = i0 / kAdamwBlock;
        const float keep = r.decay ? a.keep : 1.f;
        float ms = 0.f, vs = 0.f;
        if (codes && n) { ms = r.m_scale[blk]; vs = r.v_scale[blk]; }
        float m[kPer], q[kPer];                      // the moments; q: the second one, or its root for 8 bits
        float m_most = 0.f, q_most = 0.f;
        for (int e = 0; e < kPer; ++e) {
            m[e] = q[e] = 0.f;
            if (e >= n) continue;
            const long long i = i0 + e;
            const float g = load_as_f32(r.grad, r.grad_dtype, i) * a.grad_scale * clip;
            const float p = r.master ? r.master[i] : load_as_f32(r.param, r.param_dtype, i);
            float v;
            if (codes) {
                m[e] = decode8(((const uint8_t*)r.m)[i]) * ms;
                v = decode8(((const uint8_t*)r.v)[i]) * vs;
                v *= v;
            } else {
                m[e] = ((const float*)r.m)[i];
                v = ((const float*)r.v)[i];
            }
            moments(a, g, m[e], v);
            const float root = sqrtf(v);
            const float pn = p * keep - a.step_size * m[e] / (root * a.root_scale + a.eps);
            if (r.master) r.master[i] = pn;
            store_f32(r.param, r.param_dtype, i, pn);
            if (codes) {
                q[e] = root;
                m_most = fmaxf(m_most, fabsf(m[e]));
                q_most = fmaxf(q_most, root);
            } else {
                ((float*)r.m)[i] = m[e];
                ((float*)r.v)[i] = v;
            }
        }
        if (codes) {                                 // the same for all threads of a workgroup
            m_most = half_wave_max(m_most);
            q_most = half_wave_max(q_most);
            const float m_inv = code_factor(m_most), q_inv = code_factor(q_most);
            for (int e = 0; e < n; ++e) {
                ((uint8_t*)r.m)[i0 + e] = encode8(m[e] * m_inv);
                uint8_t code = encode8(q[e] * q_inv);
                if (code == 0 && q[e] > 0.f && q_inv > 0.f) code = 1;
                ((uint8_t*)r.v)[i0 + e] = code;
            }
            if (n && (threadIdx.x & 31) == 0) {
                r.m_scale[blk] = block_scale(m_most);
                r.v_scale[blk] = block_scale(q_most);
            }
        }
    }
}

long long adamw_chunks(long long n) { return (n + kChunk - 1) / kChunk; }

hipError_t launch_adamw(const AdamwArgs& a, hipStream_t s) {
    AdamwArgs g = a;
    const int wgs = (int)(a.chunks < kAdamwParts ? a.chunks : kAdamwParts);
    if (a.norm || a.max_norm > 0.f) {
        g.n_part = wgs;
        hipLaunchKernelGGL(adamw_norm_kernel, dim3(wgs), dim3(kThreads), 0, s, g);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    hipLaunchKernelGGL(adamw_step_kernel, dim3(wgs), dim3(kThreads), 0, s, g);
    return hipGetLastError();
}

}  // namespace spiral
