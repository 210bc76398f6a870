// Log-probabilities of given tokens and the gradient of the policy objective in the logits.
#include "spiral_internal.h"

namespace spiral {

namespace {

constexpr int kThreads = 256;

template <class T> __device__ __forceinline__ float get(const T* p, size_t i) { return (float)p[i]; }
template <class T> __device__ __forceinline__ void put(T* p, size_t i, float v) { p[i] = (T)v; }

}  // namespace

// d(-scale J)/d logit_v = slope (p_v - 1{v = target}),  slope = scale mask A r [r A <= clip(r) A] / T, or without the ratio: scale mask A / T
__device__ __forceinline__ float policy_slope(const GradArgs& a, long long row, float logp) {
    const float A = a.advantage[row];
    float d = logp == logp ? A : NAN;
    if (a.logp_old) {
        const float r = expf(logp - a.logp_old[row]);
        const float rc = fminf(fmaxf(r, 1.f - a.clip_eps), 1.f + a.clip_eps);
        d = r * A <= rc * A ? r * A : r * A > rc * A ? 0.f : NAN;
    }
    return d * (a.scale * a.inv_t);
}

// A row by a workgroup: one sweep for the maximum and the sum, one for the gradient.
template <class T>
__global__ __launch_bounds__(kThreads) void policy_grad_kernel(GradArgs a) {
    __shared__ float s_m[kThreads / 64], s_s[kThreads / 64];
    const long long row = blockIdx.x;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const T* lr = (const T*)a.logits + (size_t)row * a.row_stride;
    T* gr = (T*)a.grad + (size_t)row * a.grad_stride;
    const int target = a.targets[row];
    if (target < 0 || (a.mask && a.mask[row] == 0)) {
        for (uint32_t v = tid; v < (uint32_t)a.V; v += kThreads) put(gr, v, 0.f);
        if (tid == 0) a.logp[row] = 0.f;
        return;
    }
    const float zt = target < a.V ? get(lr, target) * a.inv_t : NAN;       // read before an element of a gradient in place is written
    float m = -INFINITY, s = 0.f;
    for (uint32_t v = tid; v < (uint32_t)a.V; v += kThreads) {
        const float z = get(lr, v) * a.inv_t;
        if (z > m) { s = s * expf(m - z) + 1.f; m = z; }
        else if (z != -INFINITY) s += expf(z - m);
    }
    auto join = [](float& m, float& s, float om, float os) {
        const float mm = fmaxf(m, om);
        s = (m == mm ? s : s * expf(m - mm)) + (om == mm ? os : os * expf(om - mm));
        m = mm;
    };
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) join(m, s, __shfl_xor(m, o, 64), __shfl_xor(s, o, 64));
    if (lane == 0) { s_m[wave] = m; s_s[wave] = s; }
    __syncthreads();
    m = s_m[0]; s = s_s[0];
    for (int w = 1; w < kThreads / 64; ++w) join(m, s, s_m[w], s_s[w]);
    if (m == -INFINITY || m == INFINITY) s = NAN;                        // a row without a distribution
    const float log_sum = logf(s);
    const float logp = (zt - m) - log_sum;
    if (tid == 0) a.logp[row] = logp;
    const float slope = policy_slope(a, row, logp);
    const float c = slope / s;
    for (uint32_t v = tid; v < (uint32_t)a.V; v += kThreads) {
        const float p = c * expf(get(lr, v) * a.inv_t - m);
        put(gr, v, (int)v == target ? p - slope : p);
    }
}

size_t policy_grad_workspace_bytes(long long, int) { return 256; }

hipError_t launch_policy_grad(const GradArgs& a, int dtype, void*, hipStream_t s) {
    if (dtype == SPIRAL_DTYPE_FP32) hipLaunchKernelGGL(policy_grad_kernel<float>, dim3((unsigned)a.n_rows), dim3(kThreads), 0, s, a);
    else if (dtype == SPIRAL_DTYPE_BF16) hipLaunchKernelGGL(policy_grad_kernel<__bf16>, dim3((unsigned)a.n_rows), dim3(kThreads), 0, s, a);
    else hipLaunchKernelGGL(policy_grad_kernel<_Float16>, dim3((unsigned)a.n_rows), dim3(kThreads), 0, s, a);
    return hipGetLastError();
}

}  // namespace spiral
