// What a decoder block has beside its matrix products and its attention, for the learner: addition to the residual stream with RMSNorm, and the
// norm and rotation of the q and k heads, each forward and backward.
#include "spiral_internal.h"

namespace spiral {

namespace {

constexpr int kThreads = 256;
constexpr float kE4m3Least = 1e-30f;          // a row whose largest |out| is no more holds zeros

template <int N> __device__ __forceinline__ float group_sum(float v, float* s) {       // of N waves, in every thread
    v = wave_sum(v);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = v;
    __syncthreads();
    v = 0.f;
#pragma unroll
    for (int w = 0; w < N; ++w) v += s[w];
    return v;
}
template <int N> __device__ __forceinline__ float group_max(float v, float* s) {       // NaN where any is
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) { const float x = __shfl_xor(v, o, 64); v = v != v || x != x ? NAN : fmaxf(v, x); }
    __syncthreads();
    if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = v;
    __syncthreads();
    v = s[0];
#pragma unroll
    for (int w = 1; w < N; ++w) v = v != v || s[w] != s[w] ? NAN : fmaxf(v, s[w]);
    return v;
}

__device__ __forceinline__ uint8_t to_e4m3(float v) { return (uint8_t)(__builtin_amdgcn_cvt_pk_fp8_f32(v, v, 0, false) & 0xFF); }

// a row a workgroup, swept three times
template <class T>
__global__ __launch_bounds__(kThreads) void add_norm_rows_kernel(NormRowsArgs a) {
    __shared__ float s[kThreads / 64];
    const long long r = blockIdx.x;
    const T* x = (const T*)a.x + r * a.x_stride;
    const T* res = a.residual ? (const T*)a.residual + r * a.residual_stride : nullptr;
    auto sum_at = [&](int c) { return (float)x[c] + (res ? (float)res[c] : 0.f); };
    float sq = 0.f;
    for (int c = threadIdx.x; c < a.d; c += kThreads) { const float h = sum_at(c); sq = fmaf(h, h, sq); }
    const float rstd = 1.f / sqrtf(group_sum<kThreads / 64>(sq, s) / a.d + a.eps);
    if (a.rstd && threadIdx.x == 0) a.rstd[r] = rstd;
    float inv = 0.f;
    if (a.out_scale) {
        float most = 0.f;
        for (int c = threadIdx.x; c < a.d; c += kThreads) {
            const float y = fabsf(sum_at(c) * rstd * a.gain[c]);
            most = most != most || y != y ? NAN : fmaxf(most, y);
        }
        most = group_max<kThreads / 64>(most, s);
        const bool some = !(most <= kE4m3Least);
        if (!(most < INFINITY)) most = NAN;
        inv = some ? 448.f / most : 0.f;
        if (threadIdx.x == 0) a.out_scale[r] = some ? most / 448.f : 0.f;
    }
    for (int c = threadIdx.x; c < a.d; c += kThreads) {
        const float h = sum_at(c), y = h * rstd * a.gain[c];
        if (a.sum) ((T*)a.sum)[r * a.sum_stride + c] = (T)h;
        if (a.out_scale) ((uint8_t*)a.out)[r * a.out_stride + c] = to_e4m3(y * inv);
        else ((T*)a.out)[r * a.out_stride + c] = (T)y;
    }
}

template <class T>
__global__ __launch_bounds__(kThreads) void norm_grad_kernel(NormGradArgs a) {
    __shared__ float s[kThreads / 64];
    const long long r = blockIdx.x;
    const T* dy = (const T*)a.dout + r * a.dout_stride;
    const T* h = (const T*)a.sum + r * a.sum_stride;
    const float rstd = a.rstd[r];
    float along = 0.f;
    for (int c = threadIdx.x; c < a.d; c += kThreads) along = fmaf((float)dy[c] * a.gain[c], (float)h[c] * rstd, along);
    along = group_sum<kThreads / 64>(along, s) / a.d;
    for (int c = threadIdx.x; c < a.d; c += kThreads) {
        float g = rstd * ((float)dy[c] * a.gain[c] - (float)h[c] * rstd * along);
        if (a.dsum) g += (float)((const T*)a.dsum)[r * a.dsum_stride + c];
        ((T*)a.dx)[r * a.dx_stride + c] = (T)g;
    }
}
constexpr int kGainRows = 128;                // rows of a partial sum
template <class T>
__global__ __launch_bounds__(kThreads) void gain_part_kernel(NormGradArgs a) {
    const int c = blockIdx.x * kThreads + threadIdx.x;
    if (c >= a.d) return;
    const long long r0 = (long long)blockIdx.y * kGainRows, r1 = r0 + kGainRows < a.n_rows ? r0 + kGainRows : a.n_rows;
    float g = 0.f;
    for (long long r = r0; r < r1; ++r) g = fmaf((float)((const T*)a.dout)[r * a.dout_stride + c], (float)((const T*)a.sum)[r * a.sum_stride + c] * a.rstd[r], g);
    a.part[(size_t)blockIdx.y * a.d + c] = g;
}
__global__ __launch_bounds__(kThreads) void add_parts_kernel(const float* part, long long parts, int d, float* out) {
    const int c = blockIdx.x * kThreads + threadIdx.x;
    if (c >= d) return;
    float g = 0.f;
    for (long long p = 0; p < parts; ++p) g += part[(size_t)p * d + c];
    out[c] = g;
}

// a head a wave: lane c holds the pair (c, c + HD / 2)
template <class T, int HD>
__global__ __launch_bounds__(kThreads) void norm_rope_kernel(RopeArgs a, RopeFreq f) {
    const int lane = threadIdx.x & 63, heads = a.side[0].heads + a.side[1].heads;
    const long long unit = (long long)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (unit >= a.n_rows * heads) return;
    const long long r = unit / heads;
    int h = (int)(unit % heads);
    const bool second = h >= a.side[0].heads;
    const RopeSide& s = a.side[second];
    if (second) h -= a.side[0].heads;
    const bool in = lane < HD / 2;
    const int c = in ? lane : 0;
    const T* x = (const T*)s.x + r * s.x_stride + h * HD;
    float lo = in ? (float)x[c] : 0.f, hi = in ? (float)x[c + HD / 2] : 0.f;
    if (s.gain) {
        const float rstd = 1.f / sqrtf(wave_sum(fmaf(lo, lo, hi * hi)) / HD + a.eps);
        lo *= rstd * s.gain[c];
        hi *= rstd * s.gain[c + HD / 2];
    }
    double sn, cs;
    sincos((double)a.positions[r] * f.inv_freq[c], &sn, &cs);
    const float2 y = rotate_pair(lo, hi, (float)cs, (float)sn);
    T* out = (T*)s.out + r * s.out_stride + h * HD;
    if (in) { out[c] = (T)y.x; out[c + HD / 2] = (T)y.y; }
}

constexpr int kRopeParts = 1024;              // workgroups of the backward kernel at most: partial sums of the gains' gradients
template <class T, int HD>
__global__ __launch_bounds__(kThreads) void norm_rope_grad_kernel(RopeArgs a, RopeFreq f) {
    __shared__ float s_part[4][2 * HD];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, heads = a.side[0].heads + a.side[1].heads;
    const bool in = lane < HD / 2;
    const int c = in ? lane : 0;
    float dg[2][2] = {};
    for (long long unit = (long long)blockIdx.x * 4 + wave; unit < a.n_rows * heads; unit += (long long)gridDim.x * 4) {
        const long long r = unit / heads;
        int h = (int)(unit % heads);
        const bool second = h >= a.side[0].heads;
        const RopeSide& s = a.side[second];
        if (second) h -= a.side[0].heads;
        const T* dy = (const T*)s.dout + r * s.dout_stride + h * HD;
        double sn, cs;
        sincos((double)a.positions[r] * f.inv_freq[c], &sn, &cs);
        float2 g = rotate_pair((float)dy[c], (float)dy[c + HD / 2], (float)cs, -(float)sn);
        if (s.gain) {
            const T* x = (const T*)s.x + r * s.x_stride + h * HD;
            float lo = in ? (float)x[c] : 0.f, hi = in ? (float)x[c + HD / 2] : 0.f;
            const float rstd = 1.f / sqrtf(wave_sum(fmaf(lo, lo, hi * hi)) / HD + a.eps);
            lo *= rstd; hi *= rstd;
            if (second) { dg[1][0] = fmaf(g.x, lo, dg[1][0]); dg[1][1] = fmaf(g.y, hi, dg[1][1]); }
            else        { dg[0][0] = fmaf(g.x, lo, dg[0][0]); dg[0][1] = fmaf(g.y, hi, dg[0][1]); }
            g.x *= s.gain[c]; g.y *= s.gain[c + HD / 2];
            const float along = wave_sum(in ? fmaf(g.x, lo, g.y * hi) : 0.f) / HD;
            g.x = rstd * (g.x - lo * along);
            g.y = rstd * (g.y - hi * along);
        }
        T* out = (T*)s.out + r * s.out_stride + h * HD;
        if (in) { out[c] = (T)g.x; out[c + HD / 2] = (T)g.y; }
    }
    if (!a.part) return;
    if (in) {
#pragma unroll
        for (int i = 0; i < 2; ++i) { s_part[wave][i * HD + c] = dg[i][0]; s_part[wave][i * HD + c + HD / 2] = dg[i][1]; }
    }
    __syncthreads();
    for (int e = threadIdx.x; e < 2 * HD; e += kThreads)
        a.part[(size_t)blockIdx.x * 2 * HD + e] = s_part[0][e] + s_part[1][e] + s_part[2][e] + s_part[3][e];
}
__global__ __launch_bounds__(kThreads) void rope_gain_kernel(const float* part, int parts, int hd, float* dq, float* dk) {
    const int e = threadIdx.x;
    if (e >= 2 * hd) return;
    float g = 0.f;
    for (int p = 0; p < parts; ++p) g += part[(size_t)p * 2 * hd + e];
    float* to = e < hd ? dq : dk;
    if (to) to[e % hd] = g;
}

int rope_grad_blocks(long long n_rows, int heads) {
    const long long units = (n_rows * heads + 3) / 4;
    return (int)(units < kRopeParts ? units : kRopeParts);
}

template <class T> hipError_t norm_grad_impl(const NormGradArgs& a, hipStream_t s) {
    hipLaunchKernelGGL((norm_grad_kernel<T>), dim3((unsigned)a.n_rows), dim3(kThreads), 0, s, a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || !a.dgain) return e;
    const int cols = (a.d + kThreads - 1) / kThreads;
    const long long parts = (a.n_rows + kGainRows - 1) / kGainRows;
    if (parts > 65535) return hipErrorInvalidValue;
    hipLaunchKernelGGL((gain_part_kernel<T>), dim3(cols, (unsigned)parts), dim3(kThreads), 0, s, a);
    if ((e = hipGetLastError()) != hipSuccess) return e;
    hipLaunchKernelGGL(add_parts_kernel, dim3(cols), dim3(kThreads), 0, s, a.part, parts, a.d, a.dgain);
    return hipGetLastError();
}

template <class T, int HD> hipError_t rope_impl(const RopeArgs& a, const RopeFreq& f, hipStream_t s) {
    const long long blocks = (a.n_rows * (a.side[0].heads + a.side[1].heads) + 3) / 4;
    if (blocks > 0x7FFFFFFF) return hipErrorInvalidValue;
    hipLaunchKernelGGL((norm_rope_kernel<T, HD>), dim3((unsigned)blocks), dim3(kThreads), 0, s, a, f);
    return hipGetLastError();
}
template <class T, int HD> hipError_t rope_grad_impl(const RopeArgs& a, const RopeFreq& f, hipStream_t s) {
    const int blocks = rope_grad_blocks(a.n_rows, a.side[0].heads + a.side[1].heads);
    hipLaunchKernelGGL((norm_rope_grad_kernel<T, HD>), dim3(blocks), dim3(kThreads), 0, s, a, f);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || !a.part) return e;
    hipLaunchKernelGGL(rope_gain_kernel, dim3(1), dim3(kThreads), 0, s, a.part, blocks, HD, a.side[0].dgain, a.side[1].dgain);
    return hipGetLastError();
}
template <class T> hipError_t rope_of(const RopeArgs& a, const RopeFreq& f, int hd, bool grad, hipStream_t s) {
    if (hd == 32) return grad ? rope_grad_impl<T, 32>(a, f, s) : rope_impl<T, 32>(a, f, s);
    if (hd == 64) return grad ? rope_grad_impl<T, 64>(a, f, s) : rope_impl<T, 64>(a, f, s);
    return grad ? rope_grad_impl<T, 128>(a, f, s) : rope_impl<T, 128>(a, f, s);
}
hipError_t rope_any(const RopeArgs& a, const RopeFreq& f, int dtype, int hd, bool grad, hipStream_t s) {
    return dtype == SPIRAL_DTYPE_FP32 ? rope_of<float>(a, f, hd, grad, s) : dtype == SPIRAL_DTYPE_BF16 ? rope_of<__bf16>(a, f, hd, grad, s) : rope_of<_Float16>(a, f, hd, grad, s);
}

}  // namespace

hipError_t launch_add_norm_rows(const NormRowsArgs& a, int dtype, hipStream_t s) {
    const dim3 grid((unsigned)a.n_rows), block(kThreads);
    if (dtype == SPIRAL_DTYPE_FP32) hipLaunchKernelGGL((add_norm_rows_kernel<float>), grid, block, 0, s, a);
    else if (dtype == SPIRAL_DTYPE_BF16) hipLaunchKernelGGL((add_norm_rows_kernel<__bf16>), grid, block, 0, s, a);
    else hipLaunchKernelGGL((add_norm_rows_kernel<_Float16>), grid, block, 0, s, a);
    return hipGetLastError();
}
size_t norm_grad_workspace_bytes(long long n_rows, int d) { return (size_t)((n_rows + kGainRows - 1) / kGainRows) * d * 4; }
hipError_t launch_norm_grad(const NormGradArgs& a, int dtype, hipStream_t s) {
    return dtype == SPIRAL_DTYPE_FP32 ? norm_grad_impl<float>(a, s) : dtype == SPIRAL_DTYPE_BF16 ? norm_grad_impl<__bf16>(a, s) : norm_grad_impl<_Float16>(a, s);
}
hipError_t launch_norm_rope(const RopeArgs& a, const RopeFreq& f, int dtype, int hd, hipStream_t s) { return rope_any(a, f, dtype, hd, false, s); }
size_t norm_rope_grad_workspace_bytes(long long n_rows, int n_heads, int hd) { return (size_t)rope_grad_blocks(n_rows, n_heads) * 2 * hd * 4; }
hipError_t launch_norm_rope_grad(const RopeArgs& a, const RopeFreq& f, int dtype, int hd, hipStream_t s) { return rope_any(a, f, dtype, hd, true, s); }

}  // namespace spiral
