// Causal attention over packed sequences, forward and backward, for the learner.
//
// A row alone: one wave computes one (row, head) of the outputs, of dq, or of dk and dv, token by token, and reads nothing that
// the row does not see.  All sums are fp32.
#include "spiral_internal.h"

namespace spiral {

namespace {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr float kLeast = -3.0e38f;            // below every score but -inf

template <class T> using Vec8 = T __attribute__((ext_vector_type(8)));

template <class T> __device__ __forceinline__ float dot8(const T* x, const T* y, float s) {
    const Vec8<T> a = *(const Vec8<T>*)x, b = *(const Vec8<T>*)y;
#pragma unroll
    for (int e = 0; e < 8; ++e) s = fmaf((float)a[e], (float)b[e], s);
    return s;
}
template <class T, int HD> __device__ __forceinline__ float dot(const T* x, const T* y) {
    float s = 0.f;
#pragma unroll 1
    for (int d = 0; d < HD; d += 8) s = dot8(x + d, y + d, s);
    return s;
}
__device__ __forceinline__ float wave_most(float v) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor(v, o, 64));
    return v;
}

// the sequence of a row: the last that starts at or before it and is not empty
__device__ __forceinline__ int sequence_of(const PackArgs& a, int row) {
    int lo = 0, hi = a.n_seqs;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (a.starts[mid] <= row) lo = mid; else hi = mid;
    }
    return lo;
}

// A lane holds dimensions lane and lane + 64 (HD = 32: the upper half of the wave repeats the lower)
template <int HD> constexpr int kDims = (HD + 63) / 64;

// out and lse of one row; k, v: the sequence's first row
template <class T, int HD>
__device__ void forward_row(const PackArgs& a, const T* k, const T* v, const T* q, int last, T* out, float* lse, int lane) {
    constexpr int DL = kDims<HD>;
    float m = kLeast, l = 0.f, o[DL] = {};
    for (int t0 = 0; t0 <= last; t0 += 64) {
        const int t = t0 + lane;
        const float s = t <= last ? dot<T, HD>(q, k + (size_t)t * a.k_stride) * a.scale_log2e : -INFINITY;
        const float m_new = fmaxf(m, wave_most(s)), shrink = exp2f(m - m_new);
        const float p = exp2f(s - m_new);
        l = l * shrink + wave_sum(t <= last ? p : 0.f);
        m = m_new;
#pragma unroll
        for (int j = 0; j < DL; ++j) o[j] *= shrink;
        for (int i = 0; i < 64 && t0 + i <= last; ++i) {
            const float pi = __shfl(p, i, 64);
            const T* row = v + (size_t)(t0 + i) * a.v_stride;
#pragma unroll
            for (int j = 0; j < DL; ++j) o[j] = fmaf(pi, (float)row[(lane + 64 * j) & (HD - 1)], o[j]);
        }
    }
#pragma unroll
    for (int j = 0; j < DL; ++j)
        if (lane + 64 * j < HD) out[lane + 64 * j] = (T)(o[j] / l);
    if (lane == 0) *lse = (m + log2f(l)) * kLn2;
}

// dq of one row
template <class T, int HD>
__device__ void dq_row(const PackArgs& a, const T* k, const T* v, const T* q, const T* dout, float lse, float delta, int last, T* dq, int lane) {
    constexpr int DL = kDims<HD>;
    float g[DL] = {};
    const float lse2 = lse * kLog2e;
    for (int t0 = 0; t0 <= last; t0 += 64) {
        const int t = t0 + lane;
        float ds = 0.f;
        if (t <= last) {
            const float p = exp2f(dot<T, HD>(q, k + (size_t)t * a.k_stride) * a.scale_log2e - lse2);
            ds = p * (dot<T, HD>(dout, v + (size_t)t * a.v_stride) - delta);
        }
        for (int i = 0; i < 64 && t0 + i <= last; ++i) {
            const float di = __shfl(ds, i, 64);
            const T* row = k + (size_t)(t0 + i) * a.k_stride;
#pragma unroll
            for (int j = 0; j < DL; ++j) g[j] = fmaf(di, (float)row[(lane + 64 * j) & (HD - 1)], g[j]);
        }
    }
#pragma unroll
    for (int j = 0; j < DL; ++j)
        if (lane + 64 * j < HD) dq[lane + 64 * j] = (T)(g[j] * a.scale);
}

// dk and dv of one token and kv head; row0: the sequence's first row, len: its length, t: the token's position
template <class T, int HD>
__device__ void dkv_row(const PackArgs& a, int row0, int len, int t, int kvh, int lane) {
    constexpr int DL = kDims<HD>;
    const int G = a.n_q_heads / a.n_kv_heads;
    const T* k = (const T*)a.k + (size_t)(row0 + t) * a.k_stride + kvh * HD;
    const T* v = (const T*)a.v + (size_t)(row0 + t) * a.v_stride + kvh * HD;
    float gk[DL] = {}, gv[DL] = {};
    for (int h = kvh * G; h < (kvh + 1) * G; ++h) {
        const T* q = (const T*)a.q + (size_t)row0 * a.q_stride + h * HD;
        const T* dout = (const T*)a.dout + (size_t)row0 * a.dout_stride + h * HD;
        const float* lse = a.lse + (size_t)h * a.n_rows + row0;
        const float* delta = a.delta + (size_t)h * a.n_rows + row0;
        for (int i0 = t; i0 < len; i0 += 64) {
            const int i = i0 + lane;
            float p = 0.f, ds = 0.f;
            if (i < len) {
                p = exp2f(dot<T, HD>(q + (size_t)i * a.q_stride, k) * a.scale_log2e - lse[i] * kLog2e);
                ds = p * (dot<T, HD>(dout + (size_t)i * a.dout_stride, v) - delta[i]);
            }
            for (int e = 0; e < 64 && i0 + e < len; ++e) {
                const float pe = __shfl(p, e, 64), de = __shfl(ds, e, 64);
                const T* qr = q + (size_t)(i0 + e) * a.q_stride;
                const T* dr = dout + (size_t)(i0 + e) * a.dout_stride;
#pragma unroll
                for (int j = 0; j < DL; ++j) {
                    gk[j] = fmaf(de, (float)qr[(lane + 64 * j) & (HD - 1)], gk[j]);
                    gv[j] = fmaf(pe, (float)dr[(lane + 64 * j) & (HD - 1)], gv[j]);
                }
            }
        }
    }
    T* dk = (T*)a.dk + (size_t)(row0 + t) * a.dk_stride + kvh * HD;
    T* dv = (T*)a.dv + (size_t)(row0 + t) * a.dv_stride + kvh * HD;
#pragma unroll
    for (int j = 0; j < DL; ++j)
        if (lane + 64 * j < HD) {
            dk[lane + 64 * j] = (T)(gk[j] * a.scale);
            dv[lane + 64 * j] = (T)gv[j];
        }
}

template <class T, int HD>
__global__ __launch_bounds__(256) void pack_forward_kernel(PackArgs a) {
    const int lane = threadIdx.x & 63, row = blockIdx.x * 4 + (threadIdx.x >> 6), h = blockIdx.y;
    if (row >= a.n_rows) return;
    const int first = a.starts[sequence_of(a, row)], kvh = h / (a.n_q_heads / a.n_kv_heads);
    forward_row<T, HD>(a, (const T*)a.k + (size_t)first * a.k_stride + kvh * HD, (const T*)a.v + (size_t)first * a.v_stride + kvh * HD,
                       (const T*)a.q + (size_t)row * a.q_stride + h * HD, row - first, (T*)a.out + (size_t)row * a.out_stride + h * HD,
                       a.lse + (size_t)h * a.n_rows + row, lane);
}

template <class T, int HD>
__global__ __launch_bounds__(256) void pack_dq_kernel(PackArgs a) {
    const int lane = threadIdx.x & 63, row = blockIdx.x * 4 + (threadIdx.x >> 6), h = blockIdx.y;
    if (row >= a.n_rows) return;
    const int first = a.starts[sequence_of(a, row)], kvh = h / (a.n_q_heads / a.n_kv_heads);
    const T* dout = (const T*)a.dout + (size_t)row * a.dout_stride + h * HD;
    const T* out = (const T*)a.out_in + (size_t)row * a.out_stride + h * HD;
    const float delta = wave_sum(lane < HD / 8 ? dot8(dout + lane * 8, out + lane * 8, 0.f) : 0.f);
    if (lane == 0) a.delta[(size_t)h * a.n_rows + row] = delta;
    dq_row<T, HD>(a, (const T*)a.k + (size_t)first * a.k_stride + kvh * HD, (const T*)a.v + (size_t)first * a.v_stride + kvh * HD,
                  (const T*)a.q + (size_t)row * a.q_stride + h * HD, dout, a.lse[(size_t)h * a.n_rows + row], delta, row - first,
                  (T*)a.dq + (size_t)row * a.dq_stride + h * HD, lane);
}

template <class T, int HD>
__global__ __launch_bounds__(256) void pack_dkv_kernel(PackArgs a) {
    const int lane = threadIdx.x & 63, row = blockIdx.x * 4 + (threadIdx.x >> 6);
    if (row >= a.n_rows) return;
    const int b = sequence_of(a, row), first = a.starts[b];
    dkv_row<T, HD>(a, first, a.starts[b + 1] - first, row - first, blockIdx.y, lane);
}

template <class T, int HD> hipError_t forward_impl(const PackArgs& a, hipStream_t s) {
    hipLaunchKernelGGL((pack_forward_kernel<T, HD>), dim3((unsigned)((a.n_rows + 3) / 4), a.n_q_heads), dim3(256), 0, s, a);
    return hipGetLastError();
}
template <class T, int HD> hipError_t backward_impl(const PackArgs& a, hipStream_t s) {
    const unsigned blocks = (unsigned)((a.n_rows + 3) / 4);
    hipLaunchKernelGGL((pack_dq_kernel<T, HD>), dim3(blocks, a.n_q_heads), dim3(256), 0, s, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((pack_dkv_kernel<T, HD>), dim3(blocks, a.n_kv_heads), dim3(256), 0, s, a);
    return hipGetLastError();
}

template <class T> hipError_t forward_of(const PackArgs& a, int hd, hipStream_t s) {
    return hd == 32 ? forward_impl<T, 32>(a, s) : hd == 64 ? forward_impl<T, 64>(a, s) : hd == 128 ? forward_impl<T, 128>(a, s) : hipErrorInvalidValue;
}
template <class T> hipError_t backward_of(const PackArgs& a, int hd, hipStream_t s) {
    return hd == 32 ? backward_impl<T, 32>(a, s) : hd == 64 ? backward_impl<T, 64>(a, s) : hd == 128 ? backward_impl<T, 128>(a, s) : hipErrorInvalidValue;
}

}  // namespace

hipError_t launch_pack_forward(const PackArgs& a, int dtype, int hd, hipStream_t s) {
    return dtype == SPIRAL_DTYPE_BF16 ? forward_of<__bf16>(a, hd, s) : forward_of<_Float16>(a, hd, s);
}
hipError_t launch_pack_backward(const PackArgs& a, int dtype, int hd, hipStream_t s) {
    return dtype == SPIRAL_DTYPE_BF16 ? backward_of<__bf16>(a, hd, s) : backward_of<_Float16>(a, hd, s);
}

}  // namespace spiral
