// One AdamW step over many tensors: the global norm of the gradients, then the update.
//
// Bound by memory: 28 bytes an element for bf16 weights with fp32 masters and states, 12 + 4 with 8-bit states, of which the norm's sweep reads the
// gradient's 2 once more.  A workgroup walks chunks of 4,096 elements of whatever tensor they fall in; all of a chunk's loads (4 runs of 4
// neighbouring elements a thread) are in flight before the first is used, four workgroups a compute unit (128 registers, no spill; five
// spill and gain 1% with 32-bit states, lose as much with 8-bit ones; chunks of 2,048 with eight: 9% and 5% slower).  Over 303 M elements, bf16 with masters: 1,676 us with 32-bit
// states (103 in the norm and 5.3 TB/s in the step, where a copy of 4 GiB moves 4.8), 1,027 us with 8-bit states.  What brought them there from 10,279 and 5,624 us: wide loads of any alignment, all
// ahead (2,005, 2,026); as many workgroups as fit (1,779, 1,627); streaming loads and stores that nothing else evicts the gradients for (1,685, 1,502); records by scalar loads instead of
// two dependent vector loads a chunk (8 bits: 1,108); chunks of four runs (1,670, 1,058).
// The update's quotient is a product with the hardware's reciprocal, off by one step of 2^-23 where a division would be by half of one; all else is fp32, each operation rounded.
#include "spiral_internal.h"

namespace spiral {

namespace {

constexpr int kThreads = 256;
constexpr int kPer = 4;                             // neighbouring elements of a thread: a wave has a block of 8-bit states
constexpr int kRun = kThreads * kPer;                // a workgroup's; a chunk is one of them or kLong
constexpr int kLong = 4, kLongWgs = 4;
static_assert(kAdamwBlock == 64 * kPer, "a block is a wave's");

// vectors that are aligned to an element only, as the tensors are: the wide loads take any address
typedef uint32_t Words __attribute__((ext_vector_type(kPer), aligned(4)));
typedef uint16_t Halves __attribute__((ext_vector_type(kPer), aligned(2)));
typedef uint8_t Bytes __attribute__((ext_vector_type(kPer), aligned(1)));

__device__ __forceinline__ float from16(uint16_t b, bool bf16) {
    return bf16 ? __uint_as_float((uint32_t)b << 16) : (float)__builtin_bit_cast(_Float16, b);
}
__device__ __forceinline__ uint16_t to16(float v, bool bf16) {
    return bf16 ? __builtin_bit_cast(uint16_t, (__bf16)v) : __builtin_bit_cast(uint16_t, (_Float16)v);
}

// The table is constant while a kernel runs: its records come by scalar loads.
typedef const __attribute__((address_space(4))) AdamwRec* Table;
__device__ __forceinline__ AdamwRec record(Table table, int t) {
    static_assert(sizeof(AdamwRec) % 8 == 0, "copied in words");
    const auto* from = (const __attribute__((address_space(4))) uint64_t*)(table + t);
    uint64_t words[sizeof(AdamwRec) / 8];
#pragma unroll
    for (int i = 0; i < (int)(sizeof(AdamwRec) / 8); ++i) words[i] = from[i];
    AdamwRec r;
    __builtin_memcpy(&r, words, sizeof(r));
    return r;
}

// the tensor that chunk `c` lies in: the last one whose first chunk is at most c; a wave looks at 64 of them at a time
__device__ __forceinline__ int tensor_of(Table table, int n, long long c) {
    int lo = 0, len = n;
    while (len > 1) {
        const int stride = (len + 63) >> 6, i = lo + (int)(threadIdx.x & 63) * stride;
        const bool at_most = i < lo + len && table[i].first_chunk <= c;
        const int last = (__popcll(__builtin_amdgcn_ballot_w64(at_most)) - 1) * stride;
        lo += last;
        len = min(stride, len - last);
    }
    return __builtin_amdgcn_readfirstlane(lo);
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

// of a block whose largest magnitude is `most`: what its values are multiplied by to be encoded, and its codes to be decoded
__device__ __forceinline__ float code_factor(float most) { return most > kAdamwTiny ? kE4m3Max * (1.f / most) : 0.f; }
__device__ __forceinline__ float block_scale(float most) { return most > kAdamwTiny ? most * (1.f / kE4m3Max) : 0.f; }

// of values that are not negative, as the integers that order them alike: four rotations within rows of 16 lanes, two exchanges of rows, and no trip
// through LDS
template <int N> __device__ __forceinline__ int row_ror(int x) { return __builtin_amdgcn_update_dpp(x, x, 0x120 + N, 0xF, 0xF, false); }
__device__ __forceinline__ float wave_max(float v) {
    int x = __float_as_int(v);
    x = max(x, row_ror<8>(x));
    x = max(x, row_ror<4>(x));
    x = max(x, row_ror<2>(x));
    x = max(x, row_ror<1>(x));
    auto r = __builtin_amdgcn_permlane16_swap(x, x, false, false);
    x = max((int)r[0], (int)r[1]);
    r = __builtin_amdgcn_permlane32_swap(x, x, false, false);
    return __int_as_float(max((int)r[0], (int)r[1]));
}

// Every operation of the moments is rounded by itself: an 8-bit code next to a border is then the one that any other evaluation in 32 bits comes to,
// and not, once in 10^5 elements, its neighbour, which moves the next step by a sixteenth.  (A fused multiply-add would be no faster: the kernel waits
// for memory.)
__device__ __forceinline__ void moments(const AdamwArgs& a, float g, float& m, float& v) {
#pragma clang fp contract(off)
    m = a.beta1 * m + a.rest1 * g;
    v = a.beta2 * v + a.rest2 * (g * g);
}

// Addresses that come out of a table in memory are not known to be global ones: flat accesses would count as LDS accesses too.
template <class T> using Global = __attribute__((address_space(1))) T;

// four neighbouring elements of a tensor, from i on; past its end they are zero and not written (FULL: none of the chunk's are).
// ONCE: nothing reads them again soon.
template <bool FULL, class W, bool ONCE = true, class T>
__device__ __forceinline__ W load4(const T* base, long long i, long long n) {
    const Global<T>* p = (const Global<T>*)base + i;
    W w = 0;
    if (FULL || i + kPer <= n) return ONCE ? __builtin_nontemporal_load((const Global<W>*)p) : *(const Global<W>*)p;
#pragma unroll
    for (int e = 0; e < kPer; ++e)
        if (i + e < n) w[e] = p[e];
    return w;
}
template <bool FULL, class W, class T>
__device__ __forceinline__ void store4(T* base, long long i, long long n, W w) {
    Global<T>* p = (Global<T>*)base + i;
    if (FULL || i + kPer <= n) { __builtin_nontemporal_store(w, (Global<W>*)p); return; }
#pragma unroll
    for (int e = 0; e < kPer; ++e)
        if (i + e < n) p[e] = w[e];
}

// STEPS runs of a tensor from `first` on.  Everything is loaded before anything is computed, and before `clip` is asked for, the factor of the norm, which
// the workgroup's first chunk waits for; it is negative where nothing is to be changed.
// G32: gradients of 32 bits.  P16: the parameter itself is read, of 16 bits without a master.  CODES: 8-bit states.
template <int STEPS, bool FULL, bool G32, bool P16, bool CODES, class Clip>
__device__ __forceinline__ void step_runs(const AdamwArgs& a, const AdamwRec& r, long long first, Clip& clip) {
    const long long n = r.n;
    Words g32[STEPS], p32[STEPS], m32[STEPS], v32[STEPS];
    Halves g16[STEPS], p16[STEPS];
    Bytes mc[STEPS], vc[STEPS];
    float ms[STEPS], vs[STEPS];
    const float* master = r.master ? r.master : (const float*)r.param;
#pragma unroll
    for (int k = 0; k < STEPS; ++k) {
        const long long i = first + k * kRun + threadIdx.x * kPer;
        if (G32) g32[k] = load4<FULL, Words>((const uint32_t*)r.grad, i, n);
        else g16[k] = load4<FULL, Halves>((const uint16_t*)r.grad, i, n);
        if (P16) p16[k] = load4<FULL, Halves>((const uint16_t*)r.param, i, n);
        else p32[k] = load4<FULL, Words>((const uint32_t*)master, i, n);
        if constexpr (CODES) {
            mc[k] = load4<FULL, Bytes>((const uint8_t*)r.m, i, n);
            vc[k] = load4<FULL, Bytes>((const uint8_t*)r.v, i, n);
            const long long blk = i / kAdamwBlock;
            ms[k] = FULL || i < n ? ((const Global<float>*)r.m_scale)[blk] : 0.f;
            vs[k] = FULL || i < n ? ((const Global<float>*)r.v_scale)[blk] : 0.f;
        } else {
            m32[k] = load4<FULL, Words>((const uint32_t*)r.m, i, n);
            v32[k] = load4<FULL, Words>((const uint32_t*)r.v, i, n);
        }
    }
    const float c = clip();
    if (c < 0.f) return;
    const bool g_bf16 = r.grad_dtype == SPIRAL_DTYPE_BF16, p_bf16 = r.param_dtype == SPIRAL_DTYPE_BF16;
    const float decay = r.decay ? a.decay : 0.f;
#pragma unroll
    for (int k = 0; k < STEPS; ++k) {
        const long long i = first + k * kRun + threadIdx.x * kPer;
        float m[kPer], v[kPer], p[kPer];
        float m_most = 0.f, q_most = 0.f;
        const uint32_t mw = CODES ? __builtin_bit_cast(uint32_t, mc[k]) : 0u, vw = CODES ? __builtin_bit_cast(uint32_t, vc[k]) : 0u;
        if (CODES) {
            m[0] = __builtin_amdgcn_cvt_f32_fp8(mw, 0); m[1] = __builtin_amdgcn_cvt_f32_fp8(mw, 1);
            m[2] = __builtin_amdgcn_cvt_f32_fp8(mw, 2); m[3] = __builtin_amdgcn_cvt_f32_fp8(mw, 3);
            v[0] = __builtin_amdgcn_cvt_f32_fp8(vw, 0); v[1] = __builtin_amdgcn_cvt_f32_fp8(vw, 1);
            v[2] = __builtin_amdgcn_cvt_f32_fp8(vw, 2); v[3] = __builtin_amdgcn_cvt_f32_fp8(vw, 3);
        }
#pragma unroll
        for (int e = 0; e < kPer; ++e) {
            const float g = (G32 ? __uint_as_float(g32[k][e]) : from16(g16[k][e], g_bf16)) * a.grad_scale * c;
            p[e] = P16 ? from16(p16[k][e], p_bf16) : __uint_as_float(p32[k][e]);
            if (CODES) {
                m[e] *= ms[k];
                v[e] *= vs[k];
                v[e] *= v[e];
            } else {
                m[e] = __uint_as_float(m32[k][e]);
                v[e] = __uint_as_float(v32[k][e]);
            }
            moments(a, g, m[e], v[e]);
            const float root = sqrtf(v[e]);
            // lr wd itself, not 1 - lr wd, which 32 bits know to 6e-8: at lr = 1e-6 a decay of 0.01 would be none and one of 0.1 a fifth too strong.  (An infinite
            // parameter, as fp16 may have without a master, stays what it is.)
            const float shrink = decay * __builtin_amdgcn_fmed3f(p[e], -3.402823466e38f, 3.402823466e38f);
            p[e] -= shrink + a.step_size * m[e] * __builtin_amdgcn_rcpf(root * a.root_scale + a.eps);
            if (CODES) {
                v[e] = root;
                m_most = fmaxf(m_most, fabsf(m[e]));
                q_most = fmaxf(q_most, root);
            }
        }
        Words out;
        if (!P16) {
#pragma unroll
            for (int e = 0; e < kPer; ++e) out[e] = __float_as_uint(p[e]);
            store4<FULL>((uint32_t*)master, i, n, out);
        }
        if (P16 || r.master) {
            Halves h;
#pragma unroll
            for (int e = 0; e < kPer; ++e) h[e] = to16(p[e], p_bf16);
            store4<FULL>((uint16_t*)r.param, i, n, h);
        }
        if (!CODES) {
#pragma unroll
            for (int e = 0; e < kPer; ++e) out[e] = __float_as_uint(m[e]);
            store4<FULL>((uint32_t*)r.m, i, n, out);
#pragma unroll
            for (int e = 0; e < kPer; ++e) out[e] = __float_as_uint(v[e]);
            store4<FULL>((uint32_t*)r.v, i, n, out);
        } else {
            m_most = wave_max(m_most);
            q_most = wave_max(q_most);
            const float mf = code_factor(m_most), qf = code_factor(q_most);
            int mo = __builtin_amdgcn_cvt_pk_fp8_f32(m[0] * mf, m[1] * mf, 0, false);
            mo = __builtin_amdgcn_cvt_pk_fp8_f32(m[2] * mf, m[3] * mf, mo, true);
            int vo = __builtin_amdgcn_cvt_pk_fp8_f32(v[0] * qf, v[1] * qf, 0, false);
            vo = __builtin_amdgcn_cvt_pk_fp8_f32(v[2] * qf, v[3] * qf, vo, true);
#pragma unroll
            for (int e = 0; e < kPer; ++e)          // a positive root keeps the least code at least
                if (qf > 0.f && v[e] > 0.f && (vo & (0xFF << (8 * e))) == 0) vo |= 1 << (8 * e);
            store4<FULL>((uint8_t*)r.m, i, n, __builtin_bit_cast(Bytes, mo));
            store4<FULL>((uint8_t*)r.v, i, n, __builtin_bit_cast(Bytes, vo));
            if ((threadIdx.x & 63) == 0 && (FULL || i < n)) {
                ((Global<float>*)r.m_scale)[i / kAdamwBlock] = block_scale(m_most);
                ((Global<float>*)r.v_scale)[i / kAdamwBlock] = block_scale(q_most);
            }
        }
    }
}

// A chunk: whole, all of it at once, else a run at a time.
template <int STEPS, bool G32, bool P16, bool CODES, class Clip>
__device__ __forceinline__ void step_chunk(const AdamwArgs& a, const AdamwRec& r, long long first, Clip& clip) {
    if (first + STEPS * kRun <= r.n) { step_runs<STEPS, true, G32, P16, CODES>(a, r, first, clip); return; }
#pragma unroll 1
    for (int k = 0; k < STEPS && first < r.n; ++k, first += kRun) step_runs<1, false, G32, P16, CODES>(a, r, first, clip);
}

template <int STEPS, bool G32, bool P16, class Clip>
__device__ __forceinline__ void step_any(const AdamwArgs& a, const AdamwRec& r, long long first, Clip& clip) {
    if (r.state_dtype == SPIRAL_DTYPE_E4M3) step_chunk<STEPS, G32, P16, true>(a, r, first, clip);
    else step_chunk<STEPS, G32, P16, false>(a, r, first, clip);
}

// A chunk's squares.  The loads leave the gradients in the last-level cache (256 MB), from which the step then has what fits.
template <int STEPS, bool FULL>
__device__ __forceinline__ double squares(const AdamwRec& r, long long first) {
    double sum = 0.0;
    if (r.grad_dtype == SPIRAL_DTYPE_FP32) {
        Words w[STEPS];
#pragma unroll
        for (int k = 0; k < STEPS; ++k) w[k] = load4<FULL, Words, false>((const uint32_t*)r.grad, first + k * kRun + threadIdx.x * kPer, r.n);
#pragma unroll
        for (int k = 0; k < STEPS; ++k)
#pragma unroll
            for (int e = 0; e < kPer; ++e) { const double g = __uint_as_float(w[k][e]); sum = fma(g, g, sum); }
    } else {
        const bool bf16 = r.grad_dtype == SPIRAL_DTYPE_BF16;
        Halves w[STEPS];
#pragma unroll
        for (int k = 0; k < STEPS; ++k) w[k] = load4<FULL, Halves, false>((const uint16_t*)r.grad, first + k * kRun + threadIdx.x * kPer, r.n);
#pragma unroll
        for (int k = 0; k < STEPS; ++k)
#pragma unroll
            for (int e = 0; e < kPer; ++e) { const double g = from16(w[k][e], bf16); sum = fma(g, g, sum); }
    }
    return sum;
}

}  // namespace

// part[workgroup]: sum of squares of its chunks, in 64 bits (16-bit gradients of 1e20 square past 32); the order is fixed
template <int STEPS>
__global__ __launch_bounds__(kThreads) void adamw_norm_kernel(AdamwArgs a) {
    __shared__ double s_sum[kThreads / 64];
    double sum = 0.0;
    const Table table = (Table)a.table;
    int t = tensor_of(table, a.n_tensors, blockIdx.x);
    for (long long c = blockIdx.x; c < a.chunks; c += gridDim.x) {
        while (t + 1 < a.n_tensors && table[t + 1].first_chunk <= c) ++t;
        const AdamwRec r = record(table, t);
        const long long first = (c - r.first_chunk) * (STEPS * kRun);
        sum += first + STEPS * kRun <= r.n ? squares<STEPS, true>(r, first) : squares<STEPS, false>(r, first);
    }
    sum = block_sum(sum, s_sum);
    if (threadIdx.x == 0) a.part[blockIdx.x] = sum;
}

template <int STEPS, int WGS>
__global__ __launch_bounds__(kThreads, WGS) void adamw_step_kernel(AdamwArgs a) {
    __shared__ double s_sum[kThreads / 64];
    const Table table = (Table)a.table;
    int t = tensor_of(table, a.n_tensors, blockIdx.x);
    float known = 0.f;                               // 0: not yet
    auto clip = [&] {
        if (known != 0.f) return known;
        known = 1.f;
        if (a.n_part) {
            double sum = 0.0;
            for (int i = threadIdx.x; i < a.n_part; i += kThreads) sum += a.part[i];
            const float norm = (float)(sqrt(block_sum(sum, s_sum)) * fabs((double)a.grad_scale));
            if (a.norm && blockIdx.x == 0 && threadIdx.x == 0) *a.norm = norm;
            if (a.max_norm > 0.f && norm > a.max_norm) known = fmaxf(a.max_norm / norm, 1e-45f);
            if (!(norm < INFINITY)) known = -1.f;
        }
        return known;
    };
    for (long long c = blockIdx.x; c < a.chunks && known >= 0.f; c += gridDim.x) {
        while (t + 1 < a.n_tensors && table[t + 1].first_chunk <= c) ++t;
        const AdamwRec r = record(table, t);
        const long long first = (c - r.first_chunk) * (STEPS * kRun);
        const bool p16 = r.param_dtype != SPIRAL_DTYPE_FP32 && !r.master;
        if (r.grad_dtype == SPIRAL_DTYPE_FP32) {
            if (p16) step_any<STEPS, true, true>(a, r, first, clip);
            else step_any<STEPS, true, false>(a, r, first, clip);
        } else {
            if (p16) step_any<STEPS, false, true>(a, r, first, clip);
            else step_any<STEPS, false, false>(a, r, first, clip);
        }
    }
}

// Chunks of one run as long as a long chunk would leave compute units without work: 2.6 M elements 20.9 us (73 MB: 15.7 in the step), with long ones 21.1.
int adamw_steps(long long elements) { return elements <= (long long)kAdamwParts * kRun * kLong ? 1 : kLong; }
long long adamw_chunks(long long n, int steps) { return (n + steps * kRun - 1) / (steps * kRun); }

template <int STEPS, int WGS>
static hipError_t launch_steps(const AdamwArgs& a, hipStream_t s) {
    AdamwArgs g = a;
    const long long most = 256 * WGS;
    const int wgs = (int)(a.chunks < most ? a.chunks : most);
    if (a.norm || a.max_norm > 0.f) {
        g.n_part = wgs;
        hipLaunchKernelGGL(adamw_norm_kernel<STEPS>, dim3(wgs), dim3(kThreads), 0, s, g);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    hipLaunchKernelGGL((adamw_step_kernel<STEPS, WGS>), dim3(wgs), dim3(kThreads), 0, s, g);
    return hipGetLastError();
}

hipError_t launch_adamw(const AdamwArgs& a, int steps, hipStream_t s) {
    return steps == 1 ? launch_steps<1, 8>(a, s) : launch_steps<kLong, kLongWgs>(a, s);
}

}  // namespace spiral
