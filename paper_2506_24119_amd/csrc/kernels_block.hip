// Rows of a decoder block, for the learner: addition to the residual stream with RMSNorm, and the norm and rotation of the q and k heads, each forward and backward.
//
// All are bound by memory: a row's elements are read once, kept in registers while their sum is formed, and written once.  Figures, other inputs each time (a copy of 4 GiB moves 4.8
// TB/s): addition + norm to 8 bits, 15,271 rows of 2,560 bf16, 274 MB in 51 us; gradient, 16,384 rows of 3,584 bf16, 470 MB in 97 us and 4.4 for the gain's sums; heads 32 + 8
// of 128, 15,271 rows bf16, 313 MB in 65 us; their gradient, 16,384 rows, 503 MB in 96 and 4.6.  A workgroup a row swept three times took 167, 298, and a wave a head with an angle of
// its own a lane 213 and 616.
#include <algorithm>

#include "spiral_internal.h"

namespace spiral {

namespace {

constexpr int kThreads = 256;
constexpr float kE4m3Least = 1e-30f;          // a row whose largest |out| is no more holds zeros

// Sums and maxima over a wave without a trip through LDS: rotations within rows of 16 lanes, then exchanges of rows.  Every lane adds the same pairs, so all have
// the same bits.
template <int N> __device__ __forceinline__ int row_ror(int x) { return __builtin_amdgcn_update_dpp(0, x, 0x120 + N, 0xF, 0xF, false); }
template <class Move, class Op> __device__ __forceinline__ float moved(float v, Move move, Op op) {
    const auto r = move(__float_as_int(v));
    return op(__int_as_float(r[0]), __int_as_float(r[1]));
}
template <class Move, class Op> __device__ __forceinline__ double moved(double v, Move move, Op op) {
    const auto lo = move(__double2loint(v)), hi = move(__double2hiint(v));
    return op(__hiloint2double(hi[0], lo[0]), __hiloint2double(hi[1], lo[1]));
}
template <class V, class Op> __device__ __forceinline__ V over_wave(V v, Op op) {
    typedef int Two __attribute__((ext_vector_type(2)));
    v = moved(v, [](int x) { return Two{x, row_ror<8>(x)}; }, op);
    v = moved(v, [](int x) { return Two{x, row_ror<4>(x)}; }, op);
    v = moved(v, [](int x) { return Two{x, row_ror<2>(x)}; }, op);
    v = moved(v, [](int x) { return Two{x, row_ror<1>(x)}; }, op);
    v = moved(v, [](int x) { const auto r = __builtin_amdgcn_permlane16_swap(x, x, false, false); return Two{(int)r[0], (int)r[1]}; }, op);
    return moved(v, [](int x) { const auto r = __builtin_amdgcn_permlane32_swap(x, x, false, false); return Two{(int)r[0], (int)r[1]}; }, op);
}
struct Add { __device__ __forceinline__ float operator()(float x, float y) const { return x + y; } };
struct Most { template <class V> __device__ __forceinline__ V operator()(V x, V y) const { return x != x || y != y ? (V)NAN : x > y ? x : y; } };      // undefined where any is
// over the WAVES waves that share a row
template <int WAVES, class V, class Op> __device__ __forceinline__ V over_row(V v, V* s, Op op) {
    v = over_wave(v, op);
    if (WAVES == 1) return v;
    __syncthreads();
    if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = v;
    __syncthreads();
    v = s[0];
#pragma unroll
    for (int w = 1; w < WAVES; ++w) v = op(v, s[w]);
    return v;
}

__device__ __forceinline__ uint8_t to_e4m3(float v) { return (uint8_t)(__builtin_amdgcn_cvt_pk_fp8_f32(v, v, 0, false) & 0xFF); }
__device__ __forceinline__ uint32_t to_e4m3x4(const float* v) {
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(v[2], v[3], __builtin_amdgcn_cvt_pk_fp8_f32(v[0], v[1], 0, false), true);
}
// Codes are those of the sum times the gain, exact in 64 bits, times 448 over the row's largest (1 / rms is in both and left out), rounded once.  Almost all of them 32 bits
// tell as well: where less and more than what can be off there give the same code.  (In 32 bits alone 25 of 39 M were others; in 64 bits alone the kernel takes 55 us, this way 51.)
// The sum itself is one of 64 bits where its parts are of 32 (in 32 bits half as many codes were others as with no 64 bits at all); of 16-bit parts 32 bits hold it, but for the last
// bits of parts 2^13 and more apart: one code in 10^8, for which the kernel would take 54 us.
template <class T> constexpr bool kWideSum = sizeof(T) == 4;
// six of 2^-24: the largest, the factor, its margin, the product and their product are off by one each; eight where the sum and that of the largest are, too
template <class T> constexpr float kOff = kWideSum<T> ? 0x1p-21f : 0x1.8p-22f;
__device__ __forceinline__ double exact_product(float x, float y) { return (double)x * y; }
__device__ __forceinline__ double exact_product(float x, float residual, float y) {
    const float sum = x + residual;
    return (fabsf(sum) < INFINITY ? (double)x + residual : (double)sum) * y;
}
// of 20 bits, the last one set where anything is cut off, so that the rounding to 4 bits goes the way it would from all of them
__device__ __forceinline__ float before_code(double v) { return (float)__hiloint2double(__double2hiint(v) | (int)min((uint32_t)__double2loint(v), 1u), 0); }
// Where the row's largest product is below this bound, those that still have a code may be subnormal in 32 bits, off by more than that, and below 2^-119.2 the factor passes 32
// bits; where it is infinite, the product of a finite sum and gain may be: such rows are left to the 64 bits (but for those that hold zeros in any case).
constexpr float kLeastProduct = 0x1p-100f;
__device__ __forceinline__ bool in_32_bits(float most, float rstd) { return (most >= kLeastProduct || (most + 0x1p-148f) * rstd < 0.99f * kE4m3Least) && most < INFINITY; }
// The larger magnitude, where what is infinite or undefined is larger than all that is not (asked for by comparisons the kernel took 51.7 us, this way 51.0)
__device__ __forceinline__ double larger(double x, double y) {
    const uint64_t a = __double_as_longlong(x), b = __double_as_longlong(fabs(y));
    return __longlong_as_double(a > b ? a : b);
}
// What the products are multiplied by, and what their codes are multiplied by to be decoded; undefined where the row's largest is undefined.
template <class V> __device__ __forceinline__ bool no_codes(V most, float rstd) { return most * rstd <= kE4m3Least; }
template <class V> __device__ __forceinline__ V code_factor(V most, float rstd) { return no_codes(most, rstd) ? (V)0 : (V)448 / most; }
template <class V> __device__ __forceinline__ float code_scale(V most, float rstd) { return no_codes(most, rstd) ? 0.f : (float)(most * rstd / (V)448); }

// Eight neighbouring elements, aligned to one: the wide accesses take any address
template <class T> struct Eight { typedef T type __attribute__((ext_vector_type(8), aligned(sizeof(T)))); };
template <class T> using Eights = typename Eight<T>::type;

// ONCE: a call that reads and writes more than the caches keep goes past their order of use.
template <bool ONCE, class E, class V> __device__ __forceinline__ void store(E* p, V x) {
    typedef V Any __attribute__((aligned(sizeof(E))));
    if constexpr (ONCE) __builtin_nontemporal_store(x, (Any*)p);
    else *(Any*)p = x;
}

// A lane's v-th eight elements of a row of d >= 8.  Those of the last v that would pass the row's end are read from d - 8 on, without a branch, and the first `skip` of
// them (all: 8) are another lane's: they are left out of sums and not written, as their place may hold the output already.
template <int LANES, int NV> struct Share {
    int t, d;
    __device__ __forceinline__ int begin(int v) const { return (v * LANES + t) * 8; }
    __device__ __forceinline__ int at(int v) const { return v < NV - 1 ? begin(v) : min(begin(v), d - 8); }
    __device__ __forceinline__ int skip(int v) const { return v < NV - 1 ? 0 : min(begin(v) - at(v), 8); }
    template <bool ONCE, class V, class E> __device__ __forceinline__ void put(E* row, int v, V x) const {
        const int n = skip(v);
        if (n == 0) store<ONCE>(row + at(v), x);
        else
#pragma unroll
            for (int e = 1; e < 8; ++e)
                if (e >= n) row[at(v) + e] = __builtin_bit_cast(E __attribute__((ext_vector_type(8))), x)[e];
    }
};
template <bool ONCE = false, class T> __device__ __forceinline__ Eights<T> eight(const T* p) {
    if constexpr (ONCE) return __builtin_nontemporal_load((const Eights<T>*)p);
    else return *(const Eights<T>*)p;
}
// What a second sweep over the same values widens again: kept from the first, they would take three times the registers (16,384 rows of 3,584 bf16: 160 us and spills, now 97).
template <class T> __device__ __forceinline__ void forget(Eights<T>& x) { asm volatile("" : "+v"(x)); }
template <> __device__ __forceinline__ void forget<float>(Eights<float>&) {}

// A row by one wave or by four, in registers: NV times eight elements a lane.  One read of what there is to read, one write; every load of a row is on its way before
// its first element is needed.
template <class T, bool OUT8, int WAVES, int NV, bool ONCE>
__global__ __launch_bounds__(kThreads, NV <= 2 ? 4 : NV <= 5 ? 3 : 2) void add_norm_kernel(NormRowsArgs a) {
    __shared__ float s[WAVES];
    __shared__ double s_most[WAVES];
    constexpr int LANES = 64 * WAVES;
    const Share<LANES, NV> mine{(int)(threadIdx.x % LANES), a.d};
    for (long long r = (long long)blockIdx.x * (4 / WAVES) + threadIdx.x / LANES; r < a.n_rows; r += (long long)gridDim.x * (4 / WAVES)) {
        const T* x = (const T*)a.x + r * a.x_stride;
        const T* res = a.residual ? (const T*)a.residual + r * a.residual_stride : nullptr;
        Eights<T> xv[NV], rv[NV];
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            xv[v] = eight<ONCE>(x + mine.at(v));
            if (res) rv[v] = eight<ONCE>(res + mine.at(v));
        }
        float h[NV][8], sq = 0.f;
#pragma unroll
        for (int v = 0; v < NV; ++v)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                h[v][e] = (float)xv[v][e] + (res ? (float)rv[v][e] : 0.f);
                const float in = e >= mine.skip(v) ? h[v][e] : 0.f;
                sq = fmaf(in, in, sq);
            }
        const float rstd = 1.f / sqrtf(over_row<WAVES>(sq, s, Add()) / a.d + a.eps);
        if (a.rstd && mine.t == 0) a.rstd[r] = rstd;
        float most = 0.f, bad = 0.f;              // bad: undefined where a product is infinite or undefined
        const float* gain = a.gain;
        const bool late = OUT8 && kWideSum<T> && (a.sum == a.x || a.sum == a.residual);      // over what open codes are made of
        auto put_sum = [&](int v) {
            if (!a.sum) return;
            Eights<T> y;
#pragma unroll
            for (int e = 0; e < 8; ++e) y[e] = (T)h[v][e];
            mine.template put<ONCE>((T*)a.sum + r * a.sum_stride, v, y);
        };
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            if (!late) put_sum(v);
            const Eights<float> g = eight(gain + mine.at(v));
            if (OUT8) {                           // (elements that are another lane's as well: they are of the same row)
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float p = h[v][e] * g[e];
                    most = fmaxf(most, fabsf(p));
                    bad = fmaf(p, 0.f, bad);
                }
            } else {
                Eights<T> y;
#pragma unroll
                for (int e = 0; e < 8; ++e) y[e] = (T)(h[v][e] * rstd * g[e]);      // (in this order: at most sqrt(d) times the gain on the way)
                mine.template put<ONCE>((T*)a.out + r * a.out_stride, v, y);
            }
        }
        if (OUT8) {
            typedef uint32_t Codes __attribute__((ext_vector_type(2)));
            most = over_row<WAVES>(bad != bad ? NAN : most, s, Most());
            const float factor = code_factor(most, rstd), less = factor * (1.f - kOff<T>), more = factor * (1.f + kOff<T>);
            if (mine.t == 0) a.out_scale[r] = code_scale(most, rstd);
            uint32_t differ = !in_32_bits(most, rstd);
            asm volatile("" : "+s"(gain));        // read again, not kept
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                const Eights<float> g = eight(gain + mine.at(v));
                float x[8], y[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) x[e] = h[v][e] * g[e] * less, y[e] = h[v][e] * g[e] * more;
                const Codes codes{to_e4m3x4(x), to_e4m3x4(x + 4)};
                differ |= (codes[0] ^ to_e4m3x4(y)) | (codes[1] ^ to_e4m3x4(y + 4));
                mine.template put<ONCE>((uint8_t*)a.out + r * a.out_stride, v, codes);
            }
            if (WAVES == 1 ? __builtin_amdgcn_ballot_w64(differ != 0) != 0 : __syncthreads_or(differ != 0)) {
                if constexpr (!kWideSum<T>) {
                    double exact = 0.0;
#pragma unroll
                    for (int v = 0; v < NV; ++v) {
                        asm volatile("" : "+s"(gain) : : "memory");      // eight at a time: a rare path is not to take registers from the other
                        const Eights<float> g = eight(gain + mine.at(v));
#pragma unroll
                        for (int e = 0; e < 8; ++e) exact = larger(exact, exact_product(h[v][e], g[e]));
                    }
                    exact = over_row<WAVES>(exact < INFINITY ? exact : (double)NAN, s_most, Most());
                    const double f = code_factor(exact, rstd);
                    if (!in_32_bits(most, rstd) && mine.t == 0) a.out_scale[r] = code_scale(exact, rstd);
#pragma unroll
                    for (int v = 0; v < NV; ++v) {
                        asm volatile("" : "+s"(gain) : : "memory");
                        const Eights<float> g = eight(gain + mine.at(v));
                        float x[8];
#pragma unroll
                        for (int e = 0; e < 8; ++e) asm volatile("" : "+v"(h[v][e]));      // nor widened values kept
#pragma unroll
                        for (int e = 0; e < 8; ++e) x[e] = before_code(exact_product(h[v][e], g[e]) * f);
                        mine.template put<ONCE>((uint8_t*)a.out + r * a.out_stride, v, Codes{to_e4m3x4(x), to_e4m3x4(x + 4)});
                    }
                } else {
                    // The elements that may be the largest and those whose codes are open, one by one, read again.  (All of them, from registers: 11.1 us for 200 rows of 8,192, this
                    // way 8.9, and 62 for 8,192 of 2,560, this way 63.)
                    const bool told = in_32_bits(most, rstd);
                    uint32_t largest = 0, open = 0;
                    if (told) {
#pragma unroll
                        for (int v = 0; v < NV; ++v) {
                            const Eights<float> g = eight(gain + mine.at(v));
                            float below[8], above[8];
#pragma unroll
                            for (int e = 0; e < 8; ++e) {
                                const float p = h[v][e] * g[e];
                                below[e] = p * less, above[e] = p * more;
                                if (fabsf(p) >= most * (1.f - kOff<T>)) largest |= 1u << (8 * v + e);
                            }
#pragma unroll
                            for (int b = 0; b < 8; b += 4) {
                                const uint32_t d = to_e4m3x4(below + b) ^ to_e4m3x4(above + b);
#pragma unroll
                                for (int e = 0; e < 4; ++e)
                                    if ((d >> (8 * e)) & 0xFF) open |= 1u << (8 * v + b + e);
                            }
                        }
                    } else largest = open = ~0u >> (32 - 8 * NV);
                    auto next = [&](uint32_t& left, int& v, int& e) { const int i = __builtin_ctz(left); left &= left - 1; v = i >> 3; e = i & 7; };
                    auto product = [&](int c) { return exact_product(x[c], res ? res[c] : 0.f, gain[c]); };
                    double exact = 0.0;
                    int v, e;
                    while (largest) {
                        next(largest, v, e);
                        exact = larger(exact, product(mine.at(v) + e));
                    }
                    exact = over_row<WAVES>(exact < INFINITY ? exact : (double)NAN, s_most, Most());
                    const double f = code_factor(exact, rstd);
                    if (!told && mine.t == 0) a.out_scale[r] = code_scale(exact, rstd);
                    while (open) {
                        next(open, v, e);
                        if (e >= mine.skip(v)) ((uint8_t*)a.out)[r * a.out_stride + mine.at(v) + e] = to_e4m3(before_code(product(mine.at(v) + e) * f));
                    }
                }
            }
#pragma unroll
            for (int v = 0; v < NV; ++v)
                if (late) put_sum(v);
        }
    }
}

// rows that registers do not hold, and those of fewer than eight elements: a row a workgroup, swept three times
template <class T>
__global__ __launch_bounds__(kThreads) void add_norm_long_kernel(NormRowsArgs a) {
    __shared__ float s[kThreads / 64];
    __shared__ double s_most[kThreads / 64];
    for (long long r = blockIdx.x; r < a.n_rows; r += gridDim.x) {
        const T* x = (const T*)a.x + r * a.x_stride;
        const T* res = a.residual ? (const T*)a.residual + r * a.residual_stride : nullptr;
        auto sum_at = [&](int c) { return (float)x[c] + (res ? (float)res[c] : 0.f); };
        auto product_at = [&](int c, float h) { return kWideSum<T> && res ? exact_product((float)x[c], (float)res[c], a.gain[c]) : exact_product(h, a.gain[c]); };
        float sq = 0.f;
        for (int c = threadIdx.x; c < a.d; c += kThreads) { const float h = sum_at(c); sq = fmaf(h, h, sq); }
        const float rstd = 1.f / sqrtf(over_row<4>(sq, s, Add()) / a.d + a.eps);
        if (a.rstd && threadIdx.x == 0) a.rstd[r] = rstd;
        double factor = 0.0;
        if (a.out_scale) {
            double most = 0.0;
            for (int c = threadIdx.x; c < a.d; c += kThreads) most = larger(most, product_at(c, sum_at(c)));
            most = over_row<4>(most < INFINITY ? most : (double)NAN, s_most, Most());
            factor = code_factor(most, rstd);
            if (threadIdx.x == 0) a.out_scale[r] = code_scale(most, rstd);
        }
        for (int c = threadIdx.x; c < a.d; c += kThreads) {
            const float h = sum_at(c), g = a.gain[c];
            if (a.out_scale) ((uint8_t*)a.out)[r * a.out_stride + c] = to_e4m3(before_code(product_at(c, h) * factor));
            else ((T*)a.out)[r * a.out_stride + c] = (T)(h * rstd * g);
            if (a.sum) ((T*)a.sum)[r * a.sum_stride + c] = (T)h;
        }
    }
}

// Gradient: rows as above, workgroups take every gridDim.x-th (group of four) and keep the gain's sums over their rows in registers.
template <class T, int WAVES, int NV, bool ONCE>
__global__ __launch_bounds__(kThreads, 2) void norm_grad_kernel(NormGradArgs a) {
    constexpr int LANES = 64 * WAVES;
    __shared__ float s[WAVES];
    const int d = a.d;
    const Share<LANES, NV> mine{(int)(threadIdx.x % LANES), d};
    float dg[NV][8] = {};
    for (long long r = (long long)blockIdx.x * (4 / WAVES) + threadIdx.x / LANES; r < a.n_rows; r += (long long)gridDim.x * (4 / WAVES)) {
        const T* dy = (const T*)a.dout + r * a.dout_stride;
        const T* h = (const T*)a.sum + r * a.sum_stride;
        const T* ds = a.dsum ? (const T*)a.dsum + r * a.dsum_stride : nullptr;
        Eights<T> yv[NV], hv[NV], sv[NV];
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            yv[v] = eight<ONCE>(dy + mine.at(v));
            hv[v] = eight<ONCE>(h + mine.at(v));
            if (ds) sv[v] = eight<ONCE>(ds + mine.at(v));
        }
        const float rstd = a.rstd[r];
        const float* gain = a.gain;
        float along = 0.f;
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const Eights<float> g = eight(gain + mine.at(v));
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float p = (float)yv[v][e] * ((float)hv[v][e] * rstd), in = e >= mine.skip(v) ? p : 0.f;
                along = fmaf(in, g[e], along);
                dg[v][e] += in;
            }
        }
        along = over_row<WAVES>(along, s, Add()) / d;
        asm volatile("" : "+s"(gain));            // read again, not kept, like the rest
        T* dx = (T*)a.dx + r * a.dx_stride;
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            forget<T>(yv[v]);
            forget<T>(hv[v]);
            const Eights<float> g = eight(gain + mine.at(v));
            Eights<T> x;
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = (T)(rstd * ((float)yv[v][e] * g[e] - (float)hv[v][e] * rstd * along) + (ds ? (float)sv[v][e] : 0.f));
            mine.template put<ONCE>(dx, v, x);
        }
    }
    if (!a.dgain) return;
    // the workgroup's sums: of four waves that had rows of their own, through LDS
    __shared__ float s_gain[WAVES == 1 ? 3 * 64 * 8 : 1];
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        if (WAVES == 1) {
            const int wave = threadIdx.x >> 6, t = mine.t;
            __syncthreads();
            if (wave)
#pragma unroll
                for (int e = 0; e < 8; ++e) s_gain[((wave - 1) * 8 + e) * 64 + t] = dg[v][e];
            __syncthreads();
            if (wave) continue;
#pragma unroll
            for (int w = 0; w < 3; ++w)
#pragma unroll
                for (int e = 0; e < 8; ++e) dg[v][e] += s_gain[(w * 8 + e) * 64 + t];
        }
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (e >= mine.skip(v)) a.part[(size_t)blockIdx.x * d + mine.at(v) + e] = dg[v][e];
    }
}
// Sums over the parts: 32 columns a workgroup, its 32 groups of 32 lanes take every 32nd part.
__global__ __launch_bounds__(1024) void add_parts_kernel(const float* part, long long parts, int d, float* out, float* out2, int split) {
    __shared__ float s[32][33];
    const int lane = threadIdx.x & 31, g = threadIdx.x >> 5, c = blockIdx.x * 32 + lane;
    float x = 0.f;
    if (c < d)
#pragma unroll 8
        for (long long p = g; p < parts; p += 32) x += part[(size_t)p * d + c];
    s[g][lane] = x;
    __syncthreads();
    if (g || c >= d) return;
    x = 0.f;
#pragma unroll
    for (int w = 0; w < 32; ++w) x += s[w][lane];
    float* to = c < split ? out : out2;
    if (to) to[c < split ? c : c - split] = x;
}

// rows that registers do not hold
template <class T>
__global__ __launch_bounds__(kThreads) void norm_grad_long_kernel(NormGradArgs a) {
    __shared__ float s[kThreads / 64];
    for (long long r = blockIdx.x; r < a.n_rows; r += gridDim.x) {
        const T* dy = (const T*)a.dout + r * a.dout_stride;
        const T* h = (const T*)a.sum + r * a.sum_stride;
        const float rstd = a.rstd[r];
        float along = 0.f;
        for (int c = threadIdx.x; c < a.d; c += kThreads) along = fmaf((float)dy[c] * a.gain[c], (float)h[c] * rstd, along);
        along = over_row<4>(along, s, Add()) / a.d;
        for (int c = threadIdx.x; c < a.d; c += kThreads) {
            float g = rstd * ((float)dy[c] * a.gain[c] - (float)h[c] * rstd * along);
            if (a.dsum) g += (float)((const T*)a.dsum)[r * a.dsum_stride + c];
            ((T*)a.dx)[r * a.dx_stride + c] = (T)g;
        }
    }
}
// their gain's sums, before dx may overwrite what they are made of: every gridDim.y-th row a part
template <class T>
__global__ __launch_bounds__(kThreads) void gain_part_kernel(NormGradArgs a) {
    const int c = blockIdx.x * kThreads + threadIdx.x;
    if (c >= a.d) return;
    float g = 0.f;
    for (long long r = blockIdx.y; r < a.n_rows; r += gridDim.y)
        g = fmaf((float)((const T*)a.dout)[r * a.dout_stride + c], (float)((const T*)a.sum)[r * a.sum_stride + c] * a.rstd[r], g);
    a.part[(size_t)blockIdx.y * a.d + c] = g;
}

// Cosine and sine of the eight angles position * freq of a lane, freq in turns: the turns' fraction and its quarter in 64 bits, then the Taylor polynomials of the at most
// pi / 4 that is left, off by 2^-29.
__device__ __forceinline__ void turn8(int position, const double* freq, float (&cs)[8], float (&sn)[8]) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const double turns = (double)position * freq[e], quarters = turns * 4.0, q = rint(quarters);
        const float x = (float)(quarters - q) * 1.57079632679489662f, x2 = x * x;
        const float si = fmaf(x * x2, fmaf(x2, fmaf(x2, fmaf(x2, 1.f / 362880.f, -1.f / 5040.f), 1.f / 120.f), -1.f / 6.f), x);
        const float co = fmaf(x2, fmaf(x2, fmaf(x2, fmaf(x2, fmaf(x2, -1.f / 3628800.f, 1.f / 40320.f), -1.f / 720.f), 1.f / 24.f), -0.5f), 1.f);
        const int k = (int)(long long)q & 3;
        const float c0 = k & 1 ? si : co, s0 = k & 1 ? co : si;
        cs[e] = k == 1 || k == 2 ? -c0 : c0;
        sn[e] = k & 2 ? -s0 : s0;
    }
}
// over the HD / 16 lanes that share a head, bit for bit the same in each: exchanges within four lanes, then of four with four
template <int HD> __device__ __forceinline__ float over_head(float v) {
    v += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0xB1, 0xF, 0xF, false));
    if (HD >= 64) v += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x4E, 0xF, 0xF, false));
    if (HD >= 128) v += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x141, 0xF, 0xF, false));
    return v;
}

// A row a wave.  HD / 16 lanes share a head: each has eight pairs (c, c + HD / 2) of neighbouring c, whose angles it evaluates once for all heads of the row.
template <class T, int HD, bool GRAD, bool ONCE>
__global__ __launch_bounds__(kThreads) void norm_rope_kernel(RopeArgs a, RopeFreq f) {
    constexpr int LANES = HD / 16, SLOTS = 64 / LANES;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c = (lane % LANES) * 8, slot = lane / LANES;
    float gain[2][2][8], dg[2][2][8];
    double freq[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) freq[e] = f.inv_freq[c + e];
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            gain[i][0][e] = a.side[i].gain ? a.side[i].gain[c + e] : 1.f;
            gain[i][1][e] = a.side[i].gain ? a.side[i].gain[c + HD / 2 + e] : 1.f;
            dg[i][0][e] = dg[i][1][e] = 0.f;
        }
    for (long long r = (long long)blockIdx.x * 4 + wave; r < a.n_rows; r += (long long)gridDim.x * 4) {
        float cs[8], sn[8];
        turn8(a.positions[r], freq, cs, sn);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const RopeSide& s = a.side[i];
            const T* x = (const T*)s.x + r * s.x_stride + c;
            const T* dy = (const T*)s.dout + r * s.dout_stride + c;
            T* out = (T*)s.out + r * s.out_stride + c;
            const bool norm = s.gain != nullptr;
            for (int h = slot; h < s.heads; h += SLOTS) {
                Eights<T> lo, hi, ylo, yhi;
                if (!GRAD || norm) lo = eight<ONCE>(x + h * HD), hi = eight<ONCE>(x + h * HD + HD / 2);
                if (GRAD) ylo = eight<ONCE>(dy + h * HD), yhi = eight<ONCE>(dy + h * HD + HD / 2);
                float rstd = 1.f;
                if (norm) {
                    float sq = 0.f;
#pragma unroll
                    for (int e = 0; e < 8; ++e) sq = fmaf((float)lo[e], (float)lo[e], fmaf((float)hi[e], (float)hi[e], sq));
                    rstd = 1.f / sqrtf(over_head<HD>(sq) / HD + a.eps);
                }
                Eights<T> olo, ohi;
                if (!GRAD) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        float p = (float)lo[e], q = (float)hi[e];
                        if (norm) p = p * rstd * gain[i][0][e], q = q * rstd * gain[i][1][e];
                        const float2 y = rotate_pair(p, q, cs[e], sn[e]);
                        olo[e] = (T)y.x; ohi[e] = (T)y.y;
                    }
                } else {
                    float p[8], q[8], along = 0.f;
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const float2 g = rotate_pair((float)ylo[e], (float)yhi[e], cs[e], -sn[e]);
                        p[e] = g.x; q[e] = g.y;
                        if (norm) {
                            const float u = (float)lo[e] * rstd, w = (float)hi[e] * rstd;
                            dg[i][0][e] = fmaf(g.x, u, dg[i][0][e]);
                            dg[i][1][e] = fmaf(g.y, w, dg[i][1][e]);
                            p[e] *= gain[i][0][e]; q[e] *= gain[i][1][e];
                            along = fmaf(p[e], u, fmaf(q[e], w, along));
                        }
                    }
                    if (norm) along = over_head<HD>(along) / HD;
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        olo[e] = (T)(norm ? rstd * (p[e] - (float)lo[e] * rstd * along) : p[e]);
                        ohi[e] = (T)(norm ? rstd * (q[e] - (float)hi[e] * rstd * along) : q[e]);
                    }
                }
                store<ONCE>(out + h * HD, olo);
                store<ONCE>(out + h * HD + HD / 2, ohi);
            }
        }
    }
    if (!GRAD || !a.part) return;
    // the gains' sums: over the slots of a wave, then the waves
    __shared__ float s_part[4][2 * HD];
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                float x = dg[i][b][e];
#pragma unroll
                for (int o = LANES; o < 64; o <<= 1) x += __shfl_xor(x, o, 64);
                if (slot == 0) s_part[wave][i * HD + b * (HD / 2) + c + e] = x;
            }
    __syncthreads();
    if (threadIdx.x < 2 * HD)
        a.part[(size_t)blockIdx.x * 2 * HD + threadIdx.x] = s_part[0][threadIdx.x] + s_part[1][threadIdx.x] + s_part[2][threadIdx.x] + s_part[3][threadIdx.x];
}

// ------------------------------------------------------------------------------------------------ launches
// A wave holds rows of up to kMostVecs times 512 elements (the gradient, which has three rows and a sum to hold, fewer: 3,584 bf16 by one wave 97 us and
// by four 98, but 4,096 by one spill), four waves, which also take shorter ones where there are few rows, four times as many.
constexpr int kFewRows = 2048;
constexpr long long kMostBlocks = 1 << 22;    // of a launch: workgroups of more rows take several
template <class T> constexpr int kMostVecs = sizeof(T) == 4 ? 4 : 8;
template <class T> constexpr int kMostGradVecs = sizeof(T) == 4 ? 4 : 6;
int norm_waves(long long n_rows, int d, int most_vecs) {      // 0: not in registers (fewer than eight elements neither)
    return d < 8 || d > 4 * 512 * most_vecs ? 0 : d > 512 * most_vecs || n_rows < kFewRows ? 4 : 1;
}
constexpr int kGradBlocks = 512, kLongParts = 128;
template <class T> long long norm_grad_parts(long long n_rows, int d) {
    const int waves = norm_waves(n_rows, d, kMostGradVecs<T>);
    return std::min<long long>(waves == 1 ? (n_rows + 3) / 4 : n_rows, waves ? kGradBlocks : kLongParts);
}
// Whether a call of so many bytes goes past the caches' order of use: from half of the largest one (256 MB) on.  Eight elements a lane are read or written once, and what the
// last call left or the next one takes does not stay anyway.  Between a launch that writes the inputs and one that reads the outputs (15,271 rows, 16,384 of gradients): norm to 8 bits
// 56 -> 45 us, its gradient 104 -> 96, rotation 69 -> 46, its gradient 105 -> 91.  With a quarter of the rows, 68 to 126 MB: 16.2 and 17.6, 30.0 and 31.8, 19.2 and 17.2, 31.3 and
// 31.9; with a thirty-second 5.2 and 5.8, 12.0, 8.6 and 9.3, 17 and 19.
bool passes_by(long long bytes) { return bytes >= 128ll << 20; }
unsigned at_most(long long blocks, long long most) { return (unsigned)(blocks < most ? blocks : most); }

template <class T, bool OUT8, int WAVES, bool ONCE> void add_norm_rows(const NormRowsArgs& a, hipStream_t s) {
    const dim3 grid(at_most((a.n_rows + 4 / WAVES - 1) / (4 / WAVES), kMostBlocks)), block(kThreads);
    switch ((a.d + 512 * WAVES - 1) / (512 * WAVES)) {
        case 1: hipLaunchKernelGGL((add_norm_kernel<T, OUT8, WAVES, 1, ONCE>), grid, block, 0, s, a); return;
        case 2: hipLaunchKernelGGL((add_norm_kernel<T, OUT8, WAVES, 2, ONCE>), grid, block, 0, s, a); return;
        case 3: hipLaunchKernelGGL((add_norm_kernel<T, OUT8, WAVES, 3, ONCE>), grid, block, 0, s, a); return;
        case 4: hipLaunchKernelGGL((add_norm_kernel<T, OUT8, WAVES, 4, ONCE>), grid, block, 0, s, a); return;
        case 5: if constexpr (kMostVecs<T> > 4) hipLaunchKernelGGL((add_norm_kernel<T, OUT8, WAVES, 5, ONCE>), grid, block, 0, s, a); return;
        case 6: if constexpr (kMostVecs<T> > 4) hipLaunchKernelGGL((add_norm_kernel<T, OUT8, WAVES, 6, ONCE>), grid, block, 0, s, a); return;
        case 7: if constexpr (kMostVecs<T> > 4) hipLaunchKernelGGL((add_norm_kernel<T, OUT8, WAVES, 7, ONCE>), grid, block, 0, s, a); return;
        case 8: if constexpr (kMostVecs<T> > 4) hipLaunchKernelGGL((add_norm_kernel<T, OUT8, WAVES, 8, ONCE>), grid, block, 0, s, a); return;
    }
}
template <class T, bool OUT8, bool ONCE> void add_norm_wide(const NormRowsArgs& a, int waves, hipStream_t s) {
    waves == 1 ? add_norm_rows<T, OUT8, 1, ONCE>(a, s) : add_norm_rows<T, OUT8, 4, ONCE>(a, s);
}
template <class T> hipError_t add_norm_of(const NormRowsArgs& a, hipStream_t s) {
    const int waves = norm_waves(a.n_rows, a.d, kMostVecs<T>);
    const bool out8 = a.out_scale != nullptr;
    if (!waves) hipLaunchKernelGGL((add_norm_long_kernel<T>), dim3(at_most(a.n_rows, kMostBlocks)), dim3(kThreads), 0, s, a);
    else if (passes_by(a.n_rows * a.d * (long long)(sizeof(T) * (1 + (a.residual != nullptr) + (a.sum != nullptr)) + (out8 ? 1 : sizeof(T)))))
        out8 ? add_norm_wide<T, true, true>(a, waves, s) : add_norm_wide<T, false, true>(a, waves, s);
    else out8 ? add_norm_wide<T, true, false>(a, waves, s) : add_norm_wide<T, false, false>(a, waves, s);
    return hipGetLastError();
}

template <class T, int WAVES, bool ONCE> void norm_grad_rows(const NormGradArgs& a, unsigned blocks, hipStream_t s) {
    const dim3 grid(blocks), block(kThreads);
    switch ((a.d + 512 * WAVES - 1) / (512 * WAVES)) {
        case 1: hipLaunchKernelGGL((norm_grad_kernel<T, WAVES, 1, ONCE>), grid, block, 0, s, a); return;
        case 2: hipLaunchKernelGGL((norm_grad_kernel<T, WAVES, 2, ONCE>), grid, block, 0, s, a); return;
        case 3: hipLaunchKernelGGL((norm_grad_kernel<T, WAVES, 3, ONCE>), grid, block, 0, s, a); return;
        case 4: hipLaunchKernelGGL((norm_grad_kernel<T, WAVES, 4, ONCE>), grid, block, 0, s, a); return;
        case 5: if constexpr (kMostGradVecs<T> > 4) hipLaunchKernelGGL((norm_grad_kernel<T, WAVES, 5, ONCE>), grid, block, 0, s, a); return;
        case 6: if constexpr (kMostGradVecs<T> > 4) hipLaunchKernelGGL((norm_grad_kernel<T, WAVES, 6, ONCE>), grid, block, 0, s, a); return;
    }
}
template <class T> hipError_t norm_grad_of(const NormGradArgs& a, hipStream_t s) {
    const int waves = norm_waves(a.n_rows, a.d, kMostGradVecs<T>);
    const long long parts = norm_grad_parts<T>(a.n_rows, a.d);
    if (!waves) {
        if (a.dgain) hipLaunchKernelGGL((gain_part_kernel<T>), dim3((a.d + kThreads - 1) / kThreads, (unsigned)parts), dim3(kThreads), 0, s, a);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        hipLaunchKernelGGL((norm_grad_long_kernel<T>), dim3(at_most(a.n_rows, kMostBlocks)), dim3(kThreads), 0, s, a);
    } else if (passes_by(a.n_rows * a.d * (long long)sizeof(T) * (3 + (a.dsum != nullptr))))
        waves == 1 ? norm_grad_rows<T, 1, true>(a, (unsigned)parts, s) : norm_grad_rows<T, 4, true>(a, (unsigned)parts, s);
    else waves == 1 ? norm_grad_rows<T, 1, false>(a, (unsigned)parts, s) : norm_grad_rows<T, 4, false>(a, (unsigned)parts, s);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || !a.dgain) return e;
    hipLaunchKernelGGL(add_parts_kernel, dim3((a.d + 31) / 32), dim3(1024), 0, s, a.part, parts, a.d, a.dgain, nullptr, a.d);
    return hipGetLastError();
}

constexpr int kRopeBlocks = 512;              // of the gradient: as many parts
int rope_grad_blocks(long long n_rows) { return (int)at_most((n_rows + 3) / 4, kRopeBlocks); }

template <class T, int HD> hipError_t rope_impl(const RopeArgs& a, const RopeFreq& f, bool grad, hipStream_t s) {
    const bool once = passes_by(a.n_rows * (a.side[0].heads + a.side[1].heads) * HD * (long long)sizeof(T) * (grad ? 3 : 2));
    if (!grad) {
        hipLaunchKernelGGL((once ? norm_rope_kernel<T, HD, false, true> : norm_rope_kernel<T, HD, false, false>), dim3(at_most((a.n_rows + 3) / 4, kMostBlocks)), dim3(kThreads), 0, s, a, f);
        return hipGetLastError();
    }
    const int blocks = rope_grad_blocks(a.n_rows);
    hipLaunchKernelGGL((once ? norm_rope_kernel<T, HD, true, true> : norm_rope_kernel<T, HD, true, false>), dim3(blocks), dim3(kThreads), 0, s, a, f);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || !a.part) return e;
    hipLaunchKernelGGL(add_parts_kernel, dim3(2 * HD / 32), dim3(1024), 0, s, a.part, (long long)blocks, 2 * HD, a.side[0].dgain, a.side[1].dgain, HD);
    return hipGetLastError();
}
template <class T> hipError_t rope_of(const RopeArgs& a, const RopeFreq& f, int hd, bool grad, hipStream_t s) {
    return hd == 32 ? rope_impl<T, 32>(a, f, grad, s) : hd == 64 ? rope_impl<T, 64>(a, f, grad, s) : rope_impl<T, 128>(a, f, grad, s);
}
hipError_t rope_any(const RopeArgs& a, const RopeFreq& f, int dtype, int hd, bool grad, hipStream_t s) {
    return dtype == SPIRAL_DTYPE_FP32 ? rope_of<float>(a, f, hd, grad, s) : dtype == SPIRAL_DTYPE_BF16 ? rope_of<__bf16>(a, f, hd, grad, s) : rope_of<_Float16>(a, f, hd, grad, s);
}

}  // namespace

hipError_t launch_add_norm_rows(const NormRowsArgs& a, int dtype, hipStream_t s) {
    return dtype == SPIRAL_DTYPE_FP32 ? add_norm_of<float>(a, s) : dtype == SPIRAL_DTYPE_BF16 ? add_norm_of<__bf16>(a, s) : add_norm_of<_Float16>(a, s);
}
// as many parts as any type's rows of that width are cut into
size_t norm_grad_workspace_bytes(long long n_rows, int d) {
    const bool long_rows = d < 8 || d > 4 * 512 * std::max(kMostGradVecs<float>, kMostGradVecs<__bf16>);
    return (size_t)std::min<long long>(n_rows, long_rows ? kLongParts : kGradBlocks) * d * 4;
}
hipError_t launch_norm_grad(const NormGradArgs& a, int dtype, hipStream_t s) {
    return dtype == SPIRAL_DTYPE_FP32 ? norm_grad_of<float>(a, s) : dtype == SPIRAL_DTYPE_BF16 ? norm_grad_of<__bf16>(a, s) : norm_grad_of<_Float16>(a, s);
}
hipError_t launch_norm_rope(const RopeArgs& a, const RopeFreq& f, int dtype, int hd, hipStream_t s) { return rope_any(a, f, dtype, hd, false, s); }
size_t norm_rope_grad_workspace_bytes(long long n_rows, int hd) { return (size_t)rope_grad_blocks(n_rows) * 2 * hd * 4; }
hipError_t launch_norm_rope_grad(const RopeArgs& a, const RopeFreq& f, int dtype, int hd, hipStream_t s) { return rope_any(a, f, dtype, hd, true, s); }

}  // namespace spiral
