// One token a row from given uniform numbers: the inverse of the running sum of the kept weights, in index order.
//
// Rows of less than 16,384 logits are a workgroup's (draw_row).  Longer ones are pieces of 2,048, a wave's each, so that 128 rows fill the card and one row still
// has 75 waves; the sums of the pieces tell in which the number falls, and only that is looked at again.  An uncut batch is one sweep (draw_sum_kernel) and that
// (draw_pick_kernel): 128 x 151,936 fp32 logits 18.9 + 5.2 us, 4.1 TB/s in the sweep (bf16 21.7 us in all: the sweep takes as long for half the bytes).  Its 6.7 M vector instructions, 22 an
// entry and 14 of those in 64 bits, are 11 us of issue on every SIMD; the table's bank conflicts are 1 us, and the waves wait for half of their cycles.
// Cut batches: a sweep that counts entries in bins (draw_count_kernel, 18.2 us), the bins between which the cuts fall (draw_plan_kernel, 9.1), a sweep that sums what is
// kept for sure and lists the entries of those bins (draw_cut_kernel, 26.8), and the exact border among them (draw_pick_kernel, 13.9).  Counts are 32-bit LDS additions; 64-bit masses in
// the histogram would take 46 us.  The line, both sides measured, 16,383 and 16,384 fp32 logits: uncut one row 12.5 and 8.2 us, 128 rows 16.7 and 9.5; top-p 0.9 25.2 and
// 25.7, 29.5 and 28.7; top-k 50, which the workgroup finds in one sweep less, 18.5 and 21.6, 19.7 and 24.1.
//
// What is held in fewer bits than the weights: the masses between which a border is sought are whole numbers, of candidates multiples of 2^-50 of the largest weight (8,192 of them
// fit 64 bits), of a row by a workgroup of 2^-44 at 151,936 logits, so that they add up alike in any order.  A candidate lighter than 2^-51 of the largest has none, and
// a piece with nothing else is not drawn from: less than 2^-38 of the row, where the given numbers have 24 bits.  The weights of the token's own piece are summed as they are.
#include <type_traits>

#include "spiral_internal.h"

namespace spiral {

namespace {

// larger float <=> larger key; -0 and +0 share a key
__device__ __forceinline__ uint32_t order_key(float z) {
    const uint32_t b = __float_as_uint(z + 0.0f);
    return (b & 0x80000000u) ? ~b : (b | 0x80000000u);
}
__device__ __forceinline__ float key_value(uint32_t k) { return __uint_as_float((k & 0x80000000u) ? (k & 0x7FFFFFFFu) : ~k); }

__device__ __forceinline__ float clean(float l) { return fmaxf(l, -INFINITY); }      // an undefined logit is never drawn

// 16 bytes of a row, aligned to an element only: the wide loads take any address
template <class T> struct RowVec;
template <> struct RowVec<float> { static constexpr int N = 4; typedef float type __attribute__((ext_vector_type(4), aligned(4))); };
template <> struct RowVec<__bf16> { static constexpr int N = 8; typedef __bf16 type __attribute__((ext_vector_type(8), aligned(2))); };
template <> struct RowVec<_Float16> { static constexpr int N = 8; typedef _Float16 type __attribute__((ext_vector_type(8), aligned(2))); };

// Sums and maxima over a wave without a trip through LDS (an exchange of lanes there takes a hundred cycles, and a sum of 64 bits needs two for each of its six
// steps): within rows of 16 lanes by shifts, then the last lane of a row to the next row and that of the second to the third and fourth.  All lanes are active.
template <int CTRL, int ROWS> __device__ __forceinline__ uint32_t moved(uint32_t x, uint32_t none) {
    return (uint32_t)__builtin_amdgcn_update_dpp((int)none, (int)x, CTRL, ROWS, 0xF, false);
}
template <int CTRL, int ROWS> __device__ __forceinline__ uint64_t moved(uint64_t x) {
    return ((uint64_t)moved<CTRL, ROWS>((uint32_t)(x >> 32), 0u) << 32) | moved<CTRL, ROWS>((uint32_t)x, 0u);
}
template <int CTRL, int ROWS> __device__ __forceinline__ double moved(double x) {
    return __longlong_as_double((long long)moved<CTRL, ROWS>((uint64_t)__double_as_longlong(x)));
}
template <int CTRL, int ROWS> __device__ __forceinline__ uint32_t moved(uint32_t x) { return moved<CTRL, ROWS>(x, 0u); }
// the sum over the lanes up to this one
template <class V> __device__ __forceinline__ V wave_scan(V v) {
    v += moved<0x111, 0xF>(v);
    v += moved<0x112, 0xF>(v);
    v += moved<0x114, 0xF>(v);
    v += moved<0x118, 0xF>(v);
    v += moved<0x142, 0xA>(v);
    v += moved<0x143, 0xC>(v);
    return v;
}
__device__ __forceinline__ uint32_t last_lane(uint32_t v) { return (uint32_t)__builtin_amdgcn_readlane((int)v, 63); }
__device__ __forceinline__ uint64_t last_lane(uint64_t v) { return ((uint64_t)last_lane((uint32_t)(v >> 32)) << 32) | last_lane((uint32_t)v); }
__device__ __forceinline__ double last_lane(double v) { return __longlong_as_double((long long)last_lane((uint64_t)__double_as_longlong(v))); }
template <class V> __device__ __forceinline__ V wave_total(V v) { return last_lane(wave_scan(v)); }
template <int CTRL, int ROWS> __device__ __forceinline__ float larger(float v) {
    const uint32_t x = __float_as_uint(v);
    return fmaxf(v, __uint_as_float(moved<CTRL, ROWS>(x, x)));
}
__device__ __forceinline__ float wave_largest(float v) {
    v = larger<0x111, 0xF>(v);
    v = larger<0x112, 0xF>(v);
    v = larger<0x114, 0xF>(v);
    v = larger<0x118, 0xF>(v);
    v = larger<0x142, 0xA>(v);
    v = larger<0x143, 0xC>(v);
    return __uint_as_float(last_lane(__float_as_uint(v)));
}

// 2^(j / 64), j = 0 .. 63, evaluated by the host's compiler from the definition
struct Exp2Table { double v[64]; };
constexpr Exp2Table make_exp2_table() {
    Exp2Table t = {};
    for (int j = 0; j < 64; ++j) {                    // e^(j ln 2 / 64) by its series
        const double x = j * (0.69314718055994530942 / 64.0);
        double term = 1.0, sum = 0.0, lost = 0.0;
        for (int n = 1; n < 30; ++n) {                // the small terms' rounding is carried along
            const double y = term - lost, s = sum + y;
            lost = (s - sum) - y;
            sum = s;
            term *= x / n;
        }
        t.v[j] = sum;
    }
    return t;
}
__device__ const Exp2Table kExp2 = make_exp2_table();

// w = exp((l - m) / T) in 64 bits: the tokens follow from where u falls between sums of up to 10^5 of them, and an error of 1e-7 in those
// would draw another token once in a few dozen rows.  With t = 64 (l - m) / (T ln 2), k the nearest integer and f = t - k: 2^(k / 64) from a table and
// an exponent, 2^(f / 64) by four terms (|f ln 2 / 64| <= 0.0055: 4e-14 off).  Adding 1.5 2^52 rounds to the integer and leaves it in the lower word.
// The largest logit, +inf too, weighs 1; without a temperature all others weigh 0.
// p f + c with the constant where a scalar register holds it: as the accumulator of the two-address form it is moved there anew each time.
__device__ __forceinline__ double fma_const(double p, double f, double c) {
    double r;
    asm("v_fma_f64 %0, %1, %2, %3" : "=v"(r) : "v"(p), "v"(f), "s"(c));
    return r;
}
struct Weight {
    double m, c;                                      // c = 64 / (T ln 2)
    const double* table;
    bool greedy, infinite;
    __device__ __forceinline__ Weight(float largest, float temperature, const double* table_)
        : m(largest == INFINITY ? 0.0 : (double)largest), c(92.33248261689366 / (double)temperature), table(table_), greedy(temperature == 0.f),
          infinite(largest == INFINITY) {}
    // what takes the place of a logit where the largest is +inf, whose differences are undefined
    __device__ __forceinline__ float tame(float l) const { return infinite ? l == INFINITY ? 0.f : -INFINITY : l; }
    // of a row with a temperature and a finite maximum, N at a time, so that neither a table's entry nor a product is waited for; an undefined logit
    // weighs nothing (the maximum drops it).  The difference comes first: l c - m c in one operation is off by m c's rounding, which for logits of 1e38 or temperatures
    // of 1e-30 is larger than any exponent.
    template <int N> __device__ __forceinline__ void plain(const float (&l)[N], double (&w)[N]) const {
        double f[N], e[N];
        int k[N];
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const double t = fmax(((double)l[i] - m) * c, -80000.0), s = t + 6755399441055744.0;
            f[i] = t - (s - 6755399441055744.0);
            k[i] = (int)(uint32_t)__double_as_longlong(s);
            e[i] = table[k[i] & 63];
        }
        if (N > 1) __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < N; ++i) w[i] = fma_const(5.732851688640402e-10, f[i], 2.1173137155464774e-07);            // (ln 2 / 64)^4 / 24, ^3 / 6, ^2 / 2, ^1
#pragma unroll
        for (int i = 0; i < N; ++i) w[i] = fma_const(w[i], f[i], 5.864904955056169e-05);
#pragma unroll
        for (int i = 0; i < N; ++i) w[i] = fma_const(w[i], f[i], 0.010830424696249145);
#pragma unroll
        for (int i = 0; i < N; ++i) w[i] = ldexp(e[i] * fma(w[i], f[i], 1.0), k[i] >> 6);
    }
    __device__ __forceinline__ double operator()(float l) const {
        const float x[1] = {tame(l)};
        double w[1];
        plain(x, w);
        return (double)x[0] == m ? 1.0 : greedy ? 0.0 : w[0];
    }
    // log of a token's weight
    __device__ __forceinline__ double log_of(float l, float temperature) const { return greedy ? 0.0 : ((double)tame(l) - m) / (double)temperature; }
};

struct Select {
    uint32_t prefix;       // digits fixed so far (high bits)
    uint64_t remaining;    // how much (count or mass) must still be covered from the top of the current digit
};

// Among 256 bins, walking from bin 255 down, the one in which the running total first reaches `remaining`.  By one wave.  The sum over COPIES of them,
// kCopyBins apart.
constexpr int kCopyBins = 260;         // the copies of a bin lie in different banks
template <int COPIES>
__device__ __forceinline__ void pick_digit(const uint64_t* hist, int shift, Select* sel, int lane) {
    const int top = 255 - 4 * lane;                  // a lane has four bins down from here
    uint64_t b[4] = {}, mine = 0;
#pragma unroll
    for (int c = 0; c < COPIES; ++c)
#pragma unroll
        for (int i = 0; i < 4; ++i) b[i] += hist[c * kCopyBins + top - i];
#pragma unroll
    for (int i = 0; i < 4; ++i) mine += b[i];
    const uint64_t incl = wave_scan(mine);
    uint64_t acc = incl - mine;
    const uint64_t need = sel->remaining;
    if (acc < need && need <= incl) {               // exactly one lane
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (acc + b[i] >= need) { sel->prefix |= (uint32_t)(top - i) << shift; sel->remaining = need - acc; break; }
            acc += b[i];
        }
    }
}

// the sum of 256 bins, by a wave
__device__ __forceinline__ uint64_t sum_of(const uint64_t* hist, int lane) {
    uint64_t z = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) z += hist[lane * 4 + i];
    return wave_total(z);
}
__device__ __forceinline__ uint64_t share_of(double p, uint64_t z) {
    const uint64_t target = (uint64_t)ceil(p * (double)z);
    return target < 1 ? 1 : target > z ? z : target;
}
__device__ __forceinline__ double number_of(float u) { return (double)fminf(fmaxf(u, 0.f), 0.99999994f); }      // fmaxf: a NaN counts as 0

constexpr int kCached = 16384;         // entries of a row that fit LDS (64 KB)

struct RowSettings {
    float temperature;
    int top_k;
    double top_p, min_p;
    bool greedy;
    __device__ __forceinline__ RowSettings(const DrawRows& rows, int r, int V) {
        temperature = rows.temperature[r];
        greedy = temperature == 0.f;
        top_k = greedy || rows.top_k[r] >= V || rows.top_k[r] < 0 ? 0 : rows.top_k[r];
        top_p = greedy ? 1.0 : rows.top_p[r];
        min_p = greedy ? 0.0 : rows.min_p[r];
    }
};

__device__ __forceinline__ void nothing_to_draw(const DrawArgs& a, int r) {
    a.tokens[r] = 0;
    if (a.logp) a.logp[r] = -INFINITY;
}

constexpr int kBins = 1024, kPerNat = 32;          // bins over the 32 below the maximum of (l - m) / T, and the last for what lies further down
// monotone in l, and their floors whole numbers that floats hold exactly
__device__ __forceinline__ float bin_scale(float temperature) { return (float)kPerNat / temperature; }
__device__ __forceinline__ float bin_place(float l, float scale) { return fminf(fmaxf(l * scale, -4194304.f), 4194304.f); }
__device__ __forceinline__ float bin_floor(float l, float scale) { return floorf(bin_place(l, scale)); }
__device__ __forceinline__ int bin_of(float l, float top, float scale) { return min((int)(top - bin_floor(l, scale)), kBins - 1); }
// Where the last bin's candidates end: below, weights are 0 in 64 bits too, so that a mask's -inf or lowest number is none.  Kept or not, such an entry is never drawn.
// (Where 30 of 151,936 are allowed and 50 are asked for, 64 rows: 48 us, and 1,008 with all of them as candidates, which the list does not hold.)
__device__ __forceinline__ float least_candidate(float m, float temperature) { return fmaxf(m - 1000.f * temperature, -3.402823466e38f); }

// The cuts of a row that lies in LDS, in two or three sweeps: counts and masses of its bins, then the entries of the bin in which a border falls, each by a thread
// that adds up those above it (up to a thread each; more, e.g. equal logits, are left to the descent below).  The masses are the integers that the descent
// adds, so the border is the same.  128 rows of 16,000 fp32 logits, top-k 300 and top-p 0.95: 43 us by eight sweeps of the descent, 29 so; 2,039 of them 15.2 and 12.8 (one
// cut of 600: 7.9 and 8.2).
struct RowBins {
    uint64_t mass[kBins];             // of bins, then of listed entries
    uint32_t count[kBins];            // of bins, then keys
    uint64_t wave_mass[kBins / 64], above_mass, kept_mass;
    uint32_t wave_count[kBins / 64], above, n, border;
    int bin;
};
struct NoBins { uint64_t mass[256]; };
struct Cuts { uint32_t floor_key; bool by_count, by_mass; };      // and which of them are done
__device__ __forceinline__ Cuts cut_by_bins(RowBins& s, const float* cache, uint32_t V, float m, const Weight& weight, const RowSettings& set, double unit) {
    constexpr int THREADS = kBins;    // a bin a thread
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const bool by_mass = set.top_p < 1.0;
    auto amount = [&](float l) { return (uint64_t)rint(weight(l) * unit); };
    Cuts cuts = {0u, !set.top_k, !by_mass};
    s.count[tid] = 0;
    s.mass[tid] = 0;
    if (tid == 0) s.n = s.border = 0;
    __syncthreads();
    const float scale = bin_scale(set.temperature), top = bin_floor(m, scale);
    for (uint32_t v = tid; v < V; v += THREADS) {
        const float l = cache[v];
        const int b = bin_of(l, top, scale);
        if (set.top_k) atomicAdd(&s.count[b], 1u);
        if (by_mass) {
            const uint64_t x = amount(l);
            if (x) atomicAdd((unsigned long long*)&s.mass[b], (unsigned long long)x);
        }
    }
    __syncthreads();
    const uint32_t n = s.count[tid];
    const uint64_t q = s.mass[tid];
    uint32_t n_upto = wave_scan(n);
    uint64_t q_upto = wave_scan(q), all = 0;
    if (lane == 63) { s.wave_count[wave] = n_upto; s.wave_mass[wave] = q_upto; }
    __syncthreads();
    for (int i = 0; i < THREADS / 64; ++i) {
        if (i < wave) { n_upto += s.wave_count[i]; q_upto += s.wave_mass[i]; }
        all += s.wave_mass[i];
    }
    uint64_t target = 0;
    auto find_mass = [&] {                           // exactly one bin
        if (q_upto - q < target && target <= q_upto) { s.bin = tid; s.above_mass = q_upto - q; }
    };
    if (set.top_k) {
        if (n_upto - n < (uint32_t)set.top_k && (uint32_t)set.top_k <= n_upto) { s.bin = tid; s.above = n_upto - n; s.above_mass = q_upto - q; }
    } else {
        target = share_of(set.top_p, all);
        find_mass();
    }
    uint32_t key = 0, upto_n = 0, over_n = 0;        // of this thread's entry of the list: how much from it on, and above it
    uint64_t upto_q = 0, over_q = 0;
    bool mine = false;
    auto listed = [&] {                              // the bin's entries; false: more than threads
        __syncthreads();
        const int bin = s.bin;
        const float least = bin == kBins - 1 ? least_candidate(m, set.temperature) : -INFINITY;
        for (uint32_t v = tid; v < V; v += THREADS) {
            const float l = cache[v];
            if (l < least || bin_of(l, top, scale) != bin) continue;
            const uint32_t at = atomicAdd(&s.n, 1u);
            if (at < (uint32_t)THREADS) s.count[at] = order_key(l);
        }
        __syncthreads();
        const uint32_t entries = s.n;
        if (entries > (uint32_t)THREADS) return false;
        mine = (uint32_t)tid < entries;
        if (mine) {
            key = s.count[tid];
            s.mass[tid] = by_mass ? amount(key_value(key)) : 0;
        }
        __syncthreads();
        if (mine) {
            upto_n = over_n = 0;
            upto_q = over_q = 0;
            for (uint32_t j = 0; j < entries; ++j) {
                const uint32_t k = s.count[j];
                const uint64_t x = s.mass[j];
                upto_n += k >= key;
                over_n += k > key;
                upto_q += k >= key ? x : 0;
                over_q += k > key ? x : 0;
            }
        }
        return true;
    };
    if (!listed()) return cuts;
    if (set.top_k) {
        const uint32_t need = (uint32_t)set.top_k - s.above;
        const bool reaches = need <= s.n;            // else it lies where nothing weighs anything
        if (mine && over_n < need && need <= upto_n) { s.border = key; s.kept_mass = upto_q; }          // equal ones write the same
        __syncthreads();
        cuts = {s.border, true, !by_mass};
        if (!by_mass) return cuts;
        target = share_of(set.top_p, reaches ? s.above_mass + s.kept_mass : all);
        if (target <= s.above_mass) {                // in a bin above
            __syncthreads();
            find_mass();
            if (tid == 0) s.n = 0;
            if (!listed()) return cuts;
        }
    }
    const uint64_t need = target - s.above_mass;
    if (mine && over_q < need && need <= upto_q) s.border = key;
    __syncthreads();
    return {s.border, true, true};
}

// A row by a workgroup, in as many sweeps of it as the cuts need: one for the maximum, those of cut_by_bins or four digits of the k-th largest key and four of
// the key at which the mass reaches p, one for the sum of what is kept and a part of one for the token.
// cache: or null, LDS for the row (short ones), which is then read once.
template <class T, int THREADS>
__device__ __forceinline__ void draw_row(const DrawArgs& a, const DrawRows& rows, int r, const double* table, float* cache) {
    constexpr int WAVES = THREADS / 64;
    constexpr bool BINS = THREADS == kBins;
    __shared__ std::conditional_t<BINS, RowBins, NoBins> bins;
    uint64_t* hist = bins.mass;
    __shared__ Select sel;
    __shared__ double s_sum[WAVES];
    __shared__ float s_max[WAVES];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const T* row = (const T*)a.logits + (size_t)r * a.row_stride;
    const uint32_t V = a.V;
    auto logit_at = [&](uint32_t v) { return cache ? cache[v] : clean((float)row[v]); };

    float m = -INFINITY;
    for (uint32_t v = tid; v < V; v += THREADS) {
        const float l = clean((float)row[v]);
        if (cache) cache[v] = l;
        m = fmaxf(m, l);
    }
    m = wave_largest(m);
    if (lane == 0) s_max[wave] = m;
    __syncthreads();
    for (int w = 0; w < WAVES; ++w) m = fmaxf(m, s_max[w]);
    if (m == -INFINITY) {
        if (tid == 0) nothing_to_draw(a, r);
        return;
    }
    const RowSettings set(rows, r, a.V);
    const Weight weight(m, set.temperature, table);
    uint32_t floor_key = 0;

    auto descend = [&](auto&& amount, auto&& total_known) {
        for (int shift = 24; shift >= 0; shift -= 8) {
            __syncthreads();
            if (tid < 256) hist[tid] = 0;
            __syncthreads();
            const uint32_t prefix = sel.prefix;
            for (uint32_t v = tid; v < V; v += THREADS) {
                const float l = logit_at(v);
                const uint32_t key = order_key(l);
                if (key >= floor_key && (shift == 24 || (key >> (shift + 8)) == (prefix >> (shift + 8)))) {
                    const uint64_t x = amount(l);
                    if (x) atomicAdd((unsigned long long*)&hist[key >> shift & 255u], (unsigned long long)x);
                }
            }
            __syncthreads();
            if (shift == 24) {
                if (wave == 0) total_known();
                __syncthreads();
            }
            if (wave == 0) pick_digit<1>(hist, shift, &sel, lane);
        }
        __syncthreads();
        floor_key = sel.prefix > floor_key ? sel.prefix : floor_key;
        __syncthreads();
    };
    // integers add in any order: 2^-b of the largest weight, b as V of them leave room for
    const double unit = ldexp(1.0, 30 + __clz(V));
    Cuts cuts = {0u, !set.top_k, !(set.top_p < 1.0)};
    if constexpr (BINS)
        if (cache && !(cuts.by_count && cuts.by_mass)) {
            cuts = cut_by_bins(bins, cache, V, m, weight, set, unit);
            floor_key = cuts.floor_key;
        }
    if (!cuts.by_count) {
        if (tid == 0) { sel.prefix = 0; sel.remaining = (uint64_t)set.top_k; }
        descend([](float) { return (uint64_t)1; }, [] {});
    }
    if (!cuts.by_mass) {
        if (tid == 0) { sel.prefix = 0; sel.remaining = 0; }
        descend([&](float l) { return (uint64_t)rint(weight(l) * unit); }, [&] {
            const uint64_t z = sum_of(hist, lane);
            if (lane == 0) sel.remaining = share_of(set.top_p, z);
        });
    }

    auto kept = [&](float l) {
        if (order_key(l) < floor_key) return 0.0;
        const double w = weight(l);
        return w >= set.min_p ? w : 0.0;
    };
    // a wave has a run of neighbouring entries
    const uint32_t run = ((V + WAVES - 1) / WAVES + 63) & ~63u;
    const uint32_t lo = min((uint32_t)wave * run, V), hi = min(lo + run, V);
    double sum = 0.0;
    for (uint32_t v = lo + lane; v < hi; v += 64) sum += kept(logit_at(v));
    sum = wave_total(sum);
    if (lane == 0) s_sum[wave] = sum;
    __syncthreads();
    double total = 0.0;
    for (int w = 0; w < WAVES; ++w) total += s_sum[w];
    const double target = set.greedy ? 0.0 : number_of(a.uniform[r]) * total;
    double before = 0.0;
    int mine = 0;
    for (int w = 0, done = 0; w < WAVES && !done; ++w) {
        if (s_sum[w] > 0.0) mine = w;               // rounding may leave none: then the last with anything in it
        done = before + s_sum[w] > target;
        before += s_sum[w];
    }
    if (wave != mine) return;
    uint32_t token = 0;
    bool found = false;
    before = 0.0;
    for (int w = 0; w < mine; ++w) before += s_sum[w];
    for (uint32_t v0 = lo; v0 < hi && !found; v0 += 64) {
        const uint32_t v = v0 + lane;
        const double w = v < hi ? kept(logit_at(v)) : 0.0;
        const double c = wave_scan(w);
        const uint64_t over = __builtin_amdgcn_ballot_w64(w > 0.0 && before + c > target), any = __builtin_amdgcn_ballot_w64(w > 0.0);
        if (over) { token = v0 + __builtin_ctzll(over); found = true; }
        else if (any) token = v0 + 63 - __builtin_clzll(any);
        before += last_lane(c);
    }
    if (lane == 0) {
        a.tokens[r] = (int32_t)token;
        if (a.logp) a.logp[r] = set.greedy ? 0.f : (float)(weight.log_of(logit_at(token), set.temperature) - log(total));
    }
}

// ---- long rows, in pieces -----------------------------------------------------------------------------------------------

constexpr int kPiece = 2048;          // neighbouring entries of a wave: 32 a lane, all loaded at once
constexpr int kMaxPieces = 256;       // of a row
constexpr int kWgWaves = 8;           // waves of a workgroup
constexpr int kSlice = kPiece * kWgWaves;
constexpr int kCopies = 4;            // of a histogram: neighbouring lanes do not meet in one
constexpr uint32_t kOne = 1u << 19;   // an entry in it; below, the sum of places of seven bits.  Room for all that lanes of one copy have:
static_assert(kSlice / kCopies * 127 < (int)kOne && kSlice / kCopies < (1 << 13) && kSlice < (1 << 16), "a bin overflows");
constexpr int kCap = 8192;            // candidates of a row
constexpr int kApart = 64;            // words between the counters of rows: atomics of different rows do not queue for one cache line
constexpr int kTakeAll = 0, kTakeSome = 1, kTakeListed = 2, kTakeSlow = 3;

// What the histogram decides of a row.  Cut by count, the border lies among the logits from k_list up to below k_keep (-inf both: not cut so); cut by mass, from
// list up to below keep.  Those are the candidates; from keep on all are kept.
struct DrawPlan {
    float m;
    int take;                         // kTakeAll: all are kept but for min-p's; Some: as above; Listed: all from `list` on are candidates; Slow: a workgroup does the row
    float keep, list, k_keep, k_list;
    uint32_t k_above;                 // entries from k_keep on
    int k_last;                       // the count's border lies in the last bin or below the candidates
};
// What a piece has: kept weights relative to exp(ref), and of a row cut by mass all weights and those in bins below lo.
struct PieceSums { double kept, all, above; float ref; int pad; };

// the piece's entries in index order: vector q of lane i starts at (64 q + i) N
template <class T>
struct Piece {
    static constexpr int N = RowVec<T>::N, Q = kPiece / 64 / N;
    typename RowVec<T>::type x[Q];
    uint32_t first, V;
    __device__ __forceinline__ Piece(const T* row, uint32_t start, uint32_t V_, int lane) : first(start + lane * N), V(V_) {
        if (start + kPiece <= V) {                  // the same for the whole wave
#pragma unroll
            for (int q = 0; q < Q; ++q) x[q] = *(const typename RowVec<T>::type*)(row + first + q * 64 * N);
            return;
        }
#pragma unroll
        for (int q = 0; q < Q; ++q)
#pragma unroll
            for (int e = 0; e < N; ++e) x[q][e] = index(q, e) < V ? row[index(q, e)] : (T)-INFINITY;
    }
    __device__ __forceinline__ uint32_t index(int q, int e) const { return first + q * 64 * N + e; }
    __device__ __forceinline__ bool whole() const { return __builtin_amdgcn_readfirstlane(first) + kPiece <= V; }
    __device__ __forceinline__ float at(int q, int e) const { return clean((float)x[q][e]); }
    __device__ __forceinline__ float largest() const {
        float m = -INFINITY;
#pragma unroll
        for (int q = 0; q < Q; ++q)
#pragma unroll
            for (int e = 0; e < N; ++e) m = fmaxf(m, (float)x[q][e]);
        return m;
    }
};

// the least logit whose floor is at least f (NaN, which none reaches: there is none), for every 16 lanes of a wave one f: four bits of its key at a time, lane i
// of the 16 tries the last key of the i-th range
__device__ __forceinline__ float least_logit(float f, float scale, int lane) {
    const uint32_t bottom = order_key(-INFINITY), top = order_key(INFINITY);
    auto reaches = [&](uint32_t key) { return key >= bottom && (key > top || bin_floor(key_value(key), scale) >= f); };
    uint32_t at = 0;
#pragma unroll
    for (int shift = 28; shift >= 0; shift -= 4) {
        const uint32_t last = at + ((uint32_t)(lane & 15) << shift) + ((1u << shift) - 1u);
        const uint32_t hit = (uint32_t)(__builtin_amdgcn_ballot_w64(reaches(last)) >> (lane & 48)) & 0xFFFFu;
        at += (uint32_t)__builtin_ctz(hit) << shift;           // the last range's reaches always
    }
    return at > top ? NAN : key_value(at);
}

struct DrawSpace {                    // the workspace of a launch's rows
    PieceSums* pieces;                // [rows][kMaxPieces]: n_pieces of them used
    float* largest;                   // [rows][slices]
    uint32_t* hist;                   // [rows][slices][kBins]: entries, and below their number 512 times the mean of their places
    DrawPlan* plan;                   // [rows]
    uint32_t* n_listed;               // [rows][kApart]
    uint2* list;                      // [rows][kCap]: key, index
    int slices, n_pieces;
};

// f(four logits, the first's number) for a lane's entries.  The values, and what has been added so far (settle), are opaque to the compiler, which would convert
// all 32 ahead, for every branch that may need them, and add them when all are there: 222 registers for what takes 80, and two waves a SIMD for six.
template <class V> __device__ __forceinline__ void settle(V& v) { asm volatile("" : "+v"(v)); }
template <class T, class F>
__device__ __forceinline__ void for_each_four(const Piece<T>& p, F&& f) {
#pragma unroll
    for (int i = 0; i < p.Q * p.N; i += 4) {
        float l[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            l[j] = (float)p.x[(i + j) / p.N][(i + j) % p.N];
            asm volatile("" : "+v"(l[j]));
        }
        f(l, i);
        __builtin_amdgcn_sched_barrier(0);
    }
}

// a piece whose entries are all kept, relative to its own maximum
template <class T>
__device__ __forceinline__ void sum_whole_piece(const Piece<T>& p, float temperature, const double* table, int lane, PieceSums* out) {
    const float m = wave_largest(p.largest());
    double sum = 0.0;
    if (m != -INFINITY) {
        const Weight weight(m, temperature, table);
        double x[4];
        if (weight.infinite || weight.greedy)
            for_each_four(p, [&](const float (&l)[4], int) {
#pragma unroll
                for (int j = 0; j < 4; ++j) sum += weight(clean(l[j]));
                settle(sum);
            });
        else
            for_each_four(p, [&](const float (&l)[4], int) {
                weight.plain(l, x);
                sum += (x[0] + x[1]) + (x[2] + x[3]);
                settle(sum);
            });
        sum = wave_total(sum);
    }
    if (lane == 0) { out->kept = sum; out->ref = m; }
}

__device__ __forceinline__ void copy_table(double* s_table) {
    if (threadIdx.x < 64) s_table[threadIdx.x] = kExp2.v[threadIdx.x];
    __syncthreads();
}

}  // namespace

template <class T>
__global__ __launch_bounds__(1024) void draw_row_kernel(DrawArgs a, DrawRows rows) {
    extern __shared__ uint4 lds_raw[];
    __shared__ double s_table[64];
    copy_table(s_table);
    draw_row<T, 1024>(a, rows, blockIdx.x, s_table, a.V <= kCached ? (float*)lds_raw : nullptr);
}

// Batches without a cut: one sweep.
template <class T>
__global__ __launch_bounds__(kWgWaves * 64) void draw_sum_kernel(DrawArgs a, DrawRows rows, DrawSpace w) {
    __shared__ double s_table[64];
    const int r = blockIdx.y, lane = threadIdx.x & 63, i = blockIdx.x * kWgWaves + (threadIdx.x >> 6);
    const Piece<T> p((const T*)a.logits + (size_t)r * a.row_stride, min((uint32_t)i * kPiece, (uint32_t)a.V), a.V, lane);
    copy_table(s_table);
    if (i < w.n_pieces) sum_whole_piece(p, rows.temperature[r], s_table, lane, &w.pieces[(size_t)r * kMaxPieces + i]);
}

// The maximum of a slice and, where the row is cut by count or mass, how many of its entries lie in which bin below it.
template <class T>
__global__ __launch_bounds__(kWgWaves * 64) void draw_count_kernel(DrawArgs a, DrawRows rows, DrawSpace w) {
    __shared__ uint32_t h[kBins * kCopies];
    __shared__ float s_max[kWgWaves];
    const int r = blockIdx.y, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const uint32_t first = (uint32_t)(blockIdx.x * kWgWaves + wave) * kPiece;
    const Piece<T> p((const T*)a.logits + (size_t)r * a.row_stride, min(first, (uint32_t)a.V), a.V, lane);
    const RowSettings set(rows, r, a.V);
    const bool binned = set.top_k || set.top_p < 1.0;
    if (binned)
        for (int i = tid; i < kBins * kCopies; i += kWgWaves * 64) h[i] = 0;
    float m = wave_largest(p.largest());
    if (lane == 0) s_max[wave] = m;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kWgWaves; ++i) m = fmaxf(m, s_max[i]);
    const size_t seg = (size_t)r * w.slices + blockIdx.x;
    if (tid == 0) w.largest[seg] = m;
    if (!binned) return;
    const float scale = bin_scale(set.temperature), top = bin_floor(m, scale);
#pragma unroll
    for (int q = 0; q < p.Q; ++q)
#pragma unroll
        for (int e = 0; e < p.N; ++e) {
            const float y = bin_place(p.at(q, e), scale), f = floorf(y);
            const int b = min((int)(top - f), kBins - 1);
            const uint32_t down = (uint32_t)((f + 1.f - y) * 127.99f);          // of 128 parts of the bin
            if (p.index(q, e) < p.V) atomicAdd(&h[b * kCopies + (lane & (kCopies - 1))], kOne | down);
        }
    __syncthreads();
    for (int b = tid; b < kBins; b += kWgWaves * 64) {
        uint2 n = make_uint2(0, 0);
#pragma unroll
        for (int i = 0; i < kCopies; ++i) {
            const uint32_t x = h[b * kCopies + i];
            n.x += x / kOne;
            n.y += x % kOne;
        }
        w.hist[seg * kBins + b] = n.x ? n.x << 16 | n.y * 512 / n.x : 0u;
    }
}

// The row's histogram, and the logits between which its cuts fall.  By mass they are estimated, an entry by the mean place of its bin's: 2.4e-4 off at most, one
// alone in its bin 1.2e-4.  The sums of the next sweep show whether the cut lies among the candidates.  (With whole bins for places a distribution of a few
// likely tokens over a flat rest was 2e-2 off, and the candidates a third of the row.)
__global__ __launch_bounds__(kBins) void draw_plan_kernel(DrawArgs a, DrawRows rows, DrawSpace w) {
    __shared__ uint32_t s_count[kBins], s_down[kBins];
    __shared__ double s_mass[kBins / 64], s_share, s_more;
    __shared__ uint32_t s_wave[kBins / 64], s_above, s_upto;
    __shared__ int s_lo, s_hi, s_cut;
    const int r = blockIdx.x, b = threadIdx.x, lane = b & 63, wave = b >> 6;
    const RowSettings set(rows, r, a.V);
    static_assert(kMaxPieces / kWgWaves <= 64, "a lane has a slice");
    const float mine = lane < w.slices ? w.largest[(size_t)r * w.slices + lane] : -INFINITY;
    uint32_t n8[8], next8[8];                                   // the first slices' bins are on their way meanwhile
    const uint32_t* hist = w.hist + (size_t)r * w.slices * kBins + b;
    const bool binned = set.top_k || set.top_p < 1.0;
    if (binned)
#pragma unroll
        for (int s = 0; s < 8; ++s) {
            n8[s] = s < w.slices ? hist[(size_t)s * kBins] : 0u;
            next8[s] = 8 + s < w.slices ? hist[(size_t)(8 + s) * kBins] : 0u;
        }
    const float m = wave_largest(mine);
    DrawPlan plan = {m, kTakeAll, -INFINITY, -INFINITY, -INFINITY, -INFINITY, 0u, 0};
    if (b == 0) w.n_listed[(size_t)r * kApart] = 0;
    if (m == -INFINITY || !binned) {
        if (b == 0) w.plan[r] = plan;
        return;
    }
    const float scale = bin_scale(set.temperature), top = bin_floor(m, scale);
    s_count[b] = s_down[b] = 0;
    if (b == 0) { s_lo = kBins; s_hi = s_cut = kBins - 1; }
    __syncthreads();
    const float down = top - bin_floor(mine, scale);
    for (int s0 = 0; s0 < w.slices; s0 += 8) {
#pragma unroll
        for (int s = 0; s < 8; ++s) {
            const int to = (int)fminf((float)b + __shfl(down, s0 + s, 64), (float)(kBins - 1));
            if (n8[s]) {
                atomicAdd(&s_count[to], n8[s] >> 16);
                atomicAdd(&s_down[to], (n8[s] >> 16) * (n8[s] & 0xFFFFu) >> 5);          // 16 times the places' sum
            }
        }
#pragma unroll
        for (int s = 0; s < 8; ++s) {
            n8[s] = next8[s];
            next8[s] = s0 + 16 + s < w.slices ? hist[(size_t)(s0 + 16 + s) * kBins] : 0u;
        }
    }
    __syncthreads();
    const uint32_t n = s_count[b];
    const double mid = n && b < kBins - 1 ? (double)((float)n * expf(-((float)b + ((float)s_down[b] / (float)n * (1.f / 16.f) + 0.5f) * (1.f / 128.f)) * (1.f / kPerNat))) : 0.0;
    uint32_t count = wave_scan(n);
    double mass = wave_scan(mid);
    if (lane == 63) { s_wave[wave] = count; s_mass[wave] = mass; }
    __syncthreads();
    double all = 0.0;
    for (int i = 0; i < kBins / 64; ++i) {
        if (i < wave) { count += s_wave[i]; mass += s_mass[i]; }
        all += s_mass[i];
    }
    double off = 0.0;
    if (set.top_k) {                                            // exactly one bin; of its mass, the share of its entries that count
        if (count - n < (uint32_t)set.top_k && (uint32_t)set.top_k <= count) {
            s_cut = b;
            s_above = count - n;
            s_upto = count;
            s_share = mass - mid + mid * ((double)((uint32_t)set.top_k - (count - n)) / n);
            s_more = mid;
        }
        __syncthreads();
        all = s_share;
        off = s_more;
    }
    const bool listed = set.top_k && s_upto <= kCap;
    const int cut = s_cut;
    if (set.top_p < 1.0 && !listed) {
        const double target = set.top_p * all;
        // every bin's mass is off by a share e in [-2.4e-4, 1.2e-4] of itself (the curve of exp over 1/32 nat, places of 1/128 bin), so the running sum less p times the
        // whole one by at most 2.4e-4 ((1 - p) p + p (1 - p)) of it, and by what lies in the last bin, 2^19 e^-32.  (With 3e-4 of the target for all p, the candidates of
        // p = 0.9999 were more than the list holds: 64 rows of 151,936 normal bf16 logits, deviation 3, 587 us; 43 now.)
        off += target * (5e-4 * (1.0 - set.top_p) + 1e-8);
        if (mass - mid < target - off && target - off <= mass) s_lo = b;
        if (mass - mid < target + off && target + off <= mass) s_hi = b;
        if (b == 0 && target - off <= 0.0) s_lo = 0;
        __syncthreads();
    }
    if (wave != 0) return;
    int lo = set.top_p < 1.0 && !listed ? s_lo : cut, hi = set.top_p < 1.0 && !listed ? s_hi : cut;
    if (hi >= cut || lo > cut) hi = cut;                        // both borders in one run of bins
    if (lo > cut && lo < kBins) lo = cut;
    // 16 lanes each: keep, list, k_keep, k_list; a bin's entries are those from its floor on
    const int bin = lane < 16 ? lo - 1 : lane < 32 ? hi : lane < 48 ? cut - 1 : cut;
    float t = least_logit(bin < 0 ? NAN : top - (float)bin, scale, lane);
    if (bin < 0) t = NAN;                                       // above every logit
    if (bin == kBins - 1) t = least_candidate(m, set.temperature);
    plan.keep = __shfl(t, 0, 64);
    plan.list = __shfl(t, 16, 64);
    if (set.top_k) {
        plan.k_keep = __shfl(t, 32, 64);
        plan.k_list = __shfl(t, 48, 64);
        plan.k_above = s_above;
        plan.k_last = cut == kBins - 1;
    }
    plan.take = lo >= kBins ? kTakeSlow : listed ? kTakeListed : kTakeSome;
    if (lane == 0) w.plan[r] = plan;
}

// The second sweep: sums of what is kept for sure, piece by piece, and the list of candidates.
template <class T>
__global__ __launch_bounds__(kWgWaves * 64, 5) void draw_cut_kernel(DrawArgs a, DrawRows rows, DrawSpace w) {
    __shared__ double s_table[64];
    const int r = blockIdx.y, lane = threadIdx.x & 63, i = blockIdx.x * kWgWaves + (threadIdx.x >> 6);
    const T* row = (const T*)a.logits + (size_t)r * a.row_stride;
    const Piece<T> p(row, min((uint32_t)i * kPiece, (uint32_t)a.V), a.V, lane);
    copy_table(s_table);
    const DrawPlan plan = w.plan[r];
    if (i >= w.n_pieces || plan.take == kTakeSlow || plan.m == -INFINITY) return;
    const RowSettings set(rows, r, a.V);
    PieceSums* out = &w.pieces[(size_t)r * kMaxPieces + i];
    if (plan.take == kTakeAll && set.min_p == 0.0) {
        sum_whole_piece(p, set.temperature, s_table, lane, out);
        return;
    }
    const Weight weight(plan.m, set.temperature, s_table);
    const bool odd = weight.infinite || weight.greedy;
    double kept = 0.0, all = 0.0, above = 0.0;
    uint32_t mine = 0;                                          // one bit an entry: a candidate
    const bool limited = set.min_p > 0.0, by_count = set.top_k != 0;
    // `all`: what counts for the mass that top-p goes by; `kept`, where min-p is at work, and `above`: what is kept for sure; and the candidates
    auto each = [&](auto&& f) {
        double x[4];
        if (odd)
            for_each_four(p, [&](const float (&l)[4], int i) {
#pragma unroll
                for (int j = 0; j < 4; ++j) x[j] = weight(clean(l[j]));
                f(l, i, x);
            });
        else
            for_each_four(p, [&](const float (&l)[4], int i) {
                weight.plain(l, x);
                f(l, i, x);
            });
    };
    if (plan.take == kTakeListed) {
        for_each_four(p, [&](const float (&l)[4], int i) {
#pragma unroll
            for (int j = 0; j < 4; ++j) mine |= l[j] >= plan.list ? 1u << (i + j) : 0u;
            settle(mine);
        });
    } else if (plan.take == kTakeAll) {
        each([&](const float (&)[4], int, double (&x)[4]) {
#pragma unroll
            for (int j = 0; j < 4; ++j) x[j] = x[j] >= set.min_p ? x[j] : 0.0;
            kept += (x[0] + x[1]) + (x[2] + x[3]);
            settle(kept);
        });
    } else if (odd || limited || by_count) {
        each([&](const float (&l)[4], int i, double (&x)[4]) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const bool sure = l[j] >= plan.keep, counted = !by_count || l[j] >= plan.k_keep;
                above += sure ? x[j] : 0.0;
                kept += sure && x[j] >= set.min_p ? x[j] : 0.0;
                all += counted ? x[j] : 0.0;
                mine |= (!sure && l[j] >= plan.list) || (!counted && l[j] >= plan.k_list) ? 1u << (i + j) : 0u;
            }
            settle(all); settle(above); settle(kept); settle(mine);
        });
    } else {
        double x[4];
        for_each_four(p, [&](const float (&l)[4], int i) {
            weight.plain(l, x);
            all += (x[0] + x[1]) + (x[2] + x[3]);
            settle(all);
            // of a distribution with few likely tokens most are below the candidates
            if (!__builtin_amdgcn_ballot_w64(fmaxf(fmaxf(l[0], l[1]), fmaxf(l[2], l[3])) >= plan.list)) return;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const bool sure = l[j] >= plan.keep;
                x[j] = sure ? x[j] : 0.0;
                mine |= !sure && l[j] >= plan.list ? 1u << (i + j) : 0u;
            }
            above += (x[0] + x[1]) + (x[2] + x[3]);
            settle(above); settle(mine);
        });
    }
    if (plan.take == kTakeSome) {
        all = wave_total(all);
        above = wave_total(above);
    }
    kept = wave_total(kept);
    if (plan.take == kTakeSome && !limited) kept = above;
    if (lane == 0) *out = {kept, all, above, plan.m, 0};
    if (!p.whole())                                             // past the row's end there are none
#pragma unroll
        for (int q = 0; q < p.Q; ++q)
#pragma unroll
            for (int e = 0; e < p.N; ++e)
                if (p.index(q, e) >= p.V) mine &= ~(1u << (q * p.N + e));
    if (!__builtin_amdgcn_ballot_w64(mine != 0)) return;
    const uint32_t n = __popc(mine);
    uint32_t at = wave_scan(n), base = 0;
    if (lane == 63) base = atomicAdd(&w.n_listed[(size_t)r * kApart], at);
    at += last_lane(base) - n;
    // a lane has few, in any of 32 places: it reads them again rather than ask for each place
    for (; mine && at < kCap; mine &= mine - 1, ++at) {
        const int i = __builtin_ctz(mine);
        const uint32_t v = p.first + i / p.N * 64 * p.N + i % p.N;
        w.list[(size_t)r * kCap + at] = make_uint2(order_key(clean((float)row[v])), v);
    }
}

// The end of a row: with CUTS the exact border among the candidates (a radix descent, as in draw_row) and their weights' place among the pieces; the piece in
// which the number falls; the token in it.
template <class T, bool CUTS>
__global__ __launch_bounds__(CUTS ? 512 : 256) void draw_pick_kernel(DrawArgs a, DrawRows rows, DrawSpace w) {
    constexpr int THREADS = CUTS ? 512 : 256;
    extern __shared__ uint4 lds_raw[];
    uint2* list = (uint2*)lds_raw;                              // [kCap]
    uint64_t* mass = (uint64_t*)(list + kCap);                  // [kCap], 2^-50 of the largest weight
    constexpr int kDigitCopies = 8;
    __shared__ double s_table[64];
    __shared__ uint64_t hist[CUTS ? kDigitCopies * kCopyBins : 1];
    __shared__ uint64_t s_cand[CUTS ? kMaxPieces : 1];
    __shared__ Select sel;
    __shared__ double s_all, s_above;
    __shared__ uint64_t s_z, s_zk;
    __shared__ uint32_t s_differ, s_below;
    __shared__ bool s_found;
    const int r = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    copy_table(s_table);
    const RowSettings set(rows, r, a.V);
    const T* row = (const T*)a.logits + (size_t)r * a.row_stride;
    const PieceSums* pieces = w.pieces + (size_t)r * kMaxPieces;
    constexpr int PER = kMaxPieces / 64;
    double sum[PER];                                            // a lane has PER neighbouring pieces
    float ref[PER];
    float m = -INFINITY;
    DrawPlan plan = {};
    constexpr int AHEAD = CUTS ? 4 : 1;                         // entries of the list, read before it is known whether there are so many
    uint2 ahead[AHEAD], first_entry = {};
    const uint2* from = w.list + (size_t)r * kCap;
    if (CUTS) {
        plan = w.plan[r];
        m = plan.m;
        first_entry = from[0];
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) ahead[j] = from[tid + j * THREADS];
    }
#pragma unroll
    for (int j = 0; j < PER; ++j) {
        const int i = lane * PER + j;
        ref[j] = i < w.n_pieces ? pieces[i].ref : -INFINITY;
        sum[j] = i < w.n_pieces ? pieces[i].kept : 0.0;
        if (!CUTS) m = fmaxf(m, ref[j]);
    }
    if (!CUTS) m = wave_largest(m);
    if (m == -INFINITY) {
        if (tid == 0) nothing_to_draw(a, r);
        return;
    }
    const Weight weight(m, set.temperature, s_table);
    uint32_t floor_key = 0;
    constexpr double UNIT = 1125899906842624.0;                 // 2^50: kCap of them fit 64 bits
    bool slow = false;
    if constexpr (CUTS) {
        const uint32_t n = w.n_listed[(size_t)r * kApart];
        slow = plan.take == kTakeSlow || ((plan.take == kTakeSome || plan.take == kTakeListed) && n > kCap);
        const bool listed = !slow && (plan.take == kTakeSome || plan.take == kTakeListed);
        if (listed) {
            if (wave == 0) {
                double all = 0.0, above = 0.0;
#pragma unroll
                for (int j = 0; j < PER; ++j) {
                    const int i = lane * PER + j;
                    if (i < w.n_pieces) { all += pieces[i].all; above += pieces[i].above; }
                }
                all = wave_total(all);
                above = wave_total(above);
                if (lane == 0) { s_all = all; s_above = above; s_z = s_zk = 0; s_differ = s_below = 0; }
            }
            for (int i = tid; i < kMaxPieces; i += THREADS) s_cand[i] = 0;
            __syncthreads();
            const uint32_t key0 = first_entry.x;
            uint32_t differ = 0;
            auto enter = [&](uint32_t i, uint2 e) {
                list[i] = e;
                mass[i] = (uint64_t)rint(weight(key_value(e.x)) * UNIT);
                differ |= e.x ^ key0;
            };
#pragma unroll
            for (int j = 0; j < AHEAD; ++j)
                if (tid + j * THREADS < n) enter(tid + j * THREADS, ahead[j]);
            for (uint32_t i = tid + AHEAD * THREADS; i < n; i += THREADS) enter(i, from[i]);
#pragma unroll
            for (int o = 32; o > 0; o >>= 1) differ |= __shfl_xor(differ, o, 64);
            if (lane == 0 && differ) atomicOr(&s_differ, differ);
            __syncthreads();
            const uint32_t any = s_differ;
            // digits that all candidates share are not looked at (16-bit logits: two of four)
            uint32_t shared_digits = 0;
            for (int shift = 0; shift < 32; shift += 8)
                if ((any >> shift & 255u) == 0) shared_digits |= key0 & (255u << shift);
            auto descend = [&](auto&& amount) {                 // sel.remaining is set
                if (tid == 0) sel.prefix = shared_digits;
                for (int shift = 24; shift >= 0; shift -= 8) {
                    if ((any >> shift & 255u) == 0) continue;
                    for (int i = tid; i < kDigitCopies * kCopyBins; i += THREADS) hist[i] = 0;
                    __syncthreads();
                    const uint32_t prefix = sel.prefix;
                    for (uint32_t i = tid; i < n; i += THREADS) {
                        const uint32_t key = list[i].x;
                        if (key >= floor_key && (shift == 24 || (key >> (shift + 8)) == (prefix >> (shift + 8)))) {
                            const uint64_t x = amount(key, i);
                            if (x) atomicAdd((unsigned long long*)&hist[(lane & (kDigitCopies - 1)) * kCopyBins + (key >> shift & 255u)], (unsigned long long)x);
                        }
                    }
                    __syncthreads();
                    if (wave == 0) pick_digit<kDigitCopies>(hist, shift, &sel, lane);
                    __syncthreads();
                }
                __syncthreads();
                floor_key = sel.prefix > floor_key ? sel.prefix : floor_key;
                __syncthreads();
            };
            // only those below k_keep are counted: the others are in number known
            const uint32_t sure_key = plan.take == kTakeListed || plan.k_keep != plan.k_keep ? 0xFFFFFFFFu : order_key(plan.k_keep);
            // A count that reaches past all candidates of the last bin cuts nothing that weighs anything.
            const uint32_t to_count = set.top_k - (plan.take == kTakeListed ? 0u : plan.k_above);
            bool counts = set.top_k != 0;
            if (counts && plan.k_last) {
                uint32_t below = 0;
                for (uint32_t i = tid; i < n; i += THREADS) below += list[i].x < sure_key ? 1u : 0u;
                below = wave_total(below);
                if (lane == 0 && below) atomicAdd(&s_below, below);
                __syncthreads();
                counts = to_count <= s_below;
            }
            if (counts) {
                if (tid == 0) sel.remaining = to_count;
                descend([&](uint32_t key, uint32_t) { return key < sure_key ? (uint64_t)1 : (uint64_t)0; });
            }
            if (set.top_p < 1.0) {
                // the mass of what the count leaves: all candidates', and of that what lies below k_keep (the rest is in s_all already)
                uint64_t z = 0, zk = 0;
                for (uint32_t i = tid; i < n; i += THREADS) {
                    const uint32_t key = list[i].x;
                    if (key < floor_key) continue;
                    z += mass[i];
                    if (set.top_k && key < sure_key) zk += mass[i];
                }
                z = wave_total(z);
                zk = wave_total(zk);
                if (lane == 0) { atomicAdd((unsigned long long*)&s_z, (unsigned long long)z); atomicAdd((unsigned long long*)&s_zk, (unsigned long long)zk); }
                __syncthreads();
                if (tid == 0) {
                    // how much of it the cut still needs; none, or more than there is: it does not lie among the candidates
                    const double of = (plan.take == kTakeListed ? 0.0 : s_all) + (double)s_zk * (1.0 / UNIT), over = plan.take == kTakeListed ? 0.0 : s_above;
                    const double need = ceil((set.top_p * of - over) * UNIT);
                    sel.remaining = need >= 1.0 && need <= (double)s_z ? (uint64_t)need : 0;
                    if (need > (double)s_z && over + (double)s_z * (1.0 / UNIT) >= of * (1.0 - 1e-12)) sel.remaining = s_z;      // by rounding alone
                    s_found = sel.remaining != 0;
                }
                __syncthreads();
                slow = !s_found;
                if (!slow) {
                    descend([&](uint32_t, uint32_t i) { return mass[i]; });
                    // below its run of candidates there is a gap down to those of the count
                    slow = plan.take == kTakeSome && floor_key < order_key(plan.list);
                }
            }
            if (!slow) {
                // A thread has neighbours of the list, which come from one piece mostly: it adds them up before it adds to the piece's sum.  (Neighbouring lanes on
                // neighbouring entries would all wait for one sum.)
                const uint32_t per = (n + THREADS - 1) / THREADS, first = tid * per, end = min(first + per, n);
                uint32_t piece = 0;
                uint64_t x = 0;
                for (uint32_t i = first; i < end; ++i) {
                    const uint2 e = list[i];
                    if (e.x < floor_key || (set.min_p > 0.0 && weight(key_value(e.x)) < set.min_p)) continue;
                    if (e.y / kPiece != piece) {
                        if (x) atomicAdd((unsigned long long*)&s_cand[piece], (unsigned long long)x);
                        piece = e.y / kPiece;
                        x = 0;
                    }
                    x += mass[i];
                }
                if (x) atomicAdd((unsigned long long*)&s_cand[piece], (unsigned long long)x);
                __syncthreads();
            }
        }
        if (slow) {
            draw_row<T, THREADS>(a, rows, r, s_table, nullptr);
            return;
        }
        if (wave >= 4) { __syncthreads(); return; }             // the barrier of the four waves below
        if (listed)
#pragma unroll
            for (int j = 0; j < PER; ++j) sum[j] += (double)s_cand[lane * PER + j] * (1.0 / UNIT);
    }
    // relative to the row's maximum: pieces whose entries are all kept have their own
    double mine = 0.0;
#pragma unroll
    for (int j = 0; j < PER; ++j) {
        if (ref[j] != m) sum[j] = sum[j] > 0.0 ? sum[j] * weight(ref[j]) : 0.0;
        mine += sum[j];
    }
    const double upto = wave_scan(mine), total = last_lane(upto);
    const double target = set.greedy ? 0.0 : number_of(a.uniform[r]) * total;
    // the first piece whose running sum exceeds the target, else the last that has anything
    double c = upto - mine, before = 0.0;
    int hit = -1, last = -1;
    double hit_before = 0.0, last_before = 0.0;
#pragma unroll
    for (int j = 0; j < PER; ++j) {
        if (sum[j] > 0.0) { last = lane * PER + j; last_before = c; }
        const double next = c + sum[j];
        if (hit < 0 && sum[j] > 0.0 && next > target) { hit = lane * PER + j; hit_before = c; }
        c = next;
    }
    const double log_total = log(total);
    const uint64_t hits = __builtin_amdgcn_ballot_w64(hit >= 0), lasts = __builtin_amdgcn_ballot_w64(last >= 0);
    int piece;
    if (hits) {
        const int from = __builtin_ctzll(hits);
        piece = __shfl(hit, from, 64); before = __shfl(hit_before, from, 64);
    } else {
        const int from = lasts ? 63 - __builtin_clzll(lasts) : 0;
        piece = max(__shfl(last, from, 64), 0); before = __shfl(last_before, from, 64);
    }
    // the piece by four waves, RUNS runs of 64 N entries each
    constexpr int N = RowVec<T>::N, RUNS = kPiece / 64 / N / 4;
    __shared__ double s_run[4 * RUNS];
    const uint32_t start = (uint32_t)piece * kPiece + wave * RUNS * 64 * N + lane * N;
    typename RowVec<T>::type x[RUNS];
    double own[RUNS], to[RUNS];
#pragma unroll
    for (int q = 0; q < RUNS; ++q) {
        const uint32_t v = start + q * 64 * N;
        if (v + N <= (uint32_t)a.V) x[q] = *(const typename RowVec<T>::type*)(row + v);
        else
#pragma unroll
            for (int e = 0; e < N; ++e) x[q][e] = v + e < (uint32_t)a.V ? row[v + e] : (T)-INFINITY;
    }
    auto kept = [&](float l) {
        const double w = !CUTS || order_key(l) >= floor_key ? weight(l) : 0.0;
        return CUTS && w < set.min_p ? 0.0 : w;
    };
#pragma unroll
    for (int q = 0; q < RUNS; ++q) {
        own[q] = 0.0;
#pragma unroll
        for (int e = 0; e < N; ++e) own[q] += kept(clean((float)x[q][e]));
        to[q] = wave_scan(own[q]);
    }
#pragma unroll
    for (int q = 0; q < RUNS; ++q)
        if (lane == 63) s_run[wave * RUNS + q] = to[q];
    __syncthreads();
    int run = -1;
    double run_before = 0.0;
    for (int i = 0, found = 0; i < 4 * RUNS && !found; ++i) {    // the first whose end exceeds, else the last that has anything
        if (s_run[i] > 0.0) {
            run = i;
            run_before = before;
            found = before + s_run[i] > target;
        }
        before += s_run[i];
    }
#pragma unroll
    for (int q = 0; q < RUNS; ++q) {
        if (run != wave * RUNS + q) continue;
        const uint64_t over = __builtin_amdgcn_ballot_w64(own[q] > 0.0 && run_before + to[q] > target), any = __builtin_amdgcn_ballot_w64(own[q] > 0.0);
        if (lane != (over ? __builtin_ctzll(over) : 63 - __builtin_clzll(any))) continue;
        double s = run_before + (to[q] - own[q]);               // in that lane: its first entry that exceeds, else its last with a weight
        uint32_t token = 0;
        float logit = 0.f;
        bool done = false;
#pragma unroll
        for (int e = 0; e < N; ++e) {
            const float l = clean((float)x[q][e]);
            const double w = kept(l);
            s += w;
            if (!done && w > 0.0) { token = start + q * 64 * N + e; logit = l; done = s > target; }
        }
        a.tokens[r] = (int32_t)token;
        if (a.logp) a.logp[r] = set.greedy ? 0.f : (float)(weight.log_of(logit, set.temperature) - log_total);
    }
}

namespace {
bool in_pieces(int V) { return V >= kCached && V <= kPiece * kMaxPieces; }
size_t take(size_t& at, size_t bytes) {
    const size_t o = at;
    at += (bytes + 255) & ~(size_t)255;
    return o;
}
DrawSpace draw_space(uintptr_t base, int rows, int V, size_t* bytes) {
    DrawSpace w;
    w.n_pieces = (V + kPiece - 1) / kPiece;
    w.slices = (V + kSlice - 1) / kSlice;
    size_t at = 0;
    w.pieces = (PieceSums*)(base + take(at, (size_t)rows * kMaxPieces * sizeof(PieceSums)));
    w.largest = (float*)(base + take(at, (size_t)rows * w.slices * sizeof(float)));
    w.hist = (uint32_t*)(base + take(at, (size_t)rows * w.slices * kBins * sizeof(uint32_t)));
    w.plan = (DrawPlan*)(base + take(at, (size_t)rows * sizeof(DrawPlan)));
    w.n_listed = (uint32_t*)(base + take(at, (size_t)rows * kApart * sizeof(uint32_t)));
    w.list = (uint2*)(base + take(at, (size_t)rows * kCap * sizeof(uint2)));
    *bytes = at;
    return w;
}

template <class T>
hipError_t launch_chunk(const DrawArgs& g, const DrawRows& rows, const DrawSpace& w, bool pieces, bool cuts, hipStream_t s) {
    if (!pieces) {
        hipLaunchKernelGGL(draw_row_kernel<T>, dim3(g.B), dim3(1024), g.V <= kCached ? (unsigned)(g.V * sizeof(float)) : 0, s, g, rows);
        return hipGetLastError();
    }
    const dim3 grid(w.slices, g.B), threads(kWgWaves * 64);
    if (!cuts) {
        hipLaunchKernelGGL(draw_sum_kernel<T>, grid, threads, 0, s, g, rows, w);
        hipLaunchKernelGGL((draw_pick_kernel<T, false>), dim3(g.B), dim3(256), 0, s, g, rows, w);
        return hipGetLastError();
    }
    const int list_lds = kCap * (sizeof(uint2) + sizeof(uint64_t));          // and 23 KB of its own: one workgroup a compute unit, which has one row at most
    hipLaunchKernelGGL(draw_count_kernel<T>, grid, threads, 0, s, g, rows, w);
    hipLaunchKernelGGL(draw_plan_kernel, dim3(g.B), dim3(kBins), 0, s, g, rows, w);
    hipLaunchKernelGGL(draw_cut_kernel<T>, grid, threads, 0, s, g, rows, w);
    hipError_t e = hipFuncSetAttribute((const void*)draw_pick_kernel<T, true>, hipFuncAttributeMaxDynamicSharedMemorySize, list_lds);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((draw_pick_kernel<T, true>), dim3(g.B), dim3(512), list_lds, s, g, rows, w);
    return hipGetLastError();
}
}  // namespace

// rows are processed kDrawRows at a time (their settings travel by value), one chunk after the other on the stream
size_t draw_workspace_bytes(int B, int V) {
    if (!in_pieces(V)) return 256;
    size_t bytes = 0;
    draw_space(0, B < kDrawRows ? B : kDrawRows, V, &bytes);
    return bytes;
}

hipError_t launch_draw(const DrawArgs& a, int dtype, const float* temperature, const int32_t* top_k, const float* top_p, const float* min_p,
                       void* workspace, hipStream_t s) {
    const size_t size = dtype == SPIRAL_DTYPE_FP32 ? 4 : 2;
    const bool pieces = in_pieces(a.V);
    for (int off = 0; off < a.B; off += kDrawRows) {
        DrawRows rows;
        const int n = a.B - off < kDrawRows ? a.B - off : kDrawRows;
        bool cuts = false;
        for (int i = 0; i < n; ++i) {
            rows.temperature[i] = temperature ? temperature[off + i] : 1.f;
            rows.top_k[i] = top_k ? top_k[off + i] : 0;
            rows.top_p[i] = top_p ? top_p[off + i] : 1.f;
            rows.min_p[i] = min_p ? min_p[off + i] : 0.f;
            cuts = cuts || (rows.temperature[i] > 0.f && ((rows.top_k[i] > 0 && rows.top_k[i] < a.V) || rows.top_p[i] < 1.f || rows.min_p[i] > 0.f));
        }
        DrawArgs g = a;
        g.B = n;
        g.logits = (const char*)a.logits + (size_t)off * a.row_stride * size;
        g.uniform = a.uniform + off;
        g.tokens = a.tokens + off;
        g.logp = a.logp ? a.logp + off : nullptr;
        size_t bytes;
        const DrawSpace w = draw_space((uintptr_t)workspace, n, a.V, &bytes);
        const hipError_t e = dtype == SPIRAL_DTYPE_FP32 ? launch_chunk<float>(g, rows, w, pieces, cuts, s)
                           : dtype == SPIRAL_DTYPE_BF16 ? launch_chunk<__bf16>(g, rows, w, pieces, cuts, s) : launch_chunk<_Float16>(g, rows, w, pieces, cuts, s);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace spiral
