// Causal attention over packed sequences, forward and backward, for the learner.
//
//   forward   s = scale q k^T, one pass over a row's tokens with a running reference m and sum l of exp2(s log2e - m); out = (sum exp2(..) v) / l, lse = ln 2 (m + log2 l)
//   dq        p = exp2(s log2e - lse log2e), dp = dout v^T, t = p (dp - D), dq = scale t k; D = dout . out, or sum p dp where a row's tokens are all at hand
//   dk, dv    the same p and t by columns: dv = p^T dout, dk = scale t^T q, over the group's heads
//
// All products are 32x32x16 matrix instructions on 16-bit operands with fp32 sums.  The scores come out transposed (a lane holds one row, its registers tokens; in the
// dk/dv kernel one token, and rows), which is the layout in which weights are the second operand of the product that follows, so they never leave their
// registers: rounded to the operands' type, to nearest, they are off by half a step, as q, k and v themselves are.  D, lse, m, l and all sums are fp32.
//
// Three kernels, seven products where the mathematics has five in the backward pass (s and dp are made twice): one kernel for all would have to add dq from many
// workgroups, by atomics whose order changes results or by partial sums that take longer than the two products (16 sequences of U[1024, 4096]: 15 GB, 3.1 ms).
//
// Bound: the chip's power, and waits.  The compute units are busy, the matrix pipes 54 to 62 % of their time, at 1.9 GHz in place of 2.4; with zeros for all inputs the same launches take
// 17, 23 and 27 % less time.  Waves wait for 31 to 36 % of their cycles, for operands from LDS for 4 to 6 %; how much of the rest is for stages' loads and how much at their barriers is
// not told apart.  16 sequences of U[1024, 4096], 32 heads on 8, hd 128, bf16 (41 k rows): forward 1.02 ms (1.04 PFLOP/s), dq 1.72 (0.93), dk and dv 2.08 (1.03 of what is computed; cards differ by 4 %);
// a library product of 16384^3 makes 1.35.  A row alone by one wave, token by token, took 534 ms for the three.
// On the way: bank-free tiles (64 banks, not 32, serve a wave's reads) 5.1 -> 2.65 ms of dk and dv, whose addresses had been spilled; values in LDS and stages of 32 rows there 2.65 -> 2.24; three
// forward workgroups a compute unit 1.16 -> 1.06.  Without effect, within 2 %: products interleaved with exponentials instruction by instruction, operand reads further ahead, the two score
// chains in turn, s_setprio around products or for long workgroups, the group's heads one after the other or stage by stage (L2 hits 28 -> 74 %).  Worse: 64 rows a wave (512 registers, one wave a SIMD: forward
// 1.16 -> 2.44 ms), eight waves a workgroup with three stages in flight (1.16 -> 1.39).
//
// A row alone: one wave computes one (row, head) of the outputs or of dq, token by token, and reads nothing that the row does not see.  For rows in whose sums a
// weight of 0 has met an infinite or undefined value only.
#include <type_traits>

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

// A lane holds dimensions lane and lane + 64 (HD = 32: the upper half of the wave repeats the lower)
template <int HD> constexpr int kDims = (HD + 63) / 64;

// out and lse of one row; k, v: the sequence's first row.
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

// ------------------------------------------------------------------------------------------------
// Tiles of 64 (or 32) rows of one head in LDS, brought there by loads that write LDS themselves: for each 32 dimensions a part of 64 bytes a row.  LDS serves 256
// bytes a cycle from as many banks.  Within four rows the transposing read (32 lanes: 64 bytes of four consecutive rows each) meets no bank twice as it
// is; for 16 lanes that read one 16-byte piece of 16 consecutive rows each, a row's four pieces are permuted by its number's bits 2 and 3.  Operand
// addresses are then two of a lane and constants, for either read.
template <int HD, int ROWS = 64> struct Tile {
    static constexpr int PARTS = HD / 32, PART = ROWS * 64, BYTES = PARTS * PART;
};
__device__ __forceinline__ int swizzle(int row) { return (row >> 2) & 3; }
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

template <class T> __device__ __forceinline__ f32x16 mma(const u32x4& x, const u32x4& y, const f32x16& c) {
    if constexpr (std::is_same_v<T, __bf16>) return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(Vec8<__bf16>, x), __builtin_bit_cast(Vec8<__bf16>, y), c, 0, 0, 0);
    else return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(Vec8<_Float16>, x), __builtin_bit_cast(Vec8<_Float16>, y), c, 0, 0, 0);
}
template <class T> __device__ __forceinline__ uint32_t pack2(float x, float y) {            // rounded to nearest
    typedef T Pair __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, Pair{(T)x, (T)y});
}
__device__ __forceinline__ f32x16 zeros() {
    f32x16 z;
#pragma unroll
    for (int r = 0; r < 16; ++r) z[r] = 0.f;
    return z;
}

// 64 lanes x 16 bytes straight to 1 KB of LDS at `to` (wave-uniform), IMM counted on both sides; what lies beyond the buffer's end comes as zeros
template <int IMM> __device__ __forceinline__ void to_lds(__amdgpu_buffer_rsrc_t from, char* to, uint32_t off) {
    __builtin_amdgcn_raw_ptr_buffer_load_lds(from, (__attribute__((address_space(3))) void*)to, 16, off, 0, IMM, 0);
}
__device__ __forceinline__ __amdgpu_buffer_rsrc_t buffer_upto(const void* p, uint32_t bytes) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), 0, bytes, 0x00027000);
}

// What a wave of four brings of a tile: 16 of its rows.  Rows past the sequence's end come as zeros: the buffer descriptor ends there.
template <int HD> struct Bring {
    uint32_t off, row_bytes;
    __device__ __forceinline__ Bring(long long stride, int wave, int lane) : row_bytes((uint32_t)stride * 2u) {
        const int row = wave * 16 + (lane >> 2);
        off = row * row_bytes + (((lane & 3) ^ swizzle(row)) * 16);
    }
    // first: the tile's first row, of `rows` that are there
    __device__ __forceinline__ void operator()(const void* first, int rows, char* lds, int wave) const {
        // (a descriptor has to be in scalar registers: one that the compiler keeps in vector registers costs a loop a load)
        const __amdgpu_buffer_rsrc_t r = buffer_upto(first, __builtin_amdgcn_readfirstlane((uint32_t)max(0, min(rows, 64)) * row_bytes));
        char* to = lds + wave * 1024;
        to_lds<0>(r, to, off);
        if constexpr (HD >= 64) to_lds<64>(r, to + Tile<HD>::PART - 64, off);
        if constexpr (HD >= 128) {
            to_lds<128>(r, to + 2 * Tile<HD>::PART - 128, off);
            to_lds<192>(r, to + 3 * Tile<HD>::PART - 192, off);
        }
    }
};

// The same of a tile of 32 rows, 16 rows of a part a load: HD / 16 loads, of which a wave of four makes every fourth.
template <int HD> struct Bring32 {
    static constexpr int LOADS = HD / 16;
    uint32_t off, row_bytes;
    __device__ __forceinline__ Bring32(long long stride, int wave, int lane) : row_bytes((uint32_t)stride * 2u) {
        const int row = (wave & 1) * 16 + (lane >> 2);
        off = row * row_bytes + (((lane & 3) ^ swizzle(row)) * 16) + (wave >> 1) * 64;
    }
    __device__ __forceinline__ void operator()(const void* first, int rows, char* lds, int wave) const { bring(first, rows, lds, wave, off); }
    // with the last row in the place of those past the end; rows >= 1, row: the lane's
    __device__ __forceinline__ void repeat_last(const void* first, int rows, char* lds, int wave, int row) const {
        uint32_t at = off;
        if (__builtin_amdgcn_readfirstlane(rows) < 32) at -= (uint32_t)max(0, row - (rows - 1)) * row_bytes;      // (asked for, whole tiles do not pay: 62 -> 60 us, 37 of U[3, 999])
        bring(first, rows, lds, wave, at);
    }
    __device__ __forceinline__ void bring(const void* first, int rows, char* lds, int wave, uint32_t at) const {
        const __amdgpu_buffer_rsrc_t r = buffer_upto(first, __builtin_amdgcn_readfirstlane((uint32_t)max(0, min(rows, 32)) * row_bytes));
        char* to = lds + wave * 1024;
        if (LOADS >= 4 || wave < LOADS) to_lds<0>(r, to, at);
        if constexpr (LOADS > 4) to_lds<128>(r, to + 4096 - 128, at);
    }
};

// A matrix operand's lane holds a row (l32 of 32) and eight of 16 contracted elements (the half that lh says).
// By rows: the contraction runs along the row.  Transposed: operand rows are dimensions, the contraction runs over the tile's rows, of 16 in the order
// 4 lh .. + 3, 8 + 4 lh .. + 3: that in which a product's result leaves them.
template <int HD, int ROWS = 64> struct Reads {
    int row[2], col[2];                       // of a lane: its row's piece of the first 16 elements and of the second; its transposed corner, and that 8 rows on
    __device__ __forceinline__ Reads(int lane) {
        const int l32 = lane & 31, lh = lane >> 5, i = lane & 15, r = 4 * lh + (i >> 2);
        row[0] = l32 * 64 + ((lh ^ swizzle(l32)) * 16);
        row[1] = row[0] ^ 32;
        col[0] = r * 64 + (((2 * ((lane >> 4) & 1) + ((i & 3) >> 1)) ^ swizzle(r)) * 16) + (i & 1) * 8;
        col[1] = (col[0] ^ 32) + 8 * 64;
    }
    // rows 32 half .. + 31, elements 16 ks .. + 15
    __device__ __forceinline__ u32x4 by_row(const char* tile, int half, int ks) const {
        return *(const u32x4*)(tile + row[ks & 1] + (ks >> 1) * Tile<HD, ROWS>::PART + half * 32 * 64);
    }
    // dimensions 32 dt .. + 31, rows 16 group .. + 15
    __device__ __forceinline__ u32x4 transposed(const char* tile, int group, int dt) const {
        typedef __attribute__((address_space(3))) s16x4 Corner;
        const char* p = tile + dt * Tile<HD, ROWS>::PART + group * 16 * 64;
        const u32x2 lo = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((Corner*)(p + col[0])));
        const u32x2 hi = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((Corner*)(p + col[1])));
        return u32x4{lo.x, lo.y, hi.x, hi.y};
    }
};

// 32 rows of a head in registers, as a matrix operand: row l32 (zeros where `there` is false), elements 16 ks + 8 lh .. + 7
template <int HD> __device__ __forceinline__ void hold(u32x4 (&f)[HD / 16], const void* row, bool there, int lh) {
#pragma unroll
    for (int ks = 0; ks < HD / 16; ++ks) {
        const u32x4 v = *(const u32x4*)((const char*)row + ks * 32 + lh * 16);
        f[ks] = there ? v : u32x4{0u, 0u, 0u, 0u};
    }
}

// Writes 32 rows of results whose transpose the wave holds (lane: row l32; registers 4b .. 4b + 3 of tile dt: dimensions 32 dt + 8 b + 4 lh .. + 3), each times its
// row's factor, through a private part of LDS, so that whole rows leave.  Nothing here reads them again: stored past the caches' order of use, they leave it to keys and
// values (forward, 24 sequences of U[256, 1024]: 144 -> 130 us).  Loads of the same kind, of q, cost 153: a line serves eight of them.
template <class T, int HD>
__device__ __forceinline__ void put_rows(const f32x16 (&acc)[HD / 32], float factor, char* lds, T* first, long long stride, int n_valid, int lane) {
    constexpr int ROW = HD * 2 + 16;          // bytes between rows: 16 lanes that write 8 bytes of 16 rows each
    const int l32 = lane & 31, lh = lane >> 5;
#pragma unroll
    for (int dt = 0; dt < HD / 32; ++dt)
#pragma unroll
        for (int b = 0; b < 4; ++b)
            *(u32x2*)(lds + l32 * ROW + (dt * 32 + b * 8 + lh * 4) * 2) = u32x2{pack2<T>(acc[dt][4 * b] * factor, acc[dt][4 * b + 1] * factor),
                                                                            pack2<T>(acc[dt][4 * b + 2] * factor, acc[dt][4 * b + 3] * factor)};
    __builtin_amdgcn_wave_barrier();
    constexpr int LANES = HD / 8;             // of a row
#pragma unroll
    for (int u = 0; u < 32 * LANES / 64; ++u) {
        const int row = u * (64 / LANES) + lane / LANES, piece = lane % LANES;
        const u32x4 v = *(const u32x4*)(lds + row * ROW + piece * 16);
        if (row < n_valid) __builtin_nontemporal_store(v, (u32x4*)(first + (size_t)row * stride + piece * 8));
    }
}
template <int HD> constexpr int kPutBytes = 32 * (HD * 2 + 16);

template <int N> __device__ __forceinline__ bool any_undefined(const f32x16 (&acc)[N]) {
    bool bad = false;
#pragma unroll
    for (int t = 0; t < N; ++t)
#pragma unroll
        for (int r = 0; r < 16; ++r) bad = bad || acc[t][r] != acc[t][r];
    return bad;
}
// whether a row of HD elements has one that is infinite or undefined
template <class T, int HD> __device__ __forceinline__ bool not_finite(const T* row) {
    float s = 0.f;
#pragma unroll 1
    for (int d = 0; d < HD; d += 8) {
        const Vec8<T> x = *(const Vec8<T>*)(row + d);
#pragma unroll
        for (int e = 0; e < 8; ++e) s = fmaf((float)x[e], 0.f, s);
    }
    return s != s;
}

// A workgroup's place: four units of a (sequence, kv head), a unit being 32 positions of one query head; units are counted heads first.  Stages of so many tokens,
// of the workgroup and of the wave.
template <int TOKENS> struct Unit {
    int row0, len, kvh, h, pos0, n_valid, stages, my_stages;
    bool active;
    __device__ __forceinline__ Unit(const PackArgs& a, int wave) {
        const int4 it = a.q_items[a.first_item + blockIdx.y];
        const int G = a.n_q_heads / a.n_kv_heads;
        row0 = it.x; len = it.y; kvh = blockIdx.x;
        const int tiles = (len + 31) >> 5, u = it.z * 4 + wave, tile = u / G, last = min(it.z * 4 + 3, tiles * G - 1) / G;
        active = tile < tiles;
        h = kvh * G + (active ? u - tile * G : 0);
        pos0 = active ? tile * 32 : 0;
        n_valid = active ? min(32, len - pos0) : 0;
        stages = (last * 32 + 32 + TOKENS - 1) / TOKENS;
        my_stages = active ? (pos0 + 32 + TOKENS - 1) / TOKENS : 0;
    }
};

// Powers of two that weights reach before the reference moves, and that the largest has when it has moved.  Half precision's normal numbers end at 2^-14 and at 2^16: there the
// largest is 2^7 at least, so that weights keep their 11 bits down to 2^-21 of it, and 2^12 at most: scores of 2^26 are off by 4 themselves.
template <class T> constexpr float kMost = std::is_same_v<T, _Float16> ? 12.f : 8.f;
template <class T> constexpr float kTop = std::is_same_v<T, _Float16> ? 7.f : 0.f;
// Stages of 32 tokens, of which the wave's last is the one on the diagonal.  Three workgroups share a compute unit, and what one waits for (its tiles, its barrier, the
// matrix pipe, its exponentials) the others fill: two of them with stages of 64 tokens, the next stage's scores made under the weights of this one, took
// 1,160 us where this took 1,054 (16 sequences of U[1024, 4096], 32 heads on 8), 164 where it took 143 (24 of U[256, 1024]).
template <class T, int HD>
__global__ __launch_bounds__(256, 3) void pack_forward_kernel(PackArgs a) {
    constexpr int KS = HD / 16, DT = HD / 32, TB = Tile<HD, 32>::BYTES;
    __shared__ __attribute__((aligned(1024))) char lds[4 * TB > 4 * kPutBytes<HD> ? 4 * TB : 4 * kPutBytes<HD>];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l32 = lane & 31, lh = lane >> 5;
    const Unit<32> w(a, wave);
    const T* k = (const T*)a.k + (size_t)w.row0 * a.k_stride + w.kvh * HD;
    const T* v = (const T*)a.v + (size_t)w.row0 * a.v_stride + w.kvh * HD;
    const Bring32<HD> bring_k(a.k_stride, wave, lane), bring_v(a.v_stride, wave, lane);
    const Reads<HD, 32> at(lane);
    auto bring = [&](int st) {
        char* to = lds + (st & 1) * 2 * TB;
        bring_k(k + (size_t)st * 32 * a.k_stride, w.len - st * 32, to, wave);
        bring_v(v + (size_t)st * 32 * a.v_stride, w.len - st * 32, to + TB, wave);
    };
    bring(0);
    const bool there = l32 < w.n_valid;
    const size_t my_row = (size_t)w.row0 + (there ? w.pos0 + l32 : 0);
    u32x4 qf[KS];
    hold<HD>(qf, (const T*)a.q + my_row * a.q_stride + w.h * HD, there, lh);
    f32x16 acc[DT];
#pragma unroll
    for (int d = 0; d < DT; ++d) acc[d] = zeros();
    float m = kLeast, l = 0.f;
    for (int st = 0; st < w.stages; ++st) {
        // This stage's tiles are here, and those that the next loads go over have been read (a barrier does not wait for either by itself).
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        if (st + 1 < w.stages) bring(st + 1);
        if (st >= w.my_stages) continue;
        const char* kt = lds + (st & 1) * 2 * TB;
        f32x16 s = zeros();
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) s = mma<T>(at.by_row(kt, 0, ks), qf[ks], s);
        if (st == w.my_stages - 1) {
#pragma unroll
            for (int r = 0; r < 16; ++r)
                if (8 * (r >> 2) + 4 * lh + (r & 3) > l32) s[r] = -INFINITY;
        }
        float mx = s[0];
#pragma unroll
        for (int r = 1; r < 16; ++r) mx = fmaxf(mx, s[r]);
        const auto both = __builtin_amdgcn_permlane32_swap(__float_as_int(mx), __float_as_int(mx), false, false);
        mx = fmaxf(__int_as_float(both[0]), __int_as_float(both[1])) * a.scale_log2e;
        if (__builtin_amdgcn_ballot_w64(mx > m + kMost<T>) != 0) {     // the reference moves only where weights would pass 2^kMost
            const float m_new = fmaxf(m, mx - kTop<T>), shrink = __builtin_amdgcn_exp2f(m - m_new);
            l *= shrink;
#pragma unroll
            for (int d = 0; d < DT; ++d)
#pragma unroll
                for (int r = 0; r < 16; ++r) acc[d][r] *= shrink;
            m = m_new;
        }
        u32x4 p[2];
#pragma unroll
        for (int r = 0; r < 16; r += 2) {
            const float x = __builtin_amdgcn_exp2f(fmaf(s[r], a.scale_log2e, -m)), y = __builtin_amdgcn_exp2f(fmaf(s[r + 1], a.scale_log2e, -m));
            l += x + y;
            p[r >> 3][(r >> 1) & 3] = pack2<T>(x, y);
        }
#pragma unroll
        for (int g = 0; g < 2; ++g)
#pragma unroll
            for (int d = 0; d < DT; ++d) acc[d] = mma<T>(at.transposed(kt + TB, g, d), p[g], acc[d]);
    }
    __syncthreads();                              // the last tiles have been read
    if (!w.active) return;
    l += __shfl_xor(l, 32, 64);
    T* out = (T*)a.out + ((size_t)w.row0 + w.pos0) * a.out_stride + w.h * HD;
    float* lse = a.lse + (size_t)w.h * a.n_rows + w.row0 + w.pos0;
    put_rows<T, HD>(acc, 1.f / l, lds + wave * kPutBytes<HD>, out, a.out_stride, w.n_valid, lane);
    if (lh == 0 && there) lse[l32] = (m + __builtin_amdgcn_logf(l)) * kLn2;
    // A weight of 0 times an infinite or undefined value of a token that the row does not see: such rows are computed alone.  (Where l is undefined, so is the row.)
    uint64_t rows = __builtin_amdgcn_ballot_w64(there && l == l && any_undefined(acc));
    rows = (rows | (rows >> 32)) & 0xFFFFFFFFull;
    if (rows) {
        const int t0 = w.pos0, t = t0 + lane;
        const uint64_t odd = __builtin_amdgcn_ballot_w64(lane < 32 && t < w.len && not_finite<T, HD>(v + (size_t)t * a.v_stride));
        while (rows) {
            const int r = __builtin_ctzll(rows);
            rows &= rows - 1;
            if (odd >> (w.pos0 + r - t0) >> 1)
                forward_row<T, HD>(a, k, v, (const T*)a.q + ((size_t)w.row0 + w.pos0 + r) * a.q_stride + w.h * HD, w.pos0 + r, out + (size_t)r * a.out_stride, lse + r, lane);
        }
    }
}

template <class T, int HD>
__global__ __launch_bounds__(256, 2) void pack_dq_kernel(PackArgs a) {
    constexpr int KS = HD / 16, DT = HD / 32, TB = Tile<HD>::BYTES;
    __shared__ __attribute__((aligned(1024))) char lds[4 * TB > 4 * kPutBytes<HD> ? 4 * TB : 4 * kPutBytes<HD>];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l32 = lane & 31, lh = lane >> 5;
    const Unit<64> w(a, wave);
    const T* k = (const T*)a.k + (size_t)w.row0 * a.k_stride + w.kvh * HD;
    const T* v = (const T*)a.v + (size_t)w.row0 * a.v_stride + w.kvh * HD;
    const Bring<HD> bring_k(a.k_stride, wave, lane), bring_v(a.v_stride, wave, lane);
    const Reads<HD> at(lane);
    auto bring = [&](int st) {
        char* to = lds + (st & 1) * 2 * TB;
        bring_k(k + (size_t)st * 64 * a.k_stride, w.len - st * 64, to, wave);
        bring_v(v + (size_t)st * 64 * a.v_stride, w.len - st * 64, to + TB, wave);
    };
    bring(0);
    const bool there = l32 < w.n_valid;
    const size_t my_row = (size_t)w.row0 + (there ? w.pos0 + l32 : 0);
    u32x4 qf[KS], df[KS];
    hold<HD>(qf, (const T*)a.q + my_row * a.q_stride + w.h * HD, there, lh);
    hold<HD>(df, (const T*)a.dout + my_row * a.dout_stride + w.h * HD, there, lh);
    float delta = 0.f;
    {
        const T* o = (const T*)a.out_in + my_row * a.out_stride + w.h * HD + lh * 8;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            const Vec8<T> x = *(const Vec8<T>*)(o + ks * 16), y = __builtin_bit_cast(Vec8<T>, df[ks]);
#pragma unroll
            for (int e = 0; e < 8; ++e) delta = fmaf((float)x[e], (float)y[e], delta);
        }
        delta += __shfl_xor(delta, 32, 64);
    }
    const float lse = there ? a.lse[(size_t)w.h * a.n_rows + my_row] : INFINITY, lse2 = lse * kLog2e;
    if (!there) delta = 0.f;
    f32x16 acc[DT];
#pragma unroll
    for (int d = 0; d < DT; ++d) acc[d] = zeros();
    const int limit = w.pos0 + l32;

    auto arrive = [&](int st) {
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        if (st + 1 < w.stages) bring(st + 1);
    };
    auto products = [&](f32x16& s, f32x16& dp, int st, int half) {
        const char* kt = lds + (st & 1) * 2 * TB;
        s = zeros(); dp = zeros();
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) s = mma<T>(at.by_row(kt, half, ks), qf[ks], s);
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) dp = mma<T>(at.by_row(kt + TB, half, ks), df[ks], dp);
    };
    auto add = [&](const u32x4 (&t)[2], int st, int half) {
        const char* kt = lds + (st & 1) * 2 * TB;
#pragma unroll
        for (int g = 0; g < 2; ++g)
#pragma unroll
            for (int d = 0; d < DT; ++d) acc[d] = mma<T>(at.transposed(kt, half * 2 + g, d), t[g], acc[d]);
    };
    auto hidden = [&](int st, int half, int r) { return st * 64 + half * 32 + 8 * (r >> 2) + 4 * lh + (r & 3) > limit; };
    arrive(0);
    if (w.my_stages == 1) {
        // All that the rows see is here, so that D can be had as sum p dp.  From `out`, whose rounding is in it, it is off by 2^-9 of what dp - D, where a
        // row sees few tokens, nearly cancels to (dq of sequences of 2 to 20 tokens: 0.4 % off, now 0.24).
        // Divided by sum p, which the rounding of lse leaves off 1 by 2^-24 of a large score: where one token has nearly all the weight, that times dp would stand for dp - D.
        float sum = 0.f, weight = 0.f;
#pragma unroll 1
        for (int half = 0; half < 2; ++half) {
            f32x16 s, dp;
            products(s, dp, 0, half);
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const float p = __builtin_amdgcn_exp2f(fmaf(s[r], a.scale_log2e, -lse2));
                sum += hidden(0, half, r) ? 0.f : p * dp[r];
                weight += hidden(0, half, r) ? 0.f : p;
            }
        }
        delta = there ? (sum + __shfl_xor(sum, 32, 64)) / (weight + __shfl_xor(weight, 32, 64)) : 0.f;
    }
    auto both_products = [&](int st, int half, auto cut) {
        f32x16 s, dp;
        products(s, dp, st, half);
        u32x4 t[2];
#pragma unroll
        for (int r = 0; r < 16; r += 2) {
            float x[2];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                x[e] = __builtin_amdgcn_exp2f(fmaf(s[r + e], a.scale_log2e, -lse2)) * (dp[r + e] - delta);
                if (cut && hidden(st, half, r + e)) x[e] = 0.f;
            }
            t[r >> 3][(r >> 1) & 3] = pack2<T>(x[0], x[1]);
        }
        add(t, st, half);
    };
    const int whole = w.my_stages - 1;            // stages that all of the wave's rows see
    for (int st = 0; st < w.stages; ++st) {
        if (st > 0) arrive(st);
        if (st < whole) {
            // (one copy of the body at 128 dimensions, two leave it too few registers to read operands ahead: 1.76 -> 1.69 ms; below it is 3 % the other way)
#pragma unroll(HD == 128 ? 1 : 2)
            for (int half = 0; half < 2; ++half) both_products(st, half, std::false_type());
        } else if (st == whole) {
            both_products(st, 0, std::true_type());
            if (st * 64 + 32 <= w.pos0 + 31) both_products(st, 1, std::true_type());
        }
    }
    __syncthreads();
    if (!w.active) return;
    if (there && lh == 0) a.delta[(size_t)w.h * a.n_rows + my_row] = delta;          // the kernel of dk and dv takes it from there
    T* dq = (T*)a.dq + ((size_t)w.row0 + w.pos0) * a.dq_stride + w.h * HD;
    put_rows<T, HD>(acc, a.scale, lds + wave * kPutBytes<HD>, dq, a.dq_stride, w.n_valid, lane);
    uint64_t rows = __builtin_amdgcn_ballot_w64(there && lse == lse && delta == delta && any_undefined(acc));      // as in the forward kernel, of keys
    rows = (rows | (rows >> 32)) & 0xFFFFFFFFull;
    if (rows) {
        const int t0 = (w.my_stages - 1) * 64, t = t0 + lane;
        const uint64_t odd = __builtin_amdgcn_ballot_w64(t < w.len && not_finite<T, HD>(k + (size_t)t * a.k_stride));
        while (rows) {
            const int r = __builtin_ctzll(rows);
            rows &= rows - 1;
            const size_t row = (size_t)w.row0 + w.pos0 + r;
            if (odd >> (w.pos0 + r - t0) >> 1)
                dq_row<T, HD>(a, k, v, (const T*)a.q + row * a.q_stride + w.h * HD, (const T*)a.dout + row * a.dout_stride + w.h * HD, __shfl(lse, r, 64), __shfl(delta, r, 64),
                              w.pos0 + r, dq + (size_t)r * a.dq_stride, lane);
        }
    }
}

// 128 tokens of a kv head a workgroup, 32 a wave; rows pass by, 32 at a time, from the sequence's end to the tokens, each time of all heads of the group (or a part of
// them).  Keys stay in registers, values in LDS: with both in registers, beside two accumulators, there are too few left to read operands ahead.
// A wave's last stages are those of its tokens' own rows, some of which do not see some tokens.  Where one of these rows is not finite, as its lse (of q) or D (of dout) then
// is, the stage is left out, as a weight of 0 would not keep it out of the sums; this head's rows and those of the heads behind it are then added pair by pair.
// In half precision, whose normal numbers end at 2^-14, the p of dv are 2^12 times as large, from exponents that are 12 more, and their sums 2^12 times less at the end: p of long
// histories, and of tokens beside one that takes nearly all, keep their bits down to 2^-26 (p is at most 1, but for the roundings of large scores, so none passes the range).
// dp - D is made 2^12 times less, and t is what it was.
template <class T> constexpr int kUp = std::is_same_v<T, _Float16> ? 12 : 0;
template <class T> constexpr float kDown = 1.f / (1 << kUp<T>);
template <int HD> constexpr int kDkvBytes = 2 * Tile<HD>::BYTES + 4 * Tile<HD, 32>::BYTES + 512;
template <class T, int HD, bool PARTS>
__global__ __launch_bounds__(256, 2) void pack_dkv_kernel(PackArgs a) {
    constexpr int KS = HD / 16, DT = HD / 32, TB = Tile<HD, 32>::BYTES;
    extern __shared__ __attribute__((aligned(1024))) char lds[];
    static_assert(4 * kPutBytes<HD> <= kDkvBytes<HD>, "results leave through the same LDS");
    char* const stages_lds = lds + 2 * Tile<HD>::BYTES;                          // [stage parity][queries, gradients]
    float* const s_row = (float*)(stages_lds + 4 * TB);                         // [stage parity][lse2, -delta][row]
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l32 = lane & 31, lh = lane >> 5;
    const int4 it = a.k_items[a.first_item + blockIdx.y];
    const int row0 = it.x, len = it.y, block0 = it.z * 128, G = a.n_q_heads / a.n_kv_heads;
    const int kvh = blockIdx.x % a.n_kv_heads, part = blockIdx.x / a.n_kv_heads;
    const int h0 = kvh * G + part * G / a.parts, h1 = kvh * G + (part + 1) * G / a.parts;
    const int tok0 = block0 + wave * 32, n_valid = max(0, min(32, len - tok0));
    const int q_stages = (len - block0 + 31) >> 5, stages = q_stages * (h1 - h0);
    const Bring32<HD> bring_q(a.q_stride, wave, lane), bring_d(a.dout_stride, wave, lane);
    int next_h = h0, next_q = block0 + (q_stages - 1) * 32;      // of the stage to be brought next
    float row_value = 0.f;                        // its row l32's lse or delta
    bool row_there = false;
    auto bring = [&](int st) {
        char* to = stages_lds + (st & 1) * 2 * TB;
        // Rows behind the last weigh exp2(s - inf): 0, if their score is that of a row that is there.  Zeros would meet a key's infinity, which for the sequence's rows may be
        // a score of -inf.
        bring_q.repeat_last((const T*)a.q + (size_t)(row0 + next_q) * a.q_stride + next_h * HD, len - next_q, to, wave, (wave & 1) * 16 + (lane >> 2));
        bring_d((const T*)a.dout + (size_t)(row0 + next_q) * a.dout_stride + next_h * HD, len - next_q, to + TB, wave);
        if (wave == 0) row_value = ((lh ? a.delta : a.lse) + (size_t)next_h * a.n_rows + row0 + next_q)[min(l32, len - 1 - next_q)];
        row_there = next_q + l32 < len;
        if (++next_h == h1) { next_h = h0; next_q -= 32; }
    };
    auto park = [&](int st) {                     // rows that are not there weigh nothing
        if (wave == 0) s_row[(st & 1) * 64 + lane] = lh ? (row_there ? -row_value : 0.f) : row_there ? fmaf(row_value, kLog2e, (float)-kUp<T>) : INFINITY;
    };
    {
        const Bring<HD> bring_v(a.v_stride, wave, lane);
        const T* v = (const T*)a.v + (size_t)(row0 + block0) * a.v_stride + kvh * HD;
        bring_v(v, len - block0, lds, wave);
        bring_v(v + (size_t)64 * a.v_stride, len - block0 - 64, lds + Tile<HD>::BYTES, wave);
    }
    bring(0);
    const bool there = l32 < n_valid;
    u32x4 kf[KS];
    hold<HD>(kf, (const T*)a.k + ((size_t)row0 + (there ? tok0 + l32 : 0)) * a.k_stride + kvh * HD, there, lh);
    f32x16 dk[DT], dv[DT];
#pragma unroll
    for (int d = 0; d < DT; ++d) dk[d] = zeros(), dv[d] = zeros();
    park(0);
    const Reads<HD> at_v(lane);
    const Reads<HD, 32> at(lane);
    const char* vt = lds + (wave >> 1) * Tile<HD>::BYTES;
    int q0 = block0 + (q_stages - 1) * 32, h = h0, alone_from = h1;
    for (int st = 0; st < stages; ++st) {
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        const bool more = st + 1 < stages;
        if (more) bring(st + 1);
        const char* qt = stages_lds + (st & 1) * 2 * TB;
        const char* ot = qt + TB;
        const float* rows = s_row + (st & 1) * 64 + lh * 4;
        if (n_valid > 0 && q0 == tok0) {
            const float x = s_row[(st & 1) * 64 + lane];
            if (__builtin_amdgcn_ballot_w64(there && !(fabsf(x) < INFINITY)) != 0) alone_from = min(alone_from, h);
        }
        if (n_valid > 0 && (q0 > tok0 || (q0 == tok0 && h < alone_from))) {
            f32x16 s = zeros(), dp;               // dp - D: its sums start at -D, which pays for the factor below (37 of U[3, 999], fp16: 151.5 us, 154.5 with the factor alone, 151 so)
#pragma unroll
            for (int b = 0; b < 4; ++b) {
                const f32x4 d = *(const f32x4*)(rows + 32 + b * 8);
#pragma unroll
                for (int e = 0; e < 4; ++e) dp[4 * b + e] = d[e];
            }
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) s = mma<T>(at.by_row(qt, 0, ks), kf[ks], s);
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) dp = mma<T>(at.by_row(ot, 0, ks), at_v.by_row(vt, wave & 1, ks), dp);
            // Rows before the lane's token.  Asked with a uniform `cut` first, whole stages pay nothing (128 dimensions, 16 sequences of U[1024, 4096]: 2.18 -> 2.09 ms);
            // where products are half as long, a comparison and two choices an element are cheaper than what becomes of that (64 dimensions, 37 of U[3, 999], forward and backward:
            // 156 us, this way 151.5; 154 with t itself chosen).  dp - D is chosen as well as p: 0 times what passes 32 bits, dout . v of rows that do not see a large v, would be undefined.
            const bool cut = q0 < tok0 + 31;
            const int first_row = cut ? tok0 + l32 - q0 - lh * 4 : -1;
            u32x4 p[2], t[2];
#pragma unroll
            for (int b = 0; b < 4; ++b) {
                const f32x4 lse2 = *(const f32x4*)(rows + b * 8);
                float x[4], y[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    x[e] = __builtin_amdgcn_exp2f(fmaf(s[4 * b + e], a.scale_log2e, -lse2[e]));
                    float along = dp[4 * b + e] * kDown<T>;
                    if (HD < 128 && b * 8 + e < first_row) x[e] = along = 0.f;
                    y[e] = x[e] * along;
                    if (HD == 128 && cut && q0 + b * 8 + lh * 4 + e < tok0 + l32) x[e] = y[e] = 0.f;
                }
                p[b >> 1][(b & 1) * 2] = pack2<T>(x[0], x[1]); p[b >> 1][(b & 1) * 2 + 1] = pack2<T>(x[2], x[3]);
                t[b >> 1][(b & 1) * 2] = pack2<T>(y[0], y[1]); t[b >> 1][(b & 1) * 2 + 1] = pack2<T>(y[2], y[3]);
            }
#pragma unroll
            for (int g = 0; g < 2; ++g)
#pragma unroll
                for (int d = 0; d < DT; ++d) dv[d] = mma<T>(at.transposed(ot, g, d), p[g], dv[d]);
#pragma unroll
            for (int g = 0; g < 2; ++g)
#pragma unroll
                for (int d = 0; d < DT; ++d) dk[d] = mma<T>(at.transposed(qt, g, d), t[g], dk[d]);
        }
        if (++h == h1) { h = h0; q0 -= 32; }
        if (more) park(st + 1);
    }
    __syncthreads();
    if (n_valid <= 0) return;
    const size_t first = (size_t)row0 + tok0;
#pragma unroll 1
    for (int g = alone_from; g < h1; ++g) {
        const T* k = (const T*)a.k + (first + (there ? l32 : 0)) * a.k_stride + kvh * HD + lh * 8;
        const T* v = (const T*)a.v + (first + (there ? l32 : 0)) * a.v_stride + kvh * HD + lh * 8;
#pragma unroll 1
        for (int i = 0; i < n_valid; ++i) {
            const T* q = (const T*)a.q + (first + i) * a.q_stride + g * HD;
            const T* o = (const T*)a.dout + (first + i) * a.dout_stride + g * HD;
            float sc = 0.f, dp = 0.f;                 // the lane's half of the dimensions, then both
#pragma unroll 1
            for (int c = 0; c < HD; c += 16) sc = dot8(q + c + lh * 8, k + c, sc), dp = dot8(o + c + lh * 8, v + c, dp);
            sc += __shfl_xor(sc, 32, 64);
            dp += __shfl_xor(dp, 32, 64);
            const float p = exp2f(sc * a.scale_log2e - a.lse[(size_t)g * a.n_rows + first + i] * kLog2e), t = p * (dp - a.delta[(size_t)g * a.n_rows + first + i]);
            const float up = p * (float)(1 << kUp<T>);
            if (l32 <= i && there)
#pragma unroll
                for (int d = 0; d < DT; ++d)
#pragma unroll
                    for (int r = 0; r < 16; ++r) {
                        const int at_d = d * 32 + 8 * (r >> 2) + 4 * lh + (r & 3);
                        dv[d][r] = fmaf(up, (float)o[at_d], dv[d][r]);
                        dk[d][r] = fmaf(t, (float)q[at_d], dk[d][r]);
                        asm volatile("" ::: "memory");      // a few loads at a time: more would take the registers that the loop above needs
                    }
        }
    }
    if constexpr (PARTS) {                        // fp32 [part][dk or dv][row][kv head][HD]: the lane's row, four dimensions at a time
        if (there) {
            const size_t width = (size_t)a.n_kv_heads * HD, plane = (size_t)a.n_rows * width;
            float* to = a.part + (size_t)part * 2 * plane + (first + l32) * width + kvh * HD + lh * 4;
#pragma unroll
            for (int d = 0; d < DT; ++d)
#pragma unroll
                for (int b = 0; b < 4; ++b) {
                    *(f32x4*)(to + d * 32 + b * 8) = f32x4{dk[d][4 * b], dk[d][4 * b + 1], dk[d][4 * b + 2], dk[d][4 * b + 3]};
                    *(f32x4*)(to + plane + d * 32 + b * 8) = f32x4{dv[d][4 * b], dv[d][4 * b + 1], dv[d][4 * b + 2], dv[d][4 * b + 3]};
                }
        }
    } else {
        char* mine = lds + wave * kPutBytes<HD>;
        put_rows<T, HD>(dk, a.scale, mine, (T*)a.dk + first * a.dk_stride + kvh * HD, a.dk_stride, n_valid, lane);
        __builtin_amdgcn_wave_barrier();
        put_rows<T, HD>(dv, kDown<T>, mine, (T*)a.dv + first * a.dv_stride + kvh * HD, a.dv_stride, n_valid, lane);
    }
}

// dk and dv as the sums of their parts: eight dimensions a thread
template <class T>
__global__ __launch_bounds__(256) void pack_join_kernel(PackArgs a, int width) {
    const size_t i = ((size_t)blockIdx.x * 256 + threadIdx.x) * 8, plane = (size_t)a.n_rows * width;
    if (i >= 2 * plane) return;
    const bool is_v = i >= plane;
    float g[8] = {};
    for (int p = 0; p < a.parts; ++p) {
        const f32x4 x = *(const f32x4*)(a.part + (size_t)p * 2 * plane + i), y = *(const f32x4*)(a.part + (size_t)p * 2 * plane + i + 4);
#pragma unroll
        for (int e = 0; e < 4; ++e) g[e] += x[e], g[4 + e] += y[e];
    }
    const size_t j = is_v ? i - plane : i, row = j / width;
    T* to = (is_v ? (T*)a.dv + row * a.dv_stride : (T*)a.dk + row * a.dk_stride) + (j - row * width);
    const float c = is_v ? kDown<T> : a.scale;
    *(u32x4*)to = u32x4{pack2<T>(g[0] * c, g[1] * c), pack2<T>(g[2] * c, g[3] * c), pack2<T>(g[4] * c, g[5] * c), pack2<T>(g[6] * c, g[7] * c)};
}

constexpr int kMostItems = 65535;                 // of a launch: its second dimension

hipError_t in_launches(void (*kernel)(PackArgs), PackArgs a, int items, int wide, int lds, hipStream_t s) {
    if (lds > 65536) {
        const hipError_t e = hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, lds);
        if (e != hipSuccess) return e;
    }
    for (a.first_item = 0; a.first_item < items; a.first_item += kMostItems) {
        hipLaunchKernelGGL(kernel, dim3(wide, items - a.first_item < kMostItems ? items - a.first_item : kMostItems), dim3(256), lds, s, a);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

template <class T, int HD> hipError_t forward_impl(const PackArgs& a, hipStream_t s) {
    return in_launches(pack_forward_kernel<T, HD>, a, a.n_q_items, a.n_kv_heads, 0, s);
}
template <class T, int HD> hipError_t backward_impl(const PackArgs& a, hipStream_t s) {
    hipError_t e = in_launches(pack_dq_kernel<T, HD>, a, a.n_q_items, a.n_kv_heads, 0, s);
    if (e != hipSuccess) return e;
    e = in_launches(a.parts > 1 ? pack_dkv_kernel<T, HD, true> : pack_dkv_kernel<T, HD, false>, a, a.n_k_items, a.n_kv_heads * a.parts, kDkvBytes<HD>, s);
    if (e != hipSuccess || a.parts == 1) return e;
    const size_t vecs = (size_t)a.n_rows * a.n_kv_heads * HD / 4;
    hipLaunchKernelGGL((pack_join_kernel<T>), dim3((unsigned)((vecs + 255) / 256)), dim3(256), 0, s, a, a.n_kv_heads * HD);
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
