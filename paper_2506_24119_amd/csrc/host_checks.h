// What the host sides of the learner's operators check their arguments with.
#pragma once
#include <cstdarg>
#include <cstdio>

#include "spiral_internal.h"

namespace spiral {

static inline int fail(int code, const char* fmt, ...) {
    char text[384];
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(text, sizeof(text), fmt, ap);
    va_end(ap);
    return spiral_set_error(code, text);
}
static inline int done(hipError_t e, const char* who) { return e == hipSuccess ? SPIRAL_OK : fail(SPIRAL_ERR_HIP, "%s: %s", who, hipGetErrorString(e)); }

static inline int dtype_size(int dtype) {          // of logits, parameters and gradients; 0: none of them
    return dtype == SPIRAL_DTYPE_FP32 ? 4 : dtype == SPIRAL_DTYPE_BF16 || dtype == SPIRAL_DTYPE_FP16 ? 2 : 0;
}
static inline bool aligned(const void* p, size_t to) { return ((uintptr_t)p & (to - 1)) == 0; }

// Of a call's buffers none that is written may be another one too: workgroups would read what others have already written.
struct Span { uintptr_t lo, hi; bool written; };
static inline Span span_of(const void* p, size_t bytes, bool written) { return {(uintptr_t)p, (uintptr_t)p + (p ? bytes : 0), written}; }
static inline uintptr_t matrix_bytes(long long rows, long long stride, int V, int size) { return ((uintptr_t)(rows - 1) * stride + V) * size; }
static inline bool any_overlap(const Span* s, int n) {
    for (int i = 0; i < n; ++i)
        for (int j = 0; j < i; ++j)
            if ((s[i].written || s[j].written) && s[i].lo < s[j].hi && s[j].lo < s[i].hi) return true;
    return false;
}

// A matrix whose rows of `width` bytes start `stride` bytes apart.  Two of one stride may lie in each other's gaps, as the heads of one fused projection do.
struct Rows { uintptr_t lo; uintptr_t stride, width; long long n; bool written; };
static inline Rows rows_of(const void* p, long long stride, long long width, long long n, int size, bool written) {
    return {(uintptr_t)p, (uintptr_t)stride * size, (uintptr_t)width * size, p ? n : 0, written};
}
static inline bool rows_meet(const Rows& a, const Rows& b) {
    if (!a.n || !b.n) return false;
    const uintptr_t a_end = a.lo + (uintptr_t)(a.n - 1) * a.stride + a.width, b_end = b.lo + (uintptr_t)(b.n - 1) * b.stride + b.width;
    if (a.lo >= b_end || b.lo >= a_end) return false;
    if (a.n == 1 || b.n == 1 || a.stride != b.stride) return true;          // unequal strides would meet somewhere, or nearly
    const uintptr_t apart = a.lo <= b.lo ? (b.lo - a.lo) % a.stride : (a.stride - (a.lo - b.lo) % a.stride) % a.stride;
    return apart < a.width || apart + b.width > a.stride;
}
static inline bool any_meet(const Rows* r, int n) {
    for (int i = 0; i < n; ++i)
        for (int j = 0; j < i; ++j)
            if ((r[i].written || r[j].written) && rows_meet(r[i], r[j])) return true;
    return false;
}

}  // namespace spiral
