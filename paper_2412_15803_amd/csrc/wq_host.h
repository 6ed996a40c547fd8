// Argument checks shared by the entry points of the cache, window-attention
// and logits sources (host only).
#pragma once

#include <cstdarg>
#include <cstdint>
#include <cstdio>

#include "wq_internal.h"

namespace wq {
namespace host {

// Records a formatted message as the thread's last error and returns `st`.
__attribute__((format(printf, 2, 3))) inline wq_status err(wq_status st, const char* fmt, ...) {
    char msg[512];
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(msg, sizeof(msg), fmt, ap);
    va_end(ap);
    return record_error(st, msg);
}

inline bool aligned(const void* p, uintptr_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }

constexpr bool is_pow2(int64_t v) { return v > 0 && (v & (v - 1)) == 0; }

constexpr int log2_of(int64_t v) {
    int r = 0;
    while ((int64_t(1) << r) < v) ++r;
    return r;
}

struct Span {
    uintptr_t lo, hi;
};
inline Span span(const void* p, uint64_t bytes) {
    const uintptr_t lo = reinterpret_cast<uintptr_t>(p);
    return Span{lo, lo + (uintptr_t)bytes};
}
inline bool overlaps(Span a, Span b) { return a.lo < a.hi && b.lo < b.hi && a.lo < b.hi && b.lo < a.hi; }

// INVALID_ARG unless lo <= v <= hi.
inline wq_status in_range(const char* fn, const char* name, int64_t v, int64_t lo, int64_t hi) {
    if (v >= lo && v <= hi) return WQ_OK;
    return err(WQ_ERR_INVALID_ARG, "%s: %s must be in [%lld, %lld] (got %lld)", fn, name, (long long)lo, (long long)hi, (long long)v);
}

inline wq_status hip_result(const char* fn, hipError_t e) {
    if (e == hipSuccess) return WQ_OK;
    return err(WQ_ERR_HIP, "%s: HIP error %d (%s)", fn, (int)e, hipGetErrorString(e));
}

#define WQ_TRY(expr)                      \
    do {                                  \
        const wq_status st_ = (expr);     \
        if (st_ != WQ_OK) return st_;     \
    } while (0)

}  // namespace host
}  // namespace wq
