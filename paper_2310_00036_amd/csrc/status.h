// What the C entry points share: the calling thread's error message and argument checks.
#pragma once

#include <stddef.h>
#include <stdint.h>

#include "../../include/cleanba_learner.h"

namespace cb {

__attribute__((format(printf, 2, 3))) impala_status_t fail(impala_status_t code, const char* fmt, ...);
impala_status_t ok();
impala_status_t hip_status(hipError_t e, const char* where);

#define CHECK_PTR(p) \
    if (!(p)) return fail(IMPALA_EINVAL, "%s: argument '%s' is NULL", __func__, #p)

inline bool valid_prec(int p) { return p == IMPALA_PREC_BF16 || p == IMPALA_PREC_FP32; }

// Whether the byte ranges [a, a + an) and [b, b + bn) share a byte.
inline bool ranges_overlap(const void* a, size_t an, const void* b, size_t bn) {
    const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
    return an > 0 && bn > 0 && x < y + bn && y < x + an;
}

// Whether the byte ranges [a, a + bytes) and [b, b + bytes) overlap without being the same.
inline bool partial_overlap(const void* a, const void* b, size_t bytes) {
    return a != b && ranges_overlap(a, bytes, b, bytes);
}

}  // namespace cb
