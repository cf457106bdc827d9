// What the C entries of the language operators share: failures, overlaps of tensors, strides.
#pragma once
#include <cuda_runtime.h>

#include <algorithm>
#include <cstdarg>
#include <cstdint>
#include <cstdio>
#include <limits>

#include "../../include/mafat.h"

mafat_status mafat_internal_fail(mafat_status s, const char* msg);
void mafat_internal_clear_error();

namespace mafat_lm {

// Nothing that throws passes a C entry: messages are made on the stack, and keeping one may fail.
inline mafat_status fail(mafat_status s, const char* format, ...) {
    char msg[256];
    va_list args;
    va_start(args, format);
    vsnprintf(msg, sizeof(msg), format, args);
    va_end(args);
    try {
        return mafat_internal_fail(s, msg);
    } catch (...) {
        return s;
    }
}
inline mafat_status cuda_fail(cudaError_t e, const char* what) {
    return fail(e == cudaErrorMemoryAllocation ? MAFAT_ENOMEM : MAFAT_ECUDA, "%s: %s", what, cudaGetErrorString(e));
}

// What was copied to the device from pageable memory, or set there, may still be on its way when the call returns, and streams that
// the legacy stream does not hold up would not wait for it: a plan's maker waits itself.
inline cudaError_t transfers_done() { return cudaStreamSynchronize(nullptr); }

constexpr int64_t kMaxI32 = std::numeric_limits<int32_t>::max();

inline bool aligned(const void* p, uintptr_t n = 16) { return ((uintptr_t)p & (n - 1)) == 0; }

// Bytes from a tensor's first element to past its last one, for sizes and strides in elements.
inline int64_t extent(const int64_t n[3], const int64_t st[3], int64_t inner, int64_t esz) {
    int64_t last = inner;
    for (int i = 0; i < 3; ++i) last += (n[i] - 1) * st[i];
    return last * esz;
}

inline bool overlap(const void* a, int64_t an, const void* b, int64_t bn) {
    const char *x = (const char*)a, *y = (const char*)b;
    return x && y && an > 0 && bn > 0 && x < y + bn && y < x + an;
}

// Strides given by the caller (all 0: packed), in elements.  They have to keep every 16-byte
// vector of channels aligned, and what they span with the sizes inside 62 bits of bytes, so that no offset passes 64.
// Where there is nothing to step to (one element of a dimension, or none at all) any stride is taken, and a valid one kept.
inline mafat_status take_strides(const char* what, const int64_t given[3], const int64_t n[3], int64_t dim, int64_t esz,
                          int64_t out[3]) {
    const int64_t most = ((int64_t)1 << 40) / esz;
    const bool packed = given[0] == 0 && given[1] == 0 && given[2] == 0, empty = n[0] == 0 || n[1] == 0 || n[2] == 0;
    __int128 span = dim, next = dim;  // of the packed: the stride of a dimension by those inside it
    for (int i = 2; i >= 0; --i) {
        out[i] = dim;
        if (n[i] <= 1 || empty) continue;
        const __int128 st = packed ? next : (__int128)given[i];
        if (st < dim) return fail(MAFAT_EINVAL, "%s: a stride is smaller than a head's channels", what);
        if (st * esz % 16 != 0) return fail(MAFAT_EINVAL, "%s: strides must be multiples of 16 bytes", what);
        if (st >= most) return fail(MAFAT_EUNSUPPORTED, "%s: strides must be below 2^40 bytes", what);
        out[i] = (int64_t)st;
        span += (n[i] - 1) * st;
        next *= n[i];
    }
    if (span * esz > (__int128)1 << 62) return fail(MAFAT_EUNSUPPORTED, "%s: the tensor spans more than 2^62 bytes", what);
    return MAFAT_OK;
}

// Two elements of a written tensor must not share a place: sorted by stride, each stride has to
// pass what the dimensions inside it span.
inline bool places_distinct(const int64_t n[3], const int64_t st[3], int64_t dim) {
    int at[3] = {0, 1, 2};
    std::sort(at, at + 3, [&](int a, int b) { return st[a] < st[b]; });
    int64_t span = dim;
    for (int i : at) {
        if (n[i] == 1) continue;
        if (st[i] < span) return false;
        span = (n[i] - 1) * st[i] + span;
    }
    return true;
}

}  // namespace mafat_lm
