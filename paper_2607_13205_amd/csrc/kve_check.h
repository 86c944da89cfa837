// Error reporting and argument checks shared by the C entry points.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdarg>
#include <cstdint>
#include <cstdio>

#include "../../include/kve.h"
#include "kve_internal.h"

namespace kve {
namespace check {

// The calling thread's last error message.  A plain character array, so that
// the library registers no thread-exit or process-exit destructor.
inline thread_local char g_error[512];

inline kve_status_t fail(kve_status_t st, const char* fmt, ...) {
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(g_error, sizeof(g_error), fmt, ap);
    va_end(ap);
    return st;
}

inline kve_status_t ok() {
    g_error[0] = '\0';
    return KVE_OK;
}

inline kve_status_t from_hip(hipError_t e, const char* what) {
    if (e == hipSuccess) return ok();
    return fail(KVE_ERR_HIP, "%s: HIP error %d (%s)", what, (int)e, hipGetErrorString(e));
}

inline bool aligned(const void* p) { return (reinterpret_cast<uintptr_t>(p) & (kve::kAlign - 1)) == 0; }

constexpr long long kMaxGrid = 2147483647LL;
// Largest token stride of a view, in bytes: the chunk loads keep the offsets
// of 64 rows in 32 bits.
constexpr long long kMaxTokenStrideBytes = 1LL << 25;

// The view of a [L, B, H, T, d] input: dense when st is null, else checked
// against the view rules of kve.h.
inline kve_status_t make_view(const char* fn, const char* name, const void* p, const kve_strides_t* st, int B, int H,
                       int T, int d, int es, kve::RowView* out) {
    if (st == nullptr) {
        *out = kve::dense_view(p, B, H, T, d, es);
        return KVE_OK;
    }
    const long long s[4] = {st->layer, st->batch, st->head, st->token};
    for (int i = 0; i < 4; ++i) {
        if (s[i] < 0) return fail(KVE_ERR_INVALID_ARG, "%s: %s has a negative stride", fn, name);
        if (s[i] > (1LL << 40)) return fail(KVE_ERR_INVALID_ARG, "%s: %s stride too large", fn, name);
        if ((s[i] * es) % 16 != 0)
            return fail(KVE_ERR_INVALID_ARG, "%s: %s stride %lld is not a multiple of 16 bytes", fn, name, s[i]);
    }
    if (s[3] * es > kMaxTokenStrideBytes)
        return fail(KVE_ERR_INVALID_ARG, "%s: %s token stride of %lld bytes exceeds %lld", fn, name, s[3] * es,
                    kMaxTokenStrideBytes);
    if ((reinterpret_cast<uintptr_t>(p) & 15u) != 0)
        return fail(KVE_ERR_INVALID_ARG, "%s: %s not 16-byte aligned", fn, name);
    *out = kve::RowView{static_cast<const char*>(p), s[0] * es, s[1] * es, s[2] * es, s[3] * es};
    return KVE_OK;
}

}  // namespace check
}  // namespace kve
