// Argument checks shared by the C entry points of the paged caches.
#pragma once

#include "../../include/kve_pages.h"
#include "kve_check.h"

namespace kve {
namespace check {

// Workgroups of 256 threads in one launch: the dispatch counts threads in 32 bits.
constexpr long long kMaxGroups = (1LL << 24) - 1;

inline bool misaligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) != 0; }

inline bool valid_page(int page) { return page >= kve::kPageMin && page <= kve::kPageMax && (page & (page - 1)) == 0; }

// Checks the cache and translates it for the kernels.  rows: the call touches
// the pool.
inline kve_status_t check_pages(const char* fn, const kve_pages_t* c, bool rows, kve::PagePool* out) {
    if (c == nullptr) return fail(KVE_ERR_INVALID_ARG, "%s: null pages", fn);
    if (c->refs == nullptr || c->table == nullptr || c->held == nullptr || c->length == nullptr ||
        (rows && c->pool == nullptr))
        return fail(KVE_ERR_INVALID_ARG, "%s: null buffer in pages", fn);
    if (c->L <= 0 || c->n_pages <= 0 || c->Hkv <= 0 || c->S <= 0 || c->M <= 0)
        return fail(KVE_ERR_INVALID_ARG, "%s: sizes must be positive (L=%d n_pages=%d Hkv=%d S=%d M=%d)", fn, c->L,
                    c->n_pages, c->Hkv, c->S, c->M);
    if (!valid_page(c->page))
        return fail(KVE_ERR_INVALID_ARG, "%s: page=%d is not a power of two in [%d, %d]", fn, c->page, kve::kPageMin,
                    kve::kPageMax);
    if (c->d != 64 && c->d != 128)
        return fail(KVE_ERR_UNSUPPORTED, "%s: head_dim %d not built (64 or 128)", fn, c->d);
    if (rows && misaligned16(c->pool)) return fail(KVE_ERR_INVALID_ARG, "%s: pool not 16-byte aligned", fn);
    if ((long long)c->M * c->page > (1LL << 30) || c->n_pages > (1 << 30) || (long long)c->S * c->M > kMaxGrid ||
        c->L > (1 << 20) || c->Hkv > (1 << 20))
        return fail(KVE_ERR_UNSUPPORTED, "%s: cache too large", fn);
    int shift = 0;
    while ((1 << shift) < c->page) ++shift;
    *out = kve::PagePool{static_cast<char*>(c->pool), c->refs, c->table, c->held, c->length, c->L,
                         c->n_pages,                  c->Hkv,  c->S,     c->M,    shift};
    return KVE_OK;
}

inline kve_status_t check_entries(const char* fn, const kve_pages_t* c, const int32_t* seq, int n) {
    if (n < 1) return fail(KVE_ERR_INVALID_ARG, "%s: n=%d < 1", fn, n);
    if (seq == nullptr && n > c->S)
        return fail(KVE_ERR_INVALID_ARG, "%s: %d entries without slots, the cache has %d", fn, n, c->S);
    return KVE_OK;
}

// B samples of `cap` rows each in a call on the cache's rows.
inline kve_status_t check_rows(const char* fn, const kve_pages_t* c, int B, int cap, const int32_t* seq,
                               bool need_seq) {
    if (B <= 0 || cap < 0) return fail(KVE_ERR_INVALID_ARG, "%s: invalid sizes (B=%d rows=%d)", fn, B, cap);
    if (need_seq && seq == nullptr) return fail(KVE_ERR_INVALID_ARG, "%s: null slots", fn);
    if (seq == nullptr && B > c->S)
        return fail(KVE_ERR_INVALID_ARG, "%s: %d samples without slots, the cache has %d", fn, B, c->S);
    const double groups = (double)c->L * B * c->Hkv * (cap / kve::kPagesRows + 1);
    if (cap > (1 << 30) || groups > (double)kMaxGroups) return fail(KVE_ERR_UNSUPPORTED, "%s: shape too large", fn);
    return KVE_OK;
}

inline kve_status_t check_dtype(const char* fn, kve_dtype_t dtype) {
    if (dtype != KVE_DTYPE_BF16 && dtype != KVE_DTYPE_F32)
        return fail(KVE_ERR_UNSUPPORTED, "%s: unknown dtype %d", fn, (int)dtype);
    return KVE_OK;
}

}  // namespace check
}  // namespace kve
