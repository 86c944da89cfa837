// C ABI of the paged 4-bit cache: argument validation and dispatch to the HIP
// launchers.  Declarations and contracts: include/kve_pages.h.
#include "../../include/kve_pages.h"

#include <hip/hip_runtime.h>

#include <cmath>

#include "kve_check.h"
#include "kve_internal.h"

namespace {

using namespace kve::check;

// Workgroups of 256 threads in one launch: the dispatch counts threads in 32 bits.
constexpr long long kMaxGroups = (1LL << 24) - 1;

bool misaligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) != 0; }

bool valid_page(int page) { return page >= kve::kPageMin && page <= kve::kPageMax && (page & (page - 1)) == 0; }

// Checks the cache and translates it for the kernels.  rows: the call touches
// the pool.
kve_status_t check_pages(const char* fn, const kve_pages_t* c, bool rows, kve::PagePool* out) {
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

kve_status_t check_entries(const char* fn, const kve_pages_t* c, const int32_t* seq, int n) {
    if (n < 1) return fail(KVE_ERR_INVALID_ARG, "%s: n=%d < 1", fn, n);
    if (seq == nullptr && n > c->S)
        return fail(KVE_ERR_INVALID_ARG, "%s: %d entries without slots, the cache has %d", fn, n, c->S);
    return KVE_OK;
}

kve_status_t check_bookkeeping(const char* fn, const kve_pages_t* c, int n, const void* workspace,
                               size_t workspace_bytes) {
    if (n > kve::kPagesMaxEntries)
        return fail(KVE_ERR_UNSUPPORTED, "%s: n=%d exceeds %d", fn, n, kve::kPagesMaxEntries);
    const size_t need = kve::pages_workspace(c->n_pages, n);
    if (workspace_bytes < need || workspace == nullptr)
        return fail(KVE_ERR_WORKSPACE, "%s: workspace of %zu bytes < %zu needed", fn, workspace_bytes, need);
    if (!aligned(workspace)) return fail(KVE_ERR_INVALID_ARG, "%s: workspace not 256-byte aligned", fn);
    return KVE_OK;
}

// B samples of `cap` rows each in a call on the cache's rows.
kve_status_t check_rows(const char* fn, const kve_pages_t* c, int B, int cap, const int32_t* seq, bool need_seq) {
    if (B <= 0 || cap < 0) return fail(KVE_ERR_INVALID_ARG, "%s: invalid sizes (B=%d rows=%d)", fn, B, cap);
    if (need_seq && seq == nullptr) return fail(KVE_ERR_INVALID_ARG, "%s: null slots", fn);
    if (seq == nullptr && B > c->S)
        return fail(KVE_ERR_INVALID_ARG, "%s: %d samples without slots, the cache has %d", fn, B, c->S);
    const double groups = (double)c->L * B * c->Hkv * (cap / kve::kPagesRows + 1);
    if (cap > (1 << 30) || groups > (double)kMaxGroups) return fail(KVE_ERR_UNSUPPORTED, "%s: shape too large", fn);
    return KVE_OK;
}

kve_status_t check_dtype(const char* fn, kve_dtype_t dtype) {
    if (dtype != KVE_DTYPE_BF16 && dtype != KVE_DTYPE_F32)
        return fail(KVE_ERR_UNSUPPORTED, "%s: unknown dtype %d", fn, (int)dtype);
    return KVE_OK;
}

// Checks of kve_pages_append and kve_pages_compact.
kve_status_t pack_common(const char* fn, const void* k, const kve_strides_t* k_st, const void* v,
                         const kve_strides_t* v_st, kve_dtype_t dtype, int B, int N, const int32_t* idx,
                         const int32_t* count, int cap, const int32_t* start, const int32_t* seq,
                         const kve_pages_t* pages, void* stream) {
    kve::PagePool p;
    kve_status_t st = check_pages(fn, pages, true, &p);
    if (st != KVE_OK || (st = check_dtype(fn, dtype)) != KVE_OK) return st;
    if ((st = check_rows(fn, pages, B, cap, seq, false)) != KVE_OK) return st;
    if (N < 0 || N > (1 << 30)) return fail(KVE_ERR_INVALID_ARG, "%s: invalid N=%d", fn, N);
    if (start == nullptr) return fail(KVE_ERR_INVALID_ARG, "%s: null start", fn);
    if (N == 0 || (cap == 0 && (k == nullptr || v == nullptr))) return ok();
    if (k == nullptr || v == nullptr) return fail(KVE_ERR_INVALID_ARG, "%s: null tensor pointer", fn);
    const int es = dtype == KVE_DTYPE_BF16 ? 2 : 4;
    kve::RowView kv, vv;
    if ((st = make_view(fn, "k", k, k_st, B, pages->Hkv, N, pages->d, es, &kv)) != KVE_OK) return st;
    if ((st = make_view(fn, "v", v, v_st, B, pages->Hkv, N, pages->d, es, &vv)) != KVE_OK) return st;
    if (misaligned16(k) || misaligned16(v)) return fail(KVE_ERR_INVALID_ARG, "%s: k or v not 16-byte aligned", fn);
    if (cap == 0) return ok();  // nothing to do, but what would be refused with rows has been
    return from_hip(kve::launch_pages_pack(kv, vv, (int)dtype, pages->d, B, N, idx, count, cap, start, seq, p,
                                           static_cast<hipStream_t>(stream)),
                    fn);
}

}  // namespace

extern "C" {

size_t kve_page_bytes(int page, int d) {
    if (!valid_page(page) || (d != 64 && d != 128)) return 0;
    return kve::page_block_bytes(page, d);
}

size_t kve_pages_workspace_size(int n_pages, int S, int n) {
    if (n_pages <= 0 || n_pages > (1 << 30) || S <= 0 || n < 1 || n > kve::kPagesMaxEntries) return 0;
    return kve::pages_workspace(n_pages, n);
}

kve_status_t kve_pages_extend(const kve_pages_t* pages, const int32_t* seq, const int32_t* add, int n,
                              int32_t* start, int32_t* missing, void* workspace, size_t workspace_bytes,
                              void* stream) {
    const char* fn = "kve_pages_extend";
    kve::PagePool p;
    kve_status_t st = check_pages(fn, pages, false, &p);
    if (st != KVE_OK || (st = check_entries(fn, pages, seq, n)) != KVE_OK) return st;
    if (add == nullptr || start == nullptr || missing == nullptr)
        return fail(KVE_ERR_INVALID_ARG, "%s: null pointer", fn);
    if ((st = check_bookkeeping(fn, pages, n, workspace, workspace_bytes)) != KVE_OK) return st;
    return from_hip(kve::launch_pages_extend(p, seq, add, n, start, missing, workspace,
                                             static_cast<hipStream_t>(stream)),
                    fn);
}

kve_status_t kve_pages_fork(const kve_pages_t* pages, const int32_t* src, const int32_t* dst, int n, int32_t* done,
                            int32_t* missing, void* workspace, size_t workspace_bytes, void* stream) {
    const char* fn = "kve_pages_fork";
    kve::PagePool p;
    kve_status_t st = check_pages(fn, pages, true, &p);
    if (st != KVE_OK) return st;
    if (src == nullptr || dst == nullptr || done == nullptr || missing == nullptr)
        return fail(KVE_ERR_INVALID_ARG, "%s: null pointer", fn);
    if ((st = check_entries(fn, pages, src, n)) != KVE_OK) return st;
    if ((st = check_bookkeeping(fn, pages, n, workspace, workspace_bytes)) != KVE_OK) return st;
    const double parts = 1.0 + (double)pages->L * pages->Hkv *
                                   (kve::page_block_bytes(pages->page, pages->d) / kve::kPagesCopyBytes + 1);
    if (n * parts > (double)kMaxGroups) return fail(KVE_ERR_UNSUPPORTED, "%s: shape too large", fn);
    return from_hip(kve::launch_pages_fork(p, pages->d, src, dst, n, done, missing, workspace,
                                           static_cast<hipStream_t>(stream)),
                    fn);
}

kve_status_t kve_pages_free(const kve_pages_t* pages, const int32_t* seq, int n, void* stream) {
    const char* fn = "kve_pages_free";
    kve::PagePool p;
    kve_status_t st = check_pages(fn, pages, false, &p);
    if (st != KVE_OK || (st = check_entries(fn, pages, seq, n)) != KVE_OK) return st;
    if (n > kMaxGroups) return fail(KVE_ERR_UNSUPPORTED, "%s: n=%d too large", fn, n);
    return from_hip(kve::launch_pages_free(p, seq, n, static_cast<hipStream_t>(stream)), fn);
}

kve_status_t kve_pages_append(const void* k, const kve_strides_t* k_strides, const void* v,
                              const kve_strides_t* v_strides, kve_dtype_t dtype, int B, int T, const int32_t* n_new,
                              const int32_t* start, const int32_t* seq, const kve_pages_t* pages, void* stream) {
    return pack_common("kve_pages_append", k, k_strides, v, v_strides, dtype, B, T, nullptr, n_new, T, start, seq,
                       pages, stream);
}

kve_status_t kve_pages_compact(const void* k, const kve_strides_t* k_strides, const void* v,
                               const kve_strides_t* v_strides, kve_dtype_t dtype, int B, int N, const int32_t* idx,
                               const int32_t* count, int k_cap, const int32_t* start, const int32_t* seq,
                               const kve_pages_t* pages, void* stream) {
    const char* fn = "kve_pages_compact";
    if (count == nullptr || (idx == nullptr && k_cap != 0))
        return fail(KVE_ERR_INVALID_ARG, "%s: null idx or count", fn);
    if (N < 1) return fail(KVE_ERR_INVALID_ARG, "%s: N must be positive", fn);
    return pack_common(fn, k, k_strides, v, v_strides, dtype, B, N, idx, count, k_cap, start, seq, pages, stream);
}

kve_status_t kve_pages_select(const kve_pages_t* pages, int B, const int32_t* src, const int32_t* idx,
                              const int32_t* count, int k_cap, const int32_t* dst, const int32_t* start,
                              void* stream) {
    const char* fn = "kve_pages_select";
    kve::PagePool p;
    kve_status_t st = check_pages(fn, pages, true, &p);
    if (st != KVE_OK) return st;
    if (src == nullptr || dst == nullptr || count == nullptr || start == nullptr || (idx == nullptr && k_cap != 0))
        return fail(KVE_ERR_INVALID_ARG, "%s: null pointer", fn);
    if ((st = check_rows(fn, pages, B, k_cap, src, true)) != KVE_OK) return st;
    if (k_cap == 0) return ok();
    return from_hip(kve::launch_pages_select(p, pages->d, B, src, idx, count, k_cap, dst, start,
                                             static_cast<hipStream_t>(stream)),
                    fn);
}

kve_status_t kve_pages_read(const kve_pages_t* pages, kve_dtype_t dtype, int B, int T, const int32_t* seq,
                            const int32_t* start, const int32_t* count, void* k_out, void* v_out, void* stream) {
    const char* fn = "kve_pages_read";
    kve::PagePool p;
    kve_status_t st = check_pages(fn, pages, true, &p);
    if (st != KVE_OK || (st = check_dtype(fn, dtype)) != KVE_OK) return st;
    if ((st = check_rows(fn, pages, B, T, seq, false)) != KVE_OK) return st;
    if (T == 0) return ok();
    if (k_out == nullptr && v_out == nullptr) return fail(KVE_ERR_INVALID_ARG, "%s: null outputs", fn);
    if (misaligned16(k_out) || misaligned16(v_out))
        return fail(KVE_ERR_INVALID_ARG, "%s: output not 16-byte aligned", fn);
    return from_hip(kve::launch_pages_read(p, (int)dtype, pages->d, B, T, seq, start, count, k_out, v_out,
                                           static_cast<hipStream_t>(stream)),
                    fn);
}

size_t kve_decode_pages_workspace_size(int L, int B, int Hq, int Hkv, int max_tokens, int d) {
    if (L <= 0 || B <= 0 || Hq <= 0 || Hkv <= 0 || max_tokens <= 0 || Hq % Hkv != 0) return 0;
    if ((d != 64 && d != 128) || (double)L * B * Hq > (double)kMaxGroups || max_tokens > (1 << 30)) return 0;
    return kve::decode_pages_size(L, B, Hq, Hkv, max_tokens, d);
}

kve_status_t kve_decode_pages(const void* q, kve_dtype_t dtype, const kve_pages_t* pages, int B, int Hq,
                              int max_tokens, const int32_t* seq, float scale, float* out, void* workspace,
                              size_t workspace_bytes, void* stream) {
    const char* fn = "kve_decode_pages";
    kve::PagePool p;
    kve_status_t st = check_pages(fn, pages, true, &p);
    if (st != KVE_OK || (st = check_dtype(fn, dtype)) != KVE_OK) return st;
    if ((st = check_rows(fn, pages, B, 0, seq, false)) != KVE_OK) return st;
    if (q == nullptr || out == nullptr) return fail(KVE_ERR_INVALID_ARG, "%s: null tensor pointer", fn);
    if (misaligned16(q)) return fail(KVE_ERR_INVALID_ARG, "%s: q not 16-byte aligned", fn);
    if (Hq <= 0 || Hq % pages->Hkv != 0)
        return fail(KVE_ERR_INVALID_ARG, "%s: Hq=%d is not a positive multiple of Hkv=%d", fn, Hq, pages->Hkv);
    if (Hq / pages->Hkv > kve::kPagesMaxGroup)
        return fail(KVE_ERR_UNSUPPORTED, "%s: Hq/Hkv=%d exceeds %d", fn, Hq / pages->Hkv, kve::kPagesMaxGroup);
    if (max_tokens < 1 || max_tokens > (long long)pages->M * pages->page)
        return fail(KVE_ERR_INVALID_ARG, "%s: max_tokens=%d outside [1, M * page]", fn, max_tokens);
    if (!(std::isfinite(scale) && scale >= 0.0f))
        return fail(KVE_ERR_INVALID_ARG, "%s: scale must be finite and >= 0", fn);
    if ((double)pages->L * B * Hq > (double)kMaxGroups) return fail(KVE_ERR_UNSUPPORTED, "%s: shape too large", fn);
    const kve::PagesPlan plan = kve::decode_pages_plan(pages->L, B, Hq, pages->Hkv, max_tokens, pages->d);
    if ((long long)plan.pairs * plan.groups > kMaxGroups)
        return fail(KVE_ERR_UNSUPPORTED, "%s: shape too large", fn);
    if (workspace_bytes < plan.total || workspace == nullptr)
        return fail(KVE_ERR_WORKSPACE, "%s: workspace of %zu bytes < %zu needed", fn, workspace_bytes, plan.total);
    if (!aligned(workspace)) return fail(KVE_ERR_INVALID_ARG, "%s: workspace not 256-byte aligned", fn);
    if (scale == 0.0f) scale = 1.0f / std::sqrt((float)pages->d);
    return from_hip(kve::launch_decode_pages(q, (int)dtype, p, pages->d, B, Hq, max_tokens, seq, scale, out,
                                             workspace, static_cast<hipStream_t>(stream)),
                    fn);
}

}  // extern "C"
