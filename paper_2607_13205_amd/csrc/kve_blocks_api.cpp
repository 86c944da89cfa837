// C ABI of the paged 8-bit cache: argument validation and dispatch to the HIP
// launchers.  Declarations and contracts: include/kve_blocks.h.
#include "../../include/kve_blocks.h"

#include <hip/hip_runtime.h>

#include <cmath>

#include "kve_check.h"
#include "kve_internal.h"
#include "kve_pages_check.h"

namespace {

using namespace kve::check;

bool valid_block(int page) { return valid_page(page) && page <= kve::kBlockMax; }

kve_status_t check_blocks(const char* fn, const kve_pages_t* c, kve::PagePool* out) {
    const kve_status_t st = check_pages(fn, c, true, out);
    if (st != KVE_OK) return st;
    if (!valid_block(c->page))
        return fail(KVE_ERR_INVALID_ARG, "%s: page=%d exceeds %d", fn, c->page, kve::kBlockMax);
    return KVE_OK;
}

// Checks of kve_blocks_append and kve_blocks_compact.
kve_status_t write_common(const char* fn, const void* k, const kve_strides_t* k_st, const void* v,
                          const kve_strides_t* v_st, kve_dtype_t dtype, int B, int N, const int32_t* idx,
                          const int32_t* count, int cap, const int32_t* start, const int32_t* seq,
                          const kve_pages_t* blocks, const kve_rotation_t* rotation, const void* q,
                          const kve_strides_t* q_st, int Hq, void* q_out, void* stream) {
    kve::PagePool p;
    kve_status_t st = check_blocks(fn, blocks, &p);
    if (st != KVE_OK || (st = check_dtype(fn, dtype)) != KVE_OK) return st;
    if ((st = check_rows(fn, blocks, B, cap, seq, false)) != KVE_OK) return st;
    if (N < 0 || N > (1 << 30)) return fail(KVE_ERR_INVALID_ARG, "%s: invalid N=%d", fn, N);
    if (start == nullptr) return fail(KVE_ERR_INVALID_ARG, "%s: null start", fn);
    kve::BlockRotation rot{};
    if (rotation != nullptr) {
        rot = kve::BlockRotation{rotation->cos, rotation->sin,      rotation->position,
                                 rotation->P,   rotation->r, rotation->pairs != 0};
        if (rot.r < 16 || rot.r > blocks->d || rot.r % 16 != 0)
            return fail(KVE_ERR_INVALID_ARG, "%s: %d rotated channels are not a multiple of 16 up to %d", fn, rot.r,
                        blocks->d);
        if (rot.P < 1) return fail(KVE_ERR_INVALID_ARG, "%s: a rotation of %d positions", fn, rot.P);
        if (N != 0 && (rot.cos == nullptr || rot.sin == nullptr || rot.position == nullptr))
            return fail(KVE_ERR_INVALID_ARG, "%s: null pointer in the rotation", fn);
        if (misaligned16(rot.cos) || misaligned16(rot.sin))
            return fail(KVE_ERR_INVALID_ARG, "%s: cos or sin not 16-byte aligned", fn);
    }
    // a call of no rows may lack its rows' tensors; what is given is checked as with rows
    if (cap != 0 && (k == nullptr || v == nullptr)) return fail(KVE_ERR_INVALID_ARG, "%s: null tensor pointer", fn);
    const int es = dtype == KVE_DTYPE_BF16 ? 2 : 4;
    kve::RowView kv{}, vv{}, qv{};
    if (k != nullptr && (st = make_view(fn, "k", k, k_st, B, blocks->Hkv, N, blocks->d, es, &kv)) != KVE_OK) return st;
    if (v != nullptr && (st = make_view(fn, "v", v, v_st, B, blocks->Hkv, N, blocks->d, es, &vv)) != KVE_OK) return st;
    if (misaligned16(k) || misaligned16(v)) return fail(KVE_ERR_INVALID_ARG, "%s: k or v not 16-byte aligned", fn);
    const long long touched = kve::blocks_touched(cap, blocks->page);
    double groups = 2.0 * blocks->L * B * blocks->Hkv * touched;
    if (q != nullptr || q_out != nullptr) {
        if (q == nullptr || q_out == nullptr || rotation == nullptr)
            return fail(KVE_ERR_INVALID_ARG, "%s: queries need an output and a rotation", fn);
        if (q == q_out) return fail(KVE_ERR_INVALID_ARG, "%s: q_out is q", fn);
        if (Hq < 1) return fail(KVE_ERR_INVALID_ARG, "%s: Hq=%d < 1", fn, Hq);
        if ((st = make_view(fn, "q", q, q_st, B, Hq, N, blocks->d, es, &qv)) != KVE_OK) return st;
        if (misaligned16(q) || misaligned16(q_out))
            return fail(KVE_ERR_INVALID_ARG, "%s: q or q_out not 16-byte aligned", fn);
        const double rows = (double)blocks->L * B * Hq * cap;
        if (rows > (double)(1 << 30)) return fail(KVE_ERR_UNSUPPORTED, "%s: shape too large", fn);
        groups += (double)blocks->L * ((long long)B * cap / 32 + 1) * (Hq / kve::kBlocksQueryHeads + 1);
    }
    if (groups > (double)kMaxGroups) return fail(KVE_ERR_UNSUPPORTED, "%s: shape too large", fn);
    if (cap == 0) return ok();
    return from_hip(kve::launch_blocks_write(kv, vv, qv, q_out, Hq, (int)dtype, blocks->d, B, N, idx, count, cap, start,
                                             seq, rot, p, static_cast<hipStream_t>(stream)),
                    fn);
}

// Checks of the calls that read `cap` rows of each segment.
kve_status_t read_common(const char* fn, const kve_pages_t* blocks, kve_dtype_t dtype, int B, int cap,
                         const int32_t* seq, const void* a, const void* b, kve::PagePool* p) {
    kve_status_t st = check_blocks(fn, blocks, p);
    if (st != KVE_OK || (st = check_dtype(fn, dtype)) != KVE_OK) return st;
    if ((st = check_rows(fn, blocks, B, cap, seq, false)) != KVE_OK) return st;
    if (cap != 0 && a == nullptr && b == nullptr) return fail(KVE_ERR_INVALID_ARG, "%s: null outputs", fn);
    if (misaligned16(a) || misaligned16(b)) return fail(KVE_ERR_INVALID_ARG, "%s: output not 16-byte aligned", fn);
    // 16 rows to a workgroup and a 32-bit number for each
    if ((double)blocks->L * B * blocks->Hkv * cap > 16.0 * (double)kMaxGroups)
        return fail(KVE_ERR_UNSUPPORTED, "%s: shape too large", fn);
    return KVE_OK;
}

// Checks of the calls on queries.
kve_status_t check_queries(const char* fn, const void* q, kve_dtype_t dtype, const kve_pages_t* blocks, int B, int Hq,
                           int T, int max_tokens, const int32_t* seq, kve::PagePool* p) {
    kve_status_t st = check_blocks(fn, blocks, p);
    if (st != KVE_OK || (st = check_dtype(fn, dtype)) != KVE_OK) return st;
    if ((st = check_rows(fn, blocks, B, 0, seq, false)) != KVE_OK) return st;
    if (q == nullptr) return fail(KVE_ERR_INVALID_ARG, "%s: null tensor pointer", fn);
    if (misaligned16(q)) return fail(KVE_ERR_INVALID_ARG, "%s: q not 16-byte aligned", fn);
    if (T < 1) return fail(KVE_ERR_INVALID_ARG, "%s: T=%d < 1", fn, T);
    if (Hq <= 0 || Hq % blocks->Hkv != 0)
        return fail(KVE_ERR_INVALID_ARG, "%s: Hq=%d is not a positive multiple of Hkv=%d", fn, Hq, blocks->Hkv);
    if (max_tokens < 1 || max_tokens > (long long)blocks->M * blocks->page)
        return fail(KVE_ERR_INVALID_ARG, "%s: max_tokens=%d outside [1, M * page]", fn, max_tokens);
    if ((double)blocks->L * B * Hq * T > (double)kMaxGroups)
        return fail(KVE_ERR_UNSUPPORTED, "%s: shape too large", fn);
    return KVE_OK;
}

kve_status_t check_workspace(const char* fn, const void* workspace, size_t have, size_t need) {
    if (have < need || workspace == nullptr)
        return fail(KVE_ERR_WORKSPACE, "%s: workspace of %zu bytes < %zu needed", fn, have, need);
    if (!aligned(workspace)) return fail(KVE_ERR_INVALID_ARG, "%s: workspace not 256-byte aligned", fn);
    return KVE_OK;
}

}  // namespace

extern "C" {

size_t kve_block_bytes(int page, int d) {
    if (!valid_block(page) || (d != 64 && d != 128)) return 0;
    return kve::block_bytes(page, d);
}

kve_status_t kve_blocks_append(const void* k, const kve_strides_t* k_strides, const void* v,
                               const kve_strides_t* v_strides, kve_dtype_t dtype, int B, int T, const int32_t* n_new,
                               const int32_t* start, const int32_t* seq, const kve_pages_t* blocks,
                               const kve_rotation_t* rotation, const void* q, const kve_strides_t* q_strides, int Hq,
                               void* q_out, void* stream) {
    return write_common("kve_blocks_append", k, k_strides, v, v_strides, dtype, B, T, nullptr, n_new, T, start, seq,
                        blocks, rotation, q, q_strides, Hq, q_out, stream);
}

kve_status_t kve_blocks_compact(const void* k, const kve_strides_t* k_strides, const void* v,
                                const kve_strides_t* v_strides, kve_dtype_t dtype, int B, int N, const int32_t* idx,
                                const int32_t* count, int k_cap, const int32_t* start, const int32_t* seq,
                                const kve_pages_t* blocks, void* stream) {
    const char* fn = "kve_blocks_compact";
    if (count == nullptr || (idx == nullptr && k_cap != 0))
        return fail(KVE_ERR_INVALID_ARG, "%s: null idx or count", fn);
    if (N < 1) return fail(KVE_ERR_INVALID_ARG, "%s: N must be positive", fn);
    return write_common(fn, k, k_strides, v, v_strides, dtype, B, N, idx, count, k_cap, start, seq, blocks, nullptr,
                        nullptr, nullptr, 0, nullptr, stream);
}

kve_status_t kve_blocks_read(const kve_pages_t* blocks, kve_dtype_t dtype, int B, int T, const int32_t* seq,
                             const int32_t* start, const int32_t* count, void* k_out, void* v_out, void* stream) {
    const char* fn = "kve_blocks_read";
    kve::PagePool p;
    const kve_status_t st = read_common(fn, blocks, dtype, B, T, seq, k_out, v_out, &p);
    if (st != KVE_OK) return st;
    if (T == 0) return ok();
    return from_hip(kve::launch_blocks_read(p, (int)dtype, blocks->d, B, T, seq, start, count, k_out, v_out,
                                            static_cast<hipStream_t>(stream)),
                    fn);
}

kve_status_t kve_blocks_bounds(const kve_pages_t* blocks, kve_dtype_t dtype, int B, int n, const int32_t* seq,
                               const int32_t* first, void* lo_out, void* hi_out, void* stream) {
    const char* fn = "kve_blocks_bounds";
    kve::PagePool p;
    const kve_status_t st = read_common(fn, blocks, dtype, B, n, seq, lo_out, hi_out, &p);
    if (st != KVE_OK) return st;
    if (n == 0) return ok();
    return from_hip(kve::launch_blocks_bounds(p, (int)dtype, blocks->d, B, n, seq, first, lo_out, hi_out,
                                              static_cast<hipStream_t>(stream)),
                    fn);
}

size_t kve_blocks_top_workspace_size(int L, int B, int Hkv, int T, int max_tokens, int page) {
    if (L <= 0 || B <= 0 || Hkv <= 0 || T <= 0 || max_tokens <= 0 || max_tokens > (1 << 30) || !valid_block(page))
        return 0;
    if ((double)L * B * Hkv * T > (double)kMaxGroups) return 0;
    return kve::top_size(L, B, Hkv, T, max_tokens, page);
}

kve_status_t kve_blocks_top(const void* q, kve_dtype_t dtype, const kve_pages_t* blocks, int B, int Hq, int T,
                            int max_tokens, const int32_t* start, const int32_t* seq, int k, int first, int last,
                            int32_t* top, void* workspace, size_t workspace_bytes, void* stream) {
    const char* fn = "kve_blocks_top";
    kve::PagePool p;
    kve_status_t st = check_queries(fn, q, dtype, blocks, B, Hq, T, max_tokens, seq, &p);
    if (st != KVE_OK) return st;
    if (top == nullptr) return fail(KVE_ERR_INVALID_ARG, "%s: null output", fn);
    if (first < 0 || last < 0 || k < 1 || (long long)first + last > k)
        return fail(KVE_ERR_INVALID_ARG, "%s: k=%d does not hold first=%d and last=%d blocks", fn, k, first, last);
    const long long chunks = kve::top_blocks(max_tokens, blocks->page) / 64 + 1;
    if ((double)blocks->L * B * blocks->Hkv * T * chunks > (double)kMaxGroups || k > (1 << 25))
        return fail(KVE_ERR_UNSUPPORTED, "%s: shape too large", fn);
    const size_t need = kve::top_size(blocks->L, B, blocks->Hkv, T, max_tokens, blocks->page);
    if ((st = check_workspace(fn, workspace, workspace_bytes, need)) != KVE_OK) return st;
    const kve::BlockView view{seq, start, B, T, max_tokens};
    return from_hip(kve::launch_blocks_top(q, (int)dtype, p, blocks->d, view, Hq, k, first, last, top, workspace,
                                           static_cast<hipStream_t>(stream)),
                    fn);
}

size_t kve_decode_blocks_workspace_size(int L, int B, int Hq, int Hkv, int T, int d) {
    if (L <= 0 || B <= 0 || Hq <= 0 || Hkv <= 0 || T <= 0 || Hq % Hkv != 0) return 0;
    if ((d != 64 && d != 128) || (double)L * B * Hq * T > (double)kMaxGroups) return 0;
    return kve::decode_blocks_size(L, B, Hq, Hkv, T, d);
}

kve_status_t kve_decode_blocks(const void* q, kve_dtype_t dtype, const kve_pages_t* blocks, int B, int Hq, int T,
                               int max_tokens, const int32_t* start, const int32_t* seq, const int32_t* top, int k,
                               float scale, float* out, void* workspace, size_t workspace_bytes, void* stream) {
    const char* fn = "kve_decode_blocks";
    kve::PagePool p;
    kve_status_t st = check_queries(fn, q, dtype, blocks, B, Hq, T, max_tokens, seq, &p);
    if (st != KVE_OK) return st;
    if (out == nullptr) return fail(KVE_ERR_INVALID_ARG, "%s: null output", fn);
    if (Hq / blocks->Hkv > kve::kPagesMaxGroup)
        return fail(KVE_ERR_UNSUPPORTED, "%s: Hq/Hkv=%d exceeds %d", fn, Hq / blocks->Hkv, kve::kPagesMaxGroup);
    if ((top == nullptr) != (k == 0) || k < 0)
        return fail(KVE_ERR_INVALID_ARG, "%s: k=%d blocks %s a list", fn, k, top != nullptr ? "with" : "without");
    if (!(std::isfinite(scale) && scale >= 0.0f))
        return fail(KVE_ERR_INVALID_ARG, "%s: scale must be finite and >= 0", fn);
    if ((long long)k * blocks->page > (1LL << 30)) return fail(KVE_ERR_UNSUPPORTED, "%s: k=%d too large", fn, k);
    const long long tokens = top != nullptr ? (long long)k * blocks->page : max_tokens;
    const kve::BlocksPlan plan =
        kve::decode_blocks_plan(blocks->L, B, Hq, blocks->Hkv, T, tokens, top != nullptr, blocks->d);
    if ((long long)plan.pairs * plan.groups > kMaxGroups || (long long)plan.pairs * plan.entries * plan.R > kMaxGroups)
        return fail(KVE_ERR_UNSUPPORTED, "%s: shape too large", fn);
    if ((st = check_workspace(fn, workspace, workspace_bytes, plan.total)) != KVE_OK) return st;
    if (scale == 0.0f) scale = 1.0f / std::sqrt((float)blocks->d);
    const kve::BlockView view{seq, start, B, T, max_tokens};
    return from_hip(kve::launch_decode_blocks(q, (int)dtype, p, blocks->d, view, Hq, top, k, scale, out, workspace,
                                              static_cast<hipStream_t>(stream)),
                    fn);
}

}  // extern "C"
