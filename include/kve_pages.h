/*
 * kve_pages.h -- C ABI of the paged 4-bit cache (libkve.so)
 *
 * What an eviction step keeps can be held in pages of four-bit rows: the kept
 * rows are packed into pages, decode attends to them through a page table, new
 * tokens are appended, a sequence is forked into continuations that share its
 * full pages, its rows are thinned out again by a second eviction, and its
 * pages return to the pool when it ends.  All of it runs on the device, so that
 * a decode loop needs no host synchronisation and can be captured in a graph.
 *
 * The conventions of kve.h hold here: every call returns a kve_status_t, checks
 * its arguments before anything is launched, allocates nothing, and enqueues
 * its work on `stream` of the current device.
 *
 * Rows
 * ----
 * A row of d channels is held as d four-bit floats (sign, two exponent bits,
 * one mantissa bit: 0, 0.5, 1, 1.5, 2, 3, 4, 6 and their negatives) and one scale
 * byte s for every 32 channels, which stands for the power of two 2^(s - 127).
 * With m the largest magnitude of the 32 and 2^e <= m < 2^(e+1),
 *     s = clamp(e + 125, 2, 252), with e + 1 in place of e when m >= 1.75 * 2^e
 * (the largest element is then off by least: at 1.75 * 2^e and above, 2^(e+1) is
 * at least as near as 1.5 * 2^e), and an element x is held as the nearest
 * four-bit float to x / 2^(s - 127): ties go to the even mantissa, larger ones to
 * +-6, the sign of zero is kept.  A block with a NaN or an infinity has s = 255
 * and reads as 32 NaN.  Every choice is exact in float32, and every value is
 * exact in bfloat16 and float32.  A row costs 17/32 bytes per channel: 3.76
 * times less than bfloat16.
 *
 * Pages
 * -----
 * A page holds `page` tokens of one layer and KV head, keys and values:
 *     key codes    [page, d / 2]   bytes, channel 2 i in the low half of byte i
 *     value codes  [page, d / 2]
 *     key scales   [d / 32, page]  bytes
 *     value scales [d / 32, page]
 * that is kve_page_bytes(page, d) = 17/16 page d bytes.  The pool is
 * [L, n_pages, Hkv, page bytes].  An eviction keeps equally many tokens of a
 * sample in every layer and KV head, so one list of page numbers per sequence
 * serves them all.  The bookkeeping is int32 and on the device:
 *     refs   [n_pages]  sequences that hold a page (0: free)
 *     table  [S, M]     page numbers of the sequence in each of S slots
 *     held   [S]        how many of them the sequence holds
 *     length [S]        tokens of the sequence
 * An empty cache has refs, held and length all zero; table entries at and beyond
 * `held` and the bytes of free pages are never used, whatever they are.  Only
 * full pages are shared, and appending writes only behind a sequence's length,
 * so no call changes a row that another sequence reads.
 *
 * Bookkeeping values are not trusted: slots outside [0, S) count as empty
 * sequences, page numbers outside [0, n_pages) as missing rows, held as at most
 * M, length as at most held * page.  No call reads or writes outside the
 * buffers whatever they hold.
 *
 * Calls on one cache are ordered by the caller, on one stream or by events, where
 * one changes bookkeeping or rows that the other uses.  Calls that only read
 * (kve_pages_read, kve_decode_pages) may overlap, and so may calls that write
 * rows of different sequences.
 */
#ifndef KVE_PAGES_H
#define KVE_PAGES_H

#include "kve.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * A paged cache: its buffers (device) and sizes.  `pool` must be 16-byte
 * aligned.  A call that works on rows of some of the layers passes the pool from
 * their first one on and L = their number; kve_pages_fork takes all layers in one
 * call, since it advances the bookkeeping that they share.  d is 64 or 128; page is a power of two, 32 .. 1024;
 * M * page and n_pages are at most 2^30, S * M at most 2^31 - 1.
 */
typedef struct kve_pages {
    void* pool;
    int32_t* refs;
    int32_t* table;
    int32_t* held;
    int32_t* length;
    int L, n_pages, Hkv, d, page, S, M;
} kve_pages_t;

/* Bytes of a page of one layer and KV head (0 if page or d is invalid). */
size_t kve_page_bytes(int page, int d);

/* Workspace bytes of kve_pages_extend and kve_pages_fork for up to n entries
 * (0 if invalid). */
size_t kve_pages_workspace_size(int n_pages, int S, int n);

/*
 * Makes room for add[i] more tokens in the sequence of slot seq[i], i < n, and
 * advances its length; the rows are the caller's to write (kve_pages_append,
 * kve_pages_compact, kve_pages_select), from position start[i] on.
 *
 * Entries are taken in order.  One is refused, and its sequence left as it is,
 * when its slot is outside [0, S) or named by an earlier entry, when add[i] < 0,
 * when the new length exceeds M * page, or when it needs pages and the free ones
 * at the call minus those that earlier entries need (also such as were refused
 * for want of pages) do not suffice.  The free pages are handed out in ascending order.
 *
 *   seq      [n] int32 (device), or NULL: entry i is slot i
 *   add      [n] int32 (device)
 *   start    [n] int32 out (device): the length before the call, -1 for a
 *            refused entry
 *   missing  [1] int32 out (device): pages that the entries needed beyond the
 *            free ones (0: every entry's need was met)
 *   workspace kve_pages_workspace_size bytes, 256-byte aligned, owned by the
 *            caller; contents on entry do not matter
 *
 * Errors: KVE_ERR_INVALID_ARG (null pointers, bad sizes, n < 1, n > S without
 * seq), KVE_ERR_UNSUPPORTED (n > 1024, d not 64/128, sizes above the limits),
 * KVE_ERR_WORKSPACE, KVE_ERR_HIP.
 */
kve_status_t kve_pages_extend(const kve_pages_t* pages, const int32_t* seq, const int32_t* add, int n,
                              int32_t* start, int32_t* missing, void* workspace, size_t workspace_bytes,
                              void* stream);

/*
 * Makes slot dst[i] a continuation of the sequence in slot src[i], i < n: the
 * full pages are shared, the rows of a partial last page are copied to a fresh
 * page, and pages that the source holds beyond its length are not passed on.
 * Page numbers outside [0, n_pages) are passed on as they are: rows that the
 * source lacks are missing from the continuation too.  A source may be named any
 * number of times.
 *
 * Entries are taken in order, the sources as they were before the call.  One
 * is refused, and its slot left as it is, when src or dst is outside [0, S),
 * when slot dst[i] holds pages or tokens or is named as dst by an earlier entry,
 * or when it needs a page and earlier entries need all that are free at the
 * call.  Free pages are handed out in ascending order.
 *
 *   src, dst [n] int32 (device)
 *   done     [n] int32 out (device): 1, or 0 for a refused entry
 *   missing, workspace and errors as for kve_pages_extend
 */
kve_status_t kve_pages_fork(const kve_pages_t* pages, const int32_t* src, const int32_t* dst, int n,
                            int32_t* done, int32_t* missing, void* workspace, size_t workspace_bytes,
                            void* stream);

/*
 * Empties the slots seq[i], i < n: held and length become 0 and the count of
 * each page that they held falls by one.  A slot named twice is emptied once;
 * slots outside [0, S) are passed over.  table keeps its entries.
 *
 *   seq  [n] int32 (device), or NULL: entry i is slot i (n <= S)
 *
 * Errors: KVE_ERR_INVALID_ARG, KVE_ERR_UNSUPPORTED (sizes), KVE_ERR_HIP.
 */
kve_status_t kve_pages_free(const kve_pages_t* pages, const int32_t* seq, int n, void* stream);

/*
 * Packs rows k[l, b, j, i], v[l, b, j, i], i < min(n_new[b], T), into positions
 * start[b] + i of the sequence in slot seq[b].  Rows whose position has no page
 * are dropped, as are all rows of a sequence whose start is negative (a refused
 * kve_pages_extend).  Positions below a sequence's length at a fork are shared:
 * start must not be below it.
 *
 *   k, v   [L, B, Hkv, T, d] (device, dtype), views as in kve.h (strides NULL:
 *          dense)
 *   n_new  [B] int32 (device), or NULL: T each
 *   start  [B] int32 (device), as kve_pages_extend returned it
 *   seq    [B] int32 (device), or NULL: sample b is slot b.  Two samples that
 *          write the same positions leave either's bytes.
 *
 * T = 0 is a valid size.  Errors: KVE_ERR_INVALID_ARG (null pointers, bad
 * sizes or strides, B > S without seq), KVE_ERR_UNSUPPORTED (dtype, d, sizes),
 * KVE_ERR_HIP.
 */
kve_status_t kve_pages_append(const void* k, const kve_strides_t* k_strides, const void* v,
                              const kve_strides_t* v_strides, kve_dtype_t dtype, int B, int T,
                              const int32_t* n_new, const int32_t* start, const int32_t* seq,
                              const kve_pages_t* pages, void* stream);

/*
 * kve_kv_compact into pages: packs rows k[l, b, j, idx[l, b, j, m]] and the same
 * of v into positions start[b] + m of the sequence in slot seq[b], for m <
 * min(count[l, b, j], k_cap).  Index values outside [0, N) are skipped (the
 * position's bytes are not written).
 *
 *   k, v   [L, B, Hkv, N, d] (device, dtype), views as in kve.h
 *   idx    [L, B, Hkv, k_cap] int32 (device)
 *   count  [L, B, Hkv] int32 (device)
 *   others as for kve_pages_append; k_cap = 0 is a valid size (nothing is launched;
 *          k and v, where not NULL, are checked all the same)
 */
kve_status_t kve_pages_compact(const void* k, const kve_strides_t* k_strides, const void* v,
                               const kve_strides_t* v_strides, kve_dtype_t dtype, int B, int N,
                               const int32_t* idx, const int32_t* count, int k_cap, const int32_t* start,
                               const int32_t* seq, const kve_pages_t* pages, void* stream);

/*
 * A second eviction: moves rows idx[l, b, j, m] of the sequence in slot src[b],
 * unchanged, to positions start[b] + m of the sequence in slot dst[b], for m <
 * min(count[l, b, j], k_cap).  Index values outside [0, length of the source) and
 * rows without a page are skipped (the position's bytes are not written).  The
 * source keeps its rows (kve_pages_free returns its pages).  src
 * and dst may name one slot when the rows read lie below start.
 *
 *   src, start, dst [B] int32 (device); idx, count as for kve_pages_compact
 *
 * Errors: KVE_ERR_INVALID_ARG, KVE_ERR_UNSUPPORTED, KVE_ERR_HIP.
 */
kve_status_t kve_pages_select(const kve_pages_t* pages, int B, const int32_t* src, const int32_t* idx,
                              const int32_t* count, int k_cap, const int32_t* dst, const int32_t* start,
                              void* stream);

/*
 * The values that rows of the cache stand for: k_out[l, b, j, i] is the key row
 * at position start[b] + i of the sequence in slot seq[b], and v_out the value
 * row, for i < min(count[b], T) and positions below the sequence's length.
 * Other rows of the outputs are left untouched.
 *
 *   T            rows of the outputs (0 is a valid size)
 *   seq          [B] int32 (device), or NULL: sample b is slot b
 *   start        [B] int32 (device), or NULL: 0 each; a negative one reads nothing
 *   count        [B] int32 (device), or NULL: T each
 *   k_out, v_out [L, B, Hkv, T, d] (device, dtype), 16-byte aligned; one may be
 *                NULL
 *
 * Errors: KVE_ERR_INVALID_ARG, KVE_ERR_UNSUPPORTED, KVE_ERR_HIP.
 */
kve_status_t kve_pages_read(const kve_pages_t* pages, kve_dtype_t dtype, int B, int T, const int32_t* seq,
                            const int32_t* start, const int32_t* count, void* k_out, void* v_out,
                            void* stream);

/* Workspace bytes that suffice for kve_decode_pages with these shapes, and for
 * any that have no more layers, samples, query heads and tokens (0 if invalid). */
size_t kve_decode_pages_workspace_size(int L, int B, int Hq, int Hkv, int max_tokens, int d);

/*
 * kve_decode_attention over paged sequences: one query per head attends to the
 * first n = min(length, max_tokens) rows of the sequence in slot seq[b],
 *   out[l, b, h] = sum_t softmax_t(scale * <q[l, b, h], k_t>) v_t,
 * k_t and v_t the rows of KV head h / (Hq/Hkv) as kve_pages_read gives them.  A
 * sequence with n = 0 gives zeros; rows whose page number is invalid are left out.
 * A NaN row makes the heads that read it NaN.  Logits are float32: one that falls
 * below its range has no weight.  A weight may grow to 2^16 before the sums are
 * rescaled, so n values of less than 2^112 / n each never overflow; larger ones may
 * become infinite.
 *
 *   q          [L, B, Hq, d] bf16 or fp32 (device), 16-byte aligned
 *   max_tokens a bound of the lengths that the caller knows (at most M * page):
 *              the work is split by it, and sequences under a bound of up to 2048
 *              need no second kernel where they are many
 *   scale      softmax scale; 0 means 1/sqrt(d)
 *   seq        [B] int32 (device), or NULL: sample b is slot b
 *   out        [L, B, Hq, d] float32 (device)
 *   workspace  kve_decode_pages_workspace_size bytes, 256-byte aligned, owned by
 *              the caller; contents on entry do not matter
 *
 * Products and sums are those of float32 numbers: the four-bit rows are exact in
 * bfloat16, and float32 queries and softmax weights go through the bfloat16
 * matrix instructions as three bfloat16 parts that add up to them.
 *
 * Requires Hq/Hkv <= 16.  Errors: KVE_ERR_INVALID_ARG (null pointers, bad sizes,
 * Hq not a multiple of Hkv, max_tokens outside [1, M * page], negative or
 * non-finite scale, B > S without seq), KVE_ERR_UNSUPPORTED (dtype, d, Hq/Hkv >
 * 16, sizes), KVE_ERR_WORKSPACE, KVE_ERR_HIP.
 */
kve_status_t kve_decode_pages(const void* q, kve_dtype_t dtype, const kve_pages_t* pages, int B, int Hq,
                              int max_tokens, const int32_t* seq, float scale, float* out, void* workspace,
                              size_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* KVE_PAGES_H */
