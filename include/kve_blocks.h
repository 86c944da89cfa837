/*
 * kve_blocks.h -- C ABI of the paged 8-bit cache (libkve.so)
 *
 * Next to the four-bit pages of kve_pages.h: a cache in pages of eight-bit rows
 * with one scale for each block of tokens and head.  It is filled by an eviction
 * step (kve_blocks_compact) or by a model's projections, whose keys and queries
 * are rotated to their positions on the way (kve_blocks_append); decode attends
 * to all of a sequence (kve_decode_blocks), or to the blocks that a score over
 * the bounds of their keys selects for each query token (kve_blocks_top).
 *
 * The conventions of kve.h hold here: every call returns a kve_status_t, checks
 * its arguments before anything is launched, allocates nothing, and enqueues
 * its work on `stream` of the current device.
 *
 * Blocks
 * ------
 * A block is one page: `page` tokens (32, 64 or 128) of one layer and KV head.
 * Its rows are eight-bit floats of type E4M3 (a sign, four exponent bits, three
 * of mantissa; no infinities, a NaN, largest value 448) times a power of two, one
 * for the block's keys and one for its values:
 *     key codes    [page, d]  bytes
 *     value codes  [page, d]
 *     key scale, value scale: a byte s each, for 2^(s - 127); 126 bytes unused
 *     key minima   [d]        codes: the smallest key of each channel
 *     key maxima   [d]
 * that is kve_block_bytes(page, d) = 2 page d + 128 + 2 d bytes.  With m the
 * largest finite magnitude of the rows that a call writes into a block, the block's
 * scale becomes
 *     s = clamp(smallest s with m <= 448 * 2^(s - 127), 27, 246),
 * or stays what it was where that is larger and the block held rows before.  An
 * element x is held as the E4M3 nearest to x / 2^(s - 127), ties to the even one,
 * magnitudes above 448 (only where s = 246) as 448; an infinity or a NaN is held
 * as a NaN.  Where the scale rises, the rows and bounds that the block held are
 * rounded once more in the same way: multiplying by a power of two changes only
 * those that become smaller than 2^-6 of the new scale.  The bounds are those of
 * the codes that calls have left in the block since a row was written at its first
 * position; a channel with a NaN has NaN bounds.  Every value is exact in bfloat16
 * and float32.
 *
 * The cache is a kve_pages_t whose pool is [L, n_pages, Hkv, block bytes] and
 * whose page is 32, 64 or 128.  The bookkeeping is that of kve_pages.h, and
 * kve_pages_extend and kve_pages_free, which do not touch the pool, serve it;
 * the other calls of kve_pages.h are for four-bit pools only.  As there,
 * bookkeeping values are not trusted, and no call reads or writes outside the
 * buffers whatever they hold.
 *
 * Calls on one cache are ordered by the caller, on one stream or by events, where
 * one changes bookkeeping or blocks that the other uses.  Calls that only read
 * may overlap, and so may calls that write rows of different sequences.
 */
#ifndef KVE_BLOCKS_H
#define KVE_BLOCKS_H

#include "kve_pages.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Bytes of a block (0 if page or d is invalid). */
size_t kve_block_bytes(int page, int d);

/*
 * A rotation of the first r channels of a row, in pairs: channels i and i + r/2,
 * or with `pairs` not 0 channels 2 i and 2 i + 1, for i < r/2.  A row at position
 * p has its pair (a, b) replaced by
 *     (a cos[p, i] - b sin[p, i],  b cos[p, i] + a sin[p, i]).
 *
 *   cos, sin   [P, r/2] float32 (device), 16-byte aligned
 *   position   [B, T] int32 (device): the position of each token
 *   r          a multiple of 16, 16 .. d
 *
 * Products and sums are exact to 53 bits and what they give is rounded once, to
 * what holds it.  A row whose position is outside [0, P) becomes NaN.
 */
typedef struct kve_rotation {
    const float* cos;
    const float* sin;
    const int32_t* position;
    int P, r, pairs;
} kve_rotation_t;

/*
 * Writes rows k[l, b, j, i], v[l, b, j, i], i < min(n_new[b], T), into positions
 * start[b] + i of the sequence in slot seq[b], the keys rotated.  Rows whose
 * position has no page are dropped, as are all rows of a sequence whose start is
 * negative (a refused kve_pages_extend).  A block that holds positions below
 * start[b] keeps them (see above); what it held at start[b] and beyond is gone, but
 * its scale and bounds may stay as wide as that made them.
 * With q, also writes the queries, rotated in the same way and rounded to their
 * type, to q_out: all of them, whatever start and n_new are.
 *
 *   k, v     [L, B, Hkv, T, d] (device, dtype), views as in kve.h (strides NULL:
 *            dense)
 *   n_new    [B] int32 (device), or NULL: T each
 *   start    [B] int32 (device), as kve_pages_extend returned it
 *   seq      [B] int32 (device), or NULL: sample b is slot b.  Two samples that
 *            write into one block leave it with rows, scale and bounds of either.
 *   rotation NULL: keys as they are
 *   q        [L, B, Hq, T, d] (device, dtype), a view, or NULL; needs a rotation
 *   q_out    [L, B, Hq, T, d] (device, dtype), dense, 16-byte aligned, not q itself
 *
 * T = 0 is a valid size: nothing is launched, k, v and the rotation's tables may be
 * NULL, and what is given is checked all the same.  Errors: KVE_ERR_INVALID_ARG
 * (null pointers, bad sizes, strides or rotation, B > S without seq, q without q_out
 * or rotation), KVE_ERR_UNSUPPORTED (dtype, d, sizes), KVE_ERR_HIP.
 */
kve_status_t kve_blocks_append(const void* k, const kve_strides_t* k_strides, const void* v,
                               const kve_strides_t* v_strides, kve_dtype_t dtype, int B, int T,
                               const int32_t* n_new, const int32_t* start, const int32_t* seq,
                               const kve_pages_t* blocks, const kve_rotation_t* rotation, const void* q,
                               const kve_strides_t* q_strides, int Hq, void* q_out, void* stream);

/*
 * kve_kv_compact into blocks: writes rows k[l, b, j, idx[l, b, j, m]] and the
 * same of v, as they are, into positions start[b] + m of the sequence in slot
 * seq[b], for m < min(count[l, b, j], k_cap).  Index values outside [0, N) leave
 * rows of zeros.
 *
 *   k, v   [L, B, Hkv, N, d] (device, dtype), views as in kve.h
 *   idx    [L, B, Hkv, k_cap] int32 (device)
 *   count  [L, B, Hkv] int32 (device)
 *   others as for kve_blocks_append; k_cap = 0 is a valid size (nothing is launched;
 *          k and v, where not NULL, are checked all the same)
 */
kve_status_t kve_blocks_compact(const void* k, const kve_strides_t* k_strides, const void* v,
                                const kve_strides_t* v_strides, kve_dtype_t dtype, int B, int N,
                                const int32_t* idx, const int32_t* count, int k_cap, const int32_t* start,
                                const int32_t* seq, const kve_pages_t* blocks, void* stream);

/* kve_pages_read for blocks: the values that rows of the cache stand for. */
kve_status_t kve_blocks_read(const kve_pages_t* blocks, kve_dtype_t dtype, int B, int T, const int32_t* seq,
                             const int32_t* start, const int32_t* count, void* k_out, void* v_out,
                             void* stream);

/*
 * The bounds of the keys of blocks first[b] + i, i < n, of the sequence in slot
 * seq[b]: lo_out[l, b, j, i] and hi_out[l, b, j, i], rows of d channels.  Rows for
 * blocks that the sequence does not have are left untouched.
 *
 *   n              0 is a valid size
 *   seq            [B] int32 (device), or NULL: sample b is slot b
 *   first          [B] int32 (device), or NULL: 0 each; a negative one reads nothing
 *   lo_out, hi_out [L, B, Hkv, n, d] (device, dtype), 16-byte aligned; one may be NULL
 *
 * Errors: KVE_ERR_INVALID_ARG, KVE_ERR_UNSUPPORTED, KVE_ERR_HIP.
 */
kve_status_t kve_blocks_bounds(const kve_pages_t* blocks, kve_dtype_t dtype, int B, int n, const int32_t* seq,
                               const int32_t* first, void* lo_out, void* hi_out, void* stream);

/*
 * What query token t < T of a sample sees: the first
 *     n(b, t) = min(start[b] + t + 1, length, max_tokens)
 * rows of its sequence, none where start[b] < 0; without start, start[b] is
 * length - T: the queries are those of the sequence's last T tokens.
 *
 * Workspace bytes that suffice for kve_blocks_top with these shapes, and for any
 * that have no more layers, samples, query tokens and tokens (0 if invalid).
 */
size_t kve_blocks_top_workspace_size(int L, int B, int Hkv, int T, int max_tokens, int page);

/*
 * For each query token and KV head the k blocks, of the ceil(n(b, t) / page) that
 * hold rows it sees, whose keys can reach the highest product with its queries: with
 * lo and hi a block's bounds, and up and down the sums over the G query heads of
 * the KV head of max(q, 0) and min(q, 0), a block's score is
 *     sum_c up[c] hi[c] + down[c] lo[c],
 * an upper bound of sum_h <q_h, k_t> over the block's keys.  The first `first`
 * blocks and the last `last` are always taken; the others by falling score, equal
 * ones and zeros of either sign by rising index, NaN and blocks without a page
 * last.  Scores are summed in 64 bits and rounded once to float32.
 *
 *   q     [L, B, Hq, T, d] (device, dtype), dense, 16-byte aligned
 *   start [B] int32 (device), or NULL
 *   seq   [B] int32 (device), or NULL: sample b is slot b
 *   k     at least max(1, first + last)
 *   top   [L, B, Hkv, T, k] int32 out (device): the blocks, ascending, then -1
 *   workspace kve_blocks_top_workspace_size bytes, 256-byte aligned, owned by the
 *         caller; contents on entry do not matter
 *
 * Errors: KVE_ERR_INVALID_ARG (null pointers, bad sizes, Hq not a multiple of Hkv,
 * max_tokens outside [1, M * page], k < max(1, first + last), B > S without seq),
 * KVE_ERR_UNSUPPORTED (dtype, d, sizes), KVE_ERR_WORKSPACE, KVE_ERR_HIP.
 */
kve_status_t kve_blocks_top(const void* q, kve_dtype_t dtype, const kve_pages_t* blocks, int B, int Hq, int T,
                            int max_tokens, const int32_t* start, const int32_t* seq, int k, int first, int last,
                            int32_t* top, void* workspace, size_t workspace_bytes, void* stream);

/* Workspace bytes that suffice for kve_decode_blocks with these shapes, and for any
 * that have no more layers, samples, query heads and query tokens (0 if invalid). */
size_t kve_decode_blocks_workspace_size(int L, int B, int Hq, int Hkv, int T, int d);

/*
 * Attention of T query tokens of each sample to the rows they see,
 *   out[l, b, h, t] = sum_i softmax_i(scale * <q[l, b, h, t], k_i>) v_i,  i < n(b, t),
 * k_i and v_i the rows of KV head h / (Hq/Hkv) as kve_blocks_read gives them; with
 * `top`, i runs over the rows seen in blocks top[l, b, h / (Hq/Hkv), t, 0 .. k).
 * Entries of top outside [0, M) are passed over; a block named twice counts twice.
 * No rows give zeros; rows whose page number is invalid are left out.  A NaN row
 * makes the outputs that see it NaN, and no others.  Logits are float32: one
 * that falls below its range has no weight.  A weight may grow to 2^16 before the
 * sums are rescaled, so n values of less than 2^112 / n each never overflow; larger
 * ones may become infinite.
 *
 *   q          [L, B, Hq, T, d] bf16 or fp32 (device), dense, 16-byte aligned
 *   max_tokens a bound of the lengths that the caller knows (at most M * page):
 *              the work is split by it
 *   start, seq as above
 *   top        [L, B, Hkv, T, k] int32 (device), or NULL with k = 0
 *   scale      softmax scale; 0 means 1/sqrt(d)
 *   out        [L, B, Hq, T, d] float32 (device)
 *   workspace  kve_decode_blocks_workspace_size bytes, 256-byte aligned, owned by
 *              the caller; contents on entry do not matter
 *
 * Products and sums are those of float32 numbers, as in kve_decode_pages.  Query
 * tokens share a read of the sequence while Hq/Hkv times their number is at most
 * 16; with `top` each reads its own blocks.
 *
 * Requires Hq/Hkv <= 16.  Errors: KVE_ERR_INVALID_ARG (null pointers, bad sizes,
 * Hq not a multiple of Hkv, max_tokens outside [1, M * page], negative or
 * non-finite scale, k < 1 with top, B > S without seq), KVE_ERR_UNSUPPORTED
 * (dtype, d, Hq/Hkv > 16, sizes), KVE_ERR_WORKSPACE, KVE_ERR_HIP.
 */
kve_status_t kve_decode_blocks(const void* q, kve_dtype_t dtype, const kve_pages_t* blocks, int B, int Hq, int T,
                               int max_tokens, const int32_t* start, const int32_t* seq, const int32_t* top, int k,
                               float scale, float* out, void* workspace, size_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* KVE_BLOCKS_H */
