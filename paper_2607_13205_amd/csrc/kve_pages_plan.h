// The paged 4-bit cache: what its kernels and the C ABI share.  Plain C++.
#pragma once

#include <stddef.h>
#include <stdint.h>

#include "kve_decode_plan.h"

namespace kve {

constexpr int kPageMin = 32, kPageMax = 1024;  // tokens per page, powers of two
constexpr int kPagesMaxEntries = 1024;         // entries of one bookkeeping call: one per thread of its workgroup
constexpr int kPagesMaxGroup = 16;             // query heads per KV head: the columns of a 16x16 product
constexpr int kPagesRows = 64;                 // rows per workgroup of a call on rows
constexpr int kPagesPlanBytes = 32;            // what a fork notes for an entry

// The cache as kernels see it.  shift: log2 of the page size.
struct PagePool {
    char* pool;
    int32_t *refs, *table, *held, *length;
    int L, n_pages, Hkv, S, M, shift;
};

// Bytes of one page of one (layer, KV head): two codes per byte and a scale byte
// per 32 channels, keys and values.  A multiple of 16 for every valid size.
inline size_t page_block_bytes(int page, int d) { return (size_t)page * d / 16 * 17; }

// Parts of a page of all KV heads of a layer that kve_pages_fork copies, one per workgroup.
constexpr int kPagesCopyBytes = 16384;
inline int pages_copy_blocks(int Hkv, int page, int d) {
    return (int)((Hkv * page_block_bytes(page, d) + kPagesCopyBytes - 1) / kPagesCopyBytes);
}

// Workspace of extend and fork: a note per entry, then the free pages found, at
// most as many as there are.
inline size_t pages_workspace(int n_pages, int n) {
    return align_up((size_t)n * kPagesPlanBytes) + align_up((size_t)n_pages * sizeof(int32_t));
}

// Plan of a decode over pages.  The lengths are on the device, so the splits are
// cut there: in whole quanta of kDecodeQuantum tokens, all of the same size, which
// is a `share`-th of all sequences' quanta, `share` being one round of resident
// workgroups over all (layer, KV head) pairs.  That makes at most share + B splits
// (a sequence's last one may be short).  They are numbered one sequence after the
// other, and workgroup x of each pair takes split x.  More than kPagesSlice sequences that
// are cut are taken by layers and in slices of equally many, calls of their own.
struct PagesPlan {
    int pairs, G, groups;  // groups: workgroups per (layer, KV head)
    int slice;             // sequences of a launch; where not all, the other fields but `total` do not count
    bool whole;            // one split per sequence: nothing to merge
    int per_unit;          // workgroups that share a compute unit: 1, 2 or 4
    size_t off_ml, off_ranges, total;
};

// `whole`, one split per sequence with no search and no merge, where none can be
// long (longer ones may differ too much) or long for their number; a workgroup
// then has all waves of a compute unit, half of them or four, so that the
// sequences fill the chip once.  Device time of a captured call, 8 KV heads of 4
// query heads, so and split: 32 sequences of 1000 tokens 11.7 and 17.2 us, of 2000
// 17 and 22.2, 64 of 1000 17 and 22.9, 100 of 500 16.2 and 20.2, 120 of 2000 49 and
// 78, 16 of 2000 15.0 and 16.3, 4 of 500 8.5 and 9.1, but 4 of 1639 12.5 and 10.4,
// one of 1000 10.3 and 9.0, 32 of 4000 28.2 and 33.  Lengths that differ, up to the
// same ones: 100 of 2000 24.3 and 28.5, 64 of 2000 16.7 and 17.9, 64 of 1000 11.4
// and 14.6, 32 of 2000 14.5 and 14.1, but 16 of 2000 14.2 and 12.1, 8 of 1000 10.2
// and 9.1, 32 of 4000 21.4 and 18.2.
constexpr int kPagesMostResident = 4 * kDecodeUnits;  // workgroups, at four per compute unit
constexpr int kPagesWhole = 4;                        // quanta up to which every sequence is one split

// Most sequences of one launch that are cut into splits.  Every workgroup finds its split
// among them by itself, so that more in one launch would cost their square; as many as
// have their lengths kept in LDS.
constexpr int kPagesSlice = 4096;

// Workspace of a decode whose splits leave `parts` partial results.
inline size_t decode_pages_bytes(size_t parts, int B, int d, PagesPlan* p) {
    p->off_ml = align_up(parts * d * sizeof(float));
    p->off_ranges = p->off_ml + align_up(parts * 2 * sizeof(float));
    return p->off_ranges + align_up((size_t)B * 2 * sizeof(int32_t));  // every sequence's first split and count
}

inline PagesPlan decode_pages_plan(int L, int B, int Hq, int Hkv, int max_tokens, int d) {
    PagesPlan p{};
    p.pairs = L * Hkv;
    p.G = Hq / Hkv;
    const long long quanta = ((long long)max_tokens + kDecodeQuantum - 1) / kDecodeQuantum;
    const long long segs = (long long)p.pairs * B;
    p.whole = quanta <= kDecodeLongest && quanta <= (segs / 8 > kPagesWhole ? segs / 8 : kPagesWhole);
    p.per_unit = !p.whole ? 4 : segs <= kDecodeUnits ? 1 : segs <= 2 * kDecodeUnits ? 2 : 4;
    const int share = p.pairs < kPagesMostResident ? kPagesMostResident / p.pairs : 1;
    long long groups = (long long)share + B;
    if (groups > B * quanta) groups = B * quanta;
    if (p.whole) groups = B;
    p.groups = (int)groups;
    const int slices = p.whole ? 1 : (B + kPagesSlice - 1) / kPagesSlice;
    p.slice = (B + slices - 1) / slices;
    if (slices > 1) {  // a slice that is not the last, and the last
        const int last = B - (slices - 1) * p.slice;
        const size_t a = decode_pages_plan(1, p.slice, Hq, Hkv, max_tokens, d).total;
        const size_t b = decode_pages_plan(1, last, Hq, Hkv, max_tokens, d).total;
        p.total = a > b ? a : b;
        return p;
    }
    p.total = decode_pages_bytes(p.whole ? 0 : (size_t)p.pairs * p.groups * p.G, B, d, &p);
    return p;
}

// Workspace that suffices for this call and for every one of no more layers,
// samples, query heads and tokens, whose sequences may be split where this call's
// are not: the splits, at most share + B, of the largest call that has any.
inline size_t decode_pages_size(int L, int B, int Hq, int Hkv, int max_tokens, int d) {
    const long long quanta = ((long long)max_tokens + kDecodeQuantum - 1) / kDecodeQuantum;
    long long pairs = (long long)L * Hkv, segs = pairs * B;
    if (quanta <= kPagesWhole)
        segs = 0;
    else if (quanta <= kDecodeLongest && segs > 8 * quanta - 1)
        segs = 8 * quanta - 1;  // more are whole
    if (pairs > segs) pairs = segs;
    const long long most = (pairs > kPagesMostResident ? pairs : kPagesMostResident) + segs;
    PagesPlan p{};
    return decode_pages_bytes((size_t)(most < segs * quanta ? most : segs * quanta) * (Hq / Hkv), B, d, &p);
}

}  // namespace kve
