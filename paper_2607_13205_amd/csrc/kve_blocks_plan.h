// The paged 8-bit cache: what its kernels and the C ABI share.  Plain C++.
#pragma once

#include <stddef.h>
#include <stdint.h>

#include "kve_pages_plan.h"

namespace kve {

constexpr int kBlockMax = 128;    // tokens per block: 32, 64 or 128
constexpr int kBlockScales = 128;  // bytes of a block's tail before its bounds
constexpr int kBlockScaleMin = 27, kBlockScaleMax = 246;

inline size_t block_bytes(int page, int d) { return (size_t)2 * page * d + kBlockScales + 2 * d; }

// A rotation as kernels see it; cos null: none.
struct BlockRotation {
    const float *cos, *sin;
    const int32_t* position;
    int P, r, pairs;
};

// Blocks that `rows` rows can touch, wherever the first one lies.
inline long long blocks_touched(long long rows, int page) { return rows == 0 ? 0 : (rows + page - 2) / page + 1; }

constexpr int kBlocksQueryHeads = 4;  // heads per workgroup that rotates queries, of 32 tokens or more

// What query tokens see (kve_blocks.h): start null: the last T tokens.
struct BlockView {
    const int32_t *seq, *start;
    int B, T, max_tokens;
};

// Workgroups per compute unit that a decode is cut for.  One reads as fast as two that
// a unit holds, and leaves the fewest partial results (8 sequences of 32768 tokens, 8 KV
// heads: 102.6 us with one, 103.6, 109 and 104 with two, three and four; 16 tokens' pairs
// of 100 blocks of 32 41, 46 and 53).  Sequences whose lengths differ leave units without
// work at the end, the fewer the shorter the splits are (64 of up to 32768: 251 us with
// one, 231, 216 and 211; 8 57, 54, 53 and 52; but 4 33, 33, 36 and 35, 2 20, 21, 25 and
// 27): from kBlocksSeveral entries on those are cut for four.
// Rows of 64 channels are half as many bytes to a step, too few in flight in one workgroup
// to read at full rate: level ones are cut for two where there are kBlocksLong quanta to
// a unit (8 sequences of 122844, 2 KV heads 47.7 us for 53.6, 4 of 20000, 4 heads 14.5 for
// 15.4, but 2 heads, five quanta to a unit, 12.5 for 11.9).
constexpr int kBlocksLevel = 1, kBlocksRagged = 4, kBlocksSeveral = 8, kBlocksLong = 8;

// Plan of a decode over blocks.  Query tokens of a sample are taken `per` at a time,
// an entry each: as many as the sixteen columns of a product hold heads for, or one
// where each has its own blocks.  The entries' tokens are cut as PagesPlan's, up to
// kPagesSlice entries at a time.
struct BlocksPlan {
    int pairs, G, per, tiles, entries, R;  // R: query rows of an entry, per * G
    int slice;                             // entries of a launch
    int share, level;                      // splits of all entries together, and where their lengths are level
    int groups;                            // workgroups per (layer, KV head) and launch
    bool whole;                            // one split per entry: nothing to merge
    size_t off_ml, off_ranges, total;
};

inline size_t decode_blocks_bytes(size_t parts, long long entries, int d, BlocksPlan* p) {
    p->off_ml = align_up(parts * d * sizeof(float));
    p->off_ranges = p->off_ml + align_up(parts * 2 * sizeof(float));
    return p->off_ranges + align_up((size_t)entries * 2 * sizeof(int32_t));  // every entry's first split and count
}

// tokens: a bound of an entry's tokens.
inline BlocksPlan decode_blocks_plan(int L, int B, int Hq, int Hkv, int T, long long tokens, bool sparse, int d) {
    BlocksPlan p{};
    p.pairs = L * Hkv;
    p.G = Hq / Hkv;
    p.per = sparse ? 1 : kPagesMaxGroup / p.G;
    if (p.per > T) p.per = T;
    p.tiles = (T + p.per - 1) / p.per;
    p.entries = B * p.tiles;
    p.R = p.per * p.G;
    const long long quanta = (tokens + kDecodeQuantum - 1) / kDecodeQuantum;
    const long long segs = (long long)p.pairs * p.entries;
    p.whole = quanta <= kDecodeLongest && quanta <= (segs / 8 > kPagesWhole ? segs / 8 : kPagesWhole);
    auto splits = [&](int per_unit) {
        return p.pairs < per_unit * kDecodeUnits ? per_unit * kDecodeUnits / p.pairs : 1;
    };
    p.level = splits(d == 64 && segs * quanta >= kBlocksLong * kDecodeUnits ? 2 * kBlocksLevel : kBlocksLevel);
    // chosen blocks are equally many
    p.share = sparse || p.entries < kBlocksSeveral ? p.level : splits(kBlocksRagged);
    const int slices = p.whole ? 1 : (p.entries + kPagesSlice - 1) / kPagesSlice;
    p.slice = (p.entries + slices - 1) / slices;
    long long groups = (long long)p.share + p.slice;
    if (groups > p.slice * quanta) groups = p.slice * quanta;
    if (p.whole) groups = p.slice;
    p.groups = (int)groups;
    p.total = decode_blocks_bytes(p.whole ? 0 : (size_t)p.pairs * p.groups * p.R, p.slice, d, &p);
    return p;
}

// Workspace that suffices for this call and for every one of no more layers,
// samples, query heads and query tokens: at most one round of workgroups, or one
// of every pair, and one of every entry, of R rows each; the last entry of a
// sample may have fewer query tokens than its rows, which at most doubles them.
inline size_t decode_blocks_size(int L, int B, int Hq, int Hkv, int T, int d) {
    const long long pairs = (long long)L * Hkv, G = Hq / Hkv;
    const long long most = G * T < kPagesMaxGroup ? G * T : kPagesMaxGroup;
    const long long round = pairs > kBlocksRagged * kDecodeUnits ? pairs : kBlocksRagged * kDecodeUnits;
    BlocksPlan p{};
    return decode_blocks_bytes((size_t)(round * most + pairs * B * G * T * (T > 1 ? 2 : 1)), (long long)B * T, d, &p);
}

// Blocks that max_tokens tokens can lie in.
inline int top_blocks(int max_tokens, int page) { return (max_tokens + page - 1) / page; }

// Keys from one segment's first to the next one's: four are loaded at once.
inline int top_pitch(int blocks) { return (blocks + 3) / 4 * 4; }

inline size_t top_size(int L, int B, int Hkv, int T, int max_tokens, int page) {
    return align_up((size_t)L * B * Hkv * T * top_pitch(top_blocks(max_tokens, page)) * sizeof(uint32_t));
}

}  // namespace kve
