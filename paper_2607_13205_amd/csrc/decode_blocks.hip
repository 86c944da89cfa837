// Attention over paged 8-bit sequences: the queries of one or a few tokens of each
// sample attend to the rows of its sequence, or of the blocks chosen for them,
// through the page table (kve_decode_blocks).
//
// The products are those of the decode over four-bit pages (decode_pages.hip): eight-
// bit rows times their power of two are exact in bf16 as well, S^T = K Q^T and
// O^T = V^T P^T on the bf16 matrix instructions, 32 tokens to a wave's step, the
// weights in their registers between the two.  The sixteen columns hold the query
// heads of one or several query tokens.  A token that is masked for a column has no
// weight in it whatever its row holds.
//
// A step's bytes go straight to LDS, two steps ahead, twice those of four-bit rows:
// two workgroups share a compute unit.  Twice the bytes for the same products also
// leave the vector unit further from being the bound.
#include <type_traits>

#include "kve_blocks_device.h"
#include "kve_decode_merge.h"
#include "kve_decode_split.h"
#include "kve_device.h"
#include "kve_internal.h"
#include "kve_stream.h"

namespace kve {
namespace {

constexpr int kThreads = kMergeThreads;
constexpr int kWaves = kThreads / kWave;
constexpr int kBlk = 32;       // tokens per wave step

// What a wave loads for 32 tokens of a block: key codes, value codes and, in every
// lane, the two scale bytes.  16-byte pieces of a key row are permuted so that the
// sixteen rows that a quarter wave reads at once lie in distinct banks: piece ^ row /
// 2 % 8 of the eight in a row of 128 channels, ^ row / 4 % 4 of the four in one of 64.
template <int D>
struct Slot {
    static constexpr int kCodes = kBlk * D;  // bytes of the key, and of the value codes
    static constexpr int kLoads = 2 * kCodes / 1024 + 1;
    static constexpr int kBytes = 2 * kCodes + 256;
    static constexpr int kSlots = 2;  // steps ahead

    __device__ __forceinline__ static int swizzle(int row) { return D == 128 ? (row >> 1) & 7 : (row >> 2) & 3; }

    // The wave's loads of tokens tok .. + 32 of a block into `slot`: kLoads of them.
    __device__ __forceinline__ static void load(const char* block, int tok, int shift, const char* slot) {
        const int lane = threadIdx.x & (kWave - 1);
        const char* keys = block + tok * D;
        const char* values = keys + ((size_t)D << shift);
        // rows of a load: 8 of 128 channels, and every second load has its pieces four on; 16 of 64
        const uint32_t piece = (uint32_t)(lane ^ swizzle(D == 128 ? lane >> 3 : lane >> 2)) * 16;
#pragma unroll
        for (int i = 0; i < kCodes / 1024; ++i)
            lds_dma16<true>(keys + i * 1024, D == 128 && i % 2 != 0 ? piece ^ 64u : piece, slot + i * 1024);
#pragma unroll
        for (int i = 0; i < kCodes / 1024; ++i)
            lds_dma16<true>(values + i * 1024, lane * 16, slot + kCodes + i * 1024);
        lds_dma4(block + tail_at<D>(shift), 0, slot + 2 * kCodes);
    }
};

// Eight codes as bf16.
__device__ __forceinline__ bf16x8 unpack8(u32x2 w, float scale) {
    u32x4 r;
    r[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[0], scale, false));
    r[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[0], scale, true));
    r[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[1], scale, false));
    r[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[1], scale, true));
    return __builtin_bit_cast(bf16x8, r);
}

// Half HI of eight dwords as bf16 pairs (two channels of a token each), regrouped
// into the eight tokens of either channel.
template <bool HI>
__device__ __forceinline__ void unpack_tokens(const uint32_t (&w)[8], float scale, bf16x8& even, bf16x8& odd) {
    uint32_t c[8];
#pragma unroll
    for (int i = 0; i < 8; ++i)
        c[i] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[i], scale, HI));
    u32x4 e, o;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        e[i] = __builtin_amdgcn_perm(c[2 * i + 1], c[2 * i], 0x05040100u);
        o[i] = __builtin_amdgcn_perm(c[2 * i + 1], c[2 * i], 0x07060302u);
    }
    even = __builtin_bit_cast(bf16x8, e);
    odd = __builtin_bit_cast(bf16x8, o);
}

// The running softmax sums of a wave over its tokens.  NH columns of query rows: up
// to 4 of three copies each, 8 of two, or 16.
template <typename T, int D, int NH>
struct Sums {
    using S = Slot<D>;
    static constexpr int NP = std::is_same<T, float>::value ? 3 : 1;  // bf16 parts of a query
    static constexpr int NK = D / 32;  // products per 16 tokens
    static constexpr int NC = D / 16;  // channels per lane of V^T
    static constexpr int NW = NH == 4 ? 1 : NH == 8 ? 2 : 3;  // parts of the weights per lane
    bf16x8 q[NK][NP];
    float m;
    f32x4 den, o[NC];  // o[i][r]: channel NC (4 (lane / 16) + r) + i of column lane % 16

    // row: the query row of the lane's column, null for none
    __device__ __forceinline__ void start(const T* row) {
        const int quarter = (threadIdx.x & (kWave - 1)) >> 4;
#pragma unroll
        for (int s = 0; s < NK; ++s) {
            if constexpr (NP == 1) {
                u32x4 y = zero16();
                if (row != nullptr) y = ld16(row + D / 4 * quarter + 8 * s);
                q[s][0] = __builtin_bit_cast(bf16x8, y);
            } else {
                float y[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) y[i] = row != nullptr ? (float)row[D / 4 * quarter + 8 * s + i] : 0.0f;
                split3(y, q[s]);
            }
        }
        m = kLowest;
        den = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int i = 0; i < NC; ++i) o[i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    }

    __device__ __forceinline__ void settle_queries() {
#pragma unroll
        for (int s = 0; s < NK; ++s)
#pragma unroll
            for (int a = 0; a < NP; ++a) settle(q[s][a]);
    }

    // The logits of 32 tokens, before scaling: row m of tile T is token 16 T + 4 (m % 4)
    // + m / 4, so that a lane receives tokens 4 i + quarter, i < 8.
    __device__ __forceinline__ void logits(const char* slot, float scale, f32x4 (&acc)[2]) const {
        const int lane = threadIdx.x & (kWave - 1);
        const int c = lane & 15, quarter = lane >> 4;
        const int tok = 4 * (c & 3) + (c >> 2);
        const char* row = slot + tok * D;
        const int swz = S::swizzle(tok);
#pragma unroll
        for (int tile = 0; tile < 2; ++tile) {
            u32x4 k[NK / 2];
#pragma unroll
            for (int e = 0; e < NK / 2; ++e)
                k[e] = ld16(row + tile * 16 * D + (((quarter * (D / 64) + e) ^ swz) << 4));
            acc[tile] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int e = 0; e < NK; ++e) {
                const bf16x8 kf = unpack8(u32x2{k[e / 2][e % 2 * 2], k[e / 2][e % 2 * 2 + 1]}, scale);
#pragma unroll
                for (int a = NP - 1; a >= 0; --a) acc[tile] = mma(kf, q[e][a], acc[tile]);
            }
        }
    }

    // The tokens' share of the sums.  left: tokens that count for the lane's column;
    // most: for any column; even: for all columns alike, and tile the query token of
    // the column where not (Several).  tiles: query tokens of the entry.
    template <bool Several>
    __device__ __forceinline__ void add(const char* slot, float scale, f32x4 (&acc)[2], int left, int most, bool even,
                                        int tile, int tiles, float sl2) {
        const int lane = threadIdx.x & (kWave - 1);
        const int c = lane & 15, quarter = lane >> 4;
        const char* rows = slot + S::kCodes + quarter * D + c * NC;
        uint32_t v[NC / 4][8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if constexpr (D == 128) {
                const u32x2 w = *reinterpret_cast<const u32x2*>(rows + 4 * i * D);
                v[0][i] = w[0];
                v[1][i] = w[1];
            } else {
                v[0][i] = *reinterpret_cast<const uint32_t*>(rows + 4 * i * D);
            }
        }
        if (most < kBlk || (Several && !even)) {
            __builtin_amdgcn_sched_barrier(0);  // a branch, not selects in every step
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                if (4 * i + quarter >= left) acc[i >> 2][i & 3] = -INFINITY;
                // rows behind the sequence hold anything: no weight, and zeros under it
                if (4 * i + quarter >= most)
#pragma unroll
                    for (int e = 0; e < NC / 4; ++e) v[e][i] = 0;
            }
        }
        float top = acc[0][0];
#pragma unroll
        for (int i = 1; i < 8; ++i) top = fmaxf(top, acc[i >> 2][i & 3]);
        if (__builtin_amdgcn_ballot_w64(top * sl2 > m + kRaise) != 0) {
            top = fmaxf(top, __shfl_xor(top, 16));
            top = fmaxf(top, __shfl_xor(top, 32));
            const float mn = fmaxf(m, top * sl2);
            const float alpha = fast_exp2(m - mn);
            m = mn;
            den *= alpha;
#pragma unroll
            for (int i = 0; i < NC; ++i) o[i] *= alpha;
        }
        float w[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) w[i] = fast_exp2(fmaf(acc[i >> 2][i & 3], sl2, -m));
        bf16x8 part[NW];
        weight_parts<NH>(w, c, part);
        const u32x4 ones = {0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u};
#pragma unroll
        for (int a = NW - 1; a >= 0; --a) den = mma(__builtin_bit_cast(bf16x8, ones), part[a], den);
        if (!Several || even) {
            values<false>(v, scale, part, true);
            return;
        }
        // a product takes no weight times a NaN for a NaN: without one, all query tokens at
        // once, the rows that a column does not see with no weight
        uint32_t bad = 0;
#pragma unroll
        for (int e = 0; e < NC / 4; ++e)
#pragma unroll
            for (int i = 0; i < 8; ++i) bad |= nan_codes(v[e][i]);
        const int turns = __builtin_amdgcn_ballot_w64(bad != 0) == 0 ? 1 : tiles;
        // with one, query token by query token: the rows behind what it sees as zeros, and only
        // its columns' sums kept
#pragma unroll 1
        for (int t = 0; t < turns; ++t) {
            const bool all = turns == 1;
            const uint64_t mine = __builtin_amdgcn_ballot_w64(all || tile == t);
            if (mine == 0) continue;
            const int seen = all ? kBlk : __builtin_amdgcn_readlane(left, __builtin_ctzll(mine));
            uint32_t vt[NC / 4][8];
#pragma unroll
            for (int e = 0; e < NC / 4; ++e)
#pragma unroll
                for (int i = 0; i < 8; ++i) vt[e][i] = 4 * i + quarter < seen ? v[e][i] : 0u;
            values<true>(vt, scale, part, all || tile == t);
        }
    }

    // Some: of the lane's column only where `keep`.
    template <bool Some>
    __device__ __forceinline__ void values(const uint32_t (&v)[NC / 4][8], float scale, const bf16x8 (&part)[NW],
                                           bool keep) {
#pragma unroll
        for (int e = 0; e < NC / 4; ++e) {
            half<false, Some>(v[e], scale, part, keep, o[4 * e], o[4 * e + 1]);
            half<true, Some>(v[e], scale, part, keep, o[4 * e + 2], o[4 * e + 3]);
        }
    }

    template <bool HI, bool Some>
    __device__ __forceinline__ static void half(const uint32_t (&v)[8], float scale, const bf16x8 (&part)[NW],
                                                bool keep, f32x4& a, f32x4& b) {
        bf16x8 even, odd;
        unpack_tokens<HI>(v, scale, even, odd);
        f32x4 na = a, nb = b;
#pragma unroll
        for (int x = NW - 1; x >= 0; --x) {
            na = mma(even, part[x], na);
            nb = mma(odd, part[x], nb);
        }
        if constexpr (Some) {
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                a[r] = keep ? na[r] : a[r];
                b[r] = keep ? nb[r] : b[r];
            }
        } else {
            a = na;
            b = nb;
        }
    }

    // the parts of a column's sums added up in its first copy
    __device__ __forceinline__ void finish() {
        if constexpr (NH == 4) {
            den[0] = den[0] + (row_from<4>(den[0]) + row_from<8>(den[0]));
#pragma unroll
            for (int i = 0; i < NC; ++i)
#pragma unroll
                for (int r = 0; r < 4; ++r) o[i][r] = o[i][r] + (row_from<4>(o[i][r]) + row_from<8>(o[i][r]));
        }
        if constexpr (NH == 8) {
            den[0] += row_from<8>(den[0]);
#pragma unroll
            for (int i = 0; i < NC; ++i)
#pragma unroll
                for (int r = 0; r < 4; ++r) o[i][r] += row_from<8>(o[i][r]);
        }
    }
};

// The entries of a launch, query tokens of a sample `per` at a time: `count` of the
// call's from number `first` on.
struct Entries {
    BlockView view;
    const int32_t* top;  // [L, B, Hkv, T, k], null: all blocks
    int k, Hq, G, per, tiles, first, count;
    // sample and first query token of entry e of the launch
    __device__ __forceinline__ int sample(int e) const { return (first + e) / tiles; }
    __device__ __forceinline__ int token(int e) const { return (first + e) % tiles * per; }
};

// An entry as a lane holds it: the rows to go through, and those that its last query
// token sees.
struct Entry : Sequence {
    int seen;
};

__device__ __forceinline__ Entry entry_of(const PagePool& p, const Entries& n, int e) {
    if (e >= n.count) return Entry{{-1, 0}, 0};
    const int b = n.sample(e), t0 = n.token(e);
    const int slot = slot_of(n.view.seq, b, p.S);
    const int seen = seen_by(p, n.view, slot, b, min(t0 + n.per, n.view.T) - 1);
    return Entry{{slot, n.top == nullptr ? seen : seen > 0 ? n.k << p.shift : 0}, seen};
}

// Output row of row r (query token r / G of the entry, head r % G of the group).
__device__ __forceinline__ size_t row_at(const Entries& n, int l, int b, int j, int t0, int r) {
    const int t = r / n.G, h = r - t * n.G;
    return (((size_t)l * n.view.B + b) * n.Hq + (size_t)j * n.G + h) * n.view.T + t0 + t;
}

// One workgroup per split of an entry and (layer, KV head); its waves take 32
// tokens in turn.  Several: entries of more than one query token.  Bound by the loads:
// 8 sequences of 131072 tokens, 8 KV heads (2.1 GB) 323 us, 6.6 TB/s; without the
// non-temporal hint 387.  A short call is a chain of latencies: 4 sequences of 32 tokens
// 5.4 us, of 1639 11.0 with the merge, 30 to 40 KB to a compute unit.  For these the code
// is kept short, a loop over the steps that is not unrolled over the slots and no masks by
// query token where there is one: three and four slots, unrolled, lose up to a quarter
// (one sequence of 32768: 19 us with two, 24 with either).
template <typename T, int D, int NH, bool Several>
__global__ __launch_bounds__(kThreads, 2) void blocks_split(const T* __restrict__ q, PagePool p, Entries n, int share,
                                                            int level, int groups, int R, int whole, float sl2,
                                                            float* __restrict__ ws_o, float2* __restrict__ ws_ml,
                                                            SplitRange* __restrict__ ranges, float* __restrict__ out) {
    constexpr int NC = D / 16, NWV = kWaves;
    using S = Slot<D>;
    // the waves' rings, and behind their last use the waves' sums
    constexpr int kRing = S::kSlots * S::kBytes, kSums = NH * D * (int)sizeof(float);
    static_assert(kSums <= kRing, "a wave's sums fit its ring");
    __shared__ __attribute__((aligned(16))) char s_ring[NWV * kRing];
    __shared__ float s_ml[NWV][2][NH];
    float(*s_o)[NH][D] = reinterpret_cast<float(*)[NH][D]>(s_ring);

    const int pairs = p.L * p.Hkv;
    const int x = blockIdx.x / pairs, pair = blockIdx.x - x * pairs;
    const int l = pair / p.Hkv, j = pair - l * p.Hkv;
    const int lane = threadIdx.x & (kWave - 1);
    const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int c = lane & 15, quarter = lane >> 4;

    Work work{x, -1, 0, 0, {x, 1}};
    int seen_most;
    if (whole) {
        const Entry s = entry_of(p, n, x);
        work.slot = __builtin_amdgcn_readfirstlane(s.slot);
        work.k1 = __builtin_amdgcn_readfirstlane(s.tokens);
        seen_most = __builtin_amdgcn_readfirstlane(s.seen);
    } else {
        // up to 64 entries: looked up once, by the lane of their number
        const bool few = n.count <= kWave;
        Entry mine{{-1, 0}, 0};
        if (few) mine = entry_of(p, n, lane);
        auto of = [&](int e) -> Sequence { return few ? mine : entry_of(p, n, e); };
        int* staged = nullptr;
        if (!few) {
            static_assert(kPagesSlice * (int)sizeof(int) <= (int)sizeof(s_ring), "the lengths fit the rings");
            staged = reinterpret_cast<int*>(s_ring);
            for (int e = threadIdx.x; e < n.count; e += NWV * kWave) staged[e] = of(e).tokens;
            __syncthreads();
        }
        // the first workgroup's first wave leaves the ranges for the merge
        work = find_work(of, n.count, share, x, staged, blockIdx.x == 0 && wv == 0 ? ranges : nullptr,
                         level);
        if (staged != nullptr) __syncthreads();  // the rings take the lengths' place
        if (work.b < 0) return;
        seen_most = few ? __builtin_amdgcn_readlane(mine.seen, work.b)
                        : __builtin_amdgcn_readfirstlane(entry_of(p, n, work.b).seen);
    }
    const int slot = work.slot, k0 = work.k0, k1 = work.k1;
    const int b = n.sample(work.b), t0 = n.token(work.b);
    const int here = min(n.per, n.view.T - t0);  // query tokens of the entry
    const int rows = here * n.G;
    const int page = 1 << p.shift;

    // the lane's column: its query token, and the rows that it sees
    const int col = c & (NH - 1);
    const bool used = col < rows && c < (NH == 4 ? 12 : 16);
    const int tile = used ? col / n.G : -1;
    int seen = used ? seen_most : 0, seen_least = seen_most;
    if constexpr (Several) {
        if (used) seen = seen_by(p, n.view, slot, b, t0 + tile);
        seen_least = __builtin_amdgcn_readfirstlane(seen_by(p, n.view, slot, b, t0));
    }

    Sums<T, D, NH> sums;
    sums.start(used ? q + row_at(n, l, b, j, t0, col) * D : nullptr);

    // block numbers and page numbers of 64 places at a time, one per lane; a step's
    // tokens lie in one block.  A step whose block has no page loads page 0 and is
    // passed over.
    const int32_t* row = p.table + (size_t)max(slot, 0) * p.M;
    const int32_t* chosen = n.top != nullptr
        ? n.top + ((((size_t)l * n.view.B + b) * p.Hkv + j) * n.view.T + t0) * n.k : nullptr;
    const int places = chosen != nullptr ? n.k : p.M;
    const char* ring = s_ring + wv * kRing;
    int ids = 0, blks = 0, ids0 = -kWave;
    // loads 32 tokens into slot i; their first position, or seen_most: to be passed over
    auto issue = [&](int t, int i) -> int {
        const int at = t >> p.shift;
        if (at >= ids0 + kWave || ids0 < 0) {
            ids0 = at;
            const int place = min(at + lane, places - 1);
            blks = chosen != nullptr ? chosen[place] : place;
            const bool in = blks >= 0 && blks < p.M;
            ids = in ? row[blks] : -1;
            settle(ids);
            settle(blks);
        }
        const int pg = __builtin_amdgcn_readlane(ids, at - ids0), blk = __builtin_amdgcn_readlane(blks, at - ids0);
        const bool ok = pg >= 0 && pg < p.n_pages;
        const int tok = t & (page - 1);
        S::load(block_at<D>(p, l, ok ? pg : 0, j), tok, p.shift, ring + i * S::kBytes);
        return ok ? (blk << p.shift) + tok : seen_most;
    };
    constexpr int kStride = NWV * kBlk;
    static_assert(S::kSlots == 2, "a step's position and the next one's");
    int at0 = k0 + wv * kBlk, pos = 0, next = 0;
    sums.settle_queries();
    settle(seen);
    if (at0 < k1) pos = issue(at0, 0);
    if (at0 + kStride < k1) next = issue(at0 + kStride, 1);
#pragma unroll 1
    for (int i = 0; at0 < k1; at0 += kStride, i ^= 1) {
        // the slot's loads are the oldest: those of the other slot may be in flight
        if (at0 + kStride < k1)
            wait_vmcnt<S::kLoads>();
        else
            wait_vmcnt<0>();
        asm volatile("" ::: "memory");
        const int most = seen_most - pos;
        if (most > 0) {
            const char* slot_at = ring + i * S::kBytes;
            const uint32_t scales = *reinterpret_cast<const uint16_t*>(slot_at + 2 * S::kCodes);
            f32x4 acc[2];
            sums.logits(slot_at, scale_float(scale_of((uint8_t)scales)), acc);
            sums.template add<Several>(slot_at, scale_float(scale_of((uint8_t)(scales >> 8))), acc, seen - pos, most,
                                       seen_least == seen_most || seen_least - pos >= kBlk, tile, here, sl2);
        }
        pos = next;
        if (at0 + 2 * kStride < k1) {
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // the slot is read
            next = issue(at0 + 2 * kStride, i);
        }
    }
    sums.finish();

    __syncthreads();  // every wave is done with its ring
    if (c < rows) {
        if (quarter == 0) {
            s_ml[wv][0][c] = sums.m;
            s_ml[wv][1][c] = sums.den[0];
        }
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int i = 0; i < NC; ++i) s_o[wv][c][NC * (4 * quarter + r) + i] = sums.o[i][r];
    }
    __syncthreads();
    // merge the waves' partial results of this split
    for (int e = threadIdx.x; e < rows * D; e += NWV * kWave) {
        const int h = e / D, ch = e - h * D;
        float mx = kLowest;
#pragma unroll
        for (int w = 0; w < NWV; ++w) mx = fmaxf(mx, s_ml[w][0][h]);
        float lt = 0.0f, ot = 0.0f;
#pragma unroll
        for (int w = 0; w < NWV; ++w) {
            const float a = fast_exp2(s_ml[w][0][h] - mx);
            lt = fmaf(a, s_ml[w][1][h], lt);
            ot = fmaf(a, s_o[w][h][ch], ot);
        }
        if (work.range.count == 1) {  // the whole entry: the result itself
            out[row_at(n, l, b, j, t0, h) * D + ch] = lt != 0.0f ? ot / lt : 0.0f;
        } else {
            const size_t place = ((size_t)pair * groups + x) * R + h;
            ws_o[place * D + ch] = ot;
            if (ch == 0) ws_ml[place] = make_float2(mx, lt);
        }
    }
}

// Merge the splits of entries that have several, and write zeros for empty ones.
// Rows (layer, entry, KV head, row of the entry), kMergeWaves / WPR per workgroup.
template <int D, int WPR>
__global__ __launch_bounds__(kThreads) void blocks_merge(int Hkv, Entries n, int R, int groups,
                                                         const float* __restrict__ ws_o,
                                                         const float2* __restrict__ ws_ml,
                                                         const SplitRange* __restrict__ ranges, int n_rows,
                                                         float* __restrict__ out) {
    const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int row = blockIdx.x * (kWaves / WPR) + wv / WPR;
    if (row >= n_rows) return;  // WPR > 1: the whole workgroup
    const int seg = row / R, r = row - seg * R;
    const int le = seg / Hkv, j = seg - le * Hkv;
    const int l = le / n.count, e = le - l * n.count;
    const int b = n.sample(e), t0 = n.token(e);
    if (r >= min(n.per, n.view.T - t0) * n.G) return;
    const SplitRange range = ranges[e];
    if (range.count == 1) return;  // written by its only split
    const size_t base = (((size_t)l * Hkv + j) * groups + range.first) * R + r;
    merge_row<D, WPR, true>(ws_o + base * D, ws_ml + base, R, range.count, true,
                            out + row_at(n, l, b, j, t0, r) * D);
}

template <typename T, int D, int NH>
hipError_t run_columns(const void* q, const PagePool& p, const Entries& call, const BlocksPlan& plan, float scale,
                       float* out, void* ws, hipStream_t st) {
    float* wo = static_cast<float*>(ws);
    float2* wml = reinterpret_cast<float2*>(static_cast<char*>(ws) + plan.off_ml);
    SplitRange* ranges = reinterpret_cast<SplitRange*>(static_cast<char*>(ws) + plan.off_ranges);
    for (Entries n = call; n.first < plan.entries; n.first += plan.slice) {
        n.count = min(plan.slice, plan.entries - n.first);
        auto launch = [&](auto kernel) {
            hipLaunchKernelGGL(kernel, dim3((unsigned)plan.pairs * plan.groups), dim3(kThreads), 0, st,
                               static_cast<const T*>(q), p, n, plan.share, plan.level, plan.groups, plan.R,
                               (int)plan.whole, scale * kLog2e, wo, wml, ranges, out);
        };
        if (plan.per > 1)
            launch(blocks_split<T, D, NH, true>);
        else
            launch(blocks_split<T, D, NH, false>);
        // up to 16 splits of a level entry: one wave per row; more: four, as over four-bit pages.
        // Ragged ones may have four times as many and leave it open which is better (8 KV heads,
        // microseconds with one wave and with four: two layers, one sequence of 131072 among 8
        // of 500 92.8 and 91.5, of 64 channels 51.5 and 50.0, one of 32768 among 16 39.6 and 38.9,
        // one of 40000 among 64 of 700 40.7 and 42.3, 16 of up to 32768 185.7 and 187.3, eight
        // layers 662.7 and 665.6; level, 16 of 8192, 84.8 and 85.1).
        const int rows = plan.pairs * n.count * plan.R;
        if (!plan.whole && plan.level > 16)
            hipLaunchKernelGGL((blocks_merge<D, kWaves>), dim3((unsigned)rows), dim3(kThreads), 0, st, p.Hkv, n, plan.R,
                               plan.groups, wo, wml, ranges, rows, out);
        else if (!plan.whole)
            hipLaunchKernelGGL((blocks_merge<D, 1>), dim3((unsigned)((rows + kWaves - 1) / kWaves)), dim3(kThreads), 0,
                               st, p.Hkv, n, plan.R, plan.groups, wo, wml, ranges, rows, out);
    }
    return hipGetLastError();
}

template <typename T, int D>
hipError_t run(const void* q, const PagePool& p, const Entries& n, const BlocksPlan& plan, float scale, float* out,
               void* ws, hipStream_t st) {
    if (plan.R <= 4) return run_columns<T, D, 4>(q, p, n, plan, scale, out, ws, st);
    if (plan.R <= 8) return run_columns<T, D, 8>(q, p, n, plan, scale, out, ws, st);
    return run_columns<T, D, kPagesMaxGroup>(q, p, n, plan, scale, out, ws, st);
}

}  // namespace

hipError_t launch_decode_blocks(const void* q, int dtype, const PagePool& p, int d, const BlockView& view, int Hq,
                                const int32_t* top, int k, float scale, float* out, void* ws, hipStream_t st) {
    const long long tokens = top != nullptr ? (long long)k << p.shift : view.max_tokens;
    const BlocksPlan plan = decode_blocks_plan(p.L, view.B, Hq, p.Hkv, view.T, tokens, top != nullptr, d);
    const Entries n{view, top, k, Hq, plan.G, plan.per, plan.tiles, 0, 0};
    if (dtype == 0) {
        if (d == 128) return run<__bf16, 128>(q, p, n, plan, scale, out, ws, st);
        return run<__bf16, 64>(q, p, n, plan, scale, out, ws, st);
    }
    if (d == 128) return run<float, 128>(q, p, n, plan, scale, out, ws, st);
    return run<float, 64>(q, p, n, plan, scale, out, ws, st);
}

}  // namespace kve
