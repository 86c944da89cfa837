// The choice of blocks for block-sparse attention (kve_blocks_top): a score for each
// block from the bounds of its keys, and the k highest for each query token.
//
// With up and down the sums over the group's heads of max(q, 0) and min(q, 0) a
// block's score is <up, hi> + <down, lo>: two products of d channels whatever the
// number of heads.  They are summed in 64 bits, so that the order of the sum does not
// decide which of two blocks is chosen.
#include <algorithm>
#include <type_traits>

#include "kve_blocks_device.h"
#include "kve_device.h"
#include "kve_internal.h"

namespace kve {
namespace {

constexpr int kThreads = 256;
constexpr int kScored = 64;              // blocks per workgroup of top_scores,
constexpr int kTokens = 4;               // and query tokens that share its read of their bounds
// Workgroups from which each takes more blocks, up to eight times as many: 16 sequences
// of 4096 blocks 46, 50 and 49 us for 1024, 2048 and 4096; of up to that many 36, 29 and
// 30, with two query tokens of 3125 47, 37 and 43.  The first blocks of all sequences come
// first, so that workgroups without blocks are the last ones (sequence after sequence:
// the first two 50 and 35 for 2048, the third 33).
constexpr int kScoreGroups = 2048, kMostTiles = 8;

template <int N>
using Int = std::integral_constant<int, N>;

// What a call chooses.
struct TopGrid {
    BlockView view;
    int Hq, G, k, first, last, pitch;  // pitch: keys of a segment in the workspace
};

struct Segment {
    int l, b, j, t, slot, blocks;  // blocks: that hold rows which the token sees
};

// Segment (l, b, j, t) of index s, in that order.
__device__ __forceinline__ Segment segment_of(const PagePool& p, const TopGrid& g, unsigned s) {
    Segment x;
    const unsigned lbj = s / (unsigned)g.view.T, lb = lbj / (unsigned)p.Hkv;
    x.t = (int)(s - lbj * g.view.T);
    x.j = (int)(lbj - lb * p.Hkv);
    x.l = (int)(lb / (unsigned)g.view.B);
    x.b = (int)(lb - (unsigned)x.l * g.view.B);
    x.slot = slot_of(g.view.seq, x.b, p.S);
    x.blocks = (int)(((long long)seen_by(p, g.view, x.slot, x.b, x.t) + (1 << p.shift) - 1) >> p.shift);
    return x;
}

// x of the lane that a step of a sum over sixteen lanes adds.
template <int CTRL>
__device__ __forceinline__ double row_move(double x) {
    const uint64_t bits = __builtin_bit_cast(uint64_t, x);
    const uint32_t lo = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)bits, CTRL, 0xf, 0xf, false);
    const uint32_t hi = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)(bits >> 32), CTRL, 0xf, 0xf, false);
    return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}

// Sum over the LANES lanes (4 or 8) of a block, in every lane.
template <int LANES>
__device__ __forceinline__ double row_sum(double x) {
    x += row_move<0xb1>(x);  // lanes 1 0 3 2
    x += row_move<0x4e>(x);  // lanes 2 3 0 1
    if constexpr (LANES == 8) x += row_move<0x141>(x);  // mirrored within eight
    return x;
}

// Code K of a dword as a double times 2^-1016, but NaN codes as +-480: an E4M3's bits,
// denormal or not, are the top bits of a double's exponent and mantissa as they are.
// Three full-rate instructions, where the conversions from float take a quarter of the rate.
template <int K>
__device__ __forceinline__ double tiny(uint32_t w) {
    const int top = (int)(w << (24 - 8 * K)) >> 7;
    return __builtin_bit_cast(double, (uint64_t)((uint32_t)top & 0x80fe0000u) << 32);
}
constexpr double kUp = 0x1p800, kDown = 0x1p216;  // what brings products of such doubles back to scale, in two steps

template <int W>
__device__ __forceinline__ double add4(const double (&up)[16], const double (&down)[16], uint32_t lo, uint32_t hi,
                                       double sum) {
    sum = fma(up[4 * W], tiny<0>(hi), fma(down[4 * W], tiny<0>(lo), sum));
    sum = fma(up[4 * W + 1], tiny<1>(hi), fma(down[4 * W + 1], tiny<1>(lo), sum));
    sum = fma(up[4 * W + 2], tiny<2>(hi), fma(down[4 * W + 2], tiny<2>(lo), sum));
    return fma(up[4 * W + 3], tiny<3>(hi), fma(down[4 * W + 3], tiny<3>(lo), sum));
}

// What a lane holds of kItems blocks: sixteen channels of both bounds.
template <int D>
struct Bounds {
    static constexpr int kRow = D / 16, kStep = kThreads / kRow, kItems = kScored / kStep;
    u32x4 lo[kItems], hi[kItems];
    uint8_t unit[kItems];
    __device__ __forceinline__ static void pages(const PagePool& p, const Segment& x, int first, int (&page)[kItems]) {
#pragma unroll
        for (int i = 0; i < kItems; ++i) {
            const int at = first + i * kStep + (int)threadIdx.x / kRow;
            page[i] = at < x.blocks ? p.table[(size_t)x.slot * p.M + at] : -1;
        }
    }
    __device__ __forceinline__ void load(const PagePool& p, const Segment& x, const int (&page)[kItems]) {
        const int part = threadIdx.x % kRow;
#pragma unroll
        for (int i = 0; i < kItems; ++i) {
            // a block without a page: any page's bounds, and not their score
            const int pg = page[i] >= 0 && page[i] < p.n_pages ? page[i] : 0;
            const char* tail = block_at<D>(p, x.l, pg, x.j) + tail_at<D>(p.shift);
            lo[i] = ld16(tail + kBlockScales + 16 * part);
            hi[i] = ld16(tail + kBlockScales + D + 16 * part);
            unit[i] = (uint8_t)tail[0];
        }
    }
    // the keys of a query token
    __device__ __forceinline__ void score(const PagePool& p, const Segment& x, int first, const int (&page)[kItems],
                                          const double (&up)[16], const double (&down)[16], uint32_t* keys) const {
#pragma unroll
        for (int i = 0; i < kItems; ++i) {
            // two chains, which hide each other's latency
            double sum = add4<1>(up, down, lo[i][1], hi[i][1], add4<0>(up, down, lo[i][0], hi[i][0], 0.0)) +
                         add4<3>(up, down, lo[i][3], hi[i][3], add4<2>(up, down, lo[i][2], hi[i][2], 0.0));
            uint32_t bad = 0;
#pragma unroll
            for (int w = 0; w < 4; ++w) bad |= nan_codes(lo[i][w]) | nan_codes(hi[i][w]);
            if (bad != 0) sum = __builtin_nan("");
            sum = row_sum<kRow>(sum);
            const int at = first + i * kStep + (int)threadIdx.x / kRow;
            if (threadIdx.x % kRow == 0 && at < x.blocks) {
                const bool ok = page[i] >= 0 && page[i] < p.n_pages;
                const double score = sum * kDown * (double)scale_float(scale_of(unit[i]));
                keys[at] = ok ? score_key((float)score) : 0u;
            }
        }
    }
};

// Keys of `tiles` times kScored blocks of a (layer, sample, KV head) for up to TOKENS
// query tokens.  The next tile's bounds, and the page numbers of the one after it, are
// on their way while a tile is scored.  16 sequences of 4096 blocks, 8 KV heads: 42 us for
// three lines of 128 bytes to a block, 4.8 TB/s; the sums take half of that beside it
// (two query tokens for one, 3125 blocks: 54 us and 41, the choice included).  Small calls
// are latency: 4.8 us for one sequence of 1024 blocks.
template <typename T, int D, int TOKENS>
__global__ __launch_bounds__(kThreads) void top_scores(const T* __restrict__ q, PagePool p, TopGrid g, int sets,
                                                       int tiles, int groups, uint32_t* __restrict__ keys) {
    using B = Bounds<D>;
    // channels 2 e, 2 e + 1 of every sixteen, side by side
    __shared__ __attribute__((aligned(16))) double s_up[TOKENS][2][8][B::kRow][2];
    const unsigned chunk = blockIdx.x / (unsigned)sets, y = blockIdx.x - chunk * sets, lbj = y / (unsigned)groups;
    const int first = (int)chunk * tiles * kScored, t0 = (int)(y - lbj * groups) * TOKENS;
    const int tokens = min(TOKENS, g.view.T - t0);
    const Segment x = segment_of(p, g, lbj * (unsigned)g.view.T + (t0 + tokens - 1));  // the token that sees most
    if (x.blocks <= g.k || first >= x.blocks) return;  // all are taken, or none here
    const int end = min(x.blocks, first + tiles * kScored);
    int now[B::kItems], next[B::kItems], then[B::kItems];
    B::pages(p, x, first, now);
    B::pages(p, x, first + kScored, next);
    // the heads' sums: a thread to each channel of either
    if (threadIdx.x < 2 * D) {
        const int c = threadIdx.x % D;
        const bool lower = threadIdx.x >= D;
        const T* row = q + ((((size_t)x.l * g.view.B + x.b) * g.Hq + (size_t)x.j * g.G) * g.view.T + t0) * D + c;
#pragma unroll 1
        for (int t = 0; t < tokens; ++t, row += D) {
            double sum = 0.0;
#pragma unroll 8
            for (int h = 0; h < g.G; ++h) {
                const float z = (float)row[(size_t)h * g.view.T * D];
                sum += (lower ? z > 0.0f : z < 0.0f) ? 0.0 : (double)z;
            }
            s_up[t][lower][c % 16 / 2][c / 16][c % 2] = sum * kUp;
        }
    }
    B mine;
    mine.load(p, x, now);
    __syncthreads();
    const int part = threadIdx.x % B::kRow;
    double up[16], down[16];
    auto token = [&](int t) {
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            up[e] = s_up[t][0][e / 2][part][e % 2];
            down[e] = s_up[t][1][e / 2][part][e % 2];
        }
    };
    if constexpr (TOKENS == 1) token(0);
#pragma unroll 1
    for (int at = first; at < end; at += kScored) {
        B ahead;
        ahead.load(p, x, next);
        B::pages(p, x, at + 2 * kScored, then);
        if constexpr (TOKENS == 1) {
            mine.score(p, x, at, now, up, down, keys + (size_t)(lbj * (unsigned)g.view.T + t0) * g.pitch);
        } else {
#pragma unroll 1
            for (int t = 0; t < tokens; ++t) {
                token(t);
                // the codes as doubles are made again for each token: held, they would leave two
                // waves to a compute unit's quarter
#pragma unroll
                for (int i = 0; i < B::kItems; ++i) {
                    asm volatile("" : "+v"(mine.lo[i]));
                    asm volatile("" : "+v"(mine.hi[i]));
                }
                mine.score(p, x, at, now, up, down, keys + (size_t)(lbj * (unsigned)g.view.T + t0 + t) * g.pitch);
            }
        }
        mine = ahead;
#pragma unroll
        for (int i = 0; i < B::kItems; ++i) {
            now[i] = next[i];
            next[i] = then[i];
        }
    }
}

// Exclusive sum over the threads of a workgroup of WAVES waves, and over all in `total`.
// s: WAVES words of LDS, free again behind the next barrier.
template <int WAVES>
__device__ __forceinline__ uint32_t scan(uint32_t x, uint32_t* s, uint32_t& total) {
    const int lane = threadIdx.x & (kWave - 1), w = threadIdx.x / kWave;
    auto step = [](uint32_t v, auto ctrl, auto rows) {
        return v + (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, decltype(ctrl)::value, decltype(rows)::value, 0xf,
                                                         false);
    };
    auto wave = [&](uint32_t v) {
        v = step(v, Int<0x111>{}, Int<0xf>{});
        v = step(v, Int<0x112>{}, Int<0xf>{});
        v = step(v, Int<0x114>{}, Int<0xf>{});
        v = step(v, Int<0x118>{}, Int<0xf>{});
        v = step(v, Int<0x142>{}, Int<0xa>{});
        return step(v, Int<0x143>{}, Int<0xc>{});
    };
    const uint32_t inc = wave(x);
    if (lane == kWave - 1) s[w] = inc;
    __syncthreads();
    const uint32_t sums = wave(lane < WAVES ? s[lane] : 0u);
    total = (uint32_t)__builtin_amdgcn_readlane((int)sums, WAVES - 1);
    const int last = __builtin_amdgcn_readfirstlane(w) - 1;  // the wave before
    const uint32_t before = last >= 0 ? (uint32_t)__builtin_amdgcn_readlane((int)sums, last) : 0u;
    return before + inc - x;
}

// One workgroup per segment.  The blocks that are not forced compete for the places
// that the forced ones leave: the lowest key that gets one is found in digits of BITS
// bits, from the highest bit in which the keys differ on (keys of one sign and a few
// binades, as scores are, spread over the digits of the first pass, and the counts in
// LDS do not collide), until all that share its digits get one.  4096 blocks: 6 us; with
// digits of 8 bits from the top one, 256 threads and the keys loaded again for each, 25.
template <int THREADS, int BITS>
__global__ __launch_bounds__(THREADS) void top_select(PagePool p, TopGrid g, const uint32_t* __restrict__ keys,
                                                      int32_t* __restrict__ top) {
    constexpr int kWaves = THREADS / kWave, kBins = 1 << BITS, kOwn = kBins / THREADS, kTile = 4 * THREADS;
    __shared__ uint32_t s_hist[kBins], s_scan[2][kWaves], s_ends[2][kWaves], s_pick[3];
    const unsigned seg = blockIdx.x;
    const Segment x = segment_of(p, g, seg);
    int32_t* out = top + (size_t)seg * g.k;
    const int n = x.blocks, tid = threadIdx.x;
    if (n <= g.k) {
        for (int i = tid; i < g.k; i += THREADS) out[i] = i < n ? i : -1;
        return;
    }
    const uint32_t* key = keys + (size_t)seg * g.pitch;
    const int open0 = g.first, open1 = n - g.last;  // blocks that compete
    uint32_t want = (uint32_t)(g.k - g.first - g.last);
    // four neighbouring keys of a tile; the first tile is loaded once
    const u32x4 mine = tid * 4 < n ? *reinterpret_cast<const u32x4*>(key + tid * 4) : zero16();
    auto load = [&](int i0) {
        if (i0 == 0) return mine;
        return i0 + tid * 4 < n ? *reinterpret_cast<const u32x4*>(key + i0 + tid * 4) : zero16();
    };
    auto each = [&](auto&& body) {
        for (int i0 = 0; i0 < n; i0 += kTile) {
            const u32x4 y = load(i0);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int i = i0 + tid * 4 + e;
                if (i >= open0 && i < open1) body(y[e]);
            }
        }
    };
    for (int i = tid; i < kBins; i += THREADS) s_hist[i] = 0;
    uint32_t least = 0xffffffffu, most = 0;
    each([&](uint32_t y) {
        least = min(least, y);
        most = max(most, y);
    });
#pragma unroll
    for (int d = 1; d < kWave; d <<= 1) {
        least = min(least, (uint32_t)__shfl_xor((int)least, d));
        most = max(most, (uint32_t)__shfl_xor((int)most, d));
    }
    const int lane = tid & (kWave - 1);
    if (lane == 0) {
        s_ends[0][tid / kWave] = least;
        s_ends[1][tid / kWave] = most;
    }
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
        least = min(least, s_ends[0][w]);
        most = max(most, s_ends[1][w]);
    }
    // `prefix`: the bits from `shift` on of the lowest key that gets a place
    int shift = least < most ? 32 - __builtin_clz(least ^ most) : 0;
    uint32_t prefix = shift < 32 ? most >> shift : 0u;
    bool done = want == 0 || shift == 0;
    while (!done) {
        const int low = max(0, shift - BITS), bits = shift - low;
        each([&](uint32_t y) {
            if (shift == 32 || y >> shift == prefix) atomicAdd(&s_hist[(y >> low) & ((1u << bits) - 1)], 1u);
        });
        __syncthreads();
        // thread e: kOwn digits, from kBins - 1 - kOwn e downwards
        uint32_t* own = s_hist + kBins - kOwn * (tid + 1);
        uint32_t counts[kOwn], sum = 0;
#pragma unroll
        for (int i = 0; i < kOwn; ++i) {
            counts[i] = own[kOwn - 1 - i];
            sum += counts[i];
        }
        uint32_t total, above = scan<kWaves>(sum, s_scan[0], total);
#pragma unroll
        for (int i = 0; i < kOwn; ++i) {
            if (above < want && above + counts[i] >= want) {
                s_pick[0] = (uint32_t)(kBins - 1 - kOwn * tid - i);
                s_pick[1] = want - above;
                s_pick[2] = counts[i];
            }
            above += counts[i];
            own[i] = 0;  // the next pass counts from zero
        }
        __syncthreads();
        prefix = prefix << bits | s_pick[0];
        want = s_pick[1];
        shift = low;
        done = low == 0 || s_pick[2] == want;
        if (!done) __syncthreads();  // s_pick and s_scan are read
    }
    // in ascending order: forced ones, keys above the prefix, and the first `want` that
    // have it; both are counted in one sum, 16 bits each per tile
    uint32_t placed = 0, equal = 0;
    for (int i0 = 0, turn = 0; i0 < n; i0 += kTile, turn ^= 1) {
        const u32x4 y = load(i0);
        uint32_t own = 0;
        bool take[4], same[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int i = i0 + tid * 4 + e;
            const bool competes = i >= open0 && i < open1;
            const uint32_t h = shift < 32 ? y[e] >> shift : 0u;
            take[e] = i < n && (!competes || h > prefix);
            same[e] = competes && h == prefix;
            own += (take[e] ? 1u : 0u) + (same[e] ? 0x10000u : 0u);
        }
        uint32_t total;
        const uint32_t before = scan<kWaves>(own, s_scan[turn], total);
        uint32_t at = placed + (before & 0xffffu), ties = equal + (before >> 16);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const bool in = same[e] && ties < want;
            if (take[e] || in) out[at + min(ties, want)] = i0 + tid * 4 + e;
            at += take[e] ? 1u : 0u;
            ties += same[e] ? 1u : 0u;
        }
        placed += total & 0xffffu;
        equal += total >> 16;
    }
}

}  // namespace

hipError_t launch_blocks_top(const void* q, int dtype, const PagePool& p, int d, const BlockView& view, int Hq, int k,
                             int first, int last, int32_t* top, void* ws, hipStream_t st) {
    const int most = top_blocks(view.max_tokens, 1 << p.shift);
    const TopGrid g{view, Hq, Hq / p.Hkv, k, first, last, top_pitch(most)};
    const unsigned segs = (unsigned)p.L * view.B * p.Hkv * view.T;
    uint32_t* keys = static_cast<uint32_t*>(ws);
    if (most > k) {
        const int tokens = view.T == 1 ? 1 : kTokens, groups = (view.T + tokens - 1) / tokens;
        const int all = (most + kScored - 1) / kScored;
        const long long pairs = (long long)p.L * view.B * p.Hkv * groups;
        const int tiles = (int)std::min(std::max(pairs * all / kScoreGroups, 1LL), (long long)kMostTiles);
        const int chunks = (all + tiles - 1) / tiles;
        auto launch = [&](auto kernel, auto rows) {
            hipLaunchKernelGGL(kernel, dim3((unsigned)(pairs * chunks)), dim3(kThreads), 0, st, rows, p, g, (int)pairs,
                               tiles, groups, keys);
        };
        auto by_size = [&](auto rows) {
            using T = std::remove_const_t<std::remove_pointer_t<decltype(rows)>>;
            if (tokens == 1)
                launch(d == 128 ? top_scores<T, 128, 1> : top_scores<T, 64, 1>, rows);
            else
                launch(d == 128 ? top_scores<T, 128, kTokens> : top_scores<T, 64, kTokens>, rows);
        };
        if (dtype == 0)
            by_size(static_cast<const __bf16*>(q));
        else
            by_size(static_cast<const float*>(q));
    }
    // as few threads as hold a segment with four keys each: one sequence of 1024 blocks, 8
    // segments, 8.6 us with 256 threads, 9.9 with 1024, scores included, 64 of 128 blocks
    // 13.0 and 16.2; 16 of 2048 blocks 29.5 with 512, 30.2 with 1024; in two tiles they lose
    // (4 of 4096 blocks, 2 KV heads: 13.2 with 512, 12.7 with 1024)
    auto select = [&](auto threads, auto bits) {
        constexpr int kThreadsOf = decltype(threads)::value;
        hipLaunchKernelGGL((top_select<kThreadsOf, decltype(bits)::value>), dim3(segs), dim3(kThreadsOf), 0, st, p, g,
                           keys, top);
    };
    if (g.pitch <= 4 * 256)
        select(Int<256>{}, Int<10>{});
    else if (g.pitch <= 4 * 512)
        select(Int<512>{}, Int<11>{});
    else
        select(Int<1024>{}, Int<11>{});
    return hipGetLastError();
}

}  // namespace kve
