// The choice of blocks for block-sparse attention (kve_blocks_top): a score for each
// block from the bounds of its keys, and the k highest for each query token.
//
// With up and down the sums over the group's heads of max(q, 0) and min(q, 0) a
// block's score is <up, hi> + <down, lo>: two products of d channels whatever the
// number of heads, which is why the kernel reads 2 d bytes per block and does little
// else.  They are summed in 64 bits, so that the order of the sum does not decide
// which of two blocks is chosen.
#include "kve_blocks_device.h"
#include "kve_device.h"
#include "kve_internal.h"

namespace kve {
namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / kWave;
constexpr int kScored = 64;              // blocks per workgroup of top_scores
constexpr uint32_t kForced = 0xffffffffu;  // key of the first and last blocks: above every score's

// What a call chooses.
struct TopGrid {
    BlockView view;
    int Hq, G, k, first, last, most;  // most: blocks that max_tokens can lie in
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

// Keys of kScored blocks of a segment.  D / 8 lanes to a block, eight channels of
// both bounds each.
template <typename T, int D>
__global__ __launch_bounds__(kThreads) void top_scores(const T* __restrict__ q, PagePool p, TopGrid g, int chunks,
                                                       uint32_t* __restrict__ keys) {
    constexpr int kRow = D / 8, kStep = kThreads / kRow;
    const unsigned seg = blockIdx.x / (unsigned)chunks;
    const int chunk = (int)(blockIdx.x - seg * chunks);
    const Segment x = segment_of(p, g, seg);
    if (x.blocks <= g.k || chunk * kScored >= x.blocks) return;  // all are taken, or none here
    const int part = threadIdx.x % kRow, in = threadIdx.x / kRow;
    double up[8], down[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) up[e] = down[e] = 0.0;
    const T* rows = q + ((((size_t)x.l * g.view.B + x.b) * g.Hq + (size_t)x.j * g.G) * g.view.T + x.t) * D + 8 * part;
#pragma unroll 1
    for (int h = 0; h < g.G; ++h)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const double y = (double)(float)rows[(size_t)h * g.view.T * D + e];
            up[e] += y < 0.0 ? 0.0 : y;
            down[e] += y > 0.0 ? 0.0 : y;
        }
#pragma unroll 1
    for (int i = 0; i < kScored; i += kStep) {
        const int at = chunk * kScored + i + in;
        const bool there = at < x.blocks;
        const int pg = there ? p.table[(size_t)x.slot * p.M + at] : -1;
        const bool ok = pg >= 0 && pg < p.n_pages;
        double sum = 0.0;
        float unit = 0.0f;
        if (ok) {
            const char* tail = block_at<D>(p, x.l, pg, x.j) + tail_at<D>(p.shift);
            const u32x2 lo = reinterpret_cast<const u32x2*>(tail + kBlockScales)[part];
            const u32x2 hi = reinterpret_cast<const u32x2*>(tail + kBlockScales + D)[part];
            unit = scale_float(scale_of((uint8_t)tail[0]));
#pragma unroll
            for (int w = 0; w < 2; ++w) {
                float a[4], c[4];
                floats4(lo[w], 1.0f, a);
                floats4(hi[w], 1.0f, c);
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    sum = fma(up[4 * w + e], (double)c[e], fma(down[4 * w + e], (double)a[e], sum));
            }
        }
#pragma unroll
        for (int s = 1; s < kRow; s <<= 1) sum += __shfl_xor(sum, s);
        if (part == 0 && there) {
            const bool forced = at < g.first || at >= x.blocks - g.last;
            keys[(size_t)seg * g.most + at] = forced ? kForced : ok ? score_key((float)(sum * (double)unit)) : 0u;
        }
    }
}

// Sum over the threads before, and over all in `total`.  s: kWaves words of LDS.
__device__ __forceinline__ uint32_t scan(uint32_t x, uint32_t* s, uint32_t& total) {
    const int lane = threadIdx.x & (kWave - 1), w = threadIdx.x / kWave;
    uint32_t inc = x;
#pragma unroll
    for (int d = 1; d < kWave; d <<= 1) {
        const uint32_t y = (uint32_t)__shfl_up((int)inc, d);
        inc += lane >= d ? y : 0u;
    }
    __syncthreads();
    if (lane == kWave - 1) s[w] = inc;
    __syncthreads();
    uint32_t before = 0;
    total = 0;
#pragma unroll
    for (int e = 0; e < kWaves; ++e) {
        before += e < w ? s[e] : 0u;
        total += s[e];
    }
    return before + inc - x;
}

// One workgroup per segment: the k-th highest key digit by digit, then the blocks
// above it and the first of those equal to it in ascending order.
__global__ __launch_bounds__(kThreads) void top_select(PagePool p, TopGrid g, const uint32_t* __restrict__ keys,
                                                       int32_t* __restrict__ top) {
    __shared__ uint32_t s_hist[256], s_scan[kWaves], s_pick[2];
    const unsigned seg = blockIdx.x;
    const Segment x = segment_of(p, g, seg);
    int32_t* out = top + (size_t)seg * g.k;
    const int n = x.blocks;
    if (n <= g.k) {
        for (int i = threadIdx.x; i < g.k; i += kThreads) out[i] = i < n ? i : -1;
        return;
    }
    const uint32_t* key = keys + (size_t)seg * g.most;
    uint32_t prefix = 0, want = (uint32_t)g.k;  // of the keys that share the prefix, the want-th highest
    for (int shift = 24; shift >= 0; shift -= 8) {
        s_hist[threadIdx.x] = 0;
        __syncthreads();
        for (int i = threadIdx.x; i < n; i += kThreads) {
            const uint32_t y = key[i];
            if (shift == 24 || (y >> (shift + 8)) == prefix) atomicAdd(&s_hist[(y >> shift) & 255u], 1u);
        }
        __syncthreads();
        // thread e: digit 255 - e, the counts above it
        const uint32_t mine = s_hist[255 - threadIdx.x];
        uint32_t total;
        const uint32_t above = scan(mine, s_scan, total);
        if (above < want && above + mine >= want) {
            s_pick[0] = 255u - threadIdx.x;
            s_pick[1] = want - above;
        }
        __syncthreads();
        prefix = prefix << 8 | s_pick[0];
        want = s_pick[1];
    }
    // in ascending order: keys above the prefix, and the first `want` equal to it
    uint32_t placed = 0, equal = 0;
    for (int i0 = 0; i0 < n; i0 += kThreads) {
        const int i = i0 + (int)threadIdx.x;
        const uint32_t y = i < n ? key[i] : 0u;
        const bool same = i < n && y == prefix;
        uint32_t sames, takes;
        const uint32_t rank = scan(same ? 1u : 0u, s_scan, sames);
        const bool take = i < n && (y > prefix || (same && equal + rank < want));
        const uint32_t at = scan(take ? 1u : 0u, s_scan, takes);
        if (take) out[placed + at] = i;
        placed += takes;
        equal += sames;
    }
}

}  // namespace

hipError_t launch_blocks_top(const void* q, int dtype, const PagePool& p, int d, const BlockView& view, int Hq, int k,
                             int first, int last, int32_t* top, void* ws, hipStream_t st) {
    const TopGrid g{view, Hq, Hq / p.Hkv, k, first, last, top_blocks(view.max_tokens, 1 << p.shift)};
    const unsigned segs = (unsigned)p.L * view.B * p.Hkv * view.T;
    uint32_t* keys = static_cast<uint32_t*>(ws);
    if (g.most > k) {
        const int chunks = (g.most + kScored - 1) / kScored;
        const dim3 grid(segs * (unsigned)chunks), block(kThreads);
        if (dtype == 0 && d == 128)
            hipLaunchKernelGGL((top_scores<__bf16, 128>), grid, block, 0, st, static_cast<const __bf16*>(q), p, g,
                               chunks, keys);
        if (dtype == 0 && d == 64)
            hipLaunchKernelGGL((top_scores<__bf16, 64>), grid, block, 0, st, static_cast<const __bf16*>(q), p, g,
                               chunks, keys);
        if (dtype == 1 && d == 128)
            hipLaunchKernelGGL((top_scores<float, 128>), grid, block, 0, st, static_cast<const float*>(q), p, g,
                               chunks, keys);
        if (dtype == 1 && d == 64)
            hipLaunchKernelGGL((top_scores<float, 64>), grid, block, 0, st, static_cast<const float*>(q), p, g,
                               chunks, keys);
    }
    hipLaunchKernelGGL(top_select, dim3(segs), dim3(kThreads), 0, st, p, g, keys, top);
    return hipGetLastError();
}

}  // namespace kve
