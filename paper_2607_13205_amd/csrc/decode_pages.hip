// Decode attention over paged 4-bit sequences: one query per head attends to the
// rows of its sequence through the page table (kve_decode_pages).
//
// The four-bit values times their power of two are exact in bf16, so both
// products run on the bf16 matrix instructions without an error beyond float32
// sums: bf16 queries are one operand as they are, float32 queries and the softmax
// weights three bf16 parts that add up to them (truncation leaves 8 bits per part).
//
// Both products are taken transposed, so that the weights never leave their
// registers.  A wave takes 32 tokens per step.  S^T = K Q^T, 16 tokens by 16 query
// heads per 16x16x32 product: row m of tile T is token 16 T + 4 (m % 4) + m / 4,
// and lane l (head l % 16, quarter q = l / 16) receives rows 4 q .. + 4, that is
// tokens 4 i + q, i < 8, from its two tiles.  Those are what the second product
// O^T = V^T P^T wants from that lane.  The value rows' dwords hold eight channels
// of one token and the product eight tokens of one channel: the scaled conversion
// gives two channels of a token, and a byte permutation pairs the tokens.
//
// The bytes of a step go straight to LDS, into the wave's own ring of slots, two
// steps ahead and without a register held for them; four workgroups share a
// compute unit.
//
// With up to four heads per KV head the sixteen columns hold every head three
// times, and each copy's lanes make another of the three parts of the weights: a
// third of the second products, and fewer vector instructions, which are what
// bounds the kernel beside the loads.  With up to eight they hold every head
// twice: the first copy takes the top and the last part, the second the middle one.
//
// Split-K and the lazy softmax reference are those of the dense decode
// (decode.hip): weights are exp2(x - m) with m raised only when a logit exceeds it
// by more than kRaise.  The denominators are one more row of the second product, a
// row of ones.
#include <type_traits>

#include "kve_decode_merge.h"
#include "kve_decode_split.h"
#include "kve_device.h"
#include "kve_internal.h"
#include "kve_pages_device.h"
#include "kve_stream.h"

namespace kve {
namespace {

constexpr int kThreads = kMergeThreads;
constexpr int kWaves = kThreads / kWave;
constexpr int kBlk = 32;    // tokens per wave step

// Waves per SIMD that the registers are kept to, and so workgroups per compute
// unit: four where the registers suffice without spills (8 layers, 4 sequences of
// 8192: float32 queries 60 us at three and 70 at four, 16 heads per KV head 64.5
// and 67).
template <typename T, int D, int NH>
constexpr int kPerSimd = D == 128 && (std::is_same<T, float>::value || NH > 8) ? 3 : 4;

// Eight codes of a dword as bf16.
__device__ __forceinline__ bf16x8 unpack8(uint32_t w, float scale) {
    u32x4 r;
    r[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 0));
    r[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 1));
    r[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 2));
    r[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 3));
    return __builtin_bit_cast(bf16x8, r);
}

// Byte `sel` of eight dwords as bf16 pairs (two channels of a token each),
// regrouped into the eight tokens of either channel.
template <int SEL>
__device__ __forceinline__ void unpack_tokens(const uint32_t (&w)[8], const float (&scale)[8], bf16x8& even,
                                              bf16x8& odd) {
    uint32_t c[8];
#pragma unroll
    for (int i = 0; i < 8; ++i)
        c[i] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[i], scale[i], SEL));
    u32x4 e, o;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        e[i] = __builtin_amdgcn_perm(c[2 * i + 1], c[2 * i], 0x05040100u);
        o[i] = __builtin_amdgcn_perm(c[2 * i + 1], c[2 * i], 0x07060302u);
    }
    even = __builtin_bit_cast(bf16x8, e);
    odd = __builtin_bit_cast(bf16x8, o);
}

__device__ __forceinline__ Sequence sequence_of(const PagePool& p, const int32_t* seq, int b, int B,
                                                int max_tokens) {
    const int slot = b < B ? slot_of(seq, b, p.S) : -1;
    return Sequence{slot, slot < 0 ? 0 : min(length_of(p, slot), max_tokens)};
}

// What a wave loads for 32 tokens of a page block: key codes, value codes, and the
// scale bytes of both, [2 D / 32][32 tokens], in a slot of LDS.  The 16-byte
// pieces of a 64-byte key row are permuted by the row's place in groups of
// sixteen (piece ^ row / 4 % 4), so that the sixteen rows a quarter wave reads at
// once lie in distinct banks.
template <int D>
struct Slot {
    static constexpr int kCodes = kBlk * D / 2;  // bytes of the key, and of the value codes
    static constexpr int kLoads = 2 * kCodes / 1024 + 1;
    static constexpr int kBytes = 2 * kCodes + 256;
    static constexpr int kSlots = 2;  // steps ahead; four of 64 channels gain nothing (61.5 and 61.8 us for 286 MB)
    static constexpr int kRow = D / 2;

    // The wave's loads of tokens tok .. + 32 of a block into `slot`: kLoads of them.
    __device__ __forceinline__ static void load(const char* block, int tok, int shift, const char* slot) {
        const int lane = threadIdx.x & (kWave - 1);
        const char* keys = block + tok * kRow;
        const char* values = keys + ((size_t)kRow << shift);
        const uint32_t piece = D == 128 ? (lane ^ ((lane >> 4) & 3)) * 16 : lane * 16;
#pragma unroll
        for (int i = 0; i < kCodes / 1024; ++i) lds_dma16<true>(keys + i * 1024, piece, slot + i * 1024);
#pragma unroll
        for (int i = 0; i < kCodes / 1024; ++i)
            lds_dma16<true>(values + i * 1024, lane * 16, slot + kCodes + i * 1024);
        // 2 D / 32 rows of 32 bytes, eight lanes each; lanes beyond them load the last one again
        const uint32_t row = min(lane >> 3, 2 * D / 32 - 1);
        lds_dma4(block + ((size_t)D << shift) + tok, (row << shift) + (lane & 7) * 4, slot + 2 * kCodes);
    }
};

// The running softmax sums of a wave over its tokens.  NH: up to 4 heads of three
// columns each, 8 of two, or 16.
template <typename T, int D, int NH>
struct Sums {
    using S = Slot<D>;
    static constexpr int NP = std::is_same<T, float>::value ? 3 : 1;  // bf16 parts of a query
    static constexpr int NK = D / 32;  // products per 16 tokens: dwords of a lane's quarter row
    static constexpr int NC = D / 16;  // channels per lane of V^T
    static constexpr int NW = NH == 4 ? 1 : NH == 8 ? 2 : 3;  // parts of the weights per lane
    bf16x8 q[NK][NP];
    float m;
    f32x4 den, o[NC];  // o[i][r]: channel NC (4 (lane / 16) + r) + i of column lane % 16

    __device__ __forceinline__ void start(const T* rows, int G) {
        const int lane = threadIdx.x & (kWave - 1);
        const int c = lane & 15, quarter = lane >> 4, h = c & (NH - 1);
        const bool used = h < G && c < (NH == 4 ? 12 : 16);
#pragma unroll
        for (int s = 0; s < NK; ++s) {
            if constexpr (NP == 1) {
                u32x4 y = zero16();
                if (used) y = ld16(rows + (size_t)h * D + D / 4 * quarter + 8 * s);
                q[s][0] = __builtin_bit_cast(bf16x8, y);
            } else {
                float y[8];
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    y[i] = used ? (float)rows[(size_t)h * D + D / 4 * quarter + 8 * s + i] : 0.0f;
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

    // The logits of 32 tokens, before scaling.
    __device__ __forceinline__ void logits(const char* slot, f32x4 (&acc)[2]) const {
        const int lane = threadIdx.x & (kWave - 1);
        const int c = lane & 15, quarter = lane >> 4;
        const int tok = 4 * (c & 3) + (c >> 2);
        const char* row = slot + tok * S::kRow + (D == 128 ? (quarter ^ (c & 3)) * 16 : quarter * 8);
        const uint8_t* scale = reinterpret_cast<const uint8_t*>(slot + 2 * S::kCodes + quarter * D / 128 * kBlk + tok);
#pragma unroll
        for (int tile = 0; tile < 2; ++tile) {
            uint32_t k[NK];
#pragma unroll
            for (int e = 0; e < NK; ++e) k[e] = reinterpret_cast<const uint32_t*>(row + tile * 16 * S::kRow)[e];
            const float sc = scale_float(scale[16 * tile]);
            acc[tile] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int e = 0; e < NK; ++e) {
                const bf16x8 kf = unpack8(k[e], sc);
#pragma unroll
                for (int a = NP - 1; a >= 0; --a) acc[tile] = mma(kf, q[e][a], acc[tile]);
            }
        }
    }

    // The tokens' share of the sums; the first `left` (at least one) count.
    __device__ __forceinline__ void add(const char* slot, f32x4 (&acc)[2], int left, float sl2) {
        const int lane = threadIdx.x & (kWave - 1);
        const int c = lane & 15, quarter = lane >> 4;
        const char* rows = slot + S::kCodes + quarter * S::kRow + c * (D / 32);
        const uint8_t* scales =
            reinterpret_cast<const uint8_t*>(slot + 2 * S::kCodes + (D / 32 + c * (D / 16) / 32) * kBlk + quarter);
        uint32_t v[8], vs[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if constexpr (D == 128)
                v[i] = *reinterpret_cast<const uint32_t*>(rows + 4 * i * S::kRow);
            else
                v[i] = *reinterpret_cast<const uint16_t*>(rows + 4 * i * S::kRow);
            vs[i] = scales[4 * i];
        }
        if (left < kBlk) {
            // rows behind the sequence hold anything: no weight, and zeros under it
            __builtin_amdgcn_sched_barrier(0);  // a branch, not selects in every step
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (4 * i + quarter >= left) {
                    acc[i >> 2][i & 3] = -INFINITY;
                    v[i] = 0;
                    vs[i] = 0;
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
        float sc[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) sc[i] = scale_float(vs[i]);
        const u32x4 ones = {0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u};
#pragma unroll
        for (int a = NW - 1; a >= 0; --a) den = mma(__builtin_bit_cast(bf16x8, ones), part[a], den);
        values<0>(v, sc, part);
        values<1>(v, sc, part);
        if constexpr (D == 128) {
            values<2>(v, sc, part);
            values<3>(v, sc, part);
        }
    }

    template <int SEL>
    __device__ __forceinline__ void values(const uint32_t (&v)[8], const float (&sc)[8], const bf16x8 (&part)[NW]) {
        bf16x8 even, odd;
        unpack_tokens<SEL>(v, sc, even, odd);
#pragma unroll
        for (int a = NW - 1; a >= 0; --a) {
            o[2 * SEL] = mma(even, part[a], o[2 * SEL]);
            o[2 * SEL + 1] = mma(odd, part[a], o[2 * SEL + 1]);
        }
    }

    // the parts of a head's sums added up in its first column
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

// One workgroup per split of a sequence and (layer, KV head); its waves take 32
// tokens in turn.  Bound by the loads: 32 layers, 4 sequences of 1639 tokens, 8 KV
// heads of 4 query heads (228 MB of pages): 42 us, 5.4 TB/s, and 38.8 without any
// arithmetic.  The vector unit is busy for about half of that; it converts K and V
// (64 instructions per 32 tokens), pairs V's tokens (36), splits the weights (32)
// and takes 8 exponentials and multiply-adds.
// NWV: waves per workgroup, kWaves, or all or half that a compute unit holds.
template <typename T, int D, int NH, int NWV>
__global__ __launch_bounds__(NWV * kWave, (kPerSimd<T, D, NH>)) void pages_split(const T* __restrict__ q, PagePool p,
                                                                  const int32_t* __restrict__ seq, int B, int G,
                                                                  int max_tokens, int share, int groups, int whole,
                                                                  float sl2, float* __restrict__ ws_o,
                                                                  float2* __restrict__ ws_ml,
                                                                  SplitRange* __restrict__ ranges,
                                                                  float* __restrict__ out) {
    constexpr int NC = D / 16;
    using S = Slot<D>;
    // the waves' rings, and behind their last use the waves' sums
    constexpr int kRing = S::kSlots * S::kBytes, kSums = NH * D * (int)sizeof(float);
    __shared__ __attribute__((aligned(16))) char s_ring[NWV * (kRing > kSums ? kRing : kSums)];
    __shared__ float s_ml[NWV][2][NH];
    float(*s_o)[NH][D] = reinterpret_cast<float(*)[NH][D]>(s_ring);

    const int pairs = p.L * p.Hkv;
    const int x = blockIdx.x / pairs, pair = blockIdx.x - x * pairs;
    const int l = pair / p.Hkv, j = pair - l * p.Hkv;
    const int lane = threadIdx.x & (kWave - 1);
    const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int c = lane & 15, quarter = lane >> 4;

    Work work{x, -1, 0, 0, {x, 1}};
    if (whole) {
        const Sequence s = sequence_of(p, seq, x, B, max_tokens);
        work.slot = s.slot;
        work.k1 = s.tokens;
    } else {
        // many sequences: their lengths are loaded once, by all waves (200 ragged ones of
        // up to 4000 tokens, 8 KV heads: 86 us with every wave loading them, 74 so)
        int* staged = nullptr;
        if (B > kWave) {
            static_assert(kPagesSlice * (int)sizeof(int) <= (int)sizeof(s_ring), "the lengths fit the rings");
            staged = reinterpret_cast<int*>(s_ring);
            for (int e = threadIdx.x; e < B; e += NWV * kWave) staged[e] = sequence_of(p, seq, e, B, max_tokens).tokens;
            __syncthreads();
        }
        // the first workgroup's first wave leaves the ranges for the merge
        auto of = [&](int e) { return sequence_of(p, seq, e, B, max_tokens); };
        work = find_work(of, B, share, x, staged, blockIdx.x == 0 && wv == 0 ? ranges : nullptr);
        if (staged != nullptr) __syncthreads();  // the rings take the lengths' place
        if (work.b < 0) return;
    }
    const int b = work.b, slot = work.slot, k0 = work.k0, k1 = work.k1;
    const int page = 1 << p.shift;
    const size_t row0 = ((size_t)l * B + b) * p.Hkv + j;  // the segment's first query row, over G

    Sums<T, D, NH> sums;
    sums.start(q + row0 * G * D, G);

    // page numbers of 64 pages at a time, one per lane; a step's tokens lie in one
    // page.  A step whose page number is invalid loads page 0 and is passed over.
    const int32_t* row = p.table + (size_t)max(slot, 0) * p.M;
    const char* ring = s_ring + wv * kRing;
    int ids = 0, ids0 = -kWave;
    uint32_t there = 0;  // by slot
    auto issue = [&](int t, int at_slot) {
        const int at = t >> p.shift;
        if (at >= ids0 + kWave || ids0 < 0) {
            ids0 = at;
            ids = row[min(at + lane, p.M - 1)];
            settle(ids);
        }
        const int pg = __builtin_amdgcn_readlane(ids, at - ids0);
        const bool ok = pg >= 0 && pg < p.n_pages;
        there = (there & ~(1u << at_slot)) | (uint32_t)ok << at_slot;
        S::load(page_block<D>(p, l, ok ? pg : 0, j), t & (page - 1), p.shift, ring + at_slot * S::kBytes);
    };
    constexpr int kStride = NWV * kBlk;
    int t0 = k0 + wv * kBlk;
    sums.settle_queries();
#pragma unroll
    for (int i = 0; i < S::kSlots; ++i)
        if (t0 + i * kStride < k1) issue(t0 + i * kStride, i);
    for (int at = 0; t0 < k1; t0 += kStride) {
        // the slot's loads are the oldest: those of the slots behind it may be in flight
        if (t0 + (S::kSlots - 1) * kStride < k1)
            wait_vmcnt<(S::kSlots - 1) * S::kLoads>();
        else
            wait_vmcnt<0>();
        asm volatile("" ::: "memory");
        if ((there >> at) & 1u) {
            const char* slot_at = ring + at * S::kBytes;
            f32x4 acc[2];
            sums.logits(slot_at, acc);
            sums.add(slot_at, acc, k1 - t0, sl2);
        }
        if (t0 + S::kSlots * kStride < k1) {
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // the slot is read
            issue(t0 + S::kSlots * kStride, at);
        }
        at = at + 1 == S::kSlots ? 0 : at + 1;
    }
    sums.finish();

    __syncthreads();  // every wave is done with its ring
    if (c < G) {
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
    for (int e = threadIdx.x; e < G * D; e += NWV * kWave) {
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
        if (work.range.count == 1) {  // the whole sequence: the result itself
            out[(row0 * G + h) * D + ch] = lt != 0.0f ? ot / lt : 0.0f;
        } else {
            const size_t part = ((size_t)pair * groups + x) * G + h;
            ws_o[part * D + ch] = ot;
            if (ch == 0) ws_ml[part] = make_float2(mx, lt);
        }
    }
}

// Merge the splits of sequences that have several, and write zeros for empty
// ones.  Rows (layer, sample, KV head, head), kMergeWaves / WPR per workgroup.
template <int D, int WPR>
__global__ __launch_bounds__(kThreads) void pages_merge(int Hkv, int B, int G, int groups,
                                                        const float* __restrict__ ws_o,
                                                        const float2* __restrict__ ws_ml,
                                                        const SplitRange* __restrict__ ranges, int n_rows,
                                                        float* __restrict__ out) {
    const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int row = blockIdx.x * (kWaves / WPR) + wv / WPR;
    if (row >= n_rows) return;  // WPR > 1: the whole workgroup
    const int seg = row / G, h = row - seg * G;
    const int lb = seg / Hkv, j = seg - lb * Hkv;
    const int l = lb / B, b = lb - l * B;
    const SplitRange range = ranges[b];
    if (range.count == 1) return;  // written by its only split
    const size_t base = (((size_t)l * Hkv + j) * groups + range.first) * G + h;
    merge_row<D, WPR, true>(ws_o + base * D, ws_ml + base, G, range.count, true, out + (size_t)row * D);
}

template <typename T, int D, int NH>
hipError_t run_heads(const void* q, const PagePool& p, int B, int Hq, int max_tokens, const int32_t* seq, float scale,
               float* out, void* ws, hipStream_t st) {
    const PagesPlan plan = decode_pages_plan(p.L, B, Hq, p.Hkv, max_tokens, D);
    const int share = max(1, kDecodeUnits * kPerSimd<T, D, NH> / plan.pairs);  // one round of workgroups
    float* wo = static_cast<float*>(ws);
    float2* wml = reinterpret_cast<float2*>(static_cast<char*>(ws) + plan.off_ml);
    SplitRange* ranges = reinterpret_cast<SplitRange*>(static_cast<char*>(ws) + plan.off_ranges);
    auto launch = [&](auto waves) {
        constexpr int NWV = decltype(waves)::value;
        hipLaunchKernelGGL((pages_split<T, D, NH, NWV>), dim3((unsigned)plan.pairs * plan.groups), dim3(NWV * kWave),
                           0, st, static_cast<const T*>(q), p, seq, B, plan.G, max_tokens, share, plan.groups,
                           (int)plan.whole, scale * kLog2e, wo, wml, ranges, out);
    };
    constexpr int kAll = 4 * kPerSimd<T, D, NH>;  // waves of a compute unit
    if (plan.per_unit == 1)
        launch(std::integral_constant<int, kAll>{});
    else if (plan.per_unit == 2)
        launch(std::integral_constant<int, kAll / 2>{});
    else
        launch(std::integral_constant<int, kWaves>{});
    // up to 16 splits: one wave per row; more: four, which cut the chain of loads in four
    // (8 KV heads of 4 query heads; one sequence of 32000 in 128 splits 21.5 us with one
    // wave and 17.2 with four, four layers of four of 8192 level, eight of them, up to 16
    // splits, 54 and 56, sixteen 99 and 101).  The bound counts, not the splits there are.
    const int rows = plan.pairs * B * plan.G;
    if (!plan.whole && share > 16)
        hipLaunchKernelGGL((pages_merge<D, kWaves>), dim3((unsigned)rows), dim3(kThreads), 0, st, p.Hkv, B, plan.G,
                           plan.groups, wo, wml, ranges, rows, out);
    else if (!plan.whole)
        hipLaunchKernelGGL((pages_merge<D, 1>), dim3((unsigned)((rows + kWaves - 1) / kWaves)), dim3(kThreads), 0, st,
                           p.Hkv, B, plan.G, plan.groups, wo, wml, ranges, rows, out);
    return hipGetLastError();
}

template <typename T, int D>
hipError_t run(const void* q, const PagePool& p, int B, int Hq, int max_tokens, const int32_t* seq, float scale,
               float* out, void* ws, hipStream_t st) {
    // fewer columns per part of the weights are more products: with the sixteen-head
    // form 4 heads take 57.6 us in place of 54.1 (8 layers, 4 sequences of 8192, d =
    // 128), 70.8 in place of 61 (d = 64, 16 layers), 8 heads 88 in place of 71 (32
    // ragged sequences of up to 32768)
    if (Hq / p.Hkv <= 4) return run_heads<T, D, 4>(q, p, B, Hq, max_tokens, seq, scale, out, ws, st);
    if (Hq / p.Hkv <= 8) return run_heads<T, D, 8>(q, p, B, Hq, max_tokens, seq, scale, out, ws, st);
    return run_heads<T, D, kPagesMaxGroup>(q, p, B, Hq, max_tokens, seq, scale, out, ws, st);
}

}  // namespace

hipError_t launch_decode_pages(const void* q, int dtype, const PagePool& p, int d, int B, int Hq, int max_tokens,
                               const int32_t* seq, float scale, float* out, void* ws, hipStream_t st) {
    const int slice = decode_pages_plan(p.L, B, Hq, p.Hkv, max_tokens, d).slice;
    if (slice < B) {  // each layer's slices as calls of their own
        const size_t row = (size_t)Hq * d, layer = (size_t)p.n_pages * p.Hkv * page_block_bytes(1 << p.shift, d);
        for (int l = 0; l < p.L; ++l)
            for (int b = 0; b < B; b += slice) {
                PagePool part = p;
                part.L = 1;
                part.pool += l * layer;
                if (seq == nullptr) {  // sample b is slot b
                    part.S -= b;
                    part.held += b;
                    part.length += b;
                    part.table += (size_t)b * p.M;
                }
                const size_t at = ((size_t)l * B + b) * row;
                const hipError_t e = launch_decode_pages(
                    static_cast<const char*>(q) + at * (dtype == 0 ? 2 : 4), dtype, part, d, B - b < slice ? B - b : slice,
                    Hq, max_tokens, seq != nullptr ? seq + b : nullptr, scale, out + at, ws, st);
                if (e != hipSuccess) return e;
            }
        return hipSuccess;
    }
    if (dtype == 0) {
        if (d == 128) return run<__bf16, 128>(q, p, B, Hq, max_tokens, seq, scale, out, ws, st);
        return run<__bf16, 64>(q, p, B, Hq, max_tokens, seq, scale, out, ws, st);
    }
    if (d == 128) return run<float, 128>(q, p, B, Hq, max_tokens, seq, scale, out, ws, st);
    return run<float, 64>(q, p, B, Hq, max_tokens, seq, scale, out, ws, st);
}

}  // namespace kve
