// The paged 4-bit cache: bookkeeping (extend, fork, free) and the kernels that
// pack rows into pages, move them between sequences and read them back.
//
// Rows are four-bit floats with a power of two per 32 channels (kve_pages.h).
// Eight channels make a dword, four neighbouring lanes a block: a lane packs or
// unpacks its dword with the scaled conversions of gfx950, whose scale operand is
// the float 2^(s - 127), that is s << 23, and the block's largest magnitude is
// two lane exchanges away.  The conversions round to the nearest, ties to even,
// and saturate; a scale of 255 << 23 reads as NaN (checked over all scales, codes
// and bf16 inputs).
#include "kve_device.h"
#include "kve_internal.h"
#include "kve_pages_device.h"

namespace kve {
namespace {

constexpr int kThreads = 256;

typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));

// ---------------------------------------------------------------------------
// eight channels of a row as a dword of codes, and back
// ---------------------------------------------------------------------------

// Once: non-temporal, for rows of a large tensor that are read once.
template <bool Once>
__device__ __forceinline__ u32x4 load16(const char* at) {
    if constexpr (Once) return __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(at));
    return ld16(at);
}

template <typename T>
struct Eight;

template <>
struct Eight<__bf16> {
    u32x4 v;
    template <bool Once>
    __device__ __forceinline__ void load(const char* row, int part) {
        v = load16<Once>(row + part * 16);
    }
    // bits of the largest magnitude, as a float32
    __device__ __forceinline__ uint32_t top() const {
        u16x2 m = __builtin_bit_cast(u16x2, v[0] & 0x7fff7fffu);
#pragma unroll
        for (int i = 1; i < 4; ++i) m = __builtin_elementwise_max(m, __builtin_bit_cast(u16x2, v[i] & 0x7fff7fffu));
        return (uint32_t)max((int)m[0], (int)m[1]) << 16;
    }
    __device__ __forceinline__ uint32_t codes(float scale) const {
        // whole elements first: a bit cast of v[i] itself reads element 0
        const uint32_t a = v[0], b = v[1], c = v[2], d = v[3];
        uint32_t w = 0;
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_bit_cast(bf16x2, a), scale, 0);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_bit_cast(bf16x2, b), scale, 1);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_bit_cast(bf16x2, c), scale, 2);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_bit_cast(bf16x2, d), scale, 3);
        return w;
    }
    __device__ __forceinline__ static void store(char* row, int part, uint32_t w, float scale) {
        u32x4 o;
        o[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 0));
        o[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 1));
        o[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 2));
        o[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 3));
        __builtin_nontemporal_store(o, reinterpret_cast<u32x4*>(row) + part);
    }
};

template <>
struct Eight<float> {
    u32x4 v[2];
    template <bool Once>
    __device__ __forceinline__ void load(const char* row, int part) {
        v[0] = load16<Once>(row + part * 32);
        v[1] = load16<Once>(row + part * 32 + 16);
    }
    __device__ __forceinline__ uint32_t top() const {
        uint32_t m = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) m = max(m, max(v[0][i] & 0x7fffffffu, v[1][i] & 0x7fffffffu));
        return m;
    }
    __device__ __forceinline__ uint32_t codes(float scale) const {
        uint32_t w = 0;
        const f32x4 a = __builtin_bit_cast(f32x4, v[0]), b = __builtin_bit_cast(f32x4, v[1]);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, a[0], a[1], scale, 0);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, a[2], a[3], scale, 1);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, b[0], b[1], scale, 2);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, b[2], b[3], scale, 3);
        return w;
    }
    __device__ __forceinline__ static void store(char* row, int part, uint32_t w, float scale) {
        const f32x2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 0);
        const f32x2 b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 1);
        const f32x2 c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 2);
        const f32x2 d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 3);
        const f32x4 lo = {a[0], a[1], b[0], b[1]}, hi = {c[0], c[1], d[0], d[1]};
        __builtin_nontemporal_store(lo, reinterpret_cast<f32x4*>(row) + 2 * part);
        __builtin_nontemporal_store(hi, reinterpret_cast<f32x4*>(row) + 2 * part + 1);
    }
};

// The largest of x over the four lanes of a block.
__device__ __forceinline__ uint32_t quad_max(uint32_t x) {
    x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0xb1, 0xf, 0xf, false));  // lanes 1 0 3 2
    return max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x4e, 0xf, 0xf, false));  // lanes 2 3 0 1
}

// Scale byte of a block whose largest magnitude has these float32 bits.  A
// quarter added to the mantissa carries into the exponent from 1.75 on.
__device__ __forceinline__ uint32_t scale_byte(uint32_t top) {
    const int e = (int)((top + 0x200000u) >> 23) - 2;
    return top >= 0x7f800000u ? 255u : (uint32_t)min(max(e, 2), 252);
}

// Codes of a lane's eight channels, the block's scale byte in s.
template <typename T>
__device__ __forceinline__ uint32_t pack_eight(const Eight<T>& x, uint32_t& s) {
    s = scale_byte(quad_max(x.top()));
    return s == 255u ? 0u : x.codes(scale_float(s));
}

// ---------------------------------------------------------------------------
// rows: into pages (kve_pages_append, kve_pages_compact), between sequences
// (kve_pages_select) and out of them (kve_pages_read)
// ---------------------------------------------------------------------------

constexpr int kRows = kPagesRows;  // per workgroup

// The rows of a call: `cap` of each of L B Hkv segments (layer, sample, KV head).
// A workgroup takes kRows rows of one segment, the heads of a page side by side,
// or, Flat, kRows rows of all segments one after the other, where a segment has
// few: a decode step's single rows would else be a workgroup each.
struct RowGrid {
    int B, Hkv, cap, nblk;  // nblk: workgroups per segment
    uint32_t rows;          // of all segments (Flat)
};

// Rows per segment up to which workgroups take several segments.  Captured calls,
// so and with a workgroup each, 4096 segments of 128 channels: of one row appended
// 5.6 and 7.1 us, read 4.9 and 7.1, selected 3.9 and 5.4; of 8 6.8 and 7.7, 6.3 and
// 7.5, 4.3 and 5.8; of 16 10.9 and 9.6, 8.7 and 8.2, 6.5 and 7.6; of 32 17.2 and
// 15.6 (the divisions per row), 14.1 and 12.6, level.  Few segments are the other
// way round, since 64 rows to a workgroup leave most compute units idle: 128 of one
// row appended 5.0 and 2.7 us, read 4.5 and 2.8, selected 3.4 and 3.0; the rule does
// not look at their number.
constexpr int kFlatRows = 8;

struct RowAt {
    int m, l, b, j;  // row m of segment (l, b, j)
    size_t seg;
};

template <bool Flat>
__device__ __forceinline__ RowAt row_at(const RowGrid& g, int in) {
    RowAt r;
    uint32_t lb;
    if constexpr (Flat) {
        const uint32_t at = min(blockIdx.x * (uint32_t)kRows + in, g.rows - 1);
        const uint32_t seg = at / (uint32_t)g.cap;
        r.m = (int)(at - seg * g.cap);
        lb = seg / (uint32_t)g.Hkv;
        r.j = (int)(seg - lb * g.Hkv);
    } else {
        const uint32_t x = blockIdx.x / (uint32_t)g.Hkv;
        r.j = (int)(blockIdx.x - x * g.Hkv);
        lb = x / (uint32_t)g.nblk;
        r.m = (int)(x - lb * g.nblk) * kRows + in;
    }
    r.l = (int)(lb / (uint32_t)g.B);
    r.b = (int)(lb - (uint32_t)r.l * g.B);
    r.seg = (size_t)lb * g.Hkv + r.j;
    return r;
}

// Whether a workgroup's row `in` exists (it may lie behind its segment's count).
template <bool Flat>
__device__ __forceinline__ bool row_there(const RowGrid& g, int in) {
    return !Flat || blockIdx.x * (uint32_t)kRows + in < g.rows;
}

// The page block and token of position first + m of a slot for a (layer, KV
// head); null where the position has no page or is not below `limit`.
template <int D>
__device__ __forceinline__ char* find_row(const PagePool& p, int slot, int first, int m, int limit, const RowAt& r,
                                          int& tok) {
    if (slot < 0 || first < 0 || m >= limit - first) return nullptr;
    const int pos = first + m;
    const int pg = p.table[(size_t)slot * p.M + (pos >> p.shift)];
    tok = pos & ((1 << p.shift) - 1);
    return pg >= 0 && pg < p.n_pages ? page_block<D>(p, r.l, pg, r.j) : nullptr;
}

// Byte offsets in a page block: codes of token tok from channel 8 part on, and
// the scale byte of the channels' block; the values' are behind the keys'.
template <int D>
struct PageAt {
    size_t codes, scales;
    __device__ __forceinline__ PageAt(int tok, int part, int shift)
        : codes((size_t)tok * (D / 2) + part * 4),
          scales(((size_t)D << shift) + ((size_t)(part / 4) << shift) + tok) {}
    __device__ __forceinline__ static size_t values(int shift) { return (size_t)(D / 2) << shift; }
    __device__ __forceinline__ static size_t value_scales(int shift) { return (size_t)(D / 32) << shift; }
};

// D / 8 lanes to a row.  All of a thread's rows are looked up, then loaded, then
// packed, so that a workgroup waits for memory once per stage.  Gather: rows idx of
// a prompt's keys and values, which are read once (32 layers, 1639 of 32768 rows:
// 207 us with non-temporal loads, 218 without, 5.3 TB/s); else all rows of what a
// projection has just left in the caches (1003 rows of four sequences, 8 layers:
// 31 and 24 us).
template <typename T, int D, bool Flat, bool Gather>
__global__ __launch_bounds__(kThreads) void pack_rows(RowView kv, RowView vv, RowGrid g, int N,
                                                      const int32_t* __restrict__ idx,
                                                      const int32_t* __restrict__ count,
                                                      const int32_t* __restrict__ start,
                                                      const int32_t* __restrict__ seq, PagePool p) {
    constexpr int kLanes = D / 8;
    constexpr int kStep = kThreads / kLanes;
    constexpr int kItems = kRows / kStep;
    const int part = threadIdx.x % kLanes;
    char* block[kItems];
    int tok[kItems];
    Eight<T> x[kItems], y[kItems];
#pragma unroll
    for (int i = 0; i < kItems; ++i) {
        const int in = i * kStep + threadIdx.x / kLanes;
        const RowAt r = row_at<Flat>(g, in);
        const int n = Gather ? min(count[r.seg], g.cap) : count != nullptr ? min(count[r.b], g.cap) : g.cap;
        block[i] = nullptr;
        if (row_there<Flat>(g, in) && r.m < n) {
            const int t = Gather ? idx[r.seg * g.cap + r.m] : r.m;
            const int slot = slot_of(seq, r.b, p.S);
            if (t >= 0 && t < N && slot >= 0)
                block[i] = find_row<D>(p, slot, start[r.b], r.m, held_of(p, slot) << p.shift, r, tok[i]);
            if (block[i] != nullptr) {
                x[i].template load<Gather>(kv.base + (size_t)r.l * kv.s_layer + (size_t)r.b * kv.s_batch + (size_t)r.j * kv.s_head +
                              (size_t)t * kv.s_token, part);
                y[i].template load<Gather>(vv.base + (size_t)r.l * vv.s_layer + (size_t)r.b * vv.s_batch + (size_t)r.j * vv.s_head +
                              (size_t)t * vv.s_token, part);
            }
        }
    }
#pragma unroll
    for (int i = 0; i < kItems; ++i) {
        if (block[i] == nullptr) continue;  // the same for all lanes of a row
        uint32_t sk, sv;
        const uint32_t wk = pack_eight(x[i], sk), wv = pack_eight(y[i], sv);
        const PageAt<D> at(tok[i], part, p.shift);
        *reinterpret_cast<uint32_t*>(block[i] + at.codes) = wk;
        *reinterpret_cast<uint32_t*>(block[i] + at.codes + at.values(p.shift)) = wv;
        if (part % 4 == 0) {
            block[i][at.scales] = (char)sk;
            block[i][at.scales + at.value_scales(p.shift)] = (char)sv;
        }
    }
}

// D / 32 lanes to a row, each a block of 32 channels (16 bytes of codes, one
// scale byte) of a key and a value row.  The source rows are read once and their
// sequence ends, as a rule: non-temporal loads (16 layers, 4 sequences, 4001 of
// 16001 rows: 105 us, 5.3 TB/s read and written; 115 without).  Rows of 64 channels
// leave half of a workgroup without work; random rows of 16001 move at 3.6 TB/s
// so, those of 128 at 3.8.
template <int D, bool Flat>
__global__ __launch_bounds__(kThreads) void select_rows(PagePool p, RowGrid g, const int32_t* __restrict__ src,
                                                        const int32_t* __restrict__ idx,
                                                        const int32_t* __restrict__ count,
                                                        const int32_t* __restrict__ dst,
                                                        const int32_t* __restrict__ start) {
    constexpr int kLanes = D / 32;
    const int in = threadIdx.x / kLanes, part = threadIdx.x % kLanes * 4;
    if (in >= kRows) return;  // rows of 64 channels: two lanes each
    const RowAt r = row_at<Flat>(g, in);
    if (!row_there<Flat>(g, in) || r.m >= min(count[r.seg], g.cap)) return;
    const int from = slot_of(src, r.b, p.S), to = slot_of(dst, r.b, p.S);
    if (from < 0 || to < 0) return;
    const int t = idx[r.seg * g.cap + r.m];
    int ta = 0, tb = 0;
    const char* a = t < 0 ? nullptr : find_row<D>(p, from, 0, t, length_of(p, from), r, ta);
    char* o = find_row<D>(p, to, start[r.b], r.m, held_of(p, to) << p.shift, r, tb);
    if (a == nullptr || o == nullptr) return;
    const PageAt<D> at_a(ta, part, p.shift), at_o(tb, part, p.shift);
    const size_t values = at_a.values(p.shift), value_scales = at_a.value_scales(p.shift);
    const u32x4 wk = load16<true>(a + at_a.codes), wv = load16<true>(a + at_a.codes + values);
    const char sk = a[at_a.scales], sv = a[at_a.scales + value_scales];
    st16(o + at_o.codes, wk);
    st16(o + at_o.codes + values, wv);
    o[at_o.scales] = sk;
    o[at_o.scales + value_scales] = sv;
}

// D / 8 lanes to a row, as in pack_rows.  Bound by HBM: 2 M rows of a pool of
// 1.1 GB in 267 us, 5.0 TB/s read and written; 1.7 M rows just packed in 155 us;
// as float32 0.4 M of them take 175 us, 2.8 TB/s (bf16: 44).
// Non-temporal loads of the codes gain 8% on the former and lose 7% on the
// latter; cached stores lose 30%.
template <typename T, int D, bool Flat>
__global__ __launch_bounds__(kThreads) void read_rows(PagePool p, RowGrid g, const int32_t* __restrict__ seq,
                                                      const int32_t* __restrict__ start,
                                                      const int32_t* __restrict__ count, char* __restrict__ k_out,
                                                      char* __restrict__ v_out) {
    constexpr int kLanes = D / 8;
    constexpr int kStep = kThreads / kLanes;
    constexpr int kItems = kRows / kStep;
    const int part = threadIdx.x % kLanes;
    size_t out[kItems];
    bool there[kItems];
    uint32_t wk[kItems], wv[kItems], sk[kItems], sv[kItems];
#pragma unroll
    for (int i = 0; i < kItems; ++i) {
        const int in = i * kStep + threadIdx.x / kLanes;
        const RowAt r = row_at<Flat>(g, in);
        const int n = count != nullptr ? min(count[r.b], g.cap) : g.cap;
        const int slot = slot_of(seq, r.b, p.S);
        out[i] = (r.seg * g.cap + r.m) * (D * sizeof(T));
        there[i] = row_there<Flat>(g, in) && r.m < n && slot >= 0;
        if (there[i]) {
            int tok = 0;
            const char* block = find_row<D>(p, slot, start != nullptr ? start[r.b] : 0, r.m, length_of(p, slot), r,
                                            tok);
            there[i] = block != nullptr;
            if (there[i]) {
                const PageAt<D> at(tok, part, p.shift);
                wk[i] = *reinterpret_cast<const uint32_t*>(block + at.codes);
                wv[i] = *reinterpret_cast<const uint32_t*>(block + at.codes + at.values(p.shift));
                sk[i] = (uint8_t)block[at.scales];
                sv[i] = (uint8_t)block[at.scales + at.value_scales(p.shift)];
            }
        }
    }
#pragma unroll
    for (int i = 0; i < kItems; ++i) {
        if (!there[i]) continue;
        if (k_out != nullptr) Eight<T>::store(k_out + out[i], part, wk[i], scale_float(sk[i]));
        if (v_out != nullptr) Eight<T>::store(v_out + out[i], part, wv[i], scale_float(sv[i]));
    }
}

// ---------------------------------------------------------------------------
// bookkeeping
// ---------------------------------------------------------------------------

// These kernels are chains of a few memory latencies, and their code comes from
// memory too when other kernels have run since: it is kept short (loops are not
// unrolled; scans are lane moves).
constexpr int kPlanThreads = kPagesMaxEntries;
constexpr int kPlanWaves = kPlanThreads / kWave;
constexpr int kLoads = 16;                                // pages per thread and round of find_free
constexpr int kTallies = kLoads * kPlanWaves;             // counts of one round, in page order
constexpr int kTalliesPerLane = kTallies / kWave;
constexpr uint32_t kMostPages = 0x7fffffffu;              // where sums of needs stay

// Sum of needs that stays at kMostPages.
__device__ __forceinline__ uint32_t add_needs(uint32_t a, uint32_t b) { return min(a + b, kMostPages); }

// Inclusive sum of needs over the lanes of a wave.
__device__ __forceinline__ uint32_t wave_scan(uint32_t x) {
#define KVE_SCAN_STEP(ctrl, rows) \
    x = add_needs(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, ctrl, rows, 0xf, false))
    KVE_SCAN_STEP(0x111, 0xf);  // the lane before
    KVE_SCAN_STEP(0x112, 0xf);  // two before
    KVE_SCAN_STEP(0x114, 0xf);
    KVE_SCAN_STEP(0x118, 0xf);
    KVE_SCAN_STEP(0x142, 0xa);  // lane 15 of a row to the next row
    KVE_SCAN_STEP(0x143, 0xc);  // lane 31 to the upper half
#undef KVE_SCAN_STEP
    return x;
}

// Sum of needs over the threads before, and over all in `total`.  s: kPlanWaves words of LDS.
__device__ __forceinline__ uint32_t scan_exclusive(uint32_t x, uint32_t* s, uint32_t& total) {
    const int lane = threadIdx.x & (kWave - 1), w = threadIdx.x / kWave;
    const uint32_t inc = wave_scan(x);
    if (lane == kWave - 1) s[w] = inc;
    __syncthreads();
    const uint32_t sums = wave_scan(lane < kPlanWaves ? s[lane] : 0u);
    total = (uint32_t)__builtin_amdgcn_readlane((int)sums, kPlanWaves - 1);
    const uint32_t before = w > 0 ? (uint32_t)__shfl((int)sums, w - 1) : 0u;
    return add_needs(before, (uint32_t)__shfl_up((int)inc, 1) * (lane > 0));
}

// The first `want` free pages in ascending order into list; returns how many
// there are (all free pages, where fewer than `want`).  Every wave takes 64
// neighbouring pages per load: a ballot ranks them, and the tallies of a round
// are summed by every wave for itself.  A round is 16384 pages and about 6.5 us: a
// call passes over all full pages below the ones it takes (extend of 16 sequences
// by a page: 10 us in an empty pool of 300000, 126 with its first 297000 full).
__device__ __noinline__ int find_free(const int32_t* refs, int n_pages, int want, int32_t* list) {
    __shared__ uint32_t s_tally[kTallies];
    const int lane = threadIdx.x & (kWave - 1), w = threadIdx.x / kWave;
    int found = 0;
    for (int base = 0; base < n_pages && found < want; base += kPlanThreads * kLoads) {
        uint32_t free = 0;
        const int at = base + (int)threadIdx.x;
        const int loads = min(kLoads, (n_pages - base + kPlanThreads - 1) / kPlanThreads);
        int32_t ref[kLoads];
#pragma unroll
        for (int i = 0; i < kLoads; ++i) ref[i] = refs[min(at + i * kPlanThreads, n_pages - 1)];
#pragma unroll
        for (int i = 0; i < kLoads; ++i) free |= (uint32_t)(ref[i] == 0 && at + i * kPlanThreads < n_pages) << i;
        __syncthreads();  // the last round's tallies are read
#pragma unroll 1
        for (int i = 0; i < loads; ++i) {
            const uint64_t mask = __builtin_amdgcn_ballot_w64((free >> i) & 1u);
            if (lane == 0) s_tally[i * kPlanWaves + w] = (uint32_t)__popcll(mask);
        }
        __syncthreads();
        // lane: the tallies kTalliesPerLane lane .. of this round, those before them in `before`
        uint32_t own = 0;
#pragma unroll 1
        for (int e = 0; e < kTalliesPerLane; ++e) {
            const int t = lane * kTalliesPerLane + e;
            own += t < loads * kPlanWaves ? s_tally[t] : 0u;
        }
        const uint32_t inc = wave_scan(own), before = inc - own;
#pragma unroll 1
        for (int i = 0; i < loads; ++i) {
            const int t = i * kPlanWaves + w, first = t / kTalliesPerLane * kTalliesPerLane;
            uint32_t r = (uint32_t)__builtin_amdgcn_readlane((int)before, __builtin_amdgcn_readfirstlane(t / kTalliesPerLane));
            for (int e = first; e < t; ++e) r += s_tally[e];
            const uint64_t mask = __builtin_amdgcn_ballot_w64((free >> i) & 1u);
            r += (uint32_t)found + __builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mask, 0u));
            if (((free >> i) & 1u) != 0 && r < (uint32_t)want) list[r] = at + i * kPlanThreads;
        }
        found += __builtin_amdgcn_readlane((int)inc, kWave - 1);
    }
    __syncthreads();  // list is whole
    return found;
}

// Whether an earlier entry names the same slot.  s_seq holds the entries' slots.
__device__ __forceinline__ bool named_before(const int* s_seq, int i, int slot) {
    bool hit = false;
#pragma unroll 1
    for (int e = 0; e < i; e += 4) {
        const int4 four = *reinterpret_cast<const int4*>(s_seq + e);
        hit |= four.x == slot | ((four.y == slot) & (e + 1 < i)) | ((four.z == slot) & (e + 2 < i)) |
               ((four.w == slot) & (e + 3 < i));
    }
    return hit;
}

// Entry that owns page r of the list: the last one with off <= r.  Entries
// without a need share their successor's offset and are passed over.
__device__ __forceinline__ int owner_of(const int* s_off, int n, int r) {
    int lo = 0, hi = n - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (s_off[mid] <= r)
            lo = mid;
        else
            hi = mid - 1;
    }
    return lo;
}

// kve_pages_extend: one workgroup, one thread per entry.  Needs are summed over
// the entries before, the free pages listed, and every listed page given to the
// entry whose range of the list it falls in.
__global__ __launch_bounds__(kPlanThreads) void extend_kernel(PagePool p, const int32_t* seq, const int32_t* add, int n,
                                                              int32_t* start, int32_t* missing, int32_t* list) {
    __shared__ __attribute__((aligned(16))) int s_seq[kPlanThreads];
    __shared__ int s_off[kPlanThreads], s_held[kPlanThreads], s_ok[kPlanThreads];
    __shared__ uint32_t s_scan[kPlanWaves];
    const int i = threadIdx.x;
    const int slot = i < n ? slot_of(seq, i, p.S) : -1;
    s_seq[i] = slot;
    __syncthreads();
    int held = 0, len = 0, more = -1;
    if (slot >= 0) {
        held = held_of(p, slot);
        len = length_of(p, slot);
        more = add[i];
    }
    bool valid = slot >= 0 && !named_before(s_seq, i, slot);
    const long long now = (long long)len + more;
    valid = valid && more >= 0 && now <= (long long)p.M << p.shift;
    const uint32_t need = valid ? (uint32_t)max(0, (int)((now + (1 << p.shift) - 1) >> p.shift) - held) : 0u;
    uint32_t total;
    const uint32_t off = scan_exclusive(need, s_scan, total);
    const int want = min((int)total, p.n_pages);
    const int found = find_free(p.refs, p.n_pages, want, list);
    const bool given = valid && (need == 0 || off + need <= (uint32_t)found);
    s_off[i] = min((int)off, p.n_pages);
    s_held[i] = held;
    s_ok[i] = given;
    __syncthreads();
    for (int r = i; r < min(want, found); r += kPlanThreads) {
        const int e = owner_of(s_off, n, r);
        if (s_ok[e]) {
            p.table[(size_t)s_seq[e] * p.M + s_held[e] + (r - s_off[e])] = list[r];
            p.refs[list[r]] = 1;
        }
    }
    if (i < n) {
        start[i] = given ? len : -1;
        if (given) {
            p.held[slot] = held + (int)need;
            p.length[slot] = len + more;
        }
    }
    if (i == 0) *missing = (int)total - min(want, found);
}

// What fork_copy does for an entry: full pages shared (-1: refused), the partial
// page's source and copy (copy < 0: none) and its rows, and the two slots.  The
// caller's arrays are read once: `done` may be one of them.
struct ForkPlan {
    int full, from, to, rows, src, dst, unused[2];
};

__global__ __launch_bounds__(kPlanThreads) void fork_kernel(PagePool p, const int32_t* src, const int32_t* dst, int n,
                                                            int32_t* done, int32_t* missing, ForkPlan* plan,
                                                            int32_t* list) {
    __shared__ __attribute__((aligned(16))) int s_dst[kPlanThreads];
    __shared__ uint32_t s_scan[kPlanWaves];
    const int i = threadIdx.x;
    const int from = i < n ? slot_of(src, i, p.S) : -1, to = i < n ? slot_of(dst, i, p.S) : -1;
    s_dst[i] = to;
    __syncthreads();
    const bool free = from >= 0 && to >= 0 && p.held[to] == 0 && p.length[to] == 0;
    int len = free ? length_of(p, from) : 0;
    const bool valid = free && !named_before(s_dst, i, to);
    if (!valid) len = 0;
    const int full = len >> p.shift, rows = len & ((1 << p.shift) - 1);
    const int last = rows != 0 ? p.table[(size_t)from * p.M + full] : -1;
    // a last page that is not there is passed on as such: a fresh one would hold another's rows
    const uint32_t need = last >= 0 && last < p.n_pages ? 1u : 0u;
    uint32_t total;
    const uint32_t off = scan_exclusive(need, s_scan, total);
    // all sources are read (the scan's barrier); destinations may be written
    const int found = find_free(p.refs, p.n_pages, (int)total, list);
    const bool given = valid && (need == 0 || off < (uint32_t)found);
    if (i < n) {
        ForkPlan f{given ? full : -1, -1, -1, rows, from, to, {0, 0}};
        if (given) {
            if (need != 0) {
                f.from = last;
                f.to = list[off];
                p.refs[f.to] = 1;
            }
            if (rows != 0) p.table[(size_t)to * p.M + full] = need != 0 ? f.to : last;
            p.held[to] = full + (rows != 0);
            p.length[to] = len;
        }
        plan[i] = f;
        done[i] = given;
    }
    if (i == 0) *missing = max(0, (int)total - found);
}

// Workgroup (entry, part): part 0 shares the full pages, the others copy the
// written rows of the partial page, kPagesCopyBytes of one layer's heads each.  A
// 16-byte piece is copied when it holds a byte of a written row.
template <int D>
__global__ __launch_bounds__(kThreads) void fork_copy(PagePool p, const ForkPlan* __restrict__ plan, int nblk) {
    const int i = blockIdx.x / (1 + p.L * nblk), part = blockIdx.x - i * (1 + p.L * nblk);
    const ForkPlan f = plan[i];
    if (f.full < 0) return;
    if (part == 0) {
        const int32_t* a = p.table + (size_t)f.src * p.M;
        int32_t* o = p.table + (size_t)f.dst * p.M;
        for (int e = threadIdx.x; e < f.full; e += kThreads) {
            const int pg = a[e];
            o[e] = pg;
            if (pg >= 0 && pg < p.n_pages) atomicAdd(p.refs + pg, 1);
        }
        return;
    }
    if (f.to < 0) return;
    const int l = (part - 1) / nblk, blk = (part - 1) % nblk;
    const int page = 1 << p.shift;
    const int bytes = (D / 16 * 17) << p.shift;
    const size_t whole = (size_t)bytes * p.Hkv;
    const char* a = page_block<D>(p, l, f.from, 0);
    char* o = page_block<D>(p, l, f.to, 0);
    const size_t end = min((size_t)(blk + 1) * kPagesCopyBytes, whole);
    for (size_t at = (size_t)blk * kPagesCopyBytes + threadIdx.x * 16; at < end; at += kThreads * 16) {
        const int in = (int)(at % (unsigned)bytes);
        const int tok = in < page * D ? (in % (page * (D / 2))) / (D / 2) : (in - page * D) % page;
        if (tok < f.rows) st16(o + at, ld16(a + at));
    }
}

// kve_pages_free: one workgroup per entry.  Whoever takes `held` first empties the slot.
__global__ __launch_bounds__(kThreads) void free_kernel(PagePool p, const int32_t* __restrict__ seq) {
    __shared__ int s_held;
    const int slot = slot_of(seq, blockIdx.x, p.S);
    if (slot < 0) return;
    if (threadIdx.x == 0) {
        s_held = min(max(atomicExch(p.held + slot, 0), 0), p.M);
        p.length[slot] = 0;
    }
    __syncthreads();
    for (int e = threadIdx.x; e < s_held; e += kThreads) {
        const int pg = p.table[(size_t)slot * p.M + e];
        if (pg >= 0 && pg < p.n_pages) atomicSub(p.refs + pg, 1);
    }
}

RowGrid row_grid(const PagePool& p, int B, int cap) {
    return RowGrid{B, p.Hkv, cap, (cap + kRows - 1) / kRows, (uint32_t)p.L * B * p.Hkv * (uint32_t)cap};
}

bool is_flat(const RowGrid& g) { return g.cap <= kFlatRows; }

dim3 row_blocks(const PagePool& p, const RowGrid& g) {
    return dim3(is_flat(g) ? (g.rows + kRows - 1) / kRows : (unsigned)p.L * g.B * g.Hkv * g.nblk);
}

template <typename T, int D, bool Flat, bool Gather>
void launch_pack(const RowView& k, const RowView& v, const RowGrid& g, int N, const int32_t* idx,
                 const int32_t* count, const int32_t* start, const int32_t* seq, const PagePool& p, hipStream_t st) {
    hipLaunchKernelGGL((pack_rows<T, D, Flat, Gather>), row_blocks(p, g), dim3(kThreads), 0, st, k, v, g, N, idx,
                       count, start, seq, p);
}

template <typename T, int D>
void run_pack(const RowView& k, const RowView& v, int B, int N, const int32_t* idx, const int32_t* count, int cap,
              const int32_t* start, const int32_t* seq, const PagePool& p, hipStream_t st) {
    const RowGrid g = row_grid(p, B, cap);
    if (is_flat(g) && idx != nullptr)
        launch_pack<T, D, true, true>(k, v, g, N, idx, count, start, seq, p, st);
    else if (is_flat(g))
        launch_pack<T, D, true, false>(k, v, g, N, idx, count, start, seq, p, st);
    else if (idx != nullptr)
        launch_pack<T, D, false, true>(k, v, g, N, idx, count, start, seq, p, st);
    else
        launch_pack<T, D, false, false>(k, v, g, N, idx, count, start, seq, p, st);
}

template <int D>
void run_select(const PagePool& p, int B, const int32_t* src, const int32_t* idx, const int32_t* count, int cap,
                const int32_t* dst, const int32_t* start, hipStream_t st) {
    const RowGrid g = row_grid(p, B, cap);
    if (is_flat(g))
        hipLaunchKernelGGL((select_rows<D, true>), row_blocks(p, g), dim3(kThreads), 0, st, p, g, src, idx, count, dst,
                           start);
    else
        hipLaunchKernelGGL((select_rows<D, false>), row_blocks(p, g), dim3(kThreads), 0, st, p, g, src, idx, count,
                           dst, start);
}

template <typename T, int D>
void run_read(const PagePool& p, int B, int cap, const int32_t* seq, const int32_t* start, const int32_t* count,
              void* k_out, void* v_out, hipStream_t st) {
    const RowGrid g = row_grid(p, B, cap);
    if (is_flat(g))
        hipLaunchKernelGGL((read_rows<T, D, true>), row_blocks(p, g), dim3(kThreads), 0, st, p, g, seq, start, count,
                           static_cast<char*>(k_out), static_cast<char*>(v_out));
    else
        hipLaunchKernelGGL((read_rows<T, D, false>), row_blocks(p, g), dim3(kThreads), 0, st, p, g, seq, start, count,
                           static_cast<char*>(k_out), static_cast<char*>(v_out));
}

}  // namespace

hipError_t launch_pages_extend(const PagePool& p, const int32_t* seq, const int32_t* add, int n, int32_t* start,
                               int32_t* missing, void* ws, hipStream_t st) {
    int32_t* list = reinterpret_cast<int32_t*>(static_cast<char*>(ws) + align_up((size_t)n * sizeof(ForkPlan)));
    hipLaunchKernelGGL(extend_kernel, dim3(1), dim3(kPlanThreads), 0, st, p, seq, add, n, start, missing, list);
    return hipGetLastError();
}

hipError_t launch_pages_fork(const PagePool& p, int d, const int32_t* src, const int32_t* dst, int n, int32_t* done,
                             int32_t* missing, void* ws, hipStream_t st) {
    static_assert(sizeof(ForkPlan) == kPagesPlanBytes, "the workspace holds a plan per entry");
    ForkPlan* plan = static_cast<ForkPlan*>(ws);
    int32_t* list = reinterpret_cast<int32_t*>(static_cast<char*>(ws) + align_up((size_t)n * sizeof(ForkPlan)));
    hipLaunchKernelGGL(fork_kernel, dim3(1), dim3(kPlanThreads), 0, st, p, src, dst, n, done, missing, plan, list);
    const int nblk = pages_copy_blocks(p.Hkv, 1 << p.shift, d);
    const dim3 grid((unsigned)n * (1 + p.L * nblk));
    if (d == 128)
        hipLaunchKernelGGL(fork_copy<128>, grid, dim3(kThreads), 0, st, p, plan, nblk);
    else
        hipLaunchKernelGGL(fork_copy<64>, grid, dim3(kThreads), 0, st, p, plan, nblk);
    return hipGetLastError();
}

hipError_t launch_pages_free(const PagePool& p, const int32_t* seq, int n, hipStream_t st) {
    hipLaunchKernelGGL(free_kernel, dim3((unsigned)n), dim3(kThreads), 0, st, p, seq);
    return hipGetLastError();
}

hipError_t launch_pages_pack(const RowView& k, const RowView& v, int dtype, int d, int B, int N, const int32_t* idx,
                             const int32_t* count, int cap, const int32_t* start, const int32_t* seq,
                             const PagePool& p, hipStream_t st) {
    if (cap == 0) return hipSuccess;
    if (dtype == 0 && d == 128) run_pack<__bf16, 128>(k, v, B, N, idx, count, cap, start, seq, p, st);
    if (dtype == 0 && d == 64) run_pack<__bf16, 64>(k, v, B, N, idx, count, cap, start, seq, p, st);
    if (dtype == 1 && d == 128) run_pack<float, 128>(k, v, B, N, idx, count, cap, start, seq, p, st);
    if (dtype == 1 && d == 64) run_pack<float, 64>(k, v, B, N, idx, count, cap, start, seq, p, st);
    return hipGetLastError();
}

hipError_t launch_pages_select(const PagePool& p, int d, int B, const int32_t* src, const int32_t* idx,
                               const int32_t* count, int cap, const int32_t* dst, const int32_t* start,
                               hipStream_t st) {
    if (cap == 0) return hipSuccess;
    if (d == 128)
        run_select<128>(p, B, src, idx, count, cap, dst, start, st);
    else
        run_select<64>(p, B, src, idx, count, cap, dst, start, st);
    return hipGetLastError();
}

hipError_t launch_pages_read(const PagePool& p, int dtype, int d, int B, int T, const int32_t* seq,
                             const int32_t* start, const int32_t* count, void* k_out, void* v_out, hipStream_t st) {
    if (T == 0) return hipSuccess;
    if (dtype == 0 && d == 128) run_read<__bf16, 128>(p, B, T, seq, start, count, k_out, v_out, st);
    if (dtype == 0 && d == 64) run_read<__bf16, 64>(p, B, T, seq, start, count, k_out, v_out, st);
    if (dtype == 1 && d == 128) run_read<float, 128>(p, B, T, seq, start, count, k_out, v_out, st);
    if (dtype == 1 && d == 64) run_read<float, 64>(p, B, T, seq, start, count, k_out, v_out, st);
    return hipGetLastError();
}

}  // namespace kve
