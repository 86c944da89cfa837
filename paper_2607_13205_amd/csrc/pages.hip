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

template <typename T>
struct Eight;

template <>
struct Eight<__bf16> {
    u32x4 v;
    __device__ __forceinline__ void load(const char* row, int part) {
        v = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(row) + part);
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
    __device__ __forceinline__ void load(const char* row, int part) {
        v[0] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(row) + 2 * part);
        v[1] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(row) + 2 * part + 1);
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
// rows into pages: kve_pages_append (idx null) and kve_pages_compact
// ---------------------------------------------------------------------------

constexpr int kRows = 64;  // rows per workgroup

// One workgroup per (segment, kRows rows), D / 8 lanes to a row.
template <typename T, int D>
__global__ __launch_bounds__(kThreads) void pack_rows(RowView kv, RowView vv, int B, int N,
                                                      const int32_t* __restrict__ idx,
                                                      const int32_t* __restrict__ count, int cap,
                                                      const int32_t* __restrict__ start,
                                                      const int32_t* __restrict__ seq, PagePool p, int nblk) {
    constexpr int kLanes = D / 8;
    constexpr int kStep = kThreads / kLanes;
    const int blk = blockIdx.x % nblk, seg = blockIdx.x / nblk;
    const int j = seg % p.Hkv, lb = seg / p.Hkv;
    const int l = lb / B, b = lb - l * B;
    const int n = idx != nullptr ? min(count[seg], cap) : count != nullptr ? min(count[b], cap) : cap;
    const int slot = slot_of(seq, b, p.S), first = start[b];
    if (blk * kRows >= n || slot < 0 || first < 0) return;
    const int rows_held = held_of(p, slot) << p.shift;
    const char* k = kv.base + (size_t)l * kv.s_layer + (size_t)b * kv.s_batch + (size_t)j * kv.s_head;
    const char* v = vv.base + (size_t)l * vv.s_layer + (size_t)b * vv.s_batch + (size_t)j * vv.s_head;
    const int part = threadIdx.x % kLanes;
    const int page = 1 << p.shift;
    for (int m = blk * kRows + (int)threadIdx.x / kLanes; m < min(n, (blk + 1) * kRows); m += kStep) {
        const int t = idx != nullptr ? idx[(size_t)seg * cap + m] : m;
        if (t < 0 || t >= N || m >= rows_held - first) continue;
        const int pos = first + m;
        const int pg = p.table[(size_t)slot * p.M + (pos >> p.shift)];
        if (pg < 0 || pg >= p.n_pages) continue;
        Eight<T> x, y;
        x.load(k + (size_t)t * kv.s_token, part);
        y.load(v + (size_t)t * vv.s_token, part);
        char* block = page_block<D>(p, l, pg, j);
        const int tok = pos & (page - 1);
        uint32_t sk, sv;
        const uint32_t wk = pack_eight(x, sk), wv = pack_eight(y, sv);
        char* row = block + (size_t)tok * (D / 2) + part * 4;
        *reinterpret_cast<uint32_t*>(row) = wk;
        *reinterpret_cast<uint32_t*>(row + (size_t)page * (D / 2)) = wv;
        if (part % 4 == 0) {
            char* scales = block + (size_t)page * D + (size_t)(part / 4) * page + tok;
            scales[0] = (char)sk;
            scales[(size_t)page * (D / 32)] = (char)sv;
        }
    }
}

// ---------------------------------------------------------------------------
// rows of one sequence to another, unchanged: kve_pages_select
// ---------------------------------------------------------------------------

// One workgroup per (segment, kRows rows); a lane moves a block of 32 channels
// (16 bytes of codes, one scale byte) of a key and a value row.
template <int D>
__global__ __launch_bounds__(kThreads) void select_rows(PagePool p, int B, const int32_t* __restrict__ src,
                                                        const int32_t* __restrict__ idx,
                                                        const int32_t* __restrict__ count, int cap,
                                                        const int32_t* __restrict__ dst,
                                                        const int32_t* __restrict__ start, int nblk) {
    constexpr int kLanes = D / 32;
    constexpr int kStep = kThreads / kLanes;
    const int blk = blockIdx.x % nblk, seg = blockIdx.x / nblk;
    const int j = seg % p.Hkv, lb = seg / p.Hkv;
    const int l = lb / B, b = lb - l * B;
    const int n = min(count[seg], cap);
    const int from = slot_of(src, b, p.S), to = slot_of(dst, b, p.S), first = start[b];
    if (blk * kRows >= n || from < 0 || to < 0 || first < 0) return;
    const int have = length_of(p, from), rows_held = held_of(p, to) << p.shift;
    const int part = threadIdx.x % kLanes;
    const int page = 1 << p.shift;
    for (int m = blk * kRows + (int)threadIdx.x / kLanes; m < min(n, (blk + 1) * kRows); m += kStep) {
        const int t = idx[(size_t)seg * cap + m];
        if (t < 0 || t >= have || m >= rows_held - first) continue;
        const int pos = first + m;
        const int pa = p.table[(size_t)from * p.M + (t >> p.shift)];
        const int pb = p.table[(size_t)to * p.M + (pos >> p.shift)];
        if (pa < 0 || pa >= p.n_pages || pb < 0 || pb >= p.n_pages) continue;
        const char* a = page_block<D>(p, l, pa, j);
        char* o = page_block<D>(p, l, pb, j);
        const int ta = t & (page - 1), to_ = pos & (page - 1);
        const size_t ca = (size_t)ta * (D / 2) + part * 16, co = (size_t)to_ * (D / 2) + part * 16;
        const size_t sa = (size_t)page * D + (size_t)part * page + ta, so = (size_t)page * D + (size_t)part * page + to_;
        const u32x4 wk = ld16(a + ca), wv = ld16(a + (size_t)page * (D / 2) + ca);
        const char sk = a[sa], sv = a[sa + (size_t)page * (D / 32)];
        st16(o + co, wk);
        st16(o + (size_t)page * (D / 2) + co, wv);
        o[so] = sk;
        o[so + (size_t)page * (D / 32)] = sv;
    }
}

// ---------------------------------------------------------------------------
// rows of the cache as the values they stand for: kve_pages_read
// ---------------------------------------------------------------------------

// One workgroup per (segment, kRows rows), D / 8 lanes to a row.
template <typename T, int D>
__global__ __launch_bounds__(kThreads) void read_rows(PagePool p, int B, int cap, const int32_t* __restrict__ seq,
                                                      const int32_t* __restrict__ start,
                                                      const int32_t* __restrict__ count, char* __restrict__ k_out,
                                                      char* __restrict__ v_out, int nblk) {
    constexpr int kLanes = D / 8;
    constexpr int kStep = kThreads / kLanes;
    const int blk = blockIdx.x % nblk, seg = blockIdx.x / nblk;
    const int j = seg % p.Hkv, lb = seg / p.Hkv;
    const int l = lb / B, b = lb - l * B;
    const int n = count != nullptr ? min(count[b], cap) : cap;
    const int slot = slot_of(seq, b, p.S), first = start != nullptr ? start[b] : 0;
    if (blk * kRows >= n || slot < 0 || first < 0) return;
    const int have = length_of(p, slot);
    const int part = threadIdx.x % kLanes;
    const int page = 1 << p.shift;
    for (int m = blk * kRows + (int)threadIdx.x / kLanes; m < min(n, (blk + 1) * kRows); m += kStep) {
        if (m >= have - first) break;
        const int pos = first + m;
        const int pg = p.table[(size_t)slot * p.M + (pos >> p.shift)];
        if (pg < 0 || pg >= p.n_pages) continue;
        const char* block = page_block<D>(p, l, pg, j);
        const int tok = pos & (page - 1);
        const char* row = block + (size_t)tok * (D / 2) + part * 4;
        const char* scales = block + (size_t)page * D + (size_t)(part / 4) * page + tok;
        const size_t o = ((size_t)seg * cap + m) * (D * sizeof(T));
        if (k_out != nullptr)
            Eight<T>::store(k_out + o, part, *reinterpret_cast<const uint32_t*>(row),
                            scale_float((uint8_t)scales[0]));
        if (v_out != nullptr)
            Eight<T>::store(v_out + o, part, *reinterpret_cast<const uint32_t*>(row + (size_t)page * (D / 2)),
                            scale_float((uint8_t)scales[(size_t)page * (D / 32)]));
    }
}

// ---------------------------------------------------------------------------
// bookkeeping
// ---------------------------------------------------------------------------

constexpr int kPlanThreads = kPagesMaxEntries;
constexpr int kPlanWaves = kPlanThreads / kWave;

// Exclusive prefix sum over the workgroup; total in `total`.  s: kPlanWaves words of LDS.
__device__ __forceinline__ unsigned long long scan_exclusive(unsigned long long x, unsigned long long* s,
                                                             unsigned long long& total) {
    const int lane = threadIdx.x & (kWave - 1), w = threadIdx.x / kWave;
    unsigned long long inc = x;
#pragma unroll
    for (int o = 1; o < kWave; o <<= 1) {
        const unsigned long long y = __shfl_up(inc, o);
        if (lane >= o) inc += y;
    }
    __syncthreads();  // the last scan's sums are read
    if (lane == kWave - 1) s[w] = inc;
    __syncthreads();
    unsigned long long before = 0;
    total = 0;
#pragma unroll
    for (int i = 0; i < kPlanWaves; ++i) {
        const unsigned long long y = s[i];
        if (i < w) before += y;
        total += y;
    }
    return before + inc - x;
}

// The first `want` free pages in ascending order into list; returns how many
// there are (all free pages counted, where fewer than `want`).  Sixteen pages per
// thread and round, as four loads of four: the counts of the four loads, at most
// 4096 each, are scanned together as 16-bit fields.
__device__ int find_free(const int32_t* __restrict__ refs, int n_pages, int want, int32_t* __restrict__ list,
                         unsigned long long* s) {
    constexpr int kPer = 4, kLoads = 4;
    int found = 0;
    for (int base = 0; base < n_pages && found < want; base += kPlanThreads * kPer * kLoads) {
        uint32_t free[kLoads];
        unsigned long long counts = 0;
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            free[i] = 0;
            const int at = base + (i * kPlanThreads + (int)threadIdx.x) * kPer;
#pragma unroll
            for (int e = 0; e < kPer; ++e)
                if (at + e < n_pages && refs[at + e] == 0) free[i] |= 1u << e;
            counts |= (unsigned long long)__popc(free[i]) << (16 * i);
        }
        unsigned long long total;
        const unsigned long long before = scan_exclusive(counts, s, total);
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            int r = found + (int)((before >> (16 * i)) & 0xffff);
            const int at = base + (i * kPlanThreads + (int)threadIdx.x) * kPer;
            for (uint32_t f = free[i]; f != 0; f &= f - 1, ++r)
                if (r < want) list[r] = at + __ffs(f) - 1;
            found += (int)((total >> (16 * i)) & 0xffff);
        }
    }
    __syncthreads();  // list is whole
    return found;
}

// Whether an earlier entry names the same slot.  s_seq holds the entries' slots.
__device__ __forceinline__ bool named_before(const int* s_seq, int i, int slot) {
    bool hit = false;
    for (int e = 0; e < i; ++e) hit |= s_seq[e] == slot;
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
__global__ __launch_bounds__(kPlanThreads) void extend_kernel(PagePool p, const int32_t* __restrict__ seq,
                                                              const int32_t* __restrict__ add, int n,
                                                              int32_t* __restrict__ start,
                                                              int32_t* __restrict__ missing,
                                                              int32_t* __restrict__ list) {
    __shared__ int s_seq[kPlanThreads], s_off[kPlanThreads], s_held[kPlanThreads], s_ok[kPlanThreads];
    __shared__ unsigned long long s_scan[kPlanWaves];
    const int i = threadIdx.x;
    const int slot = i < n ? slot_of(seq, i, p.S) : -1;
    s_seq[i] = slot;
    __syncthreads();
    bool valid = slot >= 0 && !named_before(s_seq, i, slot);
    int held = 0, len = 0, more = 0;
    long long need = 0;
    if (valid) {
        held = held_of(p, slot);
        len = length_of(p, slot);
        more = add[i];
        const long long now = (long long)len + more;
        valid = more >= 0 && now <= (long long)p.M << p.shift;
        if (valid) need = max(0LL, ((now + (1 << p.shift) - 1) >> p.shift) - held);
    }
    unsigned long long total;
    const unsigned long long off = scan_exclusive((unsigned long long)need, s_scan, total);
    const int want = (int)min(total, (unsigned long long)p.n_pages);
    const int found = find_free(p.refs, p.n_pages, want, list, s_scan);
    const bool given = valid && (need == 0 || off + need <= (unsigned long long)found);
    s_off[i] = (int)min(off, (unsigned long long)p.n_pages);
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
    if (i == 0) *missing = (int)min(total - (unsigned long long)min(want, found), 2147483647ULL);
}

// What fork_copy does for an entry: full pages shared (-1: refused), the partial
// page's source and copy (copy < 0: none) and its rows.
struct ForkPlan {
    int full, from, to, rows;
};

__global__ __launch_bounds__(kPlanThreads) void fork_kernel(PagePool p, const int32_t* __restrict__ src,
                                                            const int32_t* __restrict__ dst, int n,
                                                            int32_t* __restrict__ done,
                                                            int32_t* __restrict__ missing,
                                                            ForkPlan* __restrict__ plan,
                                                            int32_t* __restrict__ list) {
    __shared__ int s_dst[kPlanThreads];
    __shared__ unsigned long long s_scan[kPlanWaves];
    const int i = threadIdx.x;
    const int from = i < n ? slot_of(src, i, p.S) : -1, to = i < n ? slot_of(dst, i, p.S) : -1;
    s_dst[i] = to;
    __syncthreads();
    const bool valid = from >= 0 && to >= 0 && !named_before(s_dst, i, to) && p.held[to] == 0 && p.length[to] == 0;
    const int len = valid ? length_of(p, from) : 0;
    const int full = len >> p.shift, rows = len & ((1 << p.shift) - 1);
    const int need = rows != 0 ? 1 : 0;
    unsigned long long total;
    const unsigned long long off = scan_exclusive((unsigned long long)need, s_scan, total);
    // all sources are read (the scan's barriers); destinations may be written
    const int found = find_free(p.refs, p.n_pages, (int)total, list, s_scan);
    const bool given = valid && (need == 0 || off < (unsigned long long)found);
    if (i < n) {
        ForkPlan f{given ? full : -1, -1, -1, rows};
        if (given) {
            if (need != 0) {
                f.from = p.table[(size_t)from * p.M + full];
                f.to = list[off];
                p.table[(size_t)to * p.M + full] = f.to;
                p.refs[f.to] = 1;
            }
            p.held[to] = full + need;
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
__global__ __launch_bounds__(kThreads) void fork_copy(PagePool p, const int32_t* __restrict__ src,
                                                      const int32_t* __restrict__ dst,
                                                      const ForkPlan* __restrict__ plan, int nblk) {
    const int i = blockIdx.x / (1 + p.L * nblk), part = blockIdx.x - i * (1 + p.L * nblk);
    const ForkPlan f = plan[i];
    if (f.full < 0) return;
    if (part == 0) {
        const int32_t* a = p.table + (size_t)src[i] * p.M;
        int32_t* o = p.table + (size_t)dst[i] * p.M;
        for (int e = threadIdx.x; e < f.full; e += kThreads) {
            const int pg = a[e];
            o[e] = pg;
            if (pg >= 0 && pg < p.n_pages) atomicAdd(p.refs + pg, 1);
        }
        return;
    }
    if (f.to < 0 || f.from < 0 || f.from >= p.n_pages) return;
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

template <typename T, int D>
void run_pack(const RowView& k, const RowView& v, int B, int N, const int32_t* idx, const int32_t* count, int cap,
              const int32_t* start, const int32_t* seq, const PagePool& p, hipStream_t st) {
    const int nblk = (cap + kRows - 1) / kRows;
    hipLaunchKernelGGL((pack_rows<T, D>), dim3((unsigned)p.L * B * p.Hkv * nblk), dim3(kThreads), 0, st, k, v, B, N,
                       idx, count, cap, start, seq, p, nblk);
}

template <typename T, int D>
void run_read(const PagePool& p, int B, int T_, const int32_t* seq, const int32_t* start, const int32_t* count,
              void* k_out, void* v_out, hipStream_t st) {
    const int nblk = (T_ + kRows - 1) / kRows;
    hipLaunchKernelGGL((read_rows<T, D>), dim3((unsigned)p.L * B * p.Hkv * nblk), dim3(kThreads), 0, st, p, B, T_,
                       seq, start, count, static_cast<char*>(k_out), static_cast<char*>(v_out), nblk);
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
    static_assert(sizeof(ForkPlan) == 16, "pages_workspace counts 16 bytes per entry");
    ForkPlan* plan = static_cast<ForkPlan*>(ws);
    int32_t* list = reinterpret_cast<int32_t*>(static_cast<char*>(ws) + align_up((size_t)n * sizeof(ForkPlan)));
    hipLaunchKernelGGL(fork_kernel, dim3(1), dim3(kPlanThreads), 0, st, p, src, dst, n, done, missing, plan, list);
    const int nblk = pages_copy_blocks(p.Hkv, 1 << p.shift, d);
    const dim3 grid((unsigned)n * (1 + p.L * nblk));
    if (d == 128)
        hipLaunchKernelGGL(fork_copy<128>, grid, dim3(kThreads), 0, st, p, src, dst, plan, nblk);
    else
        hipLaunchKernelGGL(fork_copy<64>, grid, dim3(kThreads), 0, st, p, src, dst, plan, nblk);
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
    const int nblk = (cap + kRows - 1) / kRows;
    const dim3 grid((unsigned)p.L * B * p.Hkv * nblk);
    if (d == 128)
        hipLaunchKernelGGL(select_rows<128>, grid, dim3(kThreads), 0, st, p, B, src, idx, count, cap, dst, start,
                           nblk);
    else
        hipLaunchKernelGGL(select_rows<64>, grid, dim3(kThreads), 0, st, p, B, src, idx, count, cap, dst, start,
                           nblk);
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
