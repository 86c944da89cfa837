// The paged 8-bit cache: the kernels that write rows into blocks (kve_blocks_append,
// kve_blocks_compact) and read rows and bounds back.
//
// A block's rows share one power of two (kve_blocks.h), so a workgroup takes the
// keys or the values of a whole block: it holds the new rows in registers, finds
// their largest magnitude, and packs them under the scale that comes of it.  The
// scaled conversions of gfx950 divide by the scale and round to the nearest, ties to
// even; the scales are kept where neither x nor x / scale is a denormal that counts.
#include "kve_blocks_device.h"
#include "kve_device.h"
#include "kve_internal.h"

namespace kve {
namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / kWave;

typedef short s16x2 __attribute__((ext_vector_type(2)));

// Eight channels of a row.  Once: non-temporal, for rows of a large tensor that are
// read once.
template <bool Once>
__device__ __forceinline__ u32x4 load16(const char* at) {
    if constexpr (Once) return __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(at));
    return ld16(at);
}

template <typename T>
struct Eight {
    static constexpr int kRegs = sizeof(T) / 2;
    u32x4 v[kRegs];
    template <bool Once>
    __device__ __forceinline__ void load(const char* row, int part) {
#pragma unroll
        for (int i = 0; i < kRegs; ++i) v[i] = load16<Once>(row + (part * kRegs + i) * 16);
    }
    __device__ __forceinline__ float get(int e) const {
        if constexpr (kRegs == 1) {
            const uint32_t w = v[0][e / 2];
            return __uint_as_float(e & 1 ? w & 0xffff0000u : w << 16);
        } else {
            return __uint_as_float(v[e / 4][e % 4]);
        }
    }
    __device__ __forceinline__ static void store(char* row, int part, const float (&x)[8]) {
        if constexpr (kRegs == 1) {
            u32x4 o;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const bf16x2 two = {(__bf16)x[2 * i], (__bf16)x[2 * i + 1]};
                o[i] = __builtin_bit_cast(uint32_t, two);
            }
            __builtin_nontemporal_store(o, reinterpret_cast<u32x4*>(row) + part);
        } else {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const f32x4 o = {x[4 * i], x[4 * i + 1], x[4 * i + 2], x[4 * i + 3]};
                __builtin_nontemporal_store(o, reinterpret_cast<f32x4*>(row) + 2 * part + i);
            }
        }
    }
};

// y to float32 so that a second rounding, to fewer bits, gives what rounding y
// once to those gives: truncated, with the last bit set where something was lost.
__device__ __forceinline__ float to_odd(double y) {
    const float f = (float)y;
    const double back = (double)f;
    if (back == y || !(fabs(y) < INFINITY)) return f;
    uint32_t bits = __float_as_uint(f);
    bits -= fabs(back) > fabs(y) ? 1u : 0u;
    return __uint_as_float(bits | 1u);
}

// Eight channels of a rotated row, exact to 53 bits.  row: its first byte; pos:
// position, outside [0, P) for none.
template <typename T, int D>
struct Turn {
    double y[8];
    __device__ __forceinline__ void load(const char* row, int part, int pos, const BlockRotation& r) {
        Eight<T> own;
        own.template load<false>(row, part);
        const bool there = pos >= 0 && pos < r.P;
        const int half = r.r / 2;
        if (8 * part >= r.r || !there) {
#pragma unroll
            for (int e = 0; e < 8; ++e) y[e] = there ? (double)own.get(e) : (double)__uint_as_float(0x7fc00000u);
            return;
        }
        const size_t base = (size_t)pos * half;
        if (r.pairs) {
            const f32x4 c = *reinterpret_cast<const f32x4*>(r.cos + base + 4 * part);
            const f32x4 s = *reinterpret_cast<const f32x4*>(r.sin + base + 4 * part);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const double a = own.get(2 * i), b = own.get(2 * i + 1), co = c[i], si = s[i];
                y[2 * i] = fma(a, co, -(b * si));
                y[2 * i + 1] = fma(b, co, a * si);
            }
            return;
        }
        const int parts = half / 8;
        const bool low = part < parts;
        Eight<T> other;
        other.template load<false>(row, low ? part + parts : part - parts);
        const size_t at = base + 8 * (low ? part : part - parts);
        f32x4 c[2], s[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            c[i] = *reinterpret_cast<const f32x4*>(r.cos + at + 4 * i);
            s[i] = *reinterpret_cast<const f32x4*>(r.sin + at + 4 * i);
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const double a = own.get(e), b = other.get(e), co = c[e / 4][e % 4], si = s[e / 4][e % 4];
            y[e] = fma(a, co, low ? -(b * si) : b * si);
        }
    }
};

// Scale byte of rows whose largest finite magnitude has these float32 bits.  448 is
// 1.75 * 2^8: what exceeds 1.75 of a power of two carries into the exponent.
__device__ __forceinline__ int scale_byte8(uint32_t top) {
    return min(max((int)((top + 0x1fffffu) >> 23) - 8, kBlockScaleMin), kBlockScaleMax);
}

// A float as it is rounded: infinities become NaN, and no more than 448 scales.
__device__ __forceinline__ float bounded(float x, float most) {
    return fabsf(x) < INFINITY ? fminf(fmaxf(x, -most), most) : __uint_as_float(0x7fc00000u);
}

// The smaller and the larger of two, NaN if one is.
__device__ __forceinline__ float lower(float a, float b) { return a < b || a != a ? a : b; }
__device__ __forceinline__ float higher(float a, float b) { return a > b || a != a ? a : b; }

__device__ __forceinline__ uint32_t codes4(float a, float b, float c, float d, float scale) {
    s16x2 w = {0, 0};
    w = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(w, a, b, scale, false);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(w, c, d, scale, true);
    return __builtin_bit_cast(uint32_t, w);
}

// Codes under another scale: rounded once more.
__device__ __forceinline__ uint32_t rescale4(uint32_t w, float factor) {
    float x[4];
    floats4(w, factor, x);
    return codes4(x[0], x[1], x[2], x[3], 1.0f);
}

// What a call writes.
struct WriteGrid {
    int B, T, N, nblk, nq;       // nblk: blocks per segment; nq: rows of queries
    unsigned blocks;             // workgroups that take blocks; those behind them take queries
};

// Row `in` of a step of kThreads / (D / 8).
template <int D>
struct Lanes {
    static constexpr int kRow = D / 8;                // lanes to a row
    static constexpr int kStep = kThreads / kRow;     // rows per step
    static constexpr int kInWave = kWave / kRow;
};

// A workgroup takes the keys or the values of one block of a segment (layer, sample,
// KV head), both and the heads of a page side by side: ITEMS rows per lane group.
// Behind them, kBlocksQueryRows rotated rows of the queries.
template <typename T, int D, int ITEMS, bool Gather>
__global__ __launch_bounds__(kThreads) void write_blocks(RowView kv, RowView vv, RowView qv, char* __restrict__ q_out,
                                                         int Hq, WriteGrid g, const int32_t* __restrict__ idx,
                                                         const int32_t* __restrict__ count,
                                                         const int32_t* __restrict__ start,
                                                         const int32_t* __restrict__ seq, BlockRotation rot,
                                                         PagePool p) {
    using Ln = Lanes<D>;
    const int part = threadIdx.x % Ln::kRow, in = threadIdx.x / Ln::kRow;
    if constexpr (!Gather) {
        if (blockIdx.x >= g.blocks) {
            const unsigned first = (blockIdx.x - g.blocks) * kBlocksQueryRows;
#pragma unroll 1
            for (int i = 0; i < kBlocksQueryRows; i += Ln::kStep) {
                const unsigned row = first + i + in;
                if (row >= (unsigned)g.nq) return;
                const unsigned lbh = row / (unsigned)g.T, t = row - lbh * g.T;
                const unsigned lb = lbh / (unsigned)Hq, h = lbh - lb * Hq;
                const unsigned l = lb / (unsigned)g.B, b = lb - l * g.B;
                Turn<T, D> x;
                x.load(qv.base + (size_t)l * qv.s_layer + (size_t)b * qv.s_batch + (size_t)h * qv.s_head +
                           (size_t)t * qv.s_token,
                       part, rot.position[(size_t)b * g.T + t], rot);
                float y[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) y[e] = sizeof(T) == 2 ? to_odd(x.y[e]) : (float)x.y[e];
                Eight<T>::store(q_out + (size_t)row * (D * sizeof(T)), part, y);
            }
            return;
        }
    }
    __shared__ uint32_t s_top[kWaves];
    __shared__ float s_lo[kWaves][D], s_hi[kWaves][D];
    const unsigned role = blockIdx.x & 1, x2 = blockIdx.x >> 1;
    const unsigned x1 = x2 / (unsigned)p.Hkv, lb = x1 / (unsigned)g.nblk;
    const int j = (int)(x2 - x1 * p.Hkv), i = (int)(x1 - lb * g.nblk);
    const int l = (int)(lb / (unsigned)g.B), b = (int)(lb - (unsigned)l * g.B);
    const size_t seg = (size_t)lb * p.Hkv + j;
    const int slot = slot_of(seq, b, p.S), s0 = start[b];
    const int n = Gather ? min(count[seg], g.T) : count != nullptr ? min(count[b], g.T) : g.T;
    if (slot < 0 || s0 < 0 || n <= 0) return;
    const int limit = held_of(p, slot) << p.shift;  // positions that there are
    if (s0 >= limit) return;
    const int at = (s0 >> p.shift) + i;             // block of the sequence
    const long long pos0 = (long long)at << p.shift;
    const int r0 = (int)max(0LL, s0 - pos0), r1 = (int)min((long long)1 << p.shift, s0 + (long long)n - pos0);
    if (pos0 >= limit || r1 <= r0) return;
    const int pg = p.table[(size_t)slot * p.M + at];
    if (pg < 0 || pg >= p.n_pages) return;
    char* block = block_at<D>(p, l, pg, j);
    char* tail = block + tail_at<D>(p.shift);
    char* codes = block + ((size_t)(role * D) << p.shift);
    const int old = r0 > 0 ? scale_of((uint8_t)tail[role]) : 0;

    // the rows, their largest magnitude
    float x[ITEMS][8];
    uint32_t top = 0;
    const RowView& view = role == 0 ? kv : vv;
    const char* base = view.base + (size_t)l * view.s_layer + (size_t)b * view.s_batch + (size_t)j * view.s_head;
#pragma unroll
    for (int it = 0; it < ITEMS; ++it) {
        const int row = it * Ln::kStep + in;
        if (row < r0 || row >= r1) continue;
        const int m = (int)(pos0 + row - s0);
        if (Gather) {
            const int t = idx[seg * g.T + m];
            if (t >= 0 && t < g.N) {
                Eight<T> raw;
                raw.template load<true>(base + (size_t)t * view.s_token, part);
#pragma unroll
                for (int e = 0; e < 8; ++e) x[it][e] = raw.get(e);
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) x[it][e] = 0.0f;
            }
        } else if (role == 0 && rot.cos != nullptr) {
            Turn<T, D> y;
            y.load(base + (size_t)m * view.s_token, part, rot.position[(size_t)b * g.T + m], rot);
#pragma unroll
            for (int e = 0; e < 8; ++e) x[it][e] = to_odd(y.y[e]);
        } else {
            Eight<T> raw;
            raw.template load<false>(base + (size_t)m * view.s_token, part);
#pragma unroll
            for (int e = 0; e < 8; ++e) x[it][e] = raw.get(e);
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const uint32_t bits = __float_as_uint(x[it][e]) & 0x7fffffffu;
            top = max(top, bits < 0x7f800000u ? bits : 0u);
        }
    }
#pragma unroll
    for (int s = 1; s < kWave; s <<= 1) top = max(top, (uint32_t)__shfl_xor((int)top, s));
    const int lane = threadIdx.x & (kWave - 1), wv = threadIdx.x / kWave;
    if (lane == 0) s_top[wv] = top;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kWaves; ++w) top = max(top, s_top[w]);
    const int s = max(scale_byte8(top), old);
    const float scale = scale_float(s), most = 448.0f * scale;
    // rows under another scale: 2^-60 of it is zero like any smaller share
    const float factor = scale_float(127 - min(s - old, 60));

    float lo[8], hi[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        lo[e] = INFINITY;
        hi[e] = -INFINITY;
    }
#pragma unroll
    for (int it = 0; it < ITEMS; ++it) {
        const int row = it * Ln::kStep + in;
        if (row >= r1) continue;
        u32x2* at8 = reinterpret_cast<u32x2*>(codes + (size_t)row * D) + part;
        if (row < r0) {
            if (s == old) continue;
            u32x2 w = *at8;
            w[0] = rescale4(w[0], factor);
            w[1] = rescale4(w[1], factor);
            *at8 = w;
            continue;
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            x[it][e] = bounded(x[it][e], most);
            lo[e] = lower(lo[e], x[it][e]);
            hi[e] = higher(hi[e], x[it][e]);
        }
        u32x2 w;
        w[0] = codes4(x[it][0], x[it][1], x[it][2], x[it][3], scale);
        w[1] = codes4(x[it][4], x[it][5], x[it][6], x[it][7], scale);
        *at8 = w;
    }
    if (threadIdx.x == 0) tail[role] = (char)s;
    if (role != 0) return;
    // bounds: rounding keeps the order, so the bounds of the codes are the codes of the bounds
#pragma unroll
    for (int st = Ln::kRow; st < kWave; st <<= 1)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            lo[e] = lower(lo[e], __shfl_xor(lo[e], st));
            hi[e] = higher(hi[e], __shfl_xor(hi[e], st));
        }
    if (lane < Ln::kRow)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            s_lo[wv][8 * part + e] = lo[e];
            s_hi[wv][8 * part + e] = hi[e];
        }
    __syncthreads();
    // four channels of one bound to a thread
    if (threadIdx.x >= 2 * D / 4) return;
    const int ch = threadIdx.x * 4 % D;
    const bool upper = threadIdx.x * 4 >= D;
    uint32_t* out = reinterpret_cast<uint32_t*>(tail + kBlockScales) + threadIdx.x;
    float y[4], was[4];
    if (r0 > 0) floats4(rescale4(*out, factor), 1.0f, was);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        y[e] = upper ? s_hi[0][ch + e] : s_lo[0][ch + e];
#pragma unroll
        for (int w = 1; w < kWaves; ++w)
            y[e] = upper ? higher(y[e], s_hi[w][ch + e]) : lower(y[e], s_lo[w][ch + e]);
        // in units of the scale: old bounds are codes already
        if (r0 > 0) y[e] = upper ? higher(y[e], was[e] * scale) : lower(y[e], was[e] * scale);
    }
    *out = codes4(y[0], y[1], y[2], y[3], scale);
}

// ---------------------------------------------------------------------------
// rows and bounds out of blocks
// ---------------------------------------------------------------------------

struct ReadGrid {
    int B, cap;
    uint32_t rows;  // of all segments
};

// D / 8 lanes to a row, rows of all segments one after the other.  Bounds: row m is
// block first + m's bound, else the row at position first + m.
template <typename T, int D, bool Bounds>
__global__ __launch_bounds__(kThreads) void read_blocks(PagePool p, ReadGrid g, const int32_t* __restrict__ seq,
                                                        const int32_t* __restrict__ first,
                                                        const int32_t* __restrict__ count, char* __restrict__ a_out,
                                                        char* __restrict__ b_out) {
    using Ln = Lanes<D>;
    const int part = threadIdx.x % Ln::kRow;
    const uint32_t at = blockIdx.x * (uint32_t)Ln::kStep + threadIdx.x / Ln::kRow;
    if (at >= g.rows) return;
    const uint32_t seg = at / (uint32_t)g.cap, m = at - seg * g.cap;
    const uint32_t lb = seg / (uint32_t)p.Hkv, j = seg - lb * p.Hkv;
    const uint32_t l = lb / (uint32_t)g.B, b = lb - l * g.B;
    const int slot = slot_of(seq, b, p.S);
    if (slot < 0 || (count != nullptr && (int)m >= count[b])) return;
    const int from = first != nullptr ? first[b] : 0;
    const int len = length_of(p, slot), end = Bounds ? (len + (1 << p.shift) - 1) >> p.shift : len;
    if (from < 0 || (long long)from + m >= end) return;
    const int pos = from + (int)m, blk = Bounds ? pos : pos >> p.shift;
    const int pg = p.table[(size_t)slot * p.M + blk];
    if (pg < 0 || pg >= p.n_pages) return;
    const char* block = block_at<D>(p, l, pg, j);
    const char* tail = block + tail_at<D>(p.shift);
    const int tok = pos & ((1 << p.shift) - 1);
    const char* rows[2] = {Bounds ? tail + kBlockScales : block + (size_t)tok * D,
                           Bounds ? tail + kBlockScales + D : block + ((size_t)D << p.shift) + (size_t)tok * D};
    const u32x2 a = reinterpret_cast<const u32x2*>(rows[0])[part], c = reinterpret_cast<const u32x2*>(rows[1])[part];
    const uint32_t scales = *reinterpret_cast<const uint16_t*>(tail);
    const size_t out = (size_t)at * (D * sizeof(T));
    auto give = [&](char* o, u32x2 w, uint32_t s) {
        float x[8];
        const float unit = scale_float(scale_of((uint8_t)s));
        floats4(w[0], unit, *reinterpret_cast<float(*)[4]>(x));
        floats4(w[1], unit, *reinterpret_cast<float(*)[4]>(x + 4));
        Eight<T>::store(o + out, part, x);
    };
    if (a_out != nullptr) give(a_out, a, scales);
    if (b_out != nullptr) give(b_out, c, Bounds ? scales : scales >> 8);
}

template <typename T, int D, int ITEMS>
void run_write(const RowView& k, const RowView& v, const RowView& q, char* q_out, int Hq, const WriteGrid& g,
               unsigned groups, const int32_t* idx, const int32_t* count, const int32_t* start, const int32_t* seq,
               const BlockRotation& rot, const PagePool& p, hipStream_t st) {
    if (idx != nullptr)
        hipLaunchKernelGGL((write_blocks<T, D, ITEMS, true>), dim3(groups), dim3(kThreads), 0, st, k, v, q, q_out, Hq,
                           g, idx, count, start, seq, rot, p);
    else
        hipLaunchKernelGGL((write_blocks<T, D, ITEMS, false>), dim3(groups), dim3(kThreads), 0, st, k, v, q, q_out, Hq,
                           g, idx, count, start, seq, rot, p);
}

template <typename T, int D>
void run_write(const RowView& k, const RowView& v, const RowView& q, char* q_out, int Hq, const WriteGrid& g,
               unsigned groups, const int32_t* idx, const int32_t* count, const int32_t* start, const int32_t* seq,
               const BlockRotation& rot, const PagePool& p, hipStream_t st) {
    constexpr int kStep = Lanes<D>::kStep;
    if (p.shift == 5)
        run_write<T, D, 32 / kStep>(k, v, q, q_out, Hq, g, groups, idx, count, start, seq, rot, p, st);
    else if (p.shift == 6)
        run_write<T, D, 64 / kStep>(k, v, q, q_out, Hq, g, groups, idx, count, start, seq, rot, p, st);
    else
        run_write<T, D, 128 / kStep>(k, v, q, q_out, Hq, g, groups, idx, count, start, seq, rot, p, st);
}

template <typename T, int D, bool Bounds>
void run_read(const PagePool& p, int B, int cap, const int32_t* seq, const int32_t* first, const int32_t* count,
              void* a, void* b, hipStream_t st) {
    const ReadGrid g{B, cap, (uint32_t)p.L * B * p.Hkv * (uint32_t)cap};
    const unsigned groups = (g.rows + Lanes<D>::kStep - 1) / Lanes<D>::kStep;
    hipLaunchKernelGGL((read_blocks<T, D, Bounds>), dim3(groups), dim3(kThreads), 0, st, p, g, seq, first, count,
                       static_cast<char*>(a), static_cast<char*>(b));
}

template <bool Bounds>
hipError_t read_any(const PagePool& p, int dtype, int d, int B, int cap, const int32_t* seq, const int32_t* first,
                    const int32_t* count, void* a, void* b, hipStream_t st) {
    if (cap == 0) return hipSuccess;
    if (dtype == 0 && d == 128) run_read<__bf16, 128, Bounds>(p, B, cap, seq, first, count, a, b, st);
    if (dtype == 0 && d == 64) run_read<__bf16, 64, Bounds>(p, B, cap, seq, first, count, a, b, st);
    if (dtype == 1 && d == 128) run_read<float, 128, Bounds>(p, B, cap, seq, first, count, a, b, st);
    if (dtype == 1 && d == 64) run_read<float, 64, Bounds>(p, B, cap, seq, first, count, a, b, st);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_blocks_write(const RowView& k, const RowView& v, const RowView& q, void* q_out, int Hq, int dtype,
                               int d, int B, int N, const int32_t* idx, const int32_t* count, int cap,
                               const int32_t* start, const int32_t* seq, const BlockRotation& rot, const PagePool& p,
                               hipStream_t st) {
    if (cap == 0) return hipSuccess;
    WriteGrid g{B, cap, N, (int)blocks_touched(cap, 1 << p.shift), 0, 0};
    g.blocks = 2u * p.L * B * p.Hkv * g.nblk;
    if (q_out != nullptr) g.nq = p.L * B * Hq * cap;
    const unsigned groups = g.blocks + (unsigned)(g.nq + kBlocksQueryRows - 1) / kBlocksQueryRows;
    char* o = static_cast<char*>(q_out);
    if (dtype == 0 && d == 128) run_write<__bf16, 128>(k, v, q, o, Hq, g, groups, idx, count, start, seq, rot, p, st);
    if (dtype == 0 && d == 64) run_write<__bf16, 64>(k, v, q, o, Hq, g, groups, idx, count, start, seq, rot, p, st);
    if (dtype == 1 && d == 128) run_write<float, 128>(k, v, q, o, Hq, g, groups, idx, count, start, seq, rot, p, st);
    if (dtype == 1 && d == 64) run_write<float, 64>(k, v, q, o, Hq, g, groups, idx, count, start, seq, rot, p, st);
    return hipGetLastError();
}

hipError_t launch_blocks_read(const PagePool& p, int dtype, int d, int B, int T, const int32_t* seq,
                              const int32_t* start, const int32_t* count, void* k_out, void* v_out, hipStream_t st) {
    return read_any<false>(p, dtype, d, B, T, seq, start, count, k_out, v_out, st);
}

hipError_t launch_blocks_bounds(const PagePool& p, int dtype, int d, int B, int n, const int32_t* seq,
                                const int32_t* first, void* lo, void* hi, hipStream_t st) {
    return read_any<true>(p, dtype, d, B, n, seq, first, nullptr, lo, hi, st);
}

}  // namespace kve
