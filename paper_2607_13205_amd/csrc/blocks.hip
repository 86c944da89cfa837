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
    // Once: non-temporal, for what is not read soon.
    template <bool Once>
    __device__ __forceinline__ static void store(char* row, int part, const float (&x)[8]) {
        u32x4 o[kRegs];
        if constexpr (kRegs == 1) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const bf16x2 two = {(__bf16)x[2 * i], (__bf16)x[2 * i + 1]};
                o[0][i] = __builtin_bit_cast(uint32_t, two);
            }
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) o[i / 4][i % 4] = __float_as_uint(x[i]);
        }
#pragma unroll
        for (int i = 0; i < kRegs; ++i) {
            u32x4* at = reinterpret_cast<u32x4*>(row) + part * kRegs + i;
            if constexpr (Once)
                __builtin_nontemporal_store(o[i], at);
            else
                *at = o[i];
        }
    }
};

// y to float32 so that a second rounding, to fewer bits, gives what rounding y
// once to those gives: truncated, with the last bit set where something was lost.
__device__ __forceinline__ float to_odd(double y) {
    const float f = (float)y;
    const double back = (double)f;
    const uint32_t bits = __float_as_uint(f);
    const bool kept = back == y | !(fabs(y) < INFINITY);
    return __uint_as_float(kept ? bits : (bits - (uint32_t)(fabs(back) > fabs(y))) | 1u);
}

// A lane of a turned row takes two pieces of eight channels, `a` and `b`, which hold
// all of its pairs; they lie beside those of its neighbours where they can, so that a
// load or store of a wave covers whole lines.
struct Pieces {
    int a, b;
    bool turned;
};

template <int D>
__device__ __forceinline__ Pieces pieces_of(int part, const BlockRotation& r) {
    const int n = r.r / 16;  // lanes whose pieces are turned
    if (part >= n) return Pieces{n + part, D / 16 + part, false};
    return r.pairs ? Pieces{2 * part, 2 * part + 1, true} : Pieces{part, part + n, true};
}

// The angles of a lane's eight pairs at a position; none outside [0, P).
struct Angles {
    f32x4 cos[2], sin[2];
    bool there;
    __device__ __forceinline__ void load(int part, int pos, const BlockRotation& r, bool turned) {
        there = pos >= 0 && pos < r.P;
        if (!turned || !there) return;
        const size_t at = (size_t)pos * (r.r / 2) + 8 * part;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            cos[i] = *reinterpret_cast<const f32x4*>(r.cos + at + 4 * i);
            sin[i] = *reinterpret_cast<const f32x4*>(r.sin + at + 4 * i);
        }
    }
};

// The larger of two, NaN if one is: what float32 could not hold shows in a maximum.
__device__ __forceinline__ float larger(float a, float b) { return __builtin_elementwise_maximum(a, b); }

// How a turned channel becomes a float: as it is rounded once more, to an E4M3 or to
// bfloat16 (Odd and Half), or as the result itself (Float).
enum class Turned { Odd, Half, Float };

// Two pieces of a row.
template <typename T>
struct Sixteen {
    Eight<T> a, b;
    __device__ __forceinline__ void load(const char* row, const Pieces& at) {
        a.template load<false>(row, at.a);
        b.template load<false>(row, at.b);
    }
    // Pair i of a row's pieces: neighbours of one (Pairs), or channels i of the two.
    template <bool Pairs>
    static constexpr int first(int i) { return Pairs ? 2 * i : i; }
    template <bool Pairs>
    static constexpr int second(int i) { return Pairs ? 2 * i + 1 : 8 + i; }
    // Turned in 32 bits with the products' errors: y is off by less than three steps of
    // float32 (u c - p is rounded once, and the sum with the exact error of p once, each by
    // half a step, where the error is not what is left of it).  That decides every later
    // rounding unless a border of one lies within three steps: borders of E4M3 end in 16
    // zero bits, those of bfloat16 in a one and 15 zeros.  Returns whether all are decided;
    // 64 bits otherwise (a chunk of 1003 tokens, 32 and 8 heads: 25.6 us with 64 bits
    // throughout).  Products that leave float32, and those of infinities, make infinities or
    // NaN here where y may be neither: both are above `most`'s limit.
    template <Turned How, bool Pairs>
    __device__ __forceinline__ static bool fast(const float (&x)[16], const Angles& g, float (&y)[16]) {
        uint32_t border = 0xffffu;
        float clear = INFINITY, most = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float u = x[first<Pairs>(i)], w = x[second<Pairs>(i)];
            const float c = g.cos[i / 4][i % 4], s = g.sin[i / 4][i % 4];
            const float p = w * s, q = u * s, ep = fmaf(w, s, -p), eq = fmaf(u, s, -q);
            const float lo = fmaf(u, c, -p) - ep, hi = fmaf(w, c, q) + eq;
            constexpr uint32_t kAt = How == Turned::Half ? 0x8003u : 3u;
            border = min(border, min((__float_as_uint(lo) + kAt) & 0xffffu, (__float_as_uint(hi) + kAt) & 0xffffu));
            clear = fminf(clear, fminf(fmaf(-4.0f, fabsf(ep), fabsf(lo)), fmaf(-4.0f, fabsf(eq), fabsf(hi))));
            most = larger(most, larger(fabsf(lo), fabsf(hi)));
            y[first<Pairs>(i)] = lo;
            y[second<Pairs>(i)] = hi;
        }
        return border > 6 && clear > 0x1p-90f && most < 0x1p120f;
    }
    template <Turned How, bool Pairs>
    __device__ __forceinline__ static void turn(const Angles& g, float (&x)[16]) {
        float y[16];
        if (How == Turned::Float || !fast<How, Pairs>(x, g, y)) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const double u = x[first<Pairs>(i)], w = x[second<Pairs>(i)];
                const double c = g.cos[i / 4][i % 4], s = g.sin[i / 4][i % 4];
                const double lo = fma(u, c, -(w * s)), hi = fma(w, c, u * s);
                y[first<Pairs>(i)] = How == Turned::Float ? (float)lo : to_odd(lo);
                y[second<Pairs>(i)] = How == Turned::Float ? (float)hi : to_odd(hi);
            }
        }
#pragma unroll
        for (int e = 0; e < 16; ++e) x[e] = y[e];
    }
    template <Turned How>
    __device__ __forceinline__ void turn(const Angles& g, bool pairs, bool turned, float (&x)[16]) const {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            x[e] = a.get(e);
            x[8 + e] = b.get(e);
        }
        if (!g.there) {
#pragma unroll
            for (int e = 0; e < 16; ++e) x[e] = __uint_as_float(0x7fc00000u);
        } else if (turned) {
            if (pairs)
                turn<How, true>(g, x);
            else
                turn<How, false>(g, x);
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

template <int CTRL>
__device__ __forceinline__ uint32_t dpp(uint32_t x) {
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, 0xf, 0xf, false);
}

// Largest x of a wave, in every lane.
__device__ __forceinline__ uint32_t wave_max(uint32_t x) {
    x = max(x, dpp<0xb1>(x));   // lanes 1 0 3 2
    x = max(x, dpp<0x4e>(x));   // lanes 2 3 0 1
    x = max(x, dpp<0x141>(x));  // mirrored within eight
    x = max(x, dpp<0x140>(x));  // within sixteen
    const auto a = __builtin_amdgcn_permlane16_swap(x, x, false, false);  // lane ^ 16 and the lane itself
    x = max((uint32_t)a[0], (uint32_t)a[1]);
    const auto b = __builtin_amdgcn_permlane32_swap(x, x, false, false);
    return max((uint32_t)b[0], (uint32_t)b[1]);
}

// f over the four rows of sixteen lanes of a wave, of N values of each lane: a swap of
// halves leaves either half of the lanes with half of the values, each beside that of
// the other half.  Lane l is left with values N / 4 ((l >> 4 & 1) + 2 (l >> 5)) .. + N / 4,
// in x[0 .. N / 4).
template <int N, typename F>
__device__ __forceinline__ void over_quarters(float (&x)[N], F f) {
#pragma unroll
    for (int e = 0; e < N / 2; ++e) {
        const auto r =
            __builtin_amdgcn_permlane32_swap(__float_as_uint(x[e]), __float_as_uint(x[e + N / 2]), false, false);
        x[e] = f(__uint_as_float(r[0]), __uint_as_float(r[1]));
    }
#pragma unroll
    for (int e = 0; e < N / 4; ++e) {
        const auto r =
            __builtin_amdgcn_permlane16_swap(__float_as_uint(x[e]), __float_as_uint(x[e + N / 4]), false, false);
        x[e] = f(__uint_as_float(r[0]), __uint_as_float(r[1]));
    }
}

// The smallest and largest of three, a quiet NaN passed over (fminf spends an
// instruction on what could be a signalling one).
__device__ __forceinline__ float min3(float a, float b, float c) {
    float r;
    asm("v_min3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
    return r;
}
__device__ __forceinline__ float max3(float a, float b, float c) {
    float r;
    asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
    return r;
}

// What a call writes.
struct WriteGrid {
    int B, T, N, nblk, heads;  // nblk: blocks per segment; heads: of the queries
    unsigned blocks, tokens;   // workgroups that take blocks, those behind them take queries; B T
};

// Partial bounds that a wave leaves: its rows are D / 16 lanes wide at least.
template <int D>
constexpr int kParts = 256 / D;

// NP pieces of eight channels to a lane.
template <int D, int NP>
struct Lanes {
    static constexpr int kRow = D / 8 / NP;        // lanes to a row
    static constexpr int kStep = kThreads / kRow;  // rows per step
};

// kBlocksQueryHeads heads of the queries of Lanes::kStep tokens, whose angles are loaded
// once.  Lines: a wave's store covers whole lines.  Those go past the caches (4 samples of
// 4000 tokens, 32 heads 73 us, 80 through them); others meet their other halves there (32
// of 2173 tokens, 16 heads, 16 turned channels 137 us, 187 past them).
template <typename T, int D, bool Lines>
__device__ __forceinline__ void queries_turned(const RowView& view, char* out, const WriteGrid& g, unsigned x,
                                               const BlockRotation& rot) {
    using Ln = Lanes<D, 2>;
    const unsigned sets = (unsigned)(g.heads + kBlocksQueryHeads - 1) / kBlocksQueryHeads;
    const unsigned y = x / sets, h0 = (x - y * sets) * kBlocksQueryHeads;
    const unsigned groups = (g.tokens + Ln::kStep - 1) / Ln::kStep, l = y / groups;
    const unsigned token = (y - l * groups) * Ln::kStep + threadIdx.x / Ln::kRow;
    if (token >= g.tokens) return;
    const int part = threadIdx.x % Ln::kRow;
    const Pieces at = pieces_of<D>(part, rot);
    const unsigned b = token / (unsigned)g.T, t = token - b * g.T;
    const char* row = view.base + (size_t)l * view.s_layer + (size_t)b * view.s_batch + (size_t)t * view.s_token;
    const int pos = rot.position[token];
    Sixteen<T> raw[kBlocksQueryHeads];
#pragma unroll
    for (int h = 0; h < kBlocksQueryHeads; ++h)
        raw[h].load(row + (size_t)min((int)h0 + h, g.heads - 1) * view.s_head, at);
    Angles angles;
    angles.load(part, pos, rot, at.turned);
#pragma unroll
    for (int h = 0; h < kBlocksQueryHeads; ++h) {
        if ((int)h0 + h >= g.heads) break;
        float z[16];
        raw[h].template turn<sizeof(T) == 2 ? Turned::Half : Turned::Float>(angles, !Lines && rot.pairs, at.turned, z);
        char* o = out + ((((size_t)l * g.B + b) * g.heads + h0 + h) * g.T + t) * (D * sizeof(T));
        Eight<T>::template store<Lines>(o, at.a, *reinterpret_cast<const float(*)[8]>(z));
        Eight<T>::template store<Lines>(o, at.b, *reinterpret_cast<const float(*)[8]>(z + 8));
    }
}

template <typename T, int D>
__device__ __forceinline__ void turn_queries(const RowView& view, char* out, const WriteGrid& g, unsigned x,
                                             const BlockRotation& rot) {
    if (sizeof(T) == 2 && rot.r == D && !rot.pairs)
        queries_turned<T, D, sizeof(T) == 2>(view, out, g, x, rot);
    else
        queries_turned<T, D, false>(view, out, g, x, rot);
}

// The keys or the values (Ends: keys) of one block: NP pieces to a lane, ITEMS rows to
// a lane group.  A decode step's call is a chain of memory latencies (slot, place,
// page, the block's scale), so everything is loaded as soon as its address is known:
// the new rows and their angles beside the look-up of the block.
template <typename T, int D, int PAGE, int NP, bool Gather, bool Ends>
__device__ __forceinline__ void write_block(uint32_t* s_top, float (*s_ends)[kWaves * kParts<D>][D],
                                            const RowView& view, int role, const WriteGrid& g, int l, int b, int j,
                                            int i, size_t seg, const int32_t* idx, int slot, int s0, int n,
                                            const BlockRotation& rot, const PagePool& p) {
    using Ln = Lanes<D, NP>;
    constexpr int ITEMS = (PAGE + Ln::kStep - 1) / Ln::kStep, kShift = PAGE == 32 ? 5 : PAGE == 64 ? 6 : 7;
    const int part = threadIdx.x % Ln::kRow, in = threadIdx.x / Ln::kRow;
    const int at = min((s0 >> kShift) + i, p.M);   // block of the sequence
    const int page = p.table[(size_t)slot * p.M + min(at, p.M - 1)], held = held_of(p, slot);
    const long long pos0 = (long long)at << kShift;
    const int r0 = (int)max(0LL, s0 - pos0), r1 = (int)min((long long)PAGE, s0 + (long long)n - pos0);
    if (r1 <= r0) return;

    Pieces pc{part, 0, false};
    if constexpr (NP == 2) pc = pieces_of<D>(part, rot);
    const char* base = view.base + (size_t)l * view.s_layer + (size_t)b * view.s_batch + (size_t)j * view.s_head;
    Sixteen<T> two[NP == 2 ? ITEMS : 1];
    Eight<T> one[NP == 1 ? ITEMS : 1];
    Angles angles[NP == 2 ? ITEMS : 1];
    int from[ITEMS];  // the source row, then its position
#pragma unroll
    for (int it = 0; it < ITEMS; ++it) {
        const int row = it * Ln::kStep + in;
        const int m = (int)(pos0 + min(max(row, r0), r1 - 1) - s0);
        from[it] = Gather ? idx[seg * g.T + m] : m;
    }
#pragma unroll
    for (int it = 0; it < ITEMS; ++it) {
        const int row = it * Ln::kStep + in;
        const bool there = row >= r0 && row < r1 && (!Gather || (from[it] >= 0 && from[it] < g.N));
        const char* at_row = base + (size_t)from[it] * view.s_token;
        if constexpr (NP == 2) {
            two[it] = Sixteen<T>{};
            if (there) two[it].load(at_row, pc);
        } else {
            one[it] = Eight<T>{};
            if (there) one[it].template load<Gather>(at_row, pc.a);
        }
    }
    if constexpr (NP == 2) {
#pragma unroll
        for (int it = 0; it < ITEMS; ++it) from[it] = rot.position[(size_t)b * g.T + from[it]];
#pragma unroll
        for (int it = 0; it < ITEMS; ++it) angles[it].load(part, from[it], rot, pc.turned);
    }
    if (at >= held || page < 0 || page >= p.n_pages) return;
    char* block = block_at<D>(p, l, page, j);
    char* tail = block + tail_at<D>(kShift);
    char* codes = block + role * D * PAGE;
    const int old = r0 > 0 ? scale_of((uint8_t)tail[role]) : 0;
    // a channel of one bound to a thread
    char* end = tail + kBlockScales + threadIdx.x % (2 * D);
    const uint32_t old_end = Ends && r0 > 0 ? (uint8_t)*end : 0u;

    // the rows' largest magnitude; rows that there are not are zeros
    float x[ITEMS][NP][8];
    uint32_t top = 0;
#pragma unroll
    for (int it = 0; it < ITEMS; ++it) {
        if constexpr (NP == 2) {
            const int row = it * Ln::kStep + in;
            if (row >= r0 && row < r1) {
                float y[16];
                two[it].template turn<Turned::Odd>(angles[it], rot.pairs, pc.turned, y);
#pragma unroll
                for (int e = 0; e < 16; ++e) x[it][e / 8][e % 8] = y[e];
            } else {
#pragma unroll
                for (int e = 0; e < 16; ++e) x[it][e / 8][e % 8] = 0.0f;
            }
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) x[it][0][e] = one[it].get(e);
        }
#pragma unroll
        for (int e = 0; e < 8 * NP; ++e) top = max(top, __float_as_uint(x[it][e / 8][e % 8]) & 0x7fffffffu);
    }
    const int lane = threadIdx.x & (kWave - 1), wv = threadIdx.x / kWave;
    auto over_all = [&](uint32_t y) {
        y = wave_max(y);
        if (lane == 0) s_top[wv] = y;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < kWaves; ++w) y = max(y, s_top[w]);
        return (uint32_t)__builtin_amdgcn_readfirstlane((int)y);
    };
    top = over_all(top);
    bool careful = top >= 0x7f800000u;
    if (careful) {  // once more, of the finite ones
        uint32_t finite = 0;
#pragma unroll
        for (int it = 0; it < ITEMS; ++it)
#pragma unroll
            for (int e = 0; e < 8 * NP; ++e) {
                const uint32_t bits = __float_as_uint(x[it][e / 8][e % 8]) & 0x7fffffffu;
                finite = max(finite, bits < 0x7f800000u ? bits : 0u);
            }
        __syncthreads();  // s_top is read
        top = over_all(finite);
    }
    const int s = max(scale_byte8(top), old);
    careful |= s == kBlockScaleMax;
    const float scale = scale_float(s);
    // rows under another scale: 2^-60 of it is zero like any smaller share
    const float factor = scale_float(127 - min(s - old, 60));

    const bool single = r1 - r0 == 1;
    const bool whole = r0 == 0 && r1 == PAGE && PAGE % Ln::kStep == 0;
    float lo[8 * NP], hi[8 * NP];
    if (careful) {
#pragma unroll
        for (int it = 0; it < ITEMS; ++it)
#pragma unroll
            for (int e = 0; e < 8 * NP; ++e) {
                const int row = it * Ln::kStep + in;
                float& y = x[it][e / 8][e % 8];
                y = bounded(y, 448.0f * scale);
                const bool there = row >= r0 && row < r1;
                lo[e] = lower(it == 0 ? INFINITY : lo[e], there ? y : INFINITY);
                hi[e] = higher(it == 0 ? -INFINITY : hi[e], there ? y : -INFINITY);
            }
    }
#pragma unroll
    for (int it = 0; it < ITEMS; ++it) {
        const int row = it * Ln::kStep + in;
        if (row < r0 || row >= r1) continue;
        u32x2* here = reinterpret_cast<u32x2*>(codes + row * D);
#pragma unroll
        for (int k = 0; k < NP; ++k) {
            const float(&y)[8] = x[it][k];
            here[k == 0 ? pc.a : pc.b] =
                u32x2{codes4(y[0], y[1], y[2], y[3], scale), codes4(y[4], y[5], y[6], y[7], scale)};
        }
    }
    if (s != old && r0 > 0) {  // what was there, 16 bytes at a time
        for (int e = threadIdx.x; e < r0 * (D / 16); e += kThreads) {
            u32x4* here = reinterpret_cast<u32x4*>(codes) + e;
            u32x4 w = *here;
#pragma unroll
            for (int k = 0; k < 4; ++k) w[k] = rescale4(w[k], factor);
            *here = w;
        }
    }
    if (threadIdx.x == 0) tail[role] = (char)s;
    if constexpr (Ends) {
        // bounds: rounding keeps the order, so the bounds of the codes are the codes of the
        // bounds.  Where all is finite, NaN stand for rows that there are not.
        constexpr int kLeft = 2 * NP;  // of a lane's channels, once the wave's quarters are together
        if (!careful) {
            if (!whole)
#pragma unroll
                for (int it = 0; it < ITEMS; ++it) {
                    const int row = it * Ln::kStep + in;
                    const bool there = row >= r0 && row < r1;
#pragma unroll
                    for (int e = 0; e < 8 * NP; ++e) {
                        float& y = x[it][e / 8][e % 8];
                        y = there ? y : __uint_as_float(0x7fc00000u);
                    }
                }
#pragma unroll
            for (int e = 0; e < 8 * NP; ++e) {
                lo[e] = hi[e] = x[0][e / 8][e % 8];
#pragma unroll
                for (int it = 1; it < ITEMS; it += 2) {
                    const float a = x[it][e / 8][e % 8], c = x[it + 1 < ITEMS ? it + 1 : it][e / 8][e % 8];
                    lo[e] = min3(lo[e], a, c);
                    hi[e] = max3(hi[e], a, c);
                }
            }
        }
        const int quarter = ((lane >> 4) & 1) + 2 * (lane >> 5);
        if (!single) {
            if (careful) {
                over_quarters(lo, lower);
                over_quarters(hi, higher);
            } else {
                over_quarters(lo, [](float a, float c) { return min3(a, c, c); });
                over_quarters(hi, [](float a, float c) { return max3(a, c, c); });
            }
            const int w = wv * kParts<D> + (lane & 15) / Ln::kRow;
#pragma unroll
            for (int e = 0; e < kLeft; ++e) {
                const int at_e = quarter * kLeft + e;
                const int ch = 8 * (at_e < 8 ? pc.a : pc.b) + at_e % 8;
                s_ends[0][w][ch] = lo[e];
                s_ends[1][w][ch] = hi[e];
            }
        } else if (in == r0 % Ln::kStep) {
#pragma unroll
            for (int e = 0; e < 8 * NP; ++e) {
                const int ch = 8 * (e < 8 ? pc.a : pc.b) + e % 8;
                s_ends[0][0][ch] = lo[e];
                s_ends[1][0][ch] = hi[e];
            }
        }
        __syncthreads();
        if (threadIdx.x >= 2 * D) return;
        const int ch = threadIdx.x % D;
        const bool upper = threadIdx.x >= D;
        constexpr int kOf = Ln::kRow >= 16 ? 1 : 16 / Ln::kRow;  // of a wave's partial bounds, those written
        float y = s_ends[upper][0][ch];
        if (!single)
#pragma unroll
            for (int w = 0; w < kWaves; ++w)
#pragma unroll
                for (int k = 0; k < kOf; ++k) {
                    const float z = s_ends[upper][w * kParts<D> + k][ch];
                    if (careful)
                        y = upper ? higher(y, z) : lower(y, z);
                    else
                        y = upper ? max3(y, z, z) : min3(y, z, z);
                }
        if (r0 > 0) {  // the old bound in the new scale is a code's value
            float was[4];
            floats4(rescale4(old_end, factor), scale, was);
            y = upper ? higher(y, was[0]) : lower(y, was[0]);
        }
        *end = (char)codes4(y, y, y, y, scale);
    }
}

// A workgroup takes the keys or the values of one block of a segment (layer, sample,
// KV head), both and the heads of a page side by side.  Bound by memory: 32 layers, 4
// samples, 8 KV heads, 1639 of 32768 rows 258 us, 1.29 GB read and written at 5.0 TB/s
// (a copy: 4.85); 4 samples of 4000 tokens 21 us, 4.7 TB/s.  Turned keys take 32 us for
// the latter: 512 bytes of angles to a row, and twelve instructions to a channel; with
// 32 query heads, 360 MB, all of it takes 73 us, 4.9 TB/s.
template <typename T, int D, int PAGE, bool Gather>
__global__ __launch_bounds__(kThreads) void write_blocks(RowView kv, RowView vv, RowView qv, char* __restrict__ q_out,
                                                         WriteGrid g, const int32_t* __restrict__ idx,
                                                         const int32_t* __restrict__ count,
                                                         const int32_t* __restrict__ start,
                                                         const int32_t* __restrict__ seq, BlockRotation rot,
                                                         PagePool p) {
    if constexpr (!Gather) {
        if (blockIdx.x >= g.blocks) return turn_queries<T, D>(qv, q_out, g, blockIdx.x - g.blocks, rot);
    }
    __shared__ uint32_t s_top[kWaves];
    __shared__ float s_ends[2][kWaves * kParts<D>][D];
    const unsigned role = blockIdx.x & 1, x2 = blockIdx.x >> 1;
    const unsigned x1 = x2 / (unsigned)p.Hkv, lb = x1 / (unsigned)g.nblk;
    const int j = (int)(x2 - x1 * p.Hkv), i = (int)(x1 - lb * g.nblk);
    const int l = (int)(lb / (unsigned)g.B), b = (int)(lb - (unsigned)l * g.B);
    const size_t seg = (size_t)lb * p.Hkv + j;
    const int slot = slot_of(seq, b, p.S), s0 = start[b];
    const int n = Gather ? min(count[seg], g.T) : count != nullptr ? min(count[b], g.T) : g.T;
    if (slot < 0 || s0 < 0 || n <= 0) return;
    if (role != 0) {
        write_block<T, D, PAGE, 1, Gather, false>(s_top, s_ends, vv, 1, g, l, b, j, i, seg, idx, slot, s0, n, rot, p);
        return;
    }
    if constexpr (!Gather) {
        if (rot.cos != nullptr) {
            write_block<T, D, PAGE, 2, false, true>(s_top, s_ends, kv, 0, g, l, b, j, i, seg, idx, slot, s0, n, rot, p);
            return;
        }
    }
    write_block<T, D, PAGE, 1, Gather, true>(s_top, s_ends, kv, 0, g, l, b, j, i, seg, idx, slot, s0, n, rot, p);
}

// Eight channels of a row, one piece to a lane: the other channels of its pairs are
// loaded beside it.  Turned as Sixteen turns them.
template <typename T, int D, bool Pairs>
__device__ __forceinline__ void turn_eight(const Eight<T>& own, const Eight<T>& other, const Angles& g, bool low,
                                           float (&x)[8]) {
    uint32_t border = 0xffffu;
    float clear = INFINITY, most = 0.0f;
    float u[8], w[8], c[8], s[8];  // x[e] = u c + w s
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        u[e] = own.get(e);
        w[e] = Pairs ? own.get(e ^ 1) : other.get(e);
        const int i = Pairs ? e / 2 : e;
        c[e] = g.cos[i / 4][i % 4];
        s[e] = g.sin[i / 4][i % 4];
        s[e] = (Pairs ? e % 2 == 0 : low) ? -s[e] : s[e];
        const float p = w[e] * s[e], ep = fmaf(w[e], s[e], -p);
        x[e] = fmaf(u[e], c[e], p) + ep;
        border = min(border, (__float_as_uint(x[e]) + 3u) & 0xffffu);
        clear = fminf(clear, fmaf(-4.0f, fabsf(ep), fabsf(x[e])));
        most = larger(most, fabsf(x[e]));
    }
    if (border > 6 && clear > 0x1p-90f && most < 0x1p120f) return;
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = to_odd(fma((double)u[e], (double)c[e], (double)w[e] * s[e]));
}

// Codes of eight channels after another rounding, and NaN told.
__device__ __forceinline__ void floats8(u32x2 w, float scale, float (&x)[8]) {
    floats4(w[0], scale, *reinterpret_cast<float(*)[4]>(x));
    floats4(w[1], scale, *reinterpret_cast<float(*)[4]>(x + 4));
}

// One row of each sample, a decode step's: D / 8 lanes take a segment's key, as many its
// value, without LDS or barriers.  Bound by four latencies (slot, place and angles'
// positions, page and angles, the block's scale): 16 samples, 8 KV heads 3.1 us, turned
// 3.7, with 32 query heads 4.5; 256 samples 3.4, 4.0 and 6.0 (a workgroup to each block,
// with one row in 64 places of threads to work on: 14.7, 17.6 and 19.1).
template <typename T, int D>
__global__ __launch_bounds__(kThreads) void write_rows(RowView kv, RowView vv, RowView qv, char* __restrict__ q_out,
                                                       WriteGrid g, const int32_t* __restrict__ count,
                                                       const int32_t* __restrict__ start,
                                                       const int32_t* __restrict__ seq, BlockRotation rot, PagePool p) {
    constexpr int kRow = D / 8, kSegs = kThreads / (2 * kRow);
    if (blockIdx.x >= g.blocks) return turn_queries<T, D>(qv, q_out, g, blockIdx.x - g.blocks, rot);
    const int part = threadIdx.x % kRow, role = threadIdx.x / kRow % 2;
    const unsigned seg = blockIdx.x * kSegs + threadIdx.x / (2 * kRow);
    const unsigned lb = seg / (unsigned)p.Hkv;
    const int j = (int)(seg - lb * p.Hkv), l = (int)(lb / (unsigned)g.B), b = (int)(lb - (unsigned)l * g.B);
    if (l >= p.L) return;
    const int slot = slot_of(seq, b, p.S), s0 = start[b];
    if (slot < 0 || s0 < 0 || (count != nullptr && count[b] <= 0)) return;
    const int at = s0 >> p.shift, r0 = s0 & ((1 << p.shift) - 1);
    const int page = p.table[(size_t)slot * p.M + min(at, p.M - 1)], held = held_of(p, slot);
    const RowView& view = role == 0 ? kv : vv;
    const char* row = view.base + (size_t)l * view.s_layer + (size_t)b * view.s_batch + (size_t)j * view.s_head;
    const int half = rot.r / 16;  // pieces of half the turned channels
    const bool turn = role == 0 && rot.cos != nullptr, turned = turn && part < 2 * half, low = part < half;
    Eight<T> own, other;
    own.template load<false>(row, part);
    other = own;
    Angles angles;
    angles.there = true;
    if (turn) {
        const int pos = rot.position[b];
        if (turned && !rot.pairs) other.template load<false>(row, low ? part + half : part - half);
        angles.there = pos >= 0 && pos < rot.P;
        if (angles.there && turned) {
            const size_t first = (size_t)pos * (rot.r / 2) + (rot.pairs ? 4 * part : 8 * (low ? part : part - half));
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                // neighbouring pairs: four angles to a piece
                const size_t four = first + (rot.pairs ? 0 : 4 * i);
                angles.cos[i] = *reinterpret_cast<const f32x4*>(rot.cos + four);
                angles.sin[i] = *reinterpret_cast<const f32x4*>(rot.sin + four);
            }
        }
    }
    if (at >= held || page < 0 || page >= p.n_pages) return;
    char* block = block_at<D>(p, l, page, j);
    char* tail = block + tail_at<D>(p.shift);
    u32x2* codes = reinterpret_cast<u32x2*>(block + ((size_t)(role * D) << p.shift)) + part;  // of row 0
    u32x2* ends = reinterpret_cast<u32x2*>(tail + kBlockScales) + part;                       // minima, then maxima
    int old = 0;
    u32x2 was[2] = {};
    if (r0 > 0) {
        old = scale_of((uint8_t)tail[role]);
        if (role == 0) {
            was[0] = ends[0];
            was[1] = ends[kRow];
        }
    }
    float x[8];
    if (turned && angles.there) {
        if (rot.pairs)
            turn_eight<T, D, true>(own, other, angles, low, x);
        else
            turn_eight<T, D, false>(own, other, angles, low, x);
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = angles.there ? own.get(e) : __uint_as_float(0x7fc00000u);
    }
    uint32_t top = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const uint32_t bits = __float_as_uint(x[e]) & 0x7fffffffu;
        top = max(top, bits < 0x7f800000u ? bits : 0u);
    }
    top = max(top, dpp<0xb1>(top));
    top = max(top, dpp<0x4e>(top));
    top = max(top, dpp<0x141>(top));
    if constexpr (kRow == 16) top = max(top, dpp<0x140>(top));
    const int s = max(scale_byte8(top), old);
    const float scale = scale_float(s), factor = scale_float(127 - min(s - old, 60));
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = bounded(x[e], 448.0f * scale);
    codes[r0 * kRow] = u32x2{codes4(x[0], x[1], x[2], x[3], scale), codes4(x[4], x[5], x[6], x[7], scale)};
    if (r0 > 0 && s != old)
        for (int e0 = 0; e0 < r0; e0 += 16) {  // what was there, sixteen rows in flight
            u32x2 w[16];
#pragma unroll
            for (int e = 0; e < 16; ++e) w[e] = codes[min(e0 + e, r0 - 1) * kRow];
#pragma unroll
            for (int e = 0; e < 16; ++e)
                if (e0 + e < r0) codes[(e0 + e) * kRow] = u32x2{rescale4(w[e][0], factor), rescale4(w[e][1], factor)};
        }
    if (part == 0) tail[role] = (char)s;
    if (role != 0) return;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        float y[8];
        if (r0 > 0) {
            floats8(u32x2{rescale4(was[k][0], factor), rescale4(was[k][1], factor)}, scale, y);
#pragma unroll
            for (int e = 0; e < 8; ++e) y[e] = k == 0 ? lower(x[e], y[e]) : higher(x[e], y[e]);
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) y[e] = x[e];
        }
        ends[k * kRow] = u32x2{codes4(y[0], y[1], y[2], y[3], scale), codes4(y[4], y[5], y[6], y[7], scale)};
    }
}

// ---------------------------------------------------------------------------
// rows and bounds out of blocks
// ---------------------------------------------------------------------------

struct ReadGrid {
    int B, cap;
    uint32_t rows;  // of all segments
};

// D / 8 lanes to a row, Items rows to a lane, those of all segments one after the
// other.  Bounds: row m is block first + m's bound, else the row at position first + m.
// Past: loads past the caches, for more codes than the last one holds.  Bound by memory:
// 1.7 M rows just written, 1.29 GB read and written, 255 us, 5.1 TB/s (through the caches
// 280, and 300 with two rows to a lane; sixteen channels to a lane, whose 16-byte stores
// then lie apart: 385).
template <typename T, int D, bool Bounds, int Items, bool Past>
__global__ __launch_bounds__(kThreads) void read_blocks(PagePool p, ReadGrid g, const int32_t* __restrict__ seq,
                                                        const int32_t* __restrict__ first,
                                                        const int32_t* __restrict__ count, char* __restrict__ a_out,
                                                        char* __restrict__ b_out) {
    constexpr int kRow = D / 8, kStep = kThreads / kRow;
    const int part = threadIdx.x % kRow;
    const uint32_t at0 = blockIdx.x * (uint32_t)(kStep * Items) + threadIdx.x / kRow;
    const char* block[Items];
    int tok[Items];
#pragma unroll
    for (int it = 0; it < Items; ++it) {
        const uint32_t at = at0 + it * kStep;
        block[it] = nullptr;
        if (at >= g.rows) continue;
        const uint32_t seg = at / (uint32_t)g.cap, m = at - seg * g.cap;
        const uint32_t lb = seg / (uint32_t)p.Hkv, j = seg - lb * p.Hkv;
        const uint32_t l = lb / (uint32_t)g.B, b = lb - l * g.B;
        const int slot = slot_of(seq, b, p.S);
        if (slot < 0 || (count != nullptr && (int)m >= count[b])) continue;
        const int from = first != nullptr ? first[b] : 0;
        const int len = length_of(p, slot), end = Bounds ? (len + (1 << p.shift) - 1) >> p.shift : len;
        if (from < 0 || (long long)from + m >= end) continue;
        const int pos = from + (int)m, blk = Bounds ? pos : pos >> p.shift;
        const int pg = p.table[(size_t)slot * p.M + blk];
        tok[it] = pos & ((1 << p.shift) - 1);
        if (pg >= 0 && pg < p.n_pages) block[it] = block_at<D>(p, l, pg, j);
    }
    u32x2 a[Items], c[Items];
    uint32_t scales[Items];
#pragma unroll
    for (int it = 0; it < Items; ++it) {
        if (block[it] == nullptr) continue;
        const char* tail = block[it] + tail_at<D>(p.shift);
        const char* row = block[it] + (size_t)tok[it] * D;
        const char* rows[2] = {Bounds ? tail + kBlockScales : row,
                               Bounds ? tail + kBlockScales + D : row + ((size_t)D << p.shift)};
        const u32x2 *from = reinterpret_cast<const u32x2*>(rows[0]) + part,
                    *other = reinterpret_cast<const u32x2*>(rows[1]) + part;
        a[it] = Past ? __builtin_nontemporal_load(from) : *from;
        c[it] = Past ? __builtin_nontemporal_load(other) : *other;
        scales[it] = *reinterpret_cast<const uint16_t*>(tail);
    }
    auto give = [&](char* o, u32x2 w, uint32_t s) {
        float x[8];
        const float unit = scale_float(scale_of((uint8_t)s));
        floats4(w[0], unit, *reinterpret_cast<float(*)[4]>(x));
        floats4(w[1], unit, *reinterpret_cast<float(*)[4]>(x + 4));
        Eight<T>::template store<true>(o, part, x);
    };
#pragma unroll
    for (int it = 0; it < Items; ++it) {
        if (block[it] == nullptr) continue;
        const size_t out = (size_t)(at0 + it * kStep) * (D * sizeof(T));
        if (a_out != nullptr) give(a_out + out, a[it], scales[it]);
        if (b_out != nullptr) give(b_out + out, c[it], Bounds ? scales[it] : scales[it] >> 8);
    }
}

template <typename T, int D, int PAGE>
void run_write(const RowView& k, const RowView& v, const RowView& q, char* q_out, const WriteGrid& g, unsigned groups,
               const int32_t* idx, const int32_t* count, const int32_t* start, const int32_t* seq,
               const BlockRotation& rot, const PagePool& p, hipStream_t st) {
    if (idx != nullptr)
        hipLaunchKernelGGL((write_blocks<T, D, PAGE, true>), dim3(groups), dim3(kThreads), 0, st, k, v, q, q_out, g,
                           idx, count, start, seq, rot, p);
    else
        hipLaunchKernelGGL((write_blocks<T, D, PAGE, false>), dim3(groups), dim3(kThreads), 0, st, k, v, q, q_out, g,
                           idx, count, start, seq, rot, p);
}

template <typename T, int D>
void run_write(const RowView& k, const RowView& v, const RowView& q, char* q_out, const WriteGrid& g, unsigned groups,
               const int32_t* idx, const int32_t* count, const int32_t* start, const int32_t* seq,
               const BlockRotation& rot, const PagePool& p, hipStream_t st) {
    if (p.shift == 5)
        run_write<T, D, 32>(k, v, q, q_out, g, groups, idx, count, start, seq, rot, p, st);
    else if (p.shift == 6)
        run_write<T, D, 64>(k, v, q, q_out, g, groups, idx, count, start, seq, rot, p, st);
    else
        run_write<T, D, 128>(k, v, q, q_out, g, groups, idx, count, start, seq, rot, p, st);
}

// Codes, in bytes, from which a call reads them past the caches, two bytes an element four
// rows to a lane: 1.7 M rows as above; a read of 1 M rows (268 MB) that the last call left
// in the last-level cache 121 us through it, 141 past it, of 2 M 283 and 272.  Else a lane
// takes one row: 128 rows 3.7 us, with two 4.1 and with four 5.3.  Float32 rows are best
// one to a lane at every size: 2 M 520, two 571, four 580.
constexpr long long kReadPast = (1LL << 28) + 1;
template <typename T, int D, bool Bounds>
void run_read(const PagePool& p, int B, int cap, const int32_t* seq, const int32_t* first, const int32_t* count,
              void* a, void* b, hipStream_t st) {
    const ReadGrid g{B, cap, (uint32_t)p.L * B * p.Hkv * (uint32_t)cap};
    auto launch = [&](auto kernel, unsigned items) {
        const unsigned rows = kThreads / (D / 8) * items;
        hipLaunchKernelGGL(kernel, dim3((g.rows + rows - 1) / rows), dim3(kThreads), 0, st, p, g, seq, first, count,
                           static_cast<char*>(a), static_cast<char*>(b));
    };
    constexpr int kMost = sizeof(T) == 2 ? 4 : 1;
    if (!Bounds && 2LL * D * g.rows >= kReadPast)
        launch(read_blocks<T, D, false, kMost, true>, kMost);
    else
        launch(read_blocks<T, D, Bounds, 1, false>, 1);
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
    WriteGrid g{B, cap, N, (int)blocks_touched(cap, 1 << p.shift), Hq, 0, (unsigned)B * cap};
    const bool single = cap == 1 && idx == nullptr;
    const unsigned segs = (unsigned)p.L * B * p.Hkv, per = kThreads / (d / 4);  // write_rows' segments per workgroup
    g.blocks = single ? (segs + per - 1) / per : 2u * segs * g.nblk;
    const unsigned step = d == 128 ? Lanes<128, 2>::kStep : Lanes<64, 2>::kStep;
    const unsigned groups =
        g.blocks + (q_out == nullptr ? 0u : (unsigned)p.L * ((g.tokens + step - 1) / step) *
                                                ((unsigned)(Hq + kBlocksQueryHeads - 1) / kBlocksQueryHeads));
    char* o = static_cast<char*>(q_out);
    auto rows = [&](auto kernel) {
        hipLaunchKernelGGL(kernel, dim3(groups), dim3(kThreads), 0, st, k, v, q, o, g, count, start, seq, rot, p);
        return hipGetLastError();
    };
    if (single && dtype == 0) return d == 128 ? rows(write_rows<__bf16, 128>) : rows(write_rows<__bf16, 64>);
    if (single) return d == 128 ? rows(write_rows<float, 128>) : rows(write_rows<float, 64>);
    if (dtype == 0 && d == 128) run_write<__bf16, 128>(k, v, q, o, g, groups, idx, count, start, seq, rot, p, st);
    if (dtype == 0 && d == 64) run_write<__bf16, 64>(k, v, q, o, g, groups, idx, count, start, seq, rot, p, st);
    if (dtype == 1 && d == 128) run_write<float, 128>(k, v, q, o, g, groups, idx, count, start, seq, rot, p, st);
    if (dtype == 1 && d == 64) run_write<float, 64>(k, v, q, o, g, groups, idx, count, start, seq, rot, p, st);
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
