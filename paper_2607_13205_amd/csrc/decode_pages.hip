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
// heads per 16x16x32 product: row m of tile T is token 8 (m / 4) + 4 T + m % 4,
// and lane l (head l % 16, quarter l / 16) receives rows 4 (l / 16) .. + 4, that
// is the eight tokens 8 (l / 16) .. + 8 from its two tiles, in order.  Those are
// what the second product O^T = V^T P^T wants from that lane.  The value rows'
// dwords hold eight channels of one token and the product eight tokens of one
// channel: the scaled conversion gives two channels of a token, and a byte
// permutation pairs the tokens.
//
// Split-K and the lazy softmax reference are those of the dense decode
// (decode.hip): weights are exp2(x - m) with m raised only when a logit exceeds it
// by more than 64.
#include <type_traits>

#include "kve_decode_merge.h"
#include "kve_device.h"
#include "kve_internal.h"
#include "kve_pages_device.h"

namespace kve {
namespace {

constexpr int kThreads = kMergeThreads;
constexpr int kWaves = kThreads / kWave;
constexpr int kBlk = 32;    // tokens per wave step
constexpr int kHeads = kPagesMaxGroup;

typedef uint32_t u32x8 __attribute__((ext_vector_type(8)));

// Eight bf16, the high halves of eight floats.
__device__ __forceinline__ bf16x8 high_halves(const uint32_t (&x)[8]) {
    u32x4 r;
#pragma unroll
    for (int i = 0; i < 4; ++i) r[i] = __builtin_amdgcn_perm(x[2 * i + 1], x[2 * i], 0x07060302u);
    return __builtin_bit_cast(bf16x8, r);
}

// Eight floats as three bf16 parts whose sum they are.
__device__ __forceinline__ void split3(const float (&x)[8], bf16x8 (&part)[3]) {
    uint32_t bits[8];
    float rest[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        bits[i] = __float_as_uint(x[i]);
        rest[i] = x[i] - __uint_as_float(bits[i] & 0xffff0000u);
    }
    part[0] = high_halves(bits);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        bits[i] = __float_as_uint(rest[i]);
        rest[i] = rest[i] - __uint_as_float(bits[i] & 0xffff0000u);
    }
    part[1] = high_halves(bits);
#pragma unroll
    for (int i = 0; i < 8; ++i) bits[i] = __float_as_uint(rest[i]);
    part[2] = high_halves(bits);
}

__device__ __forceinline__ f32x4 mma(bf16x8 a, bf16x8 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}

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

// One workgroup per (segment, split); its waves take 32 tokens in turn.
template <typename T, int D>
__global__ __launch_bounds__(kThreads) void pages_split(const T* __restrict__ q, PagePool p,
                                                        const int32_t* __restrict__ seq, int B, int G,
                                                        int max_tokens, int nsplit, int split_keys, float sl2,
                                                        float* __restrict__ ws_o, float2* __restrict__ ws_ml,
                                                        float* __restrict__ out) {
    constexpr int NP = std::is_same<T, float>::value ? 3 : 1;  // bf16 parts of a query
    constexpr int NK = D / 32;                                 // products per 16 tokens: dwords of a lane's quarter row
    constexpr int NC = D / 16;                                 // channels per lane of V^T
    __shared__ float s_ml[kWaves][2][kHeads];
    __shared__ float s_o[kWaves][kHeads][D];

    const int seg = blockIdx.x / nsplit;
    const int sp = blockIdx.x - seg * nsplit;
    const int j = seg % p.Hkv, lb = seg / p.Hkv;
    const int l = lb / B, b = lb - l * B;
    const int lane = threadIdx.x & (kWave - 1);
    const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int c = lane & 15, quarter = lane >> 4;
    const int slot = slot_of(seq, b, p.S);
    const int n = slot < 0 ? 0 : min(length_of(p, slot), max_tokens);
    const int k0 = sp * split_keys;
    const int k1 = min(n, k0 + split_keys);
    const int page = 1 << p.shift;

    bf16x8 qf[NK][NP];
#pragma unroll
    for (int s = 0; s < NK; ++s) {
        if constexpr (NP == 1) {
            u32x4 x = zero16();
            if (c < G) x = ld16(q + ((size_t)seg * G + c) * D + D / 4 * quarter + 8 * s);
            qf[s][0] = __builtin_bit_cast(bf16x8, x);
        } else {
            float x[8];
#pragma unroll
            for (int i = 0; i < 8; ++i)
                x[i] = c < G ? (float)q[((size_t)seg * G + c) * D + D / 4 * quarter + 8 * s + i] : 0.0f;
            split3(x, qf[s]);
        }
    }
    float m = -INFINITY, den = 0.0f;
    f32x4 o[NC];
#pragma unroll
    for (int i = 0; i < NC; ++i) o[i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};

    for (int t0 = k0 + wv * kBlk; t0 < k1; t0 += kWaves * kBlk) {
        const int pg = p.table[(size_t)slot * p.M + (t0 >> p.shift)];
        if (pg < 0 || pg >= p.n_pages) continue;
        const char* block = page_block<D>(p, l, pg, j);
        const int tok = t0 & (page - 1);
        const int left = k1 - t0;  // tokens of this step

        // keys: a quarter row per lane and tile, and the scales of eight tokens
        uint32_t kw[2][NK];
#pragma unroll
        for (int tile = 0; tile < 2; ++tile) {
            const char* row = block + (size_t)(tok + 8 * (c >> 2) + 4 * tile + (c & 3)) * (D / 2) + quarter * (D / 8);
#pragma unroll
            for (int s = 0; s < NK; ++s) kw[tile][s] = reinterpret_cast<const uint32_t*>(row)[s];
        }
        const char* scales = block + (size_t)page * D;
        const u32x2 ks = *reinterpret_cast<const u32x2*>(scales + (size_t)(quarter * D / 128) * page + tok + 8 * (c >> 2));
        // values: NC channels of eight tokens
        uint32_t vw[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const char* row = block + (size_t)page * (D / 2) + (size_t)(tok + 8 * quarter + i) * (D / 2) + c * (D / 32);
            if constexpr (D == 128)
                vw[i] = *reinterpret_cast<const uint32_t*>(row);
            else
                vw[i] = *reinterpret_cast<const uint16_t*>(row);
        }
        u32x2 vs = *reinterpret_cast<const u32x2*>(scales + (size_t)(D / 32 + c * (D / 16) / 32) * page + tok + 8 * quarter);

        f32x4 acc[2];
#pragma unroll
        for (int tile = 0; tile < 2; ++tile) {
            const float sc = scale_float((ks[tile] >> (8 * (c & 3))) & 0xffu);
            acc[tile] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int s = 0; s < NK; ++s) {
                const bf16x8 kf = unpack8(kw[tile][s], sc);
#pragma unroll
                for (int a = NP - 1; a >= 0; --a) acc[tile] = mma(kf, qf[s][a], acc[tile]);
            }
        }
        float x[8];
        bool raise = false;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            x[i] = 8 * quarter + i < left ? acc[i >> 2][i & 3] * sl2 : -INFINITY;
            raise |= x[i] > m + 64.0f;
        }
        if (__builtin_amdgcn_ballot_w64(raise) != 0) {
            float mn = m;
#pragma unroll
            for (int i = 0; i < 8; ++i) mn = fmaxf(mn, x[i]);
            mn = fmaxf(mn, __shfl_xor(mn, 16));
            mn = fmaxf(mn, __shfl_xor(mn, 32));
            const float alpha = mn == -INFINITY ? 1.0f : fast_exp2(m - mn);
            den *= alpha;
            m = mn;
#pragma unroll
            for (int i = 0; i < NC; ++i) o[i] *= alpha;
        }
        float w[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            w[i] = 8 * quarter + i < left ? fast_exp2(x[i] - m) : 0.0f;
            den += w[i];
        }
        bf16x8 pf[3];
        split3(w, pf);

        // rows behind the sequence hold anything: zeros under their zero weights
        if (left < kBlk) {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (8 * quarter + i >= left) {
                    vw[i] = 0;
                    vs[i >> 2] &= ~(0xffu << (8 * (i & 3)));
                }
        }
        float sc[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) sc[i] = scale_float((vs[i >> 2] >> (8 * (i & 3))) & 0xffu);
        bf16x8 vf[NC];
        unpack_tokens<0>(vw, sc, vf[0], vf[1]);
        unpack_tokens<1>(vw, sc, vf[2], vf[3]);
        if constexpr (D == 128) {
            unpack_tokens<2>(vw, sc, vf[4], vf[5]);
            unpack_tokens<3>(vw, sc, vf[6], vf[7]);
        }
#pragma unroll
        for (int i = 0; i < NC; ++i)
#pragma unroll
            for (int a = 2; a >= 0; --a) o[i] = mma(vf[i], pf[a], o[i]);
    }

    den += __shfl_xor(den, 16);
    den += __shfl_xor(den, 32);
    if (den != den && m == -INFINITY) m = 0.0f;  // every logit was NaN: the split is not empty
    if (c < G) {
        if (quarter == 0) {
            s_ml[wv][0][c] = m;
            s_ml[wv][1][c] = den;
        }
        // o[i][r]: channel NC (4 quarter + r) + i of head c
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int i = 0; i < NC; ++i) s_o[wv][c][NC * (4 * quarter + r) + i] = o[i][r];
    }
    __syncthreads();
    // merge the waves' partial results of this split
    for (int e = threadIdx.x; e < G * D; e += kThreads) {
        const int h = e / D, ch = e - h * D;
        float mx = -INFINITY;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) mx = fmaxf(mx, s_ml[w][0][h]);
        float lt = 0.0f, ot = 0.0f;
        if (mx != -INFINITY) {
#pragma unroll
            for (int w = 0; w < kWaves; ++w) {
                const float a = fast_exp2(s_ml[w][0][h] - mx);
                lt = fmaf(a, s_ml[w][1][h], lt);
                ot = fmaf(a, s_o[w][h][ch], ot);
            }
        }
        const size_t row = (size_t)blockIdx.x * G + h;
        if (nsplit == 1) {  // the whole segment: the result itself
            out[row * D + ch] = lt != 0.0f ? ot / lt : 0.0f;
        } else {
            ws_o[row * D + ch] = ot;
            if (ch == 0) ws_ml[row] = make_float2(mx, lt);
        }
    }
}

template <typename T, int D>
hipError_t run(const void* q, const PagePool& p, int B, int Hq, int max_tokens, const int32_t* seq, float scale,
               float* out, void* ws, hipStream_t st) {
    const DecodePlan plan = decode_pages_plan(p.L, B, Hq, p.Hkv, max_tokens, D);
    char* w = static_cast<char*>(ws);
    float* wo = reinterpret_cast<float*>(w + plan.off_o);
    float2* wml = reinterpret_cast<float2*>(w + plan.off_ml);
    hipLaunchKernelGGL((pages_split<T, D>), dim3((unsigned)((size_t)plan.segs * plan.nsplit)), dim3(kThreads), 0, st,
                       static_cast<const T*>(q), p, seq, B, plan.G, max_tokens, plan.nsplit, plan.split_keys,
                       scale * kLog2e, wo, wml, out);
    launch_merge<D, true>(wo, wml, plan.G, plan.nsplit, plan.segs * plan.G, out, st);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_decode_pages(const void* q, int dtype, const PagePool& p, int d, int B, int Hq, int max_tokens,
                               const int32_t* seq, float scale, float* out, void* ws, hipStream_t st) {
    if (dtype == 0) {
        if (d == 128) return run<__bf16, 128>(q, p, B, Hq, max_tokens, seq, scale, out, ws, st);
        return run<__bf16, 64>(q, p, B, Hq, max_tokens, seq, scale, out, ws, st);
    }
    if (d == 128) return run<float, 128>(q, p, B, Hq, max_tokens, seq, scale, out, ws, st);
    return run<float, 64>(q, p, B, Hq, max_tokens, seq, scale, out, ws, st);
}

}  // namespace kve
