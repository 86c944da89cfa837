// What the decodes over pages share: how the sequences are cut into splits on the
// device, and float32 softmax weights as operands of bf16 products.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "kve_device.h"
#include "kve_pages_device.h"
#include "kve_stream.h"

namespace kve {
namespace {

// A weight may grow to 2^kRaise before the reference is raised: rarely after the
// first step, and far from where the value sums overflow.
constexpr float kRaise = 16.0f;
// The reference before any logit: finite, so that logits of minus infinity (products
// that leave float32) have weights of zero under it, not NaN.
constexpr float kLowest = -3.4028234663852886e38f;
constexpr int kMostQuanta = (1 << 30) / kDecodeQuantum;  // of a sequence

// One direct-to-LDS load of four bytes per lane, as lds_dma16.
__device__ __forceinline__ void lds_dma4(const char* base, unsigned voff, const char* lds_dst) {
    const unsigned m0 = __builtin_amdgcn_readfirstlane((unsigned)(uintptr_t)lds_dst);
    asm volatile("s_nop 4\n\tglobal_load_lds_dword %0, %1" ::"v"(voff), "s"(base), "{m0}"(m0) : "memory");
}

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

// Eight softmax weights of a lane in column c of the second product's sixteen, as
// the bf16 parts that the column's copies of a head make.
template <int NH, int NW>
__device__ __forceinline__ void weight_parts(const float (&w)[8], int c, bf16x8 (&part)[NW]) {
    if constexpr (NH == 4) {
        // columns 0..3 keep the top 8 bits, 4..7 the 8 after them, 8..11 the rest
        const uint32_t first = c >= 4 ? 0xffff0000u : 0u, second = c >= 8 ? 0xffff0000u : 0u;
        uint32_t bits[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            float y = w[i] - __uint_as_float(__float_as_uint(w[i]) & first);
            y = y - __uint_as_float(__float_as_uint(y) & second);
            bits[i] = __float_as_uint(y);
        }
        part[0] = high_halves(bits);
    } else if constexpr (NH == 8) {
        // columns 0..7 keep the top 8 bits and the last, 8..15 the middle ones
        uint32_t bits[8], rest[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float y = w[i] - __uint_as_float(__float_as_uint(w[i]) & 0xffff0000u);
            const float z = y - __uint_as_float(__float_as_uint(y) & 0xffff0000u);
            bits[i] = __float_as_uint(c < 8 ? w[i] : y);
            rest[i] = __float_as_uint(z);
        }
        part[0] = high_halves(bits);
        u32x4 last = __builtin_bit_cast(u32x4, high_halves(rest));
        last &= c < 8 ? 0xffffffffu : 0u;
        part[1] = __builtin_bit_cast(bf16x8, last);
    } else {
        split3(w, part);
    }
}

// Inclusive sum over the lanes of a wave, with lane moves (an LDS exchange per
// step is several times their latency).
__device__ __forceinline__ int wave_scan(int x) {
    x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false);  // the lane before
    x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false);  // two before
    x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);  // lane 15 of a row to the next row
    x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);  // lane 31 to the upper half
    return x;
}

__device__ __forceinline__ int wave_sum(int x) { return __builtin_amdgcn_readlane(wave_scan(x), kWave - 1); }

// A sequence as a lane holds it: its slot (-1: none) and its tokens.
struct Sequence {
    int slot, tokens;
};

__device__ __forceinline__ int quanta_of(int tokens) { return (tokens + kDecodeQuantum - 1) / kDecodeQuantum; }

__device__ __forceinline__ int splits_of(int quanta, int per) {
    return (int)((unsigned)(quanta + per - 1) / (unsigned)per);
}

// Splits before and of a sequence.
struct SplitRange {
    int first, count;
};

// What a workgroup works on: tokens [k0, k1) of sample b, in slot `slot`.
struct Work {
    int b, slot, k0, k1;
    SplitRange range;
};

// How the sequences are cut (PagesPlan): the quanta of a split are a `share`-th of
// all, rounded up, which makes at most share + B splits; and split x of them (b =
// -1: there is none).  Longer ones that make no more than `share` are worse: the
// longest then outlasts the others by more than a second round of short ones
// costs (64 ragged sequences of up to 16384 tokens, 8 KV heads: 87 us so, 64.5
// with a share-th; half of it and twice it 63.6 and 73).  Every wave works it out for
// itself, 64 sequences at a time.  of(b): sequence b, none from B on.  staged: the
// lengths of all sequences, null for up to 64, which the lanes hold.  ranges: where not
// null, every sequence's range is written there.
// level: where not 0, the share for sequences of which none is much longer than the
// mean.
template <typename Of>
__device__ __forceinline__ Work find_work(Of of, int B, int share, int x, const int* staged, SplitRange* ranges,
                                          int level = 0) {
    const int lane = threadIdx.x & (kWave - 1);
    Sequence mine{-1, 0};
    if (staged == nullptr) mine = of(lane);
    auto tokens_at = [&](int b0) -> int {
        if (staged != nullptr) return b0 + lane < B ? staged[b0 + lane] : 0;
        return mine.tokens;
    };
    // sums over the lanes' shares: up to 2^23 quanta each, any number of sequences
    long long total = 0;
    int longest = 0;
    for (int b0 = 0; b0 < B; b0 += kWave) {
        const int quanta = quanta_of(tokens_at(b0));
        total += wave_sum(quanta);
        if (level != 0) longest = max(longest, quanta);
    }
    if (level != 0 && __builtin_amdgcn_ballot_w64((long long)longest * B > total + total / 8) == 0) share = level;
    // no sequence has more than kMostQuanta
    int per = total < kMostQuanta ? max(1, splits_of((int)total, share))
                                  : (int)min((total + share - 1) / share, (long long)kMostQuanta);
    Work w{-1, -1, 0, 0, {0, 0}};
    int before = 0;
    for (int b0 = 0; b0 < B; b0 += kWave) {
        const int tokens = tokens_at(b0);
        const int n = splits_of(quanta_of(tokens), per), inc = wave_scan(n);
        const int first = before + inc - n;
        if (ranges != nullptr && b0 + lane < B) ranges[b0 + lane] = SplitRange{first, n};
        const uint64_t mask = __builtin_amdgcn_ballot_w64(x >= first && x < first + n);
        if (mask != 0) {
            const int at = __builtin_ctzll(mask);
            w.b = b0 + at;
            w.slot = staged == nullptr ? __builtin_amdgcn_readlane(mine.slot, at)
                                       : __builtin_amdgcn_readfirstlane(of(w.b).slot);
            w.range.first = __builtin_amdgcn_readlane(first, at);
            w.range.count = __builtin_amdgcn_readlane(n, at);
            w.k0 = (x - w.range.first) * per * kDecodeQuantum;
            w.k1 = (int)min((long long)__builtin_amdgcn_readlane(tokens, at),
                            w.k0 + (long long)per * kDecodeQuantum);
            if (ranges == nullptr) return w;
        }
        before += __builtin_amdgcn_readlane(inc, kWave - 1);
    }
    return w;
}

// Has the compiler wait for x here.  A wait for a tracked load inside the loop
// over the steps would wait for the direct-to-LDS loads behind it too.
template <typename X>
__device__ __forceinline__ void settle(X& x) {
    asm volatile("" : "+v"(x));
}

// x[i + N] of the sixteen lanes of a row, 0 behind them.
template <int N>
__device__ __forceinline__ float row_from(float x) {
    return __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(x), 0x100 + N, 0xf, 0xf,
                                                                 true));
}

}  // namespace
}  // namespace kve
