// The last step of a split decode: partial softmax sums merged and normalised.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "kve_device.h"

namespace kve {
namespace {

constexpr int kMergeThreads = 256;
constexpr int kMergeWaves = kMergeThreads / kWave;

__device__ __forceinline__ float xor_max32(float v) {
#pragma unroll
    for (int s = 1; s < 32; s <<= 1) v = fmaxf(v, __shfl_xor(v, s));
    return v;
}

__device__ __forceinline__ float xor_sum32(float v) {
#pragma unroll
    for (int s = 1; s < 32; s <<= 1) v += __shfl_xor(v, s);
    return v;
}

__device__ __forceinline__ float read_lane(float v, int lane) {
    return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), lane));
}

// The merge of one row's splits and its normalisation: WPR waves per row, each a
// contiguous share of the splits, 64 at a time: lane s takes the reference and
// denominator of split s, then the partial outputs are added kAhead loads at a
// time.  What the merge costs is round trips to memory, not bytes: a loop that
// loads split by split took 6.9 us for 13 splits of 128 rows.
// ws_o, ws_ml: the row's first split; the next one is `step` rows on.  All waves
// of a row must call it together; `store`: whether there is a row at all.
// KeepNaN: a denominator that is not a number makes the row NaN, not zero.
template <int D, int WPR, bool KeepNaN>
__device__ __forceinline__ void merge_row(const float* __restrict__ ws_o, const float2* __restrict__ ws_ml, int step,
                                          int nsplit, bool store, float* __restrict__ out) {
    constexpr int CPT = D / kWave;  // columns per lane
    constexpr int kAhead = 8;
    __shared__ float s_m[kMergeWaves], s_l[kMergeWaves], s_o[kMergeWaves][D];
    const int lane = threadIdx.x & (kWave - 1);
    const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int part = wv % WPR;
    const int s0 = nsplit * part / WPR, s1 = nsplit * (part + 1) / WPR;
    float mx = -INFINITY, lt = 0.0f, ot[CPT];
#pragma unroll
    for (int c = 0; c < CPT; ++c) ot[c] = 0.0f;
    for (int sb = s0; sb < s1; sb += kWave) {
        const int n = min(kWave, s1 - sb);
        const float2 ml = ws_ml[(size_t)(sb + min(lane, n - 1)) * step];
        const float m = lane < n ? ml.x : -INFINITY;
        float mn = fmaxf(xor_max32(m), mx);
        mn = fmaxf(mn, __shfl_xor(mn, 32));
        if (mn == -INFINITY) continue;  // uniform: only empty splits so far
        const float a = fast_exp2(m - mn), keep = fast_exp2(mx - mn);
        const float l = xor_sum32(lane < n ? a * ml.y : 0.0f);
        lt = fmaf(lt, keep, l + __shfl_xor(l, 32));
#pragma unroll
        for (int c = 0; c < CPT; ++c) ot[c] *= keep;
        mx = mn;
        for (int i = 0; i < n; i += kAhead) {
            float o[kAhead][CPT];
#pragma unroll
            for (int j = 0; j < kAhead; ++j) {
                const float* os = ws_o + (size_t)(sb + min(i + j, n - 1)) * step * D + lane * CPT;
#pragma unroll
                for (int c = 0; c < CPT; ++c) o[j][c] = os[c];
            }
#pragma unroll
            for (int j = 0; j < kAhead; ++j) {
                const float w = i + j < n ? read_lane(a, min(i + j, n - 1)) : 0.0f;
#pragma unroll
                for (int c = 0; c < CPT; ++c) ot[c] = fmaf(w, o[j][c], ot[c]);
            }
        }
    }
    if constexpr (WPR > 1) {
        s_m[wv] = mx;
        s_l[wv] = lt;
#pragma unroll
        for (int c = 0; c < CPT; ++c) s_o[wv][lane * CPT + c] = ot[c];
        __syncthreads();
        if (part != 0) return;
        float m = -INFINITY;
#pragma unroll
        for (int w = 0; w < WPR; ++w) m = fmaxf(m, s_m[wv + w]);
        lt = 0.0f;
#pragma unroll
        for (int c = 0; c < CPT; ++c) ot[c] = 0.0f;
        if (m != -INFINITY) {
#pragma unroll
            for (int w = 0; w < WPR; ++w) {
                const float a = fast_exp2(s_m[wv + w] - m);
                lt = fmaf(a, s_l[wv + w], lt);
#pragma unroll
                for (int c = 0; c < CPT; ++c) ot[c] = fmaf(a, s_o[wv + w][lane * CPT + c], ot[c]);
            }
        }
    }
    if (store) {
#pragma unroll
        for (int c = 0; c < CPT; ++c)
            out[lane * CPT + c] = (KeepNaN ? lt != 0.0f : lt > 0.0f) ? ot[c] / lt : 0.0f;
    }
}

}  // namespace
}  // namespace kve
