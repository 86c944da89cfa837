// Device-side building blocks of the paged 8-bit cache.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "kve_blocks_plan.h"
#include "kve_pages_device.h"

namespace kve {

typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

template <int D>
__device__ __forceinline__ size_t tail_at(int shift) {
    return (size_t)(2 * D) << shift;
}

// Block of page number `page` for a (layer, KV head).
template <int D>
__device__ __forceinline__ char* block_at(const PagePool& p, int l, int page, int j) {
    return p.pool + (((size_t)l * p.n_pages + page) * p.Hkv + j) * (tail_at<D>(p.shift) + kBlockScales + 2 * D);
}

// A scale byte of a block's tail, whatever the byte holds.
__device__ __forceinline__ int scale_of(uint8_t s) { return min(max((int)s, kBlockScaleMin), kBlockScaleMax); }

// Four codes of a dword as floats times `scale`.
__device__ __forceinline__ void floats4(uint32_t w, float scale, float (&x)[4]) {
    const f32x2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w, scale, false);
    const f32x2 b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w, scale, true);
    x[0] = a[0];
    x[1] = a[1];
    x[2] = b[0];
    x[3] = b[1];
}

// Not 0 if one of four codes is NaN.
__device__ __forceinline__ uint32_t nan_codes(uint32_t w) { return ((w & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u; }

// Rows that query token t of sample b sees in the sequence of `slot`.
__device__ __forceinline__ int seen_by(const PagePool& p, const BlockView& v, int slot, int b, int t) {
    if (slot < 0) return 0;
    const int len = length_of(p, slot);
    const long long start = v.start != nullptr ? v.start[b] : (long long)len - v.T;
    if (v.start != nullptr && start < 0) return 0;
    return (int)max(0LL, min(start + t + 1, (long long)min(len, v.max_tokens)));
}

}  // namespace kve
