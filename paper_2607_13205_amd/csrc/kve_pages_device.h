// Device-side building blocks of the paged 4-bit cache.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "kve_device.h"
#include "kve_pages_plan.h"

namespace kve {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

// Slot of sample b, or -1.
__device__ __forceinline__ int slot_of(const int32_t* seq, int b, int S) {
    const int s = seq != nullptr ? seq[b] : b;
    return s >= 0 && s < S ? s : -1;
}

__device__ __forceinline__ int held_of(const PagePool& p, int slot) { return min(max(p.held[slot], 0), p.M); }

// Tokens of a sequence that its pages can hold.
__device__ __forceinline__ int length_of(const PagePool& p, int slot) {
    return min(max(p.length[slot], 0), held_of(p, slot) << p.shift);
}

// Block of page number `page` for a (layer, KV head).
template <int D>
__device__ __forceinline__ char* page_block(const PagePool& p, int l, int page, int j) {
    const size_t bytes = (size_t)(D / 16 * 17) << p.shift;
    return p.pool + (((size_t)l * p.n_pages + page) * p.Hkv + j) * bytes;
}

// The power of two that scale byte s stands for, as the scaled conversions take
// it: 255 << 23 makes them give NaN.
__device__ __forceinline__ float scale_float(uint32_t s) { return __uint_as_float(s << 23); }

}  // namespace kve
