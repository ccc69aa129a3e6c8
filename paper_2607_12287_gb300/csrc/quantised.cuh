// What the kernels of the 8-bit cache share: e4m3 codes, the layout and its check.
#pragma once

#include "backbone.cuh"

namespace ivit {

// Four codes of a word as fp16 values, which hold every e4m3 value exactly.
__device__ __forceinline__ void codes_to_half4(uint32_t w, uint32_t& lo, uint32_t& hi) {
  asm("{\n\t.reg .b16 a, b;\n\tmov.b32 {a, b}, %2;\n\tcvt.rn.f16x2.e4m3x2 %0, a;\n\tcvt.rn.f16x2.e4m3x2 %1, b;\n\t}"
      : "=r"(lo), "=r"(hi)
      : "r"(w));
}
// Codes of two fp32 values, rounded to nearest even (beyond 448: 448; NaN stays NaN).
__device__ __forceinline__ uint32_t to_codes2(float lo, float hi) {
  uint16_t r;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
  return r;
}

// 8 and 4 bytes to shared memory (see copy16).
__device__ __forceinline__ void copy8(uint32_t dst, const void* src, bool ok) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 8, %2;" ::"r"(dst), "l"(src), "r"(ok ? 8 : 0) : "memory");
}
__device__ __forceinline__ void copy4(uint32_t dst, const void* src, bool ok) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(src), "r"(ok ? 4 : 0) : "memory");
}

// A paged cache of 8 bits of one layer (ivit_quantised_layout).
struct QuantisedCache {
  int n_pages, page_shift, block_shift, heads, dim;
  long long page_stride, token_stride, head_stride;  // bytes

  __device__ __forceinline__ bool holds(int slot) const { return slot >= 0 && (slot >> page_shift) < n_pages; }
  __device__ __forceinline__ long long token(int slot) const {  // byte of head 0 of a slot
    return (slot >> page_shift) * page_stride + (slot & ((1 << page_shift) - 1)) * token_stride;
  }
  // (blocks of a page follow each other, so a slot's block is slot >> block_shift)
  __device__ __forceinline__ long long scale(int slot, int head) const {
    return static_cast<long long>(slot >> block_shift) * heads + head;
  }
};

inline bool valid_quantised(const ivit_quantised_layout& c) {
  const ivit_cache_layout l = {c.n_pages, c.page_size, c.kv_heads, c.head_dim, c.dtype, 0, c.page_stride, c.token_stride, c.head_stride};
  return valid_cache(l) && page_shift(c.block) >= 0 && c.block <= c.page_size;
}

inline QuantisedCache quantised(const ivit_quantised_layout& c) {
  return {c.n_pages, page_shift(c.page_size), page_shift(c.block), c.kv_heads, c.head_dim, c.page_stride, c.token_stride,
          c.head_stride};
}

}  // namespace ivit
