// What the kernels of the language backbone share: 16-bit types, cache slots, host-side checks.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <stdint.h>

#include <atomic>
#include <initializer_list>

#include "internal.h"
#include "ivit.h"
#include "ptx.cuh"

namespace ivit {

void set_create_error(const char* msg);  // engine.cu: message for ivit_last_error(NULL)

using half = __half;

// Two values of a 32-bit word, and back (rounded to nearest even).
template <typename T>
__device__ __forceinline__ float2 unpack2(uint32_t w);
template <>
__device__ __forceinline__ float2 unpack2<bf16>(uint32_t w) {
  return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
}
template <>
__device__ __forceinline__ float2 unpack2<half>(uint32_t w) {
  return __half22float2(*reinterpret_cast<const __half2*>(&w));
}
template <typename T>
__device__ __forceinline__ uint32_t pack2(float lo, float hi);
template <>
__device__ __forceinline__ uint32_t pack2<bf16>(float lo, float hi) {
  const __nv_bfloat162 b = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&b);
}
template <>
__device__ __forceinline__ uint32_t pack2<half>(float lo, float hi) {
  const __half2 b = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&b);
}

// A paged cache of one layer (ivit_cache_layout), page size as a shift.
struct PagedCache {
  int n_pages, page_shift, heads, dim;
  long long page_stride, token_stride, head_stride;

  __device__ __forceinline__ bool holds(int slot) const { return slot >= 0 && (slot >> page_shift) < n_pages; }
  __device__ __forceinline__ long long token(int slot) const {  // element of head 0 of a slot
    return (slot >> page_shift) * page_stride + (slot & ((1 << page_shift) - 1)) * token_stride;
  }
};

inline int fail(int code, const char* msg) {
  set_create_error(msg);
  return code;
}

inline int fail_cuda(cudaError_t e) {
  set_create_error(cudaGetErrorString(e));
  return IVIT_ERR_CUDA;
}

inline bool aligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

inline bool all_aligned(std::initializer_list<const void*> ps, uintptr_t a) {  // (null is)
  for (const void* p : ps)
    if (!aligned(p, a)) return false;
  return true;
}

inline int page_shift(int page_size) {  // -1: not supported
  for (int s = 0; s <= 10; ++s)
    if (page_size == 1 << s) return s;
  return -1;
}

inline bool valid_cache(const ivit_cache_layout& c) {
  return page_shift(c.page_size) >= 0 && c.n_pages >= 1 &&
         static_cast<long long>(c.n_pages) * c.page_size < (1LL << 31) && c.kv_heads >= 1 && c.kv_heads <= 256 &&
         c.head_dim >= 8 && c.head_dim <= 256 && c.head_dim % 8 == 0 && (c.dtype == IVIT_BF16 || c.dtype == IVIT_FP16) &&
         c.page_stride >= 0 && c.token_stride >= 0 && c.head_stride >= 0 && c.page_stride % 8 == 0 &&
         c.token_stride % 8 == 0 && c.head_stride % 8 == 0;
}

inline PagedCache paged(const ivit_cache_layout& c) {
  return {c.n_pages, page_shift(c.page_size), c.kv_heads, c.head_dim, c.page_stride, c.token_stride, c.head_stride};
}

// Lets Kernel take `bytes` of dynamic shared memory, once per device.
template <auto Kernel>
cudaError_t allow_smem(int bytes) {
  static std::atomic<uint64_t> done{0};
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  const uint64_t bit = 1ull << (dev & 63);
  if (dev < 64 && (done.load(std::memory_order_relaxed) & bit)) return cudaSuccess;
  e = cudaFuncSetAttribute(Kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
  if (e == cudaSuccess && dev < 64) done.fetch_or(bit, std::memory_order_relaxed);
  return e;
}

// SMs of the current device, asked for at most once per device and thread; <= 0 on failure.
inline int sm_count() {
  thread_local int of = -1, sms = 0;
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return 0;
  if (dev != of) {
    if (cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) return 0;
    of = dev;
  }
  return sms;
}

}  // namespace ivit
