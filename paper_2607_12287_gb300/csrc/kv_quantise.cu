// Keys and values of accepted rows, of all layers at once, into their slots of a cache of 8 bits (ivit_kv_quantise), and
// cached tokens back as rows (ivit_kv_dequantise).
//
//   code = rn_e4m3(x / 2^e),  e = the smallest in [-60, 60] with max |x| <= 448 2^e
//
// over the finite values of a block of tokens and head; a block that keeps earlier tokens has an e that is not below the old
// one, and rounds them again if it grew.  e4m3 is a floating-point format, so a power of two costs no precision against
// max / 448 (but at the subnormal end), makes x / 2^e exact, and lets a block's scale grow without a second rounding.
//
// Writing: a warp has a unit of (layer, keys or values, head, some entries of the list).  Entries of one block lie next to each other; the
// first of them does the block: a row's 16-byte pieces go to neighbouring lanes, several rows at a time, and stay in
// registers between the maximum and the rounding where the block has few rows in the call.
// Reading: a warp has a unit of (layer, entry) as in kv_write.cu.
#include <algorithm>

#include "quantised.cuh"

namespace ivit {
namespace {

constexpr int THREADS = 256, WARPS = THREADS / 32;
constexpr int MIN_E = -60, MAX_E = 60;
constexpr int MAX_ROWS = 1 << 30;
constexpr int HELD = 8;  // passes over rows whose values stay in registers

struct QuantiseArgs {
  const void *k, *v;
  uint8_t *k_cache, *v_cache;
  float *k_scale, *v_scale;
  const int *row, *slot;
  long long row_stride, layer_stride, cache_layer_stride, scale_layer_stride;
  QuantisedCache cache;
  int n_layers, n, n_src, entries;  // entries of a unit
};

__device__ __forceinline__ float power(int e) { return __int_as_float((e + 127) << 23); }

// Exponent of the smallest power of two by which `size` (finite, >= 0) is at most 448 = 1.75 * 2^8.
__device__ __forceinline__ int exponent_for(float size) {
  const uint32_t b = __float_as_uint(size);
  return static_cast<int>(b >> 23) - 127 - 8 + ((b & 0x7fffffu) > 0x600000u ? 1 : 0);
}
// ... of two that is at least `scale`; very low for one that is not positive and finite.
__device__ __forceinline__ int exponent_of(float scale) {
  if (!(scale > 0.f && scale < INFINITY)) return -1000;
  const uint32_t b = __float_as_uint(scale);
  return static_cast<int>(b >> 23) - 127 + (b & 0x7fffffu ? 1 : 0);
}

// max(size, |x|) over the finite ones of the 8 values of a piece.
template <typename T>
__device__ __forceinline__ float largest(const uint4& x, float size) {
  const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 y = unpack2<T>(w[i]);
    const float a = fabsf(y.x), b = fabsf(y.y);
    size = fmaxf(size, fmaxf(a < INFINITY ? a : 0.f, b < INFINITY ? b : 0.f));
  }
  return size;
}

template <typename T>
__device__ __forceinline__ uint2 codes_of(const uint4& x, float inverse) {
  const uint32_t w[4] = {x.x, x.y, x.z, x.w};
  uint32_t c[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 y = unpack2<T>(w[i]);
    const auto one = [&](float v) { return fabsf(v) < INFINITY ? v * inverse : __uint_as_float(0x7fffffffu); };
    c[i] = to_codes2(one(y.x), one(y.y));
  }
  return make_uint2(c[0] | c[1] << 16, c[2] | c[3] << 16);
}

template <typename T>
__global__ void __launch_bounds__(THREADS) kv_quantise_kernel(const QuantiseArgs a) {
  pdl_wait();
  pdl_launch_dependents();
  constexpr unsigned ALL = 0xffffffffu;
  const int lane = threadIdx.x & 31;
  const int pieces = a.cache.dim >> 3, rows_at_once = 32 / pieces;
  const int my_row = lane / pieces, my_piece = lane - my_row * pieces;
  const bool used = my_row < rows_at_once;
  const int block = 1 << a.cache.block_shift;
  const int groups = (a.n + a.entries - 1) / a.entries;
  const long long units = static_cast<long long>(a.n_layers) * groups * 2 * a.cache.heads;
  const long long warps = static_cast<long long>(gridDim.x) * WARPS;
  for (long long unit = static_cast<long long>(blockIdx.x) * WARPS + (threadIdx.x >> 5); unit < units; unit += warps) {
    // heads side by side, as they lie in a row
    const long long rest = unit / a.cache.heads;
    const int head = static_cast<int>(unit - rest * a.cache.heads);
    const long long rest2 = rest >> 1;
    const bool values = rest & 1;
    const int layer = static_cast<int>(rest2 / groups), i0 = static_cast<int>(rest2 - static_cast<long long>(layer) * groups) * a.entries;
    // Blocks that begin among the unit's entries: an entry whose nearest one before it that counts is of another block.
    const int mine = i0 + lane;
    const int slot = lane < a.entries && mine < a.n ? a.slot[mine] : -1;
    bool first = a.cache.holds(slot);
    if (first) {
      for (int j = mine - 1; j >= 0; --j) {
        const int s = a.slot[j];
        if (!a.cache.holds(s)) continue;
        first = s >> a.cache.block_shift != slot >> a.cache.block_shift;
        break;
      }
    }
    unsigned todo = __ballot_sync(ALL, first);
    const T* const src = static_cast<const T*>(values ? a.v : a.k) + layer * a.layer_stride + static_cast<long long>(head) * a.cache.dim + 8 * my_piece;
    uint8_t* const cache = (values ? a.v_cache : a.k_cache) + layer * a.cache_layer_stride + head * a.cache.head_stride + 8 * my_piece;
    float* const scales = (values ? a.v_scale : a.k_scale) + layer * a.scale_layer_stride;
    while (todo) {
      const int at = __ffs(todo) - 1;
      todo &= todo - 1;
      const int i = i0 + at, id = __shfl_sync(ALL, slot, at) >> a.cache.block_shift;
      // How far the block's entries go, and which of its places they write (lane l: places 32 l .. 32 l + 31).
      unsigned written = 0;
      int end = i, last = -1;
      for (int j = i;; j += 32) {
        const int s = j + lane < a.n ? a.slot[j + lane] : -1;
        const bool holds = a.cache.holds(s), same = holds && s >> a.cache.block_shift == id;
        const unsigned others = __ballot_sync(ALL, holds && !same);
        const int limit = others ? __ffs(others) - 1 : 32;  // entries from here on are not the block's
        const int r = same && lane < limit ? a.row[j + lane] : -1;
        unsigned good = __ballot_sync(ALL, static_cast<unsigned>(r) < static_cast<unsigned>(a.n_src));
        if (good) end = j + 32 - __clz(good);
        while (good) {
          const int b = __ffs(good) - 1;
          good &= good - 1;
          const int place = __shfl_sync(ALL, s, b) & (block - 1);
          if (place >> 5 == lane) written |= 1u << (place & 31);
          last = max(last, place);
        }
        if (limit < 32 || j + 32 >= a.n) break;
      }
      if (last < 0) continue;  // none of them has a row
      const int before = last - 32 * lane;  // places of the lane's that are before the last
      const unsigned all_before = before >= 32 ? ALL : before > 0 ? (1u << before) - 1 : 0u;
      const unsigned stays = all_before & ~written;
      const bool keeps = __any_sync(ALL, stays != 0);

      // rows of the call, rows_at_once of them to a pass
      const auto row_of = [&](int j, int& s) {  // -1: not one of the block's
        s = j < end ? a.slot[j] : -1;
        const int r = a.cache.holds(s) ? a.row[j] : -1;
        return static_cast<unsigned>(r) < static_cast<unsigned>(a.n_src) ? r : -1;
      };
      uint4 x[HELD];
      int to[HELD];
      float size = 0.f;
#pragma unroll
      for (int p = 0; p < HELD; ++p) {
        int s;
        const int r = used && i + p * rows_at_once < end ? row_of(i + p * rows_at_once + my_row, s) : -1;
        to[p] = r >= 0 ? s : -1;
        x[p] = r >= 0 ? *reinterpret_cast<const uint4*>(src + r * a.row_stride) : make_uint4(0, 0, 0, 0);
      }
#pragma unroll
      for (int p = 0; p < HELD; ++p) size = largest<T>(x[p], size);
      const int beyond = i + HELD * rows_at_once;
      for (int j = beyond; j < end; j += rows_at_once) {
        int s;
        const int r = used ? row_of(j + my_row, s) : -1;
        if (r >= 0) size = largest<T>(*reinterpret_cast<const uint4*>(src + r * a.row_stride), size);
      }
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) size = fmaxf(size, __shfl_xor_sync(ALL, size, o));
      float* const scale = scales + static_cast<long long>(id) * a.cache.heads + head;
      int e = exponent_for(size);
      float old = 0.f;
      if (keeps) {
        old = *scale;
        e = max(e, exponent_of(old));
      }
      e = min(max(e, MIN_E), MAX_E);
      const float fresh = power(e), inverse = power(-e);
      __syncwarp();  // (the scale has been read)
      if (lane == 0 && !(keeps && old == fresh)) *scale = fresh;
      if (keeps && old != fresh) {
        const float ratio = old > 0.f && old < INFINITY ? old * inverse : 0.f;
        for (int p0 = 0; p0 < last; p0 += rows_at_once) {
          const int place = p0 + my_row;
          const unsigned bits = __shfl_sync(ALL, stays, (place >> 5) & 31);
          if (!used || place >= last || !(bits >> (place & 31) & 1)) continue;
          uint2* c = reinterpret_cast<uint2*>(cache + a.cache.token((id << a.cache.block_shift) + place));
          const uint2 w = *c;
          const auto again = [&](uint32_t word) {
            uint32_t lo, hi;
            codes_to_half4(word, lo, hi);
            const float2 p = unpack2<half>(lo), q = unpack2<half>(hi);
            return to_codes2(p.x * ratio, p.y * ratio) | to_codes2(q.x * ratio, q.y * ratio) << 16;
          };
          *c = make_uint2(again(w.x), again(w.y));
        }
      }
#pragma unroll
      for (int p = 0; p < HELD; ++p)
        if (to[p] >= 0) *reinterpret_cast<uint2*>(cache + a.cache.token(to[p])) = codes_of<T>(x[p], inverse);
      for (int j = beyond; j < end; j += rows_at_once) {
        int s;
        const int r = used ? row_of(j + my_row, s) : -1;
        if (r >= 0)
          *reinterpret_cast<uint2*>(cache + a.cache.token(s)) = codes_of<T>(*reinterpret_cast<const uint4*>(src + r * a.row_stride), inverse);
      }
    }
  }
}

struct DequantiseArgs {
  const uint8_t *k_cache, *v_cache;
  const float *k_scale, *v_scale;
  const int* slot;
  void *k, *v;
  long long row_stride, layer_stride, cache_layer_stride, scale_layer_stride;
  QuantisedCache cache;
  int n_layers, n;
};

// 8 codes times their scale.
template <typename T>
__device__ __forceinline__ uint4 values_of(uint2 c, float scale) {
  uint32_t h[4];
  codes_to_half4(c.x, h[0], h[1]);
  codes_to_half4(c.y, h[2], h[3]);
  uint32_t y[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 f = unpack2<half>(h[i]);
    y[i] = pack2<T>(f.x * scale, f.y * scale);
  }
  return make_uint4(y[0], y[1], y[2], y[3]);
}

template <typename T>
__global__ void __launch_bounds__(THREADS) kv_dequantise_kernel(const DequantiseArgs a) {
  pdl_wait();
  pdl_launch_dependents();
  constexpr int U = 4;  // pieces of a lane in flight
  const int lane = threadIdx.x & 31, pieces = a.cache.dim >> 3, wide = a.cache.heads * pieces;
  const long long warps = static_cast<long long>(gridDim.x) * WARPS, all = static_cast<long long>(a.n_layers) * a.n;
  for (long long w = static_cast<long long>(blockIdx.x) * WARPS + (threadIdx.x >> 5); w < all; w += warps) {
    const int layer = static_cast<int>(w / a.n), i = static_cast<int>(w - static_cast<long long>(layer) * a.n);
    const int slot = a.slot[i];
    if (!a.cache.holds(slot)) continue;
    const long long from = layer * a.cache_layer_stride + a.cache.token(slot), row = layer * a.layer_stride + i * a.row_stride;
    const long long scale = layer * a.scale_layer_stride + a.cache.scale(slot, 0);
    for (int c0 = lane; c0 < 2 * wide; c0 += 32 * U) {
      uint2 x[U];
      float s[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int c = c0 + 32 * u, d = c < wide ? c : c - wide, h = d / pieces;
        if (c >= 2 * wide) continue;
        x[u] = *reinterpret_cast<const uint2*>((c < wide ? a.k_cache : a.v_cache) + from + h * a.cache.head_stride + 8 * (d - h * pieces));
        s[u] = (c < wide ? a.k_scale : a.v_scale)[scale + h];
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int c = c0 + 32 * u, d = c < wide ? c : c - wide;
        if (c >= 2 * wide) continue;
        *reinterpret_cast<uint4*>(static_cast<T*>(c < wide ? a.k : a.v) + row + 8 * d) = values_of<T>(x[u], s[u]);
      }
    }
  }
}

}  // namespace
}  // namespace ivit

extern "C" int ivit_kv_quantise(const ivit_quantised_layout* cache, int32_t n_layers, int32_t n, int32_t n_src,
                                const void* k_dev, const void* v_dev, int64_t row_stride, int64_t layer_stride,
                                const int32_t* src_row_dev, const int32_t* slot_dev, void* k_cache_dev, void* v_cache_dev,
                                int64_t cache_layer_stride, float* k_scale_dev, float* v_scale_dev,
                                int64_t scale_layer_stride, void* stream) {
  using namespace ivit;
  if (!cache || n_layers < 0 || n < 0 || n_src < 0)
    return fail(IVIT_ERR_ARG, "ivit_kv_quantise: null cache layout or a negative size");
  if (!valid_quantised(*cache) || n > MAX_ROWS)
    return fail(IVIT_ERR_SHAPE, "ivit_kv_quantise: cache layout not supported, or more than 2^30 entries");
  if (row_stride < 0 || layer_stride < 0 || cache_layer_stride < 0 || scale_layer_stride < 0 || row_stride % 8 ||
      layer_stride % 8 || cache_layer_stride % 8)
    return fail(IVIT_ERR_ARG, "ivit_kv_quantise: strides must not be negative, and multiples of 8 (of scales any)");
  if (n_layers == 0 || n == 0 || n_src == 0) return IVIT_OK;
  if (!k_dev || !v_dev || !src_row_dev || !slot_dev || !k_cache_dev || !v_cache_dev || !k_scale_dev || !v_scale_dev)
    return fail(IVIT_ERR_ARG, "ivit_kv_quantise: null pointer");
  if (!all_aligned({k_dev, v_dev}, 16) || !all_aligned({k_cache_dev, v_cache_dev}, 8) ||
      !all_aligned({src_row_dev, slot_dev, k_scale_dev, v_scale_dev}, 4))
    return fail(IVIT_ERR_ARG, "ivit_kv_quantise: rows must be 16-byte aligned, caches 8-byte, indices and scales 4-byte");
  const int sms = sm_count();
  if (sms <= 0) return fail(IVIT_ERR_CUDA, "ivit_kv_quantise: no CUDA device");
  QuantiseArgs a = {k_dev, v_dev, static_cast<uint8_t*>(k_cache_dev), static_cast<uint8_t*>(v_cache_dev), k_scale_dev, v_scale_dev,
                    src_row_dev, slot_dev, row_stride, layer_stride, cache_layer_stride, scale_layer_stride, quantised(*cache),
                    n_layers, n, n_src, 1};
  // One entry to a unit while the chip has places for them all, then as many as a block can have next to each other.
  const long long parts = 2LL * n_layers * cache->kv_heads, resident = 64LL * sms;
  if (parts * n > resident) a.entries = std::min(32, std::max(8, cache->block));
  const long long blocks = (parts * ((n + a.entries - 1) / a.entries) + WARPS - 1) / WARPS;
  const int grid = static_cast<int>(std::min(blocks, 8LL * sms));
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  const cudaError_t e = cache->dtype == IVIT_BF16 ? launch_ex(kv_quantise_kernel<bf16>, dim3(grid), dim3(THREADS), 0, s, 1, a)
                                                  : launch_ex(kv_quantise_kernel<half>, dim3(grid), dim3(THREADS), 0, s, 1, a);
  return e == cudaSuccess ? IVIT_OK : fail_cuda(e);
}

extern "C" int ivit_kv_dequantise(const ivit_quantised_layout* cache, int32_t n_layers, int32_t n, const int32_t* slot_dev,
                                  const void* k_cache_dev, const void* v_cache_dev, int64_t cache_layer_stride,
                                  const float* k_scale_dev, const float* v_scale_dev, int64_t scale_layer_stride,
                                  void* k_dev, void* v_dev, int64_t row_stride, int64_t layer_stride, void* stream) {
  using namespace ivit;
  if (!cache || n_layers < 0 || n < 0)
    return fail(IVIT_ERR_ARG, "ivit_kv_dequantise: null cache layout or a negative size");
  if (!valid_quantised(*cache) || n > MAX_ROWS)
    return fail(IVIT_ERR_SHAPE, "ivit_kv_dequantise: cache layout not supported, or more than 2^30 entries");
  if (row_stride < 0 || layer_stride < 0 || cache_layer_stride < 0 || scale_layer_stride < 0 || row_stride % 8 ||
      layer_stride % 8 || cache_layer_stride % 8)
    return fail(IVIT_ERR_ARG, "ivit_kv_dequantise: strides must not be negative, and multiples of 8 (of scales any)");
  if (n_layers == 0 || n == 0) return IVIT_OK;
  if (!k_dev || !v_dev || !slot_dev || !k_cache_dev || !v_cache_dev || !k_scale_dev || !v_scale_dev)
    return fail(IVIT_ERR_ARG, "ivit_kv_dequantise: null pointer");
  if (!all_aligned({k_dev, v_dev}, 16) || !all_aligned({k_cache_dev, v_cache_dev}, 8) ||
      !all_aligned({slot_dev, k_scale_dev, v_scale_dev}, 4))
    return fail(IVIT_ERR_ARG, "ivit_kv_dequantise: rows must be 16-byte aligned, caches 8-byte, indices and scales 4-byte");
  const int sms = sm_count();
  if (sms <= 0) return fail(IVIT_ERR_CUDA, "ivit_kv_dequantise: no CUDA device");
  const DequantiseArgs a = {static_cast<const uint8_t*>(k_cache_dev), static_cast<const uint8_t*>(v_cache_dev), k_scale_dev, v_scale_dev,
                            slot_dev, k_dev, v_dev, row_stride, layer_stride, cache_layer_stride, scale_layer_stride,
                            quantised(*cache), n_layers, n};
  const long long blocks = (static_cast<long long>(n_layers) * n + WARPS - 1) / WARPS;
  const int grid = static_cast<int>(std::min(blocks, 8LL * sms));
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  const cudaError_t e = cache->dtype == IVIT_BF16 ? launch_ex(kv_dequantise_kernel<bf16>, dim3(grid), dim3(THREADS), 0, s, 1, a)
                                                  : launch_ex(kv_dequantise_kernel<half>, dim3(grid), dim3(THREADS), 0, s, 1, a);
  return e == cudaSuccess ? IVIT_OK : fail_cuda(e);
}
