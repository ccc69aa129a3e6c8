// Keys and values of accepted rows, of all layers at once, into their slots of the paged caches
// (ivit_kv_write): a copy, one warp per (layer, row), lanes over the 16-byte pieces of its keys
// and then of its values, four of them in flight.
//
// Bound: a launch and two dependent reads (slot and row, then the data) for a few rows (5 rows of 27 layers 1.6 us);
// HBM for many: 2048 rows of 32 layers of 8 heads of 128 86 us, 6240 GB/s read and written.
#include "backbone.cuh"

namespace ivit {
namespace {

constexpr int THREADS = 256;

struct WriteArgs {
  const uint4 *k, *v;                     // in 16-byte pieces, as the strides here
  uint4 *k_cache, *v_cache;
  const int *row, *slot;
  long long row_stride, layer_stride, cache_layer_stride, page_stride, token_stride, head_stride;
  int n_layers, n, n_src, n_pages, page_shift, heads, pieces;  // pieces of a head
};

__global__ void __launch_bounds__(THREADS) kv_write_kernel(const WriteArgs a) {
  pdl_wait();
  pdl_launch_dependents();
  const int lane = threadIdx.x & 31;
  const long long warps = static_cast<long long>(gridDim.x) * (THREADS / 32);
  const long long all = static_cast<long long>(a.n_layers) * a.n;
  const int wide = a.heads * a.pieces;
  for (long long w = static_cast<long long>(blockIdx.x) * (THREADS / 32) + (threadIdx.x >> 5); w < all; w += warps) {
    const int layer = static_cast<int>(w / a.n), i = static_cast<int>(w - static_cast<long long>(layer) * a.n);
    const int row = a.row[i], slot = a.slot[i];
    if (row < 0 || row >= a.n_src || slot < 0 || slot >> a.page_shift >= a.n_pages) continue;
    const long long from = layer * a.layer_stride + row * a.row_stride;
    const long long to = layer * a.cache_layer_stride + (slot >> a.page_shift) * a.page_stride +
                         (slot & ((1 << a.page_shift) - 1)) * a.token_stride;
    for (int c0 = lane; c0 < 2 * wide; c0 += 4 * 32) {
      uint4 x[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int c = c0 + 32 * u;
        if (c < 2 * wide) x[u] = c < wide ? a.k[from + c] : a.v[from + c - wide];
      }
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        int c = c0 + 32 * u;
        if (c >= 2 * wide) continue;
        uint4* cache = a.k_cache;
        if (c >= wide) {
          cache = a.v_cache;
          c -= wide;
        }
        const int h = c / a.pieces;
        cache[to + h * a.head_stride + c - h * a.pieces] = x[u];
      }
    }
  }
}

}  // namespace
}  // namespace ivit

extern "C" int ivit_kv_write(const ivit_cache_layout* cache, int32_t n_layers, int32_t n, int32_t n_src,
                             const void* k_dev, const void* v_dev, int64_t row_stride, int64_t layer_stride,
                             const int32_t* src_row_dev, const int32_t* slot_dev, void* k_cache_dev, void* v_cache_dev,
                             int64_t cache_layer_stride, void* stream) {
  using namespace ivit;
  if (!cache || n_layers < 0 || n < 0 || n_src < 0)
    return fail(IVIT_ERR_ARG, "ivit_kv_write: null cache layout or a negative size");
  if (!valid_cache(*cache)) return fail(IVIT_ERR_SHAPE, "ivit_kv_write: cache layout not supported");
  if (row_stride < 0 || layer_stride < 0 || cache_layer_stride < 0 || row_stride % 8 || layer_stride % 8 ||
      cache_layer_stride % 8)
    return fail(IVIT_ERR_ARG, "ivit_kv_write: strides must be multiples of 8 elements");
  if (n_layers == 0 || n == 0 || n_src == 0) return IVIT_OK;
  if (!k_dev || !v_dev || !src_row_dev || !slot_dev || !k_cache_dev || !v_cache_dev)
    return fail(IVIT_ERR_ARG, "ivit_kv_write: null pointer");
  if (!all_aligned({k_dev, v_dev, k_cache_dev, v_cache_dev}, 16) || !all_aligned({src_row_dev, slot_dev}, 4))
    return fail(IVIT_ERR_ARG, "ivit_kv_write: arrays must be 16-byte aligned, indices 4-byte");
  const int sms = sm_count();
  if (sms <= 0) return fail(IVIT_ERR_CUDA, "ivit_kv_write: no CUDA device");
  const WriteArgs a = {static_cast<const uint4*>(k_dev), static_cast<const uint4*>(v_dev), static_cast<uint4*>(k_cache_dev),
                       static_cast<uint4*>(v_cache_dev), src_row_dev, slot_dev, row_stride / 8, layer_stride / 8,
                       cache_layer_stride / 8, cache->page_stride / 8, cache->token_stride / 8, cache->head_stride / 8,
                       n_layers, n, n_src, cache->n_pages, page_shift(cache->page_size), cache->kv_heads,
                       cache->head_dim / 8};
  const long long blocks = (static_cast<long long>(n_layers) * n + THREADS / 32 - 1) / (THREADS / 32);
  const int grid = static_cast<int>(blocks < 8LL * sms ? blocks : 8LL * sms);
  const cudaError_t e = launch_ex(kv_write_kernel, dim3(grid), dim3(THREADS), 0, static_cast<cudaStream_t>(stream), 1, a);
  return e == cudaSuccess ? IVIT_OK : fail_cuda(e);
}
