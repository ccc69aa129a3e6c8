// The entry points of the attention over a cache of 8 bits (ivit_tree_attention_quantised; the kernel is in
// tree_attention_quantised.cuh) and its form for rows of bf16.
#include "tree_attention_quantised.cuh"

namespace ivit {

cudaError_t launch_tree_attention_quantised_bf16(const QuantisedArgs& a, int dp, int nr, int ctas, cudaStream_t s) {
  return launch<bf16>(a, dp, nr, ctas, s);
}

namespace {

bool valid(const ivit_attention_config& c, const ivit_quantised_layout& l) {
  return valid_quantised(l) && valid_attention(c, l.kv_heads, l.page_size);
}

// More rows per key head than this take the tcgen05 kernel, where a group has at most 128 heads.  Both sides, 16 requests of up to
// 8192 tokens, us: 32 rows of heads of 64 65 (tcgen05) and 43, of 128 112 and 72, of 256 233 and 258; 40 rows of 64 68 and 50, of 96
// 80 and 84, of 128 114 and 90; 48 rows of 128 99 and 103 (fp16); 20 rows of 256 232 and 186.
constexpr int tc_rows(int dp) { return dp <= 128 ? 40 : 24; }

// Tiles of 8 nr rows, or with tc the tcgen05 kernel's.
struct Plan {
  bool tc;
  int dp, nr, tile_rows, ctas_per_sm, part_floats;
};

Plan plan(const ivit_attention_config& c, const ivit_quantised_layout& l) {
  const int group = c.heads / l.kv_heads;
  const long long rows = static_cast<long long>(c.max_new) * group;  // that share a key head
  const auto of = [&](auto d) {
    constexpr int DP = decltype(d)::value;
    if (rows > tc_rows(DP) && group <= 128) return Plan{true, DP, 0, tree_tc_rows(group), DP <= 128 ? 2 : 1, tree_part_floats(128, DP)};
    if constexpr (DP <= MOST_DP)
      if (rows > 8) return Plan{false, DP, 2, 16, Cfg<DP, 2>::CTAS, Cfg<DP, 2>::PART};
    return Plan{false, DP, 1, 8, Cfg<DP, 1>::CTAS, Cfg<DP, 1>::PART};
  };
  return l.head_dim <= 64    ? of(std::integral_constant<int, 64>{})
         : l.head_dim <= 80  ? of(std::integral_constant<int, 80>{})
         : l.head_dim <= 96  ? of(std::integral_constant<int, 96>{})
         : l.head_dim <= 128 ? of(std::integral_constant<int, 128>{})
                             : of(std::integral_constant<int, 256>{});
}

// The error word, then of each CTA a note and two parts.
size_t workspace_of(const Plan& p) {
  return 16 + static_cast<size_t>(p.ctas_per_sm) * TREE_MAX_SMS * (2 * sizeof(int4) + 2 * sizeof(float) * p.part_floats);
}

}  // namespace
}  // namespace ivit

extern "C" size_t ivit_tree_attention_quantised_workspace(const ivit_attention_config* cfg, const ivit_quantised_layout* cache) {
  return cfg && cache && ivit::valid(*cfg, *cache) ? ivit::workspace_of(ivit::plan(*cfg, *cache)) : 0;
}

extern "C" int ivit_tree_attention_quantised(const ivit_attention_config* cfg, const ivit_quantised_layout* cache, int32_t n_rows,
                                             const void* q_dev, int64_t q_stride, const void* k_new_dev, int64_t k_new_stride,
                                             const void* v_new_dev, int64_t v_new_stride, const void* k_cache_dev,
                                             const void* v_cache_dev, const float* k_scale_dev, const float* v_scale_dev,
                                             const int32_t* table_dev, const int32_t* len_dev, const int32_t* cu_rows_dev,
                                             const uint32_t* mask_dev, void* out_dev, int64_t out_stride, float* lse_dev,
                                             void* workspace_dev, size_t workspace_bytes, void* stream) {
  using namespace ivit;
  if (!cfg || !cache || n_rows < 0)
    return fail(IVIT_ERR_ARG, "ivit_tree_attention_quantised: null configuration or a negative row count");
  if (!valid(*cfg, *cache))
    return fail(IVIT_ERR_SHAPE,
                "ivit_tree_attention_quantised: need 1..4096 requests, heads up to 256 and a multiple of the cache's, head_dim "
                "a multiple of 8 up to 256, max_pages * page_size below 2^31 - 2^20, max_new 1..65536, a mask mode (trees with "
                "1..32768 mask words), scale > 0 and a supported cache layout");
  if (n_rows == 0) return IVIT_OK;
  if (!q_dev || !k_new_dev || !v_new_dev || !k_cache_dev || !v_cache_dev || !k_scale_dev || !v_scale_dev || !table_dev ||
      !len_dev || !cu_rows_dev || !out_dev || !workspace_dev || (cfg->mask_mode == IVIT_MASK_TREE && !mask_dev))
    return fail(IVIT_ERR_ARG, "ivit_tree_attention_quantised: null pointer");
  if ((q_stride | k_new_stride | v_new_stride | out_stride) & 7 || q_stride <= 0 || k_new_stride <= 0 || v_new_stride <= 0 ||
      out_stride <= 0)
    return fail(IVIT_ERR_ARG, "ivit_tree_attention_quantised: row strides must be positive multiples of 8 elements");
  if (!all_aligned({q_dev, k_new_dev, v_new_dev, out_dev, workspace_dev}, 16) || !all_aligned({k_cache_dev, v_cache_dev}, 8) ||
      !all_aligned({k_scale_dev, v_scale_dev, table_dev, len_dev, cu_rows_dev, mask_dev, lse_dev}, 4))
    return fail(IVIT_ERR_ARG,
                "ivit_tree_attention_quantised: rows and the workspace must be 16-byte aligned, caches 8-byte (scales, table, "
                "lengths, offsets, mask and lse 4)");
  const Plan p = plan(*cfg, *cache);
  if (workspace_bytes < workspace_of(p)) return fail(IVIT_ERR_ARG, "ivit_tree_attention_quantised: the workspace is too small");
  const int sms = sm_count();
  if (sms <= 0) return fail(IVIT_ERR_CUDA, "ivit_tree_attention_quantised: no CUDA device");
  QuantisedArgs a = {};
  a.q = q_dev;
  a.k_new = k_new_dev;
  a.v_new = v_new_dev;
  a.k_cache = k_cache_dev;
  a.v_cache = v_cache_dev;
  a.k_scale = k_scale_dev;
  a.v_scale = v_scale_dev;
  a.table = table_dev;
  a.len = len_dev;
  a.cu = cu_rows_dev;
  a.mask = mask_dev;
  a.out = out_dev;
  a.lse = lse_dev;
  a.q_stride = q_stride;
  a.k_new_stride = k_new_stride;
  a.v_new_stride = v_new_stride;
  a.out_stride = out_stride;
  const QuantisedCache c = quantised(*cache);
  a.cache = {c.n_pages, c.page_shift, c.heads, c.dim, c.page_stride, c.token_stride, c.head_stride};
  a.block_shift = c.block_shift;
  const bool lines = all_aligned({k_cache_dev, v_cache_dev}, 16) && (c.page_stride | c.token_stride) % 16 == 0;
  // Windows are built for 72 and 88 alone, in tiles of their own width.  Other heads of 8 more than a multiple of 16 are copied by 8
  // bytes, which costs (32 requests of up to 16384 tokens, 32 + 8 heads, us): 40 113 (of 48 70), 56 131 (of 64 63), 104 185 (of 112 104),
  // 120 189 (of 128 106), 136 581 (of 144 245), 248 631 (of 256 260).  The tcgen05 form converts on the way and copies 72 in halves too
  // (views of 256 rows 59 us, of 80 56).
  a.window = !p.tc && lines && (c.dim == 72 || c.dim == 88);
  a.wide = a.window || (lines && c.dim % 16 == 0 && c.head_stride % 16 == 0);
  a.n_req = cfg->n_req;
  a.n_rows = n_rows;
  a.heads = cfg->heads;
  a.group = cfg->heads / cache->kv_heads;
  a.max_pages = cfg->max_pages;
  a.max_new = cfg->max_new;
  a.mask_mode = cfg->mask_mode;
  a.mask_words = cfg->mask_words;
  a.scale_log2 = 1.f;
  a.score_log2 = cfg->scale * 1.4426950408889634f;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  // whole runs of all key heads, at least one (more CTAs than fit at a time wait for a place, not for each other)
  const int ctas = std::max(1, p.ctas_per_sm * std::min(TREE_MAX_SMS, sms) / cache->kv_heads) * cache->kv_heads;
  a.tile_rows = p.tile_rows;
  a.err = static_cast<int*>(workspace_dev);
  a.joins = static_cast<int4*>(workspace_dev) + 1;
  a.parts = reinterpret_cast<float*>(a.joins + 2 * p.ctas_per_sm * TREE_MAX_SMS);
  const cudaError_t e = p.tc                        ? launch_tree_attention_quantised_tc(a, cache->dtype, p.dp, ctas, s)
                        : cache->dtype == IVIT_BF16 ? launch_tree_attention_quantised_bf16(a, p.dp, p.nr, ctas, s)
                                                    : launch_tree_attention_quantised_fp16(a, p.dp, p.nr, ctas, s);
  return e == cudaSuccess ? IVIT_OK : fail_cuda(e);
}
