// The attention over a cache of 8 bits for rows of fp16 (see tree_attention_quantised.cuh).
#include "tree_attention_quantised.cuh"

namespace ivit {

cudaError_t launch_tree_attention_quantised_fp16(const QuantisedArgs& a, int dp, int nr, int ctas, cudaStream_t s) {
  return launch<half>(a, dp, nr, ctas, s);
}

}  // namespace ivit
