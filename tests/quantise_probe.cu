// ivit_kv_quantise around a wait that gives up although the copies it waited for have landed: in some CTAs one thread's, at the
// first unit (expire 1) or once all stages have been filled again (expire 2); 0: none.  A shared library, for the GPU tests.
#include "../paper_2607_12287_gb300/csrc/quantised.cuh"
#include "../paper_2607_12287_gb300/csrc/tree_attention.cuh"

namespace ivit {
__device__ int g_expire;
__device__ unsigned g_expired;  // waits that gave up
namespace {
__device__ bool wait_or_give_up(uint32_t bar, uint32_t parity) {
  if (!mbar_wait(bar, parity)) return false;
  const unsigned cta = blockIdx.x + blockIdx.y + blockIdx.z;
  if (g_expire == 0 || cta % 3 == 1 || threadIdx.x != 7 + 31 * (cta & 3) || parity + 1 != g_expire) return true;
  atomicAdd(&g_expired, 1u);
  return false;
}
}  // namespace
}  // namespace ivit

#define mbar_wait wait_or_give_up
#include "../paper_2607_12287_gb300/csrc/kv_quantise.cu"
#undef mbar_wait

extern "C" int probe_expire(int expire) { return cudaMemcpyToSymbol(ivit::g_expire, &expire, sizeof expire); }
extern "C" int probe_expired() {  // how many waits gave up so far
  unsigned n = 0;
  return cudaMemcpyFromSymbol(&n, ivit::g_expired, sizeof n) == cudaSuccess ? static_cast<int>(n) : -1;
}
