// Pages, slots, positions and tree masks of a step, from the requests' lengths (ivit_step_plan).
//
// With p(x) = ceil(x / page_size), request i takes max(0, p(base + new) - p(held)) pages from the
// front of the ring of free pages and returns what it holds beyond p(base + new) to its end, in
// request order: three running sums over the requests (rows, pages taken, pages returned) give
// every row, table entry and ring place independently of the others.
//
// Bound: latency (a launch, the lengths, the page ids).  Every CTA computes the sums over all
// requests for itself -- at most eight rounds of 512, from L2 -- instead of waiting for one that
// does, and then takes its share of the rows and of the requests' pages.  The page of a row that
// this step takes is read from the ring, not from the table another CTA is writing.  Measured: 8 requests 3.0 us,
// 512 requests with trees of up to 64 drafts 6.7 us.
#include "backbone.cuh"

namespace ivit {
namespace {

constexpr int THREADS = 512, WARPS = THREADS / 32;
constexpr int MAX_REQ = 4096, MAX_SPAN = 262144;  // (their product is below 2^31: the sums fit in 32 bits)

struct PlanArgs {
  const int *held, *base, *fresh, *parent, *ring_in;
  int *ring, *table, *cu, *req, *slot, *pos, *ring_out, *status;
  uint32_t* mask;
  int n_req, max_rows, max_pages, page_shift, n_pages, mask_words;
};

__device__ __forceinline__ unsigned pages_of(long long tokens, int shift) {
  return static_cast<unsigned>((tokens + (1 << shift) - 1) >> shift);
}

__global__ void __launch_bounds__(THREADS) step_plan_kernel(const PlanArgs a) {
  extern __shared__ int sm[];
  int* cu = sm;                     // [n_req + 1] rows before request i
  int* taken = cu + a.n_req + 1;    // [n_req] pages taken before it
  int* given = taken + a.n_req;     // [n_req] pages returned before it
  __shared__ int part[3][WARPS];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  pdl_wait();
  pdl_launch_dependents();
  const unsigned head = a.ring_in[0], count = a.ring_in[1];

  int why = 0;
  int sum[3] = {0, 0, 0};
  for (int i0 = 0; i0 < a.n_req; i0 += THREADS) {
    const int i = i0 + tid;
    int v[3] = {0, 0, 0};
    if (i < a.n_req) {
      const int held = a.held[i], base = a.base[i], fresh = a.fresh[i];
      if ((held | base | fresh) < 0) {
        why |= 8;
      } else {
        const unsigned have = pages_of(held, a.page_shift);
        const unsigned need = pages_of(static_cast<long long>(base) + fresh, a.page_shift);
        const unsigned most = a.max_pages;
        if (have > most || need > most) {
          why |= 2;
        } else {
          v[1] = need > have ? need - have : 0;
          v[2] = have > need ? have - need : 0;
        }
        v[0] = min(fresh, a.max_rows + 1);
      }
    }
    int run[3];
#pragma unroll
    for (int k = 0; k < 3; ++k) {
      run[k] = v[k];
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int up = __shfl_up_sync(0xffffffffu, run[k], o);
        if (lane >= o) run[k] += up;
      }
      if (lane == 31) part[k][warp] = run[k];
    }
    __syncthreads();
    int before[3] = {0, 0, 0}, all[3] = {0, 0, 0};
#pragma unroll
    for (int w = 0; w < WARPS; ++w)
#pragma unroll
      for (int k = 0; k < 3; ++k) {
        const int x = part[k][w];
        if (w < warp) before[k] += x;
        all[k] += x;
      }
    if (i < a.n_req) {
      cu[i] = sum[0] + before[0] + run[0] - v[0];
      taken[i] = sum[1] + before[1] + run[1] - v[1];
      given[i] = sum[2] + before[2] + run[2] - v[2];
    }
#pragma unroll
    for (int k = 0; k < 3; ++k) sum[k] += all[k];
    __syncthreads();  // (the warps' sums are read before the next round's)
  }
  if (tid == 0) cu[a.n_req] = sum[0];
  const unsigned places = a.n_pages;
  if (sum[0] > a.max_rows) why |= 4;
  if (head >= places || count > places) {
    why |= 8;
  } else if (static_cast<unsigned>(sum[1]) > count) {
    why |= 1;
  } else if (count + sum[2] > places) {  // (a page that is both free and held: returned ids would land on places that are
    why |= 8;                            // being read)
  }
  // every thread's reasons, in every thread
  int all_why = 0;
#pragma unroll
  for (int b = 1; b <= 8; b <<= 1) all_why |= __syncthreads_or(why & b) ? b : 0;
  const bool refused = all_why != 0;
  const int rows = refused ? 0 : sum[0];

  const int first = blockIdx.x * THREADS + tid, stride = gridDim.x * THREADS;
  for (int i = first; i <= a.n_req; i += stride) a.cu[i] = refused ? 0 : cu[i];
  if (first == 0) {
    a.ring_out[0] = refused ? head : (head + sum[1]) % places;
    a.ring_out[1] = refused ? count : count - sum[1] + sum[2];
    a.status[0] = all_why;
  }

  // the requests' pages, a warp each
  if (!refused)
    for (int i = blockIdx.x * WARPS + warp; i < a.n_req; i += gridDim.x * WARPS) {
      const int have = pages_of(a.held[i], a.page_shift);
      const int need = pages_of(static_cast<long long>(a.base[i]) + a.fresh[i], a.page_shift);
      int* row = a.table + static_cast<size_t>(i) * a.max_pages;
      for (int k = have + lane; k < need; k += 32) row[k] = a.ring[(head + taken[i] + k - have) % places];
      for (int k = need + lane; k < have; k += 32) a.ring[(head + count + given[i] + k - need) % places] = row[k];
    }

  for (int r = first; r < a.max_rows; r += stride) {
    uint32_t* words = a.mask ? a.mask + static_cast<size_t>(r) * a.mask_words : nullptr;
    if (r >= rows) {
      if (a.req) a.req[r] = -1;
      a.slot[r] = -1;
      if (a.pos) a.pos[r] = 0;
      if (words)
        for (int w = 0; w < a.mask_words; ++w) words[w] = 0;
      continue;
    }
    int lo = 0, hi = a.n_req - 1;  // last request with cu[i] <= r (requests without rows are passed over)
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (cu[mid] <= r) lo = mid; else hi = mid - 1;
    }
    const int i = lo, j = r - cu[i], base = a.base[i], at = base + j;
    const int page = at >> a.page_shift, have = pages_of(a.held[i], a.page_shift);
    const int id = page < have ? a.table[static_cast<size_t>(i) * a.max_pages + page]
                               : a.ring[(head + taken[i] + page - have) % places];
    if (a.req) a.req[r] = i;
    a.slot[r] = (id << a.page_shift) + (at & ((1 << a.page_shift) - 1));
    int depth = j;
    if (a.parent) {  // up the tree; a parent is an earlier row, so the words come in descending order
      const int* parent = a.parent + cu[i];
      depth = 0;
      if (words)
        for (int w = 0; w < a.mask_words; ++w) words[w] = 0;
      int k = j, w = j >> 5;
      uint32_t bits = 1u << (j & 31);
      for (;;) {
        const int p = parent[k];
        if (p < 0 || p >= k) break;
        ++depth;
        k = p;
        if (k >> 5 != w) {
          if (words && w < a.mask_words) words[w] = bits;
          w = k >> 5;
          bits = 0;
        }
        bits |= 1u << (k & 31);
      }
      if (words && w < a.mask_words) words[w] = bits;
    } else if (words) {
      for (int w = 0; w < a.mask_words; ++w) {
        const int n = j + 1 - 32 * w;  // bits of this word
        words[w] = n >= 32 ? 0xffffffffu : n > 0 ? (1u << n) - 1 : 0;
      }
    }
    if (a.pos) a.pos[r] = base + depth;
  }
}

}  // namespace
}  // namespace ivit

extern "C" int ivit_step_plan(const ivit_plan_config* cfg, const int32_t* held_dev, const int32_t* base_dev,
                              const int32_t* new_dev, const int32_t* parent_dev, int32_t* ring_dev,
                              const int32_t* ring_in_dev, int32_t* table_dev, int32_t* cu_rows_dev, int32_t* req_dev,
                              int32_t* slot_dev, int32_t* pos_dev, uint32_t* mask_dev, int32_t* ring_out_dev,
                              int32_t* status_dev, void* stream) {
  using namespace ivit;
  if (!cfg || !held_dev || !base_dev || !new_dev || !ring_dev || !ring_in_dev || !table_dev || !cu_rows_dev ||
      !ring_out_dev || !status_dev || (!slot_dev && cfg->max_rows > 0))
    return fail(IVIT_ERR_ARG, "ivit_step_plan: null pointer");
  if (!all_aligned({held_dev, base_dev, new_dev, parent_dev, ring_dev, ring_in_dev, table_dev, cu_rows_dev, req_dev,
                    slot_dev, pos_dev, mask_dev, ring_out_dev, status_dev}, 4))
    return fail(IVIT_ERR_ARG, "ivit_step_plan: arrays must be 4-byte aligned");
  if (ring_in_dev == ring_out_dev) return fail(IVIT_ERR_ARG, "ivit_step_plan: ring_out may not be ring_in");
  const int shift = page_shift(cfg->page_size);
  if (cfg->n_req < 1 || cfg->n_req > MAX_REQ || cfg->max_rows < 0 || cfg->max_rows > MAX_SPAN || cfg->max_pages < 1 ||
      cfg->max_pages > MAX_SPAN || shift < 0 || cfg->n_pages < 1 ||
      static_cast<long long>(cfg->n_pages) * cfg->page_size >= (1LL << 31) || cfg->mask_words < 0 ||
      cfg->mask_words > 32768)
    return fail(IVIT_ERR_SHAPE,
                "ivit_step_plan: need 1..4096 requests, up to 262144 rows and table columns, a page size that is a "
                "power of two up to 1024, fewer than 2^31 slots, up to 32768 mask words");
  const int sms = sm_count();
  if (sms <= 0) return fail(IVIT_ERR_CUDA, "ivit_step_plan: no CUDA device");
  const PlanArgs a = {held_dev, base_dev, new_dev, parent_dev, ring_in_dev, ring_dev, table_dev, cu_rows_dev, req_dev,
                      slot_dev, pos_dev, ring_out_dev, status_dev, cfg->mask_words ? mask_dev : nullptr, cfg->n_req,
                      cfg->max_rows, cfg->max_pages, shift, cfg->n_pages, cfg->mask_words};
  const int want = max((cfg->max_rows + THREADS - 1) / THREADS, (cfg->n_req + WARPS - 1) / WARPS);
  const size_t smem = sizeof(int) * (3 * static_cast<size_t>(cfg->n_req) + 1);
  // (the limit is set to the largest call's, never lower: another thread may be about to launch with it)
  constexpr int most = sizeof(int) * (3 * MAX_REQ + 1);
  cudaError_t e = smem <= 48000 ? cudaSuccess : allow_smem<step_plan_kernel>(most);
  if (e == cudaSuccess)
    e = launch_ex(step_plan_kernel, dim3(max(1, min(want, sms))), dim3(THREADS), smem,
                                  static_cast<cudaStream_t>(stream), 1, a);
  return e == cudaSuccess ? IVIT_OK : fail_cuda(e);
}
