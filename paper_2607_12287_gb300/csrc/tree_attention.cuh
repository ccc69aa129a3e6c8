// What the two kernels of ivit_tree_attention share: the requests' bounds, the cutting of the work into
// equal runs, masks, and the join of what several runs leave of a tile of rows.
#pragma once

#include "attention.cuh"
#include "backbone.cuh"

namespace ivit {

constexpr int TREE_MAX_REQ = 4096;
constexpr int TREE_MAX_SMS = 256;   // the workspace has parts for that many
// Probabilities are kept 2^SHIFT times too large, which keeps small fp16 ones normal.
constexpr float TREE_SHIFT = 10.f;
// A row's reference maximum moves when a tile exceeds it by more than 2^GROWTH, not before: the output is
// rescaled a few times per run instead of for most tiles, and 2^(SHIFT + GROWTH) is an fp16 number.
constexpr float TREE_GROWTH = 5.f;

struct TreeArgs {
  const void *q, *k_new, *v_new, *k_cache, *v_cache;
  const int *table, *len, *cu;
  const uint32_t* mask;
  void* out;
  float *lse, *parts;
  int* err;                         // device error word of the tcgen05 kernel's bounded waits
  int4* joins;                      // [CTAs][2] the tile that CTA c's run begins and others go on with: key head
                                    // (-1: none), first of its rows in the request, the request's first row,
                                    // 2 * its parts + whether the first is c's second; rows of the tile
  long long q_stride, k_new_stride, v_new_stride, out_stride;
  PagedCache cache;
  int n_req, n_rows, heads, group, max_pages, max_new, mask_mode, mask_words;
  int tile_rows;                    // rows (new row x head of the group) of a tile
  float scale_log2;                 // scale * log2(e)
};

// Floats of a part in the workspace: output [m][dp] (of the tcgen05 kernel [m / 8][dp / 4][8][4]), then running maximum
// and sum of each row.
__host__ __device__ constexpr int tree_part_floats(int m, int dp) { return m * (dp + 2); }

// The tcgen05 kernel: dp 64, 80, 96, 128 or 256, pages of 8 tokens and more, groups of up to 128 heads; tiles of
// tree_tc_rows(group) rows, two CTAs per SM (of dp 256 one).
inline int tree_tc_rows(int group) { return 128 / group * group; }
cudaError_t launch_tree_attention_tc(const TreeArgs& a, int dtype, int dp, int ctas, cudaStream_t s);

// Rows and cached tokens of a request, within the bounds the host vouches for.
struct TreeRequest {
  int row0, n, len;
};

__device__ __forceinline__ TreeRequest tree_request(const TreeArgs& a, int i) {
  TreeRequest r;
  const int most = a.max_pages << a.cache.page_shift;
  const auto bounded = [&](int row) { return min(max(row, 0), a.n_rows); };  // (each by itself: their difference fits)
  r.row0 = bounded(a.cu[i]);
  r.n = min(max(bounded(a.cu[i + 1]) - r.row0, 0), a.max_new);
  r.len = min(max(a.len[i], 0), most);
  return r;
}

__device__ __forceinline__ int tree_row_tiles(const TreeArgs& a, const TreeRequest& r) {
  return (r.n * a.group + a.tile_rows - 1) / a.tile_rows;
}

// A place in a head's order of units (request, row tile, key tile).  Keys::tiles(r): key tiles of a request
// with rows.  Keys::LEAST: units of a run.
template <class Keys>
struct TreePlace {
  TreeRequest r;
  int req, head, rt, kt, nkt, nrt;

  __device__ __forceinline__ void enter(const TreeArgs& a, int i) {  // the first unit of request i or later
    for (req = i; req < a.n_req; ++req) {
      r = tree_request(a, req);
      if (r.n > 0) break;
    }
    nkt = Keys::tiles(r);
    nrt = tree_row_tiles(a, r);
    rt = kt = 0;
  }
  __device__ __forceinline__ void next_rows(const TreeArgs& a) {  // the first key tile of the next tile of rows
    kt = 0;
    if (++rt == nrt) enter(a, req + 1);
  }
  __device__ __forceinline__ void next(const TreeArgs& a) {
    if (++kt == nkt) next_rows(a);
  }
};

// (a division of 64-bit numbers is a subroutine; nearly all are small)
__device__ __forceinline__ unsigned long long tree_div(unsigned long long a, unsigned long long b) {
  return (a | b) >> 32 ? a / b : static_cast<unsigned>(a) / static_cast<unsigned>(b);
}

// The units [lo, hi) of this CTA: its key head's units, `total` of them, are cut into equal runs, and CTA c has
// run c / heads of head c % heads.  So the CTAs that read the heads of the same tokens, which lie side by side
// in the cache, do it at the same time: a head's 128 or 160 bytes of a token alone make poor use of DRAM.  A
// run has at least Keys::LEAST units but for the last few (none is empty between two that share a tile, and
// parts stay cheap beside the work on them).  `before` [n_req] is scratch in shared memory, free again after
// the call.
template <class Keys>
struct TreeRun {
  unsigned long long lo, hi, least, more;
  TreePlace<Keys> at;

  template <int THREADS>
  __device__ __forceinline__ bool find(const TreeArgs& a, unsigned long long* before) {
    __shared__ unsigned long long carry[THREADS / 32];
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    unsigned long long total = 0;
    for (int i0 = 0; i0 < a.n_req; i0 += THREADS) {
      const int i = i0 + tid;
      unsigned long long n = 0;
      if (i < a.n_req) {
        const TreeRequest r = tree_request(a, i);
        if (r.n > 0) n = static_cast<unsigned long long>(Keys::tiles(r)) * tree_row_tiles(a, r);
      }
      unsigned long long run = n;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const unsigned long long up = __shfl_up_sync(0xffffffffu, run, o);
        if (lane >= o) run += up;
      }
      if (lane == 31) carry[warp] = run;
      __syncthreads();
      unsigned long long ahead = total;
#pragma unroll
      for (int w = 0; w < THREADS / 32; ++w) {
        if (w < warp) ahead += carry[w];
        total += carry[w];
      }
      if (i < a.n_req) before[i] = ahead + run - n;
      __syncthreads();
    }
    if (tid == 0) a.joins[2 * blockIdx.x].x = -1;
    const unsigned run = blockIdx.x / a.cache.heads, all = gridDim.x / a.cache.heads;
    const unsigned long long most = tree_div(total + Keys::LEAST - 1, Keys::LEAST), runs = most < all ? most : all;
    if (run >= runs) return false;
    // the first `more` runs have one unit more than the others
    least = tree_div(total, runs);
    more = total - least * runs;
    lo = least * run + min(static_cast<unsigned long long>(run), more);
    hi = lo + least + (run < more ? 1 : 0);
    int i = 0, j = a.n_req - 1;  // last request with before <= lo: it has units
    while (i < j) {
      const int mid = (i + j + 1) >> 1;
      if (before[mid] <= lo) i = mid; else j = mid - 1;
    }
    const unsigned long long off = lo - before[i];
    at.enter(a, i);
    at.rt = static_cast<int>(tree_div(off, at.nkt));
    at.kt = static_cast<int>(off - static_cast<unsigned long long>(at.rt) * at.nkt);
    at.head = blockIdx.x - run * a.cache.heads;
    __syncthreads();
    return true;
  }

  // Notes that the run begins the tile of rows at `p` (as its second part or its first) and another ends it;
  // `unit`: the head's unit that is the tile's first.
  __device__ __forceinline__ void note_join(const TreeArgs& a, const TreePlace<Keys>& p, unsigned long long unit) const {
    const unsigned long long last = unit + p.nkt - 1, longer = more * (least + 1);
    const unsigned long long end = last < longer ? tree_div(last, least + 1) : more + tree_div(last - longer, least);  // its run
    const int parts = static_cast<int>(end) - static_cast<int>(blockIdx.x / a.cache.heads) + 1;
    const int x0 = p.rt * a.tile_rows;
    a.joins[2 * blockIdx.x] = make_int4(p.head, x0, p.r.row0, 2 * parts + (unit > lo ? 1 : 0));
    a.joins[2 * blockIdx.x + 1] = make_int4(min(a.tile_rows, p.r.n * a.group - x0), 0, 0, 0);
  }
};

}  // namespace ivit
