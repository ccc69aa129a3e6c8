// The second kernel of the tree attentions (16-bit and 8-bit caches): joins the parts that several runs have of a tile of rows.
#pragma once

#include <algorithm>

#include "tree_attention.cuh"

namespace ivit {
namespace {

// Joins the parts of a tile of rows that several runs have, in the order of their keys.  Blocks (i, y) take the
// tile that CTA i's run begins or, where the call has few tiles (`search`), look for the i-th of them among the
// runs' notes.  A thread has 4 columns of a row, an element of the parts.  Up to FEW parts, it reads four parts
// at a time; more parts are shared by the warps of a block, 32 elements at a time, which meet in shared memory.
// TC: the parts are the tcgen05 kernel's.
template <typename T, int DP, int M, bool TC>
__global__ void __launch_bounds__(256) tree_join_kernel(const TreeArgs a, int ctas, bool search) {
  constexpr int PART = tree_part_floats(M, DP), WARPS = 8, FEW = 16, NOTES = 4;
  static_assert(NOTES * 256 >= 4 * TREE_MAX_SMS, "the notes of all CTAs");
  __shared__ float2 ml_of[WARPS][32];
  __shared__ float4 o_of[WARPS][32];
  __shared__ int found[NOTES][WARPS], which;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  if (tid == 0) which = -1;
  pdl_wait();
  // (Dependents start when the blocks end: launched earlier, the next call's CTAs that find no room beside these
  // begin their equal shares late; 64 requests with heads of 64 took 65 us instead of 49.)
  int c = blockIdx.x;
  if (search) {
    bool has[NOTES];
    unsigned mine[NOTES];
#pragma unroll
    for (int k = 0; k < NOTES; ++k) has[k] = 256 * k + tid < ctas && a.joins[2 * (256 * k + tid)].x >= 0;
#pragma unroll
    for (int k = 0; k < NOTES; ++k) {
      mine[k] = __ballot_sync(0xffffffffu, has[k]);
      if (lane == 0) found[k][warp] = __popc(mine[k]);
    }
    __syncthreads();
    int before = 0;
#pragma unroll
    for (int k = 0; k < NOTES; ++k) {
      int rank = before + __popc(mine[k] & ((1u << lane) - 1));
#pragma unroll
      for (int w = 0; w < WARPS; ++w) {
        if (w < warp) rank += found[k][w];
        before += found[k][w];
      }
      if (has[k] && rank == static_cast<int>(blockIdx.x)) which = 256 * k + tid;
    }
    __syncthreads();
    c = which;
    if (c < 0) return;
  }
  const int4 note = a.joins[2 * c], rest = a.joins[2 * c + 1];
  if (note.x < 0) return;
  const int head = note.x, x0 = note.y, row0 = note.z, n = note.w >> 1, rows = rest.x;
  // the tile's parts: CTA c's second or first, then the first ones of the head's CTAs behind it
  const float* parts = a.parts + static_cast<size_t>(2 * c) * PART;
  const auto part = [&](int i) { return parts + static_cast<size_t>(2 * i * a.cache.heads + (i == 0 ? note.w & 1 : 0)) * PART; };
  const int elements = TC ? (rows + 7) / 8 * (2 * DP) : rows * (DP / 4);
  const auto place = [&](int e, int& row, int& col) {  // columns 4 col .. 4 col + 3 of a row; whether it is one of the tile's
    const int g = e / (TC ? 2 * DP : DP / 4), w = e - g * (TC ? 2 * DP : DP / 4);
    row = TC ? 8 * g + (w & 7) : g;
    col = TC ? w >> 3 : w;
    return e < elements && row < rows;
  };
  // element e of parts i, i + step, i + 2 step, i + 3 step, into (m, l, o)
  const auto add4 = [&](int i, int step, int e, int row, float& m, float& l, float4& o) {
    float2 ml[4];
    float4 x[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      ml[k] = make_float2(-INFINITY, 0.f);
      x[k] = make_float4(0.f, 0.f, 0.f, 0.f);
      if (i + k * step < n) {
        const float* p = part(i + k * step);
        ml[k] = *reinterpret_cast<const float2*>(p + M * DP + 2 * row);
        x[k] = reinterpret_cast<const float4*>(p)[e];
      }
    }
    const float top = fmaxf(fmaxf(m, fmaxf(ml[0].x, ml[1].x)), fmaxf(ml[2].x, ml[3].x)), ref = top == -INFINITY ? 0.f : top;
    const float f = ex2((m - ref) * a.scale_log2);
    m = top;
    l *= f;
    o = make_float4(o.x * f, o.y * f, o.z * f, o.w * f);
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (i + k * step < n) {
        const float g = ex2((ml[k].x - ref) * a.scale_log2);
        l += ml[k].y * g;
        o = make_float4(o.x + x[k].x * g, o.y + x[k].y * g, o.z + x[k].z * g, o.w + x[k].w * g);
      }
  };
  const auto write = [&](int row, int col, float m, float l, const float4& o) {
    const int x = x0 + row, node = x / a.group, h = head * a.group + x - node * a.group;
    const long long orow = row0 + node;
    const float inv = l == 0.f ? 0.f : 1.f / l;
    if (4 * col < a.cache.dim)
      *reinterpret_cast<uint2*>(static_cast<T*>(a.out) + orow * a.out_stride + static_cast<long long>(h) * a.cache.dim + 4 * col) =
          make_uint2(pack2<T>(o.x * inv, o.y * inv), pack2<T>(o.z * inv, o.w * inv));
    if (a.lse && col == 0) a.lse[orow * a.heads + h] = (m * a.scale_log2 + (log2f(l) - TREE_SHIFT)) * 0.6931471805599453f;
  };

  if (n <= FEW) {
    for (int e = blockIdx.y * 256 + tid; e < elements; e += gridDim.y * 256) {
      int row, col;
      if (!place(e, row, col)) continue;
      float m = -INFINITY, l = 0.f;
      float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
      for (int i = 0; i < n; i += 4) add4(i, 1, e, row, m, l, o);
      write(row, col, m, l, o);
    }
    return;
  }
  for (int first = blockIdx.y * 32; first < elements; first += gridDim.y * 32) {
    int row, col;
    const bool has = place(first + lane, row, col);
    float m = -INFINITY, l = 0.f;
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
    if (has)
      for (int i = warp; i < n; i += 4 * WARPS) add4(i, WARPS, first + lane, row, m, l, o);
    ml_of[warp][lane] = make_float2(m, l);
    o_of[warp][lane] = o;
    __syncthreads();
    if (warp == 0 && has) {
#pragma unroll
      for (int w = 1; w < WARPS; ++w) m = fmaxf(m, ml_of[w][lane].x);
      const float ref = m == -INFINITY ? 0.f : m;
      l = 0.f;
      o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int w = 0; w < WARPS; ++w) {
        const float2 ml = ml_of[w][lane];
        const float4 x = o_of[w][lane];
        const float g = ex2((ml.x - ref) * a.scale_log2);
        l += ml.y * g;
        o = make_float4(o.x + x.x * g, o.y + x.y * g, o.z + x.z * g, o.w + x.w * g);
      }
      write(row, col, m, l, o);
    }
    __syncthreads();  // the sums are read before the next ones
  }
}

// The join of tiles of M rows (of which a.tile_rows are used) that `ctas` CTAs have left parts of.
template <typename T, int DP, int M, bool TC>
cudaError_t launch_tree_join(const TreeArgs& a, int ctas, cudaStream_t s) {
  // at most one joined tile per run and tile of rows; a thread for 4 columns of a row, up to some 16 blocks per SM
  const long long most = static_cast<long long>(a.max_new) * a.group;  // rows that share a key head
  const long long tiles = static_cast<long long>(a.n_req) * a.cache.heads * ((most + a.tile_rows - 1) / a.tile_rows);
  const bool search = 4 * tiles < ctas;
  const int x = search ? static_cast<int>(tiles) : ctas, rows = static_cast<int>(std::min<long long>(a.tile_rows, most));
  const int elements = TC ? (rows + 7) / 8 * 2 * DP : rows * (DP / 4);
  const int blocks = ctas > 8 * x ? (elements + 31) / 32 : (elements + 255) / 256;  // (many parts: 32 elements each)
  const int y = std::max(1, std::min(blocks, 8 * ctas / x));
  return launch_ex(tree_join_kernel<T, DP, M, TC>, dim3(x, y), dim3(256), 0, s, 1, a, ctas, search);
}

}  // namespace
}  // namespace ivit
