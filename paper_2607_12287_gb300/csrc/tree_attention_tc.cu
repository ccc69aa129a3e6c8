// The form of ivit_tree_attention for many rows per key head (see tree_attention.cu for the operation), on
// the tensor cores.  A tile is up to 128 rows (new row x head of the group) of one request and key head; it
// walks the request's keys in blocks of KB: first the cached tokens, then the new rows, each with a last block
// that may be partly empty.  The blocks of the call are cut into equal runs, two CTAs per SM, as in
// tree_attention.cu; while one CTA's warps take exponentials the other's MMAs run.  (Heads above 128: one CTA,
// for O takes 256 columns of tensor memory and two blocks of K and V take 128 KB.)  KB is 96 for heads up to 96,
// else 64: S, P and O of a block fit in 256 columns of tensor memory and a row of S in registers (heads of 64,
// eight requests of up to 256 rows over up to 4096 tokens, 16 heads: 40 us, 42 at KB = 64, 50 at 128, which spills).
//
// Warps of a CTA:
//   4      TMA: Q tile (a box of heads x new rows, which is the tile's order of rows), then K and V blocks
//          through a ring.  A cached block is fetched page by page (or in boxes of the largest power of two
//          that divides KB, for larger pages), a block of new rows in one box.  64 columns of a head form a
//          slice with 128-byte swizzle, 16 or 32 that are left (heads up to 80, up to 96) one with 32- or 64-byte
//          swizzle (heads of 96, eight requests of up to 256 rows over up to 4096 tokens, 16 heads: 53 us, as 128 60).
//   5      MMA: S = Q K^T of block i + 1 is issued before O += P V of block i; P is read from tensor memory,
//          V is the B operand in MN-major form.
//   0 - 3  softmax, thread = row = tensor-memory lane: S into registers, masked where the block holds keys
//          that the row does not see; P = 2^((S - m) c + SHIFT) rounded to 16 bits into tensor memory, l the
//          sum of the fp32 values.  In blocks that hold new rows, or end, they first clear what the product
//          with V must not meet: rows past the block's keys, and new rows' values that are not finite, which
//          (0 * NaN) would reach rows that do not see them; rows that do see them get them back at the end.
//
// A tile that another run shares leaves its part in groups of 8 rows, 4 columns of each side by side, so that a
// warp's store (lane = row) is whole lines (34.2 us for the eight requests below; row after row 36.3).
//
// P is rounded once: a second 16-bit term would double the MMAs of P V and the stores of P, both on the chain of a block
// that bounds the kernel.  Errors against 64 bits, relative to the output: bf16 0.0023 (0.0017 is the rounding of
// the output alone), fp16 0.00029 (0.00021).
//
// Bound: the cache's bytes for up to about 128 rows, for more the chain of a block (1.3 us at KB = 96, two CTAs
// at a time): two thirds of it are the exponentials of both CTAs.  A quarter of them by a polynomial on the FMA
// pipe was slower (35 -> 38 us: registers).
// Measured: 16 trees of up to 31 drafts over up to 8192 tokens, 32 + 8 heads of 128, 61.6 us (mma.sync 137); eight
// requests of up to 256 rows over up to 2048 tokens, 16 heads of 72, 34 us (73), over up to 8192 tokens 68 us
// (465 TFLOP/s); 16 requests of 16 drafts over up to 4096 tokens, 16 + 2 heads of 256, 33 us (53).
#include <cudaTypedefs.h>

#include <type_traits>

#include "tree_attention.cuh"

namespace ivit {
namespace {

constexpr int AQ = 128;                // rows of a tile (MMA M)
constexpr int THREADS = 192;

template <int DP>
struct Cfg {
  static constexpr int KB = DP <= 96 ? 96 : 64;
  static constexpr int CTAS = DP <= 128 ? 2 : 1;                // of an SM
  static constexpr int FULL = DP / 64, TAIL = DP % 64;          // slices of 64 columns, and columns of a narrow last one
  static constexpr int Q1 = AQ * 128, T1 = KB * 128;            // bytes of a full slice of Q, of a K or V block
  static constexpr int Q_ROW = FULL * 128 + TAIL * 2;
  static constexpr int T_BYTES = KB * Q_ROW, TILE = (T_BYTES + 1023) / 1024 * 1024;
  static constexpr int TM_O = KB, TM_P = KB + DP, TM_COLS = 512 / CTAS;  // S at column 0
  static_assert(TM_P + KB / 2 <= TM_COLS, "tensor memory of one CTA");
  static constexpr int OFF_RING = AQ * Q_ROW;
  static constexpr int FIT = ((CTAS == 2 ? 113 : 227) * 1024 - OFF_RING - 1024 - 512) / TILE, RING = FIT < 8 ? FIT : 8;
  static constexpr int OFF_BAR = OFF_RING + RING * TILE;
  static constexpr int BYTES = OFF_BAR + 256 + 1024;  // with alignment slack
  static_assert(TREE_MAX_REQ * 8 <= OFF_BAR, "the units before each request");
  static_assert(RING >= 4, "K and V of two blocks");
};

template <int KB>
struct Blocks {
  static constexpr int LEAST = 128 / KB;
  static __device__ __forceinline__ int cached(const TreeRequest& r) { return (r.len + KB - 1) / KB; }
  static __device__ __forceinline__ int tiles(const TreeRequest& r) { return cached(r) + (r.n + KB - 1) / KB; }
};

// Maps of one array: 64 columns of a head, and the narrow last slice.
struct Maps {
  CUtensorMap lo, hi;
};
struct AllMaps {
  Maps q, k, v, k_new, v_new;
};

// Instruction descriptor, kind::f16: A and B of type T (both K-major), fp32 D.
template <typename T>
__device__ __forceinline__ uint32_t idesc(int m, int n) {
  const uint32_t d = idesc_bf16_f32(m, n);
  return std::is_same<T, bf16>::value ? d : d & ~((1u << 7) | (1u << 10));
}

// Shared-memory descriptor of a narrow slice whose rows are W columns (and one swizzle span) wide: groups of 8
// rows follow each other.  For a K-major operand the rows are its M or N index, for an MN-major one (V) its
// K index.
template <int W>
__device__ __forceinline__ uint64_t sdesc_rows(uint32_t saddr) {
  constexpr uint32_t group = 8 * W * 2;
  uint64_t d = sdesc_sw128(saddr, group, group) & ~(static_cast<uint64_t>(7) << 61);
  return d | (static_cast<uint64_t>(W == 16 ? 6 : 4) << 61);  // 32-, 64-byte swizzle
}

// 4-D tiled load (see tma_load_2d).
__device__ __forceinline__ void tma_load_4d(uint32_t dst, const CUtensorMap* map, int c0, int c1, int c2, int c3, uint32_t bar,
                                            uint64_t policy) {
  asm volatile(
      "cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes"
      ".L2::cache_hint [%0], [%1, {%2, %3, %4, %5}], [%6], %7;" ::"r"(dst),
      "l"(reinterpret_cast<uint64_t>(map)), "r"(c0), "r"(c1), "r"(c2), "r"(c3), "r"(bar), "l"(policy)
      : "memory");
}

// 32 columns of S (bits) -> 16 packed pairs of P; l gets the fp32 values.
template <typename T>
__device__ __forceinline__ void exp_chunk(const uint32_t* s, float sc, float mo, uint32_t* pk, float2 (&l)[2]) {
  const float2 c2 = make_float2(sc, sc), m2 = make_float2(mo, mo);
#pragma unroll
  for (int u = 0; u < 16; ++u) {
    const float2 t = fma_f32x2(make_float2(__uint_as_float(s[2 * u]), __uint_as_float(s[2 * u + 1])), c2, m2);
    const float2 p = make_float2(ex2(t.x), ex2(t.y));
    l[u & 1] = add_f32x2(l[u & 1], p);
    pk[u] = pack2<T>(p.x, p.y);
  }
}

// Which of the 32 new rows from j0 (a multiple of 32) on new row `node` sees.
__device__ __forceinline__ uint32_t seen32(const TreeArgs& a, const TreeRequest& r, int node, int j0) {
  const int last = a.mask_mode == IVIT_MASK_CAUSAL ? node + 1 : r.n, n = last - j0;
  const uint32_t bits = n >= 32 ? 0xffffffffu : n > 0 ? (1u << n) - 1 : 0u;
  if (a.mask_mode != IVIT_MASK_TREE) return bits;
  const int w = j0 >> 5;
  return w < a.mask_words ? bits & a.mask[static_cast<size_t>(r.row0 + node) * a.mask_words + w] : 0u;
}

template <typename T>
__device__ __forceinline__ bool not_finite(uint32_t half_word) {
  constexpr uint32_t e = std::is_same<T, bf16>::value ? 0x7f80u : 0x7c00u;
  return (half_word & e) == e;
}

// A slice of a V block (rows of WIDTH bytes at `slice`): zeros for rows from `rows` on, and with `clean` for values
// that are not finite; whether there was one.  By 128 threads.
template <typename T, int KB, int WIDTH>
__device__ __forceinline__ bool clear_slice(uint8_t* slice, int rows, bool clean, int tid) {
  bool odd = false;
  for (int e = tid; e < KB * WIDTH / 16; e += 128) {
    uint4* at = reinterpret_cast<uint4*>(slice) + e;  // (a swizzle moves pieces within a row only)
    if (e / (WIDTH / 16) >= rows) {
      *at = make_uint4(0, 0, 0, 0);
    } else if (clean) {
      uint4 x = *at;
      uint32_t* w = reinterpret_cast<uint32_t*>(&x);
      bool here = false;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const bool low = not_finite<T>(w[i]), high = not_finite<T>(w[i] >> 16);
        if (low) w[i] &= 0xffff0000u;
        if (high) w[i] &= 0x0000ffffu;
        here |= low || high;
      }
      if (here) *at = x;
      odd |= here;
    }
  }
  return odd;
}

template <typename T, int DP>
__global__ void __launch_bounds__(THREADS, Cfg<DP>::CTAS)
    tree_attention_tc_kernel(const __grid_constant__ AllMaps maps, const TreeArgs a, int box_shift) {
  using C = Cfg<DP>;
  constexpr int KB = C::KB, RING = C::RING, FULL = C::FULL, TAIL = C::TAIL, PART = tree_part_floats(AQ, DP);
  using B = Blocks<KB>;
  extern __shared__ uint8_t raw[];
  uint8_t* sm = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(raw) + 1023) & ~static_cast<uintptr_t>(1023));
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const uint32_t sb = smem_u32(sm), bar = sb + C::OFF_BAR;
  const uint32_t q_full = bar, q_empty = bar + 8, s_full = bar + 16, s_free = bar + 24, p_ready = bar + 32, o_done = bar + 40,
                 o_free = bar + 48, t_full = bar + 56, t_empty = t_full + 8 * RING;
  uint32_t* tslot = reinterpret_cast<uint32_t*>(sm + C::OFF_BAR + 56 + 16 * RING);
  volatile int* sh_abort = reinterpret_cast<volatile int*>(tslot + 1);
  // Last tile of rows, of the even ones and of the odd ones, that met a value that is not finite.  A warp may be in tile n + 1
  // while another still reads what tile n met; in n + 2 it is not, for the products of n + 1 wait for all four warps.
  volatile int* sh_odd = reinterpret_cast<volatile int*>(tslot + 2);
  if (tid == 0) {
    mbar_init(q_full, 1);
    mbar_init(q_empty, 1);
    mbar_init(s_full, 1);
    mbar_init(s_free, 4);
    mbar_init(p_ready, 4);
    mbar_init(o_done, 1);
    mbar_init(o_free, 4);
    for (int i = 0; i < RING; ++i) {
      mbar_init(t_full + 8 * i, 1);
      mbar_init(t_empty + 8 * i, 1);
    }
    fence_mbar_init();
    for (const Maps* m : {&maps.q, &maps.k, &maps.v, &maps.k_new, &maps.v_new}) {
      tma_prefetch_desc(&m->lo);
      if (TAIL > 0) tma_prefetch_desc(&m->hi);
    }
    *sh_abort = 0;
    sh_odd[0] = sh_odd[1] = 0;
  }
  if (warp == 5) {
    tmem_alloc(smem_u32(tslot), C::TM_COLS);
    tmem_relinquish();
  }
  pdl_wait();
  pdl_launch_dependents();
  if (blockIdx.x == 0 && tid == 0) *a.err = 0;  // (a wait that expires says so a second later)
  TreeRun<B> run{};
  const bool some = run.template find<THREADS>(a, reinterpret_cast<unsigned long long*>(sm));
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tslot;

  // Every wait is bounded; after one has expired no role waits again and all leave.
  auto wait = [&](uint32_t b, uint32_t parity) {
    if (*sh_abort) return false;
    if (mbar_wait(b, parity)) return true;
    atomicExch(a.err, kErrWaitTmaFull);
    *sh_abort = 1;
    return false;
  };
  // The run as segments: consecutive key blocks [first, first + n) of one tile of rows.
  const unsigned long long units = some ? run.hi - run.lo : 0;
  unsigned long long u = 0;
  auto segment = [&](const TreePlace<B>& p) {
    return static_cast<int>(min(static_cast<unsigned long long>(p.nkt - p.kt), units - u));
  };

  if (warp == 4) {
    fence_proxy_async_smem();  // (the ring was scratch)
    const uint64_t policy = l2_policy_evict_first();
    const uint32_t q_bytes = a.tile_rows * C::Q_ROW;
    const int boxes = KB >> box_shift, page_mask = (1 << a.cache.page_shift) - 1;
    TreePlace<B> p = run.at;
    uint32_t t = 0;  // K / V blocks so far
    for (uint32_t n = 0; u < units; ++n) {
      const int blocks = segment(p), cached = B::cached(p.r);
      if (!__all_sync(0xffffffffu, wait(q_empty, (n & 1) ^ 1))) break;
      if (elect_one()) {
        const int head = p.head * a.group, row = p.r.row0 + p.rt * (a.tile_rows / a.group);
        mbar_arrive_expect_tx(q_full, q_bytes);
#pragma unroll
        for (int c = 0; c < FULL; ++c) tma_load_3d(sb + c * C::Q1, &maps.q.lo, 64 * c, head, row, q_full, policy);
        if (TAIL > 0) tma_load_3d(sb + FULL * C::Q1, &maps.q.hi, 64 * FULL, head, row, q_full, policy);
      }
      __syncwarp();
      const int* table = a.table + static_cast<size_t>(p.req) * a.max_pages;
      auto look_up = [&](int kb) {  // the page of the lane's box of a cached block (past the table: none)
        const int key = kb * KB + (lane << box_shift);
        return lane < boxes && key < p.r.len ? table[key >> a.cache.page_shift] : -1;
      };
      int ids = p.kt < cached ? look_up(p.kt) : -1;
      bool ok = true;
      for (int i = 0; i < blocks && ok; ++i) {
        const int kb = p.kt + i;
        const int ids_next = kb + 1 < cached && i + 1 < blocks ? look_up(kb + 1) : -1;
        for (int kv = 0; kv < 2 && ok; ++kv, ++t) {
          const uint32_t slot = t % RING;
          ok = __all_sync(0xffffffffu, wait(t_empty + 8 * slot, ((t / RING) & 1) ^ 1));
          if (!ok) break;
          const uint32_t dst = sb + C::OFF_RING + slot * C::TILE, full = t_full + 8 * slot;
          if (elect_one()) mbar_arrive_expect_tx(full, C::T_BYTES);
          __syncwarp();
          if (kb < cached) {
            const Maps& m = kv ? maps.v : maps.k;
            for (int b = 0; b < boxes; ++b) {
              const int id = __shfl_sync(0xffffffffu, ids, b);
              if (elect_one()) {
                const int token = (kb * KB + (b << box_shift)) & page_mask;
#pragma unroll
                for (int c = 0; c < FULL; ++c)
                  tma_load_4d(dst + c * C::T1 + (b << box_shift) * 128, &m.lo, 64 * c, p.head, token, id, full, policy);
                if (TAIL > 0)
                  tma_load_4d(dst + FULL * C::T1 + (b << box_shift) * TAIL * 2, &m.hi, 64 * FULL, p.head, token, id, full, policy);
              }
              __syncwarp();
            }
          } else if (elect_one()) {
            const Maps& m = kv ? maps.v_new : maps.k_new;
            const int row = p.r.row0 + (kb - cached) * KB;
#pragma unroll
            for (int c = 0; c < FULL; ++c) tma_load_3d(dst + c * C::T1, &m.lo, 64 * c, p.head, row, full, policy);
            if (TAIL > 0) tma_load_3d(dst + FULL * C::T1, &m.hi, 64 * FULL, p.head, row, full, policy);
          }
          __syncwarp();
        }
        ids = ids_next;
      }
      if (!ok) break;
      u += blocks;
      p.next_rows(a);
    }
  } else if (warp == 5) {
    TreePlace<B> p = run.at;
    uint32_t j0 = 0;  // key blocks of the earlier segments
    bool ok = true;
    for (uint32_t n = 0; ok && u < units; ++n) {
      const int blocks = segment(p);
      ok = __all_sync(0xffffffffu, wait(q_full, n & 1));
      for (int i = 0; i <= blocks && ok; ++i) {
        if (i < blocks) {  // S of block i
          const uint32_t j = j0 + i, t = 2 * j, slot = t % RING;
          ok = __all_sync(0xffffffffu, wait(t_full + 8 * slot, (t / RING) & 1) && wait(s_free, (j & 1) ^ 1));
          if (!ok) break;
          tc_fence_after();
          if (elect_one()) {
            const uint32_t kt = sb + C::OFF_RING + slot * C::TILE, id = idesc<T>(AQ, KB);
#pragma unroll
            for (int c = 0; c < DP / 16; ++c)
              umma_bf16(tmem,
                        c < 4 * FULL ? sdesc_kmajor_sw128(sb + c / 4 * C::Q1 + c % 4 * 32)
                                     : sdesc_rows<TAIL>(sb + FULL * C::Q1 + (c - 4 * FULL) * 32),
                        c < 4 * FULL ? sdesc_kmajor_sw128(kt + c / 4 * C::T1 + c % 4 * 32)
                                     : sdesc_rows<TAIL>(kt + FULL * C::T1 + (c - 4 * FULL) * 32),
                        id, c > 0);
            umma_commit(t_empty + 8 * slot);
            umma_commit(s_full);
            if (i == blocks - 1) umma_commit(q_empty);
          }
          __syncwarp();
        }
        if (i > 0) {  // O += P V of block i - 1
          const uint32_t j = j0 + i - 1, t = 2 * j + 1, slot = t % RING;
          ok = __all_sync(0xffffffffu, wait(t_full + 8 * slot, (t / RING) & 1) && wait(p_ready, j & 1) &&
                                           (i > 1 || wait(o_free, (n & 1) ^ 1)));
          if (!ok) break;
          tc_fence_after();
          if (elect_one()) {
            const uint32_t vt = sb + C::OFF_RING + slot * C::TILE;
            const uint32_t id0 = idesc<T>(AQ, 64) | (1u << 16), id1 = idesc<T>(AQ, TAIL > 0 ? TAIL : 16) | (1u << 16);  // (V: MN-major)
#pragma unroll
            for (int c = 0; c < KB / 16; ++c) {
              const uint32_t acc = (i > 1 || c > 0) ? 1u : 0u;
#pragma unroll
              for (int f = 0; f < FULL; ++f)
                umma_bf16_ts(tmem + C::TM_O + 64 * f, tmem + C::TM_P + c * 8, sdesc_sw128(vt + f * C::T1 + c * 2048, 1024, 1024),
                             id0, acc);
              if (TAIL > 0)
                umma_bf16_ts(tmem + C::TM_O + 64 * FULL, tmem + C::TM_P + c * 8, sdesc_rows<TAIL>(vt + FULL * C::T1 + c * 32 * TAIL),
                             id1, acc);
            }
            umma_commit(t_empty + 8 * slot);
            umma_commit(o_done);
          }
          __syncwarp();
        }
      }
      j0 += blocks;
      u += blocks;
      p.next_rows(a);
    }
  } else {
    const uint32_t trow = tmem + (static_cast<uint32_t>(warp * 32) << 16);
    const int row = warp * 32 + lane;
    const float sc = a.scale_log2;
    TreePlace<B> p = run.at;
    uint32_t j = 0;  // key blocks so far
    bool ok = true;
    auto arrive = [&](uint32_t b) {
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(b);
    };
    for (int n = 1; ok && u < units; ++n) {
      const int blocks = segment(p), cached = B::cached(p.r);
      const int rows = min(a.tile_rows, p.r.n * a.group - p.rt * a.tile_rows);
      const bool wrow = warp * 32 < rows;  // warp-uniform: a warp of padding rows only keeps step
      const bool valid = row < rows;
      const int x = p.rt * a.tile_rows + row, node = valid ? x / a.group : 0;
      float m_ref = -INFINITY;
      float2 l[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
      for (int i = 0; i < blocks; ++i, ++j) {
        const int kb = p.kt + i, j0 = (kb - cached) * KB;  // j0: first new row of a block of them
        const int keys = kb < cached ? p.r.len - kb * KB : p.r.n - j0;
        if (kb >= cached || keys < KB) {
          const uint32_t t = 2 * j + 1, slot = t % RING;
          if (!(ok = __all_sync(0xffffffffu, wait(t_full + 8 * slot, (t / RING) & 1)))) break;
          uint8_t* v = sm + C::OFF_RING + slot * C::TILE;
          bool odd = false;
#pragma unroll
          for (int c = 0; c < FULL; ++c) odd |= clear_slice<T, KB, 128>(v + c * C::T1, keys, kb >= cached, tid);
          if (TAIL > 0) odd |= clear_slice<T, KB, (TAIL > 0 ? TAIL * 2 : 16)>(v + FULL * C::T1, keys, kb >= cached, tid);
          if (odd) sh_odd[n & 1] = n;
          fence_proxy_async_smem();
        }
        if (!(ok = __all_sync(0xffffffffu, wait(s_full, j & 1)))) break;
        tc_fence_after();
        if (!wrow) {
          arrive(s_free);
          if (!(ok = __all_sync(0xffffffffu, j == 0 || wait(o_done, (j & 1) ^ 1)))) break;
          arrive(p_ready);
          continue;
        }
        uint32_t r[KB];
#pragma unroll
        for (int c = 0; c < KB; c += 32) tmem_ld32_async(trow + c, *reinterpret_cast<uint32_t(*)[32]>(r + c));
#pragma unroll
        for (int c = 0; c < KB; c += 32) tmem_ld_wait_regs(*reinterpret_cast<uint32_t(*)[32]>(r + c));
        arrive(s_free);
        if (kb >= cached) {
#pragma unroll
          for (int c = 0; c < KB; c += 32) {
            const uint32_t bits = valid ? seen32(a, p.r, node, j0 + c) : 0u;
#pragma unroll
            for (int e = 0; e < 32; ++e)
              if (!(bits >> e & 1)) r[c + e] = 0xff800000u;  // -inf: P = 0
          }
        } else if (keys < KB) {
#pragma unroll
          for (int c = 0; c < KB; ++c)
            if (c >= keys) r[c] = 0xff800000u;
        }
        float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
        for (int c = 0; c < KB; ++c) mx[c & 3] = fmaxf(mx[c & 3], __uint_as_float(r[c]));
        const float m_blk = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3]));
        float alpha = 1.f;
        const bool grow = (m_blk - m_ref) * sc > TREE_GROWTH;
        if (grow) {
          alpha = ex2((m_ref - m_blk) * sc);
          m_ref = m_blk;
        }
        const float mo = TREE_SHIFT - (m_ref == -INFINITY ? 0.f : m_ref * sc);  // (nothing seen so far: P = 0)
        const bool rescale = i > 0 && __any_sync(0xffffffffu, grow);
        if (rescale) {
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            l[e].x *= alpha;
            l[e].y *= alpha;
          }
        }
        uint32_t pk[KB / 2];
#pragma unroll
        for (int c = 0; c < KB; c += 32) exp_chunk<T>(r + c, sc, mo, pk + c / 2, l);
        // P and O are free once the previous block's P V has run
        if (!(ok = __all_sync(0xffffffffu, j == 0 || wait(o_done, (j & 1) ^ 1)))) break;
        tc_fence_after();
        if (rescale) {
#pragma unroll
          for (int d = 0; d < DP; d += 16) {
            uint32_t o[16];
            tmem_ld16_async(trow + C::TM_O + d, o);
            tmem_ld_wait();
            tmem_regs_after_wait16(o);
#pragma unroll
            for (int e = 0; e < 16; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * alpha);
            tmem_st16(trow + C::TM_O + d, o);
          }
        }
#pragma unroll
        for (int c = 0; c < KB / 2; c += 16) tmem_st16(trow + C::TM_P + c, pk + c);
        tmem_st_wait();
        arrive(p_ready);
      }
      if (!ok || !(ok = __all_sync(0xffffffffu, wait(o_done, (j & 1) ^ 1)))) break;
      tc_fence_after();
      const bool whole = blocks == p.nkt;
      if (wrow) {
        const float sum = (l[0].x + l[0].y) + (l[1].x + l[1].y), inv = sum == 0.f ? 0.f : 1.f / sum;
        const bool odd = sh_odd[n & 1] == n;
        const int h = p.head * a.group + x - node * a.group;
        const long long orow = p.r.row0 + node;
        T* dst = static_cast<T*>(a.out) + orow * a.out_stride + static_cast<long long>(h) * a.cache.dim;
        // a part: the run's first, or the one it ends with
        float* part = a.parts + static_cast<size_t>(2 * blockIdx.x + (u > 0 ? 1 : 0)) * PART;
        // new rows of the segment
        const int n0 = max(p.kt - cached, 0) * KB, n1 = min((p.kt + blocks - cached) * KB, p.r.n);
#pragma unroll
        for (int d = 0; d < DP; d += 16) {
          uint32_t o[16];
          tmem_ld16_async(trow + C::TM_O + d, o);
          tmem_ld_wait();
          tmem_regs_after_wait16(o);
          if (odd && valid) {  // the values that were cleared, for the rows that see them
            for (int k = n0; k < n1; ++k) {
              if (!(seen32(a, p.r, node, k & ~31) >> (k & 31) & 1)) continue;
              const T* v = static_cast<const T*>(a.v_new) + (p.r.row0 + k) * a.v_new_stride + p.head * a.cache.dim + d;
#pragma unroll
              for (int e = 0; e < 16; e += 2)
                if (d + e < a.cache.dim) {
                  const uint32_t w = *reinterpret_cast<const uint32_t*>(v + e);
                  const float2 y = unpack2<T>(w);
                  if (not_finite<T>(w)) o[e] = __float_as_uint(__uint_as_float(o[e]) + y.x);
                  if (not_finite<T>(w >> 16)) o[e + 1] = __float_as_uint(__uint_as_float(o[e + 1]) + y.y);
                }
            }
          }
          if (!valid) continue;
          if (whole) {
#pragma unroll
            for (int h8 = 0; h8 < 16; h8 += 8) {
              uint4 y;
              uint32_t* w = reinterpret_cast<uint32_t*>(&y);
#pragma unroll
              for (int e = 0; e < 4; ++e)
                w[e] = pack2<T>(__uint_as_float(o[h8 + 2 * e]) * inv, __uint_as_float(o[h8 + 2 * e + 1]) * inv);
              if (d + h8 < a.cache.dim) *reinterpret_cast<uint4*>(dst + d + h8) = y;
            }
          } else {
#pragma unroll
            for (int e = 0; e < 16; e += 4)  // (a warp's stores are whole lines)
              *reinterpret_cast<uint4*>(part + (row >> 3) * (8 * DP) + 8 * (d + e) + 4 * (row & 7)) =
                  make_uint4(o[e], o[e + 1], o[e + 2], o[e + 3]);
          }
        }
        if (valid && whole && a.lse) a.lse[orow * a.heads + h] = (m_ref * sc + (log2f(sum) - TREE_SHIFT)) * 0.6931471805599453f;
        if (valid && !whole) *reinterpret_cast<float2*>(part + AQ * DP + 2 * row) = make_float2(m_ref, sum);
      }
      if (!whole && p.kt == 0 && tid == 0) run.note_join(a, p, run.lo + u);
      arrive(o_free);
      u += blocks;
      p.next_rows(a);
    }
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp == 5) tmem_dealloc(tmem, C::TM_COLS);
}

PFN_cuTensorMapEncodeTiled_v12000 encoder() {
  static PFN_cuTensorMapEncodeTiled_v12000 fn = [] {
    void* p = nullptr;
    cudaDriverEntryPointQueryResult q;
    const cudaError_t e = cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &q);
    return e == cudaSuccess && q == cudaDriverEntryPointSuccess ? reinterpret_cast<PFN_cuTensorMapEncodeTiled_v12000>(p) : nullptr;
  }();
  return fn;
}

// Maps of an array of `rank` dimensions, the first a head's values; box: of the others.
bool make_maps(Maps* m, int dtype, int tail, const void* base, int rank, const cuuint64_t* dims, const cuuint64_t* strides,
               const cuuint32_t* box) {
  const auto enc = encoder();
  if (!enc) return false;
  const auto make = [&](CUtensorMap* map, cuuint32_t cols) {
    const cuuint32_t b[4] = {cols, box[0], box[1], rank > 3 ? box[2] : 1}, one[4] = {1, 1, 1, 1};
    const auto swizzle = cols == 64   ? CU_TENSOR_MAP_SWIZZLE_128B
                         : cols == 32 ? CU_TENSOR_MAP_SWIZZLE_64B
                                      : CU_TENSOR_MAP_SWIZZLE_32B;
    return enc(map, dtype == IVIT_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, rank,
               const_cast<void*>(base), dims, strides, b, one, CU_TENSOR_MAP_INTERLEAVE_NONE, swizzle,
               CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
  };
  if (!make(&m->lo, 64)) return false;
  m->hi = m->lo;
  return tail == 0 || make(&m->hi, tail);
}

template <typename T, int DP>
cudaError_t launch(const TreeArgs& a, int dtype, int ctas, cudaStream_t s) {
  using C = Cfg<DP>;
  cudaError_t e = allow_smem<tree_attention_tc_kernel<T, DP>>(C::BYTES);
  if (e != cudaSuccess) return e;
  AllMaps m;
  const cuuint64_t dim = a.cache.dim, kv = a.cache.heads, rows = a.n_rows;
  const int page = 1 << a.cache.page_shift, most = C::KB & -C::KB, box = page < most ? page : most;
  const auto fresh = [&](Maps* map, const void* base, cuuint64_t heads, long long stride, cuuint32_t box_heads, cuuint32_t box_rows) {
    const cuuint64_t dims[3] = {dim, heads, rows}, strides[2] = {dim * 2, static_cast<cuuint64_t>(stride) * 2};
    const cuuint32_t b[2] = {box_heads, box_rows};
    return make_maps(map, dtype, C::TAIL, base, 3, dims, strides, b);
  };
  const auto pages = [&](Maps* map, const void* base) {
    const cuuint64_t dims[4] = {dim, kv, static_cast<cuuint64_t>(page), static_cast<cuuint64_t>(a.cache.n_pages)};
    const cuuint64_t strides[3] = {static_cast<cuuint64_t>(a.cache.head_stride) * 2, static_cast<cuuint64_t>(a.cache.token_stride) * 2,
                                   static_cast<cuuint64_t>(a.cache.page_stride) * 2};
    const cuuint32_t b[3] = {1, static_cast<cuuint32_t>(box), 1};
    return make_maps(map, dtype, C::TAIL, base, 4, dims, strides, b);
  };
  if (!fresh(&m.q, a.q, a.heads, a.q_stride, a.group, a.tile_rows / a.group) || !pages(&m.k, a.k_cache) || !pages(&m.v, a.v_cache) ||
      !fresh(&m.k_new, a.k_new, kv, a.k_new_stride, 1, C::KB) || !fresh(&m.v_new, a.v_new, kv, a.v_new_stride, 1, C::KB))
    return cudaErrorInvalidValue;
  int shift = 0;
  while (1 << shift < box) ++shift;
  return launch_ex(tree_attention_tc_kernel<T, DP>, dim3(ctas), dim3(THREADS), C::BYTES, s, 1, m, a, shift);
}

}  // namespace

cudaError_t launch_tree_attention_tc(const TreeArgs& a, int dtype, int dp, int ctas, cudaStream_t s) {
  const auto width = [&](auto type) {
    using T = decltype(type);
    return dp == 64    ? launch<T, 64>(a, dtype, ctas, s)
           : dp == 80  ? launch<T, 80>(a, dtype, ctas, s)
           : dp == 96  ? launch<T, 96>(a, dtype, ctas, s)
           : dp == 128 ? launch<T, 128>(a, dtype, ctas, s)
                       : launch<T, 256>(a, dtype, ctas, s);
  };
  return dtype == IVIT_BF16 ? width(bf16{}) : width(half{});
}

}  // namespace ivit
