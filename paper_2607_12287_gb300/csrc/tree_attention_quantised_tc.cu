// The form of ivit_tree_attention_quantised for many rows per key head (see tree_attention_quantised.cuh for the operation and what
// is done with the blocks' scales), on the tensor cores, as tree_attention_tc.cu is for caches of 16 bits: tiles of up to 128
// rows, key blocks of 64, first the cached tokens, then the new rows; S, P and O in tensor memory; equal runs of blocks.
//
// Warps of a CTA:
//   0 - 3  softmax, thread = row = tensor-memory lane, as there; scores of cached keys are scaled and shifted by their blocks' scales.
//   4      MMA: S = Q K^T of block i + 1 is issued before O += P V of block i.
//   5 - 7  K and V blocks through the ring: cached tokens' codes come by asynchronous copies, some blocks ahead, each thread's to a place of
//          its own, become 16-bit values of the rows' type (exact) and go where TMA would have put them, and their scales beside
//          them; blocks of new rows come by TMA, as does the tile of Q.
//
// Where the time goes: into the chain of a block, 3.3 us for two CTAs an SM (heads of 128), of which 2.2 are the handshakes of S, P and O
// that tree_attention_tc.cu has too; it is no limit of the machine, and the 16-bit cache's kernel, which converts nothing, takes 62 us for
// the trees below and 34 for the views; conversions wait for a place in the ring, which has three at heads of 128 beside the 32 KB of Q.
// Without conversions and copies 79 us instead of 110 for 16 trees of up to 31 drafts over up to 8192 tokens (32 + 8 heads of 128, fp16; bf16
// 124), without most of the softmax's work 101.  Eight requests of up to 256 rows over up to 2048 tokens, 16 heads of 72, 58 us.
#include <cudaTypedefs.h>

#include <type_traits>

#include "tree_attention_quantised.cuh"

namespace ivit {
namespace {

constexpr int AQ = 128;                // rows of a tile (MMA M)
constexpr int FILL = 96;               // threads of the warps that fill the ring
constexpr int TC_THREADS = 160 + FILL;
constexpr int KB = 64;                 // keys of a block
constexpr int SCALES = 4;              // blocks whose scales are kept: V blocks in the ring, and one

template <int DP>
struct TcCfg {
  static constexpr int CTAS = DP <= 128 ? 2 : 1;                // of an SM
  static constexpr int FULL = DP / 64, TAIL = DP % 64;          // slices of 64 columns, and columns of a narrow last one
  static constexpr int Q1 = AQ * 128, T1 = KB * 128;            // bytes of a full slice of Q, of a K or V block
  static constexpr int Q_ROW = FULL * 128 + TAIL * 2;
  static constexpr int T_BYTES = KB * Q_ROW, TILE = (T_BYTES + 1023) / 1024 * 1024;
  static constexpr int TM_O = KB, TM_P = KB + DP, TM_COLS = 512 / CTAS;  // S at column 0
  static_assert(TM_P + KB / 2 <= TM_COLS, "tensor memory of one CTA");
  static constexpr int PIECES = DP / 16, PASSES = (KB * PIECES + FILL - 1) / FILL;  // 16 codes each, of a row and of a thread
  static constexpr int RAW = PASSES * FILL * 16;                // bytes of codes of a block
  static constexpr int RING = DP <= 64 ? 6 : DP <= 96 ? 4 : 3, AHEAD = DP <= 96 ? 4 : 3;
  static constexpr int OFF_RING = AQ * Q_ROW;
  static constexpr int OFF_RAW = OFF_RING + RING * TILE;        // [block % AHEAD][pass][thread]
  static constexpr int OFF_RAW_SCALES = OFF_RAW + AHEAD * RAW;  // [block % AHEAD][of keys, of values][KB]
  static constexpr int OFF_SCALES = OFF_RAW_SCALES + AHEAD * 2 * KB * 4;  // [block % SCALES][of keys, log2 and inverse of values][KB]
  static constexpr int OFF_BAR = OFF_SCALES + SCALES * 3 * KB * 4;
  static constexpr int BYTES = OFF_BAR + 256 + 1024;  // with alignment slack
  static_assert(TREE_MAX_REQ * 8 <= OFF_RAW, "the units before each request");
  static_assert(CTAS * (BYTES + 1024 + 64) <= 228 * 1024, "shared memory of an SM");
  static_assert(RING >= 3 && (RING + 1) / 2 + 1 <= SCALES, "V blocks in the ring, and the one that is multiplied");
};

struct TcBlocks {
  static constexpr int LEAST = 128 / KB;
  static __device__ __forceinline__ int cached(const TreeRequest& r) { return (r.len + KB - 1) / KB; }
  static __device__ __forceinline__ int tiles(const TreeRequest& r) { return cached(r) + (r.n + KB - 1) / KB; }
};

// Maps of one array: 64 columns of a head, and the narrow last slice.
struct Maps {
  CUtensorMap lo, hi;
};
struct AllMaps {
  Maps q, k_new, v_new;
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

// 32 columns of scores y (log2 units) -> 16 packed pairs of P = 2^(y + mo); l gets the fp32 values, times iv (32 floats in shared
// memory) if there is one.
template <typename T>
__device__ __forceinline__ void exp_chunk(const uint32_t* y, float mo, const float* iv, uint32_t* pk, float2 (&l)[2]) {
  const float2 m2 = make_float2(mo, mo);
#pragma unroll
  for (int u = 0; u < 16; u += 2) {
    const float4 w = iv ? *reinterpret_cast<const float4*>(iv + 2 * u) : make_float4(1.f, 1.f, 1.f, 1.f);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const float2 t = add_f32x2(make_float2(__uint_as_float(y[2 * (u + i)]), __uint_as_float(y[2 * (u + i) + 1])), m2);
      const float2 p = make_float2(ex2(t.x), ex2(t.y));
      l[i] = fma_f32x2(p, i ? make_float2(w.z, w.w) : make_float2(w.x, w.y), l[i]);
      pk[u + i] = pack2<T>(p.x, p.y);
    }
  }
}

template <typename T>
__device__ __forceinline__ bool not_finite(uint32_t half_word) {
  constexpr uint32_t e = std::is_same<T, bf16>::value ? 0x7f80u : 0x7c00u;
  return (half_word & e) == e;
}

// A slice of a V block (rows of WIDTH bytes at `slice`): zeros for rows from `rows` on, and with `clean` for values
// that are not finite; whether there was one.  By 128 threads.
template <typename T, int WIDTH>
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

// 16 codes as 16-bit values of type T (exact).
template <typename T>
__device__ __forceinline__ void values16(const uint4& codes, uint4& lo, uint4& hi) {
  const uint32_t w[4] = {codes.x, codes.y, codes.z, codes.w};
  uint32_t y[8];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    codes_to_half4(w[i], y[2 * i], y[2 * i + 1]);
    if (std::is_same<T, bf16>::value) {
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const float2 f = unpack2<half>(y[2 * i + e]);
        y[2 * i + e] = pack2<T>(f.x, f.y);
      }
    }
  }
  lo = make_uint4(y[0], y[1], y[2], y[3]);
  hi = make_uint4(y[4], y[5], y[6], y[7]);
}

// Byte of 16-byte chunk c of row `row` in a K or V block, as TMA's swizzles place it: 8 chunks a row in a full slice, 2 or 4 in a
// narrow last one.
template <int DP>
__device__ __forceinline__ int chunk_at(int row, int c) {
  using C = TcCfg<DP>;
  if (C::TAIL == 0 || c < 8 * C::FULL) return (c >> 3) * C::T1 + row * 128 + (((c & 7) ^ (row & 7)) << 4);
  const int d = c - 8 * C::FULL;
  return C::FULL * C::T1 + row * (C::TAIL * 2) + ((C::TAIL == 16 ? d ^ (row >> 2 & 1) : d ^ (row >> 1 & 3)) << 4);
}

template <typename T, int DP>
__global__ void __launch_bounds__(TC_THREADS, TcCfg<DP>::CTAS)
    tree_attention_quantised_tc_kernel(const __grid_constant__ AllMaps maps, const QuantisedArgs a) {
  using C = TcCfg<DP>;
  constexpr int RING = C::RING, FULL = C::FULL, TAIL = C::TAIL, PART = tree_part_floats(AQ, DP);
  using B = TcBlocks;
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
      mbar_init(t_full + 8 * i, FILL / 32);  // (a warp that fills has done its part)
      mbar_init(t_empty + 8 * i, 1);
    }
    fence_mbar_init();
    for (const Maps* m : {&maps.q, &maps.k_new, &maps.v_new}) {
      tma_prefetch_desc(&m->lo);
      if (TAIL > 0) tma_prefetch_desc(&m->hi);
    }
    *sh_abort = 0;
    sh_odd[0] = sh_odd[1] = 0;
  }
  if (warp == 4) {
    tmem_alloc(smem_u32(tslot), C::TM_COLS);
    tmem_relinquish();
  }
  pdl_wait();
  pdl_launch_dependents();
  if (blockIdx.x == 0 && tid == 0) *a.err = 0;  // (a wait that expires says so a second later)
  TreeRun<B> run{};
  const bool some = run.template find<TC_THREADS>(a, reinterpret_cast<unsigned long long*>(sm));
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

  if (warp >= 5) {
    fence_proxy_async_smem();  // (the ring was scratch)
    const uint64_t policy = l2_policy_evict_first();
    const uint32_t q_bytes = a.tile_rows * C::Q_ROW;
    const int tid2 = tid - 160, page_mask = (1 << a.cache.page_shift) - 1, dim = a.cache.dim;
    // The place and the pages of the next cached block to be copied; its codes and scales.
    TreePlace<B> next = run.at;
    unsigned long long next_u = 0;
    int next_kb = next.kt, next_end = 0, ids[C::PASSES], scale_id = -1;
    const long long head = next.head * a.cache.head_stride;
    const auto bounds = [&] {  // the next segment that has cached blocks, from `next` on
      while (next_u < units) {
        const int blocks = static_cast<int>(min(static_cast<unsigned long long>(next.nkt - next.kt), units - next_u));
        next_end = min(next.kt + blocks, B::cached(next.r));
        next_kb = next.kt;
        if (next_kb < next_end) return;
        next_u += blocks;
        next.next_rows(a);
      }
    };
    const auto look_up = [&] {
      if (next_u >= units) return;
      const int* table = a.table + static_cast<size_t>(next.req) * a.max_pages;
      const auto page = [&](int row) {
        const int key = next_kb * KB + row, id = row < KB && key < next.r.len ? table[key >> a.cache.page_shift] : -1;
        return static_cast<unsigned>(id) < static_cast<unsigned>(a.cache.n_pages) ? id : -1;
      };
#pragma unroll
      for (int x = 0; x < C::PASSES; ++x) ids[x] = page((tid2 + x * FILL) / C::PIECES);
      scale_id = page(tid2);
    };
    // To where in a K or V block the thread's pieces go.
    int to_at[C::PASSES];
#pragma unroll
    for (int x = 0; x < C::PASSES; ++x) {
      const int e = tid2 + x * FILL, row = e / C::PIECES, c = e - row * C::PIECES;
      to_at[x] = row < KB ? chunk_at<DP>(row, 2 * c) : -1;
    }
    uint32_t copied = 0;  // K and V blocks, in turn
    const auto copy = [&] {
      if (next_u < units) {
        const bool values = copied & 1;
        const uint32_t raw = sb + C::OFF_RAW + copied % C::AHEAD * C::RAW + tid2 * 16;
        const uint8_t* const cache = static_cast<const uint8_t*>(values ? a.v_cache : a.k_cache) + head;
        const uint8_t* const from = cache + (next_kb * KB & page_mask) * a.cache.token_stride;  // (a page above 64 tokens has whole blocks)
#pragma unroll
        for (int x = 0; x < C::PASSES; ++x) {
          const int e = tid2 + x * FILL, row = e / C::PIECES, c = e - row * C::PIECES;  // (places kept for all pieces spilled: 112 instead of 109 us)
          const bool ok = ids[x] >= 0 && 16 * c < dim;
          const uint8_t* src = ok ? from + (row & page_mask) * a.cache.token_stride + 16 * c + ids[x] * a.cache.page_stride : cache;
          const uint32_t to = raw + x * FILL * 16;
          if (a.wide) {
            copy16(to, src, ok);
          } else {
            copy8(to, src, ok);
            const bool second = ok && 16 * c + 8 < dim;
            copy8(to + 8, second ? src + 8 : src, second);
          }
        }
        if (values) {
          if (tid2 < KB) {
            const bool ok = scale_id >= 0;
            const long long at =
                ok ? static_cast<long long>(((scale_id << a.cache.page_shift) + ((next_kb * KB + tid2) & page_mask)) >> a.block_shift) * a.cache.heads + next.head : 0;
            const uint32_t to = sb + C::OFF_RAW_SCALES + (copied % C::AHEAD * 2 * KB + tid2) * 4;
            copy4(to, a.k_scale + at, ok);
            copy4(to + KB * 4, a.v_scale + at, ok);
          }
          if (++next_kb == next_end) {
            next_u += static_cast<int>(min(static_cast<unsigned long long>(next.nkt - next.kt), units - next_u));
            next.next_rows(a);
            bounds();
          }
          look_up();
        }
      }
      ++copied;
      copies_commit();
    };
    bounds();
    look_up();
#pragma unroll 1
    for (int x = 0; x < C::AHEAD; ++x) copy();

    TreePlace<B> p = run.at;
    uint32_t t = 0, converted = 0;  // K / V blocks so far, and cached ones
    for (uint32_t n = 0; u < units; ++n) {
      const int blocks = segment(p), cached = B::cached(p.r);
      if (!__all_sync(0xffffffffu, wait(q_empty, (n & 1) ^ 1))) break;
      if (warp == 5 && elect_one()) {
        const int head = p.head * a.group, row = p.r.row0 + p.rt * (a.tile_rows / a.group);
        mbar_arrive_expect_tx(q_full, q_bytes);
#pragma unroll
        for (int c = 0; c < FULL; ++c) tma_load_3d(sb + c * C::Q1, &maps.q.lo, 64 * c, head, row, q_full, policy);
        if (TAIL > 0) tma_load_3d(sb + FULL * C::Q1, &maps.q.hi, 64 * FULL, head, row, q_full, policy);
      }
      __syncwarp();
      bool ok = true;
      for (int i = 0; i < blocks && ok; ++i) {
        const int kb = p.kt + i;
        for (int kv = 0; kv < 2 && ok; ++kv, ++t) {
          const uint32_t slot = t % RING;
          ok = __all_sync(0xffffffffu, wait(t_empty + 8 * slot, ((t / RING) & 1) ^ 1));
          if (!ok) break;
          const uint32_t dst = sb + C::OFF_RING + slot * C::TILE, full = t_full + 8 * slot;
          if (kb < cached) {
            copies_wait<C::AHEAD - 1>();  // (this thread's, of this block)
            const int stage = converted++ % C::AHEAD;
            if (kv == 1 && tid2 < KB) {  // (beside the values: their slot stays full until the block's probabilities have been multiplied)
              const float* raw = reinterpret_cast<const float*>(sm + C::OFF_RAW_SCALES) + stage * 2 * KB + tid2;
              float* scales = reinterpret_cast<float*>(sm + C::OFF_SCALES) + (t / 2 % SCALES) * 3 * KB + tid2;
              scales[0] = key_scale(raw[0]) * a.score_log2;
              value_scale(raw[KB], scales[KB], scales[2 * KB]);
            }
            uint8_t* tile = sm + C::OFF_RING + slot * C::TILE;
            const uint8_t* raw = sm + C::OFF_RAW + stage * C::RAW + tid2 * 16;
#pragma unroll
            for (int x = 0; x < C::PASSES; ++x) {
              if (C::PASSES * FILL > KB * C::PIECES && x == C::PASSES - 1 && to_at[x] < 0) break;
              uint4 lo, hi;
              values16<T>(*reinterpret_cast<const uint4*>(raw + x * FILL * 16), lo, hi);
              *reinterpret_cast<uint4*>(tile + to_at[x]) = lo;
              *reinterpret_cast<uint4*>(tile + (to_at[x] ^ 16)) = hi;  // (the swizzles leave a pair of chunks beside each other)
            }
            fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive(full);
            copy();
          } else if (elect_one()) {
            if (warp == 5) {
              mbar_arrive_expect_tx(full, C::T_BYTES);
              const Maps& m = kv ? maps.v_new : maps.k_new;
              const int row = p.r.row0 + (kb - cached) * KB;
#pragma unroll
              for (int c = 0; c < FULL; ++c) tma_load_3d(dst + c * C::T1, &m.lo, 64 * c, p.head, row, full, policy);
              if (TAIL > 0) tma_load_3d(dst + FULL * C::T1, &m.hi, 64 * FULL, p.head, row, full, policy);
            } else {
              mbar_arrive(full);
            }
          }
          __syncwarp();
        }
      }
      if (!ok) break;
      u += blocks;
      p.next_rows(a);
    }
  } else if (warp == 4) {
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
    const float sc = a.score_log2;
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
        if (kb >= cached) {
          const uint32_t t = 2 * j + 1, slot = t % RING;
          if (!(ok = __all_sync(0xffffffffu, wait(t_full + 8 * slot, (t / RING) & 1)))) break;
          uint8_t* v = sm + C::OFF_RING + slot * C::TILE;
          bool odd = false;
#pragma unroll
          for (int c = 0; c < FULL; ++c) odd |= clear_slice<T, 128>(v + c * C::T1, keys, true, tid);
          if (TAIL > 0) odd |= clear_slice<T, (TAIL > 0 ? TAIL * 2 : 16)>(v + FULL * C::T1, keys, true, tid);
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
        const float* scales = nullptr;  // of a cached block
        if (kb >= cached) {
#pragma unroll
          for (int c = 0; c < KB; c += 32) {
            const uint32_t bits = valid ? seen(a, p.r, node, j0 + c) : 0u;
#pragma unroll
            for (int e = 0; e < 32; ++e)  // -inf: P = 0
              r[c + e] = bits >> e & 1 ? __float_as_uint(__uint_as_float(r[c + e]) * sc) : 0xff800000u;
          }
        } else {
          const uint32_t t = 2 * j + 1, slot = t % RING;
          if (!(ok = __all_sync(0xffffffffu, wait(t_full + 8 * slot, (t / RING) & 1)))) break;
          scales = reinterpret_cast<const float*>(sm + C::OFF_SCALES) + (j % SCALES) * 3 * KB;
#pragma unroll
          for (int c = 0; c < KB; c += 4) {
            const float4 f = *reinterpret_cast<const float4*>(scales + c), lv = *reinterpret_cast<const float4*>(scales + KB + c);
            const float2 y0 = fma_f32x2(make_float2(__uint_as_float(r[c]), __uint_as_float(r[c + 1])), make_float2(f.x, f.y), make_float2(lv.x, lv.y));
            const float2 y1 = fma_f32x2(make_float2(__uint_as_float(r[c + 2]), __uint_as_float(r[c + 3])), make_float2(f.z, f.w), make_float2(lv.z, lv.w));
            r[c] = __float_as_uint(y0.x);
            r[c + 1] = __float_as_uint(y0.y);
            r[c + 2] = __float_as_uint(y1.x);
            r[c + 3] = __float_as_uint(y1.y);
          }
          if (keys < KB) {
#pragma unroll
            for (int c = 0; c < KB; ++c)
              if (c >= keys) r[c] = 0xff800000u;
          }
        }
        float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
        for (int c = 0; c < KB; ++c) mx[c & 3] = fmaxf(mx[c & 3], __uint_as_float(r[c]));
        const float m_blk = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3]));
        float alpha = 1.f;
        const bool grow = m_blk - m_ref > TREE_GROWTH;
        if (grow) {
          alpha = ex2(m_ref - m_blk);
          m_ref = m_blk;
        }
        const float mo = TREE_SHIFT - (m_ref == -INFINITY ? 0.f : m_ref);  // (nothing seen so far: P = 0)
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
        for (int c = 0; c < KB; c += 32) exp_chunk<T>(r + c, mo, scales ? scales + 2 * KB + c : nullptr, pk + c / 2, l);
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
              if (!(seen(a, p.r, node, k & ~31) >> (k & 31) & 1)) continue;
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
        if (valid && whole && a.lse) a.lse[orow * a.heads + h] = (m_ref + (log2f(sum) - TREE_SHIFT)) * 0.6931471805599453f;
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
  if (warp == 4) tmem_dealloc(tmem, C::TM_COLS);
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
cudaError_t launch_tc(const QuantisedArgs& a, int dtype, int ctas, cudaStream_t s) {
  using C = TcCfg<DP>;
  cudaError_t e = allow_smem<tree_attention_quantised_tc_kernel<T, DP>>(C::BYTES);
  if (e != cudaSuccess) return e;
  AllMaps m;
  const cuuint64_t dim = a.cache.dim, kv = a.cache.heads, rows = a.n_rows;
  const auto fresh = [&](Maps* map, const void* base, cuuint64_t heads, long long stride, cuuint32_t box_heads, cuuint32_t box_rows) {
    const cuuint64_t dims[3] = {dim, heads, rows}, strides[2] = {dim * 2, static_cast<cuuint64_t>(stride) * 2};
    const cuuint32_t b[2] = {box_heads, box_rows};
    return make_maps(map, dtype, C::TAIL, base, 3, dims, strides, b);
  };
  if (!fresh(&m.q, a.q, a.heads, a.q_stride, a.group, a.tile_rows / a.group) || !fresh(&m.k_new, a.k_new, kv, a.k_new_stride, 1, KB) ||
      !fresh(&m.v_new, a.v_new, kv, a.v_new_stride, 1, KB))
    return cudaErrorInvalidValue;
  e = launch_ex(tree_attention_quantised_tc_kernel<T, DP>, dim3(ctas), dim3(TC_THREADS), C::BYTES, s, 1, m, a);
  return e != cudaSuccess ? e : launch_tree_join<T, DP, AQ, true>(a, ctas, s);
}

}  // namespace

cudaError_t launch_tree_attention_quantised_tc(const QuantisedArgs& a, int dtype, int dp, int ctas, cudaStream_t s) {
  const auto width = [&](auto type) {
    using T = decltype(type);
    return dp == 64    ? launch_tc<T, 64>(a, dtype, ctas, s)
           : dp == 80  ? launch_tc<T, 80>(a, dtype, ctas, s)
           : dp == 96  ? launch_tc<T, 96>(a, dtype, ctas, s)
           : dp == 128 ? launch_tc<T, 128>(a, dtype, ctas, s)
                       : launch_tc<T, 256>(a, dtype, ctas, s);
  };
  return dtype == IVIT_BF16 ? width(bf16{}) : width(half{});
}

}  // namespace ivit
