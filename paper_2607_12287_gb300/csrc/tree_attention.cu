// New rows of every request over its cached tokens and over each other (ivit_tree_attention):
//
//   o = sum_j p_j v_j / sum_j p_j,  p_j = exp(scale q.k_j - m),  lse = m + log sum_j p_j
//
// over the keys j that a row sees: all cached ones, and the new rows that its mask names.
//
// Rows that share a key head (the new rows x the query heads of the group) form tiles of 16, 32, 64
// or 128; a tile walks its keys -- the cached tokens and, behind them, the new rows -- 64 at a time.
// All (request, row tile, 64 keys) of a key head, in this order, are cut into as many equal runs as
// there are CTAs for the head, so that ragged lengths and few requests load the chip alike.  A run
// that holds a tile's keys only in part leaves its running maximum, sum and output (fp32) in
// the workspace, and a second kernel joins the parts of a tile in the order of their keys.
//
// Tiles of 16 rows (a step of one token, small trees): the 64 keys of a tile belong to the four warps, 16 each.  A
// warp copies its own keys and values with 16-byte asynchronous copies into its part of a ring of tiles in shared
// memory, looks the pages up a tile ahead, and walks on without a barrier; its running maximum, sum and output
// meet the others' at the end of a tile of rows.  Products by mma.m16n8k16; probabilities enter the one with V
// as two 16-bit terms (16 bits and more of their fp32 value), which is free beside the cache's bytes.
// Tiles of 32 to 128 rows are for what the tcgen05 kernel (tree_attention_tc.cu) does not take: pages of fewer
// than 8 tokens, groups of more than 128 heads.  Row groups of 16 are split over four or
// eight warps that share the keys, the 64 keys too for 32 rows; probabilities are rounded once from 64 rows on, where
// the second term's products would not be free.  Sums use the fp32 values everywhere.
//
// Bound: the cache's bytes for few rows per key head (32 requests of up to 16384 tokens, 32 + 8 heads of 128, 171 us:
// 6470 GB/s; 64 of up to 8192, 16 + 4 heads of 64, 52 us: 5260 GB/s), the chain of dependent reads of a start
// for short ones (one request of 1041 tokens 7.5 us), mma.sync's rate for many rows (16 trees of up to 31 drafts over up to
// 8192 tokens, 32 + 8 heads of 128, pages of 4 tokens 150 us; of 32, on tcgen05, 62).  Heads of 256 have one stage of the
// ring, and with eight warps on an SM the cache's bytes still bound a decoding step (32 requests of up to 16384 tokens,
// 16 + 4 heads, 171 us: 6470 GB/s).
#include <algorithm>
#include <type_traits>

#include "tree_attention.cuh"

namespace ivit {
namespace {

constexpr int TK = 64;              // keys of a tile
// More rows per key head than this take the tcgen05 kernel where it can (pages of 8 tokens and more, groups of up to 128).
// Both sides, 16 requests of up to 8192 tokens, us: 32 rows of heads of 128 58 (tcgen05) and 70, 64 rows 60 and 79, 124
// rows 62 and 137; heads of 64, 32 rows 31 and 33, 64 rows 32 and 35; up to 4096 tokens, heads of 256, 32 rows 30 and 41,
// 64 rows 30 and 45, 124 rows 33 and 53; one request of 1000 tokens, 32 rows of 128, 12.3 and 11.6, of 600 tokens, 32
// rows of 256, 15.4 and 13.7 (lengths are not known when the call is made).
constexpr int TC_ROWS = 16;

struct Keys64 {
  static constexpr int LEAST = 1;
  static __device__ __forceinline__ int tiles(const TreeRequest& r) { return (r.len + r.n + TK - 1) / TK; }
};

template <typename T>
__device__ __forceinline__ void mma(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1);
template <>
__device__ __forceinline__ void mma<bf16>(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  mma_bf16_16816(d, a[0], a[1], a[2], a[3], b0, b1);
}
template <>
__device__ __forceinline__ void mma<half>(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

__device__ __forceinline__ void ldmatrix4(uint32_t (&r)[4], uint32_t addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(addr)
               : "memory");
}
__device__ __forceinline__ void ldmatrix4_trans(uint32_t (&r)[4], uint32_t addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(addr)
               : "memory");
}

// 16 bytes to shared memory, or zeros (nothing is read) if not `ok`.  Without an L2 policy: a build with one on these
// copies faulted at heads of 256, and reading showed no cause that would spare the others (it was up to 8 % faster).
__device__ __forceinline__ void copy16(uint32_t dst, const void* src, bool ok) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(ok ? 16 : 0) : "memory");
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copies_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}

template <int DP, int RW>
struct Cfg {
  static constexpr int M = 16 * RW, KW = RW < 4 ? 4 / RW : 1, WK = TK / KW;  // rows, warps along the keys, keys of a warp
  static constexpr int THREADS = 32 * RW * KW;
  // One row group: no two warps share keys, each copies its own, and the walk has no barrier.
  static constexpr bool ALONE = RW == 1;
  // Bytes of a row in shared memory: 8 rows of ldmatrix must not meet in a bank, by a swizzle of the pieces of
  // rows of 64, 128 and 256 values, by an odd number of pieces for 80 and 96.
  static constexpr bool PADDED = DP == 80 || DP == 96;
  static constexpr int ROW = 2 * DP + (PADDED ? 16 : 0);
  static constexpr int TILE = TK * ROW;
  static constexpr int CTAS = ALONE ? (DP <= 64 ? 4 : DP <= 80 ? 3 : 2) : DP <= 128 && RW < 8 ? 2 : 1;  // per SM
  static constexpr bool QSMEM = DP > 128;                                    // queries in shared memory, not registers
  static constexpr int STAGES = ALONE ? (DP <= 128 ? 3 : 1) : DP > 128 ? 2 : 3;
  static constexpr int TERMS = RW < 4 ? 2 : 1;
  // a copy of a tile (of the warp's keys if it is alone): CP lanes for the pieces of a row, RP rows at a time
  static constexpr int CP = DP <= 64 ? 8 : DP <= 128 ? 16 : 32, RP = (ALONE ? 32 : THREADS) / CP, COPIES = (ALONE ? WK : TK) / RP;
  static constexpr int MEET = DP + 4;                                        // floats of a row where the warps meet
  static constexpr int OFF_Q = STAGES * 2 * TILE;
  static constexpr int OFF_MEET = OFF_Q + (QSMEM ? M * ROW : 0);
  static constexpr int OFF_FLAGS = OFF_MEET + (ALONE ? KW * M * 8 : KW > 1 ? M * (MEET + 2) * 4 : 0);
  static constexpr int BYTES = OFF_FLAGS + 4 * 16;
  static constexpr int PART = tree_part_floats(M, DP);
  static_assert(TREE_MAX_REQ * 8 <= OFF_Q, "the units before each request");
  static_assert(CTAS * (BYTES + 1024 + 128) <= 228 * 1024, "shared memory of an SM");
};

// Shared-memory address of 16-byte piece c of a row.
template <class C>
__device__ __forceinline__ uint32_t piece(uint32_t tile, int row, int c) {
  return tile + row * C::ROW + ((C::PADDED ? c : c ^ (row & 7)) << 4);
}

// Which of the 64 keys from k0 on new row `node` of the request sees (bit j: key k0 + j).
__device__ __forceinline__ uint64_t seen(const TreeArgs& a, const TreeRequest& r, int node, int k0) {
  const auto low = [](int n) { return n >= 64 ? ~0ull : n > 0 ? (1ull << n) - 1 : 0ull; };
  const int first = k0 - r.len;  // new row of bit 0 (negative: cached tokens up to there)
  if (a.mask_mode == IVIT_MASK_CAUSAL) return low(node + 1 - first);
  if (a.mask_mode == IVIT_MASK_ALL) return low(r.n - first);
  const uint32_t* words = a.mask + static_cast<size_t>(r.row0 + node) * a.mask_words;
  const auto word = [&](int w) { return static_cast<uint64_t>(w < a.mask_words ? words[w] : 0u); };
  uint64_t bits;
  if (first < 0) {
    bits = ((word(0) | word(1) << 32) << -first) | low(-first);
  } else {
    const int w = first >> 5, s = first & 31;
    bits = (word(w) | word(w + 1) << 32) >> s;
    if (s) bits |= word(w + 2) << (64 - s);
  }
  return bits & low(r.n - first);
}

// ONE_PAGE: the 16 keys of a warp that is alone are of one page.
template <typename T, int DP, int RW, bool ONE_PAGE>
__global__ void __launch_bounds__(Cfg<DP, RW>::THREADS, Cfg<DP, RW>::CTAS) tree_attention_kernel(const TreeArgs a) {
  using C = Cfg<DP, RW>;
  constexpr int M = C::M, KW = C::KW, WK = C::WK, ROW = C::ROW, STAGES = C::STAGES, THREADS = C::THREADS;
  constexpr int PIECES = DP / 8, COPIES = C::COPIES, RP = C::RP;
  extern __shared__ __align__(128) uint8_t sm[];
  const uint32_t sb = smem_u32(sm);
  // [tile % 4][16 keys] whose values are not finite; cleared two tiles ahead, a barrier away from their use
  uint32_t* flags = reinterpret_cast<uint32_t*>(sm + C::OFF_FLAGS);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, t = lane & 3;
  const int rw = warp / KW, kw = warp % KW;  // row group and key group of the warp
  const int pieces = a.cache.dim >> 3;
  pdl_wait();
  pdl_launch_dependents();

  if (blockIdx.x == 0 && tid == 0) *a.err = 0;  // (nothing here waits on a barrier that could fail)
  TreeRun<Keys64> run{};
  if (!run.find<THREADS>(a, reinterpret_cast<unsigned long long*>(sm))) return;
  TreePlace<Keys64> load = run.at, at = run.at;
  const int units = static_cast<int>(run.hi - run.lo);
  if (pieces < PIECES) {
    // columns past a head's are zero for good: no copy touches them
    for (int x = tid; x < STAGES * 2 * TK * (PIECES - pieces); x += THREADS) {
      const int row = x / (PIECES - pieces), c = pieces + x % (PIECES - pieces);
      *reinterpret_cast<uint4*>(sm + piece<C>(0, row, c)) = make_uint4(0, 0, 0, 0);
    }
  }

  // A copy's part of this thread: piece cp of the rows r0, r0 + RP, ... of a tile.
  const int cp = tid % C::CP, r0 = C::ALONE ? warp * WK + lane / C::CP : tid / C::CP, page_mask = (1 << a.cache.page_shift) - 1;
  const uint32_t to = piece<C>(0, r0, cp);
  const auto place = [&](int x) {  // of its x-th row in a tile (8 rows repeat the swizzle)
    return (C::PADDED || RP % 8 == 0 ? to : to ^ ((x * RP & 7) << 4)) + x * RP * ROW;
  };
  // The pages of the tile at `load`, of those rows; kept a tile ahead of the copies.
  constexpr int IDS = ONE_PAGE ? 1 : COPIES;
  int ids[IDS];
  const auto look_up = [&] {
    const int* table = a.table + static_cast<size_t>(load.req) * a.max_pages;
    const int key = load.kt * TK + (ONE_PAGE ? warp * WK : r0);
    if ((load.kt + 1) * TK <= load.r.len) {
#pragma unroll
      for (int x = 0; x < IDS; ++x) ids[x] = table[(key + x * RP) >> a.cache.page_shift];
    } else {
#pragma unroll
      for (int x = 0; x < IDS; ++x) ids[x] = key + x * RP < load.r.len ? table[(key + x * RP) >> a.cache.page_shift] : -1;
    }
  };
  const auto copy = [&](int stage) {
    if (cp >= pieces) return;
    const uint32_t ks = sb + stage * 2 * C::TILE, vs = ks + C::TILE;
    const long long head = load.head * a.cache.head_stride + 8 * cp;
    const T *kc = static_cast<const T*>(a.k_cache) + head, *vc = static_cast<const T*>(a.v_cache) + head;
    const int key = load.kt * TK + r0;
    const auto cached = [&](int x, bool& ok) {  // where the x-th row is in the caches (row 0 if its page is outside)
      const int id = ids[ONE_PAGE ? 0 : x];
      ok = static_cast<unsigned>(id) < static_cast<unsigned>(a.cache.n_pages);
      return ok ? id * a.cache.page_stride + ((key + x * RP) & page_mask) * a.cache.token_stride : 0;
    };
    if ((load.kt + 1) * TK <= load.r.len) {
      bool ok;
      long long off = cached(0, ok);
      const long long step = RP * a.cache.token_stride;
#pragma unroll
      for (int x = 0; x < COPIES; ++x) {
        if (!ONE_PAGE && x > 0) off = cached(x, ok);
        copy16(ks + place(x), kc + off, ok);
        copy16(vs + place(x), vc + off, ok);
        if (ONE_PAGE) off += step;
      }
      return;
    }
#pragma unroll
    for (int x = 0; x < COPIES; ++x) {  // the new rows, and what lies behind them (zeros)
      const int fresh = key + x * RP - load.r.len;
      const T *k = kc, *v = vc;
      bool ok;
      if (fresh < 0) {
        const long long off = cached(x, ok);
        k += off;
        v += off;
      } else {
        ok = fresh < load.r.n;
        if (ok) {
          const long long row = load.r.row0 + fresh, col = load.head * a.cache.dim + 8 * cp;
          k = static_cast<const T*>(a.k_new) + row * a.k_new_stride + col;
          v = static_cast<const T*>(a.v_new) + row * a.v_new_stride + col;
        }
      }
      copy16(ks + place(x), k, ok);
      copy16(vs + place(x), v, ok);
    }
  };

  if (tid < 16) flags[tid] = 0;
  int loaded = 0;
  look_up();
  auto fill = [&](int stage) {  // the next tile's copies, if there is one
    if (loaded < units) {
      copy(stage);
      load.next(a);
      if (++loaded < units) look_up();
    }
    copies_commit();
  };
#pragma unroll 1
  for (int s = 0; s < (STAGES > 1 ? STAGES - 1 : 1); ++s) fill(s);
  __syncthreads();  // the flags are clear, and the columns past a head's

  uint32_t q[C::QSMEM ? 1 : DP / 16][4];
  float o[DP / 8][4], m[2], l[2];
  int node[2];               // new row of the lane's rows g, g + 8 (-1: none)
  bool two = true;           // the warp has rows past its first 8
  bool begun = true;         // of the tile's keys the run has seen the first

  for (int u = 0; u < units; ++u) {
    const int stage = u % STAGES;
    const bool fresh_rows = u == 0 || at.kt == 0;
    if (fresh_rows) {  // a new tile of rows
      begun = at.kt == 0;
      two = at.rt * M + rw * 16 + 8 < at.r.n * a.group;
      const T* from[2];
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        const int x = at.rt * M + rw * 16 + g + 8 * r, n = x / a.group;
        node[r] = n < at.r.n ? n : -1;
        from[r] = static_cast<const T*>(a.q) + (at.r.row0 + n) * a.q_stride +
                  static_cast<long long>(at.head * a.group + x - n * a.group) * a.cache.dim;
        m[r] = -INFINITY;
        l[r] = 0.f;
      }
      if (!C::QSMEM) {
#pragma unroll
        for (int r = 0; r < 2; ++r)
#pragma unroll
          for (int e = r; e < 4; e += 2)
#pragma unroll
            for (int c = 0; c < DP / 16; ++c) {
              const int d = 16 * c + 2 * t + 8 * (e >> 1);
              q[c][e] = (r == 0 || two) && node[r] >= 0 && d < a.cache.dim ? *reinterpret_cast<const uint32_t*>(from[r] + d) : 0u;
            }
      } else {
        __syncthreads();  // the tile before has been multiplied
        if (kw == 0) {
#pragma unroll
          for (int r = 0; r < 2; ++r)
            for (int c = t; c < PIECES; c += 4)
              *reinterpret_cast<uint4*>(sm + C::OFF_Q + (piece<C>(0, rw * 16 + g + 8 * r, c))) =
                  node[r] >= 0 && c < pieces ? *reinterpret_cast<const uint4*>(from[r] + 8 * c) : make_uint4(0, 0, 0, 0);
        }
      }
#pragma unroll
      for (int j = 0; j < DP / 8; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[j][e] = 0.f;
    }
    const uint32_t ks = sb + stage * 2 * C::TILE, vs = ks + C::TILE;
    const int k0 = at.kt * TK;
    const bool edge = k0 + TK > at.r.len;  // holds new rows, or ends
    uint32_t* odd_keys = flags + 4 * (u & 3);
    copies_wait<(STAGES > 2 ? STAGES - 2 : 0)>();
    if (edge) {
      // Values of new rows that are not finite would reach rows that do not see them (0 * NaN): they
      // become zero here, each thread looking at what it copied, and are added back below.
#pragma unroll
      for (int x = 0; x < COPIES; ++x) {
        const int row = r0 + x * RP;
        if (cp >= pieces || k0 + row < at.r.len || k0 + row >= at.r.len + at.r.n) continue;
        uint32_t* w = reinterpret_cast<uint32_t*>(sm + (vs - sb) + place(x));
        bool odd = false;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const uint32_t e16 = std::is_same<T, bf16>::value ? 0x7f80u : 0x7c00u;
          const uint32_t x0 = w[i];
          uint32_t keep = 0xffffffffu;
          if ((x0 & e16) == e16) keep &= 0xffff0000u;
          if ((x0 >> 16 & e16) == e16) keep &= 0x0000ffffu;
          if (keep != 0xffffffffu) {
            w[i] = x0 & keep;
            odd = true;
          }
        }
        if (odd) atomicOr(&odd_keys[row >> 4], 1u << (row & 15));
      }
    }
    // everyone's copies (of this warp's keys) have landed, and the stage of the tile before is free
    if (C::ALONE && !(C::QSMEM && fresh_rows)) {
      __syncwarp();
    } else {
      __syncthreads();
    }
    if (lane == 0 && warp < 4) flags[4 * (u + 2 & 3) + warp] = 0;
    if (STAGES > 1) fill((u + STAGES - 1) % STAGES);

    if (at.rt * M + rw * 16 < at.r.n * a.group) {  // (else the warp's rows are all padding)
      // scores of the warp's keys
      float s[WK / 8][4];
#pragma unroll
      for (int j = 0; j < WK / 8; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) s[j][e] = 0.f;
#pragma unroll
      for (int c = 0; c < DP / 16; ++c) {
        if (C::QSMEM) ldmatrix4(q[0], piece<C>(sb + C::OFF_Q, rw * 16 + (lane & 15), 2 * c + (lane >> 4)));
#pragma unroll
        for (int j = 0; j < WK / 16; ++j) {
          uint32_t b[4];
          const int row = kw * WK + 16 * j + (lane & 7) + ((lane & 16) >> 1);
          ldmatrix4(b, piece<C>(ks, row, 2 * c + (lane >> 3 & 1)));
          mma<T>(s[2 * j], q[C::QSMEM ? 0 : c], b[0], b[1]);
          mma<T>(s[2 * j + 1], q[C::QSMEM ? 0 : c], b[2], b[3]);
        }
      }
      if (edge) {
#pragma unroll
        for (int r = 0; r < 2; ++r) {
          const uint64_t bits = node[r] >= 0 ? seen(a, at.r, node[r], k0) >> (kw * WK) : 0;
#pragma unroll
          for (int j = 0; j < WK / 8; ++j)
#pragma unroll
            for (int e = 0; e < 2; ++e)
              if (!(bits >> (8 * j + 2 * t + e) & 1)) s[j][2 * r + e] = -INFINITY;
        }
      }
      // probabilities against the reference maximum, and their sum
      float mx[2];
      bool grow = false;
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        if (r == 1 && !two) break;
        mx[r] = s[0][2 * r];
#pragma unroll
        for (int j = 0; j < WK / 8; ++j) mx[r] = fmaxf(mx[r], fmaxf(s[j][2 * r], s[j][2 * r + 1]));
        mx[r] = fmaxf(mx[r], __shfl_xor_sync(0xffffffffu, mx[r], 1));
        mx[r] = fmaxf(mx[r], __shfl_xor_sync(0xffffffffu, mx[r], 2));
        grow |= (mx[r] - m[r]) * a.scale_log2 > TREE_GROWTH;
      }
      if (__any_sync(0xffffffffu, grow)) {
#pragma unroll
        for (int r = 0; r < 2; ++r) {
          if ((r == 1 && !two) || !(mx[r] > m[r])) continue;
          const float alpha = ex2((m[r] - mx[r]) * a.scale_log2);
          m[r] = mx[r];
          l[r] *= alpha;
#pragma unroll
          for (int j = 0; j < DP / 8; ++j) {
            o[j][2 * r] *= alpha;
            o[j][2 * r + 1] *= alpha;
          }
        }
      }
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        if (r == 1 && !two) break;
        const float mo = TREE_SHIFT - (m[r] == -INFINITY ? 0.f : m[r] * a.scale_log2);  // (nothing seen so far: P = 0)
        float sum[2] = {0.f, 0.f};
#pragma unroll
        for (int j = 0; j < WK / 8; ++j)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            s[j][2 * r + e] = ex2(fmaf(s[j][2 * r + e], a.scale_log2, mo));
            sum[e] += s[j][2 * r + e];
          }
        l[r] += sum[0] + sum[1];
      }
#pragma unroll
      for (int j = 0; j < WK / 16; ++j) {
        uint32_t p[C::TERMS][4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          if ((e & 1) && !two) {
            p[0][e] = p[C::TERMS - 1][e] = 0u;
            continue;
          }
          float& x = s[2 * j + (e >> 1)][2 * (e & 1)];
          float& y = s[2 * j + (e >> 1)][2 * (e & 1) + 1];
          p[0][e] = pack2<T>(x, y);
          if (C::TERMS == 2) {
            const float2 h = unpack2<T>(p[0][e]);
            p[C::TERMS - 1][e] = pack2<T>(x - h.x, y - h.y);
          }
        }
#pragma unroll
        for (int c = 0; c < DP / 16; ++c) {
          uint32_t b[4];
          const int row = kw * WK + 16 * j + (lane & 15);
          ldmatrix4_trans(b, piece<C>(vs, row, 2 * c + (lane >> 4)));
#pragma unroll
          for (int x = 0; x < C::TERMS; ++x) {
            mma<T>(o[2 * c], p[x], b[0], b[1]);
            mma<T>(o[2 * c + 1], p[x], b[2], b[3]);
          }
        }
      }
      if (edge && (C::ALONE ? odd_keys[kw] : odd_keys[0] | odd_keys[1] | odd_keys[2] | odd_keys[3])) {
        // values that are not finite, for the rows that see them
        for (int k = kw * WK; k < (kw + 1) * WK; ++k) {
          if (!(odd_keys[k >> 4] >> (k & 15) & 1)) continue;
          const T* v = static_cast<const T*>(a.v_new) + (at.r.row0 + k0 + k - at.r.len) * a.v_new_stride + at.head * a.cache.dim;
#pragma unroll
          for (int r = 0; r < 2; ++r)
            if (node[r] >= 0 && seen(a, at.r, node[r], k0) >> k & 1) {
#pragma unroll
              for (int j = 0; j < DP / 8; ++j)
                if (8 * j < a.cache.dim) {
                  const float2 x = unpack2<T>(*reinterpret_cast<const uint32_t*>(v + 8 * j + 2 * t));
                  if (!isfinite(x.x)) o[j][2 * r] += x.x;
                  if (!isfinite(x.y)) o[j][2 * r + 1] += x.y;
                }
            }
        }
      }
    }

    if (at.kt == at.nkt - 1 || u == units - 1) {  // the run has no more keys of this tile of rows
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        l[r] += __shfl_xor_sync(0xffffffffu, l[r], 1);
        l[r] += __shfl_xor_sync(0xffffffffu, l[r], 2);
      }
      const bool whole = begun && at.kt == at.nkt - 1;
      // a part: the first of the run, or the one it ends with
      float* part = a.parts + static_cast<size_t>(2 * blockIdx.x + (u - at.kt > 0 && begun ? 1 : 0)) * C::PART;
      const auto out_of = [&](int row, int node, int& h, long long& orow) {  // of a row of the tile
        h = at.head * a.group + at.rt * M + row - node * a.group;
        orow = at.r.row0 + node;
        return static_cast<T*>(a.out) + orow * a.out_stride + static_cast<long long>(h) * a.cache.dim;
      };
      if constexpr (C::ALONE) {
        // Each warp leaves its output in the place of its own keys and values of this tile (rows 0 - 7 and 8 - 15;
        // pieces of a row turn with it, so that the rows do not meet in a bank); all threads add them up.
        constexpr int COLS = DP / 4;
        float2* ml = reinterpret_cast<float2*>(sm + C::OFF_MEET);  // [KW][M]
        const auto at_row = [&](int w, int row) {
          return sm + stage * 2 * C::TILE + (row >> 3) * C::TILE + w * WK * ROW + (row & 7) * DP * 4;
        };
        __syncwarp();
#pragma unroll
        for (int r = 0; r < 2; ++r) {
          if (r == 1 && !two) break;
          if (t == 0) ml[warp * M + g + 8 * r] = make_float2(m[r], l[r]);
          uint8_t* dst = at_row(warp, g + 8 * r);
#pragma unroll
          for (int j = 0; j < DP / 8; ++j) {
            const int c = 2 * j + (t >> 1) + g;
            *reinterpret_cast<float2*>(dst + 16 * (c >= COLS ? c - COLS : c) + 8 * (t & 1)) = make_float2(o[j][2 * r], o[j][2 * r + 1]);
          }
        }
        __syncthreads();
        const int rows = min(M, at.r.n * a.group - at.rt * M);
#pragma unroll 1
        for (int e = tid; e < rows * COLS; e += THREADS) {
          const int row = e / COLS, col = e - row * COLS, turned = col + (row & 7);
          float top = -INFINITY, sum = 0.f;
          float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
          float2 w[KW];
#pragma unroll
          for (int k = 0; k < KW; ++k) {
            w[k] = ml[k * M + row];
            top = fmaxf(top, w[k].x);
          }
          const float ref = top == -INFINITY ? 0.f : top;
#pragma unroll
          for (int k = 0; k < KW; ++k) {
            const float4 x = *reinterpret_cast<const float4*>(at_row(k, row) + 16 * (turned >= COLS ? turned - COLS : turned));
            const float f = ex2((w[k].x - ref) * a.scale_log2);
            sum += w[k].y * f;
            y = make_float4(y.x + x.x * f, y.y + x.y * f, y.z + x.z * f, y.w + x.w * f);
          }
          if (whole) {
            int h;
            long long orow;
            T* dst = out_of(row, (at.rt * M + row) / a.group, h, orow) + 4 * col;
            const float inv = sum == 0.f ? 0.f : 1.f / sum;
            if (4 * col < a.cache.dim)
              *reinterpret_cast<uint2*>(dst) = make_uint2(pack2<T>(y.x * inv, y.y * inv), pack2<T>(y.z * inv, y.w * inv));
            if (a.lse && col == 0)
              a.lse[orow * a.heads + h] = (top * a.scale_log2 + (log2f(sum) - TREE_SHIFT)) * 0.6931471805599453f;
          } else {
            reinterpret_cast<float4*>(part + row * DP)[col] = y;
            if (col == 0) *reinterpret_cast<float2*>(part + M * DP + 2 * row) = make_float2(top, sum);
          }
        }
        __syncthreads();  // the stage is free
        for (int x = lane; x < 2 * WK * (PIECES - pieces); x += 32) {  // the columns past a head's are zero again
          const int row = x / (PIECES - pieces), c = pieces + x % (PIECES - pieces);
          const uint32_t tile = stage * 2 * C::TILE + (row >= WK ? C::TILE : 0);
          *reinterpret_cast<uint4*>(sm + piece<C>(tile, warp * WK + (row & (WK - 1)), c)) = make_uint4(0, 0, 0, 0);
        }
      } else {
        if constexpr (KW > 1) {  // the warps of a row group, one after another into the first
          float* meet = reinterpret_cast<float*>(sm + C::OFF_MEET);
          float* mm = meet + M * C::MEET;
#pragma unroll 1
          for (int w = 1; w < KW; ++w) {
            if (kw == w) {
#pragma unroll
              for (int r = 0; r < 2; ++r) {
                const int row = rw * 16 + g + 8 * r;
                if (t == 0) {
                  mm[2 * row] = m[r];
                  mm[2 * row + 1] = l[r];
                }
#pragma unroll
                for (int j = 0; j < DP / 8; ++j)
                  *reinterpret_cast<float2*>(meet + row * C::MEET + 8 * j + 2 * t) = make_float2(o[j][2 * r], o[j][2 * r + 1]);
              }
            }
            __syncthreads();
            if (kw == 0) {
#pragma unroll
              for (int r = 0; r < 2; ++r) {
                const int row = rw * 16 + g + 8 * r;
                const float m2 = mm[2 * row], l2 = mm[2 * row + 1];
                const float top = fmaxf(m[r], m2), ref = top == -INFINITY ? 0.f : top;
                const float f1 = ex2((m[r] - ref) * a.scale_log2), f2 = ex2((m2 - ref) * a.scale_log2);
                m[r] = top;
                l[r] = l[r] * f1 + l2 * f2;
#pragma unroll
                for (int j = 0; j < DP / 8; ++j) {
                  const float2 x = *reinterpret_cast<const float2*>(meet + row * C::MEET + 8 * j + 2 * t);
                  o[j][2 * r] = o[j][2 * r] * f1 + x.x * f2;
                  o[j][2 * r + 1] = o[j][2 * r + 1] * f1 + x.y * f2;
                }
              }
            }
            __syncthreads();
          }
        }
        if (kw == 0) {
#pragma unroll
          for (int r = 0; r < 2; ++r) {
            const int row = rw * 16 + g + 8 * r;
            if (whole) {
              if (node[r] < 0) continue;
              int h;
              long long orow;
              T* dst = out_of(row, node[r], h, orow);
              const float inv = l[r] == 0.f ? 0.f : 1.f / l[r];
#pragma unroll
              for (int j = 0; j < DP / 8; ++j)
                if (8 * j < a.cache.dim)
                  *reinterpret_cast<uint32_t*>(dst + 8 * j + 2 * t) = pack2<T>(o[j][2 * r] * inv, o[j][2 * r + 1] * inv);
              if (a.lse && t == 0)
                a.lse[orow * a.heads + h] = (m[r] * a.scale_log2 + (log2f(l[r]) - TREE_SHIFT)) * 0.6931471805599453f;
            } else {
              if (t == 0) {
                part[M * DP + 2 * row] = m[r];
                part[M * DP + 2 * row + 1] = l[r];
              }
#pragma unroll
              for (int j = 0; j < DP / 8; ++j)
                *reinterpret_cast<float2*>(part + row * DP + 8 * j + 2 * t) = make_float2(o[j][2 * r], o[j][2 * r + 1]);
            }
          }
        }
      }
      if (!whole && begun && tid == 0) run.note_join(a, at, run.lo + u - at.kt);
    }
    at.next(a);
    if (STAGES == 1) {  // (the warp's own keys: it alone reads them)
      __syncwarp();
      fill(0);
    }
  }
}

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

bool valid(const ivit_attention_config& c, const ivit_cache_layout& l) {
  return valid_cache(l) && c.n_req >= 1 && c.n_req <= TREE_MAX_REQ && c.heads >= 1 && c.heads <= 256 && c.heads % l.kv_heads == 0 &&
         c.max_pages >= 1 && static_cast<long long>(c.max_pages) * l.page_size < (1LL << 31) - (1 << 20) && c.max_new >= 1 &&
         c.max_new <= 65536 && c.mask_mode >= IVIT_MASK_CAUSAL && c.mask_mode <= IVIT_MASK_TREE && c.mask_words >= 0 &&
         c.mask_words <= 32768 && (c.mask_mode != IVIT_MASK_TREE || c.mask_words > 0) && c.scale > 0.f && c.scale < 1e30f;
}

// Which kernel, and its sizes: tiles of 16 * rw rows of mma.sync, or with tc the tcgen05 kernel's of up to 128.
struct Plan {
  bool tc;
  int dp, rw, tile_rows, ctas_per_sm, part_floats;
};

template <int DP, int RW>
Plan plan_of() {
  using C = Cfg<DP, RW>;
  return {false, DP, RW, C::M, C::CTAS, C::PART};
}

Plan plan(const ivit_attention_config& c, const ivit_cache_layout& l) {
  const int group = c.heads / l.kv_heads;
  const int rows = static_cast<int>(std::min<long long>(128, static_cast<long long>(c.max_new) * group));  // that share a key head
  const int dp = l.head_dim <= 64 ? 64 : l.head_dim <= 80 ? 80 : l.head_dim <= 96 ? 96 : l.head_dim <= 128 ? 128 : 256;
  if (rows > TC_ROWS && group <= 128 && l.page_size >= 8 && l.head_stride > 0 && l.token_stride > 0 && l.page_stride > 0)
    return {true, dp, 0, tree_tc_rows(group), dp <= 128 ? 2 : 1, tree_part_floats(128, dp)};
  // the smallest tile that holds the rows
  const auto groups = [&](auto d) {
    constexpr int DP = decltype(d)::value;
    return rows <= 16 ? plan_of<DP, 1>() : rows <= 32 ? plan_of<DP, 2>() : rows <= 64 ? plan_of<DP, 4>() : plan_of<DP, 8>();
  };
  return dp == 64    ? groups(std::integral_constant<int, 64>{})
         : dp == 80  ? groups(std::integral_constant<int, 80>{})
         : dp == 96  ? groups(std::integral_constant<int, 96>{})
         : dp == 128 ? groups(std::integral_constant<int, 128>{})
                     : groups(std::integral_constant<int, 256>{});
}

// The error word, then of each CTA a note and two parts.
size_t workspace_of(const Plan& p) {
  return 16 + static_cast<size_t>(p.ctas_per_sm) * TREE_MAX_SMS * (2 * sizeof(int4) + 2 * sizeof(float) * p.part_floats);
}

template <typename T, int DP, int RW, bool ONE_PAGE = false>
cudaError_t launch_rows(const TreeArgs& a, int ctas, cudaStream_t s) {
  using C = Cfg<DP, RW>;
  const auto kernel = tree_attention_kernel<T, DP, RW, ONE_PAGE>;
  const cudaError_t e = allow_smem<tree_attention_kernel<T, DP, RW, ONE_PAGE>>(C::BYTES);
  return e != cudaSuccess ? e : launch_ex(kernel, dim3(ctas), dim3(C::THREADS), C::BYTES, s, 1, a);
}

// The kernel of the plan, then the join.
template <typename T, int DP>
cudaError_t launch(const Plan& p, const TreeArgs& a, int dtype, int ctas, cudaStream_t s) {
  const auto join = [&](auto m, auto tc) {
    // at most one joined tile per run and tile of rows; a thread for 4 columns of a row, up to some 16 blocks per SM
    const long long most = static_cast<long long>(a.max_new) * a.group;  // rows that share a key head
    const long long tiles = static_cast<long long>(a.n_req) * a.cache.heads * ((most + a.tile_rows - 1) / a.tile_rows);
    const bool search = 4 * tiles < ctas;
    const int x = search ? static_cast<int>(tiles) : ctas, rows = static_cast<int>(std::min<long long>(a.tile_rows, most));
    const int elements = p.tc ? (rows + 7) / 8 * 2 * DP : rows * (DP / 4);
    const int blocks = ctas > 8 * x ? (elements + 31) / 32 : (elements + 255) / 256;  // (many parts: 32 elements each)
    const int y = std::max(1, std::min(blocks, 8 * ctas / x));
    return launch_ex(tree_join_kernel<T, DP, decltype(m)::value, decltype(tc)::value>, dim3(x, y), dim3(256), 0, s, 1, a, ctas, search);
  };
  cudaError_t e;
  if (p.tc) {
    e = launch_tree_attention_tc(a, dtype, DP, ctas, s);
    return e != cudaSuccess ? e : join(std::integral_constant<int, 128>{}, std::true_type{});
  }
  e = p.rw == 1   ? (a.cache.page_shift >= 4 ? launch_rows<T, DP, 1, true>(a, ctas, s) : launch_rows<T, DP, 1>(a, ctas, s))
      : p.rw == 2 ? launch_rows<T, DP, 2>(a, ctas, s)
      : p.rw == 4 ? launch_rows<T, DP, 4>(a, ctas, s)
                  : launch_rows<T, DP, 8>(a, ctas, s);
  if (e != cudaSuccess) return e;
  return p.rw == 1   ? join(std::integral_constant<int, 16>{}, std::false_type{})
         : p.rw == 2 ? join(std::integral_constant<int, 32>{}, std::false_type{})
         : p.rw == 4 ? join(std::integral_constant<int, 64>{}, std::false_type{})
                     : join(std::integral_constant<int, 128>{}, std::false_type{});
}

}  // namespace
}  // namespace ivit

extern "C" size_t ivit_tree_attention_workspace(const ivit_attention_config* cfg, const ivit_cache_layout* cache) {
  return cfg && cache && ivit::valid(*cfg, *cache) ? ivit::workspace_of(ivit::plan(*cfg, *cache)) : 0;
}

extern "C" int ivit_tree_attention(const ivit_attention_config* cfg, const ivit_cache_layout* cache, int32_t n_rows,
                                   const void* q_dev, int64_t q_stride, const void* k_new_dev, int64_t k_new_stride,
                                   const void* v_new_dev, int64_t v_new_stride, const void* k_cache_dev,
                                   const void* v_cache_dev, const int32_t* table_dev, const int32_t* len_dev,
                                   const int32_t* cu_rows_dev, const uint32_t* mask_dev, void* out_dev, int64_t out_stride,
                                   float* lse_dev, void* workspace_dev, size_t workspace_bytes, void* stream) {
  using namespace ivit;
  if (!cfg || !cache || n_rows < 0)
    return fail(IVIT_ERR_ARG, "ivit_tree_attention: null configuration or a negative row count");
  if (!valid(*cfg, *cache))
    return fail(IVIT_ERR_SHAPE,
                "ivit_tree_attention: need 1..4096 requests, heads up to 256 and a multiple of the cache's, head_dim a "
                "multiple of 8 up to 256, max_pages * page_size below 2^31 - 2^20, max_new 1..65536, a mask mode (trees "
                "with 1..32768 mask words), scale > 0 and a "
                "supported cache layout");
  if (n_rows == 0) return IVIT_OK;
  if (!q_dev || !k_new_dev || !v_new_dev || !k_cache_dev || !v_cache_dev || !table_dev || !len_dev || !cu_rows_dev ||
      !out_dev || !workspace_dev || (cfg->mask_mode == IVIT_MASK_TREE && !mask_dev))
    return fail(IVIT_ERR_ARG, "ivit_tree_attention: null pointer");
  if ((q_stride | k_new_stride | v_new_stride | out_stride) & 7 || q_stride <= 0 || k_new_stride <= 0 || v_new_stride <= 0 ||
      out_stride <= 0)
    return fail(IVIT_ERR_ARG, "ivit_tree_attention: row strides must be positive multiples of 8 elements");
  if (!all_aligned({q_dev, k_new_dev, v_new_dev, k_cache_dev, v_cache_dev, out_dev, workspace_dev}, 16) ||
      !all_aligned({table_dev, len_dev, cu_rows_dev, mask_dev, lse_dev}, 4))
    return fail(IVIT_ERR_ARG, "ivit_tree_attention: arrays must be 16-byte aligned (table, lengths, offsets, mask and lse 4)");
  const Plan p = plan(*cfg, *cache);
  if (workspace_bytes < workspace_of(p)) return fail(IVIT_ERR_ARG, "ivit_tree_attention: the workspace is too small");
  const int sms = sm_count();
  if (sms <= 0) return fail(IVIT_ERR_CUDA, "ivit_tree_attention: no CUDA device");
  TreeArgs a = {};
  a.q = q_dev;
  a.k_new = k_new_dev;
  a.v_new = v_new_dev;
  a.k_cache = k_cache_dev;
  a.v_cache = v_cache_dev;
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
  a.cache = paged(*cache);
  a.n_req = cfg->n_req;
  a.n_rows = n_rows;
  a.heads = cfg->heads;
  a.group = cfg->heads / cache->kv_heads;
  a.max_pages = cfg->max_pages;
  a.max_new = cfg->max_new;
  a.mask_mode = cfg->mask_mode;
  a.mask_words = cfg->mask_words;
  a.scale_log2 = cfg->scale * 1.4426950408889634f;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  // whole runs of all key heads, at least one (more CTAs than fit at a time wait for a place, not for each other)
  const int ctas = std::max(1, p.ctas_per_sm * std::min(TREE_MAX_SMS, sms) / cache->kv_heads) * cache->kv_heads;
  a.tile_rows = p.tile_rows;
  a.err = static_cast<int*>(workspace_dev);
  a.joins = static_cast<int4*>(workspace_dev) + 1;
  a.parts = reinterpret_cast<float*>(a.joins + 2 * p.ctas_per_sm * TREE_MAX_SMS);
  const auto width = [&](auto type) {
    using T = decltype(type);
    return p.dp == 64    ? launch<T, 64>(p, a, cache->dtype, ctas, s)
           : p.dp == 80  ? launch<T, 80>(p, a, cache->dtype, ctas, s)
           : p.dp == 96  ? launch<T, 96>(p, a, cache->dtype, ctas, s)
           : p.dp == 128 ? launch<T, 128>(p, a, cache->dtype, ctas, s)
                         : launch<T, 256>(p, a, cache->dtype, ctas, s);
  };
  const cudaError_t e = cache->dtype == IVIT_BF16 ? width(bf16{}) : width(half{});
  return e == cudaSuccess ? IVIT_OK : fail_cuda(e);
}
