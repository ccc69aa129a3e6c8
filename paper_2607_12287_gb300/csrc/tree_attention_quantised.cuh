// New rows of every request over its cached tokens, held in 8 bits, and over each other (ivit_tree_attention_quantised):
//
//   o = sum_j p_j v_j / sum_j p_j,  p_j = exp(scale q.k_j - m),  k_j = a_j s_j,  v_j = b_j t_j  for cached keys
//
// with e4m3 codes a_j, b_j and the scales s_j, t_j of their blocks.  The codes enter the products as fp16 values (exact; mma.sync of
// e4m3 itself is no option: it takes 37 cycles of a quarter SM for 16 x 8 x 32, two of fp16 16 and the conversions): s_j multiplies
// the score, t_j the probability, p'_j = 2^(y_j - m), y_j = s_j (q.a_j) c + log2 t_j, which stays within fp16 whatever the
// blocks' scales are, for m is the running maximum of y; the sum has p'_j / t_j.  Queries in bf16 enter as fp16 times a power of two
// that puts a row's largest value at 2^14 (exact but for values 2^-28 of it and less).  p' is rounded to fp16 for bf16 rows,
// 2^-12 of each and an eighth of what their own rounding is, and has two terms for fp16 rows.
//
// The work is cut as in tree_attention.cu, whose run, part and join it shares: tiles of 8 or 16 rows (new row x head of the
// group), 128 keys at a time, first the cached tokens, then the new rows; 32 keys of a tile belong to each of the four warps, which
// walk on without barriers.  Rows are columns of the products: S^T = K q^T, O^T = V^T P^T.  The order of a head's values
// in a product is free, so a lane reads 16 consecutive codes of a key in one load; of V, transposed loads give two values of two
// tokens, of which a byte permutation and two conversions make an operand.  New rows are few and stay in their own type, read from
// global memory, in a loop of their own behind that of the cached keys.
//
// Bound: latency and instructions (32 requests of up to 16384 tokens, 32 + 8 heads of 128, 106 us: 5240 GB/s of 128 bytes a
// key and head; 750 warp instructions to 32 keys, 44 % issue at 12 warps an SM).  Rows as columns halve the products and the outputs'
// registers of a step of 8 rows (153 -> 135 us); two CTAs an SM with three stages were slower than three with two (124 and 110), heads that
// lie together in a row read by one CTA gave nothing (one key head and eight are alike).  Others, us: 16 + 4 heads of 64 39, of 256
// 144, 16 heads of 80 172, of 72 228 (8-byte halves of their pieces), blocks of 8 tokens instead of 16 117; their floors at the
// copy rate are 20.5, 82, 102 and 92: narrow heads have nearly the same instructions to 32 keys, heads of 256 one CTA of four warps an SM.
#pragma once

#include <algorithm>
#include <type_traits>

#include "quantised.cuh"
#include "tree_join.cuh"

namespace ivit {

struct QuantisedArgs : TreeArgs {    // scale_log2 is 1: running maxima are those of y
  const float *k_scale, *v_scale;
  float score_log2;                  // scale * log2(e)
  int block_shift;
  bool wide;                         // copies of 16 bytes
  bool window;                       // ... of heads of 72 or 88: of the 16-byte pieces that a head lies in
};

namespace {

constexpr int TK = 128, WARPS = 4, WK = TK / WARPS, THREADS = 32 * WARPS;

struct QuantisedKeys {
  static constexpr int LEAST = 1;
  static __device__ __forceinline__ int cached(const TreeRequest& r) { return (r.len + TK - 1) / TK; }
  static __device__ __forceinline__ int tiles(const TreeRequest& r) { return cached(r) + (r.n + TK - 1) / TK; }
};

constexpr int MOST_DP = 128;  // of tiles of 16 rows, whose outputs and queries take 7 / 8 DP registers

// Heads of up to DP values, tiles of 8 NR rows.
template <int DP, int NR>
struct Cfg {
  static constexpr int M = 8 * NR;
  static constexpr bool PADDED = DP == 80 || DP == 96;
  static constexpr int ROW = DP == 96 ? 112 : DP;             // bytes of a row of codes: odd numbers of 16-byte pieces if padded
  static constexpr int PIECES = DP / 16, TILE = TK * ROW;
  static constexpr int CTAS = DP > 128 ? 1 : NR == 2 ? (DP <= 64 ? 3 : 2) : DP <= 64 ? 4 : 3;  // per SM
  static constexpr int STAGES = DP <= 80 || DP > 128 || (DP <= 96 && CTAS == 2) ? 3 : 2;
  // a copy of a warp's keys: CP lanes for the pieces of a row, RP rows at a time
  static constexpr int CP = DP <= 64 ? 4 : DP <= 128 ? 8 : 16, RP = 32 / CP, COPIES = WK / RP;
  static constexpr int FULL = DP / 64, TAIL = DP % 64, STEPS = DP / 16;  // of the product, of 16 values
  static constexpr int MEET = DP + 4;                          // floats of a row where the warps meet
  static constexpr int OFF_SCALES = STAGES * 2 * TILE;         // [stage][K, V][key]
  static constexpr int OFF_MEET = OFF_SCALES + STAGES * 2 * TK * 4;  // [row][MEET] fp32
  static constexpr int OFF_ML = OFF_MEET + M * MEET * 4;       // [warp][row] maximum and sum
  static constexpr int BYTES = OFF_ML + WARPS * M * 8;
  static constexpr int PART = tree_part_floats(M, DP);
  static_assert(TREE_MAX_REQ * 8 <= OFF_SCALES, "the units before each request");
  static_assert(CTAS * (BYTES + 1024 + 128) <= 228 * 1024, "shared memory of an SM");
};

// Shared-memory offset of 16-byte piece c of a row of codes.  K: a quarter of a warp reads 64 bytes of two rows.  V: ldmatrix
// reads 16 bytes of eight.
template <int DP, bool V>
__device__ __forceinline__ uint32_t piece(int row, int c) {
  using C = Cfg<DP, 1>;
  const int turned = C::PADDED ? c : DP == 64 ? c ^ (row >> 1 & 3) : V ? c ^ (row & 7) : c ^ ((row & 1) << 2);
  return row * C::ROW + (turned << 4);
}

// Which of the 32 new rows from j0 (a multiple of 32) on new row `node` of the request sees (bit j: row j0 + j).
__device__ __forceinline__ uint32_t seen(const TreeArgs& a, const TreeRequest& r, int node, int j0) {
  const int n = (a.mask_mode == IVIT_MASK_CAUSAL ? min(node + 1, r.n) : r.n) - j0;
  const uint32_t bits = n >= 32 ? 0xffffffffu : n > 0 ? (1u << n) - 1 : 0u;
  if (a.mask_mode != IVIT_MASK_TREE) return bits;
  const int w = j0 >> 5;
  return w < a.mask_words ? bits & a.mask[static_cast<size_t>(r.row0 + node) * a.mask_words + w] : 0u;
}

// An 8 x 8 matrix of 16-bit values, of which lane 4 i + j has values 2 j and 2 j + 1 of row i, turned over.
__device__ __forceinline__ uint32_t transposed8x8(uint32_t x) {
  uint32_t y;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}

template <typename T>
__device__ __forceinline__ bool odd16(uint32_t half_word) {  // infinite or not a number
  constexpr uint32_t e = std::is_same<T, bf16>::value ? 0x7f80u : 0x7c00u;
  return (half_word & e) == e;
}

// A block's scale; one that is not positive and finite counts as 0 for keys, and as 2^-80 for values (as good as 0, and the sum of
// 2^31 probabilities over it stays below 2^127).  Bits of a positive, normal one: 2^23 .. 254 * 2^23 (2^127 counts as none).
__device__ __forceinline__ float key_scale(float x) {
  return static_cast<unsigned>(__float_as_int(x)) - 0x00800000u < 0x7e800000u ? x : 0.f;
}
__device__ __forceinline__ void value_scale(float x, float& log2_of, float& inverse) {
  const int b = __float_as_int(x);
  const bool power = !(b & 0x7fffff), none = b < 0x00800000 || b >= 0x7f000000;
  log2_of = none ? -80.f : power ? static_cast<float>((b >> 23) - 127) : __log2f(x);
  inverse = none ? __int_as_float((80 + 127) << 23) : power ? __int_as_float(0x7f000000 - b) : __fdividef(1.f, x);
}

// ONE_BLOCK: 16 keys of a warp, of whose 32 there are two such halves, have their page and their scales in common.
template <typename T, int DP, int NR, bool ONE_BLOCK>
__global__ void __launch_bounds__(THREADS, Cfg<DP, NR>::CTAS) tree_attention_quantised_kernel(const QuantisedArgs a) {
  using C = Cfg<DP, NR>;
  constexpr unsigned ALL = 0xffffffffu;
  constexpr int M = C::M, STAGES = C::STAGES, COPIES = C::COPIES, RP = C::RP;
  constexpr bool BF16 = std::is_same<T, bf16>::value;
  constexpr int PT = BF16 ? 1 : 2;  // terms of probabilities
  extern __shared__ __align__(128) uint8_t sm[];
  const uint32_t sb = smem_u32(sm);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, t = lane & 3;
  const int dim = a.cache.dim;
  pdl_wait();
  pdl_launch_dependents();

  if (blockIdx.x == 0 && tid == 0) *a.err = 0;  // (nothing here waits on a barrier that could fail)
  TreeRun<QuantisedKeys> run{};
  if (!run.find<THREADS>(a, reinterpret_cast<unsigned long long*>(sm))) return;
  TreePlace<QuantisedKeys> load = run.at, at = run.at;
  const int units = static_cast<int>(run.hi - run.lo);
  // Where a head begins in a row of codes: heads of 72 or 88 bytes lie 0 or 8 bytes behind a 16-byte boundary, and stay so (8-byte
  // copies took 310 us instead of 227 for 32 requests of up to 16384 tokens, 16 heads of 72).
  const int shift = C::PADDED && a.window ? load.head * a.cache.head_stride & 15 : 0;
  if (dim < DP) {
    // bytes beside a head's are zero for good: no copy touches them
    for (int x = tid; x < STAGES * 2 * TK * (DP / 8); x += THREADS) {
      const int row = x / (DP / 8), d = 8 * (x - row * (DP / 8)), key = row & (TK - 1), tile = row / TK;
      if (d >= shift && d < shift + dim) continue;
      *reinterpret_cast<uint2*>(sm + tile * C::TILE + (tile & 1 ? piece<DP, true>(key, d >> 4) : piece<DP, false>(key, d >> 4)) + (d & 8)) =
          make_uint2(0, 0);
    }
  }

  // A copy's part of this thread: piece cp of the rows r0, r0 + RP, ... of the warp's.
  const int cp = lane % C::CP, r0 = warp * WK + lane / C::CP, page_mask = (1 << a.cache.page_shift) - 1;
  const bool first = 16 * cp >= shift, second = 16 * cp + 8 < shift + dim;  // (halves of the piece that are the head's)
  const bool copies = 16 * cp < shift + dim;
  const uint32_t k_to = sb + piece<DP, false>(r0, cp), v_to = piece<DP, true>(r0, cp);
  const auto v_place = [&](int x) { return sb + C::TILE + (C::PADDED || DP == 64 ? v_to : v_to ^ ((x * RP & 7) << 4)) + x * RP * C::ROW; };
  const uint8_t* const k_from = static_cast<const uint8_t*>(a.k_cache) + load.head * a.cache.head_stride - shift + 16 * cp;
  const uint8_t* const v_from = static_cast<const uint8_t*>(a.v_cache) + load.head * a.cache.head_stride - shift + 16 * cp;
  // Scales: lane l's are those of the warp's key l (of common ones, keys 0 and 16).
  const uint32_t scale_to = sb + C::OFF_SCALES + (warp * WK + lane) * 4;
  // The pages of the tile at `load`, of those rows (of the two halves), and of the lane's scale; kept a tile ahead of the copies.
  constexpr int IDS = ONE_BLOCK ? 2 : COPIES;
  int ids[IDS], scale_id = -1;
  const auto look_up = [&] {
    const int key0 = load.kt * TK;
    if (key0 >= load.r.len) return;  // new rows
    const int* table = a.table + static_cast<size_t>(load.req) * a.max_pages;
    const auto page = [&](int key) { return key < load.r.len ? table[key >> a.cache.page_shift] : -1; };
    if (ONE_BLOCK) {
      ids[0] = page(key0 + warp * WK);
      ids[1] = page(key0 + warp * WK + 16);
    } else {
#pragma unroll
      for (int x = 0; x < IDS; ++x) ids[x] = page(key0 + r0 + x * RP);
      scale_id = page(key0 + warp * WK + lane);
    }
  };
  const auto inside = [&](int id) { return static_cast<unsigned>(id) < static_cast<unsigned>(a.cache.n_pages); };
  const auto copy = [&](int stage) {
    const int key0 = load.kt * TK;
    if (key0 >= load.r.len) return;
    if (!ONE_BLOCK || (lane & 15) == 0) {
      const int key = key0 + warp * WK + lane, id = ONE_BLOCK ? ids[lane >> 4 ? 1 : 0] : scale_id;
      const bool ok = key < load.r.len && inside(id);
      const int block = ok ? ((id << a.cache.page_shift) + (key & page_mask)) >> a.block_shift : 0;
      const long long at = static_cast<long long>(block) * a.cache.heads + load.head;
      copy4(scale_to + 2 * stage * TK * 4, a.k_scale + at, ok);
      copy4(scale_to + (2 * stage + 1) * TK * 4, a.v_scale + at, ok);
    }
    if (!copies) return;
    const uint32_t tile = 2 * stage * C::TILE;
    const auto one = [&](uint32_t to, const uint8_t* from, bool ok) {
      if (a.wide && first && second) {
        copy16(to, from, ok);
      } else if (a.wide) {
        copy8(to + (first ? 0 : 8), from + (first ? 0 : 8), ok);
      } else {
        copy8(to, from, ok);
        if (second) copy8(to + 8, from + 8, ok);
      }
    };
    if (ONE_BLOCK && a.wide && key0 + TK <= load.r.len) {  // nearly all
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        const bool ok = inside(ids[half]);
        const long long step = ok ? RP * a.cache.token_stride : 0;
        const long long off = ok ? ids[half] * a.cache.page_stride + ((key0 + r0 + 16 * half) & page_mask) * a.cache.token_stride : 0;
        const uint8_t *k = k_from + off, *v = v_from + off;
#pragma unroll
        for (int x = half * (COPIES / 2); x < (half + 1) * (COPIES / 2); ++x, k += step, v += step) {
          if constexpr (C::PADDED) {
            one(tile + k_to + x * RP * C::ROW, k, ok);
            one(tile + v_place(x), v, ok);
          } else {
            copy16(tile + k_to + x * RP * C::ROW, k, ok);
            copy16(tile + v_place(x), v, ok);
          }
        }
      }
      return;
    }
#pragma unroll
    for (int x = 0; x < COPIES; ++x) {
      const int key = key0 + r0 + x * RP, id = ids[ONE_BLOCK ? 2 * x / COPIES : x];
      const bool ok = key < load.r.len && inside(id);
      const long long off = ok ? id * a.cache.page_stride + (key & page_mask) * a.cache.token_stride : 0;
      one(tile + k_to + x * RP * C::ROW, k_from + off, ok);
      one(tile + v_place(x), v_from + off, ok);
    }
  };

  int loaded = 0;
  look_up();
  const auto fill = [&](int stage) {  // the next tile's copies, if there is one
    if (loaded < units) {
      copy(stage);
      load.next(a);
      if (++loaded < units) look_up();
    }
    copies_commit();
  };
  __syncthreads();  // (the scratch of the search is free, the bytes past a head's are clear)
#pragma unroll 1
  for (int s = 0; s < STAGES - 1; ++s) fill(s);

  // First of the four values of a head that the lane has in a step of the product with cached keys.
  const auto value = [&](int s) {
    return s < 4 * C::FULL ? 64 * (s >> 2) + 16 * t + 4 * (s & 3) : 64 * C::FULL + (C::TAIL == 32 ? 8 * t + 4 * (s & 1) : 4 * t);
  };
  // Rows of the tile are columns of the products: S^T = K q^T with 16 keys (of the lane: g and g + 8, twice) times 8 rows (2 t and 2 t + 1),
  // O^T = V^T P^T with 16 values of a head (2 g and 2 g + 1) times 8 rows.
  int u = 0;  // units done
#pragma unroll 1
  while (u < units) {
    // A segment: consecutive key tiles [at.kt, at.kt + tiles) of one tile of rows, cached ones in front.
    const int tiles = min(at.nkt - at.kt, units - u), cached = QuantisedKeys::cached(at.r), n_old = max(0, min(tiles, cached - at.kt));
    const int rows = min(M, at.r.n * a.group - at.rt * M);
    const auto node_of = [&](int row) { return (at.rt * M + row) / a.group; };  // new row of a row of the tile
    const auto query = [&](int row) {
      const int x = at.rt * M + row, n = x / a.group;
      return static_cast<const T*>(a.q) + (at.r.row0 + n) * a.q_stride + static_cast<long long>(at.head * a.group + x - n * a.group) * dim;
    };
    float o[NR][C::PIECES][4], m[NR][2], l[NR][2];
#pragma unroll
    for (int h = 0; h < NR; ++h) {
      m[h][0] = m[h][1] = -INFINITY;
      l[h][0] = l[h][1] = 0.f;
#pragma unroll
      for (int c = 0; c < C::PIECES; ++c)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[h][c][e] = 0.f;
    }

    // Scores (log2 units, -inf where a key is not seen; of keys g and g + 8 of 16 N keys times rows 2 t, 2 t + 1) to probabilities
    // against the reference maximum, which are added to l times iv.
    const auto probabilities = [&](auto& s, const auto& iv) {
      constexpr int N = std::extent<typename std::remove_reference<decltype(s)>::type>::value;
      bool grow = false;
#pragma unroll
      for (int i = 0; i < N; ++i)
#pragma unroll
        for (int h = 0; h < NR; ++h)
#pragma unroll
          for (int e = 0; e < 4; ++e) grow |= s[i][h][e] - m[h][e & 1] > TREE_GROWTH;
      if (__any_sync(ALL, grow)) {
#pragma unroll
        for (int h = 0; h < NR; ++h) {
          float2 alpha;
#pragma unroll
          for (int r = 0; r < 2; ++r) {
            float mx = fmaxf(s[0][h][r], s[0][h][2 + r]);
            if (N == 2) mx = fmaxf(mx, fmaxf(s[N - 1][h][r], s[N - 1][h][2 + r]));
#pragma unroll
            for (int x = 4; x < 32; x <<= 1) mx = fmaxf(mx, __shfl_xor_sync(ALL, mx, x));
            const float top = fmaxf(m[h][r], mx), f = top == -INFINITY ? 1.f : ex2(m[h][r] - top);
            (r ? alpha.y : alpha.x) = f;
            m[h][r] = top;
            l[h][r] *= f;
          }
#pragma unroll
          for (int c = 0; c < C::PIECES; ++c)
#pragma unroll
            for (int e = 0; e < 4; e += 2) {
              const float2 y = mul_f32x2(make_float2(o[h][c][e], o[h][c][e + 1]), alpha);
              o[h][c][e] = y.x;
              o[h][c][e + 1] = y.y;
            }
        }
      }
#pragma unroll
      for (int h = 0; h < NR; ++h)
#pragma unroll
        for (int r = 0; r < 2; ++r) {
          const float mo = TREE_SHIFT - (m[h][r] == -INFINITY ? 0.f : m[h][r]);  // (nothing seen so far: P = 0)
#pragma unroll
          for (int i = 0; i < N; ++i)
#pragma unroll
            for (int e = r; e < 4; e += 2) {
              s[i][h][e] = ex2(s[i][h][e] + mo);
              l[h][r] = fmaf(s[i][h][e], iv[i][e >> 1], l[h][r]);
            }
        }
    };
    // 16-bit terms of the probabilities of 16 keys, as the second operand of O^T = V^T P^T.
    const auto terms = [&](auto type, const float (&s)[4], auto& p) {
      using P = decltype(type);
      constexpr int N = std::extent<typename std::remove_reference<decltype(p)>::type>::value;
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const uint32_t first = pack2<P>(s[2 * e], s[2 * e + 1]);
        p[0][e] = transposed8x8(first);
        if (N == 2) {
          const float2 back = unpack2<P>(first);
          p[N - 1][e] = transposed8x8(pack2<P>(s[2 * e] - back.x, s[2 * e + 1] - back.y));
        }
      }
    };
    const auto step = [&] {  // the next unit's copies have landed, and those of a later one begin
      copies_wait<STAGES - 2>();
      __syncwarp();  // the lanes' copies have landed, and the stage of the tile before is free
      fill((u + STAGES - 1) % STAGES);
    };

    if (n_old > 0) {
      uint32_t q[NR][C::STEPS][2];
      float factor[NR][2];  // of rows 2 t, 2 t + 1
#pragma unroll
      for (int h = 0; h < NR; ++h) {
        const T* from = query(8 * h + g);
        float size = 0.f, mine = a.score_log2;
#pragma unroll
        for (int s = 0; s < C::STEPS; ++s) {
          const int d = value(s) - shift;
          const uint2 w = 8 * h + g < rows && d >= 0 && d < dim ? *reinterpret_cast<const uint2*>(from + d) : make_uint2(0, 0);
          q[h][s][0] = w.x;
          q[h][s][1] = w.y;
        }
        if (BF16) {
#pragma unroll
          for (int s = 0; s < C::STEPS; ++s)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              const float2 y = unpack2<T>(q[h][s][e]);
              const float y0 = fabsf(y.x), y1 = fabsf(y.y);
              size = fmaxf(size, fmaxf(y0 < INFINITY ? y0 : 0.f, y1 < INFINITY ? y1 : 0.f));
            }
          size = fmaxf(size, __shfl_xor_sync(ALL, size, 1));
          size = fmaxf(size, __shfl_xor_sync(ALL, size, 2));
          const int e2 = max(static_cast<int>(__float_as_uint(size) >> 23) - 127, -100) - 14;  // (-114 .. 113)
          const float up = __int_as_float((127 - e2) << 23);
          mine *= __int_as_float((127 + e2) << 23);
#pragma unroll
          for (int s = 0; s < C::STEPS; ++s)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              const float2 y = unpack2<T>(q[h][s][e]);
              q[h][s][e] = pack2<half>(y.x * up, y.y * up);
            }
        }
        factor[h][0] = __shfl_sync(ALL, mine, 8 * t);  // (row r is that of lanes 4 r ..)
        factor[h][1] = __shfl_sync(ALL, mine, 8 * t + 4);
      }
#pragma unroll 1
      for (int kt = at.kt; kt < at.kt + n_old; ++kt, ++u) {
        const int stage = u % STAGES;
        step();
        const int keys = at.r.len - kt * TK - warp * WK;  // cached tokens from the warp's first on
        if (keys <= 0) continue;
        const uint8_t* k_tile = sm + stage * 2 * C::TILE;
        const float* scales = reinterpret_cast<const float*>(sm + C::OFF_SCALES) + 2 * stage * TK + warp * WK;
        float s[2][NR][4], iv[2][2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {  // 16 keys
          float sum[2][NR][4];  // two, for shorter chains
#pragma unroll
          for (int h = 0; h < NR; ++h)
#pragma unroll
            for (int e = 0; e < 4; ++e) sum[0][h][e] = sum[1][h][e] = 0.f;
          const auto product = [&](int st, uint32_t x, uint32_t y) {  // step st, four codes of keys g and g + 8
            uint32_t k4[4];
            codes_to_half4(x, k4[0], k4[2]);
            codes_to_half4(y, k4[1], k4[3]);
#pragma unroll
            for (int h = 0; h < NR; ++h) mma<half>(sum[st & 1][h], k4, q[h][st][0], q[h][st][1]);
          };
          const int row = warp * WK + 16 * i + g;
#pragma unroll
          for (int c = 0; c < C::FULL; ++c) {
            const uint4 x = *reinterpret_cast<const uint4*>(k_tile + piece<DP, false>(row, 4 * c + t));
            const uint4 y = *reinterpret_cast<const uint4*>(k_tile + piece<DP, false>(row + 8, 4 * c + t));
            product(4 * c, x.x, y.x);
            product(4 * c + 1, x.y, y.y);
            product(4 * c + 2, x.z, y.z);
            product(4 * c + 3, x.w, y.w);
          }
          if constexpr (C::TAIL == 32) {
            const uint2 x = *reinterpret_cast<const uint2*>(k_tile + piece<DP, false>(row, 4 * C::FULL + (t >> 1)) + 8 * (t & 1));
            const uint2 y = *reinterpret_cast<const uint2*>(k_tile + piece<DP, false>(row + 8, 4 * C::FULL + (t >> 1)) + 8 * (t & 1));
            product(C::STEPS - 2, x.x, y.x);
            product(C::STEPS - 1, x.y, y.y);
          }
          if constexpr (C::TAIL == 16)
            product(C::STEPS - 1, *reinterpret_cast<const uint32_t*>(k_tile + piece<DP, false>(row, 4 * C::FULL) + 4 * t),
                    *reinterpret_cast<const uint32_t*>(k_tile + piece<DP, false>(row + 8, 4 * C::FULL) + 4 * t));
          // Scales of keys g, g + 8: of keys, log2 and inverse of values.
          float kf[2], lv[2];
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            if (ONE_BLOCK && e == 1) {
              kf[1] = kf[0], lv[1] = lv[0], iv[i][1] = iv[i][0];
              break;
            }
            const int at_key = 16 * i + (ONE_BLOCK ? 0 : g + 8 * e);
            kf[e] = key_scale(scales[at_key]);
            value_scale(scales[TK + at_key], lv[e], iv[i][e]);
          }
#pragma unroll
          for (int h = 0; h < NR; ++h)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              s[i][h][e] = fmaf(sum[0][h][e] + sum[1][h][e], kf[e >> 1] * factor[h][e & 1], lv[e >> 1]);
            }
        }
        if (keys < WK) {
#pragma unroll
          for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int h = 0; h < NR; ++h)
#pragma unroll
              for (int e = 0; e < 4; ++e)
                if (16 * i + g + 8 * (e >> 1) >= keys) s[i][h][e] = -INFINITY;
        }
        probabilities(s, iv);
        uint32_t p[2][NR][PT][2];
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int h = 0; h < NR; ++h) terms(half{}, s[i][h], p[i][h]);
        const uint32_t v_tile = sb + (2 * stage + 1) * C::TILE;
#pragma unroll
        for (int c = 0; c < C::PIECES; c += 2) {
          const int mine = c + 1 < C::PIECES ? c + (lane >> 4) : c;
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            uint32_t b[4];
            ldmatrix4_trans(b, v_tile + piece<DP, true>(warp * WK + 16 * i + (lane & 15), mine));
#pragma unroll
            for (int d = 0; d < 2; ++d) {
              if (c + d >= C::PIECES) break;
              // (value 2 g of tokens 2 t, 2 t + 1, then value 2 g + 1; of tokens 8 further on)
              uint32_t v4[4];
              codes_to_half4(__byte_perm(b[2 * d], 0, 0x3120), v4[0], v4[1]);
              codes_to_half4(__byte_perm(b[2 * d + 1], 0, 0x3120), v4[2], v4[3]);
#pragma unroll
              for (int h = 0; h < NR; ++h)
#pragma unroll
                for (int x = 0; x < PT; ++x) mma<half>(o[h][c + d], v4, p[i][h][x][0], p[i][h][x][1]);
            }
          }
        }
      }
    }

    // New rows, in their own type, 16 at a time.
#pragma unroll 1
    for (int nt = at.kt + n_old - cached; nt < at.kt + tiles - cached; ++nt, ++u) {
      step();
#pragma unroll 1
      for (int k0 = nt * TK + warp * WK; k0 < min(nt * TK + (warp + 1) * WK, at.r.n); k0 += 16) {
        const int keys = at.r.n - k0;
        float s[1][NR][4] = {};
        const T* const k_new = static_cast<const T*>(a.k_new) + static_cast<long long>(at.r.row0 + k0) * a.k_new_stride + at.head * dim;
        const T* const v_new = static_cast<const T*>(a.v_new) + static_cast<long long>(at.r.row0 + k0) * a.v_new_stride + at.head * dim;
#pragma unroll 2
        for (int st = 0; st < DP / 16; ++st) {  // (unrolled whole, the loads of all steps took the registers of the loop above)
          const int d = 16 * st + 4 * t;
          uint32_t k4[4];
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const uint2 w = g + 8 * e < keys && d < dim ? *reinterpret_cast<const uint2*>(k_new + (g + 8 * e) * a.k_new_stride + d) : make_uint2(0, 0);
            k4[e] = w.x;
            k4[e + 2] = w.y;
          }
#pragma unroll
          for (int h = 0; h < NR; ++h) {
            const uint2 w = 8 * h + g < rows && d < dim ? *reinterpret_cast<const uint2*>(query(8 * h + g) + d) : make_uint2(0, 0);
            mma<T>(s[0][h], k4, w.x, w.y);
          }
        }
#pragma unroll
        for (int h = 0; h < NR; ++h)
#pragma unroll
          for (int r = 0; r < 2; ++r) {
            const int row = 8 * h + 2 * t + r;
            const uint32_t bits = row < rows ? seen(a, at.r, node_of(row), k0 & ~31) >> (k0 & 16) : 0u;
#pragma unroll
            for (int e = r; e < 4; e += 2) s[0][h][e] = bits >> (g + 8 * (e >> 1)) & 1 ? s[0][h][e] * a.score_log2 : -INFINITY;
          }
        const float iv[1][2] = {{1.f, 1.f}};
        probabilities(s, iv);
        uint32_t p[NR][2][2];  // two terms of each
#pragma unroll
        for (int h = 0; h < NR; ++h) terms(T{}, s[0][h], p[h]);
        bool odd = false;
#pragma unroll
        for (int c = 0; c < C::PIECES; ++c) {
          const int d = 16 * c + 2 * g - shift;
          uint32_t w[4];  // tokens 2 t, 2 t + 1, 2 t + 8, 2 t + 9
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int key = 2 * t + (i & 1) + 8 * (i >> 1);
            w[i] = key < keys && d >= 0 && d < dim ? *reinterpret_cast<const uint32_t*>(v_new + key * a.v_new_stride + d) : 0u;
            // Values that are not finite would reach rows that do not see them (0 * NaN): left out here, added below.
            const bool lo = odd16<T>(w[i]), hi = odd16<T>(w[i] >> 16);
            if (lo) w[i] &= 0xffff0000u;
            if (hi) w[i] &= 0x0000ffffu;
            odd |= lo || hi;
          }
          const uint32_t v4[4] = {__byte_perm(w[0], w[1], 0x5410), __byte_perm(w[0], w[1], 0x7632), __byte_perm(w[2], w[3], 0x5410),
                                  __byte_perm(w[2], w[3], 0x7632)};
#pragma unroll
          for (int h = 0; h < NR; ++h)
#pragma unroll
            for (int x = 0; x < 2; ++x) mma<T>(o[h][c], v4, p[h][x][0], p[h][x][1]);
          if (c & 1) asm volatile("" ::: "memory");  // (two loads of values at a time, for the same reason)
        }
        if (__any_sync(ALL, odd)) {
#pragma unroll 1
          for (int k = 0; k < min(keys, 16); ++k)
#pragma unroll
            for (int h = 0; h < NR; ++h)
#pragma unroll
              for (int r = 0; r < 2; ++r) {
                const int row = 8 * h + 2 * t + r;
                if (row >= rows || !(seen(a, at.r, node_of(row), k0 & ~31) >> ((k0 & 16) + k) & 1)) continue;
#pragma unroll
                for (int c = 0; c < C::PIECES; ++c)
                  if (const int d = 16 * c + 2 * g - shift; d >= 0 && d < dim) {
                    const float2 x = unpack2<T>(*reinterpret_cast<const uint32_t*>(v_new + k * a.v_new_stride + d));
                    if (!isfinite(x.x)) o[h][c][r] += x.x;
                    if (!isfinite(x.y)) o[h][c][2 + r] += x.y;
                  }
              }
        }
      }
    }

    // The warps meet: every output against the largest maximum, added up in the order of the warps.
    float2* ml = reinterpret_cast<float2*>(sm + C::OFF_ML);
    float* meet = reinterpret_cast<float*>(sm + C::OFF_MEET);
#pragma unroll
    for (int h = 0; h < NR; ++h)
#pragma unroll
      for (int r = 0; r < 2; ++r) {
#pragma unroll
        for (int x = 4; x < 32; x <<= 1) l[h][r] += __shfl_xor_sync(ALL, l[h][r], x);
        if (g == 0) ml[warp * M + 8 * h + 2 * t + r] = make_float2(m[h][r], l[h][r]);
      }
    __syncthreads();
#pragma unroll
    for (int h = 0; h < NR; ++h)
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        float top = -INFINITY;
#pragma unroll
        for (int w = 0; w < WARPS; ++w) top = fmaxf(top, ml[w * M + 8 * h + 2 * t + r].x);
        const float f = ex2(m[h][r] - (top == -INFINITY ? 0.f : top));
#pragma unroll
        for (int c = 0; c < C::PIECES; ++c) {
          o[h][c][r] *= f;
          o[h][c][2 + r] *= f;
        }
      }
#pragma unroll 1
    for (int w = 0; w < WARPS; ++w) {
      if (warp == w) {
#pragma unroll
        for (int h = 0; h < NR; ++h)
#pragma unroll
          for (int r = 0; r < 2; ++r)
            if (8 * h + 2 * t + r < rows) {
#pragma unroll
              for (int c = 0; c < C::PIECES; ++c) {
                float2* dst = reinterpret_cast<float2*>(meet + (8 * h + 2 * t + r) * C::MEET + 16 * c + 2 * g);
                float2 y = make_float2(o[h][c][r], o[h][c][2 + r]);
                if (w > 0) {
                  const float2 x = *dst;
                  y = make_float2(x.x + y.x, x.y + y.y);
                }
                *dst = y;
              }
            }
      }
      __syncthreads();
    }
    const bool whole = tiles == at.nkt;
    // a part: the first of the run, or the one it ends with
    float* part = a.parts + static_cast<size_t>(2 * blockIdx.x + (u > tiles ? 1 : 0)) * C::PART;
#pragma unroll 1
    for (int e = tid; e < rows * (DP / 4); e += THREADS) {
      const int row = e / (DP / 4), col = e - row * (DP / 4);  // (columns of the output)
      if (4 * col >= dim) continue;
      const float4 y = *reinterpret_cast<const float4*>(meet + row * C::MEET + 4 * col + shift);
      float top = -INFINITY, sum = 0.f;
      float2 of[WARPS];
#pragma unroll
      for (int w = 0; w < WARPS; ++w) {
        of[w] = ml[w * M + row];
        top = fmaxf(top, of[w].x);
      }
#pragma unroll
      for (int w = 0; w < WARPS; ++w) sum += of[w].y * ex2(of[w].x - (top == -INFINITY ? 0.f : top));
      if (whole) {
        const int x = at.rt * M + row, nd = x / a.group, h = at.head * a.group + x - nd * a.group;
        const long long orow = at.r.row0 + nd;
        const float inv = sum == 0.f ? 0.f : 1.f / sum;
        *reinterpret_cast<uint2*>(static_cast<T*>(a.out) + orow * a.out_stride + static_cast<long long>(h) * dim + 4 * col) =
            make_uint2(pack2<T>(y.x * inv, y.y * inv), pack2<T>(y.z * inv, y.w * inv));
        if (a.lse && col == 0) a.lse[orow * a.heads + h] = (top + (log2f(sum) - TREE_SHIFT)) * 0.6931471805599453f;
      } else {
        reinterpret_cast<float4*>(part + row * DP)[col] = y;
        if (col == 0) *reinterpret_cast<float2*>(part + M * DP + 2 * row) = make_float2(top, sum);
      }
    }
    __syncthreads();  // the place of the meeting is free
    if (!whole && at.kt == 0 && tid == 0) run.note_join(a, at, run.lo + u - tiles);
    at.next_rows(a);
  }
}

template <typename T, int DP, int NR>
cudaError_t launch_rows(const QuantisedArgs& a, int ctas, cudaStream_t s) {
  using C = Cfg<DP, NR>;
  const auto kernel = [&](auto one_block) {
    constexpr auto k = tree_attention_quantised_kernel<T, DP, NR, decltype(one_block)::value>;
    const cudaError_t e = allow_smem<k>(C::BYTES);
    return e != cudaSuccess ? e : launch_ex(k, dim3(ctas), dim3(THREADS), C::BYTES, s, 1, a);
  };
  const cudaError_t e = a.block_shift >= 4 ? kernel(std::true_type{}) : kernel(std::false_type{});
  return e != cudaSuccess ? e : launch_tree_join<T, DP, C::M, false>(a, ctas, s);
}

template <typename T>
cudaError_t launch(const QuantisedArgs& a, int dp, int nr, int ctas, cudaStream_t s) {
  const auto width = [&](auto d) {
    constexpr int DP = decltype(d)::value;
    if constexpr (DP <= MOST_DP)
      if (nr == 2) return launch_rows<T, DP, 2>(a, ctas, s);
    return launch_rows<T, DP, 1>(a, ctas, s);
  };
  return dp == 64    ? width(std::integral_constant<int, 64>{})
         : dp == 80  ? width(std::integral_constant<int, 80>{})
         : dp == 96  ? width(std::integral_constant<int, 96>{})
         : dp == 128 ? width(std::integral_constant<int, 128>{})
                     : width(std::integral_constant<int, 256>{});
}

}  // namespace

// The kernel and the join for rows of bf16 and fp16 (a source file each: there are many forms).
cudaError_t launch_tree_attention_quantised_bf16(const QuantisedArgs& a, int dp, int nr, int ctas, cudaStream_t s);
cudaError_t launch_tree_attention_quantised_fp16(const QuantisedArgs& a, int dp, int nr, int ctas, cudaStream_t s);

// The form for many rows per key head (tree_attention_quantised_tc.cu), for groups of up to 128 heads: tiles of tree_tc_rows(group)
// rows, two CTAs per SM (of dp 256 one).
cudaError_t launch_tree_attention_quantised_tc(const QuantisedArgs& a, int dtype, int dp, int ctas, cudaStream_t s);

}  // namespace ivit
