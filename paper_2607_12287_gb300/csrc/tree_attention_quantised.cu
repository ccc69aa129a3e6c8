// New rows of every request over its cached tokens, held in 8 bits, and over each other (ivit_tree_attention_quantised):
//
//   o = sum_j p_j v_j / sum_j p_j,  p_j = exp(scale q.k_j - m),  k_j = a_j s_j,  v_j = b_j t_j  for cached keys
//
// with e4m3 codes a_j, b_j and the scales s_j, t_j of their blocks.  The codes enter the products as they are, as fp16 values (exact):
// s_j multiplies the score, t_j the probability, p'_j = 2^(y_j - m), y_j = s_j (q.a_j) c + log2 t_j, which stays within
// fp16 whatever the blocks' scales are, for m is the running maximum of y; the sum has p'_j / t_j.  Queries in bf16 enter as
// fp16 times a power of two that puts a row's largest value at 2^14 (exact but for values 2^-28 of it and less).
//
// The work is cut as in tree_attention.cu, whose run, part and join it shares: tiles of 16 rows (new row x head of the group), 64 keys
// at a time, first the cached tokens, then the new rows; 16 keys of a tile belong to each of the four warps, which walk on
// without barriers.  A cached tile's codes come by asynchronous copies through a ring in shared memory, 128 bytes a key for
// heads of 128.  The order of a head's values in a product is free, so a lane reads 16 consecutive codes of a key, four steps
// of the product, in one load; of V, a transposed load gives two values of two tokens, which a byte permutation and two conversions
// make operands of two products.  New rows are few and stay in their own type, read from global memory.
#include <algorithm>
#include <type_traits>

#include "quantised.cuh"
#include "tree_join.cuh"

namespace ivit {
namespace {

constexpr int TK = 64, WARPS = 4, WK = TK / WARPS, THREADS = 32 * WARPS;

struct QuantisedArgs : TreeArgs {    // scale_log2 is 1: running maxima are those of y
  const float *k_scale, *v_scale;
  float score_log2;                  // scale * log2(e)
  int block_shift;
  bool wide;                         // copies of 16 bytes
};

struct QuantisedKeys {
  static constexpr int LEAST = 1;
  static __device__ __forceinline__ int cached(const TreeRequest& r) { return (r.len + TK - 1) / TK; }
  static __device__ __forceinline__ int tiles(const TreeRequest& r) { return cached(r) + (r.n + TK - 1) / TK; }
};

__device__ __forceinline__ void copy8(uint32_t dst, const void* src, bool ok) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 8, %2;" ::"r"(dst), "l"(src), "r"(ok ? 8 : 0) : "memory");
}
__device__ __forceinline__ void copy4(uint32_t dst, const void* src, bool ok) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(src), "r"(ok ? 4 : 0) : "memory");
}

// Heads of up to DP values, tiles of 8 NR rows.
template <int DP, int NR>
struct Cfg {
  static constexpr int M = 8 * NR;
  static constexpr bool PADDED = DP == 80 || DP == 96;
  static constexpr int ROW = DP == 96 ? 112 : DP;             // bytes of a row of codes: odd numbers of 16-byte pieces if padded
  static constexpr int PIECES = DP / 16, TILE = TK * ROW;
  static constexpr int CTAS = NR == 1 ? (DP <= 128 ? 4 : 3) : DP <= 64 ? 4 : DP <= 128 ? 3 : 2;  // per SM
  static constexpr int STAGES = DP > 128 ? 2 : DP <= 80 || CTAS == 3 ? 4 : 3;
  // a copy of a warp's keys: CP lanes for the pieces of a row, RP rows at a time
  static constexpr int CP = DP <= 64 ? 4 : DP <= 128 ? 8 : 16, RP = 32 / CP, COPIES = WK / RP;
  static constexpr int STEPS = DP / 16, FULL = DP / 64, TAIL = DP % 64;  // of the product: of 16 values, 64, and what is left
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

// Which of the 64 new rows from j0 on new row `node` of the request sees (bit j: row j0 + j).
__device__ __forceinline__ uint64_t seen(const TreeArgs& a, const TreeRequest& r, int node, int j0) {
  const auto low = [](int n) { return n >= 64 ? ~0ull : n > 0 ? (1ull << n) - 1 : 0ull; };
  if (a.mask_mode == IVIT_MASK_CAUSAL) return low(node + 1 - j0);
  if (a.mask_mode == IVIT_MASK_ALL) return low(r.n - j0);
  const uint32_t* words = a.mask + static_cast<size_t>(r.row0 + node) * a.mask_words;
  const auto word = [&](int w) { return static_cast<uint64_t>(w < a.mask_words ? words[w] : 0u); };
  return (word(j0 >> 5) | word((j0 >> 5) + 1) << 32) & low(r.n - j0);
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

// What the 16 keys of a warp have in common.
enum Common { NOTHING, PAGE, BLOCK };  // BLOCK: their page and their scales

template <typename T, int DP, int NR, Common COMMON>
__global__ void __launch_bounds__(THREADS, Cfg<DP, NR>::CTAS) tree_attention_quantised_kernel(const QuantisedArgs a) {
  using C = Cfg<DP, NR>;
  constexpr unsigned ALL = 0xffffffffu;
  constexpr int M = C::M, STAGES = C::STAGES, COPIES = C::COPIES, RP = C::RP, STEPS = C::STEPS;
  constexpr bool BF16 = std::is_same<T, bf16>::value, ONE_PAGE = COMMON != NOTHING, ONE_BLOCK = COMMON == BLOCK;
  // Probabilities of cached keys are rounded to fp16, 2^-12 of each and an eighth of what bf16 rows' own rounding is; fp16 rows have
  // them as two terms.
  constexpr int TERMS = BF16 ? 1 : 2;
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
  if (dim < DP) {
    // bytes past a head's are zero for good: no copy touches them
    const int words = (DP - dim) / 8;
    for (int x = tid; x < STAGES * 2 * TK * words; x += THREADS) {
      const int row = x / words, d = dim + 8 * (x - row * words), key = row & (TK - 1), tile = row / TK;
      *reinterpret_cast<uint2*>(sm + tile * C::TILE + (tile & 1 ? piece<DP, true>(key, d >> 4) : piece<DP, false>(key, d >> 4)) + (d & 8)) =
          make_uint2(0, 0);
    }
  }

  // A copy's part of this thread: piece cp of the rows r0, r0 + RP, ... of the warp's.
  const int cp = lane % C::CP, r0 = warp * WK + lane / C::CP, page_mask = (1 << a.cache.page_shift) - 1;
  const bool copies = 16 * cp < dim, second = 16 * cp + 8 < dim;  // (the piece, and its second half, are the head's)
  const uint32_t k_to = sb + piece<DP, false>(r0, cp), v_to = piece<DP, true>(r0, cp);
  const auto v_place = [&](int x) { return sb + C::TILE + (C::PADDED || DP == 64 ? v_to : v_to ^ ((x * RP & 7) << 4)) + x * RP * C::ROW; };
  const uint8_t* const k_from = static_cast<const uint8_t*>(a.k_cache) + load.head * a.cache.head_stride + 16 * cp;
  const uint8_t* const v_from = static_cast<const uint8_t*>(a.v_cache) + load.head * a.cache.head_stride + 16 * cp;
  // Scales: of lane l key l % 16 (the common one: 0), of keys or (l >= 16) values.
  const int scale_key = warp * WK + (ONE_BLOCK ? 0 : lane & 15);
  const uint32_t scale_to = sb + C::OFF_SCALES + ((lane >> 4) * TK + scale_key) * 4;
  const float* const scale_from = (lane < 16 ? a.k_scale : a.v_scale) + load.head;
  // The pages of the tile at `load`, of those rows, and of the lane's scale; kept a tile ahead of the copies.
  constexpr int IDS = ONE_PAGE ? 1 : COPIES;
  int ids[IDS], scale_id = -1;
  const auto look_up = [&] {
    const int key0 = load.kt * TK;
    if (key0 >= load.r.len) return;  // new rows
    const int* table = a.table + static_cast<size_t>(load.req) * a.max_pages;
    const auto page = [&](int key) { return key < load.r.len ? table[key >> a.cache.page_shift] : -1; };
    if (ONE_PAGE) {
      ids[0] = page(key0 + warp * WK);
    } else {
#pragma unroll
      for (int x = 0; x < IDS; ++x) ids[x] = page(key0 + r0 + x * RP);
      scale_id = page(key0 + scale_key);
    }
  };
  const auto inside = [&](int id) { return static_cast<unsigned>(id) < static_cast<unsigned>(a.cache.n_pages); };
  const auto copy = [&](int stage) {
    const int key0 = load.kt * TK;
    if (key0 >= load.r.len) return;
    if (!ONE_BLOCK || (lane & 15) == 0) {
      const int key = key0 + scale_key, id = ONE_PAGE ? ids[0] : scale_id;
      const bool ok = key < load.r.len && inside(id);
      const int block = ok ? ((id << a.cache.page_shift) + (key & page_mask)) >> a.block_shift : 0;
      copy4(scale_to + 2 * stage * TK * 4, scale_from + static_cast<long long>(block) * a.cache.heads, ok);
    }
    if (!copies) return;
    const uint32_t tile = 2 * stage * C::TILE;
    const auto both = [&](int x, long long off, bool ok) {
      const uint32_t kd = tile + k_to + x * RP * C::ROW, vd = tile + v_place(x);
      if (a.wide) {
        copy16(kd, k_from + off, ok);
        copy16(vd, v_from + off, ok);
      } else {
        copy8(kd, k_from + off, ok);
        copy8(vd, v_from + off, ok);
        if (second) {
          copy8(kd + 8, k_from + off + 8, ok);
          copy8(vd + 8, v_from + off + 8, ok);
        }
      }
    };
    if (ONE_PAGE && key0 + TK <= load.r.len) {  // nearly all
      const bool ok = inside(ids[0]);
      const long long step = ok ? RP * a.cache.token_stride : 0;
      long long off = ok ? ids[0] * a.cache.page_stride + ((key0 + r0) & page_mask) * a.cache.token_stride : 0;
#pragma unroll
      for (int x = 0; x < COPIES; ++x) {
        both(x, off, ok);
        off += step;
      }
      return;
    }
#pragma unroll
    for (int x = 0; x < COPIES; ++x) {
      const int key = key0 + r0 + x * RP, id = ids[ONE_PAGE ? 0 : x];
      const bool ok = key < load.r.len && inside(id);
      both(x, ok ? id * a.cache.page_stride + (key & page_mask) * a.cache.token_stride : 0, ok);
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

  // First of the four values of a head that the lane has in step s of the product with K.
  const auto value = [&](int s) {
    return s < 4 * C::FULL ? 64 * (s >> 2) + 16 * t + 4 * (s & 3) : 64 * C::FULL + (C::TAIL == 32 ? 8 * t + 4 * (s & 1) : 4 * t);
  };
  // Rows of the tile are columns of the products: S^T = K q^T with 16 keys (of the lane: g and g + 8) times 8 rows (2 t and 2 t + 1),
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

    // Scores (log2 units, -inf where a key is not seen; of keys g, g + 8 times rows 2 t, 2 t + 1) to probabilities against the reference
    // maximum, which are added to l times iv.
    const auto probabilities = [&](float (&s)[NR][4], const float (&iv)[2]) {
      bool grow = false;
#pragma unroll
      for (int h = 0; h < NR; ++h)
#pragma unroll
        for (int e = 0; e < 4; ++e) grow |= s[h][e] - m[h][e & 1] > TREE_GROWTH;
      if (__any_sync(ALL, grow)) {
#pragma unroll
        for (int h = 0; h < NR; ++h)
#pragma unroll
          for (int r = 0; r < 2; ++r) {
            float mx = fmaxf(s[h][r], s[h][2 + r]);
#pragma unroll
            for (int x = 4; x < 32; x <<= 1) mx = fmaxf(mx, __shfl_xor_sync(ALL, mx, x));
            if (!(mx > m[h][r])) continue;
            const float alpha = ex2(m[h][r] - mx);
            m[h][r] = mx;
            l[h][r] *= alpha;
#pragma unroll
            for (int c = 0; c < C::PIECES; ++c) {
              o[h][c][r] *= alpha;
              o[h][c][2 + r] *= alpha;
            }
          }
      }
#pragma unroll
      for (int h = 0; h < NR; ++h)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float mo = TREE_SHIFT - (m[h][e & 1] == -INFINITY ? 0.f : m[h][e & 1]);  // (nothing seen so far: P = 0)
          s[h][e] = ex2(s[h][e] + mo);
          l[h][e & 1] = fmaf(s[h][e], iv[e >> 1], l[h][e & 1]);
        }
    };
    // N 16-bit terms of each, as the second operand of O^T = V^T P^T.
    const auto terms = [&](auto type, const float (&s)[4], auto& p) {
      using P = decltype(type);
      constexpr int N = std::extent<typename std::remove_reference<decltype(p)>::type>::value;
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const uint32_t first = pack2<P>(s[2 * e], s[2 * e + 1]);
        p[0][e] = transposed8x8(first);
        if (N == 2) {
          const float2 h = unpack2<P>(first);
          p[N - 1][e] = transposed8x8(pack2<P>(s[2 * e] - h.x, s[2 * e + 1] - h.y));
        }
      }
    };
    const auto step = [&] {  // the next unit's copies have landed, and those of a later one begin
      copies_wait<STAGES - 2>();
      __syncwarp();  // the lanes' copies have landed, and the stage of the tile before is free
      fill((u + STAGES - 1) % STAGES);
    };

    if (n_old > 0) {
      uint32_t q[NR][STEPS][2];
      float factor[NR][2];  // of rows 2 t, 2 t + 1
#pragma unroll
      for (int h = 0; h < NR; ++h) {
        const T* from = query(8 * h + g);
#pragma unroll
        for (int s = 0; s < STEPS; ++s) {
          const int d = value(s);
          const uint2 w = 8 * h + g < rows && d < dim ? *reinterpret_cast<const uint2*>(from + d) : make_uint2(0, 0);
          q[h][s][0] = w.x;
          q[h][s][1] = w.y;
        }
        float mine = a.score_log2;
        if (BF16) {
          float size = 0.f;
#pragma unroll
          for (int s = 0; s < STEPS; ++s)
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
          for (int s = 0; s < STEPS; ++s)
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
        const uint8_t* k_row = sm + stage * 2 * C::TILE;
        // two sums of every product, for shorter chains
        float s[NR][4], s2[NR][4];
#pragma unroll
        for (int h = 0; h < NR; ++h)
#pragma unroll
          for (int e = 0; e < 4; ++e) s[h][e] = s2[h][e] = 0.f;
        const auto product = [&](int st, uint32_t w0, uint32_t w1) {  // step st, four codes of keys g and g + 8
          uint32_t k4[4];
          codes_to_half4(w0, k4[0], k4[2]);
          codes_to_half4(w1, k4[1], k4[3]);
#pragma unroll
          for (int h = 0; h < NR; ++h) mma<half>(st & 1 ? s2[h] : s[h], k4, q[h][st][0], q[h][st][1]);
        };
        const int row = warp * WK + g;
#pragma unroll
        for (int c = 0; c < C::FULL; ++c) {
          const uint4 x = *reinterpret_cast<const uint4*>(k_row + piece<DP, false>(row, 4 * c + t));
          const uint4 y = *reinterpret_cast<const uint4*>(k_row + piece<DP, false>(row + 8, 4 * c + t));
          product(4 * c, x.x, y.x);
          product(4 * c + 1, x.y, y.y);
          product(4 * c + 2, x.z, y.z);
          product(4 * c + 3, x.w, y.w);
        }
        if constexpr (C::TAIL == 32) {
          const uint2 x = *reinterpret_cast<const uint2*>(k_row + piece<DP, false>(row, 4 * C::FULL + (t >> 1)) + 8 * (t & 1));
          const uint2 y = *reinterpret_cast<const uint2*>(k_row + piece<DP, false>(row + 8, 4 * C::FULL + (t >> 1)) + 8 * (t & 1));
          product(STEPS - 2, x.x, y.x);
          product(STEPS - 1, x.y, y.y);
        }
        if constexpr (C::TAIL == 16)
          product(STEPS - 1, *reinterpret_cast<const uint32_t*>(k_row + piece<DP, false>(row, 4 * C::FULL) + 4 * t),
                  *reinterpret_cast<const uint32_t*>(k_row + piece<DP, false>(row + 8, 4 * C::FULL) + 4 * t));
        // Scales of keys g, g + 8: of keys, log2 and inverse of values (one that is none, or out of range: the values are as good as 0).
        const float* scales = reinterpret_cast<const float*>(sm + C::OFF_SCALES) + 2 * stage * TK + warp * WK;
        float kf[2], lv[2], iv[2];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          if (ONE_BLOCK && e == 1) {
            kf[1] = kf[0], lv[1] = lv[0], iv[1] = iv[0];
            break;
          }
          const int at_key = ONE_BLOCK ? 0 : g + 8 * e;
          kf[e] = scales[at_key];
          const float x = scales[TK + at_key];
          const int b = __float_as_int(x);
          const bool power = !(b & 0x7fffff), none = b < 0x00800000 || b >= 0x7f000000;
          lv[e] = none ? -100.f : power ? static_cast<float>((b >> 23) - 127) : __log2f(x);
          iv[e] = none ? __int_as_float((100 + 127) << 23) : power ? __int_as_float(0x7f000000 - b) : __fdividef(1.f, x);
        }
#pragma unroll
        for (int h = 0; h < NR; ++h)
#pragma unroll
          for (int e = 0; e < 4; ++e) s[h][e] = fmaf(s[h][e] + s2[h][e], kf[e >> 1] * factor[h][e & 1], lv[e >> 1]);
        if (keys < WK) {
#pragma unroll
          for (int h = 0; h < NR; ++h)
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if (g + 8 * (e >> 1) >= keys) s[h][e] = -INFINITY;
        }
        probabilities(s, iv);
        uint32_t p[NR][TERMS][2];
#pragma unroll
        for (int h = 0; h < NR; ++h) terms(half{}, s[h], p[h]);
#pragma unroll
        for (int c = 0; c < C::PIECES; c += 2) {
          const int mine = c + 1 < C::PIECES ? c + (lane >> 4) : c;
          uint32_t b[4];
          ldmatrix4_trans(b, sb + (2 * stage + 1) * C::TILE + piece<DP, true>(warp * WK + (lane & 15), mine));
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            if (c + i >= C::PIECES) break;
            // (value 2 g of tokens 2 t, 2 t + 1, then value 2 g + 1; of tokens 8 further on)
            uint32_t v4[4];
            codes_to_half4(__byte_perm(b[2 * i], 0, 0x3120), v4[0], v4[1]);
            codes_to_half4(__byte_perm(b[2 * i + 1], 0, 0x3120), v4[2], v4[3]);
#pragma unroll
            for (int h = 0; h < NR; ++h)
#pragma unroll
              for (int x = 0; x < TERMS; ++x) mma<half>(o[h][c + i], v4, p[h][x][0], p[h][x][1]);
          }
        }
      }
    }

    // New rows, in their own type.
#pragma unroll 1
    for (int nt = at.kt + n_old - cached; nt < at.kt + tiles - cached; ++nt, ++u) {
      step();
      const int k0 = nt * TK + warp * WK, keys = at.r.n - k0;  // first new row of the warp's
      if (keys <= 0) continue;
      float s[NR][4] = {};
      const float iv[2] = {1.f, 1.f};
      const T* const k_new = static_cast<const T*>(a.k_new) + static_cast<long long>(at.r.row0 + k0) * a.k_new_stride + at.head * dim;
      const T* const v_new = static_cast<const T*>(a.v_new) + static_cast<long long>(at.r.row0 + k0) * a.v_new_stride + at.head * dim;
#pragma unroll 2
      for (int st = 0; st < STEPS; ++st) {  // (unrolled whole, the loads of all steps took the registers of the loop above)
        const int d = value(st);
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
          mma<T>(s[h], k4, w.x, w.y);
        }
      }
#pragma unroll
      for (int h = 0; h < NR; ++h)
#pragma unroll
        for (int r = 0; r < 2; ++r) {
          const int row = 8 * h + 2 * t + r;
          const uint64_t bits = row < rows ? seen(a, at.r, node_of(row), nt * TK) >> (warp * WK) : 0;
#pragma unroll
          for (int e = r; e < 4; e += 2) s[h][e] = bits >> (g + 8 * (e >> 1)) & 1 ? s[h][e] * a.score_log2 : -INFINITY;
        }
      probabilities(s, iv);
      uint32_t p[NR][2][2];
#pragma unroll
      for (int h = 0; h < NR; ++h) terms(T{}, s[h], p[h]);
      bool odd = false;
#pragma unroll
      for (int c = 0; c < C::PIECES; ++c) {
        const int d = 16 * c + 2 * g;
        uint32_t w[4];  // tokens 2 t, 2 t + 1, 2 t + 8, 2 t + 9
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int key = 2 * t + (i & 1) + 8 * (i >> 1);
          w[i] = key < keys && d < dim ? *reinterpret_cast<const uint32_t*>(v_new + key * a.v_new_stride + d) : 0u;
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
        for (int k = 0; k < min(keys, WK); ++k)
#pragma unroll
          for (int h = 0; h < NR; ++h)
#pragma unroll
            for (int r = 0; r < 2; ++r) {
              const int row = 8 * h + 2 * t + r;
              if (row >= rows || !(seen(a, at.r, node_of(row), nt * TK) >> (warp * WK + k) & 1)) continue;
#pragma unroll
              for (int c = 0; c < C::PIECES; ++c)
                if (16 * c + 2 * g < dim) {
                  const float2 x = unpack2<T>(*reinterpret_cast<const uint32_t*>(v_new + k * a.v_new_stride + 16 * c + 2 * g));
                  if (!isfinite(x.x)) o[h][c][r] += x.x;
                  if (!isfinite(x.y)) o[h][c][2 + r] += x.y;
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
      const int row = e / (DP / 4), col = e - row * (DP / 4);
      const float4 y = *reinterpret_cast<const float4*>(meet + row * C::MEET + 4 * col);
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
        if (4 * col < dim)
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

bool valid(const ivit_attention_config& c, const ivit_quantised_layout& l) {
  return valid_quantised(l) && valid_attention(c, l.kv_heads, l.page_size);
}

struct Plan {
  int dp, nr, ctas_per_sm, part_floats;
};

Plan plan(const ivit_attention_config& c, const ivit_quantised_layout& l) {
  const long long rows = static_cast<long long>(c.max_new) * (c.heads / l.kv_heads);  // that share a key head
  const auto of = [&](auto d) {
    constexpr int DP = decltype(d)::value;
    return rows <= 8 ? Plan{DP, 1, Cfg<DP, 1>::CTAS, Cfg<DP, 1>::PART} : Plan{DP, 2, Cfg<DP, 2>::CTAS, Cfg<DP, 2>::PART};
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

template <typename T, int DP, int NR>
cudaError_t launch_rows(const QuantisedArgs& a, int ctas, cudaStream_t s) {
  using C = Cfg<DP, NR>;
  const auto kernel = [&](auto common) {
    constexpr Common COMMON = decltype(common)::value;
    const cudaError_t e = allow_smem<tree_attention_quantised_kernel<T, DP, NR, COMMON>>(C::BYTES);
    return e != cudaSuccess ? e : launch_ex(tree_attention_quantised_kernel<T, DP, NR, COMMON>, dim3(ctas), dim3(THREADS), C::BYTES, s, 1, a);
  };
  const cudaError_t e = a.block_shift >= 4          ? kernel(std::integral_constant<Common, BLOCK>{})
                        : a.cache.page_shift >= 4 ? kernel(std::integral_constant<Common, PAGE>{})
                                                    : kernel(std::integral_constant<Common, NOTHING>{});
  return e != cudaSuccess ? e : launch_tree_join<T, DP, C::M, false>(a, ctas, s);
}

template <typename T, int DP>
cudaError_t launch(const Plan& p, const QuantisedArgs& a, int ctas, cudaStream_t s) {
  return p.nr == 1 ? launch_rows<T, DP, 1>(a, ctas, s) : launch_rows<T, DP, 2>(a, ctas, s);
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
  a.wide = all_aligned({k_cache_dev, v_cache_dev}, 16) && c.dim % 16 == 0 && c.page_stride % 16 == 0 && c.token_stride % 16 == 0 &&
           c.head_stride % 16 == 0;
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
  a.tile_rows = 8 * p.nr;
  a.err = static_cast<int*>(workspace_dev);
  a.joins = static_cast<int4*>(workspace_dev) + 1;
  a.parts = reinterpret_cast<float*>(a.joins + 2 * p.ctas_per_sm * TREE_MAX_SMS);
  const auto width = [&](auto type) {
    using T = decltype(type);
    return p.dp == 64    ? launch<T, 64>(p, a, ctas, s)
           : p.dp == 80  ? launch<T, 80>(p, a, ctas, s)
           : p.dp == 96  ? launch<T, 96>(p, a, ctas, s)
           : p.dp == 128 ? launch<T, 128>(p, a, ctas, s)
                         : launch<T, 256>(p, a, ctas, s);
  };
  const cudaError_t e = cache->dtype == IVIT_BF16 ? width(bf16{}) : width(half{});
  return e == cudaSuccess ? IVIT_OK : fail_cuda(e);
}
