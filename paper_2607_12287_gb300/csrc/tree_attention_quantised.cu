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

constexpr int TK = 64, WARPS = 4, WK = TK / WARPS, THREADS = 32 * WARPS, M = 16;

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

template <int DP>
struct Cfg {
  static constexpr bool PADDED = DP == 80 || DP == 96;
  static constexpr int ROW = DP == 96 ? 112 : DP;             // bytes of a row of codes: odd numbers of 16-byte pieces if padded
  static constexpr int PIECES = DP / 16, TILE = TK * ROW;
  static constexpr int CTAS = DP <= 64 ? 4 : DP <= 96 ? 3 : 2;  // per SM
  static constexpr int STAGES = DP <= 128 ? 4 : 2;
  // a copy of a warp's keys: CP lanes for the pieces of a row, RP rows at a time
  static constexpr int CP = DP <= 64 ? 4 : DP <= 128 ? 8 : 16, RP = 32 / CP, COPIES = WK / RP;
  static constexpr int STEPS = DP / 16, FULL = DP / 64, TAIL = DP % 64;  // of the product: of 16 values, 64, and what is left
  static constexpr int OFF_SCALES = STAGES * 2 * TILE;         // [stage][K, V][key]
  static constexpr int OFF_MEET = OFF_SCALES + STAGES * 2 * TK * 4;  // [row][DP] fp32
  static constexpr int OFF_ML = OFF_MEET + M * DP * 4;         // [warp][row] maximum and sum
  static constexpr int BYTES = OFF_ML + WARPS * M * 8;
  static constexpr int PART = tree_part_floats(M, DP);
  static_assert(TREE_MAX_REQ * 8 <= OFF_SCALES, "the units before each request");
  static_assert(CTAS * (BYTES + 1024 + 128) <= 228 * 1024, "shared memory of an SM");
};

// Shared-memory offset of 16-byte piece c of a row of codes.  K: a quarter of a warp reads 64 bytes of two rows.  V: ldmatrix
// reads 16 bytes of eight.
template <int DP, bool V>
__device__ __forceinline__ uint32_t piece(int row, int c) {
  using C = Cfg<DP>;
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

template <typename T>
__device__ __forceinline__ bool odd16(uint32_t half_word) {  // infinite or not a number
  constexpr uint32_t e = std::is_same<T, bf16>::value ? 0x7f80u : 0x7c00u;
  return (half_word & e) == e;
}

// ONE_PAGE: the 16 keys of a warp are of one page.
template <typename T, int DP, bool ONE_PAGE>
__global__ void __launch_bounds__(THREADS, Cfg<DP>::CTAS) tree_attention_quantised_kernel(const QuantisedArgs a) {
  using C = Cfg<DP>;
  constexpr unsigned ALL = 0xffffffffu;
  constexpr int STAGES = C::STAGES, COPIES = C::COPIES, RP = C::RP, STEPS = C::STEPS;
  constexpr bool BF16 = std::is_same<T, bf16>::value;
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
  const bool copies = 16 * cp < dim;
  const int second = 16 * cp + 8 < dim;  // the piece's second half is the head's
  const uint32_t k_to = piece<DP, false>(r0, cp), v_to = piece<DP, true>(r0, cp);
  const auto v_place = [&](int x) { return (C::PADDED || DP == 64 ? v_to : v_to ^ ((x * RP & 7) << 4)) + x * RP * C::ROW; };
  // The pages of the tile at `load`, of those rows, and of the lane's scale; kept a tile ahead of the copies.
  constexpr int IDS = ONE_PAGE ? 1 : COPIES;
  const int scale_key = warp * WK + (lane & 15);
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
  const auto copy = [&](int stage) {
    const int key0 = load.kt * TK;
    if (key0 >= load.r.len) return;
    const uint32_t ks = sb + stage * 2 * C::TILE, vs = ks + C::TILE;
    const auto inside = [&](int id, int key) { return key < load.r.len && static_cast<unsigned>(id) < static_cast<unsigned>(a.cache.n_pages); };
    {
      const int key = key0 + scale_key, id = ONE_PAGE ? ids[0] : scale_id;
      const bool ok = inside(id, key);
      const int block = ok ? ((id << a.cache.page_shift) + (key & page_mask)) >> a.block_shift : 0;
      copy4(sb + C::OFF_SCALES + ((2 * stage + (lane >> 4)) * TK + scale_key) * 4,
            (lane < 16 ? a.k_scale : a.v_scale) + static_cast<long long>(block) * a.cache.heads + load.head, ok);
    }
    if (!copies) return;
    const long long head = load.head * a.cache.head_stride + 16 * cp;
    const uint8_t *kc = static_cast<const uint8_t*>(a.k_cache) + head, *vc = static_cast<const uint8_t*>(a.v_cache) + head;
#pragma unroll
    for (int x = 0; x < COPIES; ++x) {
      const int key = key0 + r0 + x * RP, id = ids[ONE_PAGE ? 0 : x];
      const bool ok = inside(id, key);
      const long long off = ok ? id * a.cache.page_stride + (key & page_mask) * a.cache.token_stride : 0;
      const uint32_t kd = ks + k_to + x * RP * C::ROW, vd = vs + v_place(x);
      if (a.wide) {
        copy16(kd, kc + off, ok);
        copy16(vd, vc + off, ok);
      } else {
        copy8(kd, kc + off, ok);
        copy8(vd, vc + off, ok);
        if (second) {
          copy8(kd + 8, kc + off + 8, ok);
          copy8(vd + 8, vc + off + 8, ok);
        }
      }
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
  int u = 0;  // units done
#pragma unroll 1
  while (u < units) {
    // A segment: consecutive key tiles [at.kt, at.kt + tiles) of one tile of rows, cached ones in front.
    const int tiles = min(at.nkt - at.kt, units - u), cached = QuantisedKeys::cached(at.r), n_old = max(0, min(tiles, cached - at.kt));
    const bool two = at.rt * M + 8 < at.r.n * a.group;  // the tile has rows past its first 8
    float o[DP / 8][4], m[2], l[2];
    int node[2];               // new row of the lane's rows g, g + 8 (-1: none)
    const T* from[2];          // their queries
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      const int x = at.rt * M + g + 8 * r, n = x / a.group;
      node[r] = n < at.r.n ? n : -1;
      from[r] = static_cast<const T*>(a.q) + (at.r.row0 + n) * a.q_stride + static_cast<long long>(at.head * a.group + x - n * a.group) * dim;
      m[r] = -INFINITY;
      l[r] = 0.f;
    }
#pragma unroll
    for (int j = 0; j < DP / 8; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) o[j][e] = 0.f;

    // Scores s (log2 units, -inf where a key is not seen) to probabilities against the reference maximum, added to l times iv.
    const auto probabilities = [&](float (&s)[2][4], const float (&iv)[2][2]) {
      float mx[2];
      bool grow = false;
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        if (r == 1 && !two) break;
        mx[r] = fmaxf(fmaxf(s[0][2 * r], s[0][2 * r + 1]), fmaxf(s[1][2 * r], s[1][2 * r + 1]));
        mx[r] = fmaxf(mx[r], __shfl_xor_sync(ALL, mx[r], 1));
        mx[r] = fmaxf(mx[r], __shfl_xor_sync(ALL, mx[r], 2));
        grow |= mx[r] - m[r] > TREE_GROWTH;
      }
      if (__any_sync(ALL, grow)) {
#pragma unroll
        for (int r = 0; r < 2; ++r) {
          if ((r == 1 && !two) || !(mx[r] > m[r])) continue;
          const float alpha = ex2(m[r] - mx[r]);
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
        const float mo = TREE_SHIFT - (m[r] == -INFINITY ? 0.f : m[r]);  // (nothing seen so far: P = 0)
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            s[j][2 * r + e] = ex2(s[j][2 * r + e] + mo);
            l[r] = fmaf(s[j][2 * r + e], iv[j][e], l[r]);
          }
      }
    };
    // two 16-bit terms of each
    const auto terms = [&](auto type, const float (&s)[2][4], uint32_t (&p)[2][4]) {
      using P = decltype(type);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        if ((e & 1) && !two) {
          p[0][e] = p[1][e] = 0u;
          continue;
        }
        const float x = s[e >> 1][2 * (e & 1)], y = s[e >> 1][2 * (e & 1) + 1];
        p[0][e] = pack2<P>(x, y);
        const float2 h = unpack2<P>(p[0][e]);
        p[1][e] = pack2<P>(x - h.x, y - h.y);
      }
    };
    const auto step = [&] {  // the next unit's copies have landed, and those of a later one begin
      copies_wait<STAGES - 2>();
      __syncwarp();  // the lanes' copies have landed, and the stage of the tile before is free
      fill((u + STAGES - 1) % STAGES);
    };

    if (n_old > 0) {
      uint32_t q[STEPS][4];
      float factor[2];
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        factor[r] = a.score_log2;
#pragma unroll
        for (int s = 0; s < STEPS; ++s) {
          const int d = value(s);
          const uint2 w = node[r] >= 0 && d < dim ? *reinterpret_cast<const uint2*>(from[r] + d) : make_uint2(0, 0);
          q[s][r] = w.x;
          q[s][r + 2] = w.y;
        }
        if (BF16) {
          float size = 0.f;
#pragma unroll
          for (int s = 0; s < STEPS; ++s)
#pragma unroll
            for (int e = r; e < 4; e += 2) {
              const float2 y = unpack2<T>(q[s][e]);
              const float y0 = fabsf(y.x), y1 = fabsf(y.y);
              size = fmaxf(size, fmaxf(y0 < INFINITY ? y0 : 0.f, y1 < INFINITY ? y1 : 0.f));
            }
          size = fmaxf(size, __shfl_xor_sync(ALL, size, 1));
          size = fmaxf(size, __shfl_xor_sync(ALL, size, 2));
          const int e2 = max(static_cast<int>(__float_as_uint(size) >> 23) - 127, -100) - 14;  // (-114 .. 113)
          const float up = __int_as_float((127 - e2) << 23);
          factor[r] *= __int_as_float((127 + e2) << 23);
#pragma unroll
          for (int s = 0; s < STEPS; ++s)
#pragma unroll
            for (int e = r; e < 4; e += 2) {
              const float2 y = unpack2<T>(q[s][e]);
              q[s][e] = pack2<half>(y.x * up, y.y * up);
            }
        }
      }
#pragma unroll 1
      for (int kt = at.kt; kt < at.kt + n_old; ++kt, ++u) {
        const int stage = u % STAGES;
        step();
        const int keys = at.r.len - kt * TK - warp * WK;  // cached tokens from the warp's first on
        if (keys <= 0) continue;
        float s[2][4], lv[2][2], iv[2][2];
        const uint8_t* kt8 = sm + stage * 2 * C::TILE;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
#pragma unroll
          for (int e = 0; e < 4; ++e) s[j][e] = 0.f;
          const int row = warp * WK + 8 * j + g;
#pragma unroll
          for (int c = 0; c < C::FULL; ++c) {
            const uint4 w = *reinterpret_cast<const uint4*>(kt8 + piece<DP, false>(row, 4 * c + t));
            const uint32_t ww[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              uint32_t b0, b1;
              codes_to_half4(ww[i], b0, b1);
              mma<half>(s[j], q[4 * c + i], b0, b1);
            }
          }
          if constexpr (C::TAIL == 32) {
            const uint2 w = *reinterpret_cast<const uint2*>(kt8 + piece<DP, false>(row, 4 * C::FULL + (t >> 1)) + 8 * (t & 1));
            uint32_t b0, b1;
            codes_to_half4(w.x, b0, b1);
            mma<half>(s[j], q[STEPS - 2], b0, b1);
            codes_to_half4(w.y, b0, b1);
            mma<half>(s[j], q[STEPS - 1], b0, b1);
          }
          if constexpr (C::TAIL == 16) {
            uint32_t b0, b1;
            codes_to_half4(*reinterpret_cast<const uint32_t*>(kt8 + piece<DP, false>(row, 4 * C::FULL) + 4 * t), b0, b1);
            mma<half>(s[j], q[STEPS - 1], b0, b1);
          }
        }
        const float* scales = reinterpret_cast<const float*>(sm + C::OFF_SCALES) + 2 * stage * TK + warp * WK + 2 * t;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const float2 kf = *reinterpret_cast<const float2*>(scales + 8 * j), vf = *reinterpret_cast<const float2*>(scales + TK + 8 * j);
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const float x = e ? vf.y : vf.x, f = e ? kf.y : kf.x;
            const int b = __float_as_int(x);
            const bool power = !(b & 0x7fffff);
            lv[j][e] = power ? static_cast<float>((b >> 23) - 127) : __log2f(x);
            iv[j][e] = power ? __int_as_float(0x7f000000 - b) : __fdividef(1.f, x);
            if (b < 0x00800000 || b >= 0x7f000000) {  // none (or out of range): the values are as good as 0
              lv[j][e] = -100.f;
              iv[j][e] = __int_as_float((100 + 127) << 23);
            }
#pragma unroll
            for (int r = 0; r < 2; ++r)
              s[j][2 * r + e] = 8 * j + 2 * t + e < keys ? fmaf(s[j][2 * r + e], f * factor[r], lv[j][e]) : -INFINITY;
          }
        }
        probabilities(s, iv);
        uint32_t p[2][4];
        terms(half{}, s, p);
#pragma unroll
        for (int c = 0; c < C::PIECES; c += 2) {
          const int mine = c + 1 < C::PIECES ? c + (lane >> 4) : c;
          uint32_t b[4];
          ldmatrix4_trans(b, sb + (2 * stage + 1) * C::TILE + piece<DP, true>(warp * WK + (lane & 15), mine));
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            if (c + h >= C::PIECES) break;
            // (value 2 g of tokens 2 t, 2 t + 1, then value 2 g + 1; of tokens 8 further on)
            const uint32_t x = __byte_perm(b[2 * h], 0, 0x3120), y = __byte_perm(b[2 * h + 1], 0, 0x3120);
            uint32_t x0, x1, y0, y1;
            codes_to_half4(x, x0, x1);
            codes_to_half4(y, y0, y1);
#pragma unroll
            for (int i = 0; i < 2; ++i) {
              mma<half>(o[2 * (c + h)], p[i], x0, y0);
              mma<half>(o[2 * (c + h) + 1], p[i], x1, y1);
            }
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
      float s[2][4] = {};
      const float iv[2][2] = {{1.f, 1.f}, {1.f, 1.f}};
#pragma unroll
      for (int st = 0; st < STEPS; ++st) {
        const int d = value(st);
        uint32_t qt[4];
#pragma unroll
        for (int r = 0; r < 2; ++r) {
          const uint2 w = node[r] >= 0 && d < dim ? *reinterpret_cast<const uint2*>(from[r] + d) : make_uint2(0, 0);
          qt[r] = w.x;
          qt[r + 2] = w.y;
        }
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const T* k = static_cast<const T*>(a.k_new) + static_cast<long long>(at.r.row0 + k0 + 8 * j + g) * a.k_new_stride + at.head * dim + d;
          const uint2 w = 8 * j + g < keys && d < dim ? *reinterpret_cast<const uint2*>(k) : make_uint2(0, 0);
          mma<T>(s[j], qt, w.x, w.y);
        }
      }
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        const uint64_t bits = node[r] >= 0 ? seen(a, at.r, node[r], nt * TK) >> (warp * WK) : 0;
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
          for (int e = 0; e < 2; ++e)
            s[j][2 * r + e] = bits >> (8 * j + 2 * t + e) & 1 ? s[j][2 * r + e] * a.score_log2 : -INFINITY;
      }
      probabilities(s, iv);
      uint32_t p[2][4];
      terms(T{}, s, p);
      bool odd = false;
#pragma unroll
      for (int c = 0; c < C::PIECES; ++c) {
        const int d = 16 * c + 2 * g;
        uint32_t w[4];  // tokens 2 t, 2 t + 1, 2 t + 8, 2 t + 9
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int key = 2 * t + (i & 1) + 8 * (i >> 1);
          const T* v = static_cast<const T*>(a.v_new) + static_cast<long long>(at.r.row0 + k0 + key) * a.v_new_stride + at.head * dim + d;
          w[i] = key < keys && d < dim ? *reinterpret_cast<const uint32_t*>(v) : 0u;
          // Values that are not finite would reach rows that do not see them (0 * NaN): left out here, added below.
          const bool lo = odd16<T>(w[i]), hi = odd16<T>(w[i] >> 16);
          if (lo) w[i] &= 0xffff0000u;
          if (hi) w[i] &= 0x0000ffffu;
          odd |= lo || hi;
        }
        const uint32_t x0 = __byte_perm(w[0], w[1], 0x5410), x1 = __byte_perm(w[0], w[1], 0x7632);
        const uint32_t y0 = __byte_perm(w[2], w[3], 0x5410), y1 = __byte_perm(w[2], w[3], 0x7632);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          mma<T>(o[2 * c], p[i], x0, y0);
          mma<T>(o[2 * c + 1], p[i], x1, y1);
        }
      }
      if (__any_sync(ALL, odd)) {
#pragma unroll 1
        for (int k = 0; k < min(keys, WK); ++k) {
          const T* v = static_cast<const T*>(a.v_new) + static_cast<long long>(at.r.row0 + k0 + k) * a.v_new_stride + at.head * dim + 4 * t;
#pragma unroll
          for (int r = 0; r < 2; ++r)
            if (node[r] >= 0 && seen(a, at.r, node[r], nt * TK) >> (warp * WK + k) & 1) {
#pragma unroll
              for (int c = 0; c < C::PIECES; ++c)
                if (16 * c + 4 * t < dim) {
                  const uint2 w = *reinterpret_cast<const uint2*>(v + 16 * c);
                  const float2 x = unpack2<T>(w.x), y = unpack2<T>(w.y);
                  if (!isfinite(x.x)) o[2 * c][2 * r] += x.x;
                  if (!isfinite(x.y)) o[2 * c + 1][2 * r] += x.y;
                  if (!isfinite(y.x)) o[2 * c][2 * r + 1] += y.x;
                  if (!isfinite(y.y)) o[2 * c + 1][2 * r + 1] += y.y;
                }
            }
        }
      }
    }

    // The warps meet: every output against the largest maximum, added up in the order of the warps.
    float2* ml = reinterpret_cast<float2*>(sm + C::OFF_ML);
    float* meet = reinterpret_cast<float*>(sm + C::OFF_MEET);
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      l[r] += __shfl_xor_sync(ALL, l[r], 1);
      l[r] += __shfl_xor_sync(ALL, l[r], 2);
      if (t == 0) ml[warp * M + g + 8 * r] = make_float2(m[r], l[r]);
    }
    __syncthreads();
    float f[2];
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      float top = -INFINITY;
#pragma unroll
      for (int w = 0; w < WARPS; ++w) top = fmaxf(top, ml[w * M + g + 8 * r].x);
      f[r] = ex2(m[r] - (top == -INFINITY ? 0.f : top));
    }
#pragma unroll 1
    for (int w = 0; w < WARPS; ++w) {
      if (warp == w) {
#pragma unroll
        for (int r = 0; r < 2; ++r) {
          if (r == 1 && !two) break;
#pragma unroll
          for (int c = 0; c < C::PIECES; ++c) {
            float4* dst = reinterpret_cast<float4*>(meet + (g + 8 * r) * DP + 16 * c + 4 * t);
            float4 y = make_float4(o[2 * c][2 * r] * f[r], o[2 * c + 1][2 * r] * f[r], o[2 * c][2 * r + 1] * f[r],
                                   o[2 * c + 1][2 * r + 1] * f[r]);
            if (w > 0) {
              const float4 x = *dst;
              y = make_float4(x.x + y.x, x.y + y.y, x.z + y.z, x.w + y.w);
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
    const int rows = min(M, at.r.n * a.group - at.rt * M);
#pragma unroll 1
    for (int e = tid; e < rows * (DP / 4); e += THREADS) {
      const int row = e / (DP / 4), col = e - row * (DP / 4);
      const float4 y = *reinterpret_cast<const float4*>(meet + row * DP + 4 * col);
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
  int dp, tile_rows, ctas_per_sm, part_floats;
};

Plan plan(const ivit_attention_config&, const ivit_quantised_layout& l) {
  const auto of = [](auto d) { return Plan{decltype(d)::value, M, Cfg<decltype(d)::value>::CTAS, Cfg<decltype(d)::value>::PART}; };
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

template <typename T, int DP>
cudaError_t launch(const QuantisedArgs& a, int ctas, cudaStream_t s) {
  using C = Cfg<DP>;
  const auto rows = [&](auto one_page) {
    constexpr bool ONE_PAGE = decltype(one_page)::value;
    const cudaError_t e = allow_smem<tree_attention_quantised_kernel<T, DP, ONE_PAGE>>(C::BYTES);
    return e != cudaSuccess ? e : launch_ex(tree_attention_quantised_kernel<T, DP, ONE_PAGE>, dim3(ctas), dim3(THREADS), C::BYTES, s, 1, a);
  };
  const cudaError_t e = a.cache.page_shift >= 4 ? rows(std::true_type{}) : rows(std::false_type{});
  return e != cudaSuccess ? e : launch_tree_join<T, DP, M, false>(a, ctas, s);
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
  a.tile_rows = p.tile_rows;
  a.err = static_cast<int*>(workspace_dev);
  a.joins = static_cast<int4*>(workspace_dev) + 1;
  a.parts = reinterpret_cast<float*>(a.joins + 2 * p.ctas_per_sm * TREE_MAX_SMS);
  const auto width = [&](auto type) {
    using T = decltype(type);
    return p.dp == 64    ? launch<T, 64>(a, ctas, s)
           : p.dp == 80  ? launch<T, 80>(a, ctas, s)
           : p.dp == 96  ? launch<T, 96>(a, ctas, s)
           : p.dp == 128 ? launch<T, 128>(a, ctas, s)
                         : launch<T, 256>(a, ctas, s);
  };
  const cudaError_t e = cache->dtype == IVIT_BF16 ? width(bf16{}) : width(half{});
  return e == cudaSuccess ? IVIT_OK : fail_cuda(e);
}
