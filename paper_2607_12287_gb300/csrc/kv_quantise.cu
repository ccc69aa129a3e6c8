// Keys and values of accepted rows, of all layers at once, into their slots of a cache of 8 bits (ivit_kv_quantise), and
// cached tokens back as rows (ivit_kv_dequantise).
//
//   code = rn_e4m3(x / 2^e),  e = the smallest in [-60, 60] with max |x| <= 448 2^e
//
// over the finite values of a block of tokens and head; a block that keeps earlier tokens has an e that is not below the old
// one, and rounds them again if it grew.  e4m3 is a floating-point format, so a power of two costs no precision against
// max / 448 (but at the subnormal end), makes x / 2^e exact, and lets a block's scale grow without a second rounding.
//
// Writing: entries of one block lie next to each other in the list, and the first of them does the block.  A CTA finds out which of
// 32 entries are first ones, how far their blocks' entries go and which earlier tokens stay (once, for all heads, keys and
// values); then it takes a (block, some heads, keys or values) of a layer at a time.  The rows' parts, a few heads side by side
// each, come by bulk copies, two to eight such units ahead; a warp has a head: a row's 16-byte pieces go to neighbouring lanes, several
// rows at a time, once for the maximum and once for the rounding.
// Reading: a warp has a unit of (layer, entry) as in kv_write.cu.
//
// What writing spends its time on is instructions (no limit of the machine is reached): 4608 rows of 27 layers of 16 heads of 72 213 us
// (4050 GB/s read and written), of 128 355 us (4330); blocks of a few rows, half of which round earlier tokens again, cost some 340 warp
// instructions a head whatever they hold (896 rows of 32 layers of 8 heads of 128 in 280 blocks 126 us, 1730 GB/s).  The look at
// whether a wait has expired is some 2 us of these.  What was tried: a warp to a block and head with
// its rows in registers 535 us and 191 (119 registers, latency), in shared memory by 16-byte copies 291 and 99 (144 instructions to
// 512 bytes), six CTAs an SM with less room 250 and 102, kept tokens' codes by bulk copies beside the rows 238 and 194, all layers of a chunk
// to a CTA 427 and 126.  Reading: HBM (4099 rows of 32 layers of 8 heads of 128 137 us, 5870 GB/s).
#include <algorithm>
#include <climits>
#include <type_traits>

#include "quantised.cuh"
#include "tree_attention.cuh"

namespace ivit {
namespace {

constexpr int THREADS = 256, WARPS = THREADS / 32;                 // reading
constexpr int W_THREADS = 128, W_WARPS = W_THREADS / 32;           // writing
constexpr int MIN_E = -60, MAX_E = 60;
constexpr int MAX_ROWS = 1 << 30, MAX_WRITTEN = 1 << 20, MAX_LAYERS = 4096;

struct QuantiseArgs {
  const void *k, *v;
  uint8_t *k_cache, *v_cache;
  float *k_scale, *v_scale;
  const int *row, *slot;
  long long row_stride, layer_stride, cache_layer_stride, scale_layer_stride;
  QuantisedCache cache;
  int n_layers, n, n_src;
  int layers;  // of a CTA

  // Slot and row of entry j if it counts, that is if the cache holds the slot and the row is one of the source's, else -1 and -1.
  __device__ __forceinline__ int2 entry(int j) const {
    const bool in = j >= 0 && j < n;
    const int s = in ? slot[j] : -1, r = in ? row[j] : -1;
    return cache.holds(s) && static_cast<unsigned>(r) < static_cast<unsigned>(n_src) ? make_int2(s, r) : make_int2(-1, -1);
  }
};

__device__ __forceinline__ float power(int e) { return __int_as_float((e + 127) << 23); }

// Exponent of the smallest power of two by which `size` (finite, >= 0) is at most 448 = 1.75 * 2^8.
__device__ __forceinline__ int exponent_for(float size) {
  const uint32_t b = __float_as_uint(size);
  return static_cast<int>(b >> 23) - 127 - 8 + ((b & 0x7fffffu) > 0x600000u ? 1 : 0);
}
// ... of two that is at least `scale`; very low for one that is not positive and finite.
__device__ __forceinline__ int exponent_of(float scale) {
  if (!(scale > 0.f && scale < INFINITY)) return -1000;
  const uint32_t b = __float_as_uint(scale);
  return static_cast<int>(b >> 23) - 127 + (b & 0x7fffffu ? 1 : 0);
}

template <typename T>
struct Packed;
template <>
struct Packed<bf16> {
  using Pair = __nv_bfloat162;
};
template <>
struct Packed<half> {
  using Pair = __half2;
};

// The larger magnitudes of pairs, NaN if one is: max(size, |x|) over a piece's 8 values, as its even and odd ones.
template <typename T>
__device__ __forceinline__ uint32_t largest(const uint4& x, uint32_t size) {
  using P = typename Packed<T>::Pair;
  const uint32_t w[4] = {x.x, x.y, x.z, x.w};
  P m = *reinterpret_cast<const P*>(&size);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t magnitude = w[i] & 0x7fff7fffu;
    m = __hmax2_nan(m, *reinterpret_cast<const P*>(&magnitude));
  }
  return *reinterpret_cast<const uint32_t*>(&m);
}

// max(size, |x|) over the finite ones of the 8 values of a piece.
template <typename T>
__device__ __forceinline__ float largest_finite(const uint4& x, float size) {
  const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 y = unpack2<T>(w[i]);
    const float a = fabsf(y.x), b = fabsf(y.y);
    size = fmaxf(size, fmaxf(a < INFINITY ? a : 0.f, b < INFINITY ? b : 0.f));
  }
  return size;
}

// Codes of a piece's values times `inverse`, a power of two.
// In the values' own type, where all are finite: the product is exact, or so small that its code is 0 (fp16: inverse an fp16 number).
template <typename T>
__device__ __forceinline__ uint2 codes_of(const uint4& x, typename Packed<T>::Pair inverse) {
  using P = typename Packed<T>::Pair;
  const uint32_t w[4] = {x.x, x.y, x.z, x.w};
  uint32_t c[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const P y = __hmul2(*reinterpret_cast<const P*>(&w[i]), inverse);
    if constexpr (std::is_same<T, half>::value) {
      uint16_t code;
      asm("cvt.rn.satfinite.e4m3x2.f16x2 %0, %1;" : "=h"(code) : "r"(*reinterpret_cast<const uint32_t*>(&y)));
      c[i] = code;
    } else {
      const float2 f = unpack2<T>(*reinterpret_cast<const uint32_t*>(&y));
      c[i] = to_codes2(f.x, f.y);
    }
  }
  return make_uint2(__byte_perm(c[0], c[1], 0x5410), __byte_perm(c[2], c[3], 0x5410));
}
// Any values, in fp32; those that are not finite become NaN.
template <typename T>
__device__ __forceinline__ uint2 any_codes_of(const uint4& x, float inverse) {
  const uint32_t w[4] = {x.x, x.y, x.z, x.w};
  uint32_t c[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 y = unpack2<T>(w[i]);
    const auto one = [&](float v) { return fabsf(v) < INFINITY ? v * inverse : __uint_as_float(0x7fffffffu); };
    c[i] = to_codes2(one(y.x), one(y.y));
  }
  return make_uint2(__byte_perm(c[0], c[1], 0x5410), __byte_perm(c[2], c[3], 0x5410));
}

// A block that is written.
struct Written {
  int id, first, end, last;  // of its entries (from the chunk's first on) the first, and one past the last that counts; the last place that is written
  int heads, units;          // heads of a unit (0: its rows do not fit), units of keys or values of the blocks up to here
  int gaps;                  // entries between them are skipped
};
constexpr int CHUNK = 32;    // entries whose blocks a CTA has
constexpr int ENTRIES = CHUNK + 128;  // that it looks at: up to blocks of 128 tokens
constexpr int WORDS = 32;    // of the places of a block (up to 1024)
constexpr int STAGED = 36864, MOST_STAGED = STAGED / 2;  // bytes of rows in shared memory, and of a unit
constexpr int MOST_STAGES = 8;

// Grid: (CTAs of a chunk and its layers, chunks, groups of layers).
template <typename T>
__global__ void __launch_bounds__(W_THREADS, 5) kv_quantise_kernel(const QuantiseArgs a) {
  pdl_wait();
  pdl_launch_dependents();
  constexpr unsigned ALL = 0xffffffffu;
  __shared__ __align__(128) uint8_t staged[STAGED];
  __shared__ __align__(8) uint64_t arrived[MOST_STAGES];
  // First unit a wait for whose rows has expired: from it on rows are read from where they lie, as those of blocks that do not fit
  // are, and nothing is copied any more.
  __shared__ int late_from;
  __shared__ int rows[ENTRIES];                  // of the entries (-1: skipped)
  __shared__ long long places[ENTRIES];          // their slots' bytes in the cache
  __shared__ int slots[ENTRIES];                 // (-1: skipped)
  __shared__ Written blocks[CHUNK];
  __shared__ unsigned stay[CHUNK][WORDS];        // places before the last written one that are not written themselves
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int block = 1 << a.cache.block_shift, dim = a.cache.dim, heads = a.cache.heads;
  const int i0 = blockIdx.y * CHUNK;
  for (int e = tid; e < ENTRIES; e += W_THREADS) {
    const int2 entry = a.entry(i0 + e);
    slots[e] = entry.x;
    rows[e] = entry.y;
    places[e] = entry.x >= 0 ? a.cache.token(entry.x) : 0;
  }
  if (tid < MOST_STAGES) mbar_init(smem_u32(&arrived[tid]), 1);
  if (tid == 0) late_from = INT_MAX;
  fence_mbar_init();
  __syncthreads();
  // Blocks that begin among the chunk's entries: an entry whose nearest one before it that counts is of another block.  (Skipped
  // entries may have any slot: one of another block does not end a block.)
  static_assert(CHUNK == 32, "an entry to a lane");
  const int slot0 = slots[lane];
  const unsigned holding = __ballot_sync(ALL, slot0 >= 0), holding_before = holding & ((1u << lane) - 1);
  int before = -1;  // of the chunk's first entry that counts, the nearest slot in front of the chunk
  if (holding)
    for (int j = i0 - 32; j > -32; j -= 32) {
      const int s = a.entry(j + lane).x;
      const unsigned good = __ballot_sync(ALL, s >= 0);
      if (!good) continue;
      before = __shfl_sync(ALL, s, 31 - __clz(good));
      break;
    }
  const int nearest = __shfl_sync(ALL, slot0, holding_before ? 31 - __clz(holding_before) : 0);
  const int previous = holding_before ? nearest : before;
  const bool first = slot0 >= 0 && (previous < 0 || previous >> a.cache.block_shift != slot0 >> a.cache.block_shift);
  const unsigned firsts = __ballot_sync(ALL, first);
  const int n_blocks = __popc(firsts);
  for (int k = warp; k < n_blocks; k += W_WARPS) {  // the k-th of them
    const int at = __fns(firsts, 0, k + 1);
    const int id = __shfl_sync(ALL, slot0, at) >> a.cache.block_shift;
    // How far the block's entries go, and which of its places they write (lane l: places 32 l .. 32 l + 31).
    unsigned written = 0;
    int end = at, last = -1, count = 0;
    for (int e = at;; e += 32) {
      const int s = e + lane < ENTRIES ? slots[e + lane] : a.entry(i0 + e + lane).x;
      const bool same = s >= 0 && s >> a.cache.block_shift == id;
      const unsigned others = __ballot_sync(ALL, s >= 0 && !same);
      const int limit = others ? __ffs(others) - 1 : 32;  // entries from here on are not the block's
      unsigned good = __ballot_sync(ALL, same && lane < limit);
      if (good) end = e + 32 - __clz(good);
      count += __popc(good);
      while (good) {
        const int b = __ffs(good) - 1;
        good &= good - 1;
        const int place = __shfl_sync(ALL, s, b) & (block - 1);
        if (place >> 5 == lane) written |= 1u << (place & 31);
        last = max(last, place);
      }
      if (limit < 32 || i0 + e + 32 >= a.n) break;
    }
    const int in_front = last - 32 * lane;  // places of the lane's that are before the last
    const unsigned all_before = in_front >= 32 ? ALL : in_front > 0 ? (1u << in_front) - 1 : 0u;
    stay[k][lane] = all_before & ~written;
    if (lane == 0) {
      const int fit = end > ENTRIES ? 0 : min(MOST_STAGED / ((end - at) * dim * 2), min(heads, 2 * W_WARPS));
      blocks[k] = {id, at, end, last, fit, (heads + max(fit, 1) - 1) / max(fit, 1), count < end - at};
    }
  }
  __syncthreads();
  if (warp == 0) {  // running sums of the units
    int n = lane < n_blocks ? blocks[lane].units : 0;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int up = __shfl_up_sync(ALL, n, o);
      if (lane >= o) n += up;
    }
    if (lane < n_blocks) blocks[lane].units = n;
  }
  __syncthreads();
  if (n_blocks == 0) return;
  int unit_bytes = 16;
  for (int k = 0; k < n_blocks; ++k) unit_bytes = max(unit_bytes, (blocks[k].end - blocks[k].first) * blocks[k].heads * dim * 2);
  const int stages = min(MOST_STAGES, STAGED / unit_bytes);

  const int layer0 = blockIdx.z * a.layers, of_kv = blocks[n_blocks - 1].units, of_layer = 2 * of_kv;
  const int units = min(a.layers, a.n_layers - layer0) * of_layer;
  struct Unit {
    Written w;
    int k, head0, n_heads, layer;
    bool values;
  };
  const auto unit_of = [&](int unit) {
    Unit u;
    const int in_cta = unit / of_layer, in_layer = unit - in_cta * of_layer;
    u.layer = layer0 + in_cta;
    u.values = in_layer >= of_kv;
    const int x = u.values ? in_layer - of_kv : in_layer;
    u.k = 0;
    while (blocks[u.k].units <= x) ++u.k;
    u.w = blocks[u.k];
    const int per = max(u.w.heads, 1);
    u.head0 = (x - (u.k > 0 ? blocks[u.k - 1].units : 0)) * per;
    u.n_heads = min(per, heads - u.head0);
    return u;
  };
  const auto source = [&](const Unit& u) {
    return static_cast<const T*>(u.values ? a.v : a.k) + u.layer * a.layer_stride + static_cast<long long>(u.head0) * dim;
  };
  const auto copy = [&](int unit, int stage) {  // by the first warp
    if (unit >= units) return;
    const Unit u = unit_of(unit);
    const T* src = source(u);
    const int bytes = u.n_heads * dim * 2, n = u.w.heads > 0 ? u.w.end - u.w.first : 0;
    const uint32_t bar = smem_u32(&arrived[stage]), to = smem_u32(staged) + stage * unit_bytes;
    int good = 0;
    for (int e = lane; e - lane < n; e += 32) good += __popc(__ballot_sync(ALL, e < n && rows[u.w.first + e] >= 0));
    if (lane == 0) mbar_arrive_expect_tx(bar, good * bytes);
    __syncwarp();
    for (int e = lane; e < n; e += 32) {
      const int r = rows[u.w.first + e];
      if (r >= 0) bulk_load(to + e * bytes, src + r * a.row_stride, bytes, bar);
    }
  };

  const int pieces = dim >> 3, rows_at_once = 32 / pieces;
  const int my_row = lane / pieces, my_piece = lane - my_row * pieces;
  const bool used = my_row < rows_at_once;
  int stage = 0, ahead = 0;  // of the unit at hand, of the next copy
  uint32_t phase = 0;
  if (warp == 0)
    for (int i = 0; i < stages - 1; ++i) copy(blockIdx.x + i * gridDim.x, i);
  ahead = stages - 1;
  bool late = false;  // (the same in all threads)
#pragma unroll 1
  for (int unit = blockIdx.x; unit < units; unit += gridDim.x) {
    const Unit u = unit_of(unit);
    // the unit's rows are here, and all warps are done with the one before
    if (!late && !mbar_wait(smem_u32(&arrived[stage]), phase)) atomicMin(&late_from, unit);
    __syncthreads();
    late = *static_cast<volatile int*>(&late_from) <= unit;  // (one that a thread ahead of this one sets is a later unit)
    if (warp == 0 && !late) copy(unit + (stages - 1) * gridDim.x, ahead);
    ahead = ahead == stages - 1 ? 0 : ahead + 1;
    const bool here = u.w.heads > 0 && !late;  // in shared memory

    const int n = u.w.end - u.w.first, n_heads = u.n_heads, row_bytes = n_heads * dim * 2;
    const uint8_t* held = staged + stage * unit_bytes;
    const unsigned stays = stay[u.k][lane], stays0 = stay[u.k][0];
    const bool keeps = __any_sync(ALL, stays != 0);
    float* const scales = (u.values ? a.v_scale : a.k_scale) + u.layer * a.scale_layer_stride + static_cast<long long>(u.w.id) * heads + u.head0;
    // the old scales of the warp's heads, a lane's each
    const int lane_head = warp + W_WARPS * lane;
    const float olds = keeps && lane_head < n_heads ? scales[lane_head] : 0.f;
    uint8_t* const caches = (u.values ? a.v_cache : a.k_cache) + u.layer * a.cache_layer_stride + u.head0 * a.cache.head_stride + 8 * my_piece;
    const T* const sources = source(u) + 8 * my_piece;
    uint8_t* const block_at = caches + a.cache.token(u.w.id << a.cache.block_shift) + my_row * a.cache.token_stride;  // (a block is of one page)
    const long long pass_stride = rows_at_once * a.cache.token_stride;
    const int begin = used ? my_row : n;
#pragma unroll 1
    for (int h = warp; h < n_heads; h += W_WARPS) {
      uint8_t* const cache = caches + h * a.cache.head_stride;
      const uint8_t* const mine = held + h * dim * 2 + my_piece * 16;
      const T* const from = sources + h * dim;
      // Calls f(piece, its place in the cache) for the lane's pieces: of rows in shared memory one after another, of such between which
      // some are skipped, or of a block that is not there.
      const auto each = [&](auto f) {
        if (here && !u.w.gaps) {
          const long long* place = places + u.w.first;
#pragma unroll 4
          for (int e = begin; e < n; e += rows_at_once) f(*reinterpret_cast<const uint4*>(mine + e * row_bytes), place + e);
        } else if (here) {
          for (int e = begin; e < n; e += rows_at_once)
            if (rows[u.w.first + e] >= 0) f(*reinterpret_cast<const uint4*>(mine + e * row_bytes), places + u.w.first + e);
        } else {
          for (int e = begin; e < n; e += rows_at_once) {
            const int2 entry = a.entry(i0 + u.w.first + e);
            if (entry.x < 0) continue;
            const long long place = a.cache.token(entry.x);
            f(*reinterpret_cast<const uint4*>(from + entry.y * a.row_stride), &place);
          }
        }
      };
      uint32_t pair = 0;
      each([&](const uint4& x, const long long*) { pair = largest<T>(x, pair); });
      const float2 both = unpack2<T>(pair);
      const bool finite = __all_sync(ALL, both.x < INFINITY && both.y < INFINITY);
      float size = fmaxf(both.x, both.y);
      if (!finite) {
        size = 0.f;
        each([&](const uint4& x, const long long*) { size = largest_finite<T>(x, size); });
      }
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) size = fmaxf(size, __shfl_xor_sync(ALL, size, o));
      const float old = __shfl_sync(ALL, olds, h / W_WARPS);
      int e2 = exponent_for(size);
      if (keeps) e2 = max(e2, exponent_of(old));
      e2 = min(max(e2, MIN_E), MAX_E);
      const float fresh = power(e2), inverse = power(-e2);
      if (!(keeps && old == fresh)) {
        if (lane == 0) scales[h] = fresh;
        if (keeps) {
          const float ratio = old > 0.f && old < INFINITY ? old * inverse : 0.f;
          const auto again = [&](uint32_t four) {
            uint32_t lo, hi;
            codes_to_half4(four, lo, hi);
            const float2 p = unpack2<half>(lo), q = unpack2<half>(hi);
            return to_codes2(p.x * ratio, p.y * ratio) | to_codes2(q.x * ratio, q.y * ratio) << 16;
          };
          constexpr int AT_ONCE = 4;  // passes whose codes are read together
          uint8_t* at = block_at + h * a.cache.head_stride;
#pragma unroll 1
          for (int p0 = 0; p0 < u.w.last; p0 += AT_ONCE * rows_at_once, at += AT_ONCE * pass_stride) {
            uint2 word[AT_ONCE];
            bool ok[AT_ONCE];
#pragma unroll
            for (int p = 0; p < AT_ONCE; ++p) {
              const int place = p0 + p * rows_at_once + my_row;
              const unsigned bits = block <= 32 ? stays0 : __shfl_sync(ALL, stays, (place >> 5) & 31);
              ok[p] = used && place < u.w.last && bits >> (place & 31) & 1;
              if (ok[p]) word[p] = *reinterpret_cast<const uint2*>(at + p * pass_stride);
            }
#pragma unroll
            for (int p = 0; p < AT_ONCE; ++p)
              if (ok[p]) *reinterpret_cast<uint2*>(at + p * pass_stride) = make_uint2(again(word[p].x), again(word[p].y));
          }
        }
      }
      if (finite && (!std::is_same<T, half>::value || (e2 >= -14 && e2 <= 14))) {
        typename Packed<T>::Pair factor;
        if constexpr (std::is_same<T, half>::value) factor = __float2half2_rn(inverse); else factor = __float2bfloat162_rn(inverse);
        each([&](const uint4& x, const long long* place) { *reinterpret_cast<uint2*>(cache + *place) = codes_of<T>(x, factor); });
      } else {
        each([&](const uint4& x, const long long* place) { *reinterpret_cast<uint2*>(cache + *place) = any_codes_of<T>(x, inverse); });
      }
    }
    if (++stage == stages) {
      stage = 0;
      phase ^= 1;
    }
  }
  // copies that are on their way end (or get as long again) before the shared memory may be another CTA's
  if (late)
    for (int unit = late_from, i = (unit - blockIdx.x) / gridDim.x, last = i + stages - 1; i < last && unit < units; ++i, unit += gridDim.x)
      mbar_wait(smem_u32(&arrived[i % stages]), i / stages & 1);
}

struct DequantiseArgs {
  const uint8_t *k_cache, *v_cache;
  const float *k_scale, *v_scale;
  const int* slot;
  void *k, *v;
  long long row_stride, layer_stride, cache_layer_stride, scale_layer_stride;
  QuantisedCache cache;
  int n_layers, n;
};

// 8 codes times their scale.
template <typename T>
__device__ __forceinline__ uint4 values_of(uint2 c, float scale) {
  uint32_t h[4];
  codes_to_half4(c.x, h[0], h[1]);
  codes_to_half4(c.y, h[2], h[3]);
  uint32_t y[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 f = unpack2<half>(h[i]);
    y[i] = pack2<T>(f.x * scale, f.y * scale);
  }
  return make_uint4(y[0], y[1], y[2], y[3]);
}

template <typename T>
__global__ void __launch_bounds__(THREADS) kv_dequantise_kernel(const DequantiseArgs a) {
  pdl_wait();
  pdl_launch_dependents();
  constexpr int U = 4;  // pieces of a lane in flight
  const int lane = threadIdx.x & 31, pieces = a.cache.dim >> 3, wide = a.cache.heads * pieces;
  const long long warps = static_cast<long long>(gridDim.x) * WARPS, all = static_cast<long long>(a.n_layers) * a.n;
  for (long long w = static_cast<long long>(blockIdx.x) * WARPS + (threadIdx.x >> 5); w < all; w += warps) {
    const int layer = static_cast<int>(w / a.n), i = static_cast<int>(w - static_cast<long long>(layer) * a.n);
    const int slot = a.slot[i];
    if (!a.cache.holds(slot)) continue;
    const long long from = layer * a.cache_layer_stride + a.cache.token(slot), row = layer * a.layer_stride + i * a.row_stride;
    const long long scale = layer * a.scale_layer_stride + a.cache.scale(slot, 0);
    for (int c0 = lane; c0 < 2 * wide; c0 += 32 * U) {
      uint2 x[U];
      float s[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int c = c0 + 32 * u, d = c < wide ? c : c - wide, h = d / pieces;
        if (c >= 2 * wide) continue;
        x[u] = *reinterpret_cast<const uint2*>((c < wide ? a.k_cache : a.v_cache) + from + h * a.cache.head_stride + 8 * (d - h * pieces));
        s[u] = (c < wide ? a.k_scale : a.v_scale)[scale + h];
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int c = c0 + 32 * u, d = c < wide ? c : c - wide;
        if (c >= 2 * wide) continue;
        *reinterpret_cast<uint4*>(static_cast<T*>(c < wide ? a.k : a.v) + row + 8 * d) = values_of<T>(x[u], s[u]);
      }
    }
  }
}

}  // namespace
}  // namespace ivit

extern "C" int ivit_kv_quantise(const ivit_quantised_layout* cache, int32_t n_layers, int32_t n, int32_t n_src,
                                const void* k_dev, const void* v_dev, int64_t row_stride, int64_t layer_stride,
                                const int32_t* src_row_dev, const int32_t* slot_dev, void* k_cache_dev, void* v_cache_dev,
                                int64_t cache_layer_stride, float* k_scale_dev, float* v_scale_dev,
                                int64_t scale_layer_stride, void* stream) {
  using namespace ivit;
  if (!cache || n_layers < 0 || n < 0 || n_src < 0)
    return fail(IVIT_ERR_ARG, "ivit_kv_quantise: null cache layout or a negative size");
  if (!valid_quantised(*cache) || n > MAX_WRITTEN || n_layers > MAX_LAYERS)
    return fail(IVIT_ERR_SHAPE, "ivit_kv_quantise: cache layout not supported, more than 2^20 entries or 4096 layers");
  if (row_stride < 0 || layer_stride < 0 || cache_layer_stride < 0 || scale_layer_stride < 0 || row_stride % 8 ||
      layer_stride % 8 || cache_layer_stride % 8)
    return fail(IVIT_ERR_ARG, "ivit_kv_quantise: strides must not be negative, and multiples of 8 (of scales any)");
  if (n_layers == 0 || n == 0 || n_src == 0) return IVIT_OK;
  if (!k_dev || !v_dev || !src_row_dev || !slot_dev || !k_cache_dev || !v_cache_dev || !k_scale_dev || !v_scale_dev)
    return fail(IVIT_ERR_ARG, "ivit_kv_quantise: null pointer");
  if (!all_aligned({k_dev, v_dev}, 16) || !all_aligned({k_cache_dev, v_cache_dev}, 8) ||
      !all_aligned({src_row_dev, slot_dev, k_scale_dev, v_scale_dev}, 4))
    return fail(IVIT_ERR_ARG, "ivit_kv_quantise: rows must be 16-byte aligned, caches 8-byte, indices and scales 4-byte");
  const int sms = sm_count();
  if (sms <= 0) return fail(IVIT_ERR_CUDA, "ivit_kv_quantise: no CUDA device");
  QuantiseArgs a = {k_dev, v_dev, static_cast<uint8_t*>(k_cache_dev), static_cast<uint8_t*>(v_cache_dev), k_scale_dev, v_scale_dev,
                    src_row_dev, slot_dev, row_stride, layer_stride, cache_layer_stride, scale_layer_stride, quantised(*cache),
                    n_layers, n, n_src, 1};
  // A chunk's layers are CTAs of their own up to some waves of them (rows of a layer lie together: with all layers of a chunk to a CTA,
  // 256 requests' drafts took 126 us instead of 99), or several where there are few, each with a unit for every warp.
  const long long chunks = (n + CHUNK - 1) / CHUNK, places = 5LL * sms;
  a.layers = static_cast<int>(std::max(1LL, std::min<long long>(n_layers, chunks * n_layers / (16 * places))));
  const int groups = (n_layers + a.layers - 1) / a.layers;
  const long long most = std::min<long long>(n, CHUNK) * 2 * ((cache->kv_heads + 2 * W_WARPS - 1) / (2 * W_WARPS));
  const int split = static_cast<int>(std::max(1LL, std::min(most, places / (chunks * groups))));
  const dim3 grid(split, static_cast<unsigned>(chunks), groups);
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  const cudaError_t e = cache->dtype == IVIT_BF16 ? launch_ex(kv_quantise_kernel<bf16>, grid, dim3(W_THREADS), 0, s, 1, a)
                                                  : launch_ex(kv_quantise_kernel<half>, grid, dim3(W_THREADS), 0, s, 1, a);
  return e == cudaSuccess ? IVIT_OK : fail_cuda(e);
}

extern "C" int ivit_kv_dequantise(const ivit_quantised_layout* cache, int32_t n_layers, int32_t n, const int32_t* slot_dev,
                                  const void* k_cache_dev, const void* v_cache_dev, int64_t cache_layer_stride,
                                  const float* k_scale_dev, const float* v_scale_dev, int64_t scale_layer_stride,
                                  void* k_dev, void* v_dev, int64_t row_stride, int64_t layer_stride, void* stream) {
  using namespace ivit;
  if (!cache || n_layers < 0 || n < 0)
    return fail(IVIT_ERR_ARG, "ivit_kv_dequantise: null cache layout or a negative size");
  if (!valid_quantised(*cache) || n > MAX_ROWS)
    return fail(IVIT_ERR_SHAPE, "ivit_kv_dequantise: cache layout not supported, or more than 2^30 entries");
  if (row_stride < 0 || layer_stride < 0 || cache_layer_stride < 0 || scale_layer_stride < 0 || row_stride % 8 ||
      layer_stride % 8 || cache_layer_stride % 8)
    return fail(IVIT_ERR_ARG, "ivit_kv_dequantise: strides must not be negative, and multiples of 8 (of scales any)");
  if (n_layers == 0 || n == 0) return IVIT_OK;
  if (!k_dev || !v_dev || !slot_dev || !k_cache_dev || !v_cache_dev || !k_scale_dev || !v_scale_dev)
    return fail(IVIT_ERR_ARG, "ivit_kv_dequantise: null pointer");
  if (!all_aligned({k_dev, v_dev}, 16) || !all_aligned({k_cache_dev, v_cache_dev}, 8) ||
      !all_aligned({slot_dev, k_scale_dev, v_scale_dev}, 4))
    return fail(IVIT_ERR_ARG, "ivit_kv_dequantise: rows must be 16-byte aligned, caches 8-byte, indices and scales 4-byte");
  const int sms = sm_count();
  if (sms <= 0) return fail(IVIT_ERR_CUDA, "ivit_kv_dequantise: no CUDA device");
  const DequantiseArgs a = {static_cast<const uint8_t*>(k_cache_dev), static_cast<const uint8_t*>(v_cache_dev), k_scale_dev, v_scale_dev,
                            slot_dev, k_dev, v_dev, row_stride, layer_stride, cache_layer_stride, scale_layer_stride,
                            quantised(*cache), n_layers, n};
  const long long blocks = (static_cast<long long>(n_layers) * n + WARPS - 1) / WARPS;
  const int grid = static_cast<int>(std::min(blocks, 8LL * sms));
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  const cudaError_t e = cache->dtype == IVIT_BF16 ? launch_ex(kv_dequantise_kernel<bf16>, dim3(grid), dim3(THREADS), 0, s, 1, a)
                                                  : launch_ex(kv_dequantise_kernel<half>, dim3(grid), dim3(THREADS), 0, s, 1, a);
  return e == cudaSuccess ? IVIT_OK : fail_cuda(e);
}
