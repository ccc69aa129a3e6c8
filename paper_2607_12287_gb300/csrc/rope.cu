// Norms of queries and keys per head and the rotation by positions of several axes, in one pass
// (ivit_qk_norm_rope), and its gradients (ivit_qk_norm_rope_backward):
//
//   y = x r w, r = 1 / sqrt(mean(x^2) + eps);   (u, v) -> (u c - v s, v c + u s), angle pos * freq;
//   backward, with g' the gradient rotated back:  dw = sum g' x r,  dx = r g' w - x r^3 sum(g' w x) / D.
//
// A row is one warp's work, or that of 2, 4 or 8 warps when there are few rows.  A lane holds 8
// values of a head in two pieces of 4, chosen so that both halves of its 4 pairs are its own (no
// exchange for the rotation) and its 4 cosines and sines serve all of the row's heads; D / 8 lanes
// make a head, 32 / (D / 8) heads a step of the warp, and the loads of several steps are in flight
// together.  The cosines and sines are computed, not read: 4 per lane and row are less than the
// memory a table would add.
//
// Bound: HBM for many rows, the launch and two dependent round trips for a few.
#include <type_traits>

#include "backbone.cuh"

namespace ivit {
namespace {

constexpr int THREADS = 256, WARPS = THREADS / 32;
constexpr int BWD_CTAS_MAX = 1024;  // CTAs of the backward pass: partial weight gradients

struct RopeArgs {
  const void *q, *k, *v, *q_weight, *k_weight;
  void *q_out, *k_out, *k_cache, *v_cache;  // (backward: dq, dk in q_out, k_out)
  const void *grad_q, *grad_k;
  float* partial;
  const int *pos, *axis, *slot;
  const float* freq;
  long long q_stride, k_stride, v_stride, q_out_stride, k_out_stride, grad_q_stride, grad_k_stride, pos_stride;
  PagedCache cache;
  int n_rows, heads, kv_heads, dim, rot, n_axes, interleaved, row_warps;
  float eps;
};

// Cosine and sine of p * f.  The product is carried in two fp32 terms and reduced by multiples of
// 2 pi, itself in two terms (Cody and Waite), so that large positions keep their angle; the fast
// functions are then within 2^-21 of the true values.
__device__ __forceinline__ void turn(int p, float f, float& c, float& s) {
  const float x = static_cast<float>(p), hi = x * f, lo = fmaf(x, f, -hi);
  const float n = rintf(hi * 0.15915494309189535f);
  const float r = fmaf(n, 1.7484555e-7f, fmaf(n, -6.2831854820251465f, hi)) + lo;
  __sincosf(r, &s, &c);
}

// Where a lane's values are: pieces of 4 at a and b; pairs (a[i], b[i]), or (a[0], a[1]) and so on when
// interleaved; lanes past rot / 8 hold values that are not rotated.
struct Lane {
  int group, l, per_head, heads, a, b;  // head of a step, lane of the head, lanes of a head, heads of a step
  bool active, rotated;

  __device__ __forceinline__ Lane(const RopeArgs& p, int lane) {
    per_head = p.dim >> 3;
    heads = 32 / per_head;
    group = lane / per_head;
    l = lane - group * per_head;
    active = group < heads;
    rotated = l < p.rot >> 3;
    if (rotated && !p.interleaved) {
      a = 4 * l;
      b = p.rot / 2 + 4 * l;
    } else {  // (rot is a multiple of 8: the same place for an interleaved pair and an unrotated value)
      a = 8 * l;
      b = a + 4;
    }
  }

  // The sum over a head's lanes, in each of them.
  __device__ __forceinline__ float sum(float v) const {
    if ((per_head & (per_head - 1)) == 0) {
#pragma unroll
      for (int o = 16; o > 0; o >>= 1)
        if (o < per_head) v += __shfl_xor_sync(0xffffffffu, v, o);
      return v;
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1)
      if (o < per_head) {
        const float x = __shfl_down_sync(0xffffffffu, v, o);
        if (l + o < per_head) v += x;
      }
    return __shfl_sync(0xffffffffu, v, group * per_head);
  }
};

__device__ __forceinline__ void angles(const RopeArgs& p, const Lane& ln, int row, float (&c)[4], float (&s)[4]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    c[i] = 1.f;
    s[i] = 0.f;
  }
  if (!ln.rotated) return;
  int at[4] = {p.pos[row], 0, 0, 0};
#pragma unroll
  for (int x = 1; x < 4; ++x)
    if (x < p.n_axes) at[x] = p.pos[x * p.pos_stride + row];
  float f[4];
  int ax[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    f[i] = p.freq[4 * ln.l + i];
    ax[i] = p.n_axes > 1 ? p.axis[4 * ln.l + i] : 0;
  }
#pragma unroll
  for (int i = 0; i < 4; ++i)
    turn(ax[i] == 1 ? at[1] : ax[i] == 2 ? at[2] : ax[i] == 3 ? at[3] : at[0], f[i], c[i], s[i]);
}

// Rotation of a lane's pairs.
template <bool INTERLEAVED>
__device__ __forceinline__ void rotate(float (&a)[4], float (&b)[4], const float (&c)[4], const float (&s)[4]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float& x = !INTERLEAVED ? a[i] : i < 2 ? a[2 * i] : b[2 * i - 4];
    float& y = !INTERLEAVED ? b[i] : i < 2 ? a[2 * i + 1] : b[2 * i - 3];
    const float u = x, v = y;
    x = u * c[i] - v * s[i];
    y = v * c[i] + u * s[i];
  }
}

template <typename T>
__device__ __forceinline__ uint2 load4(const T* p) {
  return *reinterpret_cast<const uint2*>(p);
}
template <typename T>
__device__ __forceinline__ void store4(T* p, const uint2& u) {
  *reinterpret_cast<uint2*>(p) = u;
}

template <typename T>
__device__ __forceinline__ void load_weight(const void* w, const Lane& ln, float (&a)[4], float (&b)[4]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) a[i] = b[i] = 1.f;
  if (w && ln.active) {
    unpack4<T>(load4(static_cast<const T*>(w) + ln.a), a);
    unpack4<T>(load4(static_cast<const T*>(w) + ln.b), b);
  }
}

// Forward: a step of a warp is up to 32 / (D / 8) heads of one kind; the warps of a row take its steps
// (queries, then keys, then values) in turn, STEPS at a time with their loads in flight together.
constexpr int STEPS = 4;

// NORM: there is a weight.
template <typename T, bool NORM, bool INTERLEAVED>
__global__ void __launch_bounds__(THREADS, 3) qk_norm_rope_kernel(const RopeArgs p) {
  const int warp = threadIdx.x >> 5;
  const Lane ln(p, threadIdx.x & 31);
  pdl_wait();
  pdl_launch_dependents();
  const int index = blockIdx.x * WARPS + warp, row = index / p.row_warps, part = index - row * p.row_warps;
  if (row >= p.n_rows) return;
  const int q_steps = (p.heads + ln.heads - 1) / ln.heads, k_steps = (p.kv_heads + ln.heads - 1) / ln.heads;
  const int steps = q_steps + (p.v ? 2 * k_steps : k_steps);
  const int my = ln.group * p.dim;
  const T* q = static_cast<const T*>(p.q) + row * p.q_stride + my;
  const T* k = static_cast<const T*>(p.k) + row * p.k_stride + my;
  const T* v = static_cast<const T*>(p.v) + row * p.v_stride + my;
  const int slot = p.slot ? p.slot[row] : -1;
  const bool cached = p.slot && p.cache.holds(slot);
  float c[4], s[4], qa[4], qb[4], ka[4], kb[4];
  bool first = true;

  for (int base = part; base < steps; base += STEPS * p.row_warps) {
    uint2 ra[STEPS], rb[STEPS];
#pragma unroll
    for (int u = 0; u < STEPS; ++u) {
      const int st = base + u * p.row_warps;
      if (st >= steps) break;  // (the same for the whole warp, as the kind of a step)
      const bool query = st < q_steps, key = st < q_steps + k_steps;
      const int h0 = (query ? st : key ? st - q_steps : st - q_steps - k_steps) * ln.heads;
      const T* src = (query ? q : key ? k : v) + h0 * p.dim;
      ra[u] = rb[u] = make_uint2(0, 0);
      if (ln.active && h0 + ln.group < (query ? p.heads : p.kv_heads)) {
        ra[u] = load4(src + ln.a);
        rb[u] = load4(src + ln.b);
      }
    }
    if (first) {  // (behind the first loads)
      first = false;
      angles(p, ln, row, c, s);
      if (NORM) {
        load_weight<T>(p.q_weight, ln, qa, qb);
        load_weight<T>(p.k_weight, ln, ka, kb);
      }
    }
#pragma unroll
    for (int u = 0; u < STEPS; ++u) {
      const int st = base + u * p.row_warps;
      if (st >= steps) break;
      const bool query = st < q_steps, key = st < q_steps + k_steps;
      const int h0 = (query ? st : key ? st - q_steps : st - q_steps - k_steps) * ln.heads;
      if (key) {
        float a[4], b[4];
        unpack4<T>(ra[u], a);
        unpack4<T>(rb[u], b);
        if (NORM && (query ? p.q_weight : p.k_weight)) {
          float ss = 0.f;
#pragma unroll
          for (int i = 0; i < 4; ++i) ss = fmaf(a[i], a[i], fmaf(b[i], b[i], ss));
          const float r = rsqrtf(ln.sum(ss) / p.dim + p.eps);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            a[i] = a[i] * r * (query ? qa[i] : ka[i]);
            b[i] = b[i] * r * (query ? qb[i] : kb[i]);
          }
        }
        rotate<INTERLEAVED>(a, b, c, s);  // (by nothing where the lane's values are not rotated)
        ra[u] = pack4<T>(a);
        rb[u] = pack4<T>(b);
      }
      if (!ln.active || h0 + ln.group >= (query ? p.heads : p.kv_heads)) continue;
      const int to = h0 * p.dim + my;
      if (query || (key && p.k_out)) {
        T* dst = (query ? static_cast<T*>(p.q_out) + row * p.q_out_stride : static_cast<T*>(p.k_out) + row * p.k_out_stride) + to;
        store4(dst + ln.a, ra[u]);
        store4(dst + ln.b, rb[u]);
      }
      if (!query && cached) {
        T* dst = static_cast<T*>(key ? p.k_cache : p.v_cache) + p.cache.token(slot) + (h0 + ln.group) * p.cache.head_stride;
        store4(dst + ln.a, ra[u]);
        store4(dst + ln.b, rb[u]);
      }
    }
  }
}

constexpr int BWD_STEPS = 2;

// Gradients of the steps of one kind of a row; its heads at x, g and dx (lane's head included).
template <typename T, bool NORM, bool INTERLEAVED>
__device__ __forceinline__ void backward_steps(const RopeArgs& p, const Lane& ln, const T* x, const T* g, T* dx, int part, int heads,
                                               const float (&c)[4], const float (&s)[4], const float (&wa)[4], const float (&wb)[4],
                                               float per, float (&dw)[8]) {
  const int step = p.row_warps * ln.heads;
  for (int base = part * ln.heads; base < heads; base += BWD_STEPS * step) {
    uint2 ga[BWD_STEPS], gb[BWD_STEPS], xa[BWD_STEPS], xb[BWD_STEPS];
#pragma unroll
    for (int u = 0; u < BWD_STEPS; ++u) {
      const int h0 = base + u * step;
      ga[u] = gb[u] = xa[u] = xb[u] = make_uint2(0, 0);
      if (ln.active && h0 + ln.group < heads) {
        ga[u] = load4(g + h0 * p.dim + ln.a);
        gb[u] = load4(g + h0 * p.dim + ln.b);
        if (NORM) {
          xa[u] = load4(x + h0 * p.dim + ln.a);
          xb[u] = load4(x + h0 * p.dim + ln.b);
        }
      }
    }
#pragma unroll
    for (int u = 0; u < BWD_STEPS; ++u) {
      const int h0 = base + u * step;
      if (h0 >= heads) break;
      float a[4], b[4];
      unpack4<T>(ga[u], a);
      unpack4<T>(gb[u], b);
      rotate<INTERLEAVED>(a, b, c, s);
      if (NORM) {
        float ya[4], yb[4];
        unpack4<T>(xa[u], ya);
        unpack4<T>(xb[u], yb);
        float ss = 0.f, dot = 0.f;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          ss = fmaf(ya[i], ya[i], fmaf(yb[i], yb[i], ss));
          dot = fmaf(a[i] * wa[i], ya[i], fmaf(b[i] * wb[i], yb[i], dot));
        }
        ss = ln.sum(ss);
        dot = ln.sum(dot);
        const float r = rsqrtf(ss * per + p.eps), m = r * r * r * dot * per;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          dw[i] = fmaf(a[i], ya[i] * r, dw[i]);
          dw[4 + i] = fmaf(b[i], yb[i] * r, dw[4 + i]);
          a[i] = a[i] * wa[i] * r - ya[i] * m;
          b[i] = b[i] * wb[i] * r - yb[i] * m;
        }
      }
      if (ln.active && h0 + ln.group < heads) {
        store4(dx + h0 * p.dim + ln.a, pack4<T>(a));
        store4(dx + h0 * p.dim + ln.b, pack4<T>(b));
      }
    }
  }
}

template <typename T, bool QNORM, bool KNORM, bool INTERLEAVED>
__global__ void __launch_bounds__(THREADS, 2) qk_norm_rope_backward_kernel(const RopeArgs p) {
  extern __shared__ float sm[];  // [16][THREADS] weight gradients of the lanes
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const Lane ln(p, lane);
  pdl_wait();
  pdl_launch_dependents();
  float dw[2][8];  // of a lane's 8 values: queries, keys
#pragma unroll
  for (int i = 0; i < 8; ++i) dw[0][i] = dw[1][i] = 0.f;
  float wa[2][4], wb[2][4];
  load_weight<T>(p.q_weight, ln, wa[0], wb[0]);
  load_weight<T>(p.k_weight, ln, wa[1], wb[1]);
  const float per = 1.f / p.dim;
  const int my = ln.group * p.dim;

  for (int index = blockIdx.x * WARPS + warp; index < p.n_rows * p.row_warps; index += gridDim.x * WARPS) {
    const int row = index / p.row_warps, part = index - row * p.row_warps;
    float c[4], s[4];
    angles(p, ln, row, c, s);
#pragma unroll
    for (int i = 0; i < 4; ++i) s[i] = -s[i];
    backward_steps<T, QNORM, INTERLEAVED>(p, ln, static_cast<const T*>(p.q) + row * p.q_stride + my,
                                          static_cast<const T*>(p.grad_q) + row * p.grad_q_stride + my,
                                          static_cast<T*>(p.q_out) + row * p.q_out_stride + my, part, p.heads, c, s, wa[0], wb[0],
                                          per, dw[0]);
    backward_steps<T, KNORM, INTERLEAVED>(p, ln, static_cast<const T*>(p.k) + row * p.k_stride + my,
                                          static_cast<const T*>(p.grad_k) + row * p.grad_k_stride + my,
                                          static_cast<T*>(p.k_out) + row * p.k_out_stride + my, part, p.kv_heads, c, s, wa[1], wb[1],
                                          per, dw[1]);
  }
  if (!p.partial) return;
  // the CTA's sums, over its warps and the heads of a step in order
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    sm[(i * 2 + 0) * THREADS + threadIdx.x] = dw[0][i];
    sm[(i * 2 + 1) * THREADS + threadIdx.x] = dw[1][i];
  }
  __syncthreads();
  const int lanes = ln.per_head;
  for (int e = threadIdx.x; e < 16 * lanes; e += THREADS) {
    const int i = e / (2 * lanes), kind = e / lanes & 1, l = e % lanes;
    float sum = 0.f;
    for (int w = 0; w < WARPS; ++w)
      for (int g = 0; g < ln.heads; ++g) sum += sm[(i * 2 + kind) * THREADS + w * 32 + g * lanes + l];
    const bool rotated = l < p.rot >> 3 && !p.interleaved;
    const int d = rotated ? (i < 4 ? 4 * l + i : p.rot / 2 + 4 * l + i - 4) : 8 * l + i;
    p.partial[(static_cast<size_t>(blockIdx.x) * 2 + kind) * p.dim + d] = sum;
  }
}

// Sums of the CTAs' partial weight gradients, 32 values per CTA, in an order that depends on n alone.
__global__ void __launch_bounds__(THREADS) weight_gradient_kernel(const float* partial, int n, int dim, float* dq, float* dk) {
  __shared__ float sm[WARPS][32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, e = blockIdx.x * 32 + lane;
  pdl_wait();
  pdl_launch_dependents();
  float sum = 0.f;
  if (e < 2 * dim)
#pragma unroll 8
    for (int i = warp; i < n; i += WARPS) sum += partial[static_cast<size_t>(i) * 2 * dim + e];
  sm[warp][lane] = sum;
  __syncthreads();
  if (warp == 0 && e < 2 * dim) {
#pragma unroll
    for (int w = 1; w < WARPS; ++w) sum += sm[w][lane];
    float* out = e < dim ? dq : dk;
    if (out) out[e < dim ? e : e - dim] = sum;
  }
}

bool valid(const ivit_rope_config& c) {
  return c.heads >= 1 && c.heads <= 256 && c.kv_heads >= 1 && c.kv_heads <= 256 && c.head_dim >= 8 && c.head_dim <= 256 &&
         c.head_dim % 8 == 0 && c.rot_dim >= 0 && c.rot_dim <= c.head_dim && c.rot_dim % 8 == 0 && c.n_axes >= 1 &&
         c.n_axes <= 4 && (c.interleaved == 0 || c.interleaved == 1) && (c.dtype == IVIT_BF16 || c.dtype == IVIT_FP16) &&
         c.eps >= 0.f && c.eps < 1e30f;
}

const char* kShape = "need heads and kv_heads 1..256, head_dim a multiple of 8 up to 256, rot_dim a multiple of 8 up to "
                     "it, 1..4 axes, interleaved 0 or 1, dtype IVIT_BF16 or IVIT_FP16, eps >= 0";

// Warps of a row: as many as it takes to give each of the chip's warp slots (of `ctas` per SM) a row's part,
// up to the steps that a row has.
int row_warps(long long rows, int steps, int ctas, int sms) {
  int w = 1;
  while (w < WARPS && w < steps && rows * w < static_cast<long long>(ctas) * sms * WARPS) w *= 2;
  return w;
}

// Calls f with the type and the order of the pairs as types.
template <typename F>
cudaError_t dispatch(const ivit_rope_config& c, F f) {
  if (c.dtype == IVIT_BF16) return c.interleaved ? f(bf16{}, std::true_type{}) : f(bf16{}, std::false_type{});
  return c.interleaved ? f(half{}, std::true_type{}) : f(half{}, std::false_type{});
}

RopeArgs common(const ivit_rope_config& c, int n_rows) {
  RopeArgs p = {};
  p.n_rows = n_rows;
  p.heads = c.heads;
  p.kv_heads = c.kv_heads;
  p.dim = c.head_dim;
  p.rot = c.rot_dim;
  p.n_axes = c.n_axes;
  p.interleaved = c.interleaved;
  p.eps = c.eps;
  return p;
}

}  // namespace
}  // namespace ivit

extern "C" int ivit_qk_norm_rope(const ivit_rope_config* cfg, int32_t n_rows, const void* q_dev, int64_t q_stride,
                                 const void* k_dev, int64_t k_stride, const void* v_dev, int64_t v_stride,
                                 const void* q_weight_dev, const void* k_weight_dev, const int32_t* pos_dev,
                                 int64_t pos_stride, const float* freq_dev, const int32_t* axis_dev, void* q_out_dev,
                                 int64_t q_out_stride, void* k_out_dev, int64_t k_out_stride,
                                 const ivit_cache_layout* cache, void* k_cache_dev, void* v_cache_dev,
                                 const int32_t* slot_dev, void* stream) {
  using namespace ivit;
  if (!cfg || n_rows < 0) return fail(IVIT_ERR_ARG, "ivit_qk_norm_rope: null configuration or a negative row count");
  if (!valid(*cfg)) return fail(IVIT_ERR_SHAPE, kShape);
  if (cache && (!valid_cache(*cache) || cache->kv_heads != cfg->kv_heads || cache->head_dim != cfg->head_dim ||
                cache->dtype != cfg->dtype))
    return fail(IVIT_ERR_SHAPE, "ivit_qk_norm_rope: cache layout not supported, or of other heads or type than the rows");
  if ((cache != nullptr) != (v_dev != nullptr) || (cache != nullptr) != (k_cache_dev != nullptr) ||
      (cache != nullptr) != (v_cache_dev != nullptr) || (cache != nullptr) != (slot_dev != nullptr))
    return fail(IVIT_ERR_ARG, "ivit_qk_norm_rope: v, the caches and the slots come together with the cache layout, or not at all");
  if (n_rows == 0) return IVIT_OK;
  if (!q_dev || !k_dev || !pos_dev || !q_out_dev || (cfg->rot_dim > 0 && (!freq_dev || !axis_dev)) || (!k_out_dev && !cache))
    return fail(IVIT_ERR_ARG, "ivit_qk_norm_rope: null pointer");
  if ((q_stride | k_stride | q_out_stride | (k_out_dev ? k_out_stride : 0) | (v_dev ? v_stride : 0)) & 7 || pos_stride < 0 ||
      q_stride < 0 || k_stride < 0 || q_out_stride < 0 || (k_out_dev && k_out_stride < 0) || (v_dev && v_stride < 0))
    return fail(IVIT_ERR_ARG, "ivit_qk_norm_rope: row strides must be multiples of 8 elements");
  if (!all_aligned({q_dev, k_dev, v_dev, q_weight_dev, k_weight_dev, q_out_dev, k_out_dev, k_cache_dev, v_cache_dev}, 16) ||
      !all_aligned({pos_dev, freq_dev, axis_dev, slot_dev}, 4))
    return fail(IVIT_ERR_ARG, "ivit_qk_norm_rope: arrays must be 16-byte aligned (positions, frequencies, axes and slots 4)");
  const int sms = sm_count();
  if (sms <= 0) return fail(IVIT_ERR_CUDA, "ivit_qk_norm_rope: no CUDA device");
  RopeArgs p = common(*cfg, n_rows);
  p.q = q_dev;
  p.k = k_dev;
  p.v = v_dev;
  p.q_weight = q_weight_dev;
  p.k_weight = k_weight_dev;
  p.q_out = q_out_dev;
  p.k_out = k_out_dev;
  p.k_cache = k_cache_dev;
  p.v_cache = v_cache_dev;
  p.pos = pos_dev;
  p.axis = axis_dev;
  p.slot = slot_dev;
  p.freq = freq_dev;
  p.q_stride = q_stride;
  p.k_stride = k_stride;
  p.v_stride = v_stride;
  p.q_out_stride = q_out_stride;
  p.k_out_stride = k_out_stride;
  p.pos_stride = pos_stride;
  if (cache) p.cache = paged(*cache);
  const int per_step = 32 / (cfg->head_dim / 8), vectors = cfg->heads + cfg->kv_heads * (v_dev ? 2 : 1);
  p.row_warps = row_warps(n_rows, (vectors + per_step - 1) / per_step, 3, sms);
  const long long blocks = (static_cast<long long>(n_rows) * p.row_warps + WARPS - 1) / WARPS;
  const dim3 grid(static_cast<unsigned>(blocks));
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  const cudaError_t e = dispatch(*cfg, [&](auto type, auto inter) {
    using T = decltype(type);
    return q_weight_dev || k_weight_dev ? launch_ex(qk_norm_rope_kernel<T, true, inter()>, grid, dim3(THREADS), 0, s, 1, p)
                                        : launch_ex(qk_norm_rope_kernel<T, false, inter()>, grid, dim3(THREADS), 0, s, 1, p);
  });
  return e == cudaSuccess ? IVIT_OK : fail_cuda(e);
}

extern "C" size_t ivit_qk_norm_rope_backward_workspace(const ivit_rope_config* cfg) {
  if (!cfg || !ivit::valid(*cfg)) return 0;
  return sizeof(float) * ivit::BWD_CTAS_MAX * 2 * cfg->head_dim;
}

extern "C" int ivit_qk_norm_rope_backward(const ivit_rope_config* cfg, int32_t n_rows, const void* grad_q_dev,
                                          int64_t grad_q_stride, const void* grad_k_dev, int64_t grad_k_stride,
                                          const void* q_dev, int64_t q_stride, const void* k_dev, int64_t k_stride,
                                          const void* q_weight_dev, const void* k_weight_dev, const int32_t* pos_dev,
                                          int64_t pos_stride, const float* freq_dev, const int32_t* axis_dev,
                                          void* dq_dev, int64_t dq_stride, void* dk_dev, int64_t dk_stride,
                                          float* dq_weight_dev, float* dk_weight_dev, void* workspace_dev, void* stream) {
  using namespace ivit;
  if (!cfg || n_rows < 0)
    return fail(IVIT_ERR_ARG, "ivit_qk_norm_rope_backward: null configuration or a negative row count");
  if (!valid(*cfg)) return fail(IVIT_ERR_SHAPE, kShape);
  if ((dq_weight_dev && !q_weight_dev) || (dk_weight_dev && !k_weight_dev))
    return fail(IVIT_ERR_ARG, "ivit_qk_norm_rope_backward: a weight's gradient without the weight");
  const bool weights = dq_weight_dev || dk_weight_dev;
  if (n_rows > 0 && (!grad_q_dev || !grad_k_dev || !q_dev || !k_dev || !pos_dev || !dq_dev || !dk_dev ||
                     (cfg->rot_dim > 0 && (!freq_dev || !axis_dev))))
    return fail(IVIT_ERR_ARG, "ivit_qk_norm_rope_backward: null pointer");
  if (weights && !workspace_dev) return fail(IVIT_ERR_ARG, "ivit_qk_norm_rope_backward: null workspace");
  if ((grad_q_stride | grad_k_stride | q_stride | k_stride | dq_stride | dk_stride) & 7 || grad_q_stride < 0 ||
      grad_k_stride < 0 || q_stride < 0 || k_stride < 0 || dq_stride < 0 || dk_stride < 0 || pos_stride < 0)
    return fail(IVIT_ERR_ARG, "ivit_qk_norm_rope_backward: row strides must be multiples of 8 elements");
  if (!all_aligned({grad_q_dev, grad_k_dev, q_dev, k_dev, q_weight_dev, k_weight_dev, dq_dev, dk_dev, workspace_dev}, 16) ||
      !all_aligned({pos_dev, freq_dev, axis_dev, dq_weight_dev, dk_weight_dev}, 4))
    return fail(IVIT_ERR_ARG,
                "ivit_qk_norm_rope_backward: arrays must be 16-byte aligned (positions, frequencies, axes and weight gradients 4)");
  const int sms = sm_count();
  if (sms <= 0) return fail(IVIT_ERR_CUDA, "ivit_qk_norm_rope_backward: no CUDA device");
  RopeArgs p = common(*cfg, n_rows);
  p.grad_q = grad_q_dev;
  p.grad_k = grad_k_dev;
  p.q = q_dev;
  p.k = k_dev;
  p.q_weight = q_weight_dev;
  p.k_weight = k_weight_dev;
  p.q_out = dq_dev;
  p.k_out = dk_dev;
  p.partial = weights ? static_cast<float*>(workspace_dev) : nullptr;
  p.pos = pos_dev;
  p.axis = axis_dev;
  p.freq = freq_dev;
  p.grad_q_stride = grad_q_stride;
  p.grad_k_stride = grad_k_stride;
  p.q_stride = q_stride;
  p.k_stride = k_stride;
  p.q_out_stride = dq_stride;
  p.k_out_stride = dk_stride;
  p.pos_stride = pos_stride;
  const int per_step = 32 / (cfg->head_dim / 8);
  p.row_warps = row_warps(n_rows, (cfg->heads + per_step - 1) / per_step, 4, sms);
  const long long blocks = (static_cast<long long>(n_rows) * p.row_warps + WARPS - 1) / WARPS;
  const int most = min(BWD_CTAS_MAX, 4 * sms), grid = static_cast<int>(blocks < most ? blocks : most);
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  cudaError_t e = cudaSuccess;
  if (grid > 0) {
    const size_t smem = weights ? sizeof(float) * 16 * THREADS : 0;
    e = dispatch(*cfg, [&](auto type, auto inter) {
      using T = decltype(type);
      const auto launch = [&](auto kernel) { return launch_ex(kernel, dim3(grid), dim3(THREADS), smem, s, 1, p); };
      return q_weight_dev ? k_weight_dev ? launch(qk_norm_rope_backward_kernel<T, true, true, inter()>)
                                         : launch(qk_norm_rope_backward_kernel<T, true, false, inter()>)
             : k_weight_dev ? launch(qk_norm_rope_backward_kernel<T, false, true, inter()>)
                            : launch(qk_norm_rope_backward_kernel<T, false, false, inter()>);
    });
  }
  if (e == cudaSuccess && weights)
    e = launch_ex(weight_gradient_kernel, dim3((2 * cfg->head_dim + 31) / 32), dim3(THREADS), 0, s, 1,
                  static_cast<const float*>(p.partial), grid, cfg->head_dim, dq_weight_dev, dk_weight_dev);
  return e == cudaSuccess ? IVIT_OK : fail_cuda(e);
}
