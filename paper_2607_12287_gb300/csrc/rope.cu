// Norms of queries and keys per head and the rotation by positions of several axes, in one pass
// (ivit_qk_norm_rope), and its gradients (ivit_qk_norm_rope_backward):
//
//   y = x r w, r = 1 / sqrt(mean(x^2) + eps);   (u, v) -> (u c - v s, v c + u s), angle pos * freq;
//   backward, with g' the gradient rotated back:  dw = sum g' x r,  dx = r g' w - x r^3 sum(g' w x) / D.
//
// A lane holds 8 values of a head in two pieces of 4, chosen so that both halves of its 4 pairs are its
// own: no exchange for the rotation.  D / 8 lanes make a head; the 32 / (D / 8) groups of a warp take a
// row each and walk its heads together, so that a lane's 4 cosines and sines (computed: a table would
// add to the memory read) serve all heads of its row, every step of the warp is of one kind (query, key
// or value), and no step is partly empty.  With few rows their heads are split over more warps, down to
// one head each.
// Heads go through a warp four at a time, loads first, so that four chains of unpack, sum, shuffle and
// scale overlap.
//
// Bound: HBM for many rows, the launch and two dependent round trips for a few.  Measured: 32768 rows of 16 + 16
// heads of 72 58.5 us (5.2 TB/s read and written), gradients of 16385 rows of 32 + 8 heads of 128 94 us (5.4 TB/s),
// 8 rows of 32 + 8 heads of 128 into the cache 2.7 us.  A step of the warp over heads of one row, with the
// cosines in every group, took 140 us instead of 58.5 (the groups' last steps partly empty, 290 instructions a step).
#include <algorithm>
#include <type_traits>

#include "backbone.cuh"

namespace ivit {
namespace {

constexpr int THREADS = 256, WARPS = THREADS / 32;
constexpr int FWD_CTAS = 3, BWD_CTAS = 2;  // per SM
constexpr int BWD_CTAS_MAX = 1024;  // CTAs of the backward pass: partial weight gradients
constexpr int MAX_ROWS = 1 << 30;   // (a warp's index, one to a row at most, is an int)

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
  int row_sets;          // groups of as many rows as a warp takes
  float eps, per_dim;    // per_dim: 1 / dim
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

// A lane's place in a head: pieces of 4 values at a and b, whose pairs are (a[i], b[i]), or (a[0], a[1]) and so
// on when interleaved; lanes past rot / 8 hold values that are not rotated.  L: lanes of a head, 0: any.
template <int L>
struct Lane {
  int group, l, per_head, heads, a, b;  // row of the warp's, lane of the head, lanes of a head, rows of a warp
  bool active, rotated;

  __device__ __forceinline__ Lane(const RopeArgs& p, int lane) {
    per_head = L ? L : p.dim >> 3;
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

  // The sum over a head's lanes, in each of them.  Powers of two: a butterfly; 9, 10 and 12 lanes: rotations
  // within the head, first by the multiples of the cofactor, then by 1, 2, ...; others: a tree and a broadcast.
  __device__ __forceinline__ float sum(float v) const {
    if constexpr (L == 8 || L == 16 || L == 32) {
#pragma unroll
      for (int o = L / 2; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
      return v;
    } else if constexpr (L > 0) {
      static_assert(L == 9 || L == 10 || L == 12, "a sum over the lanes of a head");
      if constexpr (L == 9) return rotations<3, 1>(rotations<3, 3>(v));
      if constexpr (L == 10) return rotations<5, 1>(rotations<2, 5>(v));
      if constexpr (L == 12) return rotations<3, 1>(rotations<2, 3>(rotations<2, 6>(v)));
    } else {
#pragma unroll
      for (int o = 16; o > 0; o >>= 1)
        if (o < per_head) {
          const float x = __shfl_down_sync(0xffffffffu, v, o);
          if (l + o < per_head) v += x;
        }
      return __shfl_sync(0xffffffffu, v, group * per_head);
    }
  }

  // The sum of the values of the lanes l, l + S, ..., l + (N - 1) S of the head, going round.
  template <int N, int S>
  __device__ __forceinline__ float rotations(float v) const {
    float r = v;
#pragma unroll
    for (int i = 1; i < N; ++i) {
      const int to = l + i * S >= L ? l + i * S - L : l + i * S;
      r += __shfl_sync(0xffffffffu, v, group * L + to);  // (the idle lanes of a warp add what they get)
    }
    return r;
  }
};

// Cosines and sines of a lane's pairs (0 and 1, 2 and 3), of no angle where they are not rotated.
template <int L>
__device__ __forceinline__ void angles(const RopeArgs& p, const Lane<L>& ln, int row, float2 (&c)[2], float2 (&s)[2]) {
  float c4[4] = {1.f, 1.f, 1.f, 1.f}, s4[4] = {0.f, 0.f, 0.f, 0.f};
  if (ln.rotated) {
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
      if (ax[i] >= p.n_axes) ax[i] = 0;  // (negative ones choose axis 0 below)
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
      turn(ax[i] == 1 ? at[1] : ax[i] == 2 ? at[2] : ax[i] == 3 ? at[3] : at[0], f[i], c4[i], s4[i]);
  }
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    c[i] = make_float2(c4[2 * i], c4[2 * i + 1]);
    s[i] = make_float2(s4[2 * i], s4[2 * i + 1]);
  }
}

// A lane's 8 values as 16 bits: the words of piece a and of piece b; and as the first and second values of its
// pairs, in fp32.
template <typename T, bool INTERLEAVED>
__device__ __forceinline__ void unpack(const uint2& a, const uint2& b, float2 (&u)[2], float2 (&v)[2]) {
  const float2 x[4] = {unpack2<T>(a.x), unpack2<T>(a.y), unpack2<T>(b.x), unpack2<T>(b.y)};
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    u[i] = INTERLEAVED ? make_float2(x[2 * i].x, x[2 * i + 1].x) : x[i];
    v[i] = INTERLEAVED ? make_float2(x[2 * i].y, x[2 * i + 1].y) : x[2 + i];
  }
}
template <typename T, bool INTERLEAVED>
__device__ __forceinline__ void pack(const float2 (&u)[2], const float2 (&v)[2], uint2& a, uint2& b) {
  if (INTERLEAVED) {
    a = make_uint2(pack2<T>(u[0].x, v[0].x), pack2<T>(u[0].y, v[0].y));
    b = make_uint2(pack2<T>(u[1].x, v[1].x), pack2<T>(u[1].y, v[1].y));
  } else {
    a = make_uint2(pack2<T>(u[0].x, u[0].y), pack2<T>(u[1].x, u[1].y));
    b = make_uint2(pack2<T>(v[0].x, v[0].y), pack2<T>(v[1].x, v[1].y));
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

// A norm's weights at a lane's values (1 without one).
template <typename T, bool INTERLEAVED, int L>
__device__ __forceinline__ void load_weight(const void* w, const Lane<L>& ln, float2 (&u)[2], float2 (&v)[2]) {
  u[0] = u[1] = v[0] = v[1] = make_float2(1.f, 1.f);
  if (w && ln.active) unpack<T, INTERLEAVED>(load4(static_cast<const T*>(w) + ln.a), load4(static_cast<const T*>(w) + ln.b), u, v);
}

__device__ __forceinline__ float2 neg(float2 x) { return make_float2(-x.x, -x.y); }
__device__ __forceinline__ float2 both(float x) { return make_float2(x, x); }

// What turns a lane's values into its outputs: weight times cosine and sine, or the weights alone where the
// values are not rotated.
struct Turn {
  float2 uc[2], us[2], vc[2], vs[2];

  __device__ __forceinline__ void set(const float2 (&wu)[2], const float2 (&wv)[2], const float2 (&c)[2], const float2 (&s)[2]) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      uc[i] = mul_f32x2(wu[i], c[i]);
      us[i] = mul_f32x2(wu[i], s[i]);
      vc[i] = mul_f32x2(wv[i], c[i]);
      vs[i] = neg(mul_f32x2(wv[i], s[i]));
    }
  }
  // (the two products of a value of a pair are not taken where there is no pair: infinity times 0)
  __device__ __forceinline__ void apply(float2 (&u)[2], float2 (&v)[2], bool rotated) const {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      float2 x = mul_f32x2(u[i], uc[i]), y = mul_f32x2(v[i], vc[i]);
      if (rotated) {
        x = fma_f32x2(v[i], vs[i], x);
        y = fma_f32x2(u[i], us[i], y);
      }
      u[i] = x;
      v[i] = y;
    }
  }
};

// Of the heads of a kind, which come after `before` others of the row: the first that is the warp's.
__device__ __forceinline__ int first_head(const RopeArgs& p, int part, int before) {
  const int h = (part - before) % p.row_warps;
  return h < 0 ? h + p.row_warps : h;
}

constexpr int AHEAD = 4;  // heads at a time

// Norm and rotation of N heads, `step` elements apart, to dst and dst2 (either may be null).
template <typename T, int L, bool INTERLEAVED, bool NORM, int N>
__device__ __forceinline__ void forward_heads(const RopeArgs& p, const Lane<L>& ln, bool on, const T* src, int step, T* dst,
                                              long long dst_step, T* dst2, long long dst2_step, const Turn& turn) {
  uint2 a[N], b[N];
#pragma unroll
  for (int i = 0; i < N; ++i) {
    a[i] = b[i] = make_uint2(0, 0);
    if (on) {
      a[i] = load4(src + i * step + ln.a);
      b[i] = load4(src + i * step + ln.b);
    }
  }
#pragma unroll
  for (int i = 0; i < N; ++i) {
    float2 x[2], y[2];
    unpack<T, INTERLEAVED>(a[i], b[i], x, y);
    if (NORM) {
      float2 ss = mul_f32x2(x[0], x[0]);
      ss = fma_f32x2(x[1], x[1], ss);
      ss = fma_f32x2(y[0], y[0], ss);
      ss = fma_f32x2(y[1], y[1], ss);
      const float2 r = both(rsqrtf(fmaf(ln.sum(ss.x + ss.y), p.per_dim, p.eps)));
      turn.apply(x, y, ln.rotated);
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        x[e] = mul_f32x2(x[e], r);
        y[e] = mul_f32x2(y[e], r);
      }
    } else {
      turn.apply(x, y, ln.rotated);
    }
    pack<T, INTERLEAVED>(x, y, a[i], b[i]);
  }
  if (!on) return;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    if (dst) {
      store4(dst + i * dst_step + ln.a, a[i]);
      store4(dst + i * dst_step + ln.b, b[i]);
    }
    if (dst2) {
      store4(dst2 + i * dst2_step + ln.a, a[i]);
      store4(dst2 + i * dst2_step + ln.b, b[i]);
    }
  }
}

// The warp's share of n heads of a row.
template <typename T, int L, bool INTERLEAVED, bool NORM>
__device__ __forceinline__ void forward_kind(const RopeArgs& p, const Lane<L>& ln, bool on, const T* src, T* dst, T* dst2,
                                             long long dst2_stride, int h, int n, const Turn& turn) {
  const int step = p.row_warps * p.dim;
  const long long step2 = p.row_warps * dst2_stride;
  src += h * p.dim;
  if (dst) dst += h * p.dim;
  if (dst2) dst2 += h * dst2_stride;
  const auto advance = [&](int heads) {
    h += heads * p.row_warps;
    src += heads * step;
    if (dst) dst += heads * step;
    if (dst2) dst2 += heads * step2;
  };
  for (; h + (AHEAD - 1) * p.row_warps < n; advance(AHEAD))
    forward_heads<T, L, INTERLEAVED, NORM, AHEAD>(p, ln, on, src, step, dst, step, dst2, step2, turn);
  for (; h < n; advance(1)) forward_heads<T, L, INTERLEAVED, NORM, 1>(p, ln, on, src, step, dst, step, dst2, step2, turn);
}

template <typename T, int L, bool INTERLEAVED, bool NORM>
__global__ void __launch_bounds__(THREADS, FWD_CTAS) qk_norm_rope_kernel(const RopeArgs p) {
  const Lane<L> ln(p, threadIdx.x & 31);
  pdl_wait();
  pdl_launch_dependents();
  const int index = blockIdx.x * WARPS + (threadIdx.x >> 5), set = index / p.row_warps, part = index - set * p.row_warps;
  const long long mine = static_cast<long long>(set) * ln.heads + ln.group;
  const bool on = ln.active && mine < p.n_rows;
  const int row = on ? static_cast<int>(mine) : 0;
  if (!__any_sync(0xffffffffu, on)) return;
  float2 c[2], s[2], wu[2], wv[2];
  angles(p, ln, row, c, s);
  Turn turn;
  load_weight<T, INTERLEAVED>(p.q_weight, ln, wu, wv);
  turn.set(wu, wv, c, s);
  const auto kind = [&](bool norm, const T* src, T* dst, T* dst2, long long dst2_stride, int h, int n) {
    if (NORM && norm) {
      forward_kind<T, L, INTERLEAVED, NORM>(p, ln, on, src, dst, dst2, dst2_stride, h, n, turn);
    } else {
      forward_kind<T, L, INTERLEAVED, false>(p, ln, on, src, dst, dst2, dst2_stride, h, n, turn);
    }
  };
  kind(p.q_weight != nullptr, static_cast<const T*>(p.q) + row * p.q_stride, static_cast<T*>(p.q_out) + row * p.q_out_stride,
       nullptr, 0, part, p.heads);
  load_weight<T, INTERLEAVED>(p.k_weight, ln, wu, wv);
  turn.set(wu, wv, c, s);
  const int slot = p.slot ? p.slot[row] : -1;
  const bool cached = p.slot && p.cache.holds(slot);
  const long long token = cached ? p.cache.token(slot) : 0;
  kind(p.k_weight != nullptr, static_cast<const T*>(p.k) + row * p.k_stride,
       p.k_out ? static_cast<T*>(p.k_out) + row * p.k_out_stride : nullptr, cached ? static_cast<T*>(p.k_cache) + token : nullptr,
       p.cache.head_stride, first_head(p, part, p.heads), p.kv_heads);
  if (!p.v) return;
  const T* v = static_cast<const T*>(p.v) + row * p.v_stride;
  T* to = static_cast<T*>(p.v_cache) + token;
  const bool copies = on && cached;
#pragma unroll 4
  for (int h = first_head(p, part, p.heads + p.kv_heads); h < p.kv_heads; h += p.row_warps)
    if (copies) {
      const uint2 a = load4(v + h * p.dim + ln.a), b = load4(v + h * p.dim + ln.b);
      store4(to + h * p.cache.head_stride + ln.a, a);
      store4(to + h * p.cache.head_stride + ln.b, b);
    }
}

constexpr int BWD_AHEAD = 4;

// Gradients of N heads, `step` elements apart.  dw: of the lane's first values, then of its second ones.
template <typename T, int L, bool INTERLEAVED, bool NORM, int N>
__device__ __forceinline__ void backward_heads(const RopeArgs& p, const Lane<L>& ln, bool on, const T* x, const T* g, T* dx,
                                               int step, const float2 (&c)[2], const float2 (&s)[2], const float2 (&wu)[2],
                                               const float2 (&wv)[2], float2 (&dw)[4]) {
  uint2 ga[N], gb[N], xa[N], xb[N];
#pragma unroll
  for (int i = 0; i < N; ++i) {
    ga[i] = gb[i] = xb[i] = make_uint2(0, 0);
    xa[i] = make_uint2(0x3c003c00u, 0);  // (without a row: positive, so that with eps = 0 nothing is 0 times 1 / sqrt(0))
    if (on) {
      ga[i] = load4(g + i * step + ln.a);
      gb[i] = load4(g + i * step + ln.b);
      if (NORM) {
        xa[i] = load4(x + i * step + ln.a);
        xb[i] = load4(x + i * step + ln.b);
      }
    }
  }
#pragma unroll
  for (int i = 0; i < N; ++i) {
    float2 u[2], v[2];
    unpack<T, INTERLEAVED>(ga[i], gb[i], u, v);
    if (ln.rotated) {  // back, by -a
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const float2 t = fma_f32x2(v[e], s[e], mul_f32x2(u[e], c[e]));
        v[e] = fma_f32x2(neg(u[e]), s[e], mul_f32x2(v[e], c[e]));
        u[e] = t;
      }
    }
    if (NORM) {
      float2 xu[2], xv[2], ss = make_float2(0.f, 0.f), dot = ss, tu[2], tv[2];
      unpack<T, INTERLEAVED>(xa[i], xb[i], xu, xv);
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        ss = fma_f32x2(xu[e], xu[e], ss);
        ss = fma_f32x2(xv[e], xv[e], ss);
        tu[e] = mul_f32x2(u[e], xu[e]);
        tv[e] = mul_f32x2(v[e], xv[e]);
        dot = fma_f32x2(tu[e], wu[e], dot);
        dot = fma_f32x2(tv[e], wv[e], dot);
      }
      const float r = rsqrtf(fmaf(ln.sum(ss.x + ss.y), p.per_dim, p.eps));
      const float m = -r * r * r * ln.sum(dot.x + dot.y) * p.per_dim;
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        dw[e] = fma_f32x2(tu[e], both(r), dw[e]);
        dw[2 + e] = fma_f32x2(tv[e], both(r), dw[2 + e]);
        u[e] = fma_f32x2(xu[e], both(m), mul_f32x2(mul_f32x2(u[e], wu[e]), both(r)));
        v[e] = fma_f32x2(xv[e], both(m), mul_f32x2(mul_f32x2(v[e], wv[e]), both(r)));
      }
    }
    pack<T, INTERLEAVED>(u, v, ga[i], gb[i]);
  }
  if (!on) return;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    store4(dx + i * step + ln.a, ga[i]);
    store4(dx + i * step + ln.b, gb[i]);
  }
}

template <typename T, int L, bool INTERLEAVED, bool NORM>
__global__ void __launch_bounds__(THREADS, BWD_CTAS) qk_norm_rope_backward_kernel(const RopeArgs p) {
  extern __shared__ float sm[];  // [8][THREADS] weight gradients of the lanes
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const Lane<L> ln(p, lane);
  pdl_wait();
  pdl_launch_dependents();
  // queries, then keys: the weights and their gradients of one kind are live at a time
  for (int kind = 0; kind < 2; ++kind) {
    const void* weight = kind ? p.k_weight : p.q_weight;
    const int n = kind ? p.kv_heads : p.heads;
    float2 dw[4], wu[2], wv[2];
#pragma unroll
    for (int i = 0; i < 4; ++i) dw[i] = make_float2(0.f, 0.f);
    load_weight<T, INTERLEAVED>(weight, ln, wu, wv);
    for (int index = blockIdx.x * WARPS + warp; index < p.row_sets * p.row_warps; index += gridDim.x * WARPS) {
      const int set = index / p.row_warps, part = index - set * p.row_warps, step = p.row_warps * p.dim;
      int h = kind ? first_head(p, part, p.heads) : part;
      if (h >= n) continue;
      const long long mine = static_cast<long long>(set) * ln.heads + ln.group;
      const bool on = ln.active && mine < p.n_rows;
      const int row = on ? static_cast<int>(mine) : 0;
      const T* x = static_cast<const T*>(kind ? p.k : p.q) + row * (kind ? p.k_stride : p.q_stride) + h * p.dim;
      const T* g = static_cast<const T*>(kind ? p.grad_k : p.grad_q) + row * (kind ? p.grad_k_stride : p.grad_q_stride) + h * p.dim;
      T* dx = static_cast<T*>(kind ? p.k_out : p.q_out) + row * (kind ? p.k_out_stride : p.q_out_stride) + h * p.dim;
      float2 c[2], s[2];
      angles(p, ln, row, c, s);
      const auto heads = [&](auto norm, auto count) {
        constexpr int N = decltype(count)::value;
        backward_heads<T, L, INTERLEAVED, decltype(norm)::value, N>(p, ln, on, x, g, dx, step, c, s, wu, wv, dw);
        h += N * p.row_warps;
        x += N * step;
        g += N * step;
        dx += N * step;
      };
      const auto all = [&](auto norm) {
        while (h + (BWD_AHEAD - 1) * p.row_warps < n) heads(norm, std::integral_constant<int, BWD_AHEAD>{});
        while (h < n) heads(norm, std::integral_constant<int, 1>{});
      };
      if (NORM && weight) {
        all(std::bool_constant<NORM>{});
      } else {
        all(std::false_type{});
      }
    }
    if (!p.partial) continue;
    // the CTA's sums, over its warps and rows in order
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      sm[2 * i * THREADS + threadIdx.x] = dw[i].x;
      sm[(2 * i + 1) * THREADS + threadIdx.x] = dw[i].y;
    }
    __syncthreads();
    const int lanes = ln.per_head;
    for (int e = threadIdx.x; e < 8 * lanes; e += THREADS) {
      const int i = e / lanes, l = e - i * lanes;  // i: first values 0 to 3, then second ones
      float sum = 0.f;
      for (int w = 0; w < WARPS; ++w)
        for (int g = 0; g < ln.heads; ++g) sum += sm[i * THREADS + w * 32 + g * lanes + l];
      const bool split = l < p.rot >> 3 && !INTERLEAVED;
      const int d = INTERLEAVED ? 8 * l + 2 * (i & 3) + (i >> 2) : split ? (i < 4 ? 4 * l + i : p.rot / 2 + 4 * l + i - 4) : 8 * l + i;
      p.partial[(static_cast<size_t>(blockIdx.x) * 2 + kind) * p.dim + d] = sum;
    }
    __syncthreads();  // the sums are read before the other kind's
  }
}

// Sums of the CTAs' partial weight gradients, 32 values per CTA, in an order that depends on n alone.
constexpr int SUM_WARPS = 32;
__global__ void __launch_bounds__(32 * SUM_WARPS) weight_gradient_kernel(const float* partial, int n, int dim, float* dq, float* dk) {
  __shared__ float sm[SUM_WARPS][33];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, e = blockIdx.x * 32 + lane;
  pdl_wait();
  pdl_launch_dependents();
  float sum = 0.f;
  if (e < 2 * dim)
#pragma unroll 8
    for (int i = warp; i < n; i += SUM_WARPS) sum += partial[static_cast<size_t>(i) * 2 * dim + e];
  sm[warp][lane] = sum;
  __syncthreads();
  // warp w adds up value w of the 32
  sum = sm[lane][warp];
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
  const int d = blockIdx.x * 32 + warp;
  float* out = d < dim ? dq : dk;
  if (lane == 0 && d < 2 * dim && out) out[d < dim ? d : d - dim] = sum;
}

bool valid(const ivit_rope_config& c) {
  return c.heads >= 1 && c.heads <= 256 && c.kv_heads >= 1 && c.kv_heads <= 256 && c.head_dim >= 8 && c.head_dim <= 256 &&
         c.head_dim % 8 == 0 && c.rot_dim >= 0 && c.rot_dim <= c.head_dim && c.rot_dim % 8 == 0 && c.n_axes >= 1 &&
         c.n_axes <= 4 && (c.interleaved == 0 || c.interleaved == 1) && (c.dtype == IVIT_BF16 || c.dtype == IVIT_FP16) &&
         c.eps >= 0.f && c.eps < 1e30f;
}

const char* kShape = "need heads and kv_heads 1..256, head_dim a multiple of 8 up to 256, rot_dim a multiple of 8 up to "
                     "it, 1..4 axes, interleaved 0 or 1, dtype IVIT_BF16 or IVIT_FP16, eps >= 0, up to 2^30 rows";

// Warps that share a set of rows: as many as it takes to give each of the chip's warp slots (`ctas` CTAs per
// SM) work, up to the row's heads.
int row_warps(int row_sets, int heads, int ctas, int sms) {
  const long long slots = static_cast<long long>(ctas) * sms * WARPS;
  return static_cast<int>(std::max<long long>(1, std::min<long long>(heads, slots / std::max(1, row_sets))));
}

// Calls f with the type, the lanes of a head (0: any), the order of the pairs and whether there is a weight as types.
template <typename F>
cudaError_t dispatch(const ivit_rope_config& c, bool norm, F f) {
  const auto norms = [&](auto type, auto lanes, auto order) {
    return norm ? f(type, lanes, order, std::true_type{}) : f(type, lanes, order, std::false_type{});
  };
  const auto order = [&](auto type, auto lanes) {
    return c.interleaved ? norms(type, lanes, std::true_type{}) : norms(type, lanes, std::false_type{});
  };
  const auto width = [&](auto type) {
    switch (c.head_dim) {
      case 64: return order(type, std::integral_constant<int, 8>{});
      case 72: return order(type, std::integral_constant<int, 9>{});
      case 80: return order(type, std::integral_constant<int, 10>{});
      case 96: return order(type, std::integral_constant<int, 12>{});
      case 128: return order(type, std::integral_constant<int, 16>{});
      case 256: return order(type, std::integral_constant<int, 32>{});
      default: return order(type, std::integral_constant<int, 0>{});
    }
  };
  return c.dtype == IVIT_BF16 ? width(bf16{}) : width(half{});
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
  p.per_dim = 1.f / c.head_dim;
  const int rows = 32 / (c.head_dim / 8);
  p.row_sets = n_rows / rows + (n_rows % rows != 0);
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
  if (!valid(*cfg) || n_rows > MAX_ROWS) return fail(IVIT_ERR_SHAPE, kShape);
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
  p.row_warps = row_warps(p.row_sets, cfg->heads + cfg->kv_heads * (v_dev ? 2 : 1), FWD_CTAS, sms);
  const long long blocks = (static_cast<long long>(p.row_sets) * p.row_warps + WARPS - 1) / WARPS;
  const dim3 grid(static_cast<unsigned>(blocks));
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  const cudaError_t e = dispatch(*cfg, q_weight_dev || k_weight_dev, [&](auto type, auto lanes, auto order, auto norm) {
    return launch_ex(qk_norm_rope_kernel<decltype(type), lanes(), order(), norm()>, grid, dim3(THREADS), 0, s, 1, p);
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
                                          float* dq_weight_dev, float* dk_weight_dev, void* workspace_dev,
                                          size_t workspace_bytes, void* stream) {
  using namespace ivit;
  if (!cfg || n_rows < 0)
    return fail(IVIT_ERR_ARG, "ivit_qk_norm_rope_backward: null configuration or a negative row count");
  if (!valid(*cfg) || n_rows > MAX_ROWS) return fail(IVIT_ERR_SHAPE, kShape);
  if ((dq_weight_dev && !q_weight_dev) || (dk_weight_dev && !k_weight_dev))
    return fail(IVIT_ERR_ARG, "ivit_qk_norm_rope_backward: a weight's gradient without the weight");
  const bool weights = dq_weight_dev || dk_weight_dev;
  if (n_rows > 0 && (!grad_q_dev || !grad_k_dev || !q_dev || !k_dev || !pos_dev || !dq_dev || !dk_dev ||
                     (cfg->rot_dim > 0 && (!freq_dev || !axis_dev))))
    return fail(IVIT_ERR_ARG, "ivit_qk_norm_rope_backward: null pointer");
  if (weights && (!workspace_dev || workspace_bytes < ivit_qk_norm_rope_backward_workspace(cfg)))
    return fail(IVIT_ERR_ARG, "ivit_qk_norm_rope_backward: the workspace is null or too small");
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
  p.row_warps = row_warps(p.row_sets, cfg->heads + cfg->kv_heads, BWD_CTAS, sms);
  const long long blocks = (static_cast<long long>(p.row_sets) * p.row_warps + WARPS - 1) / WARPS;
  const int most = min(BWD_CTAS_MAX, BWD_CTAS * sms), grid = static_cast<int>(blocks < most ? blocks : most);
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  cudaError_t e = cudaSuccess;
  if (grid > 0) {
    const size_t smem = weights ? sizeof(float) * 8 * THREADS : 0;
    e = dispatch(*cfg, q_weight_dev || k_weight_dev, [&](auto type, auto lanes, auto order, auto norm) {
      return launch_ex(qk_norm_rope_backward_kernel<decltype(type), lanes(), order(), norm()>, dim3(grid), dim3(THREADS), smem, s,
                       1, p);
    });
  }
  if (e == cudaSuccess && weights)
    e = launch_ex(weight_gradient_kernel, dim3((2 * cfg->head_dim + 31) / 32), dim3(32 * SUM_WARPS), 0, s, 1,
                  static_cast<const float*>(p.partial), grid, cfg->head_dim, dq_weight_dev, dk_weight_dev);
  return e == cudaSuccess ? IVIT_OK : fail_cuda(e);
}
