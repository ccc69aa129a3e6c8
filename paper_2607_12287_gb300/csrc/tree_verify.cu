// Drafted tokens against the target's probabilities, from given random numbers (ivit_tree_verify).
//
//   e_v = exp((l_v - max l) / T),  w_v = max(e_v - c q_v, 0),  W = sum_v w_v       (p, w and W of the header times sum e)
//
// A request's rows are looked at in their order: a row that hangs on the last accepted one is a draft x, accepted if
// u W q_x < w_x; then it is the last accepted row, c = 0 and the rows that hang on it are tried.  Else c grows by W, for
// max(max(e - c q, 0) - W q, 0) = max(e - (c + W) q, 0).  Drafts without probabilities (q = 1 at x) leave a list of tokens that
// were tried: w is 0 there.  W loses e_x then, in fp32 with an error of 2^-25 of W, and is summed again over the tokens that are left
// when it is below half of what the last sum gave or 32 have been taken off: the error stays near a sum's own.  In the end the token is the argmax of w_v / noise_v, an exponential race.  Only rows on
// the path are read.
//
// A cluster of up to 8 CTAs has a request, each CTA a part of the vocabulary; sums and maxima of a CTA meet in
// shared memory, those of a cluster through distributed shared memory, all in fixed order, and every thread walks
// through the rows alike.  A request's rows are walked one after another, so a pass over a row (or over a row and its drafter's
// probabilities after a draft that was not right) is what a step costs, and the requests with most passes end last: 500 requests of
// up to 4 rows of 50001 logits in 32 bits 47 us (3380 GB/s of the 794 rows that are visited; of 50000, with 16-byte loads, 42), a CTA each
// on 304 places; 304 of them, one wave of one to four rows one after another, 30.  64 trees of up to 16 rows of 131072 logits with probabilities 86 us (without 33), one
// run of five rows of 32768 8.9 us.  256 threads instead of 512 took 126 us for the trees; twice the CTAs to a request 83, but 41 instead of
// 33 without probabilities; four loads in flight at one CTA an SM 103.
#include <algorithm>
#include <type_traits>

#include "attention.cuh"
#include "backbone.cuh"

namespace ivit {
namespace {

constexpr int THREADS = 512, WARPS = THREADS / 32;
constexpr int MAX_CLUSTER = 8;
constexpr int MAX_REQ = 65536, MAX_VOCAB = 1 << 24, MAX_NEW = 1024, MAX_ROWS = 1 << 30;
constexpr int U = 8;                   // tokens of a thread at a time

struct VerifyArgs {
  const void* logits;
  const float *prob, *temperature, *uniform, *noise;
  const int *token, *parent, *cu;
  int *path, *accepted, *next;
  long long logits_stride, prob_stride, noise_stride;
  int n_rows, vocab, max_new, slice;   // slice: tokens of a CTA, a multiple of THREADS * U (or the vocabulary's rest)
};

// 8 tokens' values from v on: side by side (VEC) or 32 apart; those past `end` are `none`.
template <typename L, bool VEC>
__device__ __forceinline__ void load8(const L* row, int v, int end, float none, float (&x)[U]) {
  if (VEC && v + U <= end) {
    if (sizeof(L) == 4) {
      const float4 a = *reinterpret_cast<const float4*>(row + v), b = *reinterpret_cast<const float4*>(row + v + 4);
      x[0] = a.x, x[1] = a.y, x[2] = a.z, x[3] = a.w, x[4] = b.x, x[5] = b.y, x[6] = b.z, x[7] = b.w;
    } else {
      const uint4 a = *reinterpret_cast<const uint4*>(row + v);
      const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float2 y = unpack2<typename std::conditional<sizeof(L) == 4, bf16, L>::type>(w[i]);
        x[2 * i] = y.x;
        x[2 * i + 1] = y.y;
      }
    }
    return;
  }
#pragma unroll
  for (int i = 0; i < U; ++i) {
    const int at = v + (VEC ? i : 32 * i);
    x[i] = at < end ? static_cast<float>(row[at]) : none;
  }
}

// The larger of two (value, token) pairs, of equal values the first token; a token of -1: none.
__device__ __forceinline__ void better(float& x, int& at, float y, int y_at) {
  if (y_at >= 0 && (at < 0 || y > x || (y == x && y_at < at))) {
    x = y;
    at = y_at;
  }
}

template <typename L, bool VEC>
__global__ void __launch_bounds__(THREADS) tree_verify_kernel(const VerifyArgs a) {
  constexpr unsigned ALL = 0xffffffffu;
  __shared__ float2 of_warp[WARPS];
  __shared__ float2 of_cta[2][MAX_CLUSTER];  // every CTA's, twice: the next sum does not overwrite one that another CTA still reads
  __shared__ int tried[MAX_NEW];             // tokens without probabilities that were not accepted
  pdl_wait();
  pdl_launch_dependents();
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int rank = cluster_ctarank(), ctas = cluster_nctarank();
  const int req = blockIdx.x / ctas;
  const auto bounded = [&](int r) { return min(max(r, 0), a.n_rows); };
  const int row0 = bounded(a.cu[req]), all = max(bounded(a.cu[req + 1]) - row0, 0), n = min(all, a.max_new);
  // the path's entries past the accepted ones, and the first
  if (rank == 0)
    for (int j = tid; j < all; j += THREADS) a.path[row0 + j] = j == 0 ? row0 : -1;
  if (n == 0) {  // (the same in every CTA of the cluster)
    if (rank == 0 && tid == 0) {
      a.accepted[req] = 0;
      a.next[req] = -1;
    }
    return;
  }
  if (ctas > 1) cluster_sync();  // all have begun, so that they can write to each other's shared memory
  const int v0 = rank * a.slice, v1 = min(a.vocab, v0 + a.slice);
  const float temperature = a.temperature ? a.temperature[req] : 0.f;
  const bool greedy = !(temperature > 0.f);
  const float per = greedy ? 0.f : fminf(fmaxf(1.4426950408889634f / temperature, 1e-30f), 1e30f);
  int parity = 0;

  // (x, y) of all threads of the cluster, joined in order by op(x, y, x', y').
  const auto everywhere = [&](float& x, float& y, auto op) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      const float x2 = __shfl_xor_sync(ALL, x, o), y2 = __shfl_xor_sync(ALL, y, o);
      op(x, y, x2, y2);
    }
    __syncthreads();  // (the last sums have been read)
    if (lane == 0) of_warp[warp] = make_float2(x, y);
    __syncthreads();
    x = of_warp[0].x;
    y = of_warp[0].y;
#pragma unroll
    for (int w = 1; w < WARPS; ++w) op(x, y, of_warp[w].x, of_warp[w].y);
    if (ctas == 1) return;
    if (tid < ctas) {
      const uint32_t to = mapa_shared(smem_u32(&of_cta[parity][rank]), tid);
      asm volatile("st.shared::cluster.v2.f32 [%0], {%1, %2};" ::"r"(to), "f"(x), "f"(y) : "memory");
    }
    cluster_sync();
    x = of_cta[parity][0].x;
    y = of_cta[parity][0].y;
    for (int c = 1; c < ctas; ++c) op(x, y, of_cta[parity][c].x, of_cta[parity][c].y);
    parity ^= 1;
  };
  const auto add = [](float& x, float&, float x2, float) { x += x2; };
  const auto best_of = [](float& x, float& y, float x2, float y2) {
    int at = __float_as_int(y);
    better(x, at, x2, __float_as_int(y2));
    y = __int_as_float(at);
  };
  // Calls f(v, step) for the thread's tokens v, v + step, ..., U at a time.
  constexpr int STEP = VEC ? 1 : 32;
  const auto tokens = [&](auto f) {
#pragma unroll 2
    for (int base = v0 + warp * 32 * U; base < v1; base += THREADS * U) f(base + (VEC ? lane * U : lane));
  };
  const auto logits_of = [&](int row) { return static_cast<const L*>(a.logits) + row * a.logits_stride; };
  // exp((l - top) / T); nothing for -inf and NaN
  const auto weight = [&](float l, float top) { return !(l > -INFINITY) ? 0.f : l == top ? 1.f : ex2((l - top) * per); };

  // Bit i: the thread's token v + i STEP was tried without probabilities and not accepted.
  int n_tried = 0;
  const auto left_out = [&](int v) {
    unsigned out = 0;
    for (int i = 0; i < n_tried; ++i) {
      const int d = tried[i] - v;
      if (d >= 0 && d % STEP == 0 && d / STEP < U) out |= 1u << (d / STEP);
    }
    return out;
  };

  int at = 0, accepted = 1;                // the last accepted row of the request, how many
  float top = -INFINITY, total = 0.f, taken = 0.f;  // max l, W, c
  float summed = 0.f;                      // W as the last sum over all tokens gave it
  int best = -1;                          // greedy: the likeliest token
  const auto enter = [&] {  // of row `at`
    const L* row = logits_of(row0 + at);
    float x = -INFINITY, y;
    if (greedy) {
      int x_at = -1;
      tokens([&](int v) {
        float l[U];
        load8<L, VEC>(row, v, v1, -INFINITY, l);
#pragma unroll
        for (int i = 0; i < U; ++i)
          if (l[i] > x) {  // (a thread's tokens ascend)
            x = l[i];
            x_at = v + STEP * i;
          }
      });
      y = __int_as_float(x_at);
      everywhere(x, y, best_of);
      best = __float_as_int(y);
      return;
    }
    y = 0.f;
    tokens([&](int v) {
      float l[U];
      load8<L, VEC>(row, v, v1, -INFINITY, l);
      float m = x;
#pragma unroll
      for (int i = 0; i < U; ++i) m = fmaxf(m, l[i]);  // (NaN is passed over)
      if (m > x) {
        y *= x == -INFINITY ? 0.f : ex2((x - m) * per);
        x = m;
      }
#pragma unroll
      for (int i = 0; i < U; ++i) y += weight(l[i], x);
    });
    everywhere(x, y, [&](float& x, float& y, float x2, float y2) {
      const float m = fmaxf(x, x2);
      const auto part = [&](float m2, float s) { return m2 == m ? s : m2 == -INFINITY ? 0.f : s * ex2((m2 - m) * per); };
      y = part(x, y) + part(x2, y2);
      x = m;
    });
    top = x;
    total = summed = y;
    taken = 0.f;
    n_tried = 0;
  };

  // The next row from j on that hangs on row `on`, n if there is none.
  const auto next_draft = [&](int j, int on) {
    if (!a.parent) return j == on + 1 && j < n ? j : n;
    for (; j < n; j += 32) {
      const unsigned bits = __ballot_sync(ALL, j + lane < n && a.parent[row0 + j + lane] == on);
      if (bits) return j + __ffs(bits) - 1;
    }
    return n;
  };
  enter();
  int found = next_draft(1, 0);
  while (found < n) {
    const int row = row0 + found, x = a.token[row];
    bool ok = false, tested = x >= 0 && x < a.vocab, less = false;  // (less: W has lost a token)
    if (!tested) {
    } else if (greedy) {
      ok = x == best;
    } else {
      const float e = weight(static_cast<float>(logits_of(row0 + at)[x]), top);
      if (a.prob) {
        const float q = a.prob[(row0 + at) * a.prob_stride + x];
        ok = a.uniform[row] * total * q < fmaxf(e - taken * q, 0.f);
      } else {
        bool again = false;
        for (int i = 0; i < n_tried; ++i) again |= tried[i] == x;
        ok = !again && a.uniform[row] * total < e;
        if (!ok && !again) {
          total = fmaxf(total - e, 0.f);
          less = true;
          __syncthreads();  // (everyone has looked at the list)
          if (tid == 0) tried[n_tried] = x;
          ++n_tried;
          __syncthreads();
        }
      }
    }
    if (ok) {
      if (rank == 0 && tid == 0) a.path[row0 + accepted] = row;
      ++accepted;
      at = found;
      enter();
      found = next_draft(at + 1, at);
      continue;
    }
    found = next_draft(found + 1, at);
    if (!tested || greedy) continue;
    if (a.prob) taken += total;
    if (found >= n) break;  // (nothing is tried against what is left)
    const L* l_row = logits_of(row0 + at);
    if (!a.prob) {
      if (!less || (total >= 0.5f * summed && n_tried % 32 != 0)) continue;
      float sum = 0.f, none = 0.f;
      tokens([&](int v) {
        float l[U];
        load8<L, VEC>(l_row, v, v1, -INFINITY, l);
        const unsigned out = left_out(v);
#pragma unroll
        for (int i = 0; i < U; ++i) sum += out >> i & 1 ? 0.f : weight(l[i], top);
      });
      everywhere(sum, none, add);
      total = summed = sum;
      continue;
    }
    const float* q_row = a.prob + (row0 + at) * a.prob_stride;
    float sum = 0.f, none = 0.f;
    tokens([&](int v) {
      float l[U], q[U];
      load8<L, VEC>(l_row, v, v1, -INFINITY, l);
      load8<float, VEC>(q_row, v, v1, 0.f, q);
#pragma unroll
      for (int i = 0; i < U; ++i) sum += fmaxf(weight(l[i], top) - taken * q[i], 0.f);
    });
    everywhere(sum, none, add);
    total = sum;
  }

  if (!greedy) {
    const L* l_row = logits_of(row0 + at);
    const float* q_row = a.prob && taken > 0.f ? a.prob + (row0 + at) * a.prob_stride : nullptr;
    const float* noise = a.noise + req * a.noise_stride;
    for (int turn = 0; turn < 2; ++turn) {  // the second without what was tried, if nothing else is left
      float x = 0.f, y;
      int x_at = -1;
      tokens([&](int v) {
        float l[U], z[U], q[U];
        load8<L, VEC>(l_row, v, v1, -INFINITY, l);
        load8<float, VEC>(noise, v, v1, 0.f, z);
        if (q_row) load8<float, VEC>(q_row, v, v1, 0.f, q);
        const unsigned out = left_out(v);
#pragma unroll
        for (int i = 0; i < U; ++i) {
          float w = weight(l[i], top);
          if (q_row) w = w - taken * q[i];
          const float r = __fdividef(w, z[i]);
          if (w > 0.f && z[i] > 0.f && r > x && !(out >> i & 1)) {
            x = r;
            x_at = v + STEP * i;
          }
        }
      });
      y = __int_as_float(x_at);
      everywhere(x, y, best_of);
      best = __float_as_int(y);
      if (best >= 0 || (!q_row && n_tried == 0)) break;
      q_row = nullptr;
      n_tried = 0;
    }
  }
  if (rank == 0 && tid == 0) {
    a.accepted[req] = accepted;
    a.next[req] = best;
  }
  if (ctas > 1) cluster_sync();  // no CTA leaves while another may still write to its shared memory
}

template <typename L>
cudaError_t launch(const VerifyArgs& a, int n_req, int cluster, bool vec, cudaStream_t s) {
  return vec ? launch_ex(tree_verify_kernel<L, true>, dim3(n_req * cluster), dim3(THREADS), 0, s, cluster, a)
             : launch_ex(tree_verify_kernel<L, false>, dim3(n_req * cluster), dim3(THREADS), 0, s, cluster, a);
}

}  // namespace
}  // namespace ivit

extern "C" int ivit_tree_verify(const ivit_verify_config* cfg, int32_t n_rows, const void* logits_dev, int64_t logits_stride,
                                const float* draft_prob_dev, int64_t draft_prob_stride, const int32_t* token_dev,
                                const int32_t* parent_dev, const int32_t* cu_rows_dev, const float* temperature_dev,
                                const float* uniform_dev, const float* noise_dev, int64_t noise_stride, int32_t* path_dev,
                                int32_t* accepted_dev, int32_t* next_dev, void* stream) {
  using namespace ivit;
  if (!cfg || n_rows < 0) return fail(IVIT_ERR_ARG, "ivit_tree_verify: null configuration or a negative row count");
  const ivit_verify_config& c = *cfg;
  if (c.n_req < 1 || c.n_req > MAX_REQ || c.vocab < 1 || c.vocab > MAX_VOCAB || c.max_new < 1 || c.max_new > MAX_NEW ||
      n_rows > MAX_ROWS || (c.dtype != IVIT_BF16 && c.dtype != IVIT_FP16 && c.dtype != IVIT_FP32))
    return fail(IVIT_ERR_SHAPE,
                "ivit_tree_verify: need 1..65536 requests, a vocabulary of 1..2^24, max_new 1..1024, up to 2^30 rows and bf16, "
                "fp16 or fp32 logits");
  if (!cu_rows_dev || !accepted_dev || !next_dev ||
      (n_rows > 0 && (!logits_dev || !token_dev || !path_dev || (temperature_dev && (!uniform_dev || !noise_dev)))))
    return fail(IVIT_ERR_ARG, "ivit_tree_verify: null pointer");
  const bool rows = n_rows > 0, prob = rows && temperature_dev && draft_prob_dev, noise = rows && temperature_dev;
  if ((rows && logits_stride < c.vocab) || (prob && draft_prob_stride < c.vocab) || (noise && noise_stride < c.vocab))
    return fail(IVIT_ERR_ARG, "ivit_tree_verify: row strides must be at least the vocabulary");
  const int size = c.dtype == IVIT_FP32 ? 4 : 2;
  if (!aligned(logits_dev, size) || !all_aligned({draft_prob_dev, token_dev, parent_dev, cu_rows_dev, temperature_dev, uniform_dev,
                                                  noise_dev, path_dev, accepted_dev, next_dev}, 4))
    return fail(IVIT_ERR_ARG, "ivit_tree_verify: arrays must be aligned to their elements");
  const int sms = sm_count();
  if (sms <= 0) return fail(IVIT_ERR_CUDA, "ivit_tree_verify: no CUDA device");
  VerifyArgs a = {logits_dev, prob ? draft_prob_dev : nullptr, rows ? temperature_dev : nullptr, uniform_dev, noise_dev,
                  token_dev, parent_dev, cu_rows_dev, path_dev, accepted_dev, next_dev,
                  logits_stride, draft_prob_stride, noise_stride, n_rows, c.vocab, c.max_new, 0};
  // 16-byte loads where every row that is read allows them
  const auto wide = [](const void* p, int64_t stride, int bytes) { return aligned(p, 16) && stride * bytes % 16 == 0; };
  const bool vec = wide(logits_dev, logits_stride, size) && (!prob || wide(draft_prob_dev, draft_prob_stride, 4)) &&
                   (!noise || wide(noise_dev, noise_stride, 4));
  // As many CTAs to a request as find a place at once, each with some work.
  int cluster = MAX_CLUSTER;
  while (cluster > 1 && (static_cast<long long>(c.n_req) * cluster > 2LL * sms || c.vocab < cluster * THREADS * U / 2)) cluster /= 2;
  const int chunks = (c.vocab + THREADS * U - 1) / (THREADS * U);
  a.slice = (chunks + cluster - 1) / cluster * (THREADS * U);
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  const cudaError_t e = c.dtype == IVIT_BF16   ? launch<bf16>(a, c.n_req, cluster, vec, s)
                        : c.dtype == IVIT_FP16 ? launch<half>(a, c.n_req, cluster, vec, s)
                                               : launch<float>(a, c.n_req, cluster, vec, s);
  return e == cudaSuccess ? IVIT_OK : fail_cuda(e);
}
