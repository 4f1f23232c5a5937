// Clipped policy loss with a KL term over a vocabulary, and its gradient
// (fe_policy_loss, fe_policy_loss_backward).
//
// With e_v = 2^((x_v - m) c), c = log2(e) / temperature and m the row's maximum,
//   logp = ((x_y - m) c - log2 sum e) ln 2,   softmax_v = e_v / sum e,
//   grad_v = k (1[v = y] - softmax_v),  k = grad_scale coef / temperature.
// The maximum comes off before the product, so the exponents' errors are relative to the
// distance from it.  All of it is fp32; a gradient is rounded once.
//
// Bound by memory: at least each logit is read once and its gradient written once.  A row's
// gradient needs the whole row's sum first, so it stays on the SM in between where it fits:
//   rows up to 64 KB   in the registers of a CTA, whose threads (32 to 512) hold up to eight
//                      pieces of 16 bytes each: 1024 threads an SM, in as many CTAs as they make
//   longer rows        the first pass keeps 64 KB of the row in shared memory and asks L2 to
//                      hold the rest, which the second pass reads again; gradients leave with
//                      the lowest claim on L2.  Few rows: up to eight CTAs share one.
//                      (Shorter rows whose gradient is aligned otherwise go this way, too.)
// What matters is rows in different phases beside one another: three CTAs of 512 threads an SM
// for long rows.  4096 tokens x 100000 words in bf16 (241 us at the copy
// rate): 292 us; without the L2 hints 315, everything read twice 397 (hints alone 313), two
// CTAs 322, one of 1024 threads 345.  A ring of bulk copies several rows deep in one CTA of
// 512 threads took 440: its phases do not overlap, and clusters that share a row pay several
// us a row (710 with the row in the registers of four CTAs).  In registers, 16384 tokens in bf16:
// x 1000 (10 us) 21 us (28 with 128 threads, where most have nothing to do), x 8192 (79) 89,
// x 16000 (154) 171 and x 32000 (309) 342 (213 and 381 by way of shared memory).
#include <algorithm>
#include <cmath>
#include <mutex>

#include "fe_ops.cuh"

namespace fe {
namespace {

struct PolicyParams {
  const void* logits;
  void* grad;
  const int32_t* tokens;
  const float *adv, *weights, *old_logp, *ref_logp, *upstream;
  float *terms, *logp, *lse, *coef;
  int32_t* status;
  int64_t logits_row, grad_row;
  int rows, vocab;
  float lo, hi, beta, t, inv_t, scale, c;  // temperature, its inverse; c: log2(e) / temperature
};

constexpr int kThreads = 512;  // of the backward kernel
constexpr float kLn2 = 0.693147180559945309f;

// Running maximum and sum of 2^((x - m) c), m -inf as long as nothing else has come
struct MaxSum {
  float m, s;
};
__device__ __forceinline__ float base_of(float m) { return m == -INFINITY ? 0.f : m; }
// a sum against maximum m0 as one against m >= m0 (m0 -inf: a sum of nothing, 0, or one that a NaN has come into, which
// a maximum does not show)
__device__ __forceinline__ float rebase(float s, float m0, float m, float c) {
  return m0 == -INFINITY ? s : s * ex2_approx((m0 - m) * c);
}
__device__ __forceinline__ MaxSum join(MaxSum a, MaxSum b, float c) {
  const float m = fmaxf(a.m, b.m);
  return {m, rebase(a.s, a.m, m, c) + rebase(b.s, b.m, m, c)};
}

template <int LANES>
__device__ __forceinline__ MaxSum warp_join(MaxSum v, float c) {
  float m = v.m;
#pragma unroll
  for (int o = LANES / 2; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
  float s = rebase(v.s, v.m, m, c);
#pragma unroll
  for (int o = LANES / 2; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
  return {m, s};
}
// the same in every thread; sh: one entry a warp, free again after the block's next barrier
template <int THREADS>
__device__ __forceinline__ MaxSum block_join(MaxSum v, float c, MaxSum* sh) {
  constexpr int W = THREADS / 32;
  v = warp_join<32>(v, c);
  if ((threadIdx.x & 31) == 0) sh[threadIdx.x >> 5] = v;
  __syncthreads();
  return warp_join<W>(sh[threadIdx.x & (W - 1)], c);
}

// What token t brings: weight, index, advantage, log probabilities before and of the reference
// (nothing is done with the loaded values here: a first use waits for its load)
struct Token {
  float w, adv, old, ref;
  int y;
  __device__ __forceinline__ bool kept() const { return w != 0.f; }
  __device__ __forceinline__ bool valid(int vocab) const { return y >= 0 && y < vocab; }
};
__device__ __forceinline__ Token token_of(const PolicyParams& p, int t) {
  Token k;
  k.w = p.weights ? __ldg(p.weights + t) : 1.f / (float)p.rows;
  k.y = __ldg(p.tokens + t);
  k.adv = p.adv ? __ldg(p.adv + t) : 0.f;
  k.old = p.old_logp ? __ldg(p.old_logp + t) : 0.f;
  k.ref = p.ref_logp ? __ldg(p.ref_logp + t) : 0.f;
  return k;
}

// terms, logp, lse and coef of a row from its chosen logit and statistics (written where asked); the gradient's factor
__device__ __forceinline__ float row_outputs(const PolicyParams& p, int t, const Token& k, float xy, MaxSum v, bool write) {
  const float l2 = log2f(v.s);
  float logp = ((xy - v.m) * p.c - l2) * kLn2, lse = v.m * p.inv_t + l2 * kLn2;
  if (v.m == -INFINITY) lse = v.s == v.s ? -INFINITY : NAN, logp = NAN;
  if (!k.valid(p.vocab)) logp = lse = NAN;
  const float r = p.old_logp ? expf(logp - k.old) : 1.f;
  const float plain = r * k.adv, clipped = fminf(fmaxf(r, 1.f - p.lo), 1.f + p.hi) * k.adv;
  float term = plain <= clipped ? -plain : -clipped, coef = plain <= clipped ? -plain : 0.f;
  if (!(plain == plain) || !(logp == logp)) term = coef = NAN;  // (clamping drops a NaN)
  if (p.ref_logp) {
    const float d = k.ref - logp, e = expm1f(d);
    term += p.beta * (e - d);
    coef -= p.beta * e;
  }
  term *= k.w;
  coef *= k.w;
  if (write) {
    p.terms[t] = term;
    p.logp[t] = logp;
    p.lse[t] = lse;
    p.coef[t] = coef;
  }
  return coef * p.scale * p.inv_t;
}

// A row's elements: `head` of them up to a 16-byte boundary, then pieces, then a tail.
template <typename T>
struct RowSplit {
  int head, pieces;
  __device__ RowSplit(const T* x, int n) {
    const unsigned mis = (unsigned)(reinterpret_cast<uintptr_t>(x) & 15u) / sizeof(T);
    head = mis ? min(n, Elem<T>::N - (int)mis) : 0;
    pieces = (n - head) / Elem<T>::N;
  }
};

template <int THREADS, typename T>
__device__ __forceinline__ void zero_row(T* g, int n) {
  const RowSplit<T> rs(g, n);
  if ((int)threadIdx.x < rs.head) g[threadIdx.x] = Elem<T>::put(0.f);
  for (int i = threadIdx.x; i < rs.pieces; i += THREADS) reinterpret_cast<uint4*>(g + rs.head)[i] = make_uint4(0u, 0u, 0u, 0u);
  for (int i = rs.head + rs.pieces * Elem<T>::N + threadIdx.x; i < n; i += THREADS) g[i] = Elem<T>::put(0.f);
}

// grad = k (1[v = y] - 2^((x - b) c) / sum) over a row
template <typename T>
__device__ void grad_row(const T* x, T* g, int n_el, int y, float k, float c, float b, float inv) {
  constexpr int N = Elem<T>::N;
  const float f = -k * inv;
  auto one = [&](int i) { g[i] = Elem<T>::put(fmaf(f, ex2_approx((Elem<T>::get(x[i]) - b) * c), i == y ? k : 0.f)); };
  const RowSplit<T> rs(x, n_el);
  if (((reinterpret_cast<uintptr_t>(x) ^ reinterpret_cast<uintptr_t>(g)) & 15u) != 0) {
    for (int i = threadIdx.x; i < n_el; i += kThreads) one(i);
    return;
  }
  if ((int)threadIdx.x < rs.head) one(threadIdx.x);
  for (int i = threadIdx.x; i < rs.pieces; i += kThreads) {
    const int at = rs.head + i * N;
    float v[N];
    piece_get<T>(*reinterpret_cast<const uint4*>(x + at), v);
#pragma unroll
    for (int j = 0; j < N; ++j) v[j] = fmaf(f, ex2_approx((v[j] - b) * c), at + j == y ? k : 0.f);
    *reinterpret_cast<uint4*>(g + at) = piece_put<T>(v);
  }
  for (int i = rs.head + rs.pieces * N + threadIdx.x; i < n_el; i += kThreads) one(i);
}

// a piece's part of the statistics, against a maximum that covers it
template <typename T>
__device__ __forceinline__ void piece_sum(const uint4& w, uint64_t nb, uint64_t c2, uint64_t* sum) {
  constexpr int N = Elem<T>::N;
  float z[N];
  piece_get<T>(w, z);
#pragma unroll
  for (int j = 0; j < N; j += 2) {
    float a, b;
    f32x2_unpack(f32x2_mul(f32x2_add(f32x2_pack(z[j], z[j + 1]), nb), c2), a, b);
    sum[(j >> 1) & 1] = f32x2_add(sum[(j >> 1) & 1], f32x2_pack(ex2_approx(a), ex2_approx(b)));
  }
}
__device__ __forceinline__ float sum_of(const uint64_t* sum) {
  float a, b, c, d;
  f32x2_unpack(sum[0], a, b);
  f32x2_unpack(sum[1], c, d);
  return (a + b) + (c + d);
}
template <typename T>
__device__ __forceinline__ float piece_max(const uint4& w, float m) {
  constexpr int N = Elem<T>::N;
  float z[N];
  piece_get<T>(w, z);
#pragma unroll
  for (int j = 0; j < N; ++j) m = fmaxf(m, z[j]);
  return m;
}
// The gradient of a piece, f = -k / sum; yj: the token's place in it (any other value: not there).  There
// k - k softmax is rounded once: the two may nearly cancel.
template <typename T>
__device__ __forceinline__ uint4 piece_grad(const uint4& w, uint64_t nb, uint64_t c2, float f, float kf, int yj) {
  constexpr int N = Elem<T>::N;
  const uint64_t f2 = f32x2_pack(f, f);
  float z[N];
  piece_get<T>(w, z);
#pragma unroll
  for (int j = 0; j < N; j += 2) {
    float a, b;
    f32x2_unpack(f32x2_mul(f32x2_add(f32x2_pack(z[j], z[j + 1]), nb), c2), a, b);
    f32x2_unpack(f32x2_mul(f32x2_pack(ex2_approx(a), ex2_approx(b)), f2), z[j], z[j + 1]);
  }
  uint4 r = piece_put<T>(z);
  if (yj >= 0 && yj < N) {
    float b, c, d;
    f32x2_unpack(nb, b, d);
    f32x2_unpack(c2, c, d);
    piece_get<T>(w, z);
    float x = z[0];
#pragma unroll
    for (int j = 1; j < N; ++j) x = j == yj ? z[j] : x;
    const float e = fmaf(f, ex2_approx((x + b) * c), kf);
    uint32_t* rw = reinterpret_cast<uint32_t*>(&r);
#pragma unroll
    for (int j = 0; j < N; ++j) {
      if (j != yj) continue;
      if constexpr (sizeof(T) == 4) {
        rw[j] = __float_as_uint(e);
      } else {
        const T t = Elem<T>::put(e);
        const uint32_t u = *reinterpret_cast<const uint16_t*>(&t);
        rw[j / 2] = j & 1 ? (rw[j / 2] & 0xffffu) | (u << 16) : (rw[j / 2] & 0xffff0000u) | u;
      }
    }
  }
  return r;
}

// ---------------------------------------------------------------------------
// short rows: in registers
// ---------------------------------------------------------------------------
__device__ __forceinline__ uint4 ld_stream(const void* p) {
  uint4 v;
  asm volatile("ld.global.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];"
               : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
               : "l"(p)
               : "memory");
  return v;
}

// A row's edges: the elements before its first 16-byte boundary and after its last one, by thread i < 2 N of a
// block: the element of thread i, or -1.
template <typename T>
__device__ __forceinline__ int edge_of(int i, const RowSplit<T>& rs, int n) {
  constexpr int N = Elem<T>::N;
  if (i < N) return i < rs.head ? i : -1;
  const int at = rs.head + rs.pieces * N + i - N;
  return i < 2 * N && at < n ? at : -1;
}

// A CTA holds a row in registers between its statistics and its gradient; with 1024 threads an SM (64 registers
// each) loads are in flight while other rows compute.
template <typename T, int THREADS, int NV>
__global__ void __launch_bounds__(THREADS, 1024 / THREADS) policy_row_kernel(const PolicyParams p) {
  constexpr int N = Elem<T>::N;
  __shared__ MaxSum sh[THREADS / 32];
  __shared__ float s_k;
  pdl_trigger();
  pdl_wait();
  const int t = blockIdx.x;
  const Token k = token_of(p, t);
  const T* x = reinterpret_cast<const T*>(p.logits) + (long long)t * p.logits_row;
  T* g = p.grad ? reinterpret_cast<T*>(p.grad) + (long long)t * p.grad_row : nullptr;
  if (!k.kept()) {
    if (threadIdx.x == 0) p.terms[t] = p.logp[t] = p.lse[t] = p.coef[t] = 0.f;
    if (g) zero_row<THREADS>(g, p.vocab);
    return;
  }
  const RowSplit<T> rs(x, p.vocab);
  const int edge = edge_of(threadIdx.x, rs, p.vocab);
  const T* xi = x + rs.head;
  uint4 w[NV];
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int at = threadIdx.x + i * THREADS;
    if (at < rs.pieces) w[i] = ld_stream(xi + at * N);
  }
  const float ze = edge >= 0 ? Elem<T>::get(x[edge]) : -INFINITY;
  const float xy = threadIdx.x == 0 && k.valid(p.vocab) ? Elem<T>::get(x[k.y]) : 0.f;
  if (!k.valid(p.vocab) && threadIdx.x == 0 && p.status) atomicOr(p.status, FE_ST_INDEX);
  MaxSum v = {ze, 0.f};
#pragma unroll
  for (int i = 0; i < NV; ++i)
    if (threadIdx.x + i * THREADS < rs.pieces) v.m = piece_max<T>(w[i], v.m);
  const uint64_t c2 = f32x2_pack(p.c, p.c);
  {
    const uint64_t nb = f32x2_pack(-base_of(v.m), -base_of(v.m));
    uint64_t sum[2] = {0ull, 0ull};
#pragma unroll
    for (int i = 0; i < NV; ++i)
      if (threadIdx.x + i * THREADS < rs.pieces) piece_sum<T>(w[i], nb, c2, sum);
    v.s = sum_of(sum) + ex2_approx((ze - base_of(v.m)) * p.c);
  }
  v = block_join<THREADS>(v, p.c, sh);
  if (threadIdx.x == 0) s_k = row_outputs(p, t, k, xy, v, true);
  if (!g) return;
  __syncthreads();
  const float kf = s_k, f = -kf * (1.f / v.s), b = base_of(v.m);
  const uint64_t nb = f32x2_pack(-b, -b);
  T* gi = g + rs.head;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int at = threadIdx.x + i * THREADS;
    if (at < rs.pieces) *reinterpret_cast<uint4*>(gi + at * N) = piece_grad<T>(w[i], nb, c2, f, kf, k.y - rs.head - at * N);
  }
  if (edge >= 0) g[edge] = Elem<T>::put(fmaf(f, ex2_approx((ze - b) * p.c), edge == k.y ? kf : 0.f));
}

// ---------------------------------------------------------------------------
// long rows: shared memory and L2
// ---------------------------------------------------------------------------
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
__device__ __forceinline__ void peer_put(const MaxSum* place, uint32_t rank, MaxSum v) {
  uint32_t at;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(smem_u32(place)), "r"(rank));
  asm volatile("st.shared::cluster.v2.f32 [%0], {%1, %2};" ::"r"(at), "f"(v.m), "f"(v.s) : "memory");
}

__device__ __forceinline__ uint4 ld_hint(const void* p, uint64_t policy) {
  uint4 v;
  asm volatile("ld.global.L1::no_allocate.L2::cache_hint.v4.u32 {%0,%1,%2,%3}, [%4], %5;"
               : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
               : "l"(p), "l"(policy)
               : "memory");
  return v;
}
__device__ __forceinline__ void st_hint(void* p, const uint4& v, uint64_t policy) {
  asm volatile("st.global.L2::cache_hint.v4.u32 [%0], {%1,%2,%3,%4}, %5;" ::"l"(p), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w),
               "l"(policy)
               : "memory");
}

// cs CTAs (a cluster) share a row; each thread keeps its first `keep` pieces, THREADS apart, and has AHEAD in flight
template <typename T, int THREADS, int MINB, int AHEAD>
__global__ void __launch_bounds__(THREADS, MINB) policy_kernel(const PolicyParams p, int cs, int keep) {
  constexpr int N = Elem<T>::N;
  extern __shared__ __align__(16) uint4 held[];  // [keep][THREADS]
  __shared__ MaxSum sh[THREADS / 32];
  __shared__ __align__(8) MaxSum s_peers[8];
  uint64_t hold, leave;  // L2's eviction priorities
  asm("createpolicy.fractional.L2::evict_last.b64 %0, 1.0;" : "=l"(hold));
  asm("createpolicy.fractional.L2::evict_first.b64 %0, 1.0;" : "=l"(leave));
  pdl_trigger();
  if (cs > 1) {  // no peer writes statistics into a CTA that has not begun
    cluster_arrive();
    cluster_wait();
  }
  pdl_wait();
  const int lane = threadIdx.x & 31, rank = (int)blockIdx.x % cs, t = (int)blockIdx.x / cs;
  const Token k = token_of(p, t);
  const T* x = reinterpret_cast<const T*>(p.logits) + (long long)t * p.logits_row;
  T* g = p.grad ? reinterpret_cast<T*>(p.grad) + (long long)t * p.grad_row : nullptr;
  const RowSplit<T> rs(x, p.vocab);
  const int per = (rs.pieces + cs - 1) / cs, from = min(rank * per, rs.pieces), n = min(from + per, rs.pieces) - from;
  const int edge = rank == 0 ? edge_of(threadIdx.x, rs, p.vocab) : -1;
  const T* xi = x + rs.head + (long long)from * N;
  T* gi = g + rs.head + (long long)from * N;
  const bool aligned = ((reinterpret_cast<uintptr_t>(xi) ^ reinterpret_cast<uintptr_t>(gi)) & 15u) == 0;
  auto store = [&](int i, const uint4& w) {
    if (aligned) {
      st_hint(gi + i * N, w, leave);
    } else {
      const T* e = reinterpret_cast<const T*>(&w);
#pragma unroll
      for (int j = 0; j < N; ++j) gi[i * N + j] = e[j];
    }
  };
  if (!k.kept()) {
    if (threadIdx.x == 0 && rank == 0) p.terms[t] = p.logp[t] = p.lse[t] = p.coef[t] = 0.f;
    if (g) {
      for (int i = threadIdx.x; i < n; i += THREADS) store(i, make_uint4(0u, 0u, 0u, 0u));
      if (edge >= 0) g[edge] = Elem<T>::put(0.f);
    }
    return;  // (the whole cluster)
  }
  if (!k.valid(p.vocab) && rank == 0 && threadIdx.x == 0 && p.status) atomicOr(p.status, FE_ST_INDEX);
  const T xy = x[k.valid(p.vocab) ? k.y : 0], xe = x[edge >= 0 ? edge : 0];
  const uint64_t c2 = f32x2_pack(p.c, p.c);
  MaxSum v = {-INFINITY, 0.f};
  const int kn = keep * THREADS;
  for (int i0 = threadIdx.x; i0 < n; i0 += AHEAD * THREADS) {
    uint4 w[AHEAD];
#pragma unroll
    for (int z = 0; z < AHEAD; ++z)
      if (i0 + z * THREADS < n) w[z] = ld_hint(xi + (i0 + z * THREADS) * N, i0 + z * THREADS < kn ? leave : hold);
#pragma unroll
    for (int z = 0; z < AHEAD; ++z)
      if (i0 + z * THREADS < min(n, kn)) held[i0 + z * THREADS] = w[z];
    float m = v.m;
#pragma unroll
    for (int z = 0; z < AHEAD; ++z)
      if (i0 + z * THREADS < n) m = piece_max<T>(w[z], m);
    const uint64_t nb = f32x2_pack(-base_of(m), -base_of(m));
    uint64_t sum[2] = {0ull, 0ull};
#pragma unroll
    for (int z = 0; z < AHEAD; ++z)
      if (i0 + z * THREADS < n) piece_sum<T>(w[z], nb, c2, sum);
    v.s = rebase(v.s, v.m, m, p.c) + sum_of(sum);
    v.m = m;
  }
  const float ze = edge >= 0 ? Elem<T>::get(xe) : -INFINITY;
  v = join(v, MaxSum{ze, ze == -INFINITY ? 0.f : 1.f}, p.c);
  v = block_join<THREADS>(v, p.c, sh);
  if (cs > 1) {
    if (threadIdx.x < cs) peer_put(&s_peers[rank], threadIdx.x, v);
    cluster_arrive();
    cluster_wait();
    v = lane < cs ? s_peers[lane] : MaxSum{-INFINITY, 0.f};
    v = warp_join<32>(v, p.c);
  }
  const float kf = row_outputs(p, t, k, Elem<T>::get(xy), v, rank == 0 && threadIdx.x == 0);
  if (!g) return;
  const float f = -kf * (1.f / v.s), b = base_of(v.m);
  const uint64_t nb = f32x2_pack(-b, -b);
  const int y0 = k.y - rs.head - from * N;
  for (int i0 = threadIdx.x + kn; i0 < n; i0 += AHEAD * THREADS) {
    uint4 w[AHEAD];
#pragma unroll
    for (int z = 0; z < AHEAD; ++z)
      if (i0 + z * THREADS < n) w[z] = ld_hint(xi + (i0 + z * THREADS) * N, leave);
#pragma unroll
    for (int z = 0; z < AHEAD; ++z) {
      const int i = i0 + z * THREADS;
      if (i < n) store(i, piece_grad<T>(w[z], nb, c2, f, kf, y0 - i * N));
    }
  }
#pragma unroll 2
  for (int i = threadIdx.x; i < min(n, kn); i += THREADS) store(i, piece_grad<T>(held[i], nb, c2, f, kf, y0 - i * N));
  if (edge >= 0) g[edge] = Elem<T>::put(fmaf(f, ex2_approx((ze - b) * p.c), edge == k.y ? kf : 0.f));
}

// The gradient from a saved lse and coef
template <typename T>
__global__ void __launch_bounds__(kThreads) policy_backward_kernel(const PolicyParams p) {
  pdl_trigger();
  pdl_wait();
  const int t = blockIdx.x;
  const Token k = token_of(p, t);
  T* g = reinterpret_cast<T*>(p.grad) + (long long)t * p.grad_row;
  if (!k.kept()) {
    zero_row<kThreads>(g, p.vocab);
    return;
  }
  if (!k.valid(p.vocab) && threadIdx.x == 0 && p.status) atomicOr(p.status, FE_ST_INDEX);
  const T* x = reinterpret_cast<const T*>(p.logits) + (long long)t * p.logits_row;
  const float f = __ldg(p.coef + t) * p.scale * p.inv_t * (p.upstream ? __ldg(p.upstream) : 1.f);
  grad_row(x, g, p.vocab, k.y, f, p.c, __ldg(p.lse + t) * p.t, 1.f);
}

// loss = sum of the terms: each thread its own in turn, then a tree, in 64 bits
// (fp64 additions are slow here, half a microsecond for a thousand: many rows are spread over a cluster's SMs, 5 us
// for 16384 terms where one CTA of 1024 threads took 13: its shuffles alone add 5000 times)
constexpr int kSumThreads = 256, kSumCtas = 8;
__global__ void __launch_bounds__(kSumThreads) policy_sum_kernel(const float* terms, int rows, float* loss) {
  constexpr int W = kSumThreads / 32;
  __shared__ double sh[W], s_parts[kSumCtas];
  pdl_trigger();
  cluster_arrive();
  pdl_wait();
  const int rank = blockIdx.x, step = gridDim.x * kSumThreads;
  double s = 0.0;
#pragma unroll 8
  for (int i = rank * kSumThreads + threadIdx.x; i < rows; i += step) s += (double)terms[i];
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
  if ((threadIdx.x & 31) == 0) sh[threadIdx.x >> 5] = s;
  __syncthreads();
  cluster_wait();  // (every CTA has begun)
  if (threadIdx.x == 0) {
    s = sh[0];
    for (int i = 1; i < W; ++i) s += sh[i];
    uint32_t at;
    asm volatile("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(at) : "r"(smem_u32(s_parts + rank)));
    asm volatile("st.shared::cluster.f64 [%0], %1;" ::"r"(at), "d"(s) : "memory");
  }
  __syncwarp();
  cluster_arrive();
  cluster_wait();
  if (rank == 0 && threadIdx.x == 0) {
    s = s_parts[0];
    for (int i = 1; i < (int)gridDim.x; ++i) s += s_parts[i];
    *loss = (float)s;
  }
}

constexpr int kKeepLong = 8, kKeepShort = 13;  // pieces a thread keeps: 64 KB of 512 threads, 52 KB of 256
template <typename T>
cudaError_t allow_smem() {
  cudaError_t e = cudaFuncSetAttribute((const void*)policy_kernel<T, 512, 3, 2>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                       kKeepLong * 512 * 16);
  if (e == cudaSuccess)
    e = cudaFuncSetAttribute((const void*)policy_kernel<T, 256, 4, 4>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                             kKeepShort * 256 * 16);
  return e;
}
struct Device {
  int sms = 0;
  cudaError_t err = cudaErrorUnknown;
};
// Once per device: its SMs and the kernels' shared-memory limits.
const Device& device() {
  static Device devs[64];
  static std::once_flag once[64];
  static const Device none;
  int d = 0;
  if (cudaGetDevice(&d) != cudaSuccess || d < 0 || d >= 64) return none;
  std::call_once(once[d], [d] {
    Device& v = devs[d];
    v.err = cudaDeviceGetAttribute(&v.sms, cudaDevAttrMultiProcessorCount, d);
    for (cudaError_t (*f)() : {allow_smem<__nv_bfloat16>, allow_smem<__half>, allow_smem<float>})
      if (v.err == cudaSuccess) v.err = f();
  });
  return devs[d];
}

template <typename T>
cudaError_t policy_go(const PolicyParams& p, cudaStream_t s) {
  constexpr int N = Elem<T>::N;
  const Device& dev = device();
  if (dev.err != cudaSuccess) return dev.err;
  const int pieces = (p.vocab + N - 1) / N;
  // a gradient whose rows start elsewhere between two 16-byte boundaries cannot leave in 16-byte pieces
  const bool aligned = !p.grad || ((((uintptr_t)p.grad ^ (uintptr_t)p.logits) & 15) == 0 && (p.grad_row - p.logits_row) % N == 0);
  if (aligned && pieces <= 512 * 8) {  // a CTA's threads by the pieces that each holds
    const dim3 g((unsigned)p.rows);
    if (pieces <= 32 * 4) return launch_k(policy_row_kernel<T, 32, 4>, g, dim3(32), 0, s, p);
    if (pieces <= 64 * 4) return launch_k(policy_row_kernel<T, 64, 4>, g, dim3(64), 0, s, p);
    if (pieces <= 128 * 4) return launch_k(policy_row_kernel<T, 128, 4>, g, dim3(128), 0, s, p);
    if (pieces <= 128 * 8) return launch_k(policy_row_kernel<T, 128, 8>, g, dim3(128), 0, s, p);
    if (pieces <= 256 * 6) return launch_k(policy_row_kernel<T, 256, 6>, g, dim3(256), 0, s, p);
    if (pieces <= 256 * 8) return launch_k(policy_row_kernel<T, 256, 8>, g, dim3(256), 0, s, p);
    if (pieces <= 512 * 6) return launch_k(policy_row_kernel<T, 512, 6>, g, dim3(512), 0, s, p);
    return launch_k(policy_row_kernel<T, 512, 8>, g, dim3(512), 0, s, p);
  }
  // few rows: several CTAs each, as long as every thread has a piece
  int cs = 1;
  while (cs < 8 && (long long)p.rows * cs < 2 * dev.sms && pieces >= cs * 1024) cs *= 2;
  const int per = (pieces + cs - 1) / cs;
  auto go = [&](auto kern, int threads, int most) {
    const int keep = !p.grad ? 0 : std::min(most, (per + threads - 1) / threads);
    return launch_kc(kern, dim3((unsigned)(p.rows * cs)), dim3((unsigned)threads), (size_t)keep * threads * 16, s, cs, p, cs, keep);
  };
  return per <= 4096 ? go(policy_kernel<T, 256, 4, 4>, 256, kKeepShort) : go(policy_kernel<T, 512, 3, 2>, 512, kKeepLong);
}

int check_policy(const fe_policy_args* a) {
  if (!a) return fail(FE_ERR_INVALID_ARG, "null arguments");
  if (a->rows < 0 || a->vocab < 1) return fail(FE_ERR_INVALID_ARG, "negative rows or empty vocabulary");
  if (a->dtype != FE_IO_BF16 && a->dtype != FE_IO_F16 && a->dtype != FE_IO_F32)
    return fail(FE_ERR_UNSUPPORTED, "logits must be bf16, f16 or fp32");
  if (!(a->temperature > 0.f) || !std::isfinite(a->temperature) || !std::isfinite(1.f / a->temperature))
    return fail(FE_ERR_INVALID_ARG, "temperature must be positive and finite");
  if (!std::isfinite(a->grad_scale)) return fail(FE_ERR_INVALID_ARG, "grad_scale must be finite");
  if (a->rows == 0) return FE_OK;
  const unsigned e = a->dtype == FE_IO_F32 ? 4 : 2;
  if (!a->logits || !a->tokens || !a->lse || !a->coef) return fail(FE_ERR_INVALID_ARG, "null pointer");
  if (misaligned(a->logits, e) || (a->grad && misaligned(a->grad, e)))
    return fail(FE_ERR_INVALID_ARG, "logits or grad not aligned to their type");
  if (a->logits_row < a->vocab || (a->grad && a->grad_row < a->vocab))
    return fail(FE_ERR_INVALID_ARG, "rows overlap");
  if (a->grad == a->logits && a->grad_row != a->logits_row)
    return fail(FE_ERR_INVALID_ARG, "grad in place of logits needs the same stride");
  return FE_OK;
}

PolicyParams policy_params(const fe_policy_args* a, const float* upstream) {
  PolicyParams p{};
  p.logits = a->logits;
  p.grad = a->grad;
  p.tokens = a->tokens;
  p.adv = a->advantages;
  p.weights = a->weights;
  p.old_logp = a->old_logp;
  p.ref_logp = a->ref_logp;
  p.upstream = upstream;
  p.terms = a->terms;
  p.logp = a->logp;
  p.lse = a->lse;
  p.coef = a->coef;
  p.status = a->status;
  p.logits_row = a->logits_row;
  p.grad_row = a->grad_row;
  p.rows = a->rows;
  p.vocab = a->vocab;
  p.lo = a->clip_low;
  p.hi = a->clip_high;
  p.beta = a->beta;
  p.t = a->temperature;
  p.inv_t = 1.f / a->temperature;
  p.scale = a->grad_scale;
  p.c = (float)(1.4426950408889634 / (double)a->temperature);
  return p;
}

}  // namespace
}  // namespace fe

extern "C" int fe_policy_loss(const fe_policy_args* a, void* stream) {
  using namespace fe;
  const int rc = check_policy(a);
  if (rc != FE_OK) return rc;
  if (!a->loss) return fail(FE_ERR_INVALID_ARG, "null pointer");
  if (a->rows > 0 && (!a->advantages || !a->terms || !a->logp)) return fail(FE_ERR_INVALID_ARG, "null pointer");
  if (!(a->clip_low >= 0.f && a->clip_low <= 1.f) || !(a->clip_high >= 0.f) || !std::isfinite(a->beta))
    return fail(FE_ERR_INVALID_ARG, "clip_low must be in [0, 1], clip_high at least 0, beta finite");
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  const PolicyParams p = policy_params(a, nullptr);
  cudaError_t e = cudaSuccess;
  if (a->rows > 0)
    e = a->dtype == FE_IO_F32 ? policy_go<float>(p, s) : a->dtype == FE_IO_BF16 ? policy_go<__nv_bfloat16>(p, s) : policy_go<__half>(p, s);
  const int cs = a->rows > 8 * kSumThreads ? kSumCtas : 1;
  if (e == cudaSuccess)
    e = launch_kc(policy_sum_kernel, dim3((unsigned)cs), dim3(kSumThreads), 0, s, cs, (const float*)a->terms, a->rows, a->loss);
  return e == cudaSuccess ? FE_OK : fail_cuda(e, "fe_policy_loss");
}

extern "C" int fe_policy_loss_backward(const fe_policy_args* a, const float* upstream, void* stream) {
  using namespace fe;
  const int rc = check_policy(a);
  if (rc != FE_OK) return rc;
  if (a->rows == 0) return FE_OK;
  if (!a->grad) return fail(FE_ERR_INVALID_ARG, "null pointer");
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  const PolicyParams p = policy_params(a, upstream);
  const dim3 g((unsigned)a->rows), b(kThreads);
  const cudaError_t e = a->dtype == FE_IO_F32    ? launch_k(policy_backward_kernel<float>, g, b, 0, s, p)
                        : a->dtype == FE_IO_BF16 ? launch_k(policy_backward_kernel<__nv_bfloat16>, g, b, 0, s, p)
                                                 : launch_k(policy_backward_kernel<__half>, g, b, 0, s, p);
  return e == cudaSuccess ? FE_OK : fail_cuda(e, "fe_policy_loss_backward");
}
