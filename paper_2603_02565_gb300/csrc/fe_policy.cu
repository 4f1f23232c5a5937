// Clipped policy loss with a KL term over a vocabulary, and its gradient
// (fe_policy_loss, fe_policy_loss_backward).
//
// With e_v = 2^((x_v - m) c), c = log2(e) / temperature and m the row's maximum,
//   logp = ((x_y - m) c - log2 sum e) ln 2,   softmax_v = e_v / sum e,
//   grad_v = k (1[v = y] - softmax_v),  k = grad_scale coef / temperature.
// The maximum comes off before the product, so the exponents' errors are relative to the
// distance from it.  All of it is fp32; a gradient is rounded once.
#include <cmath>

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

constexpr int kThreads = 512;
constexpr float kLn2 = 0.693147180559945309f;

// Running maximum and sum of 2^((x - m) c), m -inf as long as nothing else has come
struct MaxSum {
  float m, s;
};
__device__ __forceinline__ float base_of(float m) { return m == -INFINITY ? 0.f : m; }
// a sum against maximum m0 as one against m >= m0
__device__ __forceinline__ float rebase(float s, float m0, float m, float c) {
  return m0 == -INFINITY ? 0.f : s * ex2_approx((m0 - m) * c);
}
__device__ __forceinline__ MaxSum join(MaxSum a, MaxSum b, float c) {
  const float m = fmaxf(a.m, b.m);
  return {m, rebase(a.s, a.m, m, c) + rebase(b.s, b.m, m, c)};
}

__device__ __forceinline__ MaxSum block_join(MaxSum v, float c, MaxSum* sh) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    MaxSum w = {__shfl_xor_sync(0xffffffffu, v.m, o), __shfl_xor_sync(0xffffffffu, v.s, o)};
    v = join(v, w, c);
  }
  if ((threadIdx.x & 31) == 0) sh[threadIdx.x >> 5] = v;
  __syncthreads();
  v = sh[0];
  for (int i = 1; i < kThreads / 32; ++i) v = join(v, sh[i], c);
  return v;
}

// What row t's token asks for: weight, whether it takes part, its index
struct Token {
  float w;
  int y;
  bool kept, valid;
};
__device__ __forceinline__ Token token_of(const PolicyParams& p, int t) {
  Token k;
  k.w = p.weights ? __ldg(p.weights + t) : 1.f / (float)p.rows;
  k.y = __ldg(p.tokens + t);
  k.kept = k.w != 0.f;
  k.valid = k.y >= 0 && k.y < p.vocab;
  return k;
}

// terms, logp, lse and coef of a row from its chosen logit and statistics; the gradient's factor
__device__ float row_outputs(const PolicyParams& p, int t, const Token& k, float xy, MaxSum v) {
  const float l2 = log2f(v.s);
  float logp = ((xy - v.m) * p.c - l2) * kLn2, lse = v.m * p.inv_t + l2 * kLn2;
  if (v.m == -INFINITY) lse = -INFINITY, logp = NAN;
  if (!k.valid) logp = NAN;
  const float a = __ldg(p.adv + t), r = p.old_logp ? expf(logp - __ldg(p.old_logp + t)) : 1.f;
  const float plain = r * a, clipped = fminf(fmaxf(r, 1.f - p.lo), 1.f + p.hi) * a;
  float term = plain <= clipped ? -plain : -clipped, coef = plain <= clipped ? -plain : 0.f;
  if (!(plain == plain)) term = coef = NAN;  // (clamping drops a NaN)
  if (p.ref_logp) {
    const float d = __ldg(p.ref_logp + t) - logp, e = expm1f(d);
    term += p.beta * (e - d);
    coef -= p.beta * e;
  }
  term *= k.w;
  coef *= k.w;
  p.terms[t] = term;
  p.logp[t] = logp;
  p.lse[t] = lse;
  p.coef[t] = coef;
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

template <typename T>
__device__ __forceinline__ void zero_row(T* g, int n) {
  for (int i = threadIdx.x; i < n; i += kThreads) g[i] = Elem<T>::put(0.f);
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

template <typename T>
__global__ void __launch_bounds__(kThreads) policy_kernel(const PolicyParams p) {
  constexpr int N = Elem<T>::N;
  __shared__ MaxSum sh[kThreads / 32];
  __shared__ float s_k, s_xy;
  pdl_trigger();
  pdl_wait();
  const int t = blockIdx.x;
  const Token k = token_of(p, t);
  T* g = p.grad ? reinterpret_cast<T*>(p.grad) + (long long)t * p.grad_row : nullptr;
  if (!k.kept) {
    if (threadIdx.x == 0) p.terms[t] = p.logp[t] = p.lse[t] = p.coef[t] = 0.f;
    if (g) zero_row(g, p.vocab);
    return;
  }
  if (!k.valid && threadIdx.x == 0 && p.status) atomicOr(p.status, FE_ST_INDEX);
  const T* x = reinterpret_cast<const T*>(p.logits) + (long long)t * p.logits_row;
  if (threadIdx.x == 0) s_xy = k.valid ? Elem<T>::get(x[k.y]) : 0.f;
  const RowSplit<T> rs(x, p.vocab);
  MaxSum v = {-INFINITY, 0.f};
  auto add = [&](const float* z, int n) {
    float m = v.m;
    for (int j = 0; j < n; ++j) m = fmaxf(m, z[j]);
    if (m != v.m) v.s = rebase(v.s, v.m, m, p.c);
    v.m = m;
    const float b = base_of(m);
    for (int j = 0; j < n; ++j) v.s += ex2_approx((z[j] - b) * p.c);
  };
  if ((int)threadIdx.x < rs.head) {
    const float z = Elem<T>::get(x[threadIdx.x]);
    add(&z, 1);
  }
  for (int i = threadIdx.x; i < rs.pieces; i += kThreads) {
    float z[N];
    piece_get<T>(*reinterpret_cast<const uint4*>(x + rs.head + i * N), z);
    add(z, N);
  }
  for (int i = rs.head + rs.pieces * N + threadIdx.x; i < p.vocab; i += kThreads) {
    const float z = Elem<T>::get(x[i]);
    add(&z, 1);
  }
  v = block_join(v, p.c, sh);
  if (threadIdx.x == 0) s_k = row_outputs(p, t, k, s_xy, v);
  __syncthreads();
  if (g) grad_row(x, g, p.vocab, k.y, s_k, p.c, base_of(v.m), 1.f / v.s);
}

// The gradient from a saved lse and coef
template <typename T>
__global__ void __launch_bounds__(kThreads) policy_backward_kernel(const PolicyParams p) {
  pdl_trigger();
  pdl_wait();
  const int t = blockIdx.x;
  const Token k = token_of(p, t);
  T* g = reinterpret_cast<T*>(p.grad) + (long long)t * p.grad_row;
  if (!k.kept) {
    zero_row(g, p.vocab);
    return;
  }
  if (!k.valid && threadIdx.x == 0 && p.status) atomicOr(p.status, FE_ST_INDEX);
  const T* x = reinterpret_cast<const T*>(p.logits) + (long long)t * p.logits_row;
  const float f = __ldg(p.coef + t) * p.scale * p.inv_t * (p.upstream ? __ldg(p.upstream) : 1.f);
  grad_row(x, g, p.vocab, k.y, f, p.c, __ldg(p.lse + t) * p.t, 1.f);
}

// loss = sum of the terms: each thread its own in turn, then a tree, in 64 bits
__global__ void __launch_bounds__(1024) policy_sum_kernel(const float* terms, int rows, float* loss) {
  __shared__ double sh[32];
  pdl_trigger();
  pdl_wait();
  double s = 0.0;
  for (int i = threadIdx.x; i < rows; i += 1024) s += (double)terms[i];
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
  if ((threadIdx.x & 31) == 0) sh[threadIdx.x >> 5] = s;
  __syncthreads();
  if (threadIdx.x < 32) {
    s = sh[threadIdx.x];
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    if (threadIdx.x == 0) *loss = (float)s;
  }
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
  const dim3 g((unsigned)a->rows), b(kThreads);
  if (a->rows > 0)
    e = a->dtype == FE_IO_F32    ? launch_k(policy_kernel<float>, g, b, 0, s, p)
        : a->dtype == FE_IO_BF16 ? launch_k(policy_kernel<__nv_bfloat16>, g, b, 0, s, p)
                                 : launch_k(policy_kernel<__half>, g, b, 0, s, p);
  if (e == cudaSuccess) e = launch_k(policy_sum_kernel, dim3(1), dim3(1024), 0, s, (const float*)a->terms, a->rows, a->loss);
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
