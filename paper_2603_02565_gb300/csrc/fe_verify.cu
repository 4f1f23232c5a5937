// Which drafted tokens the target's probabilities accept, and the token drawn after them
// (fe_verify_drafts).
//
// Row t of a sequence that is the first not to be accepted, or its last, is the one that a token is
// drawn from: w = p, or max(p - q, 0) (p without y where there is no q) after a rejection, and
//   the first i with sum_{k <= i} w_k > u sum_k w_k.
// A whole number comes out, so the sums have to be alike however they are split: each w goes
// into them as a whole number of units of 2^-45.  Adding 1 rounds p - q to 2^-23, and adding a small constant to what is left over
// of it (within 2^-24 + 2^-25) rounds that to 2^-45; 32-bit integer sums of both parts are exact, and need no 64-bit float, of
// which the GPU has two a clock and SM.
//
// A cluster of CTAs has a sequence, each a run of its row's 16-byte pieces, each warp a run of that.
// The CTAs add up their sums through shared memory, the warp whose run has the threshold goes
// through it again (from L2), 32 pieces a step.
//
// What bounds it: for few sequences a chain of steps (offsets, tokens, their probabilities; the sums; the cluster; the search),
// for many the instructions of the sums as well: 7 an element, two at a time.  GB300, a call alone in a replayed graph, caches
// flushed, here and below: one row of 100003 bf16 14.5 us; 200 sequences of up to 5 drafts over 131072 fp32, with draft
// probabilities, 54.5 us (bytes at a copy's rate: 31); 500 of up to 7 over 32768 f16, without, 25.5 us (4.8).
#include <algorithm>

#include "fe_kernels.h"
#include "fe_ops.cuh"

namespace fe {
namespace {

struct VerifyParams {
  const void *target, *draft;
  const int32_t *tokens, *row_start;
  const float *accept, *sample;
  int32_t *out, *accepted, *status;
  int64_t target_row, draft_row;
  int n_seqs, n_rows, vocab;
};

constexpr int kThreads = 256, kWarps = kThreads / 32, kMaxCluster = 8;
// CTAs an SM: registers for several loads at once.  (Six, with half the loads of fp32: a row of 131072 24 us instead of 18, 200 of them
// 60.5 instead of 55; 500 of 32768 f16 34 instead of 26, and with four loads instead of two 30.)
constexpr int kCtas = 4;
constexpr uint32_t kOne = 0x3f800000u;

struct Sum {
  unsigned long long hi;  // units of 2^-23
  long long lo;           // units of 2^-45
  __device__ __forceinline__ unsigned long long all() const { return (hi << 22) + (unsigned long long)lo; }
};

// A w in [0, 1] added to kTop leaves it in steps of 2^-23 in the sum's last bits (2, the end of the range, follows on from those below
// it).  What is left over, up to half such a step and what 32 bits could not hold of p - q (2^-25 at most), added to kLow, leaves
// that in steps of 2^-45: the sum stays within 2^-22 .. 2^-21, where such steps are.
constexpr float kTop = 1.f, kLow = 0x1.8p-22f;
constexpr uint32_t kTopBits = 0x3f800000u, kLowBits = 0x34c00000u;

// What a token is drawn from: with q max(p - q, 0), otherwise p, and 0 at `but`
template <typename T>
struct Weights {
  static constexpr int N = 16 / (int)sizeof(T);
  const T *p, *q;
  int vocab, mis, but;  // mis: elements from the 16-byte boundary before p to p
  bool whole;           // p and q lie alike on 16-byte boundaries

  __device__ __forceinline__ int pieces() const { return (vocab + mis + N - 1) / N; }
  // Two w of values p and their q, in parts, and the constants that these bring; worst: the largest probability's bits
  template <bool Q>
  __device__ __forceinline__ static void weights(float x0, float x1, float y0, float y1, uint32_t& hi, uint32_t& lo, uint32_t& worst) {
    const uint64_t top = f32x2_pack(kTop, kTop), low = f32x2_pack(kLow, kLow), one = f32x2_pack(-1.f, -1.f);
    worst = max(max(worst, __float_as_uint(x0)), __float_as_uint(x1));
    const uint64_t m = Q ? f32x2_pack(fmaxf(x0, y0), fmaxf(x1, y1)) : f32x2_pack(x0, x1);
    uint64_t w = m, q = 0;
    if (Q) {  // max(p - q, 0) as max(p, q) - q
      worst = max(max(worst, __float_as_uint(y0)), __float_as_uint(y1));
      q = f32x2_pack(y0, y1);
      w = f32x2_fma(q, one, m);
    }
    const uint64_t a = f32x2_add(w, top);
    // m less the rounded w is exact: a multiple of m's last bit, and no larger than m or 2^-24.  Less q it is rounded, by 2^-48 at most.
    uint64_t left = f32x2_fma(f32x2_fma(top, one, a), one, m);
    if (Q) left = f32x2_fma(q, one, left);
    const uint64_t b = f32x2_add(left, low);
    float a0, a1, b0, b1;
    f32x2_unpack(a, a0, a1);
    f32x2_unpack(b, b0, b1);
    hi += __float_as_uint(a0) + __float_as_uint(a1);
    lo += __float_as_uint(b0) + __float_as_uint(b1);
  }
  // Pieces ka + lane, ka + lane + 32, ... below kb, all of them whole; `but` is not looked for
  template <bool Q>
  __device__ __forceinline__ void add_whole(int ka, int kb, Sum& v, uint32_t& worst) const {
    constexpr int U = sizeof(T) == 2 ? 2 : Q ? 4 : 8;  // loads of each at once (a piece of 16 bits is eight numbers)
    const uint4* from = reinterpret_cast<const uint4*>(p - mis);
    const uint4* less = reinterpret_cast<const uint4*>(q - (Q ? mis : 0));
    for (int k = ka + (int)(threadIdx.x & 31); k < kb; k += 32 * U) {
      uint4 x[U], y[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const bool in = k + 32 * u < kb;
        x[u] = in ? __ldg(from + k + 32 * u) : make_uint4(0u, 0u, 0u, 0u);
        if (Q) y[u] = in ? __ldg(less + k + 32 * u) : make_uint4(0u, 0u, 0u, 0u);
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        float a[N], b[N];
        piece_get<T>(x[u], a);
        if (Q) piece_get<T>(y[u], b);
        uint32_t hi = 0u - N * kTopBits, lo = 0u - N * kLowBits;
#pragma unroll
        for (int i = 0; i < N; i += 2) weights<Q>(a[i], a[i + 1], Q ? b[i] : 0.f, Q ? b[i + 1] : 0.f, hi, lo, worst);
        v.hi += hi;
        v.lo += (int32_t)lo;
      }
    }
  }
  // piece k: its sum, or that of its first `upto` elements
  __device__ __forceinline__ void add(int k, int upto, uint32_t& hi, int32_t& lo, uint32_t& worst) const {
    const long long e0 = (long long)k * N - mis;
    float x[N], y[N];
    if (whole && e0 >= 0 && e0 + N <= vocab) {
      piece_get<T>(__ldg(reinterpret_cast<const uint4*>(p + e0)), x);
      if (q) piece_get<T>(__ldg(reinterpret_cast<const uint4*>(q + e0)), y);
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const bool in = e0 + i >= 0 && e0 + i < vocab;
        x[i] = in ? Elem<T>::get(p[e0 + i]) : 0.f;
        if (q) y[i] = in ? Elem<T>::get(q[e0 + i]) : 0.f;
      }
    }
    uint32_t h = 0u - N * kTopBits, l = 0u - N * kLowBits;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      x[i] = i < upto ? __fadd_rn(x[i], 0.f) : 0.f;  // (no -0)
      if (e0 + i == but) {
        worst = max(worst, __float_as_uint(x[i]));
        x[i] = 0.f;
      }
      y[i] = q && i < upto ? __fadd_rn(y[i], 0.f) : 0.f;
    }
#pragma unroll
    for (int i = 0; i < N; i += 2) weights<true>(x[i], x[i + 1], y[i], y[i + 1], h, l, worst);
    hi += h;
    lo += (int32_t)l;
  }
};

__device__ __forceinline__ unsigned long long warp_sum(unsigned long long v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_sync_all() {
  cluster_arrive();
  cluster_wait();
}
__device__ __forceinline__ uint32_t cluster_rank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ unsigned long long remote_u64(const void* p, uint32_t rank) {
  uint32_t at;
  unsigned long long v;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(smem_u32(p)), "r"(rank));
  asm volatile("ld.shared::cluster.u64 %0, [%1];" : "=l"(v) : "r"(at) : "memory");
  return v;
}

template <typename T>
__global__ void __launch_bounds__(kThreads, kCtas) verify_kernel(const VerifyParams p, const int cluster) {
  __shared__ unsigned long long sh_hi[kWarps];
  __shared__ long long sh_lo[kWarps];
  __shared__ uint32_t sh_worst[kWarps];
  __shared__ unsigned long long total[3];  // the CTA's, for the others: hi, lo, worst
  __shared__ int sh_accepted;
  pdl_trigger();
  pdl_wait();
  const int s = blockIdx.x / cluster, rank = (int)cluster_rank(), lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const bool first = rank == 0 && threadIdx.x == 0;
  const int a = p.row_start[s], b = p.row_start[s + 1], n = b - a - 1;
  if (a < 0 || b > p.n_rows || b <= a) {  // (the whole cluster)
    if (first) {
      p.accepted[s] = 0;
      if (!(a == b && a >= 0 && b <= p.n_rows) && p.status) atomicOr(p.status, FE_ST_INDEX);
    }
    return;
  }
  const T *target = static_cast<const T*>(p.target), *draft = static_cast<const T*>(p.draft);
  if (warp == 0) {
    int got = n;
    for (int j0 = 0; j0 < n; j0 += 32) {
      const int t = a + j0 + lane;
      bool ok = j0 + lane >= n;
      if (!ok) {
        const int y = p.tokens[t];
        if (y >= 0 && y < p.vocab) {
          // (the product of two 24-bit numbers is exact in 64 bits)
          const double q = draft ? (double)Elem<T>::get(draft[(long long)t * p.draft_row + y]) : 1.0;
          ok = (double)p.accept[t] * q < (double)Elem<T>::get(target[(long long)t * p.target_row + y]);
        }
      }
      const uint32_t no = __ballot_sync(0xffffffffu, !ok);
      if (no) {
        got = j0 + __ffs(no) - 1;
        break;
      }
    }
    if (lane == 0) sh_accepted = got;
  }
  __syncthreads();
  const int accepted = sh_accepted, t = a + accepted;
  const bool rejected = accepted < n;
  const int y = rejected ? p.tokens[t] : 0;
  const float u = p.sample[s];
  if (rank == 0) {
    if (threadIdx.x == 0) p.accepted[s] = accepted;
    for (int i = a + threadIdx.x; i < b; i += kThreads)
      if (i != t) p.out[i] = i < t ? p.tokens[i] : -1;
  }
  if (y < 0 || y >= p.vocab || !(u >= 0.f && u < 1.f)) {
    if (first) {
      p.out[t] = -1;
      if (p.status) atomicOr(p.status, FE_ST_INDEX);
    }
    return;
  }
  Weights<T> w;
  w.p = target + (long long)t * p.target_row;
  w.q = rejected && draft ? draft + (long long)t * p.draft_row : nullptr;
  w.vocab = p.vocab;
  w.mis = (int)((reinterpret_cast<uintptr_t>(w.p) & 15u) / sizeof(T));
  w.whole = !w.q || ((reinterpret_cast<uintptr_t>(w.q) ^ reinterpret_cast<uintptr_t>(w.p)) & 15u) == 0;
  w.but = rejected && !draft ? y : -1;
  const int pieces = w.pieces(), runs = cluster * kWarps, each = (pieces + runs - 1) / runs;
  const int k0 = min(pieces, (rank * kWarps + warp) * each), k1 = min(pieces, k0 + each);
  uint32_t worst = 0;
  auto one = [&](int k, Sum& v) {
    uint32_t hi = 0;
    int32_t lo = 0;
    w.add(k, Weights<T>::N, hi, lo, worst);
    v.hi += hi;
    v.lo += lo;
  };
  Sum all;
  unsigned long long before;
  bool careful = false, again = false;
  while (true) {
    Sum v = {0, 0};
    worst = 0;
    // whole pieces, but for the row's ends and that of a token left out
    int ka = k0, kb = k0;
    if (w.whole && !careful) {
      ka = max(k0, w.mis > 0 ? 1 : 0);
      kb = max(ka, min(k1, (w.vocab + w.mis) / Weights<T>::N));
      if (ka > k0 && k1 > k0 && lane == 0) one(k0, v);
      if (w.q) {
        w.template add_whole<true>(ka, kb, v, worst);
      } else {
        const int out = w.but < 0 ? kb : min(kb, max(ka, (w.but + w.mis) / Weights<T>::N));
        w.template add_whole<false>(ka, out, v, worst);
        if (out < kb && lane == 0) one(out, v);
        w.template add_whole<false>(out + 1, kb, v, worst);
      }
      ka = kb;
    }
    for (int k = ka + lane; k < k1; k += 32) one(k, v);
    v.hi = warp_sum(v.hi);
    v.lo = (long long)warp_sum((unsigned long long)v.lo);
    worst = __reduce_max_sync(0xffffffffu, worst);
    if (lane == 0) {
      sh_hi[warp] = v.hi;
      sh_lo[warp] = v.lo;
      sh_worst[warp] = worst;
    }
    __syncthreads();
    if (warp == 0) {
      const bool in = lane < kWarps;
      const unsigned long long hi = warp_sum(in ? sh_hi[lane] : 0), lo = warp_sum(in ? (unsigned long long)sh_lo[lane] : 0);
      const uint32_t wo = __reduce_max_sync(0xffffffffu, in ? sh_worst[lane] : 0u);
      if (lane == 0) {
        total[0] = hi;
        total[1] = lo;
        total[2] = wo;
      }
    }
    cluster_sync_all();
    {  // a CTA's sums a lane
      Sum x = {0, 0};
      uint32_t wo = 0;
      if (lane < cluster) {
        x.hi = remote_u64(total, lane);
        x.lo = (long long)remote_u64(total + 1, lane);
        wo = (uint32_t)remote_u64(total + 2, lane);
      }
      all = {warp_sum(x.hi), (long long)warp_sum((unsigned long long)x.lo)};
      before = warp_sum(lane < rank ? x.all() : 0);
      worst = __reduce_max_sync(0xffffffffu, wo);
    }
    cluster_arrive();  // (these sums have been read)
    if (worst > kOne) {
      if (careful) break;
      careful = true;  // -0 may be all that is wrong
    } else {
      // nothing above 0 after a rejection: p itself
      if (again || !rejected || all.all() != 0) break;
      again = true;
      w.q = nullptr;
      w.but = -1;
    }
    cluster_wait();
  }
  const unsigned long long sum = all.all();
  // (units of 2^-45 of a sum below 2^17 fit 64 bits)
  if (worst > kOne || sum == 0 || (all.hi >> (23 + 17)) != 0) {
    if (first) {
      p.out[t] = -1;
      if (p.status) atomicOr(p.status, FE_ST_INDEX);
    }
  } else {
    const unsigned long long bound = __umul64hi((unsigned long long)((double)u * 18446744073709551616.0), sum);
    for (int i = 0; i < warp; ++i) before += Sum{sh_hi[i], sh_lo[i]}.all();
    if (before <= bound && before + Sum{sh_hi[warp], sh_lo[warp]}.all() > bound) {
      for (int k = k0; k < k1; k += 32) {
        uint32_t hi = 0, unused = 0;
        int32_t lo = 0;
        if (k + lane < k1) w.add(k + lane, Weights<T>::N, hi, lo, unused);
        unsigned long long c = Sum{hi, lo}.all();
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
          const unsigned long long x = __shfl_up_sync(0xffffffffu, c, o);
          if (lane >= o) c += x;
        }
        const uint32_t past = __ballot_sync(0xffffffffu, before + c > bound);
        if (past) {
          const int l = __ffs(past) - 1;
          const unsigned long long up = __shfl_sync(0xffffffffu, c, max(l - 1, 0));
          if (l > 0) before += up;
          // an element a lane: the sum of the piece up to it
          hi = 0, lo = 0;
          if (lane < Weights<T>::N) w.add(k + l, lane + 1, hi, lo, unused);
          const uint32_t at = __ballot_sync(0xffffffffu, lane < Weights<T>::N && before + Sum{hi, lo}.all() > bound);
          if (lane == 0) p.out[t] = (k + l) * Weights<T>::N - w.mis + __ffs(at) - 1;
          break;
        }
        before += __shfl_sync(0xffffffffu, c, 31);
      }
    }
  }
  __syncwarp();
  cluster_wait();  // (nobody leaves while others read its sums)
}

template <typename T>
cudaError_t verify_go(const VerifyParams& p, cudaStream_t s) {
  // CTAs a sequence: as many as the SMs hold at once, as long as each thread has a piece of 16 bytes; and until it has no more than
  // 16.  (200 sequences x 131072 fp32: 55 us with eight CTAs each, 60 with four, 81 with two; 500 x 32768 f16, which is 16 pieces: 26
  // with one, 30 with two, 40 with four; 500 x 50257 f16: 38 with two, 36 with one.  So the step past 16 costs some 4 of 28 us.)
  int cluster = 1, sms = 0;
  const cudaError_t e = device_sms(&sms);
  if (e != cudaSuccess) return e;
  const long long pieces = (long long)p.vocab * (int)sizeof(T) / 16;
  while (cluster < kMaxCluster &&
         (pieces > 16LL * kThreads * cluster ||
          (pieces > (long long)kThreads * cluster && 2LL * p.n_seqs * cluster <= (long long)kCtas * sms)))
    cluster *= 2;
  const dim3 grid((unsigned)p.n_seqs * cluster);
  return launch_kc(verify_kernel<T>, grid, dim3(kThreads), 0, s, cluster, p, cluster);
}

}  // namespace
}  // namespace fe

extern "C" int fe_verify_drafts(const fe_verify_args* a, void* stream) {
  using namespace fe;
  if (!a) return fail(FE_ERR_INVALID_ARG, "null arguments");
  if (a->n_seqs < 0 || a->n_rows < 0 || a->vocab < 1) return fail(FE_ERR_INVALID_ARG, "negative size or empty vocabulary");
  if (a->dtype != FE_IO_BF16 && a->dtype != FE_IO_F16 && a->dtype != FE_IO_F32)
    return fail(FE_ERR_UNSUPPORTED, "probabilities must be bf16, f16 or fp32");
  if (a->n_seqs == 0) return a->n_rows == 0 ? FE_OK : fail(FE_ERR_INVALID_ARG, "rows without a sequence");
  if (a->n_seqs > (1 << 27)) return fail(FE_ERR_UNSUPPORTED, "at most 2^27 sequences");
  if (a->vocab > 0x7ffffff0) return fail(FE_ERR_UNSUPPORTED, "vocabulary too large");
  if (!a->row_start || !a->accepted || !a->sample) return fail(FE_ERR_INVALID_ARG, "null pointer");
  if (a->n_rows > 0 && (!a->target || !a->tokens || !a->accept || !a->out)) return fail(FE_ERR_INVALID_ARG, "null pointer");
  if (a->out && a->out == a->tokens) return fail(FE_ERR_INVALID_ARG, "out must not be tokens");
  const unsigned size = a->dtype == FE_IO_F32 ? 4 : 2;
  if (misaligned(a->target, size) || misaligned(a->draft, size))
    return fail(FE_ERR_INVALID_ARG, "probabilities must be aligned to their type");
  if (a->target_row < a->vocab || (a->draft && a->draft_row < a->vocab))
    return fail(FE_ERR_INVALID_ARG, "rows must not overlap");
  VerifyParams p{};
  p.target = a->target;
  p.draft = a->draft;
  p.tokens = a->tokens;
  p.row_start = a->row_start;
  p.accept = a->accept;
  p.sample = a->sample;
  p.out = a->out;
  p.accepted = a->accepted;
  p.status = a->status;
  p.target_row = a->target_row;
  p.draft_row = a->draft_row;
  p.n_seqs = a->n_seqs;
  p.n_rows = a->n_rows;
  p.vocab = a->vocab;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  const cudaError_t e = a->dtype == FE_IO_BF16  ? verify_go<__nv_bfloat16>(p, s)
                        : a->dtype == FE_IO_F16 ? verify_go<__half>(p, s)
                                                : verify_go<float>(p, s);
  return e == cudaSuccess ? FE_OK : fail_cuda(e, "fe_verify_drafts");
}
