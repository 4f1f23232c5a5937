// Rows of ragged sequences into a paged cache, rotated by position on the way
// (fe_kv_append).
//
// out = x for values; for keys and queries pair i of a row at position p becomes
// (x c - y s, y c + x s), (c, s) = rope[p][i].  Nothing is reused, so the kernel is bound
// by memory: each element is read once and written once.
//
// One warp takes one row (or one of several parts of a row, when rows are few) and
// holds the row's cosines and sines in registers over its heads: a lane owns 16
// elements of a head, eight pairs, as two 16-byte pieces that hold both members of each
// pair (i and i + rot / 16 for halves, neighbours when interleaved), so a warp moves
// 1 KB a step and rope is read once a row, not once a head.  Rows are split into parts as
// long as all warps are on the SMs at once: 32 queries and 16 keys and values of 128, f16, a
// row each of 64 / 256 / 1024 sequences take 3.8 / 4.3 / 7.2 us (7.3 / 7.5 / 8.0 unsplit; the
// launch alone is 3), of 4096 18.4 (24 with more parts than that; 14.8 at the copy rate).
// 37 prompts of up to 8000 rows: 590 us, 6.4 TB/s of 6.8 measured for a copy.
#include <atomic>

#include "fe_ops.cuh"

namespace fe {
namespace {

struct AppendParams {
  const int32_t *row_start, *first, *shift, *pages;
  const void *k, *v, *q;
  void *k_out, *v_out, *q_out;
  const float* rope;
  int32_t* status;
  int64_t k_row, k_head, v_row, v_head, q_row, q_head;
  int n_seqs, n_rows, page_cols, hq, hkv, page_rows, n_pages, rope_rows, rot, parts;
};

template <typename T>
__device__ __forceinline__ void turn(uint4& a, uint4& b, const float* cs, bool half) {
  float x[8], y[8];
  piece_get<T>(a, x);
  piece_get<T>(b, y);
  if (half) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float u = x[i], w = y[i];
      x[i] = u * cs[2 * i] - w * cs[2 * i + 1];
      y[i] = w * cs[2 * i] + u * cs[2 * i + 1];
    }
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float u = x[2 * i], w = x[2 * i + 1];
      x[2 * i] = u * cs[2 * i] - w * cs[2 * i + 1];
      x[2 * i + 1] = w * cs[2 * i] + u * cs[2 * i + 1];
      u = y[2 * i], w = y[2 * i + 1];
      y[2 * i] = u * cs[8 + 2 * i] - w * cs[8 + 2 * i + 1];
      y[2 * i + 1] = w * cs[8 + 2 * i] + u * cs[8 + 2 * i + 1];
    }
  }
  a = piece_put<T>(x);
  b = piece_put<T>(y);
}

constexpr int kThreads = 256;
constexpr int kWarps = 32;  // that an SM holds (64 registers a thread)

template <typename T, int D, bool HALF>
__global__ void __launch_bounds__(kThreads) append_kernel(const AppendParams p) {
  constexpr int LH = D / 16, HS = 32 / LH;  // lanes of a head, heads of a step
  pdl_trigger();
  pdl_wait();
  const int lane = threadIdx.x & 31;
  const long long w = (long long)blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5);
  const int t = (int)(w / p.parts), part = (int)(w % p.parts);
  if (t >= p.n_rows) return;
  // the row's sequence: t's own when every sequence has one new row (as many rows as sequences, but t in another one
  // where some have none and others several)
  int s = t;
  if (p.n_rows != p.n_seqs || __ldg(p.row_start + t) != t || __ldg(p.row_start + t + 1) <= t)
    s = warp_find_row(p.row_start, p.n_seqs, t);
  const int j = t - __ldg(p.row_start + s);
  const long long c = (long long)__ldg(p.first + s) + j;
  const long long pos = c + (p.shift ? __ldg(p.shift + s) : 0);
  bool bad = j < 0 || t >= __ldg(p.row_start + s + 1);
  long long place = -1;  // row of the pages of head 0
  if (!bad && c >= 0 && c < (long long)p.page_cols * p.page_rows) {
    const int col = (int)(c / p.page_rows);
    const int page = __ldg(p.pages + (long long)s * p.page_cols + col);
    if (page >= 0 && page < p.n_pages) place = (long long)page * p.hkv * p.page_rows + (c - (long long)col * p.page_rows);
  }
  bad = bad || place < 0;
  const int li = lane % LH;
  const bool rotated = p.rope && 16 * li < p.rot;
  float cs[16];
#pragma unroll
  for (int i = 0; i < 16; ++i) cs[i] = 0.f;
  if (rotated) {
    const bool known = pos >= 0 && pos < p.rope_rows;
    bad = bad || !known;
    const float4* r = reinterpret_cast<const float4*>(p.rope + (known ? pos : 0) * p.rot) + 4 * li;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float4 f = __ldg(r + i);
      cs[4 * i] = known ? f.x : NAN;
      cs[4 * i + 1] = known ? f.y : NAN;
      cs[4 * i + 2] = known ? f.z : NAN;
      cs[4 * i + 3] = known ? f.w : NAN;
    }
  }
  if (bad && lane == 0 && p.status) atomicOr(p.status, FE_ST_INDEX);
  // the lane's two pieces of a head
  const int r16 = p.rope ? p.rot / 16 : 0;
  const int ea = !HALF ? 16 * li : rotated ? 8 * li : 16 * li;
  const int eb = HALF && rotated ? 8 * (li + r16) : ea + 8;
  const int total = p.hq + 2 * p.hkv;
  const T* q = reinterpret_cast<const T*>(p.q) + (long long)t * p.q_row;
  const T* k = reinterpret_cast<const T*>(p.k) + (long long)t * p.k_row;
  const T* v = reinterpret_cast<const T*>(p.v) + (long long)t * p.v_row;
  T* qo = reinterpret_cast<T*>(p.q_out) + (long long)t * p.hq * D;
  T* ko = reinterpret_cast<T*>(p.k_out) + place * D;
  T* vo = reinterpret_cast<T*>(p.v_out) + place * D;
  for (int h = part * HS + lane / LH; h < total; h += p.parts * HS) {
    const T* in;
    T* out;
    bool turned = rotated;
    if (h < p.hq) {
      in = q + h * p.q_head;
      out = qo + (long long)h * D;
    } else if (h < p.hq + p.hkv) {
      in = k + (h - p.hq) * p.k_head;
      out = place < 0 ? nullptr : ko + (long long)(h - p.hq) * p.page_rows * D;
    } else {
      in = v + (h - p.hq - p.hkv) * p.v_head;
      out = place < 0 ? nullptr : vo + (long long)(h - p.hq - p.hkv) * p.page_rows * D;
      turned = false;
    }
    uint4 a = *reinterpret_cast<const uint4*>(in + ea), b = *reinterpret_cast<const uint4*>(in + eb);
    if (turned) turn<T>(a, b, cs, HALF);
    if (out) {
      *reinterpret_cast<uint4*>(out + ea) = a;
      *reinterpret_cast<uint4*>(out + eb) = b;
    }
  }
}

template <typename T, int D>
cudaError_t append_go(const AppendParams& p, bool half, cudaStream_t s) {
  const long long warps = (long long)p.n_rows * p.parts;
  const dim3 grid((unsigned)((warps + kThreads / 32 - 1) / (kThreads / 32)));
  return half ? launch_k(append_kernel<T, D, true>, grid, dim3(kThreads), 0, s, p)
              : launch_k(append_kernel<T, D, false>, grid, dim3(kThreads), 0, s, p);
}

template <typename T>
cudaError_t append_dim(const AppendParams& p, int d, bool half, cudaStream_t s) {
  return d == 32 ? append_go<T, 32>(p, half, s) : d == 64 ? append_go<T, 64>(p, half, s) : append_go<T, 128>(p, half, s);
}

// SMs of the current device, asked for once
cudaError_t device_sms(int* sms) {
  static std::atomic<int> known[64];
  int d = 0;
  cudaError_t e = cudaGetDevice(&d);
  if (e != cudaSuccess) return e;
  if (d < 64 && (*sms = known[d].load(std::memory_order_relaxed)) > 0) return e;
  e = cudaDeviceGetAttribute(sms, cudaDevAttrMultiProcessorCount, d);
  if (e == cudaSuccess && d < 64) known[d].store(*sms, std::memory_order_relaxed);
  return e;
}

bool bad_strides(const void* x, int64_t row, int64_t head) { return misaligned(x, 16) || row % 8 != 0 || head % 8 != 0; }

}  // namespace
}  // namespace fe

extern "C" int fe_kv_append(const fe_append_args* a, void* stream) {
  using namespace fe;
  if (!a) return fail(FE_ERR_INVALID_ARG, "null arguments");
  const int rc = check_paged_kv(a->kv);
  if (rc != FE_OK) return rc;
  if (a->n_seqs < 0 || a->n_rows < 0 || a->page_cols < 1) return fail(FE_ERR_INVALID_ARG, "negative size or no page column");
  if (a->n_rows == 0) return FE_OK;
  if (a->n_seqs == 0) return fail(FE_ERR_INVALID_ARG, "rows without a sequence");
  if (!a->row_start || !a->first || !a->pages || !a->k || !a->v) return fail(FE_ERR_INVALID_ARG, "null pointer");
  if (a->q && (!a->q_out || a->q_heads < 1)) return fail(FE_ERR_INVALID_ARG, "queries without q_out or q_heads");
  if (a->q && a->q_out == a->q && (a->q_head != a->kv.head_dim || a->q_row != (int64_t)a->q_heads * a->kv.head_dim))
    return fail(FE_ERR_INVALID_ARG, "q_out in place of q needs contiguous queries");
  if (bad_strides(a->k, a->k_row, a->k_head) || bad_strides(a->v, a->v_row, a->v_head) ||
      (a->q && (bad_strides(a->q, a->q_row, a->q_head) || misaligned(a->q_out, 16))))
    return fail(FE_ERR_UNSUPPORTED, "rows must be 16-byte aligned, strides multiples of 8");
  if (a->pairs != FE_PAIRS_HALF && a->pairs != FE_PAIRS_INTERLEAVED) return fail(FE_ERR_INVALID_ARG, "unknown pairs");
  if (a->rope) {
    if (a->rope_rows < 1 || misaligned(a->rope, 16)) return fail(FE_ERR_INVALID_ARG, "rope: no rows or not 16-byte aligned");
    if (a->rot_dim < 16 || a->rot_dim % 16 != 0 || a->rot_dim > a->kv.head_dim)
      return fail(FE_ERR_UNSUPPORTED, "rot_dim must be a multiple of 16, at most head_dim");
  }
  AppendParams p{};
  p.row_start = a->row_start;
  p.first = a->first;
  p.shift = a->shift;
  p.pages = a->pages;
  p.k = a->k;
  p.v = a->v;
  p.q = a->q;
  p.k_out = a->kv.k;
  p.v_out = a->kv.v;
  p.q_out = a->q_out;
  p.rope = a->rope;
  p.status = a->status;
  p.k_row = a->k_row, p.k_head = a->k_head;
  p.v_row = a->v_row, p.v_head = a->v_head;
  p.q_row = a->q_row, p.q_head = a->q_head;
  p.n_seqs = a->n_seqs;
  p.n_rows = a->n_rows;
  p.page_cols = a->page_cols;
  p.hq = a->q ? a->q_heads : 0;
  p.hkv = a->kv.kv_heads;
  p.page_rows = a->kv.page_rows;
  p.n_pages = a->kv.n_pages;
  p.rope_rows = a->rope_rows;
  p.rot = a->rope ? a->rot_dim : 0;
  const int heads = 512 / a->kv.head_dim, steps = (p.hq + 2 * p.hkv + heads - 1) / heads;  // of a warp over a row
  int sms = 0;
  cudaError_t e = device_sms(&sms);
  if (e != cudaSuccess) return fail_cuda(e, "fe_kv_append");
  p.parts = 1;
  while (2 * p.parts <= steps && 2LL * p.n_rows * p.parts <= (long long)kWarps * sms) p.parts *= 2;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  const bool half = a->pairs == FE_PAIRS_HALF;
  e = a->kv.dtype == FE_IO_BF16 ? append_dim<__nv_bfloat16>(p, a->kv.head_dim, half, s)
                                : append_dim<__half>(p, a->kv.head_dim, half, s);
  return e == cudaSuccess ? FE_OK : fail_cuda(e, "fe_kv_append");
}
