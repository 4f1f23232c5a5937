// Attention of groups of sequences that share a prefix, over a paged cache
// (fe_prefix_attention).
//
// For row t of sequence s in group g, with n_s rows in the call and j = t - row_start[s]:
//   p_k = softmax_k(scale q . k) over the prefix's prefix_len[g] rows and the sequence's
//   own rows 0 .. seq_len[s] - n_s + j,  out = sum_k p_k v_k.
#include <cmath>

#include "fe_ops.cuh"

namespace fe {
namespace {

struct PrefixParams {
  const int32_t *group_start, *prefix_len, *prefix_pages, *row_start, *seq_len, *pages;
  const void *q, *k, *v;
  void* out;
  float* lse;
  int32_t* status;
  int64_t q_row, q_head;
  int n_groups, n_seqs, n_rows, hq, hkv, prefix_cols, page_cols, page_rows, n_pages;
  float scale;
};

// One warp per row and query head, 32 keys at a time.
template <typename T, int D>
__global__ void __launch_bounds__(128) prefix_simple_kernel(const PrefixParams p) {
  __shared__ float sq[4][D];
  pdl_trigger();
  pdl_wait();
  const int lane = threadIdx.x & 31, wp = threadIdx.x >> 5;
  const long long w = (long long)blockIdx.x * 4 + wp;
  const int t = (int)(w / p.hq), h = (int)(w % p.hq), hk = h / (p.hq / p.hkv);
  if (t >= p.n_rows) return;
  const int s = warp_find_row(p.row_start, p.n_seqs, t), g = warp_find_row(p.group_start, p.n_groups, s);
  const int r0 = p.row_start[s], n = p.row_start[s + 1] - r0, len = p.seq_len[s], np = p.prefix_len[g];
  bool bad = t < r0 || t >= r0 + n || s < p.group_start[g] || s >= p.group_start[g + 1] || len < 0 || np < 0 ||
             (long long)len > (long long)p.page_cols * p.page_rows || (long long)np > (long long)p.prefix_cols * p.page_rows;
  const int own = bad ? 0 : max(0, min(len, len - n + (t - r0) + 1)), pre = bad ? 0 : np;
  const T* q = reinterpret_cast<const T*>(p.q) + (long long)t * p.q_row + h * p.q_head;
  for (int i = lane; i < D; i += 32) sq[wp][i] = Elem<T>::get(q[i]);
  __syncwarp();
  float m = -INFINITY, l = 0.f, o[D / 32] = {};
  for (int part = 0; part < 2; ++part) {
    const int32_t* table = part ? p.pages + (long long)s * p.page_cols : p.prefix_pages + (long long)g * p.prefix_cols;
    const int keys = part ? own : pre;
    for (int k0 = 0; k0 < keys; k0 += 32) {
      const int k = k0 + lane;
      long long row = -1;
      float x = -INFINITY;
      if (k < keys) {
        const int page = table[k / p.page_rows];
        if (page < 0 || page >= p.n_pages) {
          bad = true;
        } else {
          row = ((long long)page * p.hkv + hk) * p.page_rows + k % p.page_rows;
          const T* kr = reinterpret_cast<const T*>(p.k) + row * D;
          float a = 0.f;
          for (int i = 0; i < D; ++i) a += sq[wp][i] * Elem<T>::get(kr[i]);
          x = a * p.scale;
        }
      }
      float mx = x;
#pragma unroll
      for (int z = 16; z > 0; z >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, z));
      const float m1 = fmaxf(m, mx), ref = m1 == -INFINITY ? 0.f : m1;
      const float f = expf(m - ref), e = expf(x - ref);
      m = m1;
      float sum = e;
#pragma unroll
      for (int z = 16; z > 0; z >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, z);
      l = l * f + sum;
#pragma unroll
      for (int i = 0; i < D / 32; ++i) o[i] *= f;
      for (int z = 0; z < 32; ++z) {
        const float pz = __shfl_sync(0xffffffffu, e, z);
        const long long rz = __shfl_sync(0xffffffffu, row, z);
        if (rz < 0) continue;
        const T* vr = reinterpret_cast<const T*>(p.v) + rz * D;
#pragma unroll
        for (int i = 0; i < D / 32; ++i) o[i] += pz * Elem<T>::get(vr[lane + 32 * i]);
      }
    }
  }
  bad = __any_sync(0xffffffffu, bad);
  if (bad && lane == 0 && p.status) atomicOr(p.status, FE_ST_INDEX);
  T* out = reinterpret_cast<T*>(p.out) + w * D;
  const float inv = bad ? NAN : l == 0.f ? 0.f : 1.f / l;
#pragma unroll
  for (int i = 0; i < D / 32; ++i) out[lane + 32 * i] = Elem<T>::put(o[i] * inv);
  if (p.lse && lane == 0) p.lse[w] = bad ? NAN : l == 0.f ? -INFINITY : m + logf(l);
}

int check_prefix(const fe_prefix_args* a) {
  if (!a) return fail(FE_ERR_INVALID_ARG, "null arguments");
  const int rc = check_paged_kv(a->kv);
  if (rc != FE_OK) return rc;
  if (a->n_groups < 0 || a->n_seqs < 0 || a->n_rows < 0 || a->prefix_cols < 1 || a->page_cols < 1)
    return fail(FE_ERR_INVALID_ARG, "negative size or no page column");
  if (a->q_heads < 1 || a->q_heads % a->kv.kv_heads != 0)
    return fail(FE_ERR_INVALID_ARG, "q_heads must be a multiple of kv_heads");
  if ((long long)a->n_rows * a->q_heads > 0x7fffffffLL)
    return fail(FE_ERR_UNSUPPORTED, "n_rows * q_heads must be below 2^31");
  if (!std::isfinite(a->scale) || a->scale < 0.f) return fail(FE_ERR_INVALID_ARG, "scale must be finite and not negative");
  if (a->n_rows == 0) return FE_OK;
  if (a->n_groups == 0 || a->n_seqs == 0) return fail(FE_ERR_INVALID_ARG, "rows without a sequence or group");
  if (!a->group_start || !a->prefix_len || !a->prefix_pages || !a->row_start || !a->seq_len || !a->pages || !a->q || !a->out)
    return fail(FE_ERR_INVALID_ARG, "null pointer");
  if (misaligned(a->q, 16) || misaligned(a->out, 16) || a->q_row % 8 != 0 || a->q_head % 8 != 0)
    return fail(FE_ERR_UNSUPPORTED, "rows must be 16-byte aligned, strides multiples of 8");
  return FE_OK;
}

template <typename T>
cudaError_t prefix_dim(const PrefixParams& p, int d, cudaStream_t s) {
  const long long warps = (long long)p.n_rows * p.hq;
  const dim3 g((unsigned)((warps + 3) / 4)), b(128);
  return d == 32   ? launch_k(prefix_simple_kernel<T, 32>, g, b, 0, s, p)
         : d == 64 ? launch_k(prefix_simple_kernel<T, 64>, g, b, 0, s, p)
                   : launch_k(prefix_simple_kernel<T, 128>, g, b, 0, s, p);
}

}  // namespace
}  // namespace fe

extern "C" uint64_t fe_prefix_attention_workspace(const fe_prefix_args* a) {
  return fe::check_prefix(a) == FE_OK ? 256 : 0;
}

extern "C" int fe_prefix_attention(const fe_prefix_args* a, void* stream) {
  using namespace fe;
  const int rc = check_prefix(a);
  if (rc != FE_OK) return rc;
  if (a->n_rows == 0) return FE_OK;
  if (!a->workspace || misaligned(a->workspace, 256)) return fail(FE_ERR_INVALID_ARG, "workspace null or not 256-byte aligned");
  if (a->workspace_bytes < fe_prefix_attention_workspace(a)) return fail(FE_ERR_WORKSPACE, "workspace too small");
  PrefixParams p{};
  p.group_start = a->group_start;
  p.prefix_len = a->prefix_len;
  p.prefix_pages = a->prefix_pages;
  p.row_start = a->row_start;
  p.seq_len = a->seq_len;
  p.pages = a->pages;
  p.q = a->q;
  p.k = a->kv.k;
  p.v = a->kv.v;
  p.out = a->out;
  p.lse = a->lse;
  p.status = a->status;
  p.q_row = a->q_row;
  p.q_head = a->q_head;
  p.n_groups = a->n_groups;
  p.n_seqs = a->n_seqs;
  p.n_rows = a->n_rows;
  p.hq = a->q_heads;
  p.hkv = a->kv.kv_heads;
  p.prefix_cols = a->prefix_cols;
  p.page_cols = a->page_cols;
  p.page_rows = a->kv.page_rows;
  p.n_pages = a->kv.n_pages;
  p.scale = a->scale;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  const cudaError_t e = a->kv.dtype == FE_IO_BF16 ? prefix_dim<__nv_bfloat16>(p, a->kv.head_dim, s)
                                                  : prefix_dim<__half>(p, a->kv.head_dim, s);
  return e == cudaSuccess ? FE_OK : fail_cuda(e, "fe_prefix_attention");
}
