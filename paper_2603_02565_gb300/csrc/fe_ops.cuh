// What the candidate generator's operators share: error reporting, element types,
// 16-byte pieces and the search for a row's sequence.
#pragma once

#include "fe_common.cuh"

namespace fe {

// Sets fe_last_error_message's text (this thread) and returns the code (fe_api.cu).
int fail(int code, const char* msg) noexcept;
int fail_cuda(cudaError_t e, const char* what) noexcept;

// cuTensorMapEncodeTiled by its driver entry point (fe_api.cu); null when unavailable.
typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*,
                                  const cuuint64_t*, const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave,
                                  CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
EncodeTiledFn encode_tiled_fn() noexcept;

template <typename T>
struct Elem;
template <>
struct Elem<__nv_bfloat16> {
  static constexpr int N = 8;  // elements of a 16-byte piece
  __device__ static __forceinline__ float get(__nv_bfloat16 x) { return __bfloat162float(x); }
  __device__ static __forceinline__ __nv_bfloat16 put(float x) { return __float2bfloat16_rn(x); }
  __device__ static __forceinline__ uint32_t put2(float a, float b) {
    __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<uint32_t*>(&h);
  }
  __device__ static __forceinline__ void get2(uint32_t w, float& a, float& b) {
    a = bf16lo_f(w);
    b = bf16hi_f(w);
  }
  __device__ static __forceinline__ uint32_t zero_fma(uint32_t w, uint32_t acc) {  // 0 w + acc, both halves
    uint32_t r;
    asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(r) : "r"(w), "r"(0u), "r"(acc));
    return r;
  }
};
template <>
struct Elem<__half> {
  static constexpr int N = 8;
  __device__ static __forceinline__ float get(__half x) { return __half2float(x); }
  __device__ static __forceinline__ __half put(float x) { return __float2half_rn(x); }
  __device__ static __forceinline__ uint32_t put2(float a, float b) { return pack_f16x2(a, b); }
  __device__ static __forceinline__ void get2(uint32_t w, float& a, float& b) {
    const float2 f = __half22float2(*reinterpret_cast<__half2*>(&w));
    a = f.x;
    b = f.y;
  }
  __device__ static __forceinline__ uint32_t zero_fma(uint32_t w, uint32_t acc) {
    uint32_t r;
    asm("fma.rn.f16x2 %0, %1, %2, %3;" : "=r"(r) : "r"(w), "r"(0u), "r"(acc));
    return r;
  }
};
template <>
struct Elem<float> {
  static constexpr int N = 4;
  __device__ static __forceinline__ float get(float x) { return x; }
  __device__ static __forceinline__ float put(float x) { return x; }
};

// a 16-byte piece as floats, and back (each rounded to nearest once)
template <typename T>
__device__ __forceinline__ void piece_get(const uint4& w, float* x) {
  if constexpr (sizeof(T) == 4) {
    x[0] = __uint_as_float(w.x);
    x[1] = __uint_as_float(w.y);
    x[2] = __uint_as_float(w.z);
    x[3] = __uint_as_float(w.w);
  } else {
    Elem<T>::get2(w.x, x[0], x[1]);
    Elem<T>::get2(w.y, x[2], x[3]);
    Elem<T>::get2(w.z, x[4], x[5]);
    Elem<T>::get2(w.w, x[6], x[7]);
  }
}
template <typename T>
__device__ __forceinline__ uint4 piece_put(const float* x) {
  if constexpr (sizeof(T) == 4)
    return make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
  else
    return make_uint4(Elem<T>::put2(x[0], x[1]), Elem<T>::put2(x[2], x[3]), Elem<T>::put2(x[4], x[5]),
                      Elem<T>::put2(x[6], x[7]));
}

// The sequence of row t by a whole warp: the largest s < n with start[s] <= t, 32 pivots
// a step.  Always in [0, n); whether the row is really its own is the caller's check.
__device__ __forceinline__ int warp_find_row(const int32_t* start, int n, int t) {
  const int lane = threadIdx.x & 31;
  int lo = 0, len = n;
  while (len > 1) {
    const int step = (len + 31) / 32, at = lane * step;
    const bool below = at < len && __ldg(start + lo + at) <= t;
    const int c = max(__popc(__ballot_sync(0xffffffffu, below)), 1) - 1;
    lo += c * step;
    len = min(step, len - c * step);
  }
  return lo;
}

inline bool misaligned(const void* p, unsigned a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) != 0; }

// The pages of fe_kv_append and fe_prefix_attention: FE_OK, or why they are refused.
inline int check_paged_kv(const fe_paged_kv& kv) {
  if (!kv.k || !kv.v || misaligned(kv.k, 128) || misaligned(kv.v, 128))
    return fail(FE_ERR_INVALID_ARG, "pages: null or not 128-byte aligned");
  if (kv.n_pages < 1 || kv.kv_heads < 1) return fail(FE_ERR_INVALID_ARG, "pages: n_pages and kv_heads must be positive");
  if (kv.dtype != FE_IO_BF16 && kv.dtype != FE_IO_F16) return fail(FE_ERR_UNSUPPORTED, "pages: type must be bf16 or f16");
  if (kv.page_rows != 16 && kv.page_rows != 32 && kv.page_rows != 64 && kv.page_rows != 128)
    return fail(FE_ERR_UNSUPPORTED, "pages: page_rows must be 16, 32, 64 or 128");
  if (kv.head_dim != 32 && kv.head_dim != 64 && kv.head_dim != 128)
    return fail(FE_ERR_UNSUPPORTED, "pages: head_dim must be 32, 64 or 128");
  if ((long long)kv.n_pages * kv.kv_heads > 0x7fffffffLL / kv.page_rows)
    return fail(FE_ERR_UNSUPPORTED, "pages: n_pages * kv_heads * page_rows must be below 2^31");
  return FE_OK;
}

}  // namespace fe
