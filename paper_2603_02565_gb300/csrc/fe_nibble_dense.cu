// The dense part of fe_nibble_attention: keys that all rows of a group see, for groups of many rows.
//
// A unit is up to 128 rows of a group that read the same key head; its keys are whole tiles of 128 (what is left of
// a prefix, and keys that only some rows see, are fe_nibble_attn.cu's).  So nothing is masked here.  Both products are
// tcgen05.mma with 16-bit operands: a code costs two instructions a pair of them, once for all 128 rows, where the
// other kernel pays for each 8 or 16.
//   S = Q K^T   queries are f16 times a power of two (bf16 to 2^-35 of a row's largest), keys n s / 8 rounded to f16
//   O += P V    weights 2^(x - m) in f16 from TMEM, values n s / 8 rounded to f16 (an eighth: the largest scale is 65504)
// Values are rounded by 2^-11 (where the other kernel rounds weights times scales as much), and so are keys where bf16's results
// (2^-8) hide it.  f16's would not, nor would the log-sum, which is fp32: with these, what is left over of a key's number (three
// bits) is a second operand of the same product, and lies in the values' place until then.  Eighths of numbers end at f16's
// 2^-24, so what is small is held to 2^-22 (half a step, times 8): scales from 2^-11 on lose nothing of a key.
// Four warps make numbers of codes, a thread a key: its codes come in registers a tile ahead, eight numbers leave as 16
// bytes.  The order of the elements within eight (0 4 1 5 2 6 3 7) is that of the codes' masks; queries are put in the
// same order, and outputs back.  Four warps are the softmax, a row a thread; one issues the products.  Two CTAs an SM fill each
// other's gaps.  Each takes an equal run of all units' tiles; a third kernel joins split units.
//
// What bounds it: the chain scores - maximum - weights - product of a tile, 3.3 us with two CTAs an SM: 2900 clocks of it are the
// softmax (128 numbers a thread, read from TMEM twice), and without arithmetic, loads and products the barriers alone
// take 1.5.  GB300 (ncu): prefixes of 20000 to 32768 under 64 rows a key head, 8 key heads of 128: 70 us (bytes 17,
// products 13); 256 prefixes of 256 under 50 rows, 4 of 32: 32 us.
// With the keys' rest, the first takes 23 us more (whole call, replayed graph: 136; 206 by the other kernel alone).
// Slower, for the first: scores of two tiles in TMEM in turn 77 us; a ring of half tiles 79, with loads two tiles ahead 72.
#include <type_traits>

#include "fe_nibble_attn.cuh"

namespace fe {
namespace {

constexpr int kThreads = 288;
constexpr int kSoftmax = 4, kMake = 4;  // warps 0 .. 3 and 4 .. 7; warp 8 issues products

template <int D>
struct DenseCfg {
  static constexpr uint32_t kRow = D >= 64 ? 128 : 64;  // bytes of a swizzled row
  static constexpr int NH = D == 128 ? 2 : 1;           // column halves of a tile
  static constexpr uint32_t kHalf = 128 * kRow, kTile = NH * kHalf;
  static constexpr uint32_t kSwz = D >= 64 ? 2u : 4u;  // descriptor swizzle code (128 B / 64 B)
  static constexpr uint32_t kCols = 256, kO = 128;     // TMEM columns: S (and P in its place), O
  static constexpr size_t kSmem = 1024 + 3 * (size_t)kTile + 256;
};

__device__ __forceinline__ uint64_t tile_desc(uint32_t saddr, uint32_t lbo, uint32_t sbo, uint32_t swz) {
  uint64_t d = 0;
  d |= (uint64_t)((saddr & 0x3FFFFu) >> 4);
  d |= (uint64_t)(lbo >> 4) << 16;
  d |= (uint64_t)(sbo >> 4) << 32;
  d |= (uint64_t)1 << 46;
  d |= (uint64_t)swz << 61;
  return d;
}
// byte of 16-byte piece c of row r
template <int D>
__device__ __forceinline__ uint32_t piece_at(int r, int c) {
  using C = DenseCfg<D>;
  constexpr int PH = C::kRow / 16;  // pieces of a row's half
  const uint32_t mask = C::kRow == 128 ? (uint32_t)r & 7u : ((uint32_t)r >> 1) & 3u;
  return (uint32_t)(c / PH) * C::kHalf + (uint32_t)r * C::kRow + ((((uint32_t)c % PH) ^ mask) << 4);
}
__device__ __forceinline__ uint32_t add2(uint32_t x, uint32_t y) {
  uint32_t z;
  asm("add.rn.f16x2 %0, %1, %2;" : "=r"(z) : "r"(x), "r"(y));
  return z;
}
__device__ __forceinline__ uint32_t mul2(uint32_t x, uint32_t y) {
  uint32_t z;
  asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(z) : "r"(x), "r"(y));
  return z;
}
// x y - z
__device__ __forceinline__ uint32_t less2(uint32_t x, uint32_t y, uint32_t z) {
  uint32_t w;
  asm("fma.rn.f16x2 %0, %1, %2, %3;" : "=r"(w) : "r"(x), "r"(y), "r"(z ^ 0x80008000u));
  return w;
}
__device__ __forceinline__ uint32_t finite2(uint32_t x) {  // infinities become NaN
  uint32_t z;
  asm("fma.rn.f16x2 %0, %1, %2, %1;" : "=r"(z) : "r"(x), "r"(0u));
  return z;
}

// A CTA's walk through its run of tiles, the same in every role
struct Walk {
  const long long* cum;
  const int* group;
  long long x, end;
  int slot, head, off, cost, n;  // the present unit's: its first tile here and how many
  RowTile tile;

  __device__ __forceinline__ void open(const NibbleParams& p) {
    cost = (int)((cum[slot + 1] - cum[slot]) / p.hkv);
    tile = row_tile(p, kDenseRows, group[slot], slot);
  }
  __device__ __forceinline__ bool start(const NibbleParams& p) {
    const long long total = cum[p.n_dslots];
    const int ctas = (int)min((long long)p.dctas, total);
    if ((int)blockIdx.x >= ctas) return false;
    const long long each = total / ctas;
    const int more = (int)(total - each * ctas);
    x = each * blockIdx.x + min((int)blockIdx.x, more);
    end = x + each + ((int)blockIdx.x < more ? 1 : 0);
    slot = warp_find(cum, p.n_dslots, x);
    open(p);
    const long long y = x - cum[slot];
    head = (int)(y / cost);
    off = (int)(y - (long long)head * cost);
    n = (int)min((long long)(cost - off), end - x);
    return true;
  }
  __device__ __forceinline__ bool next(const NibbleParams& p) {
    x += n;
    if (x >= end) return false;
    off = 0;
    if (++head == p.hkv) {
      head = 0;
      ++slot;
      while (cum[slot + 1] == cum[slot]) ++slot;
      open(p);
    }
    n = (int)min((long long)cost, end - x);
    return true;
  }
};

// Key tiles of a row tile (one head)
__device__ int dense_cost(const NibbleParams& p, int slot, int g) {
  if (row_tile(p, kDenseRows, g, slot).rows == 0) return 0;
  const int n = p.prefix_of(g);
  if (!p.prefix_ok(n)) return 0;
  return (p.group_start ? p.dense_prefix(n) : p.dense_own(g)) / kDenseKeys;
}
// Many row tiles: one CTA counts them (few: every CTA of the kernel does)
__global__ void __launch_bounds__(1024) dense_plan_kernel(const NibbleParams p) {
  __shared__ long long sh[33];
  pdl_trigger();
  pdl_wait();
  sum_slots<1024>(p, p.n_dslots, p.dcum, sh, [&](int i) {
    const int g = group_of_slot(p, kDenseRows, i);
    p.dslot_group[i] = g;
    return dense_cost(p, i, g);
  });
}

// FINE: scores of the keys as they are
template <typename T, int D, bool FINE>
__global__ void __launch_bounds__(kThreads, 2) dense_kernel(const NibbleParams p) {
  using C = DenseCfg<D>;
  constexpr int G = D / 32;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
  uint8_t *sQ = smem, *sK = sQ + C::kTile, *sV = sK + C::kTile;
  uint64_t* bars = reinterpret_cast<uint64_t*>(sV + C::kTile);
  uint64_t *k_full = bars, *k_empty = bars + 1, *v_full = bars + 2, *v_empty = bars + 3, *q_full = bars + 4, *s_full = bars + 5,
           *p_full = bars + 6, *pv_done = bars + 7, *drain = bars + 8;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + 9);
  __shared__ long long sh[kThreads / 32 + 1], sh_cum[kFewSlots + 1];
  __shared__ int sh_group[kFewSlots];
  __shared__ int status_word;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  prefetch_indices(p);
  if (threadIdx.x == 0) {
    status_word = 0;
    mbar_init(k_full, kMake);
    mbar_init(k_empty, 1);
    mbar_init(v_full, kMake);
    mbar_init(v_empty, 1);
    mbar_init(q_full, kSoftmax);
    mbar_init(s_full, 1);
    mbar_init(p_full, kSoftmax);
    mbar_init(pv_done, 1);
    mbar_init(drain, 1);
    fence_mbar_init();
  }
  if (warp == 8) tmem_alloc(tmem_slot, C::kCols);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  pdl_trigger();
  pdl_wait();
  int* status = &status_word;  // (a CTA's waits are its own)
  auto arrive = [&](uint64_t* bar) {
    __syncwarp();
    mbar_arrive_if_at(smem_u32(bar), lane == 0);
  };
  if (threadIdx.x == 0) p.drecs[blockIdx.x].count = 0;
  Walk w;
  w.cum = p.dcum;
  w.group = p.dslot_group;
  if (p.n_dslots <= kFewSlots) {
    sum_slots<kThreads>(p, p.n_dslots, sh_cum, sh, [&](int i) {
      const int g = group_of_slot(p, kDenseRows, i);
      sh_group[i] = g;
      return dense_cost(p, i, g);
    });
    w.cum = sh_cum;
    w.group = sh_group;
  }
  const bool some = w.start(p);

  if (some && warp == 8) {
    // ---------------- products ----------------
    const uint32_t go = elect_one();
    const uint32_t idesc = umma_idesc_f16(128, kDenseKeys);
    const uint32_t idesc_pv = umma_idesc_f16(128, D) | (1u << 16);  // V is MN-major
    const uint64_t qd = tile_desc(smem_u32(sQ), 16, 8 * C::kRow, C::kSwz), kd = tile_desc(smem_u32(sK), 16, 8 * C::kRow, C::kSwz);
    const uint64_t kd2 = tile_desc(smem_u32(sV), 16, 8 * C::kRow, C::kSwz);  // what rounding left over of the keys
    const uint64_t vd = tile_desc(smem_u32(sV), C::kHalf, 8 * C::kRow, C::kSwz);
    uint32_t jobs = 0, units = 0;
    bool ok = true;
    do {
      ok = mbar_wait_ok(q_full, units & 1u, status);
      ++units;
#pragma unroll 1
      for (int j = 0; ok && j < w.n; ++j, ++jobs) {
        // (P lies where S does: its product is waited for)
        if (!(ok = mbar_wait_ok(k_full, jobs & 1u, status) && (jobs == 0 || mbar_wait_ok(pv_done, (jobs - 1) & 1u, status)))) break;
        tc_fence_after();
#pragma unroll
        for (int kk = 0; kk < D / 16; ++kk) {
          const uint64_t at = (uint64_t)(((kk * 32) / C::kRow * C::kHalf + (kk * 32) % C::kRow) >> 4);
          umma_bf16_if(tmem, qd + at, kd + at, idesc, kk != 0 ? 1u : 0u, go);
          if (FINE) umma_bf16_if(tmem, qd + at, kd2 + at, idesc, 1u, go);
        }
        umma_commit_if(s_full, go);
        umma_commit_if(k_empty, go);
        if (!(ok = mbar_wait_ok(v_full, jobs & 1u, status) && mbar_wait_ok(p_full, jobs & 1u, status))) break;
        tc_fence_after();
#pragma unroll
        for (int kk = 0; kk < kDenseKeys / 16; ++kk)
          umma_bf16_tmem_a_if(tmem + C::kO, tmem + (uint32_t)(8 * kk), vd + (uint64_t)((kk * 16 * C::kRow) >> 4), idesc_pv,
                              j != 0 || kk != 0 ? 1u : 0u, go);
        umma_commit_if(pv_done, go);
        umma_commit_if(v_empty, go);
      }
    } while (ok && w.next(p));
    umma_drain(drain, status, go);
  } else if (some && warp >= kSoftmax) {
    // ---------------- numbers of codes: key `row` of each tile ----------------
    const int row = threadIdx.x - 32 * kSoftmax;
    constexpr int NW = D / 8;  // words of a row's codes
    uint32_t kc[NW], vc[NW], ks[(G + 1) / 2], vs[(G + 1) / 2];
    uint32_t jobs = 0;
    bool ok = true;
    auto place = [&](int j, int& page) -> uint32_t {  // the row of the pages of key `row` of tile j
      const int idx = j * kDenseKeys + row;
      const int32_t* table = p.group_start ? p.prefix_pages + (long long)w.tile.group * p.prefix_cols
                                           : p.pages + (long long)w.tile.group * p.page_cols;
      page = __ldg(table + (idx >> p.page_shift));
      const bool bad = page < 0 || page >= p.n_pages;
      return (uint32_t)((bad ? 0 : page) * p.hkv + w.head) * (uint32_t)p.page_rows + (uint32_t)(idx & (p.page_rows - 1));
    };
    auto fetch = [&](const uint8_t* codes, const __half* scales, uint32_t r, uint32_t* c, uint32_t* s) {
      const uint4* from = reinterpret_cast<const uint4*>(codes + (uint64_t)r * (D / 2));
#pragma unroll
      for (int i = 0; i < NW / 4; ++i) {
        const uint4 x = __ldg(from + i);
        c[4 * i] = x.x, c[4 * i + 1] = x.y, c[4 * i + 2] = x.z, c[4 * i + 3] = x.w;
      }
      if constexpr (G == 4) {
        const uint2 y = __ldg(reinterpret_cast<const uint2*>(scales + (uint64_t)r * G));
        s[0] = y.x, s[1] = y.y;
      } else if constexpr (G == 2) {
        s[0] = __ldg(reinterpret_cast<const uint32_t*>(scales + (uint64_t)r * G));
      } else {
        s[0] = __ldg(reinterpret_cast<const uint16_t*>(scales + (uint64_t)r));
      }
    };
    // (rest: what rounding leaves over of the numbers)
    auto make = [&](uint8_t* to, const uint32_t* c, const uint32_t* s, auto rest) {
#pragma unroll
      for (int b = 0; b < G; ++b) {
        uint32_t s2 = __byte_perm(s[b / 2], 0, b & 1 ? 0x3232 : 0x1010);
        s2 = finite2(s2);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          // elements 8 i .. 8 i + 7 of the group: half-words 2 i G + b and (2 i + 1) G + b
          uint32_t x;
          if constexpr (G == 1)
            x = c[i];
          else
            x = __byte_perm(c[i * G + b / 2], c[i * G + G / 2 + b / 2], b & 1 ? 0x7632 : 0x5410);
          const uint32_t x8 = x >> 8;
          auto number = [&](uint32_t n) {
            const uint32_t z = mul2(n, s2);
            if constexpr (decltype(rest)::value)
              return less2(n, s2, z);
            else
              return z;
          };
          // (128 + u / 8 and 8 + u / 8, less 129 and 9: eighths of n, exactly)
          uint4 y;
          y.x = number(add2((x & 0x000f000fu) | 0x58005800u, 0xd808d808u));
          y.y = number(add2((x & 0x00f000f0u) | 0x48004800u, 0xc880c880u));
          y.z = number(add2((x8 & 0x000f000fu) | 0x58005800u, 0xd808d808u));
          y.w = number(add2((x8 & 0x00f000f0u) | 0x48004800u, 0xc880c880u));
          *reinterpret_cast<uint4*>(to + piece_at<D>(row, 4 * b + i)) = y;
        }
      }
    };
    int page, next_page = 0;
    uint32_t at = place(w.off, page), next_at = 0;
    fetch(p.kc, p.ks, at, kc, ks);
    fetch(p.vc, p.vs, at, vc, vs);
    do {
#pragma unroll 1
      for (int j = 0; j < w.n; ++j, ++jobs) {
        if (page < 0 || page >= p.n_pages) {  // its rows are NaN
          if (p.status) atomicOr(p.status, FE_ST_INDEX);
#pragma unroll
          for (int i = 0; i < (G + 1) / 2; ++i) ks[i] = 0x7fff7fffu;
        }
        const bool last = j + 1 == w.n;
        if (!last) next_at = place(w.off + j + 1, next_page);
        if (!FINE && !(ok = mbar_wait_ok(k_empty, (jobs & 1u) ^ 1u, status))) break;  // (FINE: waited for before the last values)
        make(sK, kc, ks, std::false_type());
        if (FINE) {  // the values' place has the keys' rest until the scores are made
          if (!(ok = mbar_wait_ok(v_empty, (jobs & 1u) ^ 1u, status))) break;
#pragma unroll
          for (int i = 0; i < NW; ++i) asm volatile("" : "+r"(kc[i]));  // (made anew: no registers to keep the numbers in)
          make(sV, kc, ks, std::true_type());
        }
        fence_async_shared();
        arrive(k_full);
        if (!last) fetch(p.kc, p.ks, next_at, kc, ks);
        if (!(ok = mbar_wait_ok(FINE ? k_empty : v_empty, FINE ? jobs & 1u : (jobs & 1u) ^ 1u, status))) break;
        make(sV, vc, vs, std::false_type());
        fence_async_shared();
        arrive(v_full);
        if (!last) fetch(p.vc, p.vs, next_at, vc, vs);
        page = next_page;
      }
      if (!ok || !w.next(p)) break;
      at = place(w.off, page);
      fetch(p.kc, p.ks, at, kc, ks);
      fetch(p.vc, p.vs, at, vc, vs);
    } while (true);
  } else if (some) {
    // ---------------- softmax and output ----------------
    const int row = threadIdx.x;
    const uint32_t tl = tmem + ((uint32_t)(warp * 32) << 16), t_s = tl, t_o = tl + C::kO;
    uint32_t jobs = 0;
    bool ok = true;
    do {
      const bool mine = row < w.tile.rows;
      const bool active = 32 * warp < w.tile.rows;
      float sc = 0.f;
      int orow = 0;
      {
        const int tk = (w.tile.r0 + row) / p.hr, h = w.head * p.hr + (w.tile.r0 + row - tk * p.hr);
        orow = (w.tile.t0 + tk) * p.hq + h;
        const uint4* q = reinterpret_cast<const uint4*>(reinterpret_cast<const T*>(p.q) + (long long)(w.tile.t0 + tk) * p.q_row + h * p.q_head);
        float big = 0.f;
        if (mine) {
#pragma unroll 4
          for (int c = 0; c < D / 8; ++c) {
            float f[8];
            piece_get<T>(__ldg(q + c), f);
#pragma unroll
            for (int i = 0; i < 8; ++i) big = fmaxf(big, fabsf(f[i]));
          }
        }
        // times a power of two that brings the largest to 2^14 .. 2^15 (a row without a number above 0: times 1); a row that holds an
        // infinity is NaN throughout, or scores of -inf alone would leave no weight
        int k = 0;
        if (big > 0.f && big < INFINITY) k = min(14 - ilogbf(big), 120);
        const float up = big == INFINITY ? NAN : ldexpf(1.f, k);
        sc = fmaxf(ldexpf(p.sc, 3 - k), 1e-37f);  // (keys are an eighth)
#pragma unroll 2
        for (int c = 0; c < D / 8; ++c) {
          uint4 y = make_uint4(0u, 0u, 0u, 0u);
          if (mine) {
            float f[8];
            piece_get<T>(__ldg(q + c), f);
#pragma unroll
            for (int i = 0; i < 8; ++i) f[i] *= up;
            y = make_uint4(pack_f16x2(f[0], f[4]), pack_f16x2(f[1], f[5]), pack_f16x2(f[2], f[6]), pack_f16x2(f[3], f[7]));
          }
          *reinterpret_cast<uint4*>(sQ + piece_at<D>(row, c)) = y;
        }
        fence_async_shared();
        arrive(q_full);
      }
      constexpr float kSlack = 8.f, kLift = 7.f;  // weights up to 2^15, at least 2^-32 of the largest count
      float m = -INFINITY, l = 0.f;
#pragma unroll 1
      for (int j = 0; j < w.n; ++j, ++jobs) {
        if (!(ok = mbar_wait_ok(s_full, jobs & 1u, status))) break;
        if (active) {
          tc_fence_after();
          float mx = -INFINITY;
#pragma unroll 1
          for (int c0 = 0; c0 < 128; c0 += 32) {
            float v[32];
            tmem_ld32(t_s + (uint32_t)c0, v);
            float a[4] = {v[0], v[1], v[2], v[3]};
#pragma unroll
            for (int i = 4; i < 32; ++i) a[i & 3] = fmaxf(a[i & 3], v[i]);
            mx = fmaxf(mx, fmaxf(fmaxf(a[0], a[1]), fmaxf(a[2], a[3])));
          }
          mx = fmaf(mx, sc, -kLift);
          if (j == 0) {
            m = mx;
          } else {
            const bool up = mx > m + kSlack;
            if (__any_sync(0xffffffffu, up)) {
              // (the last product with V is complete: this tile's scores came after it)
              const float f = up ? ex2_approx(m - mx) : 1.f;
              if (up) m = mx;
              l *= f;
#pragma unroll 1
              for (int c0 = 0; c0 < D; c0 += 8) {
                uint32_t o[8];
                tmem_ld8(t_o + (uint32_t)c0, o);
#pragma unroll
                for (int i = 0; i < 8; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * f);
                tmem_st8_nowait(t_o + (uint32_t)c0, o);
              }
            }
          }
          const float ref = m == -INFINITY ? 0.f : m;
          const uint64_t sc2 = f32x2_pack(sc, sc), nm2 = f32x2_pack(-ref, -ref);
          uint64_t sum[2] = {0ull, 0ull};
#pragma unroll 1
          for (int c0 = 0; c0 < 128; c0 += 32) {
            float v[32];
            uint32_t pk[16];
            tmem_ld32(t_s + (uint32_t)c0, v);
#pragma unroll
            for (int i = 0; i < 32; i += 4) {
              float e[4];
              f32x2_unpack(f32x2_fma(f32x2_pack(v[i], v[i + 1]), sc2, nm2), e[0], e[1]);
              f32x2_unpack(f32x2_fma(f32x2_pack(v[i + 2], v[i + 3]), sc2, nm2), e[2], e[3]);
#pragma unroll
              for (int z = 0; z < 4; ++z) e[z] = ex2_approx(e[z]);
              uint64_t& acc = sum[(i >> 2) & 1];
              acc = f32x2_add(acc, f32x2_add(f32x2_pack(e[0], e[2]), f32x2_pack(e[1], e[3])));
              pk[i / 2] = pack_f16x2(e[0], e[1]);
              pk[i / 2 + 1] = pack_f16x2(e[2], e[3]);
            }
            tmem_st16_nowait(t_s + (uint32_t)(c0 / 2), pk);
          }
          float a0, a1, a2, a3;
          f32x2_unpack(sum[0], a0, a1);
          f32x2_unpack(sum[1], a2, a3);
          l += (a0 + a1) + (a2 + a3);
          tmem_st_wait();
          tc_fence_before();
        }
        arrive(p_full);
      }
      if (!ok) break;
      // ---------------- the piece's output ----------------
      if (!(ok = mbar_wait_ok(pv_done, (jobs - 1) & 1u, status))) break;
      tc_fence_after();
      const bool direct = w.n == w.cost;
      const long long slot = (2LL * blockIdx.x + (w.off == 0 ? 1 : 0)) * kDenseRows + row;
      if (!direct && w.off == 0 && threadIdx.x == 0) {
        const long long total = w.cum[p.n_dslots];
        const int ctas = (int)min((long long)p.dctas, total);
        const long long each = total / ctas, more = total - each * ctas, tile = w.x + w.cost - 1, in_large = (each + 1) * more;
        const int to = (int)(tile < in_large ? tile / (each + 1) : more + (tile - in_large) / each);
        p.drecs[blockIdx.x] = SplitRec{to - (int)blockIdx.x + 1, w.tile.t0, w.tile.r0, w.tile.rows, w.head};
      }
      float* out = direct ? p.state_o + (long long)orow * D : p.dpart_o + slot * D;
      if (active) {
#pragma unroll 1
        for (int c0 = 0; c0 < D; c0 += 8) {
          uint32_t o[8];
          float y[8];
          tmem_ld8(t_o + (uint32_t)c0, o);
#pragma unroll
          for (int i = 0; i < 8; ++i) y[(i & 1) * 4 + i / 2] = __uint_as_float(o[i]) * 8.f;
          if (mine) st_sector(out + c0, y);
        }
        if (mine) {
          if (direct)
            p.state_ml[orow] = make_float2(m, l);
          else
            p.dpart_ml[slot] = make_float2(m, l);
        }
      }
      tc_fence_before();
    } while (w.next(p));
  }
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  if (threadIdx.x == 0) p.stat[blockIdx.x] = status_word;
  if (warp == 8) tmem_dealloc(tmem, C::kCols);
}

// CTA (x, y) joins rows of the split unit that CTA x of the dense kernel has begun
template <int D>
__global__ void __launch_bounds__(256) dense_join_kernel(const NibbleParams p) {
  constexpr int N = D / 32;
  pdl_trigger();
  pdl_wait();
  const SplitRec rec = p.drecs[blockIdx.x];
  if (rec.count == 0) return;
  const int lane = threadIdx.x & 31, wp = threadIdx.x >> 5;
  struct alignas(4 * N) Values {
    float v[N];
  };
  for (int r = blockIdx.y * 8 + wp; r < rec.rows; r += 8 * gridDim.y) {
    auto slot = [&](int i) { return (2LL * ((int)blockIdx.x + i) + (i == 0)) * kDenseRows + r; };
    float m = -INFINITY, l = 0.f;
    Values o = {};
    for (int i0 = 0; i0 < rec.count; i0 += 32) {  // references and sums of 32 pieces at once, a lane each
      const float2 ml = i0 + lane < rec.count ? p.dpart_ml[slot(i0 + lane)] : make_float2(-INFINITY, 0.f);
      float top = ml.x;
#pragma unroll
      for (int z = 16; z > 0; z >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, z));
      const float m1 = fmaxf(m, top), ref = m1 == -INFINITY ? 0.f : m1;
      const float old = ex2_approx(m - ref), f = ex2_approx(ml.x - ref);
      m = m1;
      float sum = ml.y * f;
#pragma unroll
      for (int z = 16; z > 0; z >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, z);
      l = fmaf(l, old, sum);
#pragma unroll
      for (int z = 0; z < N; ++z) o.v[z] *= old;
      constexpr int U = 8;  // loads at once (those past the last piece: none, times 0)
#pragma unroll 1
      for (int i = 0; i < min(32, rec.count - i0); i += U) {
        Values x[U] = {};
#pragma unroll
        for (int c = 0; c < U; ++c)
          if (i0 + i + c < rec.count) x[c] = reinterpret_cast<const Values*>(p.dpart_o + slot(i0 + i + c) * D)[lane];
#pragma unroll
        for (int c = 0; c < U; ++c) {
          const float fi = __shfl_sync(0xffffffffu, f, i + c);
#pragma unroll
          for (int z = 0; z < N; ++z) o.v[z] = fmaf(x[c].v[z], fi, o.v[z]);
        }
      }
    }
    const int rr = rec.r0 + r;
    const long long at = (long long)(rec.t0 + rr / p.hr) * p.hq + rec.head * p.hr + rr % p.hr;
    reinterpret_cast<Values*>(p.state_o + at * D)[lane] = o;
    if (lane == 0) p.state_ml[at] = make_float2(m, l);
  }
}

template <typename T, int D, bool FINE>
cudaError_t dense_go(const NibbleParams& p, cudaStream_t s) {
  using C = DenseCfg<D>;
  cudaError_t e = cudaFuncSetAttribute((const void*)dense_kernel<T, D, FINE>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)C::kSmem);
  if (e == cudaSuccess && p.n_dslots > kFewSlots) e = launch_k(dense_plan_kernel, dim3(1), dim3(1024), 0, s, p);
  if (e == cudaSuccess) e = launch_k(dense_kernel<T, D, FINE>, dim3((unsigned)p.dctas), dim3(kThreads), C::kSmem, s, p);
  if (e == cudaSuccess) e = launch_k(dense_join_kernel<D>, dim3((unsigned)p.dctas, 8), dim3(256), 0, s, p);
  return e;
}
template <typename T, bool FINE>
cudaError_t dense_dim(const NibbleParams& p, int d, cudaStream_t s) {
  return d == 32 ? dense_go<T, 32, FINE>(p, s) : d == 64 ? dense_go<T, 64, FINE>(p, s) : dense_go<T, 128, FINE>(p, s);
}
}  // namespace

cudaError_t nibble_dense(const NibbleParams& p, int head_dim, bool f16, cudaStream_t s) {
  if (f16) return dense_dim<__half, true>(p, head_dim, s);
  return p.lse ? dense_dim<__nv_bfloat16, true>(p, head_dim, s) : dense_dim<__nv_bfloat16, false>(p, head_dim, s);
}

}  // namespace fe
