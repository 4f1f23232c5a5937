// Attention of groups of sequences that share a prefix, over a 4-bit paged cache
// (fe_nibble_attention).
//
// For row t of sequence s in group g, with n_s rows in the call and j = t - row_start[s]:
//   p_k = softmax_k(scale q . k) over the prefix's prefix_len[g] rows and the sequence's
//   own rows 0 .. seq_len[s] - n_s + j,  out = sum_k p_k v_k.
// With codes u (n = u - 8) and scales s of groups G of 32 elements,
//   q . k = sum_G s_G sum_{e in G} q_e (u_e - 8),   out_e = sum_k (p_k s_kG) (u_ke - 8).
//
// A unit is a run of up to 8 or 16 rows of a group that read the same key head (tokens x the query heads of
// that key head); its keys come in tiles of 32: first the prefix's, then the own rows of the unit's
// sequences, packed without gaps.  Each warp takes an equal run of all units' tiles, by weight, wherever it begins or
// ends: all SMs have work for a single long sequence as for thousands of short ones.  A finish kernel joins the
// pieces of split units, in order.  Up to 512 row tiles are counted by every CTA for itself, more by a plan kernel.
// Keys that all rows of a group of many rows see are fe_nibble_dense.cu's, which comes first; the first piece of a unit
// takes its sums in.
//
// What a decoding step has to read is a quarter of a 16-bit cache, so what counts is to make numbers of codes with few
// instructions.  Warps work alone, from codes in shared memory (a ring of tiles, each warp its own) to mma.sync's operands in
// registers: numbers never go through shared or tensor memory, and rows are too few for tcgen05's 128.
// Up to 8 rows are the short side of both products (keys x rows, elements x rows), so that one token of a sequence wastes
// little of them; 9 to 16 are the long one.
//   A code in the low bits of a 16-bit float is u 2^-24, one in the next four 16 u 2^-24: a mask makes two numbers of a word.
//   8 is taken off in f16 (exactly).  (Of keys, sums that start at -8 sum q saved that, and took registers and digits: the 64
//   sequences below 4 us longer, and log-sums two to three times as far off.)
//   Keys: queries are f16 times a power of two, which holds bf16 to 2^-35 of the row's largest; every second element's is
//   a sixteenth.  The groups' sums are fp32, scales come to them.
//   Values: scales go to the weights, p s in f16: p is rounded by 2^-11, p s again.  Very small and large scales are lifted or
//   lowered by a power of two, and the reference of the weights follows the largest, so that p s ends below 2^15 and a long flat
//   tail keeps its weight under a peak.  (A peak over 131071 keys of 2^-17 to 2^-18.5 of its weight: off by 3 % at scales of
//   2^-14, 55 % at 2^-24 and 12 % at 60000 when scales stayed as they are; 222 us instead of 226 for the 64 sequences below.)
//   The weights' sum is that of the rounded ones, by a product with ones; the log-sum's that of the exact ones, in fp32.
//
// What bounds it: a half tile's chain of dependent steps in the 12 or 16 warps that registers allow an SM; they issue in 55 to 58 %
// of the cycles, the tensor pipe is busy for 18 to 25.  GB300, a call alone in a replayed graph, caches flushed:
//   one sequence of 131071 rows, 32 over 8 heads of 128, f16: 60 us (bytes at a copy's rate: 22; 16 us of it are what a call
//   of a few rows takes, and beyond that keys come at 4.5 TB/s; a ring of three tiles a warp instead of two: 61)
//   64 sequences of up to 16384 rows, 1 to 5 query rows each, 32 over 8 of 128, bf16: 226 us (bytes 92)
//   256 x 50 sequences of up to 6 rows, prefixes of 256, 4 of 32, bf16: 85 us with the dense part, 97 without
//   the finish kernel is 6 to 10 us of each: 2 to start, 2 for offsets and records, the rest two or three reads that wait on another
// Steps on the way, for the 64 sequences: 16 keys a tile 428, 32 265, rows as the long side 245, runs by weight 226, numbers of keys instead of
// codes 222, scales lifted 226.
#include <cmath>

#include "fe_nibble_attn.cuh"

namespace fe {
namespace {

constexpr int kKeys = 32, kWarps = 4, kThreads = 32 * kWarps;

// What a key tile costs a warp, in parts, by how many rows the unit has.  (64 sequences of up to 5 x 4 rows: 226 us; 228 by
// 2 : 3, 237 by 3 : 5, 249 without weights.)
__host__ __device__ __forceinline__ constexpr int tile_weight(int rows) { return rows <= 8 ? 3 : 4; }

// Key tiles of a row tile (one head) times their weight: at least 1, or 0 if it is unused.  Lengths that are none count as 0, and are reported.
__device__ int slot_cost(const NibbleParams& p, int slot, int group) {
  const RowTile x = row_tile(p, p.unit_rows, group, slot);
  if (x.rows == 0) return 0;
  const int ta = x.t0 + x.r0 / p.hr, tb = x.t0 + (x.r0 + x.rows - 1) / p.hr;
  const int s0 = p.group_first(x.group), s1 = p.group_first(x.group + 1), n = p.prefix_of(x.group);
  long long own = 0;
  bool fine = p.prefix_ok(n);
  int s = seq_of(p, s0, s1, x.t0, x.t1, ta);
  int a = p.row_start[s];
#pragma unroll 4
  for (; s < s1 && a <= tb; ++s) {
    const int b = p.row_start[s + 1], len = p.seq_len[s];
    if (b > a) {
      const bool ok = p.len_ok(len);
      fine = fine && ok;
      if (ok) own += seen_by(len, a, b, min(b - 1, tb)) - p.dense_own(s);
    }
    a = b;
  }
  if (!fine && p.status) atomicOr(p.status, FE_ST_INDEX);
  return tile_weight(x.rows) * (int)max(1LL, ((p.prefix_ok(n) ? n - p.dense_prefix(n) : 0) + kKeys - 1) / kKeys + (own + kKeys - 1) / kKeys);
}

__device__ __forceinline__ void plan_barrier() {  // of the cluster, global writes included
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}

// Many row tiles: one cluster counts them, its first CTA sums up.  (Few: every CTA of the attend kernel does.)
constexpr int kPlanThreads = 1024, kPlanCtas = 8, kPlanGroups = 4096;
__global__ void __launch_bounds__(kPlanThreads) __cluster_dims__(kPlanCtas, 1, 1) nibble_plan_kernel(const NibbleParams p) {
  __shared__ long long sh[kPlanThreads / 32 + 1];
  __shared__ int first[kPlanGroups];  // the groups' first slots, as every slot looks for its group
  pdl_trigger();
  pdl_wait();
  const bool few = p.n_groups <= kPlanGroups;
  if (few) {
    for (int g = threadIdx.x; g < p.n_groups; g += kPlanThreads) first[g] = (int)slot_of(p, p.unit_rows, g);
    __syncthreads();
  }
#pragma unroll 1
  for (int i = blockIdx.x * kPlanThreads + threadIdx.x; i < p.n_slots; i += kPlanThreads * kPlanCtas) {
    const int g = few ? find_last(first, 0, p.n_groups, i) : group_of_slot(p, p.unit_rows, i);
    p.slot_group[i] = g;
    p.cum[i] = slot_cost(p, i, g);
  }
  plan_barrier();
  if (blockIdx.x == 0) sum_slots<kPlanThreads>(p, p.n_slots, p.cum, sh, [&](int i) { return p.cum[i]; });
}

// ---------------------------------------------------------------------------
// attend
// ---------------------------------------------------------------------------
// A tile in shared memory.  Key i lies in row place(i), so that what a warp reads at once of keys (eight of them) and of
// values (four pairs of keys) is in different banks.
__device__ __forceinline__ int place(int i) { return (i & 4) ? i ^ 1 : i; }

template <int D>
struct Tile {
  static constexpr int kRow = D / 2, kScale = D == 128 ? 8 : 4;  // bytes (of a single scale, its neighbour comes with it)
  static constexpr int kK = 0, kV = kKeys * kRow, kKS = 2 * kV, kVS = kKS + kKeys * kScale, kMeta = kVS + kKeys * kScale;
  static constexpr int kFlag = kMeta + kKeys * 8, kOne = kFlag + 16;  // kOne: D = 32, values' own scales
  static constexpr int kBytes = kOne + (D == 32 ? kKeys * 2 : 0);
  static constexpr int kScales = kKeys * (D / 32) * 4;  // keys' scales of the present tile in fp32
  // byte of 16-byte chunk c of a row (rows of 64 bytes: the other half of the banks for every second pair of rows)
  __device__ static __forceinline__ int chunk(int row, int c) { return row * kRow + 16 * (D == 128 ? c ^ (row & 2) : c); }
};

__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
template <int N>
__device__ __forceinline__ void cp_async_small(uint32_t dst, const void* src) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(dst), "l"(src), "n"(N) : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_async_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}
__device__ __forceinline__ void mma_f16(float* c, uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transpose8(uint32_t x) {
  uint32_t y;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}
__device__ __forceinline__ uint32_t add2(uint32_t x, uint32_t y) {
  uint32_t z;
  asm("add.rn.f16x2 %0, %1, %2;" : "=r"(z) : "r"(x), "r"(y));
  return z;
}
__device__ __forceinline__ float half_of(uint32_t w, int hi) {
  return __half2float(__ushort_as_half((unsigned short)(hi ? w >> 16 : w & 0xffffu)));
}
constexpr int kBadKey = (int)0x80000000;  // of a key's number in its sequence: its page does not exist
constexpr uint32_t kLow = 0x000f000fu, kHigh = 0x00f000f0u;       // codes as u 2^-24 and 16 u 2^-24
constexpr uint32_t kEight = 0x80088008u, kEight16 = 0x80808080u;  // -8 and -128 times 2^-24, twice
__device__ __forceinline__ uint32_t low8(uint32_t x) { return add2(x & kLow, kEight); }       // two numbers times 2^-24
__device__ __forceinline__ uint32_t high8(uint32_t x) { return add2(x & kHigh, kEight16); }  // times 2^-20
constexpr float kNoMax = 3e38f;
__device__ __forceinline__ uint32_t mul2(uint32_t x, uint32_t y) {
  uint32_t z;
  asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(z) : "r"(x), "r"(y));
  return z;
}
// infinities become NaN
__device__ __forceinline__ uint32_t finite2(uint32_t x) {
  uint32_t z;
  asm("fma.rn.f16x2 %0, %1, %2, %1;" : "=r"(z) : "r"(x), "r"(0u));
  return z;
}

// What a warp knows of its present unit, in shared memory (registers are for accumulators); seq .. orow of each row
struct alignas(16) Unit {
  int head, group, t0, r0, rows, plen, ptiles;  // plen: the prefix's end
  int pfirst, ofirst;                           // first key of the prefix and of the own rows (those before: the dense part's)
  int own_keys, all_see, first_seq, alone;      // own keys of the list; those that all rows see; all rows are of first_seq
  uint32_t cap;                                 // what the values' scales so far ask for,
  float base;                                   // and where weights start, in log2
  int seq[32], seen[32], start[32], orow[32];   // its sequence, own keys that it sees, first of its keys in the own list, row of
                                                // out / head 0
};

// CTAs an SM: registers for 16 warps, or for as many as hold the accumulators of more rows
constexpr int ctas_of(int d, int nt) { return d == 128 ? 3 : 4; }
// NT: most row tiles (of 8) of a unit
template <int D, int NT>
struct AttendCfg {
  static constexpr int kStages = D == 128 ? 2 : 3;
  static constexpr int G = D / 32;
  static constexpr int kQ = NT == 1 ? 0 : G * 32 * 2 * 16;  // queries
  static constexpr int kWarp = (int)sizeof(Unit) + Tile<D>::kScales + kStages * Tile<D>::kBytes + kQ;
  static constexpr size_t kSmem = (size_t)kWarps * kWarp;
  static constexpr int kStatic = 8 * (kFewSlots + 1 + kWarps + 1) + 4 * kFewSlots;  // the plan's
  static_assert(ctas_of(D, NT) * (kSmem + kStatic + 1024) <= 227 * 1024 + 1024, "shared memory for the CTAs that registers allow");
  static constexpr int kCtas = ctas_of(D, NT);
};

// A warp's loads of key tiles into its ring
template <int D, int ST>
struct KeyLoader {
  using L = Tile<D>;
  static constexpr int G = D / 32, NC = L::kRow / 16, NK = 32 / NC;  // 16-byte pieces of a row, keys of a step
  const NibbleParams& p;
  const Unit& u;
  uint8_t* ring;
  int lane, fill;  // fill: the ring's next stage
  uint32_t chunk0;
  const uint8_t *kc, *vc;
  int l_owner, l_idx, l_page;

  __device__ __forceinline__ KeyLoader(const NibbleParams& p_, const Unit& u_, uint8_t* ring_)
      : p(p_), u(u_), ring(ring_), lane(threadIdx.x & 31), fill(0) {
    chunk0 = L::chunk(place(lane / NC), lane % NC);
    kc = p.kc + 16 * (lane % NC);
    vc = p.vc + 16 * (lane % NC);
  }
  // Lane i looks key i of a tile up; the page's number is asked for a tile before it is used.
  __device__ __forceinline__ void look(int j) {
    l_owner = -3;
    l_idx = 0;
    l_page = 0;
    const int32_t* table = p.prefix_pages + (long long)u.group * p.prefix_cols;
    if (j < u.ptiles) {
      l_idx = u.pfirst + j * kKeys + lane;
      if (l_idx < u.plen) l_owner = -1;
    } else {
      const int o = (j - u.ptiles) * kKeys + lane;
      if (u.alone) {
        if (o < u.own_keys) {
          l_owner = u.first_seq;
          l_idx = u.ofirst + o;
        }
      } else {
        int at = 0;
#pragma unroll
        for (int z = 16; z > 0; z >>= 1) {
          if (u.start[at + z] <= o) at += z;
        }
        // (rows past the last have no keys, and the list's end as their start)
        if (o < u.own_keys) {
          l_owner = u.seq[at];
          l_idx = u.ofirst + o - u.start[at];
        }
      }
      table = p.pages + (long long)max(l_owner, 0) * p.page_cols;
    }
    if (l_owner != -3) l_page = __ldg(table + (l_idx >> p.page_shift));
  }
  __device__ __forceinline__ void load() {
    const uint32_t to = smem_u32(ring) + fill * L::kBytes;
    uint8_t* tile = ring + fill * L::kBytes;
    fill = fill + 1 == ST ? 0 : fill + 1;
    const bool bad = l_page < 0 || l_page >= p.n_pages;
    const int row = ((bad ? 0 : l_page) * p.hkv + u.head) * p.page_rows + (l_idx & (p.page_rows - 1));
#pragma unroll
    for (int z = 0; z < kKeys / NK; ++z) {
      // (place(8 z + i) = 8 z + place(i))
      const uint32_t r = __shfl_sync(0xffffffffu, (uint32_t)row, NK * z + lane / NC), at = to + chunk0 + z * NK * L::kRow;
      cp_async16(at + L::kK, kc + (uint64_t)r * L::kRow);
      cp_async16(at + L::kV, vc + (uint64_t)r * L::kRow);
    }
    const uint32_t first = D == 32 ? (uint32_t)row & ~1u : (uint32_t)row;
    cp_async_small<L::kScale>(to + L::kKS + lane * L::kScale, p.ks + (uint64_t)first * G);
    cp_async_small<L::kScale>(to + L::kVS + lane * L::kScale, p.vs + (uint64_t)first * G);
    // a tile whose keys all rows see
    const bool plain = l_owner != -3 && !bad && (l_owner == -1 || (u.alone && l_idx < u.all_see));
    const bool whole = __all_sync(0xffffffffu, plain);
    if (!whole) {
      if (bad && p.status) atomicOr(p.status, FE_ST_INDEX);
      *reinterpret_cast<int2*>(tile + L::kMeta + 8 * lane) = make_int2(l_owner, bad ? l_idx | kBadKey : l_idx);
    }
    const int halves = __any_sync(0xffffffffu, lane >= 16 && l_owner != -3) ? 2 : 1;  // (keys come without gaps)
    if (lane == 0) *reinterpret_cast<int2*>(tile + L::kFlag) = make_int2(whole ? 0 : 1, halves);
  }
  // the first of n tiles from off on
  __device__ __forceinline__ void start(int off, int n) {
    look(off);
#pragma unroll 1
    for (int i = 0; i < ST - 1; ++i) {
      if (i < n) {
        load();
        if (i + 1 < n) look(off + i + 1);
      }
      cp_async_commit();
    }
  }
  // before tile j is used
  __device__ __forceinline__ void step(int off, int n, int j) {
    cp_async_wait<ST - 2>();
    __syncwarp();
    if (j + ST - 1 < n) {
      load();
      if (j + ST < n) look(off + j + ST);
    }
    cp_async_commit();
  }
};

// What the scales of values seen so far ask for goes by `cap`, the largest scale (as f16 has it) that asks for no more:
// scales are lifted by a power of two (2^lift_of) that brings the largest to 2^-8 .. 1, or below 2^8 if it is beyond, and weights
// start at 2^(25 - exponent_of), so that a weight times a scale is below 2^15 with the slack of new_reference.  A row's largest weight is at
// least 2^3, so is that times the largest lifted scale, and f16's smallest step is 2^-24: what is not rounded to 11 bits is held to
// 2^-28 of these.  All rows and groups of a unit go by one scale.  (From 2^-8 to 1, values of 0.03 to 7, nothing is to do.)
constexpr uint32_t kSmallest = 0xffu, kUsual = 0x3bffu;
__device__ __forceinline__ uint32_t cap_of(uint32_t top) {  // borders 2^-16, 2^-8, 1
  return top < 0x100u ? kSmallest : top < 0x1c00u ? 0x1bffu : top < 0x3c00u ? kUsual : top | 0x3ffu;
}
__device__ __forceinline__ int lift_of(uint32_t cap) {  // and 2^8, 2^12
  return cap < 0x100u ? 16 : cap < 0x1c00u ? 8 : cap < 0x5c00u ? 0 : cap < 0x6c00u ? -4 : -8;
}
__device__ __forceinline__ int exponent_of(uint32_t cap) { return cap < 0x3c00u ? 14 : (int)(cap >> 10) + lift_of(cap); }
__device__ __forceinline__ float power_of_2(int e) { return __int_as_float((127 + e) << 23); }
// (by one lane, before the first tile of a unit's piece)
__device__ __forceinline__ void start_scales(Unit* u) {
  u->cap = kSmallest;
  u->base = 25 - exponent_of(kSmallest);
}

// A tile's scales before it is used: the keys' go to ks in fp32, infinities as NaN, the values' are lifted.  key: key `lane` of a mixed
// tile.  Keys that are none, or that make their rows NaN by their score, get scales of 0.  gate: up to this the largest scale asks for
// nothing (-1: all are lifted).  spoil(key, groups): a key whose scales of these groups are no numbers.  renew(lower, units): weights are
// 2^lower of what they were from here on, and the sums of weighted values count in these units of the old ones.
template <int D, typename Spoil, typename Renew>
__device__ __forceinline__ void take_scales(uint8_t* tile, float* ks, bool mixed, int2 key, Unit* u, int& gate, Spoil spoil, Renew renew) {
  using L = Tile<D>;
  constexpr int G = D / 32, W = D == 128 ? 2 : 1;  // W: words of a key's scales
  const int lane = threadIdx.x & 31;
  uint32_t vw[W], top;
  if constexpr (D == 128) {
    const uint2 y = *reinterpret_cast<const uint2*>(tile + L::kVS + 8 * lane), x = *reinterpret_cast<const uint2*>(tile + L::kKS + 8 * lane);
    const uint32_t x0 = finite2(x.x), x1 = finite2(x.y);
    *reinterpret_cast<float4*>(ks + 4 * lane) = make_float4(half_of(x0, 0), half_of(x0, 1), half_of(x1, 0), half_of(x1, 1));
    vw[0] = y.x;
    vw[1] = y.y;
    top = __vmaxu2(y.x, y.y);
  } else {
    vw[0] = *reinterpret_cast<const uint32_t*>(tile + L::kVS + 4 * lane);
    const uint32_t x = finite2(*reinterpret_cast<const uint32_t*>(tile + L::kKS + 4 * lane));
    if constexpr (D == 64) {
      *reinterpret_cast<float2*>(ks + 2 * lane) = make_float2(half_of(x, 0), half_of(x, 1));
    } else {
      // (rows of a page lie in pairs)
      const int odd = (mixed ? key.y : lane) & 1;
      vw[0] = odd ? vw[0] >> 16 : vw[0] & 0xffffu;
      ks[lane] = half_of(odd ? x >> 16 : x, 0);
      *reinterpret_cast<uint16_t*>(tile + L::kOne + 2 * lane) = (uint16_t)vw[0];
    }
    top = vw[0];
  }
  auto put_scales = [&]() {
    if constexpr (D == 128)
      *reinterpret_cast<uint2*>(tile + L::kVS + 8 * lane) = make_uint2(vw[0], vw[W - 1]);
    else if constexpr (D == 64)
      *reinterpret_cast<uint32_t*>(tile + L::kVS + 4 * lane) = vw[0];
    else
      *reinterpret_cast<uint16_t*>(tile + L::kOne + 2 * lane) = (uint16_t)vw[0];
  };
  if (mixed && (key.x < -1 || key.y < 0)) {  // no key, or one that makes its rows NaN by its score
#pragma unroll
    for (int i = 0; i < W; ++i) vw[i] = 0;
    top = 0;
    put_scales();
  }
  top = __reduce_max_sync(0xffffffffu, max(top & 0xffffu, top >> 16));
  if ((int)top > gate) {
    if (top >= 0x7c00u) {
      // Scales that are negative, or no numbers: these spoil their group in the rows that see the key (a masked weight is
      // 0, and would too), and count as 0.
      top = 0;
      uint32_t wrong = 0;  // groups of key `lane`
#pragma unroll
      for (int b = 0; b < G; ++b) {
        const uint32_t y = (vw[b / 2] >> (16 * (b & 1))) & 0x7fffu;
        if (y < 0x7c00u) {
          top = max(top, y);
        } else {
          wrong |= 1u << b;
          vw[b / 2] &= b & 1 ? 0x0000ffffu : 0xffff0000u;
        }
      }
      top = __reduce_max_sync(0xffffffffu, top);
#pragma unroll 1
      for (uint32_t left = __ballot_sync(0xffffffffu, wrong != 0); left; left &= left - 1) {
        const int i = __ffs(left) - 1;
        const int2 k = make_int2(__shfl_sync(0xffffffffu, key.x, i), __shfl_sync(0xffffffffu, key.y, i));
        const uint32_t groups = __shfl_sync(0xffffffffu, wrong, i);
        spoil(k, groups);
      }
    }
    const uint32_t old = u->cap, cap = max(old, cap_of(top));
    __syncwarp();
    const int lift = lift_of(cap);
    if (cap != old) {
      renew((float)(exponent_of(old) - exponent_of(cap)), power_of_2(lift - lift_of(old)));
      if (lane == 0) {
        u->cap = cap;
        u->base = 25 - exponent_of(cap);
      }
    }
    gate = lift == 0 ? (int)cap : -1;
    const uint32_t f = (uint32_t)(15 + min(lift, 8)) * 0x04000400u, f2 = lift > 8 ? 0x5c005c00u : 0x3c003c00u;  // (f16 has no 2^16)
#pragma unroll
    for (int i = 0; i < W; ++i) vw[i] = mul2(mul2(vw[i], f), f2);
    put_scales();
  }
  __syncwarp();  // (scales that have been written)
}

// Query row r of the unit, of a lane 8 elements of each group, as f16 times 2^k, which is returned: the largest comes to
// 2^14 .. 2^15 (a row without a number above 0: k = 0).  A row that holds an infinity is NaN throughout, or scores of -inf alone
// would leave no weight.  put(b, words): group b in the order of the codes' masks, every second element a sixteenth.
template <typename T, int D, typename Put>
__device__ __forceinline__ int load_query(const NibbleParams& p, const Unit& u, int r, int t, Put put) {
  constexpr int G = D / 32;
  const int at = u.orow[r], tk = at / p.hq;
  const T* q = reinterpret_cast<const T*>(p.q) + (long long)tk * p.q_row + ((long long)u.head * p.hr + (at - tk * p.hq)) * p.q_head;
  uint4 qw[G];
  float big = 0.f;
#pragma unroll
  for (int b = 0; b < G; ++b) {
    qw[b] = r < u.rows ? __ldg(reinterpret_cast<const uint4*>(q + 32 * b + 8 * t)) : make_uint4(0u, 0u, 0u, 0u);
    float f[8];
    piece_get<T>(qw[b], f);
#pragma unroll
    for (int i = 0; i < 8; ++i) big = fmaxf(big, fabsf(f[i]));
  }
  big = fmaxf(big, __shfl_xor_sync(0xffffffffu, big, 1));
  big = fmaxf(big, __shfl_xor_sync(0xffffffffu, big, 2));
  int k = 0;
  if (big > 0.f && big < INFINITY) k = min(14 - ilogbf(big), 120);
  const float up = big == INFINITY ? NAN : ldexpf(1.f, k);
#pragma unroll
  for (int b = 0; b < G; ++b) {
    float f[8];
    piece_get<T>(qw[b], f);
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] *= up;
    put(b, make_uint4(pack_f16x2(f[0], f[4]), pack_f16x2(f[1] * 0.0625f, f[5] * 0.0625f), pack_f16x2(f[2], f[6]),
                      pack_f16x2(f[3] * 0.0625f, f[7] * 0.0625f)));
  }
  return k;
}
template <int N>
__device__ __forceinline__ void load_floats(const float* p, float* x) {
  if constexpr (N == 4) {
    const float4 y = *reinterpret_cast<const float4*>(p);
    x[0] = y.x, x[1] = y.y, x[2] = y.z, x[3] = y.w;
  } else if constexpr (N == 2) {
    const float2 y = *reinterpret_cast<const float2*>(p);
    x[0] = y.x, x[1] = y.y;
  } else {
    x[0] = *p;
  }
}
// A lane's codes of the key in row `row` of a tile: a word a group, elements 8 t .. 8 t + 3 in its low half and + 4 .. + 7 in its high one
template <int D>
__device__ __forceinline__ void key_words(const uint8_t* tile, int row, int t, uint32_t* w) {
  using L = Tile<D>;
  if constexpr (D == 128) {
    const uint4 x = *reinterpret_cast<const uint4*>(tile + L::kK + L::chunk(row, t));
    w[0] = __byte_perm(x.x, x.z, 0x5410);
    w[1] = __byte_perm(x.x, x.z, 0x7632);
    w[2] = __byte_perm(x.y, x.w, 0x5410);
    w[3] = __byte_perm(x.y, x.w, 0x7632);
  } else if constexpr (D == 64) {
    const uint2 x = *reinterpret_cast<const uint2*>(tile + L::kK + row * L::kRow + 8 * t);
    w[0] = __byte_perm(x.x, x.y, 0x5410);
    w[1] = __byte_perm(x.x, x.y, 0x7632);
  } else {
    w[0] = *reinterpret_cast<const uint32_t*>(tile + L::kK + row * L::kRow + 4 * t);
  }
}
// Of half h: xs, a lane's codes (elements 4 g .. 4 g + 3 of each group) of the values of keys 2 t, 2 t + 1, 2 t + 8, 2 t + 9; vs, the scales
// of the first and the second two, a pair a group
template <int D>
__device__ __forceinline__ void value_words(const uint8_t* tile, int h, int g, int t, uint32_t (*xs)[D == 128 ? 2 : 1],
                                            uint32_t (*vs)[D / 32]) {
  using L = Tile<D>;
#pragma unroll
  for (int z = 0; z < 4; ++z) {
    const int row = place(2 * t + (z & 1)) + 8 * (z >> 1) + 16 * h;
    if constexpr (D == 128) {
      const uint2 y = *reinterpret_cast<const uint2*>(tile + L::kV + L::chunk(row, g >> 1) + 8 * (g & 1));
      xs[z][0] = y.x;
      xs[z][1] = y.y;
    } else if constexpr (D == 64) {
      xs[z][0] = *reinterpret_cast<const uint32_t*>(tile + L::kV + row * L::kRow + 4 * g);
    } else {
      xs[z][0] = *reinterpret_cast<const uint16_t*>(tile + L::kV + row * L::kRow + 2 * g);
    }
  }
#pragma unroll
  for (int z = 0; z < 2; ++z) {
    const int k0 = 2 * t + 8 * z + 16 * h;
    if constexpr (D == 128) {
      const uint4 y = *reinterpret_cast<const uint4*>(tile + L::kVS + 8 * k0);
      vs[z][0] = __byte_perm(y.x, y.z, 0x5410);
      vs[z][1] = __byte_perm(y.x, y.z, 0x7632);
      vs[z][2] = __byte_perm(y.y, y.w, 0x5410);
      vs[z][3] = __byte_perm(y.y, y.w, 0x7632);
    } else if constexpr (D == 64) {
      const uint2 y = *reinterpret_cast<const uint2*>(tile + L::kVS + 4 * k0);
      vs[z][0] = __byte_perm(y.x, y.y, 0x5410);
      vs[z][1] = __byte_perm(y.x, y.y, 0x7632);
    } else {
      vs[z][0] = *reinterpret_cast<const uint32_t*>(tile + L::kOne + 2 * k0);
    }
  }
}
// A weight is 2^(y + nm), y = s qs the score in log2 units, nm = 25 - e - m: m follows the row's maximum by kSlack, e is exponent_of
// the scales so far (14 at least), so that a weight is below 2^15, and times a scale, too.  Scores are compared as they are
// summed, s: lim = (m + kSlack) / qs.  This takes a new largest score in, and returns what to multiply the row's sums by.
constexpr float kSlack = 4.f;
__device__ __forceinline__ float new_reference(float most, float qs, float base, float& lim, float& nm) {
  const float old = nm;
  if (most > lim) {
    lim = most + __fdividef(kSlack, qs);
    nm = base - most * qs;
  }
  return ex2_approx(nm - old);  // (0 where there was no maximum, and nothing)
}
// The same for weights that are 2^lower of what they were (nm is rounded: by what it has changed)
__device__ __forceinline__ float lower_reference(float lower, float& nm) {
  const float old = nm;
  if (nm != kNoMax) nm += lower;
  return ex2_approx(nm - old);
}
// The warps' runs: equal ones of all units' tiles, by weight.  A tile is the warp's whose run its beginning lies in; runs are as long as
// the heaviest tile at least, so that the pieces of a unit are those of warps in a row.
struct Runs {
  int warps;
  long long each, more;  // the first `more` runs are longer by 1
  __device__ __forceinline__ Runs(const NibbleParams& p, long long total) {
    warps = (int)max(1LL, min((long long)p.warps, total / 4));
    each = total / warps;
    more = total - each * warps;
  }
  __device__ __forceinline__ long long begin(int w) const { return each * w + min((long long)w, more); }
  __device__ __forceinline__ int of(long long x) const {
    const long long in_large = (each + 1) * more;
    return (int)(x < in_large ? x / (each + 1) : more + (x - in_large) / each);
  }
};
// The record of a unit whose first tile is warp w's; last: where its last one begins
__device__ __forceinline__ SplitRec split_record(const NibbleParams& p, const Unit& u, long long last, int w, long long total) {
  return SplitRec{Runs(p, total).of(last) - w + 1, u.t0, u.r0, u.rows, u.head};
}
// The end of row r's piece, whose sums count in `unit`s: statistics are written (by the lane that `write`s); f and fs, what its sums and those
// of the dense part, if `more`, are to be multiplied by; at, its row of out
struct RowEnd {
  int at;
  float f, fs;
  bool more;
};
__device__ __forceinline__ RowEnd row_end(const NibbleParams& p, const Unit& u, int r, int off, bool direct, bool write, float nm, float sum,
                                          float exact, float unit, long long slot) {
  RowEnd z = {u.orow[r] + u.head * p.hr, unit, 0.f, off == 0 && (u.pfirst > 0 || u.ofirst > 0)};
  float ref = sum == 0.f ? -INFINITY : -nm;
  if (z.more) {  // the first piece takes what the dense part has made of its keys
    const float2 ml = p.state_ml[z.at];
    const float top = fmaxf(ref, ml.x), f1 = ex2_approx(ref - top);
    z.fs = ex2_approx(ml.x - top);
    z.f *= f1;
    sum = fmaf(ml.y, z.fs, sum * f1);
    exact = fmaf(ml.y, z.fs, exact * f1);
    ref = top;
  }
  const float inv = !direct ? 1.f : sum == 0.f ? 0.f : __fdividef(1.f, sum);
  z.f *= inv;
  z.fs *= inv;
  if (write) {
    if (!direct)
      p.part_ml[slot + r] = make_float4(ref, sum, exact, 0.f);
    else if (p.lse)
      p.lse[z.at] = sum == 0.f ? -INFINITY : (log2f(exact) + ref) * 0.693147180559945309f;
  }
  return z;
}

// Tiles off .. off + n - 1 of a unit of up to 8 rows, by one warp; last: where the unit's last tile begins.  The rows are the short
// side of both products (keys x rows, elements x rows); a lane has two of them, 2 t and 2 t + 1.
template <typename T, int D, int STAGES>
__device__ __forceinline__ void attend8(const NibbleParams& p, Unit* up, int off, int n, int cost, long long last, int w, long long total,
                                        uint8_t* smem) {
  using L = Tile<D>;
  constexpr int G = D / 32, ST = STAGES, W = D == 128 ? 2 : 1;  // W: words of a key's scales
  const Unit& u = *up;
  const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  float* ks = reinterpret_cast<float*>(smem);  // [keys][G]
  uint8_t* ring = smem + L::kScales;
  KeyLoader<D, ST> keys(p, u, ring);
  keys.start(off, n);
  float qs[2];
  uint4 hq[G];
  const int k2 = load_query<T, D>(p, u, g, t, [&](int b, const uint4& q4) { hq[b] = q4; });
  int hseq[2], hseen[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    qs[i] = fmaxf(ldexpf(p.sc, 24 - __shfl_sync(0xffffffffu, k2, 4 * (2 * t + i))), 1e-37f);
    hseq[i] = u.seq[2 * t + i];
    hseen[i] = u.seen[2 * t + i];
  }
  float o[G][2][4], lim[2], nm[2], l[4], lx[2];  // l: the rounded weights' sums, twice; lx: the exact ones'
  int gate = -1;
  if (lane == 0) start_scales(up);
#pragma unroll
  for (int i = 0; i < 2; ++i) lim[i] = -kNoMax, nm[i] = kNoMax, lx[i] = 0.f;
#pragma unroll
  for (int i = 0; i < 4; ++i) l[i] = 0.f;
#pragma unroll
  for (int b = 0; b < G; ++b)
#pragma unroll
    for (int i = 0; i < 8; ++i) o[b][i / 4][i % 4] = 0.f;
  auto seen = [&](int2 k, int i) {  // whether row 2 t + i sees a key
    return k.x == -1 || (k.x == hseq[i] && (k.y & ~kBadKey) < hseen[i]);
  };
  int use = 0;
#pragma unroll 1
  for (int j = 0; j < n; ++j) {
    keys.step(off, n, j);
    uint8_t* tile = ring + use * L::kBytes;
    use = use + 1 == ST ? 0 : use + 1;
    const int2 flags = *reinterpret_cast<const int2*>(tile + L::kFlag);
    const bool mixed = flags.x != 0;
    int2 key = {-1, 0};  // key `lane`
    if (mixed) key = *reinterpret_cast<const int2*>(tile + L::kMeta + 8 * lane);
    auto spoil = [&](int2 k, uint32_t groups) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const bool see = seen(k, i);
#pragma unroll
        for (int b = 0; b < G; ++b)
          if (see && ((groups >> b) & 1)) o[b][0][i] = o[b][0][i + 2] = o[b][1][i] = o[b][1][i + 2] = NAN;
      }
    };
    auto renew = [&](float lower, float units) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        float f = lower_reference(lower, nm[i]);
        l[i] *= f;
        l[i + 2] *= f;
        lx[i] *= f;
        f *= units;
#pragma unroll
        for (int b = 0; b < G; ++b) {
          o[b][0][i] *= f;
          o[b][0][i + 2] *= f;
          o[b][1][i] *= f;
          o[b][1][i + 2] *= f;
        }
      }
    };
    take_scales<D>(tile, ks, mixed, key, up, gate, spoil, renew);
    // Half a tile at a time (16 keys): long enough, and short code: pieces are often of a few tiles only.
#pragma unroll 1
    for (int h = 0; h < flags.y; ++h) {
      // ---- scores: of keys 16 h + 8 z + g, z = i / 2, and rows 2 t + i % 2 ----
      float s[4];
      uint32_t kw[2][G];
      float sk[2][G];
#pragma unroll
      for (int z = 0; z < 2; ++z) {
        const int i = g + 16 * h + 8 * z;
        key_words<D>(tile, place(g) + 16 * h + 8 * z, t, kw[z]);
        load_floats<G>(ks + G * i, sk[z]);
      }
#pragma unroll
      for (int b = 0; b < G; ++b) {
        const uint32_t a = kw[0][b], c = kw[1][b], a8 = a >> 8, c8 = c >> 8;
        float d[4] = {0.f, 0.f, 0.f, 0.f};
        mma_f16(d, low8(a), low8(c), high8(a), high8(c), hq[b].x, hq[b].y);
        mma_f16(d, low8(a8), low8(c8), high8(a8), high8(c8), hq[b].z, hq[b].w);
#pragma unroll
        for (int i = 0; i < 4; ++i) s[i] = b == 0 ? d[i] * sk[i / 2][0] : fmaf(d[i], sk[i / 2][b], s[i]);
      }
      if (mixed) {
#pragma unroll
        for (int z = 0; z < 2; ++z) {
          const int2 k = *reinterpret_cast<const int2*>(tile + L::kMeta + 8 * (g + 8 * z + 16 * h));
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            if (k.y < 0) s[2 * z + i] = NAN;
            if (!seen(k, i)) s[2 * z + i] = -INFINITY;
          }
        }
      }
      // ---- weights ----
      if (__any_sync(0xffffffffu, fmaxf(s[0], s[2]) > lim[0] || fmaxf(s[1], s[3]) > lim[1])) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          float y = fmaxf(s[i], s[i + 2]);
#pragma unroll
          for (int z = 4; z < 32; z <<= 1) y = fmaxf(y, __shfl_xor_sync(0xffffffffu, y, z));
          const float f = new_reference(y, qs[i], u.base, lim[i], nm[i]);
          l[i] *= f;
          l[i + 2] *= f;
          lx[i] *= f;
#pragma unroll
          for (int b = 0; b < G; ++b) {
            o[b][0][i] *= f;
            o[b][0][i + 2] *= f;
            o[b][1][i] *= f;
            o[b][1][i + 2] *= f;
          }
        }
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) s[i] = ex2_approx(fmaf(s[i], qs[i & 1], nm[i & 1]));
      if (p.lse) {
        lx[0] += s[0] + s[2];
        lx[1] += s[1] + s[3];
      }
      // weights of keys 2 t, 2 t + 1 and 2 t + 8, 2 t + 9 of the half, row g
      const uint32_t b0 = transpose8(pack_f16x2(s[0], s[1])), b1 = transpose8(pack_f16x2(s[2], s[3]));
      mma_f16(l, 0x3c003c00u, 0x3c003c00u, 0x3c003c00u, 0x3c003c00u, b0, b1);  // (ones)
      // ---- values ----
      uint32_t xs[4][W], vs[2][G];
      value_words<D>(tile, h, g, t, xs, vs);
#pragma unroll
      for (int b = 0; b < G; ++b) {
        const uint32_t pick = b & 1 ? 0x7632 : 0x5410;
        const uint32_t a = __byte_perm(xs[0][b / 2], xs[1][b / 2], pick), c = __byte_perm(xs[2][b / 2], xs[3][b / 2], pick);
        const uint32_t a8 = a >> 8, c8 = c >> 8, p0 = mul2(b0, vs[0][b]), p1 = mul2(b1, vs[1][b]);
        mma_f16(o[b][0], low8(a), high8(a), low8(c), high8(c), p0, p1);
        mma_f16(o[b][1], low8(a8), high8(a8), low8(c8), high8(c8), p0,
                p1);
      }
    }
  }
  // ---------------- the piece's output ----------------
  const bool direct = n == cost;
  const long long slot = (2LL * w + (off == 0 ? 1 : 0)) * p.unit_rows;
  if (!direct && off == 0 && lane == 0) p.recs[w] = split_record(p, u, last, w, total);
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int r = 2 * t + i;
    float sum = l[i], exact = lx[i];
#pragma unroll
    for (int z = 4; z < 32; z <<= 1) exact += __shfl_xor_sync(0xffffffffu, exact, z);
    if (u.seen[r] < 0) sum = exact = NAN;
    if (r < u.rows) {
      const RowEnd z = row_end(p, u, r, off, direct, g == 0, nm[i], sum, exact, power_of_2(24 - lift_of(u.cap)), slot);
#pragma unroll
      for (int b = 0; b < G; ++b) {
        // elements 4 g .. 4 g + 3 of the group
        float y[4] = {o[b][0][i] * z.f, o[b][0][i + 2] * (z.f * 0.0625f), o[b][1][i] * z.f, o[b][1][i + 2] * (z.f * 0.0625f)};
        const int at = 32 * b + 4 * g;
        if (z.more) {
          const float4 q = *reinterpret_cast<const float4*>(p.state_o + (long long)z.at * D + at);
          y[0] = fmaf(q.x, z.fs, y[0]);
          y[1] = fmaf(q.y, z.fs, y[1]);
          y[2] = fmaf(q.z, z.fs, y[2]);
          y[3] = fmaf(q.w, z.fs, y[3]);
        }
        if (direct)
          *reinterpret_cast<uint2*>(reinterpret_cast<T*>(p.out) + (long long)z.at * D + at) =
              make_uint2(Elem<T>::put2(y[0], y[1]), Elem<T>::put2(y[2], y[3]));
        else
          *reinterpret_cast<float4*>(p.part_o + (slot + r) * D + at) = make_float4(y[0], y[1], y[2], y[3]);
      }
    }
  }
  cp_async_wait<0>();
  __syncwarp();
}

// The same for a unit of 9 to 16 rows: these are the long side of both products (rows x keys, rows x elements), scores
// come out as the weights' operand, and a lane has two rows, g and g + 8.
template <typename T, int D, int STAGES>
__device__ __forceinline__ void attend16(const NibbleParams& p, Unit* up, int off, int n, int cost, long long last, int w, long long total,
                                         uint8_t* smem) {
  using L = Tile<D>;
  constexpr int G = D / 32, ST = STAGES, W = D == 128 ? 2 : 1;  // W: words of a key's scales
  const Unit& u = *up;
  const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  float* ks = reinterpret_cast<float*>(smem);  // [keys][G]
  uint8_t* ring = smem + L::kScales;
  uint4* sq = reinterpret_cast<uint4*>(ring + ST * L::kBytes);  // [2][G][32]
  KeyLoader<D, ST> keys(p, u, ring);
  keys.start(off, n);
  float qs[2];
  int hseq[2], hseen[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    hseq[i] = u.seq[8 * i + g];
    hseen[i] = u.seen[8 * i + g];
    const int k = load_query<T, D>(p, u, 8 * i + g, t, [&](int b, const uint4& q4) { sq[(i * G + b) * 32 + lane] = q4; });
    qs[i] = fmaxf(ldexpf(p.sc, 24 - k), 1e-37f);
  }
  float o[G][4][4], lim[2], nm[2], l[4], lx[2];
  int gate = -1;
  if (lane == 0) start_scales(up);
#pragma unroll
  for (int i = 0; i < 2; ++i) lim[i] = -kNoMax, nm[i] = kNoMax, lx[i] = 0.f;
#pragma unroll
  for (int i = 0; i < 4; ++i) l[i] = 0.f;
#pragma unroll
  for (int b = 0; b < G; ++b)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[b][i / 4][i % 4] = 0.f;
  auto seen = [&](int owner, int idx, int i) {  // whether row 8 i + g sees a key
    return owner == -1 || (owner == hseq[i] && (idx & ~kBadKey) < hseen[i]);
  };
  int use = 0;
#pragma unroll 1
  for (int j = 0; j < n; ++j) {
    keys.step(off, n, j);
    uint8_t* tile = ring + use * L::kBytes;
    use = use + 1 == ST ? 0 : use + 1;
    const int2 flags = *reinterpret_cast<const int2*>(tile + L::kFlag);
    const bool mixed = flags.x != 0;
    int2 key = {-1, 0};  // key `lane`
    if (mixed) key = *reinterpret_cast<const int2*>(tile + L::kMeta + 8 * lane);
    auto spoil = [&](int2 k, uint32_t groups) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const bool see = seen(k.x, k.y, i);
#pragma unroll
        for (int b = 0; b < G; ++b)
          if (see && ((groups >> b) & 1)) {
#pragma unroll
            for (int c = 0; c < 4; ++c) o[b][c][2 * i] = o[b][c][2 * i + 1] = NAN;
          }
      }
    };
    auto renew = [&](float lower, float units) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        float f = lower_reference(lower, nm[i]);
        l[2 * i] *= f;
        l[2 * i + 1] *= f;
        lx[i] *= f;
        f *= units;
#pragma unroll
        for (int b = 0; b < G; ++b)
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            o[b][c][2 * i] *= f;
            o[b][c][2 * i + 1] *= f;
          }
      }
    };
    take_scales<D>(tile, ks, mixed, key, up, gate, spoil, renew);
#pragma unroll 1
    for (int h = 0; h < flags.y; ++h) {
      int slot = lane;  // (made anew each time: queries that the compiler keeps in registers over the loop cost others their place)
      asm volatile("" : "+r"(slot));
      // ---- scores: of rows g and g + 8 (i / 2) and keys 16 h + 8 z + 2 t + i % 2 ----
      float s[2][4];
      uint32_t kw[2][G];
#pragma unroll
      for (int z = 0; z < 2; ++z) key_words<D>(tile, place(g) + 16 * h + 8 * z, t, kw[z]);
      float sk[2][2][G];
#pragma unroll
      for (int z = 0; z < 4; ++z) load_floats<G>(ks + G * (16 * h + 8 * (z / 2) + 2 * t + z % 2), sk[z / 2][z % 2]);
#pragma unroll
      for (int b = 0; b < G; ++b) {
        const uint4 qa = sq[b * 32 + slot], qb = sq[(G + b) * 32 + slot];
#pragma unroll
        for (int z = 0; z < 2; ++z) {
          const uint32_t a = kw[z][b], a8 = a >> 8;
          float d[4] = {0.f, 0.f, 0.f, 0.f};
          mma_f16(d, qa.x, qb.x, qa.y, qb.y, low8(a), high8(a));
          mma_f16(d, qa.z, qb.z, qa.w, qb.w, low8(a8), high8(a8));
#pragma unroll
          for (int i = 0; i < 4; ++i) s[z][i] = b == 0 ? d[i] * sk[z][i & 1][0] : fmaf(d[i], sk[z][i & 1][b], s[z][i]);
        }
      }
      if (mixed) {
#pragma unroll
        for (int z = 0; z < 2; ++z) {
          const int4 k = *reinterpret_cast<const int4*>(tile + L::kMeta + 8 * (16 * h + 8 * z + 2 * t));
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int owner = i & 1 ? k.z : k.x, idx = i & 1 ? k.w : k.y;
            if (idx < 0) s[z][i] = NAN;
            if (!seen(owner, idx, i / 2)) s[z][i] = -INFINITY;
          }
        }
      }
      // ---- weights ----
      float most[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) most[i] = fmaxf(fmaxf(s[0][2 * i], s[0][2 * i + 1]), fmaxf(s[1][2 * i], s[1][2 * i + 1]));
      if (__any_sync(0xffffffffu, most[0] > lim[0] || most[1] > lim[1])) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          float y = most[i];
          y = fmaxf(y, __shfl_xor_sync(0xffffffffu, y, 1));
          y = fmaxf(y, __shfl_xor_sync(0xffffffffu, y, 2));
          const float f = new_reference(y, qs[i], u.base, lim[i], nm[i]);
          l[2 * i] *= f;
          l[2 * i + 1] *= f;
          lx[i] *= f;
#pragma unroll
          for (int b = 0; b < G; ++b)
#pragma unroll
            for (int c = 0; c < 4; ++c) {
              o[b][c][2 * i] *= f;
              o[b][c][2 * i + 1] *= f;
            }
        }
      }
#pragma unroll
      for (int z = 0; z < 2; ++z)
#pragma unroll
        for (int i = 0; i < 4; ++i) s[z][i] = ex2_approx(fmaf(s[z][i], qs[i / 2], nm[i / 2]));
      if (p.lse) {
#pragma unroll
        for (int i = 0; i < 2; ++i) lx[i] += (s[0][2 * i] + s[0][2 * i + 1]) + (s[1][2 * i] + s[1][2 * i + 1]);
      }
      const uint32_t a0 = pack_f16x2(s[0][0], s[0][1]), a1 = pack_f16x2(s[0][2], s[0][3]), a2 = pack_f16x2(s[1][0], s[1][1]),
                     a3 = pack_f16x2(s[1][2], s[1][3]);
      mma_f16(l, a0, a1, a2, a3, 0x3c003c00u, 0x3c003c00u);  // (ones)
      // ---- values ----
      uint32_t xs[4][W], vs[2][G];
      value_words<D>(tile, h, g, t, xs, vs);
#pragma unroll
      for (int b = 0; b < G; ++b) {
        const uint32_t pick = b & 1 ? 0x7632 : 0x5410;
        const uint32_t a = __byte_perm(xs[0][b / 2], xs[1][b / 2], pick), c = __byte_perm(xs[2][b / 2], xs[3][b / 2], pick);
        const uint32_t a8 = a >> 8, c8 = c >> 8;
        const uint32_t p0 = mul2(a0, vs[0][b]), p1 = mul2(a1, vs[0][b]), p2 = mul2(a2, vs[1][b]), p3 = mul2(a3, vs[1][b]);
        mma_f16(o[b][0], p0, p1, p2, p3, low8(a), low8(c));
        mma_f16(o[b][1], p0, p1, p2, p3, high8(a), high8(c));
        mma_f16(o[b][2], p0, p1, p2, p3, low8(a8), low8(c8));
        mma_f16(o[b][3], p0, p1, p2, p3, high8(a8), high8(c8));
      }
    }
  }
  // ---------------- the piece's output ----------------
  const bool direct = n == cost;
  const long long slot = (2LL * w + (off == 0 ? 1 : 0)) * p.unit_rows;
  if (!direct && off == 0 && lane == 0) p.recs[w] = split_record(p, u, last, w, total);
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int r = 8 * i + g;
    float sum = l[2 * i], exact = lx[i];
    exact += __shfl_xor_sync(0xffffffffu, exact, 1);
    exact += __shfl_xor_sync(0xffffffffu, exact, 2);
    if (u.seen[r] < 0) sum = exact = NAN;
    if (r < u.rows) {
      const RowEnd z = row_end(p, u, r, off, direct, t == 0, nm[i], sum, exact, power_of_2(24 - lift_of(u.cap)), slot);
#pragma unroll
      for (int b = 0; b < G; ++b) {
        // elements 8 t .. 8 t + 7 of the group
        float y[8];
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          const float f = c & 1 ? z.f * 0.0625f : z.f;
          y[c] = o[b][c][2 * i] * f;
          y[4 + c] = o[b][c][2 * i + 1] * f;
        }
        const int at = 32 * b + 8 * t;
        if (z.more) {
#pragma unroll
          for (int c = 0; c < 8; c += 4) {
            const float4 q = *reinterpret_cast<const float4*>(p.state_o + (long long)z.at * D + at + c);
            y[c] = fmaf(q.x, z.fs, y[c]);
            y[c + 1] = fmaf(q.y, z.fs, y[c + 1]);
            y[c + 2] = fmaf(q.z, z.fs, y[c + 2]);
            y[c + 3] = fmaf(q.w, z.fs, y[c + 3]);
          }
        }
        if (direct) {
          *reinterpret_cast<uint4*>(reinterpret_cast<T*>(p.out) + (long long)z.at * D + at) = piece_put<T>(y);
        } else {
          float* to = p.part_o + (slot + r) * D + at;
          *reinterpret_cast<float4*>(to) = make_float4(y[0], y[1], y[2], y[3]);
          *reinterpret_cast<float4*>(to + 4) = make_float4(y[4], y[5], y[6], y[7]);
        }
      }
    }
  }
  cp_async_wait<0>();
  __syncwarp();
}

template <typename T, int D, int NT>
__global__ void __launch_bounds__(kThreads, AttendCfg<D, NT>::kCtas) nibble_attend_kernel(const NibbleParams p) {
  using C = AttendCfg<D, NT>;
  extern __shared__ __align__(16) uint8_t smem[];
  __shared__ long long sh[kWarps + 1], sh_cum[kFewSlots + 1];
  __shared__ int sh_group[kFewSlots];
  const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5;
  prefetch_indices(p);
  pdl_trigger();
  pdl_wait();
  const int w = blockIdx.x * kWarps + wid;
  // offsets that are not increasing from 0 to their ends would leave rows out: each CTA looks at some of them
  {
    bool bad = p.row_start[0] != 0 || p.row_start[p.n_seqs] != p.n_rows;
    for (int s = blockIdx.x * kThreads + threadIdx.x; s < p.n_seqs; s += gridDim.x * kThreads) bad |= p.row_start[s] > p.row_start[s + 1];
    if (p.group_start) {
      bad |= p.group_start[0] != 0 || p.group_start[p.n_groups] != p.n_seqs;
      for (int g = blockIdx.x * kThreads + threadIdx.x; g < p.n_groups; g += gridDim.x * kThreads)
        bad |= p.group_start[g] > p.group_start[g + 1];
    }
    bad = __syncthreads_or(bad);
    if (threadIdx.x == 0) p.bad[blockIdx.x] = bad;
  }
  if (lane == 0) p.recs[w].count = 0;
  const long long* cum = p.cum;
  const int* slot_group = p.slot_group;
  if (p.n_slots <= kFewSlots) {
    sum_slots<kThreads>(p, p.n_slots, sh_cum, sh, [&](int i) {
      const int group = group_of_slot(p, p.unit_rows, i);
      sh_group[i] = group;
      return slot_cost(p, i, group);
    });
    cum = sh_cum;
    slot_group = sh_group;
  }
  const long long total = cum[p.n_slots];
  const Runs runs(p, total);
  if (total == 0 || w >= runs.warps) return;
  const long long x = runs.begin(w), end = runs.begin(w + 1);
  // (unused row tiles have no key tiles: the last of equal sums is a used one)
  int slot = warp_find(cum, p.n_slots, x);
  long long weight = (cum[slot + 1] - cum[slot]) / p.hkv;  // of a unit
  int head = (int)((x - cum[slot]) / weight);
  long long begin = cum[slot] + head * weight;
  Unit* u = reinterpret_cast<Unit*>(smem + (size_t)wid * C::kWarp);
  bool opened = false;  // the row tile's rows are known
  while (begin < end) {
    if (!opened) {
      opened = true;
      while (cum[slot + 1] == cum[slot]) ++slot;
      weight = (cum[slot + 1] - cum[slot]) / p.hkv;
      const RowTile tile = row_tile(p, p.unit_rows, slot_group[slot], slot);
      int plen = p.prefix_of(tile.group);
      const bool prefix_fine = p.prefix_ok(plen);
      plen = prefix_fine ? plen : 0;
      const int pfirst = p.dense_prefix(plen), ofirst = p.dense_own(p.group_first(tile.group));
      int seq = -5, seen = 0, orow = 0;
      if (lane < tile.rows) {
        const int tk = (tile.r0 + lane) / p.hr, h = tile.r0 + lane - tk * p.hr, tt = tile.t0 + tk;
        seq = seq_of(p, p.group_first(tile.group), p.group_first(tile.group + 1), tile.t0, tile.t1, tt);
        const int a = p.row_start[seq], b = p.row_start[seq + 1], len = p.seq_len[seq];
        seen = p.len_ok(len) && prefix_fine ? seen_by(len, a, b, tt) : -1;
        orow = tt * p.hq + h;
      }
      const int next = __shfl_down_sync(0xffffffffu, seq, 1);
      const int keys = lane < tile.rows && (lane == tile.rows - 1 || next != seq) ? max(seen - ofirst, 0) : 0;
      int start = keys;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int v = __shfl_up_sync(0xffffffffu, start, o);
        if (lane >= o) start += v;
      }
      const int own_keys = __shfl_sync(0xffffffffu, start, 31), first_seq = __shfl_sync(0xffffffffu, seq, 0);
      const int last_seq = __shfl_sync(0xffffffffu, seq, tile.rows - 1);
      const int all_see = __reduce_min_sync(0xffffffffu, lane < tile.rows ? max(seen, 0) : 0x7fffffff);
      u->seq[lane] = seq;
      u->seen[lane] = seen;
      u->start[lane] = start - keys;
      u->orow[lane] = orow;
      if (lane == 0) {
        u->group = tile.group;
        u->t0 = tile.t0;
        u->r0 = tile.r0;
        u->rows = tile.rows;
        u->plen = plen;
        u->pfirst = pfirst;
        u->ofirst = ofirst;
        u->ptiles = (plen - pfirst + kKeys - 1) / kKeys;
        u->own_keys = own_keys;
        u->all_see = all_see;
        u->first_seq = first_seq;
        u->alone = first_seq == last_seq;
      }
    }
    if (lane == 0) u->head = head;
    __syncwarp();
    uint8_t* mine = reinterpret_cast<uint8_t*>(u + 1);
    const int rows = u->rows, part = tile_weight(rows), cost = (int)(weight / part);
    // the tiles that begin within the run
    const int off = begin >= x ? 0 : (int)((x - begin + part - 1) / part), n = (int)min((long long)cost, (end - begin + part - 1) / part) - off;
    const long long last = begin + (long long)(cost - 1) * part;
    if (n > 0) {
      if (NT == 1 || rows <= 8)
        attend8<T, D, C::kStages>(p, u, off, n, cost, last, w, total, mine);
      else
        attend16<T, D, C::kStages>(p, u, off, n, cost, last, w, total, mine);
    }
    begin += weight;
    if (++head == p.hkv) {
      head = 0;
      ++slot;
      opened = false;
    }
  }
}

// ---------------------------------------------------------------------------
// finish
// ---------------------------------------------------------------------------
// CTA (x, y) joins rows of the split units that warps 8 x .. 8 x + 7 have begun
constexpr int kFewPieces = 8;
template <typename T, int D>
__global__ void __launch_bounds__(256) nibble_finish_kernel(const NibbleParams p, const int ctas) {
  constexpr int N = D / 32;
  __shared__ float so[8][D];
  __shared__ float4 sml[8];
  __shared__ SplitRec recs[8];
  pdl_trigger();
  pdl_wait();
  const int lane = threadIdx.x & 31, wp = threadIdx.x >> 5, w0 = 8 * blockIdx.x;
  SplitRec mine{};
  if (lane == 0 && w0 + wp < p.warps) mine = p.recs[w0 + wp];
  int bad = 0;
  for (int i0 = 0; i0 < ctas; i0 += 1024) {  // (four loads at once)
    int x[4];
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      const int i = i0 + 256 * c + threadIdx.x;
      x[c] = i < ctas ? p.bad[i] : 0;
    }
    bad |= x[0] | x[1] | x[2] | x[3];
  }
  if (lane == 0) recs[wp] = mine;
  if (__syncthreads_or(bad)) {
    const long long rows = (long long)p.n_rows * p.hq, nw = (long long)gridDim.x * gridDim.y * 8;
    for (long long w = ((long long)blockIdx.y * gridDim.x + blockIdx.x) * 8 + wp; w < rows; w += nw) {
      T* out = reinterpret_cast<T*>(p.out) + w * D;
      for (int i = lane; i < D; i += 32) out[i] = Elem<T>::put(NAN);
      if (p.lse && lane == 0) p.lse[w] = NAN;
    }
    if (blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0 && p.status) atomicOr(p.status, FE_ST_INDEX);
    return;
  }
  if (p.dense && blockIdx.x == 0 && blockIdx.y == 0 && p.status)
    for (int i = threadIdx.x; i < p.dctas; i += 256)
      if (p.stat[i]) atomicOr(p.status, p.stat[i]);
  struct alignas(4 * N) Values {
    float v[N];
  };
  struct alignas(2 * N) Outputs {
    T v[N];
  };
  // (w: the warp that has begun the unit)
  auto slot = [&](int w, int i, int r) { return (2LL * (w + i) + (i == 0)) * p.unit_rows + r; };
  auto put = [&](const SplitRec& rec, int r, float m, float l, float lx, const float* o) {
    const int rr = rec.r0 + r;
    const long long at = (long long)(rec.t0 + rr / p.hr) * p.hq + rec.head * p.hr + rr % p.hr;
    const float inv = l == 0.f ? 0.f : 1.f / l;
    Outputs y;
#pragma unroll
    for (int z = 0; z < N; ++z) y.v[z] = Elem<T>::put(o[z] * inv);
    reinterpret_cast<Outputs*>(reinterpret_cast<T*>(p.out) + at * D)[lane] = y;
    if (p.lse && lane == 0) p.lse[at] = l == 0.f ? -INFINITY : (m + log2f(lx)) * 0.693147180559945309f;
  };
  // pieces first, first + step, ... of row r; references and sums of 32 of them at once, a lane each
  auto join = [&](const SplitRec& rec, int w, int r, int first, int step, float& m, float& l, float& lx, float* o) {
    m = -INFINITY, l = 0.f, lx = 0.f;
#pragma unroll
    for (int z = 0; z < N; ++z) o[z] = 0.f;
    for (int i0 = first; i0 < rec.count; i0 += 32 * step) {
      const int mine = i0 + lane * step, n = min(32, (rec.count - i0 + step - 1) / step);
      const float4 ml = mine < rec.count ? p.part_ml[slot(w, mine, r)] : make_float4(-INFINITY, 0.f, 0.f, 0.f);
      constexpr int U = 8;  // sums read at once (those past the last piece: none, times 0); the first ones with the references
      Values x[U];
      auto read = [&](int i) {
#pragma unroll
        for (int c = 0; c < U; ++c)
          x[c] = i + c < n ? reinterpret_cast<const Values*>(p.part_o + slot(w, i0 + (i + c) * step, r) * D)[lane] : Values{};
      };
      read(0);
      float top = ml.x;
#pragma unroll
      for (int z = 16; z > 0; z >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, z));
      const float m1 = fmaxf(m, top), ref = m1 == -INFINITY ? 0.f : m1;
      const float old = ex2_approx(m - ref), f = ex2_approx(ml.x - ref);
      m = m1;
      float sum = ml.y * f, exact = ml.z * f;
#pragma unroll
      for (int z = 16; z > 0; z >>= 1) {
        sum += __shfl_xor_sync(0xffffffffu, sum, z);
        exact += __shfl_xor_sync(0xffffffffu, exact, z);
      }
      l = fmaf(l, old, sum);
      lx = fmaf(lx, old, exact);
#pragma unroll
      for (int z = 0; z < N; ++z) o[z] *= old;
#pragma unroll 1
      for (int i = 0; i < n; i += U) {
#pragma unroll
        for (int c = 0; c < U; ++c) {
          const float fi = __shfl_sync(0xffffffffu, f, i + c);
#pragma unroll
          for (int z = 0; z < N; ++z) o[z] = fmaf(x[c].v[z], fi, o[z]);
        }
        read(i + U);
      }
    }
  };
  float m, l, lx, o[N];
  // units of few pieces: a row a warp, of all eight units
  for (int z = blockIdx.y * 8 + wp; z < 8 * p.unit_rows; z += 8 * gridDim.y) {
    const int k = z / p.unit_rows, r = z % p.unit_rows;
    const SplitRec rec = recs[k];
    if (rec.count == 0 || rec.count > kFewPieces || r >= rec.rows) continue;
    join(rec, w0 + k, r, 0, 1, m, l, lx, o);
    put(rec, r, m, l, lx, o);
  }
  // of many: a row a CTA
  for (int k = 0; k < 8; ++k) {
    const SplitRec rec = recs[k];
    if (rec.count <= kFewPieces) continue;
    for (int r = blockIdx.y; r < rec.rows; r += gridDim.y) {
      join(rec, w0 + k, r, wp, 8, m, l, lx, o);
      if (lane == 0) sml[wp] = make_float4(m, l, lx, 0.f);
#pragma unroll
      for (int z = 0; z < N; ++z) so[wp][N * lane + z] = o[z];
      __syncthreads();
      if (wp == 0) {
        m = -INFINITY, l = 0.f, lx = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) m = fmaxf(m, sml[i].x);
        const float ref = m == -INFINITY ? 0.f : m;
#pragma unroll
        for (int z = 0; z < N; ++z) o[z] = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float f = ex2_approx(sml[i].x - ref);
          l = fmaf(sml[i].y, f, l);
          lx = fmaf(sml[i].z, f, lx);
#pragma unroll
          for (int z = 0; z < N; ++z) o[z] = fmaf(so[i][N * lane + z], f, o[z]);
        }
        put(rec, r, m, l, lx, o);
      }
      __syncthreads();
    }
  }
}

int check_attention(const fe_nibble_attention_args* a) {
  if (!a) return fail(FE_ERR_INVALID_ARG, "null arguments");
  const int rc = check_nibble_kv(a->kv);
  if (rc != FE_OK) return rc;
  const bool groups = a->group_start || a->prefix_len || a->prefix_pages || a->n_groups != 0;
  if (a->n_groups < 0 || a->n_seqs < 0 || a->n_rows < 0 || a->page_cols < 1 || (groups && a->prefix_cols < 1))
    return fail(FE_ERR_INVALID_ARG, "negative size or no page column");
  if (a->q_heads < 1 || a->q_heads % a->kv.kv_heads != 0)
    return fail(FE_ERR_INVALID_ARG, "q_heads must be a multiple of kv_heads");
  if (a->q_heads / a->kv.kv_heads > 1024) return fail(FE_ERR_UNSUPPORTED, "at most 1024 query heads a key head");
  if ((long long)a->n_rows * a->q_heads > 0x7fffffffLL)
    return fail(FE_ERR_UNSUPPORTED, "n_rows * q_heads must be below 2^31");
  if ((long long)a->page_cols * a->kv.page_rows > (1 << 26) || (groups && (long long)a->prefix_cols * a->kv.page_rows > (1 << 26)))
    return fail(FE_ERR_UNSUPPORTED, "at most 2^26 rows a sequence or prefix");
  if (a->n_seqs > (1 << 27) || a->n_groups > (1 << 27)) return fail(FE_ERR_UNSUPPORTED, "at most 2^27 sequences");
  if (!std::isfinite(a->scale) || a->scale < 0.f) return fail(FE_ERR_INVALID_ARG, "scale must be finite and not negative");
  if (a->n_rows == 0) return FE_OK;
  if (a->n_seqs == 0 || (groups && a->n_groups == 0)) return fail(FE_ERR_INVALID_ARG, "rows without a sequence or group");
  if (groups && (!a->group_start || !a->prefix_len || !a->prefix_pages)) return fail(FE_ERR_INVALID_ARG, "null pointer");
  if (!a->row_start || !a->seq_len || !a->pages || !a->q || !a->out) return fail(FE_ERR_INVALID_ARG, "null pointer");
  if (a->out == a->q) return fail(FE_ERR_INVALID_ARG, "out must not be q");
  if (misaligned(a->q, 16) || misaligned(a->out, 32) || a->q_row % 8 != 0 || a->q_head % 8 != 0)
    return fail(FE_ERR_UNSUPPORTED, "q must be 16-byte aligned, its strides multiples of 8, out 32-byte aligned");
  return FE_OK;
}

// Sizes of the workspace's parts, in order, each on a 256-byte boundary
struct Layout {
  size_t bad, cum, slot_group, recs, part_o, part_ml, stat, dcum, dslot_group, drecs, dpart_o, dpart_ml, state_o, state_ml, bytes;
};
// Rows a group, on average, above which keys that they share go through the dense part.  What a call takes with it, and without |
// with it and the keys' rest (us, a replayed graph; bf16, 6 own rows a sequence), by rows a group:
//                                               16             32              48              64
//   4 prefixes of 32768, 32 over 8 of 128    110, 91 | 141   110, 130 | 147  116, 175 | 147  118, 220 | 149
//   4 of 8192                                 67, 56 | 74     69, 65 | 77     71, 79 | 78     73, 91 | 81
//   64 of 1024, 16 over 4 of 64               59, 56 | 65     65, 54 | 69     73, 64 | 75     69, 77 | 73
//   256 of 256, 4 of 32                       67, 71 | 71     77, 69 | 79     88, 80 | 91     97, 91 | 101
// So 32 lies between the crossings of long prefixes (20 and 37 rows of the first, 37 and 48 of the second) and short ones (some 55
// of the third); a rule that looked at lengths would need them on the host.
constexpr int kDenseFrom = 32;
// What a call is run with: rows of a unit and warps
struct Shape {
  int nt, ctas, groups, slots;
  bool dense;
  int dslots, dctas;
  int rows() const { return 8 * nt; }
};

// Rows of a unit: 8, unless the groups have more on average.
Shape shape_of(const fe_nibble_attention_args* a, int sms) {
  Shape s{};
  s.groups = a->group_start ? a->n_groups : a->n_seqs;
  const long long rows = (long long)a->n_rows * (a->q_heads / a->kv.kv_heads);
  // (the dense part: for groups of more rows than a warp takes; what is left then is mostly sequences' own rows, which their
  // own queries alone see)
  s.dense = rows > kDenseFrom * (long long)s.groups;
  s.nt = rows <= 8LL * (s.dense ? a->n_seqs : s.groups) ? 1 : 2;
  s.ctas = sms * ctas_of(a->kv.head_dim, s.nt);
  s.slots = (int)(rows / s.rows() + s.groups);
  s.dslots = (int)(rows / kDenseRows + s.groups);
  s.dctas = 2 * sms;
  return s;
}
Layout layout(const fe_nibble_attention_args* a, const Shape& s) {
  size_t at = 0;
  auto take = [&](size_t n) {
    const size_t x = at;
    at += (n + 255) / 256 * 256;
    return x;
  };
  Layout w;
  const size_t warps = (size_t)s.ctas * kWarps;
  w.bad = take(4 * (size_t)s.ctas);
  w.cum = take(8 * ((size_t)s.slots + 1));
  w.slot_group = take(4 * (size_t)s.slots);
  w.recs = take(sizeof(SplitRec) * warps);
  w.part_o = take(warps * 2 * s.rows() * a->kv.head_dim * 4);
  w.part_ml = take(warps * 2 * s.rows() * 16);
  w.stat = w.dcum = w.dslot_group = w.drecs = w.dpart_o = w.dpart_ml = w.state_o = w.state_ml = at;
  if (s.dense) {
    const size_t d = a->kv.head_dim, ctas = s.dctas, rows = (size_t)a->n_rows * a->q_heads;
    w.stat = take(4 * ctas);
    w.dcum = take(8 * ((size_t)s.dslots + 1));
    w.dslot_group = take(4 * (size_t)s.dslots);
    w.drecs = take(sizeof(SplitRec) * ctas);
    w.dpart_o = take(ctas * 2 * kDenseRows * d * 4);
    w.dpart_ml = take(ctas * 2 * kDenseRows * 8);
    w.state_o = take(rows * d * 4);
    w.state_ml = take(rows * 8);
  }
  w.bytes = at;
  return w;
}

template <typename T, int D, int NT>
cudaError_t attend_go(const NibbleParams& p, const Shape& sh, cudaStream_t s) {
  using C = AttendCfg<D, NT>;
  // (once per device would do; the call costs nothing that a user sees)
  cudaError_t e = cudaFuncSetAttribute((const void*)nibble_attend_kernel<T, D, NT>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)C::kSmem);
  if (e == cudaSuccess && p.n_slots > kFewSlots) e = launch_k(nibble_plan_kernel, dim3(kPlanCtas), dim3(kPlanThreads), 0, s, p);
  if (e == cudaSuccess) e = launch_k(nibble_attend_kernel<T, D, NT>, dim3((unsigned)sh.ctas), dim3(kThreads), C::kSmem, s, p);
  if (e == cudaSuccess)
    e = launch_k(nibble_finish_kernel<T, D>, dim3((unsigned)(p.warps + 7) / 8, 4), dim3(256), 0, s, p, sh.ctas);
  return e;
}
template <typename T>
cudaError_t attend_dim(const NibbleParams& p, const Shape& sh, int d, cudaStream_t s) {
  if (d == 32) return sh.nt == 1 ? attend_go<T, 32, 1>(p, sh, s) : attend_go<T, 32, 2>(p, sh, s);
  if (d == 64) return sh.nt == 1 ? attend_go<T, 64, 1>(p, sh, s) : attend_go<T, 64, 2>(p, sh, s);
  return sh.nt == 1 ? attend_go<T, 128, 1>(p, sh, s) : attend_go<T, 128, 2>(p, sh, s);
}

}  // namespace
}  // namespace fe

extern "C" uint64_t fe_nibble_attention_workspace(const fe_nibble_attention_args* a) {
  using namespace fe;
  if (check_attention(a) != FE_OK) return 0;
  int sms = 0;
  const cudaError_t e = device_sms(&sms);
  if (e != cudaSuccess) {
    fail_cuda(e, "fe_nibble_attention_workspace");
    return 0;
  }
  return layout(a, shape_of(a, sms)).bytes;
}

extern "C" int fe_nibble_attention(const fe_nibble_attention_args* a, void* stream) {
  using namespace fe;
  const int rc = check_attention(a);
  if (rc != FE_OK) return rc;
  if (a->n_rows == 0) return FE_OK;
  if (!a->workspace || misaligned(a->workspace, 256)) return fail(FE_ERR_INVALID_ARG, "workspace null or not 256-byte aligned");
  int sms = 0;
  cudaError_t e = device_sms(&sms);
  if (e != cudaSuccess) return fail_cuda(e, "fe_nibble_attention");
  const Shape sh = shape_of(a, sms);
  const Layout w = layout(a, sh);
  if (a->workspace_bytes < w.bytes) return fail(FE_ERR_WORKSPACE, "workspace too small");
  char* ws = static_cast<char*>(a->workspace);
  NibbleParams p{};
  p.slot_group = reinterpret_cast<int*>(ws + w.slot_group);
  p.bad = reinterpret_cast<int*>(ws + w.bad);
  p.cum = reinterpret_cast<long long*>(ws + w.cum);
  p.recs = reinterpret_cast<SplitRec*>(ws + w.recs);
  p.part_o = reinterpret_cast<float*>(ws + w.part_o);
  p.part_ml = reinterpret_cast<float4*>(ws + w.part_ml);
  // (not without a tile of keys that a page table has room for)
  p.dense = sh.dense && (long long)(a->group_start ? a->prefix_cols : a->page_cols) * a->kv.page_rows >= kDenseKeys;
  p.n_dslots = sh.dslots;
  p.dctas = sh.dctas;
  p.stat = reinterpret_cast<int*>(ws + w.stat);
  p.dcum = reinterpret_cast<long long*>(ws + w.dcum);
  p.dslot_group = reinterpret_cast<int*>(ws + w.dslot_group);
  p.drecs = reinterpret_cast<SplitRec*>(ws + w.drecs);
  p.dpart_o = reinterpret_cast<float*>(ws + w.dpart_o);
  p.dpart_ml = reinterpret_cast<float2*>(ws + w.dpart_ml);
  p.state_o = reinterpret_cast<float*>(ws + w.state_o);
  p.state_ml = reinterpret_cast<float2*>(ws + w.state_ml);
  p.warps = sh.ctas * kWarps;
  p.n_slots = sh.slots;
  p.unit_rows = sh.rows();
  p.group_start = a->group_start;
  p.prefix_len = a->prefix_len;
  p.prefix_pages = a->prefix_pages;
  p.row_start = a->row_start;
  p.seq_len = a->seq_len;
  p.pages = a->pages;
  p.kc = static_cast<const uint8_t*>(a->kv.k_codes);
  p.vc = static_cast<const uint8_t*>(a->kv.v_codes);
  p.ks = static_cast<const __half*>(a->kv.k_scales);
  p.vs = static_cast<const __half*>(a->kv.v_scales);
  p.q = a->q;
  p.out = a->out;
  p.lse = a->lse;
  p.status = a->status;
  p.q_row = a->q_row;
  p.q_head = a->q_head;
  p.n_groups = sh.groups;
  p.n_seqs = a->n_seqs;
  p.n_rows = a->n_rows;
  p.hq = a->q_heads;
  p.hkv = a->kv.kv_heads;
  p.hr = p.hq / p.hkv;
  p.prefix_cols = a->prefix_cols;
  p.page_cols = a->page_cols;
  p.page_rows = a->kv.page_rows;
  while ((1 << p.page_shift) < p.page_rows) ++p.page_shift;
  p.n_pages = a->kv.n_pages;
  p.sc = (float)(a->scale * 1.4426950408889634);
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (p.dense && (e = nibble_dense(p, a->kv.head_dim, a->kv.dtype == FE_IO_F16, s)) != cudaSuccess) return fail_cuda(e, "fe_nibble_attention");
  e = a->kv.dtype == FE_IO_BF16 ? attend_dim<__nv_bfloat16>(p, sh, a->kv.head_dim, s) : attend_dim<__half>(p, sh, a->kv.head_dim, s);
  return e == cudaSuccess ? FE_OK : fail_cuda(e, "fe_nibble_attention");
}
