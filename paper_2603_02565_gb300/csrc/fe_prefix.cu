// Attention of groups of sequences that share a prefix, over a paged cache
// (fe_prefix_attention).
//
// For row t of sequence s in group g, with n_s rows in the call and j = t - row_start[s]:
//   p_k = softmax_k(scale q . k) over the prefix's prefix_len[g] rows and the sequence's
//   own rows 0 .. seq_len[s] - n_s + j,  out = sum_k p_k v_k.
//
// Unit of work: up to 128 query rows of a group that read the same key head (tokens x the
// query heads of that key head), so that a prefix key is loaded once for all of them.
// Its keys come in tiles of 128: first the prefix's, then the own rows of the unit's
// sequences, packed in slots of 16 keys (a slot has one owner; a row masks the slots of
// others), so short sequences share tiles and decoding needs no second kernel for them.
//   plan kernel     counts each unit's tiles from the lengths in device memory;
//   attend kernel   two CTAs per SM, each takes an equal run of all units' tiles, wherever
//                   it begins or ends: few units with long prefixes are split over the SMs;
//   finish kernel   joins the pieces of split units by their maxima and sums, and computes
//                   some rows again, key by key (see below).
//
// A CTA of the attend kernel has four softmax warps (a row a thread) and four that feed
// them: one walks the schedule, one issues tcgen05.mma (S = Q K^T, and O += P V with P from
// TMEM), one loads queries and keys, one loads values and looks through them.  S, P and O
// live in half of the SM's TMEM.  What such a warp does is a chain of short steps: the two
// CTAs fill each other's gaps.  (One CTA per SM with two groups of softmax warps, on
// alternate tiles or on 256 rows, joined at the unit's end, had the same steps in one chain
// for both.)  Eight unlike roles compete for the instruction cache: a third of all stalls
// were for instructions while loops were unrolled; rolled ones took a quarter off.
//
// Device time of a call:
//   4 groups x 16 sequences, a token each, prefixes up to 32768 keys, 32 heads of 8 x 128:
//     112 us, 4.3 TB/s.  Bound by how much a CTA has in flight: reads alone, 64 KB in flight
//     an SM, reach 5.1 TB/s in boxes of 64 rows (a copy 6.8);
//   2 groups x 8 sequences, up to 256 rows each, prefixes of 8192, the same heads:
//     411 us, 1130 TFLOP/s (cuBLAS 1895).  The products take half of the time, the chain
//     scores - maximum - weights - product of two CTAs the rest;
//   256 groups x 50 sequences, a token each, prefixes of 256, 4 heads of 32: 88 us (bytes
//     alone 9): a tile's steps again, for nine tiles a unit of which seven are own keys, one to six of
//     them in a slot of 16;
//   1 group x 4 sequences, prefix of 300, 8 heads of 64: 17 us, of which three launches 8.
// A tile of 128 keys that a row sees whole costs it 128 exponentials, at sixteen a clock and SM 1.1 us
// for the tiles of both CTAs (a row that sees one slot of a tile: 16).
//
// 0 x NaN is NaN, so a value that is no number spoils rows that give it no weight.  The
// values' warp clears the value rows past a sequence's end, whatever the pages hold there,
// and looks through tiles of own keys, which rows of other sequences (and earlier rows of
// the same one) do not see: infinities and NaN there become 0 in the tile, and all rows of
// the sequence that has them are computed again from their visible keys alone.  Nothing is
// looked for in the prefix, which all rows see.
#include <cmath>
#include <mutex>

#include "fe_ops.cuh"

namespace fe {
namespace {

constexpr int kUnitRows = 128, kTileKeys = 128, kSlot = 16, kSlots = kTileKeys / kSlot;
constexpr int kDirty = 3, kUnitsAhead = 8;

struct PlanHead {
  int status;   // ST_ bits of this call
  int bad;      // the row or group offsets are not what they must be: all rows NaN
  int listed;   // rows to compute again
};
// A split unit: its rows, and the CTAs that have its pieces (count 0: none).  While the schedule runs, count is its
// tiles, the first of them tile.
struct SplitRec {
  int first, count, t0, r0, rows, head;
  long long tile;
};

struct PrefixParams {
  const int32_t *group_start, *prefix_len, *prefix_pages, *row_start, *seq_len, *pages;
  const void *q, *k, *v;
  void* out;
  float* lse;
  int32_t* status;
  int64_t q_row, q_head;
  int n_groups, n_seqs, n_rows, hq, hkv, hr, hr_inv, prefix_cols, page_cols, page_rows, page_shift, n_pages;
  float scale, sc;  // sc: scale log2(e), and no 0 (masked scores, -inf, are multiplied by it)
  int ctas;
  // workspace
  PlanHead* head;
  int2* tok;           // [n_rows] sequence of a row, and how many of its own rows it sees (-1: a length is none)
  int* gtile;          // [n_groups + 1] first row tile of a group
  long long* gcost;    // [n_groups + 1] key tiles of all heads before a group
  int* cost;           // [max_tiles] key tiles of a row tile (one head), at least 1
  long long* before;   // [max_tiles + 1] key tiles of one head before a row tile
  SplitRec* recs;      // [ctas][2] the split unit that a CTA begins in the middle of, the one it ends in the middle of
  int* list;           // [n_rows hq] rows of the output to compute again: those that a CTA has whole and that are NaN
  float* part_o;       // [ctas][2][kUnitRows][D]
  float2* part_ml;     // [ctas][2][kUnitRows] reference (about the maximum, log2 units) and sum of the weights
};

// The sequence's own rows that row j of its n sees, and whether its length is one
__device__ __forceinline__ bool len_ok(const PrefixParams& p, int len) {
  return len >= 0 && (long long)len <= (long long)p.page_cols * p.page_rows;
}
__device__ __forceinline__ bool prefix_ok(const PrefixParams& p, int n) {
  return n >= 0 && (long long)n <= (long long)p.prefix_cols * p.page_rows;
}
__device__ __forceinline__ int seen_rows(int len, int n, int j) { return max(0, min(len, len - n + j + 1)); }

// ---------------------------------------------------------------------------
// plan
// ---------------------------------------------------------------------------
constexpr int kPlanThreads = 1024, kPlanGroups = 2048, kPlanCtas = 8;
static_assert(kPlanThreads == 1024, "block_scan sums the totals of 32 warps");

// inclusive sum over the block's threads
template <typename V>
__device__ V block_scan(V v, V* sh) {
  const int lane = threadIdx.x & 31, wp = threadIdx.x >> 5;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const V u = __shfl_up_sync(0xffffffffu, v, o);
    if (lane >= o) v += u;
  }
  __syncthreads();
  if (lane == 31) sh[wp] = v;
  __syncthreads();
  if (wp == 0) {
    V w = sh[lane];
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const V u = __shfl_up_sync(0xffffffffu, w, o);
      if (lane >= o) w += u;
    }
    sh[lane] = w;
  }
  __syncthreads();
  return wp > 0 ? v + sh[wp - 1] : v;
}

// the largest i < n with a[i] <= x (a[0] <= x)
template <typename V>
__device__ __forceinline__ int find_last(const V* a, int n, V x) {
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (a[mid] <= x)
      lo = mid;
    else
      hi = mid;
  }
  return lo;
}

__device__ __forceinline__ void plan_barrier() {  // of the cluster, global writes included
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}

// One cluster: what is counted per sequence and row is spread over its CTAs, the sums over groups and row tiles are
// the first one's.
__global__ void __launch_bounds__(kPlanThreads) __cluster_dims__(kPlanCtas, 1, 1) prefix_plan_kernel(const PrefixParams p) {
  __shared__ long long sh[32];
  __shared__ int sh_i[32];
  __shared__ int sh_groups[kPlanGroups], sh_first[kPlanGroups], sh_tile[kPlanGroups];
  pdl_trigger();
  pdl_wait();
  const int tid = threadIdx.x, all = blockIdx.x * kPlanThreads + tid;
  constexpr int kAll = kPlanThreads * kPlanCtas;
  // offsets that are not increasing from 0 to their ends would send rows nowhere
  bool bad = p.row_start[0] != 0 || p.row_start[p.n_seqs] != p.n_rows || p.group_start[0] != 0 ||
             p.group_start[p.n_groups] != p.n_seqs;
  for (int g = tid; g < p.n_groups; g += kPlanThreads) bad |= p.group_start[g] > p.group_start[g + 1];
#pragma unroll 8
  for (int s = tid; s < p.n_seqs; s += kPlanThreads) bad |= p.row_start[s] > p.row_start[s + 1];
  bad = __syncthreads_or(bad);  // (the same in every CTA)
  if (all == 0) *p.head = PlanHead{0, bad ? 1 : 0, 0};
  if (bad) return;
  // The groups' first sequences, rows and row tiles: in shared memory, if they fit, because every sequence looks for
  // its group.
  const bool few = p.n_groups <= kPlanGroups;
  const int32_t* groups = few ? sh_groups : p.group_start;
  const int* gtile = few ? sh_tile : p.gtile;
  auto first_row = [&](int g) { return few ? sh_first[g] : p.row_start[p.group_start[g]]; };
  // row tiles of the groups (every CTA sums them up for itself, the first one writes them)
  int tiles = 0;
  for (int g0 = 0; g0 < p.n_groups; g0 += kPlanThreads) {
    const int g = g0 + tid;
    int n = 0;
    if (g < p.n_groups) {
      const int s = p.group_start[g], a = p.row_start[s];
      const long long rows = (long long)(p.row_start[p.group_start[g + 1]] - a) * p.hr;
      n = (int)((rows + kUnitRows - 1) / kUnitRows);
      if (few) {
        sh_groups[g] = s;
        sh_first[g] = a;
      }
    }
    const int incl = block_scan(n, sh_i);
    if (g < p.n_groups) {
      if (few) sh_tile[g] = tiles + incl - n;
      if (blockIdx.x == 0) p.gtile[g] = tiles + incl - n;
    }
    __syncthreads();
    tiles += sh_i[31];
    __syncthreads();
  }
  if (all == 0) p.gtile[p.n_groups] = tiles;
  for (int i = all; i < tiles; i += kAll) p.cost[i] = 0;
  // The sequence of a row: where it would be if all had as many rows, or the next one, or else searched for.
  const float per_row = (float)p.n_seqs / (float)p.n_rows;
  auto seq_of = [&](int t) {
    const int s = min(p.n_seqs - 1, (int)((float)t * per_row));
    const int a = p.row_start[s], b = p.row_start[s + 1], c = p.row_start[min(s + 2, p.n_seqs)];
    return a <= t && t < b ? s : b <= t && t < c ? s + 1 : find_last(p.row_start, p.n_seqs, t);
  };
  plan_barrier();
  // slots of own keys: a sequence's first row tile by the sequence, its further ones by the tile
  auto slots = [&](int s, int a, int n, int first, int i) {  // sequence s (its n rows from a on, the group's from first on) in tile i
    const int len = p.seq_len[s];
    const int j = min(n - 1, (int)(((uint32_t)(i + 1) * kUnitRows - 1) / (uint32_t)p.hr) - (a - first));  // (rows * hr < 2^31)
    return len_ok(p, len) ? (seen_rows(len, n, j) + kSlot - 1) / kSlot : 0;
  };
  for (int s = all; s < p.n_seqs; s += kAll) {
    const int a = p.row_start[s], n = p.row_start[s + 1] - a;
    if (n == 0) continue;
    const int g = find_last(groups, p.n_groups, s), first = first_row(g);
    const int i = (int)((long long)(a - first) * p.hr / kUnitRows);
    const int c = slots(s, a, n, first, i);
    if (c) atomicAdd(p.cost + gtile[g] + i, c);
  }
  for (int rt = all; rt < tiles; rt += kAll) {
    const int g = find_last(gtile, p.n_groups, rt), i = rt - gtile[g];
    if (i == 0) continue;
    const int first = first_row(g), t = first + (int)((uint32_t)i * kUnitRows / (uint32_t)p.hr);
    const int s = seq_of(t), a = p.row_start[s];
    if ((long long)(a - first) * p.hr / kUnitRows < i) {
      const int c = slots(s, a, p.row_start[s + 1] - a, first, i);
      if (c) atomicAdd(p.cost + rt, c);
    }
  }
  plan_barrier();
  if (blockIdx.x != 0) {
    // what the rows see, while the first CTA sums up
    for (int t = all - kPlanThreads; t < p.n_rows; t += kAll - kPlanThreads) {
      const int s = seq_of(t), a = p.row_start[s], len = p.seq_len[s];
      const int g = find_last(groups, p.n_groups, s);
      const bool fine = len_ok(p, len) && prefix_ok(p, p.prefix_len[g]);
      p.tok[t] = make_int2(s, fine ? seen_rows(len, p.row_start[s + 1] - a, t - a) : -1);
    }
    return;
  }
  // key tiles of the row tiles, and those before them
  long long run = 0;
  for (int r0 = 0; r0 < tiles; r0 += kPlanThreads) {
    const int rt = r0 + tid;
    long long c = 0;
    if (rt < tiles) {
      const int g = find_last(gtile, p.n_groups, rt), n = p.prefix_len[g];
      const int own = *reinterpret_cast<volatile int*>(p.cost + rt);  // (summed in L2)
      c = ((prefix_ok(p, n) ? n : 0) + kTileKeys - 1) / kTileKeys + (own + kSlots - 1) / kSlots;
      c = c < 1 ? 1 : c;
      p.cost[rt] = (int)c;
    }
    const long long incl = block_scan(c, sh);
    if (rt < tiles) p.before[rt] = run + incl - c;
    __syncthreads();
    run += sh[31];
    __syncthreads();
  }
  if (tid == 0) p.before[tiles] = run;
  __syncthreads();
  for (int g = tid; g <= p.n_groups; g += kPlanThreads) p.gcost[g] = p.before[p.gtile[g]] * p.hkv;
}

// ---------------------------------------------------------------------------
// attend
// ---------------------------------------------------------------------------
// What the schedule tells the others about a key tile
struct alignas(16) TileDesc {
  int flags, slots, bad, piece, pad[4];
  int owner[kSlots];  // sequence, or -1: the prefix
  int base[kSlots];   // the slot's first key
  int count[kSlots];  // its valid keys
  int row[kSlots];    // the first one's row of the pages
};
enum : int { TD_FIRST = 1, TD_LAST = 2, TD_FULL = 4, TD_END = 8, TD_SCAN = 16 };
struct UnitInfo {
  int t0, r0, rows, head;  // first token of the group, first row and rows of the unit, its key head
};
struct RowInfo {
  int seq, seen, out, pad;  // sequence (-5: no row), own keys seen (-1: spoiled), row of the output
};

// Sequences with values that are no numbers, of one of the last kUnitsAhead units
struct Dirty {
  int n, seq[kDirty];  // n > kDirty: any of them
};

// Tensor maps of the pages, a page a box
struct PageMaps {
  CUtensorMap k, v;
};

template <int D>
struct PrefixCfg {
  static constexpr int kThreads = 256;
  static constexpr uint32_t kRow = D >= 64 ? 128 : 64;  // bytes of a swizzled row
  static constexpr int NH = D == 128 ? 2 : 1;           // column halves of a tile
  static constexpr uint32_t kHalf = 128 * kRow, kTile = NH * kHalf;
  // tiles of queries, keys and values in shared memory
  static constexpr int NQ = D == 128 ? 1 : 2, NK = D == 128 ? 1 : D == 64 ? 2 : 4, NV = NK;
  static constexpr uint32_t kSwz = D >= 64 ? 2u : 4u;  // descriptor swizzle code (128 B / 64 B)
  // TMEM columns: S, P (its own columns where they fit), O
  static constexpr bool kOwnP = D <= 64;
  static constexpr uint32_t kCols = 256, kP = kOwnP ? 128 : 0, kO = kOwnP ? 192 : 128;
  static_assert(kO + D <= kCols, "TMEM budget");
  static constexpr int ND = 6;  // tile descriptors in flight
  // Weights of a tile that all rows see, so many keys at a time: short code goes faster as long as the next product
  // does not wait for P's columns (D = 128: 424 us a long reading by 32, 447 by 16; others 1 % the other way).
  static constexpr int kStep = kOwnP ? 16 : 32;
  static constexpr int kBars = 3 * NV + 2 * NK + 2 * ND + 2 * NQ + 3 + kUnitsAhead + 1;
  static constexpr size_t kFixed = sizeof(TileDesc) * ND + sizeof(UnitInfo) * kUnitsAhead + sizeof(RowInfo) * 128 * NQ +
                                   sizeof(Dirty) * kUnitsAhead + 8 * kBars + 16;
  static_assert(ND < kUnitsAhead, "a unit's entries are read before they are used again");
  static constexpr size_t kSmem = 1024 + (size_t)(NQ + NK + NV) * kTile + kFixed;
  static_assert(kSmem <= 115000, "two CTAs an SM");
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

__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void cp_async8(uint32_t dst, const void* src) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 8;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void cp_async_wait() { asm volatile("cp.async.wait_all;" ::: "memory"); }
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_async_wait_group() {
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}
// 16 bytes, or 16 zeros
__device__ __forceinline__ void cp_async16_or_zero(uint32_t dst, const void* src, bool on) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(on ? 16 : 0) : "memory");
}
__device__ __forceinline__ bool there(uint64_t* bar, uint32_t par) {  // for the whole warp
  return __all_sync(0xffffffffu, mbar_test_wait(bar, par)) != 0;
}

// A whole tile: eight full slots of a prefix, whose pages follow one another in the tile: a box a page and half.
template <int D>
__device__ __forceinline__ void load_pages(uint8_t* dst, const CUtensorMap* map, uint64_t* bar, int row, int lane0, int page_rows,
                                           uint32_t go) {
  using C = PrefixCfg<D>;
  mbar_arrive_expect_tx_if(bar, C::kTile, go);
#pragma unroll 1
  for (int i = 0; i < kSlots; i += page_rows / kSlot) {
    const int r = __shfl_sync(0xffffffffu, row, lane0 + i);
#pragma unroll
    for (int hf = 0; hf < C::NH; ++hf)
      tma_load_2d_if(dst + hf * C::kHalf + i * kSlot * C::kRow, map, 64 * hf, r, bar, go);
  }
}
// Any other tile: slot by slot, its valid rows alone, the others zeros (ZERO) or left as they are.  Boxes cost about
// 100 cycles each to issue whatever their size (16 of them 1900 of a tile's cycles); this takes a few hundred, and
// reads no row that is not used.
template <int D, bool ZERO>
__device__ __forceinline__ void load_slots(uint8_t* dst, const void* pages, int slots, int row, int count, int lane0) {
  using C = PrefixCfg<D>;
  constexpr int NP = D / 8, RP = 32 / NP;  // pieces of a row, rows of a step
  const int lane = threadIdx.x & 31, r0 = lane / NP, pc = lane % NP;
  const uint32_t at = smem_u32(dst) + (uint32_t)(pc * 16) / C::kRow * C::kHalf + (uint32_t)r0 * C::kRow;
  const uint32_t poff = (uint32_t)(pc * 16) % C::kRow;
  const char* src = static_cast<const char*>(pages) + (r0 * D + pc * 8) * 2;
#pragma unroll 1
  for (int s = 0; s < slots; ++s) {
    const int r = __shfl_sync(0xffffffffu, row, lane0 + s), n = __shfl_sync(0xffffffffu, count, lane0 + s);
    const char* from = src + (long long)r * (D * 2);
#pragma unroll
    for (int i = 0; i < kSlot; i += RP) {
      const uint32_t in = (uint32_t)(r0 + i);  // row of the slot (a slot begins a swizzle pattern)
      const uint32_t mask = C::kRow == 128 ? (in & 7u) : ((in >> 1) & 3u);
      const uint32_t to = at + (uint32_t)(s * kSlot + i) * C::kRow + (poff ^ (mask << 4));
      if (ZERO)
        cp_async16_or_zero(to, from + (r0 + i < n ? i * D * 2 : -(r0 * D * 2)), r0 + i < n);
      else if (r0 + i < n)
        cp_async16(to, from + i * D * 2);
    }
  }
}
__device__ __forceinline__ void mbar_arrive_lane0(uint64_t* bar) {
  __syncwarp();
  mbar_arrive_if_at(smem_u32(bar), (threadIdx.x & 31) == 0);
}

// A ring position: stage and the parity of its phase
template <int N>
struct Ring {
  int i = 0;
  uint32_t par = 0;
  __device__ __forceinline__ void next() {
    if (++i == N) {
      i = 0;
      par ^= 1u;
    }
  }
};

// maximum of N values, in four chains
template <int N>
__device__ __forceinline__ float maxn(const float* v) {
  float a[4] = {v[0], v[1], v[2], v[3]};
#pragma unroll
  for (int i = 4; i + 8 <= N; i += 8) {
#pragma unroll
    for (int k = 0; k < 4; ++k)
      asm("max.f32 %0, %1, %2, %3;" : "=f"(a[k]) : "f"(a[k]), "f"(v[i + 2 * k]), "f"(v[i + 2 * k + 1]));
  }
  a[0] = fmaxf(fmaxf(a[0], v[N - 4]), v[N - 3]);
  a[1] = fmaxf(fmaxf(a[1], v[N - 2]), v[N - 1]);
  return fmaxf(fmaxf(a[0], a[1]), fmaxf(a[2], a[3]));
}

template <typename T, int D>
__global__ void __launch_bounds__(PrefixCfg<D>::kThreads, 2)
    prefix_attend_kernel(const __grid_constant__ PageMaps maps, const PrefixParams p) {
  using C = PrefixCfg<D>;
  constexpr int NQ = C::NQ, NK = C::NK, NV = C::NV, ND = C::ND;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
  uint8_t* sQ = smem;                   // [NQ]
  uint8_t* sK = sQ + NQ * C::kTile;     // [NK]
  uint8_t* sV = sK + NK * C::kTile;     // [NV]
  TileDesc* descs = reinterpret_cast<TileDesc*>(sV + NV * C::kTile);
  UnitInfo* units = reinterpret_cast<UnitInfo*>(descs + ND);       // [kUnitsAhead]
  RowInfo* rinfo = reinterpret_cast<RowInfo*>(units + kUnitsAhead);  // [NQ][128]
  Dirty* dirty = reinterpret_cast<Dirty*>(rinfo + 128 * NQ);       // [kUnitsAhead]
  uint64_t* bars = reinterpret_cast<uint64_t*>(dirty + kUnitsAhead);
  uint64_t *k_full = bars, *k_empty = k_full + NK;
  uint64_t *v_full = k_empty + NK, *v_ready = v_full + NV, *v_empty = v_ready + NV;
  uint64_t *d_full = v_empty + NV, *d_empty = d_full + ND, *q_full = d_empty + ND, *q_free = q_full + NQ;
  uint64_t *s_full = q_free + NQ, *p_full = s_full + 1, *pv_done = s_full + 2;
  uint64_t *cleaned = s_full + 3, *drain = cleaned + kUnitsAhead;  // [kUnitsAhead] a unit's values have been looked through
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + C::kBars);

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    for (int i = 0; i < C::kBars; ++i) mbar_init(bars + i, 1);
    for (int i = 0; i < ND; ++i) mbar_init(d_empty + i, 7);  // all warps but the schedule's
    for (int i = 0; i < NQ; ++i) mbar_init(q_free + i, 4);
    mbar_init(p_full, 4);
    fence_mbar_init();
    prefetch_tmap(&maps.k);
    prefetch_tmap(&maps.v);
  }
  if (warp == 1) tmem_alloc(tmem_slot, C::kCols);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  pdl_trigger();
  pdl_wait();
  int* status = &p.head->status;

  if (warp < 4) {
    if (warp == 0) {
      // ---------------- schedule ----------------
      const int cta = blockIdx.x;
      const bool bad_plan = p.head->bad != 0;
      const long long total = bad_plan ? 0 : p.gcost[p.n_groups];
      // (no more CTAs than tiles: each of them has one at least)
      const int ctas = (int)min((long long)p.ctas, total);
      const long long each = ctas > 0 ? total / ctas : 0;
      const int more = (int)(total - each * ctas);  // CTAs with one tile more
      auto begin = [&](int c) { return each * c + min(c, more); };
      const long long hi = cta < ctas ? begin(cta + 1) : 0;
      long long x = cta < ctas ? begin(cta) : 0;
      Ring<ND> dr;
      bool ok = true;
      if (lane < 2) p.recs[2 * cta + lane].count = 0;
      __syncwarp();
      uint32_t unit = 0;
      // the unit that holds tile x: group, head, row tile; the next ones follow step by step
      int g = 0, head = 0, ti = 0, off = 0, first_rt = 0, n_rt = 0, s0 = 0, s1 = 0, t0 = 0, group_rows = 0, plen = 0;
      auto open_group = [&]() {
        first_rt = p.gtile[g];
        n_rt = p.gtile[g + 1] - first_rt;
        s0 = p.group_start[g];
        s1 = p.group_start[g + 1];
        plen = prefix_ok(p, p.prefix_len[g]) ? p.prefix_len[g] : 0;
        t0 = p.row_start[s0];
        group_rows = (int)min(0x7fffffffLL, (long long)(p.row_start[s1] - t0) * p.hr);
      };
      if (x < hi) {
        // (groups without rows have no tiles: the last of equal starts is the one with some)
        g = find_last(p.gcost, p.n_groups + 1, x);
        open_group();
        const long long per_head = p.before[first_rt + n_rt] - p.before[first_rt];
        long long y = x - p.gcost[g];
        while (y >= per_head) y -= per_head, ++head;
        y += p.before[first_rt];
        ti = find_last(p.before + first_rt, n_rt, y);
        off = (int)(y - p.before[first_rt + ti]);
      }
      while (ok && x < hi) {
        const int cost = p.cost[first_rt + ti];
        const int n = (int)min((long long)(cost - off), hi - x);
        const int r0 = ti * kUnitRows, rows = min(kUnitRows, group_rows - r0);
        const int piece = off == 0 && n == cost ? -1 : off == 0 ? 1 : 0;
        if (piece >= 0) {
          if (lane == 0) p.recs[2 * cta + piece] = SplitRec{0, cost, t0, r0, rows, head, x - off};
        }
        // (each reader of a unit's entry reads it before it passes on the unit's first tile)
        const UnitInfo info = {t0, r0, rows, head};
        const int ptiles = (plen + kTileKeys - 1) / kTileKeys;
        // own keys: the sequences of the unit's rows, 32 at a time, with their first slots
        const int ta = t0 + r0 / p.hr, tb = t0 + (r0 + rows - 1) / p.hr;
        int cs = 0, c_seen = 0, c_start = 0, c_end = 0;  // chunk's first sequence; lane's keys, first slot; the chunk's end
        bool own_open = false;
        auto chunk = [&](int from, int start) {
          cs = from;
          const int s = from + lane;
          int slots = 0;
          c_seen = 0;
          if (s < s1) {
            const int a = p.row_start[s], m = p.row_start[s + 1] - a, len = p.seq_len[s];
            if (m > 0 && a <= tb && a + m > ta && len_ok(p, len)) c_seen = seen_rows(len, m, min(m - 1, tb - a));
          }
          slots = (c_seen + kSlot - 1) / kSlot;
          int incl = slots;
#pragma unroll
          for (int o = 1; o < 32; o <<= 1) {
            const int u = __shfl_up_sync(0xffffffffu, incl, o);
            if (lane >= o) incl += u;
          }
          c_start = start + incl - slots;
          c_end = start + __shfl_sync(0xffffffffu, incl, 31);
        };
        // a batch of 32 slots (four tiles) of one part; this lane's slot
        int b_first = -1, b_part = -1;  // first tile of the batch, its part
        int b_owner = 0, b_base = 0, b_count = 0, b_row = 0, b_bad = 0;
        int ahead = -1, ahead_page = 0;  // the prefix batch whose pages have been asked for, this lane's page
        const int32_t* pre_table = p.prefix_pages + (long long)g * p.prefix_cols;
        auto batch = [&](int tile, int part) {
          b_first = tile;
          b_part = part;
          b_owner = -2;
          b_base = b_count = b_row = b_bad = 0;
          int page = -1;
          if (part == 0) {
            const int k = (tile * kSlots + lane) * kSlot;
            if (k < plen) {
              b_owner = -1;
              b_base = k;
              b_count = min(kSlot, plen - k);
              page = ahead == tile ? ahead_page : __ldg(pre_table + (k >> p.page_shift));
            }
            // (nothing is done with the next batch's page before its turn)
            const int next = k + 32 * kSlot;
            ahead = tile + 4;
            if (next < plen) ahead_page = __ldg(pre_table + (next >> p.page_shift));
          } else {
            const int slot = (tile - ptiles) * kSlots + lane;
            int from = -1;  // the chunk to be opened
            if (!own_open) {
              own_open = true;
              from = s0 + warp_find_row(p.row_start + s0, s1 - s0, ta);
              c_end = 0;
            }
            while (true) {
              if (from >= 0) chunk(from, c_end);
              // the chunk's sequence with the last first slot at or before this lane's (empty ones lie before it)
              int at = 0;
#pragma unroll
              for (int o = 16; o > 0; o >>= 1) {
                const int st = __shfl_sync(0xffffffffu, c_start, min(at + o, 31));
                if (at + o < 32 && st <= slot) at += o;
              }
              const int st = __shfl_sync(0xffffffffu, c_start, at), seen = __shfl_sync(0xffffffffu, c_seen, at);
              if (b_owner == -2 && slot < c_end && slot >= st && (slot - st) * kSlot < seen) {
                b_owner = cs + at;
                b_base = (slot - st) * kSlot;
                b_count = min(kSlot, seen - b_base);
                page = __ldg(p.pages + (long long)b_owner * p.page_cols + (b_base >> p.page_shift));
              }
              // past the chunk's end: the next one, as long as its sequences have rows here
              if (!__any_sync(0xffffffffu, b_owner == -2 && slot >= c_end) || cs + 32 >= s1 || p.row_start[cs + 32] > tb) break;
              from = cs + 32;
            }
          }
          if (b_owner != -2) {
            if (page < 0 || page >= p.n_pages) {
              b_bad = 1;
              page = 0;
            }
            b_row = ((page * p.hkv + head) << p.page_shift) + (b_base & (p.page_rows - 1));
          }
        };
#pragma unroll 1
        for (int j = off; j < off + n; ++j, ++x) {
          const int part = j >= ptiles;
          if (b_part != part || j >= b_first + 4) batch(j, part);
          const int l0 = (j - b_first) * kSlots;  // the tile's first lane
          const bool mine = lane >= l0 && lane < l0 + kSlots;
          // (a tile of the prefix ends with it, whatever the batch goes on with)
          const uint32_t used = __ballot_sync(0xffffffffu, mine && b_owner != -2);
          const uint32_t badm = __ballot_sync(0xffffffffu, mine && b_bad), part_m = __ballot_sync(0xffffffffu, mine && b_owner != -2 && b_count < kSlot);
          const int slots = __popc(used);
          const bool whole = part == 0 && slots == kSlots && part_m == 0 && badm == 0;
          if (!(ok = mbar_wait_ok(d_empty + dr.i, dr.par ^ 1u, status))) break;
          TileDesc* td = descs + dr.i;
          if (mine) {
            td->owner[lane - l0] = b_owner;
            td->base[lane - l0] = b_base;
            td->count[lane - l0] = b_count;
            td->row[lane - l0] = b_row;
          }
          if (lane == 0) {
            if (j == off) units[unit % kUnitsAhead] = info;
            td->flags = (j == off ? TD_FIRST : 0) | (j == off + n - 1 ? TD_LAST : 0) |
                        (whole ? TD_FULL : 0) |
                        (part == 1 && ta != tb ? TD_SCAN : 0);
            td->slots = slots;
            td->bad = (int)(badm >> l0);
            td->piece = piece;
          }
          mbar_arrive_lane0(d_full + dr.i);
          dr.next();
        }
        ++unit;
        // the next unit: row tile, head, group with rows
        off = 0;
        if (x < hi && ++ti == n_rt) {
          ti = 0;
          if (++head == p.hkv) {
            head = 0;
            do {
              ++g;
            } while (p.gtile[g + 1] == p.gtile[g]);
            open_group();
          }
        }
      }
      if (ok && mbar_wait_ok(d_empty + dr.i, dr.par ^ 1u, status)) {
        if (lane == 0) descs[dr.i].flags = TD_END;
        mbar_arrive_lane0(d_full + dr.i);
      }
      // (the equal runs are worked out once more: held until here they would cost the loop registers)
      __syncwarp();
      SplitRec* rec = p.recs + 2 * cta + (lane & 1);
      if (lane < 2 && rec->count > 0) {
        const long long all = p.gcost[p.n_groups], n = min((long long)p.ctas, all), low = all / n, large = all - low * n;
        auto cta_of = [&](long long tile) {  // that has the tile
          const long long in_large = (low + 1) * large;
          return (int)(tile < in_large ? tile / (low + 1) : large + (tile - in_large) / low);
        };
        const int first = cta_of(rec->tile);
        rec->count = cta_of(rec->tile + rec->count - 1) - first + 1;
        rec->first = first;
      }
    } else if (warp == 1) {
      // ---------------- products ----------------
      const uint32_t go = elect_one();
      constexpr uint32_t kType = std::is_same<T, __nv_bfloat16>::value ? (1u << 7) | (1u << 10) : 0u;
      const uint32_t idesc = (1u << 4) | kType | (8u << 24);
      const uint32_t idesc_pv = idesc | (1u << 16) | ((uint32_t)(D >> 3) << 17);  // V is MN-major
      const uint64_t qd0 = tile_desc(smem_u32(sQ), 16, 8 * C::kRow, C::kSwz);
      const uint64_t kd0 = tile_desc(smem_u32(sK), 16, 8 * C::kRow, C::kSwz);
      const uint64_t vd0 = tile_desc(smem_u32(sV), C::kHalf, 8 * C::kRow, C::kSwz);
      const uint32_t t_p = tmem + C::kP, t_o = tmem + C::kO;
      Ring<NK> kr;
      Ring<NV> pr;  // of the next product with V
      Ring<ND> dr;
      Ring<NQ> qr;
      uint32_t done = 0;             // products with V
      bool begun = false;            // the last job's product with V is still to come
      int p_slots = 0, p_first = 0;  // its slots, and whether it opens a unit's output
      // The tile in hand: what is waited for next, its description (0), its unit's queries (1), its keys (2), or
      // nothing any more (3).
      int need = 0, flags = 0, slots = 0, first = 0;
      int n_slots = 0, n_first = 0;  // of a job whose scores have been issued before the last one's product
#pragma unroll 1
      while (true) {
        uint64_t* bar = need == 0 ? d_full + dr.i : need == 1 ? q_full + qr.i : k_full + kr.i;
        const uint32_t par = need == 0 ? dr.par : need == 1 ? qr.par : kr.par;
        // O += P V: before the next scores where they, or P, lie in the same columns, after them elsewhere, and
        // before waiting for what may only come after it (a tile's or the queries' space)
        if (begun && (n_slots || need == 3 || (!C::kOwnP && need == 2) || !there(bar, par))) {
          if (!mbar_wait_ok(p_full, done & 1u, status) || !mbar_wait_ok(v_ready + pr.i, pr.par, status)) break;
          tc_fence_after();
          const uint64_t vd = vd0 + (uint64_t)((pr.i * C::kTile) >> 4);
          umma_bf16_tmem_a_if(t_o, t_p, vd, idesc_pv, p_first ? 0u : 1u, go);
          if (D == 128 && p_slots == kSlots) {
#pragma unroll
            for (int s = 1; s < kSlots; ++s)
              umma_bf16_tmem_a_if(t_o, t_p + (uint32_t)(8 * s), vd + (uint64_t)((s * kSlot * C::kRow) >> 4), idesc_pv, 1u, go);
          } else {
#pragma unroll 1
            for (int s = 1; s < p_slots; ++s)
              umma_bf16_tmem_a_if(t_o, t_p + (uint32_t)(8 * s), vd + (uint64_t)((s * kSlot * C::kRow) >> 4), idesc_pv, 1u, go);
          }
          umma_commit_if(pv_done, go);
          umma_commit_if(v_empty + pr.i, go);
          pr.next();
          ++done;
          begun = n_slots != 0;
          p_slots = n_slots;
          p_first = n_first;
          n_slots = 0;
          continue;
        }
        if (need == 3) break;
        if (!mbar_wait_ok(bar, par, status)) break;
        if (need == 0) {
          const TileDesc* td = descs + dr.i;
          flags = td->flags;
          slots = td->slots;
          if (flags & TD_END) {
            need = 3;
            continue;
          }
          mbar_arrive_lane0(d_empty + dr.i);
          dr.next();
          if (flags & TD_FIRST)
            need = 1;
          else if (slots)
            need = 2;
        } else if (need == 1) {
          qr.next();
          first = 1;
          need = slots ? 2 : 0;
        } else {
          // (S is free when its weights are there; without columns of its own, P lies there until its product is done)
          if (begun && !mbar_wait_ok(p_full, done & 1u, status)) break;
          if (!C::kOwnP && done > 0 && !mbar_wait_ok(pv_done, (done - 1) & 1u, status)) break;
          tc_fence_after();
          const int qi = qr.i == 0 ? NQ - 1 : qr.i - 1;
          const uint64_t qd = qd0 + (uint64_t)((qi * C::kTile) >> 4), kd = kd0 + (uint64_t)((kr.i * C::kTile) >> 4);
          const uint32_t id = idesc | ((uint32_t)(slots * 2) << 17);
#pragma unroll (D == 128 ? 8 : 1)
          for (int kk = 0; kk < D / 16; ++kk) {
            const uint64_t at = (uint64_t)(((kk * 32) / C::kRow * C::kHalf + (kk * 32) % C::kRow) >> 4);
            umma_bf16_if(tmem, qd + at, kd + at, id, kk != 0 ? 1u : 0u, go);
          }
          umma_commit_if(s_full, go);
          umma_commit_if(k_empty + kr.i, go);
          kr.next();
          if (begun) {
            n_slots = slots;
            n_first = first;
          } else {
            begun = true;
            p_slots = slots;
            p_first = first;
          }
          first = 0;
          need = 0;
        }
      }
      umma_drain(drain, status, go);
    } else if (warp == 2) {
      // ---------------- values ----------------
      // A tile is loaded, and the one before it then made ready (or at once, while the next has to wait).
      const uint32_t go = elect_one();
      Ring<NV> vr;
      Ring<ND> dr;
      uint32_t unit = 0, full = 0;  // unit: of the tile to be made ready; parities of the stages' box loads
      struct Tile {
        int flags, slots, stage, owner, row, count;  // (owner, row and count: of this lane's slot)
      };
      Tile next = {}, last = {};
      bool have = false, pending = false, issued = false, end = false, ok = true;
#pragma unroll 1
      while (true) {
        issued = false;
        if (!have && !end && (!pending || there(d_full + dr.i, dr.par))) {
          if (!(ok = mbar_wait_ok(d_full + dr.i, dr.par, status))) break;
          const TileDesc* td = descs + dr.i;
          next.flags = td->flags;
          next.slots = td->slots;
          next.owner = td->owner[lane & (kSlots - 1)];
          next.row = td->row[lane & (kSlots - 1)];
          next.count = td->count[lane & (kSlots - 1)];
          if (next.flags & TD_END) {
            end = true;
          } else {
            mbar_arrive_lane0(d_empty + dr.i);
            dr.next();
            have = true;
          }
        }
        if (have && (!pending || next.slots == 0 || there(v_empty + vr.i, vr.par ^ 1u))) {
          next.stage = vr.i;
          if (next.slots > 0) {
            if (!(ok = mbar_wait_ok(v_empty + vr.i, vr.par ^ 1u, status))) break;
            uint8_t* v = sV + vr.i * C::kTile;
            if (next.flags & TD_FULL)
              load_pages<D>(v, &maps.v, v_full + vr.i, next.row, 0, p.page_rows, go);
            else
              load_slots<D, true>(v, p.v, next.slots, next.row, next.count, 0);
            vr.next();
          }
          cp_async_commit();
          have = false;
          issued = true;
        }
        if (pending) {
          const uint32_t bit = 1u << last.stage;
          Dirty* dt = dirty + unit % kUnitsAhead;
          if ((last.flags & TD_FIRST) && lane == 0) dt->n = 0;
          if (last.flags & TD_FULL) {
            if (!(ok = mbar_wait_ok(v_full + last.stage, (full & bit) ? 1u : 0u, status))) break;
            full ^= bit;
          } else if (issued) {
            cp_async_wait_group<1>();
          } else {
            cp_async_wait_group<0>();
          }
          if (last.flags & TD_SCAN) {
            __syncwarp();
            uint8_t* v = sV + last.stage * C::kTile;
            // 0 x summed: 0 as long as every x is a number
            uint32_t acc[4] = {0u, 0u, 0u, 0u};
#pragma unroll 1
            for (int sl = 0; sl < last.slots; ++sl)
#pragma unroll
              for (int o = 0; o < (int)(C::NH * kSlot * C::kRow); o += 512) {
                const uint4 y = *reinterpret_cast<const uint4*>(v + o / (int)(kSlot * C::kRow) * C::kHalf + sl * kSlot * C::kRow +
                                                                o % (int)(kSlot * C::kRow) + lane * 16);
                acc[0] = Elem<T>::zero_fma(y.x, acc[0]);
                acc[1] = Elem<T>::zero_fma(y.y, acc[1]);
                acc[2] = Elem<T>::zero_fma(y.z, acc[2]);
                acc[3] = Elem<T>::zero_fma(y.w, acc[3]);
              }
            if (__any_sync(0xffffffffu, ((acc[0] | acc[1] | acc[2] | acc[3]) & 0x7fff7fffu) != 0)) {
#pragma unroll 1
              for (int s = 0; s < last.slots; ++s) {
                bool found = false;
#pragma unroll 1
                for (int hf = 0; hf < C::NH; ++hf)
#pragma unroll 1
                  for (uint32_t o = lane * 2; o < kSlot * C::kRow; o += 64) {
                    T* x = reinterpret_cast<T*>(v + hf * C::kHalf + s * kSlot * C::kRow + o);
                    const float f = Elem<T>::get(*x) * 0.f;
                    if (!(f == 0.f)) {
                      found = true;
                      *x = Elem<T>::put(0.f);
                    }
                  }
                found = __any_sync(0xffffffffu, found);
                const int who = __shfl_sync(0xffffffffu, last.owner, s);
                if (found && lane == 0) {
                  const int n = dt->n;
                  if (n == 0 || n > kDirty || dt->seq[n - 1] != who) {
                    if (n < kDirty) dt->seq[n] = who;
                    dt->n = n + 1;
                  }
                }
              }
            }
          }
          if (last.slots > 0) {
            fence_async_shared();
            mbar_arrive_lane0(v_ready + last.stage);
          }
          if (last.flags & TD_LAST) {
            mbar_arrive_lane0(cleaned + unit % kUnitsAhead);
            ++unit;
          }
          pending = false;
        }
        if (issued) {
          last = next;
          pending = true;
        }
        if (end && !pending) break;
      }
      // (after a timed-out wait, the loads still on their way)
      cp_async_wait();
      if (!ok && pending && (last.flags & TD_FULL)) mbar_landed(v_full + last.stage, (full >> last.stage) & 1u, status);
      if (!ok && issued && (next.flags & TD_FULL)) mbar_landed(v_full + next.stage, (full >> next.stage) & 1u, status);
    } else {
      // ---------------- queries and keys ----------------
      const uint32_t go = elect_one();
      Ring<NK> kr;
      Ring<ND> dr;
      Ring<NQ> qr;
      uint32_t unit = 0;
      // Slots on their way by cp.async, oldest first: their tiles are announced once they have landed, at the latest
      // before this warp waits for anything.
      int away = 0;
      uint64_t *away0 = nullptr, *away1 = nullptr;
      auto landed = [&](bool all) {
        if (all)
          cp_async_wait_group<0>();
        else
          cp_async_wait_group<2>();
        fence_async_shared();
        mbar_arrive_lane0(away0);
        if (all && away == 2) mbar_arrive_lane0(away1);
        away0 = away1;
        away = all ? 0 : away - 1;
      };
      auto wait = [&](uint64_t* bar, uint32_t par) {
        if (away && !there(bar, par)) landed(true);
        return mbar_wait_ok(bar, par, status);
      };
      while (true) {
        if (!wait(d_full + dr.i, dr.par)) break;
        const TileDesc* td = descs + dr.i;
        const int flags = td->flags, slots = td->slots, row = td->row[lane & (kSlots - 1)], count = td->count[lane & (kSlots - 1)];
        if (flags & TD_END) break;
        const UnitInfo u = units[unit % kUnitsAhead];
        mbar_arrive_lane0(d_empty + dr.i);
        dr.next();
        if (flags & TD_FIRST) {
          const int t_first = u.r0 / p.hr, h_first = u.r0 - t_first * p.hr;  // the unit's first row: token, query head
          auto at = [&](int r, int& t, int& h) {  // (a product instead of a division: exact below 2^16)
            const int q = (int)__umulhi((uint32_t)(h_first + r), (uint32_t)p.hr_inv);
            t = u.t0 + t_first + (p.hr == 1 ? r : q);
            h = u.head * p.hr + (p.hr == 1 ? 0 : h_first + r - q * p.hr);
          };
          if (!wait(q_free + qr.i, qr.par ^ 1u)) break;
          // the queries: pieces of 16 bytes, swizzled as TMA would have it
          constexpr int NP = D / 8, RP = 32 / NP;  // pieces of a row, rows of a step
          const int pc = lane % NP;
          const uint32_t to = smem_u32(sQ) + qr.i * C::kTile + (uint32_t)(pc * 16) / C::kRow * C::kHalf;
          const uint32_t poff = (uint32_t)(pc * 16) % C::kRow;
#pragma unroll (D == 128 ? 4 : 1)
          for (int r = lane / NP; r < u.rows; r += RP) {
            int t, h;
            at(r, t, h);
            const uint32_t mask = C::kRow == 128 ? ((uint32_t)r & 7u) : (((uint32_t)r >> 1) & 3u);
            cp_async16(to + (uint32_t)r * C::kRow + (poff ^ (mask << 4)),
                       reinterpret_cast<const T*>(p.q) + (long long)t * p.q_row + h * p.q_head + pc * 8);
          }
          RowInfo* info = rinfo + qr.i * 128;
#pragma unroll 1
          for (int r = lane; r < kUnitRows; r += 32) {
            if (r < u.rows) {
              int t, h;
              at(r, t, h);
              cp_async8(smem_u32(info + r), p.tok + t);
              info[r].out = t * p.hq + h;
            } else {
              info[r] = RowInfo{-5, 0, -1, 0};
            }
          }
          // (announced as a tile's slots are)
          cp_async_commit();
          if (away == 2) landed(false);
          (away ? away1 : away0) = q_full + qr.i;
          ++away;
          qr.next();
        }
        if (flags & TD_LAST) ++unit;
        if (slots == 0) continue;
        if (!wait(k_empty + kr.i, kr.par ^ 1u)) break;
        uint8_t* k = sK + kr.i * C::kTile;
        if (flags & TD_FULL) {
          load_pages<D>(k, &maps.k, k_full + kr.i, row, 0, p.page_rows, go);
          cp_async_commit();
        } else {
          load_slots<D, false>(k, p.k, slots, row, count, 0);
          cp_async_commit();
          if (away == 2) landed(false);
          (away ? away1 : away0) = k_full + kr.i;
          ++away;
        }
        kr.next();
      }
      if (away) landed(true);
      cp_async_wait();
      // the loads land before the shared memory goes away, whatever became of their readers
      mbar_landed_ring(k_full, kr.i, kr.par ^ 1u, NK, status);
    }
  } else {
    // ---------------- softmax and output ----------------
    const int row = threadIdx.x & 127;
    const uint32_t tl = tmem + ((uint32_t)((warp & 3) * 32) << 16), t_s = tl, t_p = tl + C::kP, t_o = tl + C::kO;
    const float sc = p.sc;
    Ring<ND> dr;
    Ring<NQ> qr;
    uint32_t jobs = 0, unit = 0;
    int mine = 0;  // jobs of this unit
    RowInfo ri = {-5, 0, -1, 0};
    float m = -INFINITY, l = 0.f;
    bool spoiled = false, active = false;
    while (true) {
      if (!mbar_wait_ok(d_full + dr.i, dr.par, status)) break;
      const TileDesc* td = descs + dr.i;
      const int flags = td->flags, slots = td->slots, piece = td->piece;
      if (flags & TD_END) break;
      if (flags & TD_FIRST) {
        if (!mbar_wait_ok(q_full + qr.i, qr.par, status)) break;
        ri = rinfo[qr.i * 128 + row];
        active = __any_sync(0xffffffffu, ri.seq >= 0);
        m = -INFINITY;
        l = 0.f;
        mine = 0;
        spoiled = ri.seen < 0;
      }
      if (slots > 0) {
        if (!mbar_wait_ok(s_full, jobs & 1u, status)) break;
        if (active) {
          tc_fence_after();
          // Scores are read twice, for the maximum and for P, and never held (code and registers: the roles'
          // instructions compete for the SM's instruction cache).  Tiles that every row sees whole go by halves,
          // others by pairs of slots, of which those that no row of the warp sees cost their zeros in P.
          const bool whole = flags & TD_FULL;
          float mx = -INFINITY;
          uint32_t pairs = 0, seen0 = 0, seen1 = 0;  // pairs with a key that a row of the warp sees; this row's keys of
                                                     // slots 0 .. 3 and 4 .. 7, a byte each
          bool single = false;
          int slot = -1;
          float one[kSlot];
          auto pair = [&](int z, float* v) {  // scores of slots 2 z and 2 z + 1, unseen ones -inf
            tmem_ld32(t_s + (uint32_t)(32 * z), v);
            const uint32_t two = (z < 2 ? seen0 : seen1) >> (16 * (z & 1));
            const uint32_t bits = ((1u << (two & 0xff)) - 1u) | ((1u << ((two >> 8) & 0xff)) - 1u) << kSlot;
#pragma unroll
            for (int i = 0; i < 2 * kSlot; ++i)
              if (!(bits & (1u << i))) v[i] = -INFINITY;
          };
          if (whole) {
#pragma unroll 1
            for (int c0 = 0; c0 < 128; c0 += 32) {
              float v[32];
              tmem_ld32(t_s + (uint32_t)c0, v);
              mx = fmaxf(mx, maxn<32>(v));
            }
          } else {
            // this row's keys of a slot: of the prefix all valid ones, of its own sequence those up to itself
            const int4 *own4 = reinterpret_cast<const int4*>(td->owner), *base4 = reinterpret_cast<const int4*>(td->base),
                       *count4 = reinterpret_cast<const int4*>(td->count);
            uint32_t mask = 0;
#pragma unroll 1
            for (int h = 0; h < 2; ++h) {
              const int4 ow = own4[h], ba = base4[h], co = count4[h];
              auto n_of = [&](int owner, int base, int count) {
                const int most = owner == -1 ? 1 << 30 : owner == ri.seq ? ri.seen : -(1 << 30);
                return (uint32_t)min(count, max(0, most - base));
              };
              const uint32_t n0 = n_of(ow.x, ba.x, co.x), n1 = n_of(ow.y, ba.y, co.y), n2 = n_of(ow.z, ba.z, co.z),
                             n3 = n_of(ow.w, ba.w, co.w);
              (h ? seen1 : seen0) = n0 | n1 << 8 | n2 << 16 | n3 << 24;
              mask |= ((n0 ? 1u : 0u) | (n1 ? 2u : 0u) | (n2 ? 4u : 0u) | (n3 ? 8u : 0u)) << (4 * h);
            }
            spoiled = spoiled || (mask & (uint32_t)td->bad);
            const uint32_t any = __reduce_or_sync(0xffffffffu, mask);
            pairs = (any & 3u ? 1u : 0u) | (any & 12u ? 2u : 0u) | (any & 48u ? 4u : 0u) | (any & 192u ? 8u : 0u);
            single = __all_sync(0xffffffffu, __popc(mask) <= 1);
            if (single) {
              // every row of the warp sees one slot at most (short sequences): 16 scores each, picked from the pairs
              slot = __ffs(mask) - 1;
              const uint32_t bits = slot < 0 ? 0u : (1u << (((slot < 4 ? seen0 : seen1) >> (8 * (slot & 3))) & 0xffu)) - 1u;
#pragma unroll
              for (int i = 0; i < kSlot; ++i) one[i] = -INFINITY;
#pragma unroll 1
              for (uint32_t left = any; left; left &= left - 1) {
                const int z = __ffs(left) - 1;
                float v[kSlot];
                tmem_ld16(t_s + (uint32_t)(kSlot * z), v);
                const uint32_t here = slot == z ? bits : 0u;
#pragma unroll
                for (int i = 0; i < kSlot; ++i)
                  if (here & (1u << i)) one[i] = v[i];
              }
              mx = maxn<kSlot>(one);
            } else {
#pragma unroll 1
            for (uint32_t left = pairs; left; left &= left - 1) {
              float v[32];
              pair(__ffs(left) - 1, v);
              mx = fmaxf(mx, maxn<32>(v));
            }
            }
          }
          // Weights are 2^(x - m) in the values' type, which the product wants of both its operands (the sum keeps them
          // in fp32): rounded once, by u of each.  m is kLift below the row's maximum and may lag kSlack more, which
          // makes weights of up to 2^15 in f16.  Its smallest numbers would otherwise drop weights below 2^-25 of
          // the largest, which thousands of keys may have; so it is 2^-32.  bf16 has fp32's range.
          constexpr float kSlack = 8.f, kLift = std::is_same<T, __half>::value ? 7.f : 0.f;
          mx = fmaf(mx, sc, -kLift);
          if (mine == 0) {
            m = mx;
          } else {
            const bool up = mx > m + kSlack;
            if (__any_sync(0xffffffffu, up)) {
              // the accumulator, complete up to the last job, to the new maximum
              if (!mbar_wait_ok(pv_done, (jobs - 1) & 1u, status)) break;
              tc_fence_after();
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
          if (C::kOwnP && jobs > 0) {  // P's columns are free once the last job's product has read them
            if (!mbar_wait_ok(pv_done, (jobs - 1) & 1u, status)) break;
            tc_fence_after();
          }
          const float ref = m == -INFINITY ? 0.f : m;
          const uint64_t sc2 = f32x2_pack(sc, sc), nm2 = f32x2_pack(-ref, -ref);
          uint64_t sum[2] = {0ull, 0ull};
          auto weights = [&](const float* x, auto count, uint32_t* pk) {  // P of some keys, in pairs
#pragma unroll
            for (int i = 0; i < decltype(count)::value; i += 4) {
              float e[4];
              f32x2_unpack(f32x2_fma(f32x2_pack(x[i], x[i + 1]), sc2, nm2), e[0], e[1]);
              f32x2_unpack(f32x2_fma(f32x2_pack(x[i + 2], x[i + 3]), sc2, nm2), e[2], e[3]);
#pragma unroll
              for (int z = 0; z < 4; ++z) e[z] = ex2_approx(e[z]);
              uint64_t& acc = sum[(i >> 2) & 1];
              acc = f32x2_add(acc, f32x2_add(f32x2_pack(e[0], e[2]), f32x2_pack(e[1], e[3])));
              pk[i / 2] = Elem<T>::put2(e[0], e[1]);
              pk[i / 2 + 1] = Elem<T>::put2(e[2], e[3]);
            }
          };
          const std::integral_constant<int, 32> c32{};
          if (whole) {
#pragma unroll 1
            for (int c0 = 0; c0 < 128; c0 += C::kStep) {
              float v[C::kStep];
              uint32_t pk[C::kStep / 2];
              if constexpr (C::kStep == 32) {
                tmem_ld32(t_s + (uint32_t)c0, v);
                weights(v, std::integral_constant<int, 32>(), pk);
                tmem_st16_nowait(t_p + (uint32_t)(c0 / 2), pk);
              } else {
                tmem_ld16(t_s + (uint32_t)c0, v);
                weights(v, std::integral_constant<int, 16>(), pk);
                tmem_st8_nowait(t_p + (uint32_t)(c0 / 2), pk);
              }
            }
          } else if (single) {
            uint32_t mine8[kSlot / 2];
            weights(one, std::integral_constant<int, kSlot>(), mine8);
#pragma unroll 1
            for (int z = 0; z < slots; ++z) {
              uint32_t pk[kSlot / 2];
#pragma unroll
              for (int i = 0; i < kSlot / 2; ++i) pk[i] = slot == z ? mine8[i] : 0u;
              tmem_st8_nowait(t_p + (uint32_t)(kSlot / 2 * z), pk);
            }
          } else {
#pragma unroll 1
            for (int z = 0; 2 * z < slots; ++z) {
              if ((pairs >> z) & 1) {
                float v[32];
                uint32_t pk[16];
                pair(z, v);
                weights(v, c32, pk);
                tmem_st16_nowait(t_p + (uint32_t)(16 * z), pk);
              } else {
                const uint32_t zero[16] = {};
                tmem_st16_nowait(t_p + (uint32_t)(16 * z), zero);
              }
            }
          }
          float a0, a1, a2, a3;
          f32x2_unpack(sum[0], a0, a1);
          f32x2_unpack(sum[1], a2, a3);
          l += (a0 + a1) + (a2 + a3);
          tmem_st_wait();
          tc_fence_before();
        }
        mbar_arrive_lane0(p_full);
        ++jobs;
        ++mine;
      }
      mbar_arrive_lane0(d_empty + dr.i);
      dr.next();
      if (!(flags & TD_LAST)) continue;

      // ---------------- the piece's output ----------------
      // (every S of the unit is complete: its queries may go)
      mbar_arrive_lane0(q_free + qr.i);
      qr.next();
      if (!mbar_wait_ok(cleaned + unit % kUnitsAhead, (unit / kUnitsAhead) & 1u, status)) break;
      {
        const Dirty dt = dirty[unit % kUnitsAhead];
        if (dt.n > 0) {
          spoiled = spoiled || dt.n > kDirty;
#pragma unroll
          for (int i = 0; i < kDirty; ++i) spoiled = spoiled || (i < dt.n && dt.seq[i] == ri.seq);
        }
        ++unit;
      }
      if (spoiled) l = NAN;
      const bool store = ri.out >= 0, direct = piece < 0;
      const float f = !direct ? 1.f : l == 0.f ? 0.f : 1.f / l;
      const long long slot = ((long long)blockIdx.x * 2 + (piece == 1)) * kUnitRows + row;
      T* out = reinterpret_cast<T*>(p.out) + (long long)ri.out * D;
      float* part = p.part_o + slot * D;
      if (mine > 0) {
        if (!mbar_wait_ok(pv_done, (jobs - 1) & 1u, status)) break;
        tc_fence_after();
      }
#pragma unroll 1
      for (int c0 = 0; c0 < D; c0 += 16) {
        float o[16];
        if (mine > 0) {
          tmem_ld16(t_o + (uint32_t)c0, o);
#pragma unroll
          for (int i = 0; i < 16; ++i) o[i] *= f;
        } else {
#pragma unroll
          for (int i = 0; i < 16; ++i) o[i] = 0.f;
        }
        if (store && direct) {
#pragma unroll
          for (int i = 0; i < 16; i += 2) o[i / 2] = __uint_as_float(Elem<T>::put2(o[i], o[i + 1]));
          // (a row a lane: whole 32-byte sectors, 12 % of a call with many rows against two halves)
          st_sector(reinterpret_cast<float*>(out + c0), o);
        } else if (store) {
#pragma unroll
          for (int i = 0; i < 16; i += 8) st_sector(part + c0 + i, o + i);
        }
      }
      tc_fence_before();
      if (store && direct) {
        if (!(l == l)) p.list[atomicAdd(&p.head->listed, 1)] = ri.out;
        if (p.lse) p.lse[ri.out] = l == 0.f ? -INFINITY : (m + log2f(l)) * 0.693147180559945309f;
      } else if (store) {
        p.part_ml[slot] = make_float2(m, l);
      }
    }
  }
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  if (warp == 1) tmem_dealloc(tmem, C::kCols);
}

// ---------------------------------------------------------------------------
// finish
// ---------------------------------------------------------------------------
// A row from its visible keys alone, 32 at a time, by one warp (sq: its D queries)
template <typename T, int D>
__device__ __noinline__ void row_by_keys(const PrefixParams& p, long long w, float* sq) {
  const int lane = threadIdx.x & 31;
  const int t = (int)(w / p.hq), h = (int)(w % p.hq), hk = h / (p.hq / p.hkv);
  const int s = warp_find_row(p.row_start, p.n_seqs, t), g = warp_find_row(p.group_start, p.n_groups, s);
  const int r0 = p.row_start[s], n = p.row_start[s + 1] - r0, len = p.seq_len[s], np = p.prefix_len[g];
  bool bad = t < r0 || t >= r0 + n || s < p.group_start[g] || s >= p.group_start[g + 1] || len < 0 || np < 0 ||
             (long long)len > (long long)p.page_cols * p.page_rows || (long long)np > (long long)p.prefix_cols * p.page_rows;
  const int own = bad ? 0 : max(0, min(len, len - n + (t - r0) + 1)), pre = bad ? 0 : np;
  __syncwarp();  // (an earlier row of this warp has been read)
  const T* q = reinterpret_cast<const T*>(p.q) + (long long)t * p.q_row + h * p.q_head;
  for (int i = lane; i < D; i += 32) sq[i] = Elem<T>::get(q[i]);
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
          for (int i = 0; i < D; ++i) a += sq[i] * Elem<T>::get(kr[i]);
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


template <typename T, int D>
__global__ void __launch_bounds__(256) prefix_finish_kernel(const PrefixParams p) {
  __shared__ float sq[8][D];
  pdl_trigger();
  pdl_wait();
  const int lane = threadIdx.x & 31, wp = threadIdx.x >> 5;
  const long long rows = (long long)p.n_rows * p.hq;
  const long long w0 = ((long long)blockIdx.y * gridDim.x + blockIdx.x) * 8 + wp, nw = (long long)gridDim.x * gridDim.y * 8;
  if (p.head->bad) {
    for (long long w = w0; w < rows; w += nw) {
      T* out = reinterpret_cast<T*>(p.out) + w * D;
      for (int i = lane; i < D; i += 32) out[i] = Elem<T>::put(NAN);
      if (p.lse && lane == 0) p.lse[w] = NAN;
    }
    if (w0 == 0 && lane == 0 && p.status) atomicOr(p.status, FE_ST_INDEX);
    return;
  }
  if (w0 == 0 && lane == 0 && p.status && p.head->status) atomicOr(p.status, p.head->status);
  // The CTAs that have the pieces of a unit join its rows, each its share: one long prefix is split over all of them
  // (two units of 98 pieces, joined by their first CTAs alone: 49 us the call, 32 this way).
  constexpr int N = D / 32;
  struct alignas(4 * N) Values {
    float v[N];
  };
  struct alignas(2 * N) Outputs {
    T v[N];
  };
  const SplitRec begins_in = p.recs[2 * blockIdx.x], ends_in = p.recs[2 * blockIdx.x + 1];
#pragma unroll 1
  for (int which = 0; which < 2; ++which) {
    const SplitRec rec = which ? ends_in : begins_in;
    if (rec.count == 0) continue;
    auto slot = [&](int i, int r) { return ((long long)(rec.first + i) * 2 + (i == 0)) * kUnitRows + r; };
    // (at most 128 rows, 2^16 CTAs; two pieces are the first one's)
    const uint32_t share = blockIdx.x - rec.first, shares = rec.count > 2 ? rec.count : 1;
    if (share >= shares) continue;
    const int r_begin = (int)(rec.rows * share / shares), r_end = (int)(rec.rows * (share + 1) / shares);
    auto values = [&](int i, int r) { return reinterpret_cast<const Values*>(p.part_o + slot(i, r) * D)[lane]; };
    auto put = [&](int r, float m, float l, float* o) {
      const int rr = rec.r0 + r;
      const long long w = (long long)(rec.t0 + rr / p.hr) * p.hq + rec.head * p.hr + rr % p.hr;
      if (!(l == l)) {
        row_by_keys<T, D>(p, w, sq[wp]);
        return;
      }
      const float inv = l == 0.f ? 0.f : 1.f / l;
      Outputs y;
#pragma unroll
      for (int z = 0; z < N; ++z) y.v[z] = Elem<T>::put(o[z] * inv);
      reinterpret_cast<Outputs*>(reinterpret_cast<T*>(p.out) + w * D)[lane] = y;
      if (p.lse && lane == 0) p.lse[w] = l == 0.f ? -INFINITY : (m + log2f(l)) * 0.693147180559945309f;
    };
#pragma unroll 1
    for (int r = r_begin + blockIdx.y * 8 + wp; r < r_end; r += gridDim.y * 8) {
      float o[N];
      if (rec.count == 2) {
        const Values x0 = values(0, r), x1 = values(1, r);
        const float2 a = p.part_ml[slot(0, r)], b = p.part_ml[slot(1, r)];
        const float m = fmaxf(a.x, b.x), ref = m == -INFINITY ? 0.f : m, f0 = ex2_approx(a.x - ref), f1 = ex2_approx(b.x - ref);
#pragma unroll
        for (int z = 0; z < N; ++z) o[z] = fmaf(x1.v[z], f1, x0.v[z] * f0);
        put(r, m, fmaf(b.y, f1, a.y * f0), o);
        continue;
      }
      // statistics of 32 pieces, a lane each
      auto stats = [&](int i) { return i < rec.count ? p.part_ml[slot(i, r)] : make_float2(-INFINITY, 0.f); };
      float m = -INFINITY, l = 0.f, f = 0.f;
#pragma unroll 1
      for (int i = lane; i < rec.count; i += 32) m = fmaxf(m, stats(i).x);
#pragma unroll
      for (int z = 16; z > 0; z >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, z));
      const float ref = m == -INFINITY ? 0.f : m;
#pragma unroll
      for (int z = 0; z < N; ++z) o[z] = 0.f;
#pragma unroll 1
      for (int i0 = 0; i0 < rec.count; i0 += 32) {
        const float2 ml = stats(i0 + lane);
        f = ex2_approx(ml.x - ref);
        l = fmaf(ml.y, f, l);
        const int n = min(32, rec.count - i0);
#pragma unroll 4
        for (int i = 0; i < n; ++i) {
          const Values x = values(i0 + i, r);
          const float fi = __shfl_sync(0xffffffffu, f, i);
#pragma unroll
          for (int z = 0; z < N; ++z) o[z] = fmaf(x.v[z], fi, o[z]);
        }
      }
#pragma unroll
      for (int z = 16; z > 0; z >>= 1) l += __shfl_xor_sync(0xffffffffu, l, z);
      put(r, m, l, o);
    }
  }
  // (in any order: a row depends on nothing but its keys)
  const uint32_t listed = p.head->listed, step = gridDim.x * gridDim.y * 8;
#pragma unroll 1
  for (uint32_t i = (blockIdx.y * gridDim.x + blockIdx.x) * 8 + wp; i < listed; i += step) row_by_keys<T, D>(p, p.list[i], sq[wp]);
}
int check_prefix(const fe_prefix_args* a) {
  if (!a) return fail(FE_ERR_INVALID_ARG, "null arguments");
  const int rc = check_paged_kv(a->kv);
  if (rc != FE_OK) return rc;
  if (a->n_groups < 0 || a->n_seqs < 0 || a->n_rows < 0 || a->prefix_cols < 1 || a->page_cols < 1)
    return fail(FE_ERR_INVALID_ARG, "negative size or no page column");
  if (a->q_heads < 1 || a->q_heads % a->kv.kv_heads != 0)
    return fail(FE_ERR_INVALID_ARG, "q_heads must be a multiple of kv_heads");
  if (a->q_heads / a->kv.kv_heads > 1024) return fail(FE_ERR_UNSUPPORTED, "at most 1024 query heads a key head");
  if ((long long)a->n_rows * a->q_heads > 0x7fffffffLL)
    return fail(FE_ERR_UNSUPPORTED, "n_rows * q_heads must be below 2^31");
  if (!std::isfinite(a->scale) || a->scale < 0.f) return fail(FE_ERR_INVALID_ARG, "scale must be finite and not negative");
  if (a->n_rows == 0) return FE_OK;
  if (a->n_groups == 0 || a->n_seqs == 0) return fail(FE_ERR_INVALID_ARG, "rows without a sequence or group");
  if (!a->group_start || !a->prefix_len || !a->prefix_pages || !a->row_start || !a->seq_len || !a->pages || !a->q || !a->out)
    return fail(FE_ERR_INVALID_ARG, "null pointer");
  if (a->out == a->q) return fail(FE_ERR_INVALID_ARG, "out must not be q");
  if (misaligned(a->q, 16) || misaligned(a->out, 32) || a->q_row % 8 != 0 || a->q_head % 8 != 0)
    return fail(FE_ERR_UNSUPPORTED, "q must be 16-byte aligned, its strides multiples of 8, out 32-byte aligned");
  return FE_OK;
}


// Sizes of the workspace's parts, in order, each on a 256-byte boundary
struct Layout {
  size_t head, tok, gtile, gcost, cost, before, recs, list, part_o, part_ml, bytes;
};
Layout layout(const fe_prefix_args* a, int ctas, int max_tiles) {
  size_t at = 0;
  auto take = [&](size_t n) {
    const size_t x = at;
    at += (n + 255) / 256 * 256;
    return x;
  };
  Layout w;
  w.head = take(sizeof(PlanHead));
  w.tok = take(8 * (size_t)a->n_rows);
  w.gtile = take(4 * ((size_t)a->n_groups + 1));
  w.gcost = take(8 * ((size_t)a->n_groups + 1));
  w.cost = take(4 * (size_t)max_tiles);
  w.before = take(8 * ((size_t)max_tiles + 1));
  w.recs = take(sizeof(SplitRec) * 2 * ctas);
  w.list = take(4 * (size_t)a->n_rows * a->q_heads);
  w.part_o = take((size_t)ctas * 2 * kUnitRows * a->kv.head_dim * 4);
  w.part_ml = take((size_t)ctas * 2 * kUnitRows * 8);
  w.bytes = at;
  return w;
}

// Row tiles at most: the groups' rows in whole tiles, and a part of one for each
int most_tiles(const fe_prefix_args* a) {
  return (int)((long long)a->n_rows * (a->q_heads / a->kv.kv_heads) / kUnitRows) + a->n_groups;
}

struct Device {
  int sms = 0;
  cudaError_t err = cudaErrorUnknown;
};
constexpr int kMaxDevices = 64;

// Once per device: its SMs and the kernels' shared-memory limits.
template <typename T, int D>
cudaError_t allow_smem() {
  return cudaFuncSetAttribute((const void*)prefix_attend_kernel<T, D>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                              (int)PrefixCfg<D>::kSmem);
}
const Device& device() {
  static Device devs[kMaxDevices];
  static std::once_flag once[kMaxDevices];
  static const Device none;
  int d = 0;
  if (cudaGetDevice(&d) != cudaSuccess || d < 0 || d >= kMaxDevices) return none;
  std::call_once(once[d], [d] {
    Device& v = devs[d];
    v.err = cudaDeviceGetAttribute(&v.sms, cudaDevAttrMultiProcessorCount, d);
    for (cudaError_t (*f)() : {allow_smem<__nv_bfloat16, 32>, allow_smem<__nv_bfloat16, 64>, allow_smem<__nv_bfloat16, 128>,
                               allow_smem<__half, 32>, allow_smem<__half, 64>, allow_smem<__half, 128>})
      if (v.err == cudaSuccess) v.err = f();
  });
  return devs[d];
}

// [n_pages * kv_heads * page_rows, head_dim] in boxes of some rows by 128 (or 64) bytes
bool encode_pages(CUtensorMap* m, const fe_paged_kv& kv, const void* base, int rows) {
  const cuuint64_t dims[2] = {(cuuint64_t)kv.head_dim, (cuuint64_t)kv.n_pages * kv.kv_heads * kv.page_rows};
  const cuuint64_t strides[1] = {(cuuint64_t)kv.head_dim * 2};
  const cuuint32_t box[2] = {(cuuint32_t)(kv.head_dim < 64 ? kv.head_dim : 64), (cuuint32_t)rows}, es[2] = {1u, 1u};
  const EncodeTiledFn fn = encode_tiled_fn();
  return fn && fn(m, kv.dtype == FE_IO_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 2,
                  const_cast<void*>(base), dims, strides, box, es, CU_TENSOR_MAP_INTERLEAVE_NONE,
                  kv.head_dim < 64 ? CU_TENSOR_MAP_SWIZZLE_64B : CU_TENSOR_MAP_SWIZZLE_128B,
                  CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <typename T, int D>
cudaError_t prefix_go(const PageMaps& m, const PrefixParams& p, cudaStream_t s) {
  using C = PrefixCfg<D>;
  cudaError_t e = launch_k(prefix_plan_kernel, dim3(kPlanCtas), dim3(kPlanThreads), 0, s, p);
  if (e == cudaSuccess)
    e = launch_k(prefix_attend_kernel<T, D>, dim3((unsigned)p.ctas), dim3(C::kThreads), C::kSmem, s, m, p);
  if (e == cudaSuccess) e = launch_k(prefix_finish_kernel<T, D>, dim3((unsigned)p.ctas, 2), dim3(256), 0, s, p);
  return e;
}
template <typename T>
cudaError_t prefix_dim(const PageMaps& m, const PrefixParams& p, int d, cudaStream_t s) {
  return d == 32 ? prefix_go<T, 32>(m, p, s) : d == 64 ? prefix_go<T, 64>(m, p, s) : prefix_go<T, 128>(m, p, s);
}

}  // namespace
}  // namespace fe

extern "C" uint64_t fe_prefix_attention_workspace(const fe_prefix_args* a) {
  using namespace fe;
  if (check_prefix(a) != FE_OK) return 0;
  const Device& dev = device();
  if (dev.err != cudaSuccess) {
    fail_cuda(dev.err, "fe_prefix_attention_workspace");
    return 0;
  }
  return layout(a, 2 * dev.sms, most_tiles(a)).bytes;
}

extern "C" int fe_prefix_attention(const fe_prefix_args* a, void* stream) {
  using namespace fe;
  const int rc = check_prefix(a);
  if (rc != FE_OK) return rc;
  if (a->n_rows == 0) return FE_OK;
  if (!a->workspace || misaligned(a->workspace, 256)) return fail(FE_ERR_INVALID_ARG, "workspace null or not 256-byte aligned");
  const Device& dev = device();
  if (dev.err != cudaSuccess) return fail_cuda(dev.err, "fe_prefix_attention");
  PrefixParams p{};
  p.ctas = 2 * dev.sms;
  const Layout w = layout(a, p.ctas, most_tiles(a));
  if (a->workspace_bytes < w.bytes) return fail(FE_ERR_WORKSPACE, "workspace too small");
  char* ws = static_cast<char*>(a->workspace);
  p.head = reinterpret_cast<PlanHead*>(ws + w.head);
  p.tok = reinterpret_cast<int2*>(ws + w.tok);
  p.gtile = reinterpret_cast<int*>(ws + w.gtile);
  p.gcost = reinterpret_cast<long long*>(ws + w.gcost);
  p.cost = reinterpret_cast<int*>(ws + w.cost);
  p.before = reinterpret_cast<long long*>(ws + w.before);
  p.recs = reinterpret_cast<SplitRec*>(ws + w.recs);
  p.list = reinterpret_cast<int*>(ws + w.list);
  p.part_o = reinterpret_cast<float*>(ws + w.part_o);
  p.part_ml = reinterpret_cast<float2*>(ws + w.part_ml);
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
  p.hr = p.hq / p.hkv;
  p.hr_inv = (int)(uint32_t)((0x100000000ull + p.hr - 1) / p.hr);
  p.prefix_cols = a->prefix_cols;
  p.page_cols = a->page_cols;
  p.page_rows = a->kv.page_rows;
  while ((1 << p.page_shift) < p.page_rows) ++p.page_shift;
  p.n_pages = a->kv.n_pages;
  p.scale = a->scale;
  p.sc = std::fmax((float)(a->scale * 1.4426950408889634), 1e-30f);
  PageMaps m;
  if (!encode_pages(&m.k, a->kv, a->kv.k, p.page_rows) || !encode_pages(&m.v, a->kv, a->kv.v, p.page_rows))
    return fail(FE_ERR_CUDA, "cuTensorMapEncodeTiled failed");
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  const cudaError_t e = a->kv.dtype == FE_IO_BF16 ? prefix_dim<__nv_bfloat16>(m, p, a->kv.head_dim, s)
                                                  : prefix_dim<__half>(m, p, a->kv.head_dim, s);
  return e == cudaSuccess ? FE_OK : fail_cuda(e, "fe_prefix_attention");
}
