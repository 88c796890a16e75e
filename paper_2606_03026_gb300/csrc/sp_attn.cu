// sp_attn.cu -- attention of a batch whose sequences share a prefix (see
// spike_proj_cache_attend): a query row r of sequence b sees the P entries of
// the prefix and its own entries,
//
//   s_j = scale q_r . k_j,   out_r = sum_j e^{s_j - lse_r} v_j,
//   weights[b][h][j] += sum over the rows of e^{s_j - lse_r}  (own entries)
//
// The rows of one K/V head are the T x G query rows (G query heads share it) of
// one sequence, R in all; for the prefix the rows of every sequence together,
// so that its entries are read once for 128 of them.
//
// attend_kernel: units of (up to 128 rows, K/V head) x all their entries, cut
// into tiles of 64 entries.  The tiles of all units, the prefix's first, are one
// line that two CTAs per SM share out evenly by cost, whatever the lengths
// (which only the device knows); a CTA's run of tiles within a unit is a
// segment, which leaves its sum over V, its maximum and its sums of
// exponentials in a slot of the workspace.  Per CTA (192 threads):
//   warp 4      copies (TMA): the query rows of a segment (a box of G heads x T
//               tokens, for the prefix x as many sequences as 128 rows hold), K
//               tiles and V tiles into rings, each as soon as its place is free.
//   warp 5      S = Q K^T one tile ahead of O += P V (tcgen05, M = 128, P from
//               tensor memory, V as an N-major operand).
//   warps 0-3   the softmax, thread = row = tensor-memory lane: per tile they
//               read the 64 scores of their row, keep the running maximum and
//               sums, and put the probabilities, rounded to the type, back over
//               the scores.
// Exponentials are powers of two of (s scale log2 e - reference).  The
// reference follows the running maximum only when that has grown by more than
// 2^kLag, so that O is rescaled seldom; half precision is offset by 2^10 so that
// its subnormals lie below 2^-34 of the largest probability.  The sum over V is
// divided by the sum of the rounded probabilities that made it, so that what
// their rounding errors have in common cancels (one entry that has all of the
// weight comes out exactly); lse and weights take the sum before rounding.
// The tiles hold the entries that every row of a unit sees.  The last T - 1 own
// entries, of which the query tokens see 0, 1, .. T - 1, are left to
// combine_kernel, so that no masked probability ever meets a value.
//
// What bounds it: K and V from memory where few rows share an entry, the tensor
// cores where 128 do (their rate at N = 64, where Q is read from shared memory
// again for every tile, is 4/5 of the peak for 128-wide heads), and in between a
// tile's way from S through the softmax to P, of which two CTAs have one each on
// their way per SM: about 1300 cycles a tile and CTA, of which the softmax's
// arithmetic is 370 at full rate.  Tiles of 64 entries with the scores one tile
// ahead, because tensor memory holds no more for 128-wide heads and two CTAs (128
// entries without: 128 drafting sequences 291 us, with 64: 212 at that state).
// Measured (a call, its three kernels together, replayed from a graph on three sets of
// inputs in turn; by itself a call takes about 1 us more, and the largest at the power
// limit's clock 145): 128 sequences of 5 tokens, 16 query heads on 4 of 128, prefix
// 16384, own 512 to 2048, with weights: 141 us, the floor of its bytes 56, of its
// operations 48, tensor pipe busy 67 to 74 % in attend_kernel (111 us); 16 sequences over
// a document of 131072: 53.4 us, 5.2 TB/s; 64 chats over 2048 with own caches of up to
// 1024: 26.6 us (floor 10.7), the kernel itself 21; 32 drafting sequences with 64-wide
// heads over 8191: 47.5 us (floor 13); one sequence of 60 entries over 512: 10.0 us, two
// launches' latency.
//
// combine_kernel: half a warp to eight warps per query row merge its partial results
// and these last entries, row by row (right for any T, meant for a few drafts: 16
// sequences with 1 / 8 / 16 / 32 tokens 16 / 23 / 27 / 41 us a call); latency, and for
// many rows the instructions of a row (10240 rows 12 us).  weights_kernel: the weights,
// from the scores of the own entries that attend_kernel left in the workspace and the
// rows' lse; 4 bytes written and read per own entry and query row (128 drafting
// sequences: 52 MB, 13 us).
#include <cuda.h>
#include <cuda_fp16.h>
#include <cudaTypedefs.h>

#include <math.h>

#include "sp_cache.h"
#include "sp_ptx.cuh"

namespace sp {
namespace {

constexpr int kTile = 64;                  // entries of a tile
constexpr int kRows = 128;                 // rows of the MMA
constexpr int kAttThreads = 192;
constexpr int kGroups = kAttThreads;
constexpr int kTmemCols = 256;             // S and P: 0 .. 63 and 64 .. 127, O (and the sum of P): from 128 on
constexpr uint32_t kTmemO = 128;
constexpr int kQBlock = kRows * 128;       // 64 elements of 128 rows
constexpr int kBlock = kTile * 128;        // 64 elements of a tile's entries
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

// Tiles of K and of V on their way: what two CTAs of an SM have room for.
template <int DK> constexpr int kStagesK = DK == 64 ? 5 : 3;
template <int DK> constexpr int kStagesV = DK == 64 ? 5 : 2;
// With 64-wide heads the product with V has 16 more columns, of ones: the sum of
// the rounded probabilities, for which tensor memory has no room at 128.
template <int DK> constexpr int kOnes = DK == 64 ? 16 : 0;
template <int DK> constexpr int kQBytes = DK / 64 * kQBlock;
template <int DK> constexpr int kTileBytes = DK / 64 * kBlock;

// The rows of units.  Of one sequence: `per_seq` tiles of `tokens` query tokens
// x `heads` query heads (all G of them, or 128 at a time).  A prefix unit has
// those of `seqs` sequences, which is 1 unless all rows of a sequence fit.
struct Rows {
  int32_t heads, tokens, seqs;
  int32_t head_tiles, per_seq;             // tiles that share a token; tiles of a sequence
  int32_t prefix_units, own_units;         // per K/V head; per sequence and K/V head
  int32_t prefix_rows, own_rows;           // of a whole unit
};

struct Costs {
  int32_t prefix_start, prefix_tile, own_start, own_tile;
};

struct AttnMaps {
  CUtensorMap pq, pk, pv, q, k, v;         // of the prefix units, of the own units
};

struct AttnParams {
  sp_attend c;
  int32_t Hq, Hkv, G, D, capacity, R;      // R = T G: query rows of a sequence and K/V head
  Rows rows;
  Costs costs;
  int32_t nt_prefix, nt_cap;               // tiles of the prefix, of the capacity
  int32_t grid;                            // CTAs of attend_kernel
  bool whole_rows;          // D is DK = 128: a tile of K or V is one copy
  float c2;                 // scale * log2 e
  int* err;
  int fault;                // kFaultStall: first copies are left out (tests of the error path)
  long long limit;          // cycles that a wait takes at most
  int2* unit_ctas;          // first and last CTA of each prefix unit, of each own unit that has tiles
  float4* p_ml;             // prefix slots: [slot][128] reference, sum, sum of the rounded
  float* p_o;               //               [slot][128][DK]
  float4* o_ml;             // own slots: [slot][own_rows], the same [DK]
  float* o_o;
  float* scores;            // [B][Hkv][nt_cap][R][64], or null
  float* lse2;              // [B][Hkv][R], base 2; +infinity where a row sees nothing
};

// ---- the line of tiles -------------------------------------------------------
__device__ __forceinline__ int used(const AttnParams& p, int b) {
  return min(max(__ldg(p.c.lens + b), 0), p.capacity);
}
// Own entries of a sequence that every query token sees.
__device__ __forceinline__ int seen_by_all(const AttnParams& p, int b) { return max(0, used(p, b) - (p.c.T - 1)); }

// The line is measured in cost: a unit costs `start` and then each of its tiles.
struct Line {
  int prefix, all;          // cost of the prefix units; of all (a call has fewer than 2^25 tiles)
  int32_t prefix_unit;      // of one
  int ctas;                 // that share it
  // CTA c has the tiles that end past first(c), up to first(c + 1)
  __device__ __forceinline__ int first(int c) const { return (int)((int64_t)c * all / ctas); }
};
__device__ __forceinline__ Line line_of(const AttnParams& p, int own_cost, int grid) {
  const Costs& k = p.costs;
  Line l;
  l.prefix_unit = k.prefix_start + p.nt_prefix * k.prefix_tile;
  l.prefix = p.nt_prefix == 0 ? 0 : p.Hkv * p.rows.prefix_units * l.prefix_unit;
  l.all = l.prefix + own_cost;
  // (as much for every CTA as a tile costs at most: a unit's tiles are of
  // CTAs without a gap)
  const int most = max(k.prefix_tile, k.own_tile);
  l.ctas = l.all / most >= grid ? grid : max(1, l.all / most);
  return l;
}
__device__ __forceinline__ int own_cost(const AttnParams& p, int b) {
  const int nt = ceil_div(seen_by_all(p, b), kTile);
  return nt == 0 ? 0 : p.Hkv * p.rows.own_units * (p.costs.own_start + nt * p.costs.own_tile);
}

struct Segment {
  bool prefix;
  int b, h, m;              // first sequence, head, row tile of the sequence
  int j0, count, nt;        // tiles, of nt that the unit has
  int seen;                 // entries of the unit
  int rows;
  int next;                 // where the following unit begins on the line
  int64_t slot;
};
// off: cost of the own units before each of the groups of sequences that
// attend_kernel's threads add up.  The segment at point x of a CTA whose tiles end at `end`; of no tiles where
// the first one past x ends past `end`.
__device__ __forceinline__ Segment segment_at(const AttnParams& p, const Line& l, const int* off, int x, int end,
                                              int cta) {
  const Rows& r = p.rows;
  Segment s;
  s.prefix = x < l.prefix;
  int start, tile, at;                     // at: where the unit begins
  if (s.prefix) {
    const int u = (uint32_t)x / (uint32_t)l.prefix_unit;
    at = u * l.prefix_unit;
    s.next = at + l.prefix_unit;
    s.nt = p.nt_prefix;
    start = p.costs.prefix_start;
    tile = p.costs.prefix_tile;
    s.h = (uint32_t)u / (uint32_t)r.prefix_units;
    const int i = u - s.h * r.prefix_units;
    s.b = i * r.seqs;
    s.m = 0;
    if (r.per_seq > 1) {                   // (then seqs is 1)
      s.b = i / r.per_seq;
      s.m = i - s.b * r.per_seq;
    }
    s.seen = p.c.prefix_len;
    s.slot = cta + u;
  } else {
    const int y = x - l.prefix;
    int lo = 0, hi = kGroups;              // off[lo] <= y < off[hi]
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (off[mid] <= y) lo = mid; else hi = mid;
    }
    int before = off[lo];
    const int per = ceil_div(p.c.B, kGroups);
    lo *= per;
    if (per > 1)
      for (int cost; before + (cost = own_cost(p, lo)) <= y; ++lo) before += cost;
    s.b = lo;
    s.seen = seen_by_all(p, lo);
    s.nt = ceil_div(s.seen, kTile);
    const int unit = p.costs.own_start + s.nt * p.costs.own_tile;
    const int u = (uint32_t)(y - before) / (uint32_t)unit;
    at = l.prefix + before + u * unit;
    s.next = at + unit;
    start = p.costs.own_start;
    tile = p.costs.own_tile;
    s.h = u;
    s.m = 0;
    if (r.own_units > 1) {
      s.h = u / r.own_units;
      s.m = u - s.h * r.own_units;
    }
    s.slot = cta + (int64_t)lo * p.Hkv * r.own_units + u;
  }
  // tile j ends at `at + start + (j + 1) tile`
  s.j0 = max(0, x - at - start) / tile;
  s.count = min(s.nt, max(0, min(end, s.next) - at - start) / tile) - s.j0;
  s.rows = r.head_tiles > 1 ? min(r.heads, p.G - s.m % r.head_tiles * r.heads)
                            : min(r.tokens, p.c.T - s.m * r.tokens) * p.G;
  if (s.prefix) s.rows *= min(r.seqs, p.c.B - s.b);
  return s;
}

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
template <bool BF16>
__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
  uint32_t r;
  if constexpr (BF16)
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  else
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
// a += the lower half of x, b += the upper one, without unpacking them first (64
// chats 27.2 -> 26.7 us a call, 32 drafting sequences 49.8 -> 48.0).
template <bool BF16>
__device__ __forceinline__ void add_halves(uint32_t x, float& a, float& b) {
  if constexpr (BF16)
    asm("{\n\t.reg .b16 l, h;\n\tmov.b32 {l, h}, %2;\n\tadd.rn.f32.bf16 %0, l, %0;\n\tadd.rn.f32.bf16 %1, h, %1;\n\t}"
        : "+f"(a), "+f"(b)
        : "r"(x));
  else
    asm("{\n\t.reg .b16 l, h;\n\tmov.b32 {l, h}, %2;\n\tadd.rn.f32.f16 %0, l, %0;\n\tadd.rn.f32.f16 %1, h, %1;\n\t}"
        : "+f"(a), "+f"(b)
        : "r"(x));
}
template <bool BF16> __device__ __forceinline__ float2 unpack2(uint32_t x) {
  if constexpr (BF16) return make_float2(__uint_as_float(x << 16), __uint_as_float(x & 0xffff0000u));
  const __half2 h = *reinterpret_cast<const __half2*>(&x);
  return __half22float2(h);
}

// Two floats in one 64-bit register, for the packed FP32 instructions.
using f32x2 = unsigned long long;
__device__ __forceinline__ f32x2 pair(float a, float b) {
  f32x2 r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ float2 halves(f32x2 x) {
  float2 r;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(x));
  return r;
}
__device__ __forceinline__ f32x2 fma2(f32x2 a, f32x2 b, f32x2 c) {
  f32x2 r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
__device__ __forceinline__ f32x2 add2(f32x2 a, f32x2 b) {
  f32x2 r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ void fence_async_shared() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

// An operand whose rows run along the MMA's N: 64 elements (128 bytes,
// swizzled) per row of K, 8 rows of K 1024 bytes apart, the next 64 elements
// of N `block` bytes on.
__device__ __forceinline__ uint64_t n_major_desc(const void* p, uint32_t block) {
  uint64_t d = smem_desc(p, 1024, kSwizzle128);
  d &= ~((uint64_t)0x3FFF << 16);
  return d | (uint64_t)(block >> 4) << 16;
}

// Bounded wait, inline (a call would cost the softmax's loop its registers);
// false too when another warp of the CTA has given up (`stop`, where given).
__device__ __forceinline__ bool wait(const AttnParams& p, uint64_t* bar, uint32_t parity, const volatile int* stop = nullptr) {
  if (mbar_try_wait(bar, parity)) return true;
  const long long t0 = clock64();
  do {
    if (mbar_try_wait(bar, parity)) return true;
  } while (!(stop && *stop) && clock64() - t0 < p.limit);
  return false;
}

// The place of the query rows in shared memory: segments of up to 64 rows have
// half of it in turn (64 rows of every block of 64 elements), so that the next
// one's rows are there in time; others the whole.  used: the parity of the times
// that each half was taken.
struct RowPlaces {
  int next = 0, used = 0;
  __device__ __forceinline__ int of(int rows) const { return rows > kRows / 2 ? 3 : 1 << next; }
  __device__ __forceinline__ void take(int halves) {
    if (halves != 3) next ^= 1;
    used ^= halves;
  }
};

// 32 bytes, a whole sector of memory.
__device__ __forceinline__ void store8(float* to, const uint32_t* v) {
  asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(to), "r"(v[0]), "r"(v[1]), "r"(v[2]),
               "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7])
               : "memory");
}

// What a softmax thread keeps of its row.
struct RowState {
  float m, ref, l, rl;      // maximum that the reference follows, reference, sums
};

// One tile: the row's scores at s_buf (left in v, -infinity past nv) become its
// probabilities.  pv: the barrier
// (and its parity) that says that the product before this tile's is complete.
template <int DK, bool BF16>
__device__ __forceinline__ bool softmax_tile(const AttnParams& p, RowState& r, uint32_t (&v)[2][32], uint32_t s_buf,
                                             uint32_t o_buf, int nv, bool first, uint64_t* pv, uint32_t pv_parity) {
  constexpr float kLag = BF16 ? 8.f : 4.f, kLift = BF16 ? 0.f : 10.f;
  tmem_ld32_issue(s_buf, v[0]);
  tmem_ld32_issue(s_buf + 32, v[1]);
  tmem_ld_wait();
  reg_pin(v[0]);
  reg_pin(v[1]);
  if (nv < kTile) {
#pragma unroll
    for (int i = 0; i < kTile; ++i)
      if (i >= nv) v[i / 32][i % 32] = 0xff800000u;
  }
  float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
  for (int i = 0; i < kTile; ++i) mx[i % 4] = fmaxf(mx[i % 4], __uint_as_float(v[i / 32][i % 32]));
  const float top = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3])) * p.c2;
  const bool grow = top > r.m + kLag;
  if (__any_sync(0xffffffffu, grow)) {
    float a = 1.f;
    if (grow) {
      a = ex2(r.m - top);                  // 0 at the first
      r.m = top;
      r.ref = top - kLift;
    }
    r.l *= a;
    r.rl *= a;
    if (!first) {
      if (!__all_sync(0xffffffffu, wait(p, pv, pv_parity))) return false;
      tc_fence_after();
#pragma unroll 1                           // (rare, and registers are short)
      for (int i = 0; i < (DK + kOnes<DK>) / 16; ++i) {
        uint32_t o[16];
        tmem_ld16_issue(o_buf + 16 * i, o);
        tmem_ld_wait();
        reg_pin(o);
#pragma unroll
        for (int e = 0; e < 16; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * a);
        tmem_st16_issue(o_buf + 16 * i, o);
      }
    }
  }
  f32x2 sum[2] = {};
  float rsum[4] = {};
  const f32x2 c2 = pair(p.c2, p.c2), base = pair(-r.ref, -r.ref);
#pragma unroll
  for (int g = 0; g < 2; ++g) {
    uint32_t pk[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const float2 x = halves(fma2(pair(__uint_as_float(v[g][2 * i]), __uint_as_float(v[g][2 * i + 1])), c2, base));
      const float2 y = make_float2(ex2(x.x), ex2(x.y));
      pk[i] = pack2<BF16>(y.x, y.y);
      sum[i % 2] = add2(sum[i % 2], pair(y.x, y.y));
      if (kOnes<DK> == 0) add_halves<BF16>(pk[i], rsum[i % 2 * 2], rsum[i % 2 * 2 + 1]);
    }
    tmem_st16_issue(s_buf + 16 * g, pk);
  }
  const float2 ls = halves(add2(sum[0], sum[1]));
  r.l += ls.x + ls.y;
  r.rl += (rsum[0] + rsum[1]) + (rsum[2] + rsum[3]);
  tmem_st_wait();
  return true;
}

// One tile of entries into shared memory, 64 elements of all of them after 64
// elements: in one copy where rows are made of whole blocks.  The whole warp
// executes it, the lane with `issue` copies.
template <int DK>
__device__ __forceinline__ void load_tile(uint32_t issue, uint8_t* to, const CUtensorMap* map, uint64_t* full, bool whole,
                                          int entry, int head, int batch, uint64_t policy) {
  if (DK == 64 || !whole) {
#pragma unroll
    for (int i = 0; i < DK / 64; ++i)
      tma_load_4d_if(issue, to + i * kBlock, map, full, 64 * i, entry, head, batch, policy);
  } else {
    tma_load_5d_if(issue, to, map, full, 0, entry, 0, head, batch, policy);
  }
}

template <int DK, bool BF16>
__global__ void __launch_bounds__(kAttThreads, 2)
attend_kernel(const __grid_constant__ AttnMaps maps, const __grid_constant__ AttnParams p) {
  constexpr int NK = kStagesK<DK>, NV = kStagesV<DK>, kBytes = kTileBytes<DK>;
  constexpr uint32_t kType = BF16 ? 1u << 7 | 1u << 10 : 0u;
  constexpr uint32_t kIdescS = 1u << 4 | kType | (uint32_t)(kTile >> 3) << 17 | (uint32_t)(kRows >> 4) << 24;
  constexpr uint32_t kIdescO = 1u << 4 | kType | 1u << 16 | (uint32_t)((DK + kOnes<DK>) >> 3) << 17 | (uint32_t)(kRows >> 4) << 24;
  extern __shared__ __align__(1024) uint8_t smem[];
  uint8_t* sQ = smem;
  uint8_t* sK = sQ + kQBytes<DK>;
  uint8_t* sV = sK + NK * kBytes;
  uint8_t* s_ones = sV + NV * kBytes;       // as a tile of 64 elements, where there are ones
  uint64_t* bars = reinterpret_cast<uint64_t*>(s_ones + (kOnes<DK> ? kBlock : 0));
  uint64_t *k_full = bars, *k_empty = bars + NK, *v_full = bars + 2 * NK, *v_empty = v_full + NV;
  uint64_t *s_full = v_empty + NV, *p_full = s_full + 2;   // [2]: by score buffer
  uint64_t *q_full = p_full + 2, *q_empty = q_full + 2,     // [2]: by half of the rows' place
           *o_full = q_full + 4, *o_empty = q_full + 5, *done = q_full + 6;
  uint32_t* s_tmem = reinterpret_cast<uint32_t*>(done + 1);
  volatile int* s_abort = reinterpret_cast<volatile int*>(s_tmem + 1);
  int* s_sum = reinterpret_cast<int*>(s_tmem + 2);         // [8]
  int* s_off = s_sum + 8;                                  // [kGroups + 1]

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    for (int i = 0; i < NK; ++i) {
      mbar_init(&k_full[i], 1);
      mbar_init(&k_empty[i], 1);
    }
    for (int i = 0; i < NV; ++i) {
      mbar_init(&v_full[i], 1);
      mbar_init(&v_empty[i], 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&s_full[i], 1);
      mbar_init(&p_full[i], 4);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&q_full[i], 1);
      mbar_init(&q_empty[i], 1);
    }
    mbar_init(o_full, 1);
    mbar_init(o_empty, 4);
    mbar_init(done, 1);
    *s_abort = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    tma_prefetch_desc(&maps.pq);
    tma_prefetch_desc(&maps.pk);
    tma_prefetch_desc(&maps.pv);
    tma_prefetch_desc(&maps.q);
    tma_prefetch_desc(&maps.k);
    tma_prefetch_desc(&maps.v);
  }
  if (warp == 5) tmem_alloc(s_tmem, kTmemCols);
  if (kOnes<DK>) {
    for (int i = threadIdx.x; i < kBlock / 4; i += kAttThreads)
      reinterpret_cast<uint32_t*>(s_ones)[i] = BF16 ? 0x3f803f80u : 0x3c003c00u;
    fence_async_shared();
  }
  pdl_launch_dependents();
  pdl_wait();

  // the own units before each sequence: every CTA adds their costs up for itself
  {
    const int per = ceil_div(p.c.B, kGroups), b0 = threadIdx.x * per, b1 = min(b0 + per, p.c.B);
    int sum = 0;
    for (int b = b0; b < b1; ++b) sum += own_cost(p, b);
    int incl = sum;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const int y = __shfl_up_sync(0xffffffffu, incl, d);
      if (lane >= d) incl += y;
    }
    if (lane == 31) s_sum[warp] = incl;
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    int at = incl - sum;
    for (int w = 0; w < warp; ++w) at += s_sum[w];
    s_off[threadIdx.x] = at;
    if (threadIdx.x == kGroups - 1) s_off[kGroups] = at + sum;
    __syncthreads();
  }
  const uint32_t tmem = *s_tmem;
  const Line line = line_of(p, s_off[kGroups], gridDim.x);
  const int cta = blockIdx.x;
  // (the same in every thread; taken from one, the compiler knows it)
  const int x0 = __shfl_sync(0xffffffffu, cta < line.ctas ? line.first(cta) : 0, 0);
  const int x1 = __shfl_sync(0xffffffffu, cta < line.ctas ? line.first(cta + 1) : 0, 0);

  if (warp == 4) {
    // ------------------------------ TMA -----------------------------------------
    // The whole warp walks the tiles and one lane issues, by predicate (as the
    // MMAs below; by a branch of lane 0 the warp was busy all the time and 128
    // drafting sequences took 141.8 us instead of 140.4).
    const uint32_t one = elect_one();
    const auto all = [](bool x) { return __all_sync(0xffffffffu, x) != 0; };
    const auto uniform = [](int x) { return __shfl_sync(0xffffffffu, x, 0); };
    // where the keys and where the values are: a tile of a segment
    struct Cursor {
      int count, j, entry, h, b, m, next, prefix;
      int st, phase;                       // place in the ring, how often it has gone round
    };
    const auto enter = [&](Cursor& c, int x) {
      c.j = c.count = 0;
      if (x >= x1) return;
      const Segment s = segment_at(p, line, s_off, x, x1, cta);
      c.count = uniform(s.count);
      c.entry = uniform(s.j0 * kTile);
      c.h = uniform(s.h);
      c.b = uniform(s.b);
      c.m = uniform(s.m);
      c.next = uniform(s.next);
      c.prefix = uniform(s.prefix);
    };
    Cursor k, v;
    enter(k, x0);
    v = k;
    k.st = v.st = k.phase = v.phase = 0;
    // Own entries that one unit reads leave L2 to the prefix, the scores and the
    // partial results (64 chats 33.7 -> 31.9 us, 128 drafting sequences 145.6 -> 143.1).
    const uint64_t normal = l2_evict_normal(), own = p.rows.own_units == 1 ? l2_evict_first() : normal;
    RowPlaces places;
    bool rows = k.count > 0;               // the query rows of the keys' segment are to come
    const auto issue = [&](Cursor& c, uint32_t copy, int n, uint8_t* ring, uint64_t* full, const CUtensorMap* of_prefix,
                           const CUtensorMap* of_own) {
      mbar_arrive_expect_tx_if(one, &full[c.st], kBytes);
      load_tile<DK>(copy, ring + c.st * kBytes, c.prefix ? of_prefix : of_own, &full[c.st], p.whole_rows, c.entry, c.h,
                    c.prefix ? 0 : c.b, c.prefix ? normal : own);
      c.entry += kTile;
      ++c.j;
      if (++c.st == n) {
        c.st = 0;
        ++c.phase;
      }
    };
    uint32_t copy = p.fault == kFaultStall ? 0u : one;       // (a test's fault leaves the first keys out)
    bool ok = true;
    int idle = 0;
    long long since = 0;
    while (k.count > 0 || v.count > 0) {
      // (a segment's keys may go ahead of its query rows, the next one's not)
      const bool k_free = mbar_test(&k_empty[k.st], k.phase & 1 ^ 1), v_free = mbar_test(&v_empty[v.st], v.phase & 1 ^ 1);
      bool moved = false;
      if (k.j < k.count && all(k_free)) {
        issue(k, copy, NK, sK, k_full, &maps.pk, &maps.k);
        copy = one;
        moved = true;
      }
      if (v.count > 0 && all(v_free)) {
        issue(v, one, NV, sV, v_full, &maps.pv, &maps.v);
        if (v.j == v.count) enter(v, v.next);
        moved = true;
      }
      if (rows) {
        const int box = k.prefix ? p.rows.prefix_rows : p.rows.own_rows, halves = places.of(box);
        if (all(((halves & 1) == 0 || mbar_test(&q_empty[0], places.used & 1 ^ 1)) &&
                ((halves & 2) == 0 || mbar_test(&q_empty[1], places.used >> 1 ^ 1)))) {
          const int head = k.h * p.G + k.m % p.rows.head_tiles * p.rows.heads;
          const int token = k.m / p.rows.head_tiles * p.rows.tokens;
          uint64_t* full = &q_full[halves == 2];
          mbar_arrive_expect_tx_if(one, full, DK / 64 * 128 * box);
          if (halves == 3) mbar_arrive_expect_tx_if(one, &q_full[1], 0);
          for (int i = 0; i < DK / 64; ++i)
            tma_load_4d_if(one, sQ + i * kQBlock + (halves == 2 ? kQBlock / 2 : 0), k.prefix ? &maps.pq : &maps.q, full, 64 * i,
                           head, token, k.b, normal);
          places.take(halves);
          rows = false;
          moved = true;
        }
      }
      if (k.j == k.count && k.count > 0 && !rows) {
        enter(k, k.next);
        rows = k.count > 0;
      }
      if (moved) {
        idle = 0;
      } else {
        if (idle++ == 0) since = clock64();
        if (!all(!*s_abort && clock64() - since <= p.limit)) {
          ok = false;
          break;
        }
      }
    }
    if (!ok) {
      *s_abort = 1;
      atomicExch(p.err, kErrMbarTimeout);
      for (int i = 0; i < 2; ++i) wait(p, &q_full[i], places.used >> i & 1 ^ 1);
    }
    // the last copies have landed
    const auto landed = [&](const Cursor& c, int n, uint64_t* full) {
      for (int i = 0; i < n; ++i)
        if (i < c.st || c.phase > 0) wait(p, &full[i], (i < c.st ? c.phase : c.phase - 1) & 1);
    };
    landed(k, NK, k_full);
    landed(v, NV, v_full);
  } else if (warp == 5) {
    // ------------------------------ MMA -----------------------------------------
    // The whole warp walks the tiles and one lane issues, by predicate: operands
    // stay in uniform registers (by a branch of lane 0, each instruction took
    // about 70 cycles to issue).
    const uint32_t one = elect_one();
    int it = 0, seg = 0;                   // it: tiles whose product with V is issued
    bool ok = true;
    RowPlaces places;
    const auto all = [](bool x) { return __all_sync(0xffffffffu, x) != 0; };
    const auto scores = [&](int i, int halves, bool last) {
      const int st = i % NK;
      if (!all(wait(p, &k_full[st], (i / NK) & 1, s_abort))) return false;
      tc_fence_after();
      // (half a place on the MMA's later rows read what is there: nobody reads theirs)
      const uint64_t qd = smem_desc(sQ + (halves == 2 ? kQBlock / 2 : 0), 1024, kSwizzle128);
      const uint64_t kd = smem_desc(sK + st * kBytes, 1024, kSwizzle128);
#pragma unroll
      for (int k = 0; k < DK / 16; ++k)
        mma_f16_if(one, tmem + (i & 1) * kTile, qd + (k / 4) * (kQBlock >> 4) + (k % 4) * 2,
                   kd + (k / 4) * (kBlock >> 4) + (k % 4) * 2, kIdescS, k > 0);
      mma_commit_if(one, &s_full[i & 1]);
      mma_commit_if(one, &k_empty[st]);
      if (last && (halves & 1)) mma_commit_if(one, &q_empty[0]);
      if (last && (halves & 2)) mma_commit_if(one, &q_empty[1]);
      return true;
    };
    Segment next;
    next.count = 0;
    if (x0 < x1) next = segment_at(p, line, s_off, x0, x1, cta);
    for (; ok && next.count > 0; ++seg) {
      const int count = __shfl_sync(0xffffffffu, next.count, 0);
      const int halves = __shfl_sync(0xffffffffu, places.of(next.prefix ? p.rows.prefix_rows : p.rows.own_rows), 0);
      // (the buffer of tile i + 1 is that of tile i - 1, whose product with V,
      // issued before, reads the probabilities there first)
      ok = all(((halves & 1) == 0 || wait(p, &q_full[0], places.used & 1, s_abort)) &&
               ((halves & 2) == 0 || wait(p, &q_full[1], places.used >> 1, s_abort))) &&
           scores(it, halves, count == 1);
      places.take(halves);
      const int x = next.next;             // (the next segment, while the first softmax runs)
      next.count = 0;
      if (x < x1) next = segment_at(p, line, s_off, x, x1, cta);
      for (int j = 0; j < count && ok; ++j, ++it) {
        const int st = it % NV;
        if (j + 1 < count) ok = scores(it + 1, halves, j + 2 == count);
        if (ok)
          ok = all(wait(p, &v_full[st], (it / NV) & 1, s_abort) && (j > 0 || wait(p, o_empty, (seg & 1) ^ 1u, s_abort)) &&
                   wait(p, &p_full[it & 1], (it >> 1) & 1, s_abort));
        if (!ok) break;
        tc_fence_after();
        const uint64_t vd = n_major_desc(sV + st * kBytes, kOnes<DK> ? (NV - st) * kBytes : kBlock);
#pragma unroll
        for (int k = 0; k < kTile / 16; ++k)
          mma_f16_ta_if(one, tmem + kTmemO, tmem + (it & 1) * kTile + 8 * k, vd + k * (2048 >> 4), kIdescO, j > 0 || k > 0);
        mma_commit_if(one, &v_empty[st]);
      }
      if (ok) mma_commit_if(one, o_full);
    }
    if (!ok) {
      *s_abort = 1;
      atomicExch(p.err, kErrMbarTimeout);
    }
    mma_commit_if(one, done);              // every MMA has retired
    wait(p, done, 0);
  } else {
    // ------------------------------ softmax -------------------------------------
    const uint32_t lanes = tmem + ((uint32_t)(warp * 32) << 16);
    int it = 0, seg = 0;
    bool ok = true;
    Segment next;
    next.count = 0;
    if (x0 < x1) next = segment_at(p, line, s_off, x0, x1, cta);
    for (; ok && next.count > 0; ++seg) {
      const Segment s = next;
      const int row = threadIdx.x;
      const bool work = warp * 32 < s.rows, mine = row < s.rows;
      const int rr = s.m / p.rows.head_tiles * p.rows.tokens * p.G + s.m % p.rows.head_tiles * p.rows.heads + row;
      RowState r = {-INFINITY, 0.f, 0.f, 0.f};
      for (int j = 0; j < s.count; ++j, ++it) {
        const int nv = min(kTile, s.seen - (s.j0 + j) * kTile);
        ok = __all_sync(0xffffffffu, wait(p, &s_full[it & 1], (it >> 1) & 1, s_abort));
        if (!ok) break;
        tc_fence_after();
        uint32_t v[2][32];
        if (work) {
          uint64_t* pv = &v_empty[(it + NV - 1) % NV];
          const uint32_t pvp = ((it + NV - 1) / NV - 1) & 1, sb = lanes + (it & 1) * kTile, ob = lanes + kTmemO;
          ok = softmax_tile<DK, BF16>(p, r, v, sb, ob, nv, j == 0, pv, pvp);
          if (!ok) break;
        }
        if (!s.prefix && nv < kTile) {
          // entries past those in use hold anything: their values become 0
          const int st = it % NV;
          ok = __all_sync(0xffffffffu, wait(p, &v_full[st], (it / NV) & 1, s_abort));
          if (!ok) break;
          if (threadIdx.x >= nv && threadIdx.x < kTile) {
#pragma unroll
            for (int i = 0; i < DK / 64; ++i)
#pragma unroll
              for (int e = 0; e < 8; ++e)
                *reinterpret_cast<uint4*>(sV + st * kBytes + i * kBlock + threadIdx.x * 128 + 16 * e) =
                    make_uint4(0u, 0u, 0u, 0u);
          }
          fence_async_shared();
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&p_full[it & 1]);
        if (!s.prefix && p.scores && mine) {
          // (after the probabilities are on their way: the stores hold a warp up)
          float* sc = p.scores + ((((int64_t)s.b * p.Hkv + s.h) * p.nt_cap + s.j0 + j) * p.R + rr) * kTile;
#pragma unroll
          for (int i = 0; i < kTile / 8; ++i) store8(sc + 8 * i, &v[i / 4][i % 4 * 8]);
        }
      }
      if (!ok) break;
      next.count = 0;                      // (the next segment, while the last product is computed)
      if (s.next < x1) next = segment_at(p, line, s_off, s.next, x1, cta);
      ok = __all_sync(0xffffffffu, wait(p, o_full, seg & 1, s_abort));
      if (!ok) break;
      tc_fence_after();
      if (work) {
        const int64_t at = s.slot * (s.prefix ? kRows : p.rows.own_rows) + row;
        float* o = (s.prefix ? p.p_o : p.o_o) + at * DK;
        if (kOnes<DK>) {
          uint32_t x[16];
          tmem_ld16_issue(lanes + kTmemO + DK, x);
          tmem_ld_wait();
          reg_pin(x);
          r.rl = __uint_as_float(x[0]);
        }
        if (mine) (s.prefix ? p.p_ml : p.o_ml)[at] = make_float4(r.ref, r.l, r.rl, 0.f);
#pragma unroll 1
        for (int i = 0; i < DK / 32; ++i) {
          uint32_t v[32];
          tmem_ld32(lanes + kTmemO + 32 * i, v);
          reg_pin(v);
          if (mine) {
#pragma unroll
            for (int e = 0; e < 4; ++e) store8(o + 32 * i + 8 * e, &v[8 * e]);
          }
        }
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(o_empty);
      if (threadIdx.x == 0) {
        // (the unit: prefix units are numbered first)
        const int64_t u = s.slot - cta + (s.prefix ? 0 : p.Hkv * p.rows.prefix_units);
        if (s.j0 == 0) p.unit_ctas[u].x = cta;
        if (s.j0 + s.count == s.nt) p.unit_ctas[u].y = cta;
      }
    }
    if (!ok) {
      *s_abort = 1;
      atomicExch(p.err, kErrMbarTimeout);
    }
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp == 5) tmem_dealloc(tmem, kTmemCols);
}

// ---- merging ------------------------------------------------------------------
// A lane has E consecutive elements of a row, from l * E on.
template <int E>
__device__ __forceinline__ void load_raw(const void* base, int64_t at, int D, int l, uint32_t (&w)[E / 2]) {
  const uint16_t* p = static_cast<const uint16_t*>(base) + at + l * E;
#pragma unroll
  for (int i = 0; i < E / 2; ++i) w[i] = 0u;
  if (l * E < D) {                         // (D is a multiple of 8)
    if constexpr (E == 8) {
      const uint4 u = __ldg(reinterpret_cast<const uint4*>(p));
      w[0] = u.x, w[1] = u.y, w[2] = u.z, w[3] = u.w;
    } else if constexpr (E == 4) {
      const uint2 u = __ldg(reinterpret_cast<const uint2*>(p));
      w[0] = u.x, w[1] = u.y;
    } else {
      w[0] = __ldg(reinterpret_cast<const uint32_t*>(p));
    }
  }
}

// A running result: sum over V and sum of exponentials, both relative to 2^m.
template <int E> struct Part {
  float m, l, r, o[E];      // r: the sum that o is divided by
  __device__ __forceinline__ void rebase(float to) {       // to >= m
    const float a = m == -INFINITY ? 0.f : ex2(m - to);
    if (m != -INFINITY) {
      l *= a;
      r *= a;
#pragma unroll
      for (int i = 0; i < E; ++i) o[i] *= a;
    }
    m = to;
  }
};

// W warps of a CTA; per query row WPR of them, each with its share of the row's
// partial results and of its last entries, or where there are many rows half a
// one.  Two rounds of loads: what the shares are, and what they hold.
template <int DK, int W, int WPR> constexpr int kCombineCtas = WPR == 1 ? 5 : (DK == 64 ? 24 : 16) / W;   // per SM
template <int DK, bool BF16, int W, int WPR>
__global__ void __launch_bounds__(32 * W, kCombineCtas<DK, W, WPR>) combine_kernel(const __grid_constant__ AttnParams p) {
  constexpr int L = WPR > 1 ? 32 : 16, E = DK / L;             // lanes of a row, elements of a lane
  constexpr int kBatch = WPR > 1 ? 8 : 16 / E, kLast = WPR > 1 ? 4 : 2;    // results and last entries on their way
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, l = lane % L, sub = warp % WPR;
  // over the lanes of a row; of the rows of a warp the larger
  const auto row_max = [](float x) {
#pragma unroll
    for (int d = L / 2; d >= 1; d >>= 1) x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, d));
    return x;
  };
  const auto row_sum = [](float x) {
#pragma unroll
    for (int d = L / 2; d >= 1; d >>= 1) x += __shfl_xor_sync(0xffffffffu, x, d);
    return x;
  };
  const auto larger = [](int x) { return L == 32 ? x : max(x, __shfl_xor_sync(0xffffffffu, x, 16)); };
  pdl_launch_dependents();
  pdl_wait();
  const uint32_t id = (blockIdx.x * (W / WPR) + warp / WPR) * (32 / L) + lane / L;     // (b, h, row)
  const bool real = id < (uint32_t)(p.c.B * p.Hkv * p.R);
  Part<E> a;
  a.m = -INFINITY;
  a.l = a.r = 0.f;
#pragma unroll
  for (int i = 0; i < E; ++i) a.o[i] = 0.f;
  const uint32_t bh = real ? id / (uint32_t)p.R : 0;
  const int rr = real ? id - bh * p.R : 0, b = bh / (uint32_t)p.Hkv, h = bh - b * p.Hkv;
  const int t = (uint32_t)rr / (uint32_t)p.G, g = rr - t * p.G, hq = h * p.G + g;
  {
    const Rows& rw = p.rows;
    int m = 0, ro = rr;                                        // tile of the sequence, row of the tile
    if (rw.per_seq > 1) {
      m = t / rw.tokens * rw.head_tiles + g / rw.heads;
      ro = (t % rw.tokens) * p.G + g % rw.heads;
    }
    const int group = (uint32_t)b / (uint32_t)rw.seqs;
    const int up = h * rw.prefix_units + group * rw.per_seq + m, prefix_units = p.Hkv * rw.prefix_units;
    const int64_t uo = (int64_t)(b * p.Hkv + h) * rw.own_units + m;
    const int n = real ? used(p, b) : 0;
    Results cp = {0, -1}, co = {0, -1};                        // of the row's prefix unit, of its own one
    const auto noted = [&](int64_t unit) {
      const int2 x = __ldcg(p.unit_ctas + unit);
      return noted_results(x.x, x.y, p.grid);
    };
    if (real && p.nt_prefix > 0) cp = noted(up);
    if (n > p.c.T - 1) co = noted(prefix_units + uo);
    const int np = cp.count(), no = co.count();
    const int64_t at_p = (int64_t)(cp.first + up) * kRows + (b - group * rw.seqs) * p.R + ro;
    const int64_t at_o = (co.first + uo) * rw.own_rows + ro;
    // the last T - 1 own entries, of which this row sees the first few: j_first
    // on, this warp every WPR-th, the first kLast on their way from here
    const int far = n - (p.c.T - 1 - t), j_first = p.c.T > 1 ? max(0, n - (p.c.T - 1)) + sub : n;
    uint32_t qw[E / 2], kw[kLast][E / 2], vw[kLast][E / 2];
    const auto fetch = [&](int j0) {
#pragma unroll
      for (int i = 0; i < kLast; ++i) {
        const int64_t j = j0 + i * WPR;
        if (j < far) {
          load_raw<E>(p.c.k, b * p.c.k_batch + j * p.c.k_entry + h * p.c.k_head, p.D, l, kw[i]);
          load_raw<E>(p.c.v, b * p.c.v_batch + j * p.c.v_entry + h * p.c.v_head, p.D, l, vw[i]);
        }
      }
    };
    if (j_first < n) {
      load_raw<E>(p.c.q, b * p.c.q_batch + t * p.c.q_token + hq * p.c.q_head, p.D, l, qw);
      fetch(j_first);
    }
    const auto [begin, end] = share_of(np + no, sub, WPR);
    const int most = larger(end - begin);
    for (int e0 = 0; e0 < most; e0 += L) {
      const int s0 = begin + e0, s = s0 + l, some = min(L, end - s0);
      const auto row_of = [&](int i) {                         // of result i
        return i < np ? at_p + (int64_t)i * kRows : at_o + (int64_t)(i - np) * rw.own_rows;
      };
      float4 ml = make_float4(0.f, 0.f, 0.f, 0.f);
      if (l < some) ml = __ldcg((s < np ? p.p_ml : p.o_ml) + row_of(s));
      float o[kBatch][E];
      const auto load = [&](int i0) {
#pragma unroll
        for (int i = 0; i < kBatch; ++i)
          if (i0 + i < some) {
            const int si = s0 + i0 + i;
            const float* from = (si < np ? p.p_o : p.o_o) + row_of(si) * DK + l * E;
            if constexpr (E == 2) {
              const float2 f = __ldcg(reinterpret_cast<const float2*>(from));
              o[i][0] = f.x, o[i][1] = f.y;
            } else {
#pragma unroll
              for (int e = 0; e < E; e += 4) {
                const float4 f = __ldcg(reinterpret_cast<const float4*>(from + e));
                o[i][e] = f.x, o[i][e + 1] = f.y, o[i][e + 2] = f.z, o[i][e + 3] = f.w;
              }
            }
          }
      };
      load(0);
      const float mi = ml.y == 0.f ? -INFINITY : ml.x;         // (a NaN sum stays in)
      const float top = row_max(mi);
      if (top > a.m) a.rebase(top);
      const float w = mi == -INFINITY ? 0.f : ex2(mi - a.m);
      a.l += row_sum(mi == -INFINITY ? 0.f : w * ml.y);
      a.r += row_sum(mi == -INFINITY ? 0.f : w * ml.z);
      for (int i0 = 0; i0 < min(L, most - e0); i0 += kBatch) {
        if (i0 > 0) load(i0);
#pragma unroll
        for (int i = 0; i < kBatch; ++i) {
          // (a result without weight too: what it has of NaN stays)
          const float wi = __shfl_sync(0xffffffffu, w, lane - l + i0 + i);
          if (i0 + i < some) {
#pragma unroll
            for (int e = 0; e < E; ++e) a.o[e] = fmaf(wi, o[i][e], a.o[e]);
          }
        }
      }
    }
    const int last = larger(n - j_first);
    for (int e0 = 0; e0 < last; e0 += kLast * WPR) {
      if (e0 > 0) fetch(j_first + e0);
#pragma unroll
      for (int i = 0; i < kLast; ++i) {
        const int j = j_first + e0 + i * WPR;
        float s = 0.f;
        if (j < far) {
#pragma unroll
          for (int e = 0; e < E / 2; ++e) {
            const float2 x = unpack2<BF16>(qw[e]), y = unpack2<BF16>(kw[i][e]);
            s = fmaf(x.x, y.x, fmaf(x.y, y.y, s));
          }
        }
        s = row_sum(s);
        if (j < far) {
          const float x = s * p.c2;
          if (x > a.m) a.rebase(x);
          const float w = ex2(fmaf(s, p.c2, a.m == -INFINITY ? 0.f : -a.m));
          a.l += w;
          a.r += w;
#pragma unroll
          for (int e = 0; e < E / 2; ++e) {
            const float2 v = unpack2<BF16>(vw[i][e]);
            a.o[2 * e] = fmaf(w, v.x, a.o[2 * e]);
            a.o[2 * e + 1] = fmaf(w, v.y, a.o[2 * e + 1]);
          }
          if (a.m == -INFINITY && w != 0.f) a.m = 0.f;      // (a NaN score)
        } else {
          s = -INFINITY;
        }
        if (p.scores && l == 0 && j < n)
          p.scores[((((int64_t)b * p.Hkv + h) * p.nt_cap + j / kTile) * p.R + rr) * kTile + j % kTile] = s;
      }
    }
  }
  if constexpr (WPR > 1) {
    __shared__ float s_ml[W][3], s_o[W][DK];
#pragma unroll
    for (int e = 0; e < E; ++e) s_o[warp][lane * E + e] = a.o[e];
    if (lane == 0) {
      s_ml[warp][0] = a.m;
      s_ml[warp][1] = a.l;
      s_ml[warp][2] = a.r;
    }
    __syncthreads();
    if (sub != 0) return;
    for (int w = 1; w < WPR; ++w) {
      const float m = s_ml[warp + w][0];
      if (m > a.m) a.rebase(m);
      const float x = m == -INFINITY ? 0.f : ex2(m - a.m);
      a.l = fmaf(x, s_ml[warp + w][1], a.l);
      a.r = fmaf(x, s_ml[warp + w][2], a.r);
#pragma unroll
      for (int e = 0; e < E; ++e) a.o[e] = fmaf(x, s_o[warp + w][lane * E + e], a.o[e]);
    }
  }
  if (!real) return;
  const bool empty = a.l == 0.f;
  const float inv = empty ? 0.f : 1.f / a.r;
  if (l * E < p.D) {
    uint16_t* out = static_cast<uint16_t*>(p.c.out) + b * p.c.out_batch + t * p.c.out_token + hq * p.c.out_head + l * E;
    uint32_t w[E / 2];
#pragma unroll
    for (int i = 0; i < E / 2; ++i)
      w[i] = empty ? 0u : pack2<BF16>(a.o[2 * i] * inv, a.o[2 * i + 1] * inv);
    if constexpr (E == 8) *reinterpret_cast<uint4*>(out) = make_uint4(w[0], w[1], w[2], w[3]);
    else if constexpr (E == 4) *reinterpret_cast<uint2*>(out) = make_uint2(w[0], w[1]);
    else *reinterpret_cast<uint32_t*>(out) = w[0];
  }
  if (l == 0) {
    const float l2 = a.m + log2f(a.l);
    if (p.c.lse) p.c.lse[((int64_t)b * p.c.T + t) * p.Hq + hq] = empty ? -INFINITY : l2 * kLn2;
    if (p.scores) p.lse2[id] = empty ? INFINITY : l2;
  }
}

// Eight tiles per CTA, one thread per four entries: the scores of their rows, a
// few rows' on their way at a time, added up.
constexpr int kWeightThreads = 128, kWeightEntries = 4 * kWeightThreads;
__global__ void __launch_bounds__(kWeightThreads) weights_kernel(const __grid_constant__ AttnParams p) {
  constexpr int kBatch = 8;
  pdl_launch_dependents();
  pdl_wait();
  for (int bh = blockIdx.y; bh < p.c.B * p.Hkv; bh += gridDim.y) {   // (more than 65535 heads)
    const int b = bh / p.Hkv, h = bh - b * p.Hkv, n = used(p, b);
    const float* lse2 = p.lse2 + (int64_t)bh * p.R;
    const int j = blockIdx.x * kWeightEntries + 4 * threadIdx.x;
    if (j < n) {
      const float* s = p.scores + ((int64_t)bh * p.nt_cap + j / kTile) * p.R * kTile + j % kTile;
      float* w = p.c.weights + b * p.c.weights_batch + h * p.c.weights_head + j;
      float sum[4] = {}, had[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) had[e] = j + e < n ? w[e] : 0.f;
      for (int r0 = 0; r0 < p.R; r0 += kBatch) {
        float4 x[kBatch];
        float l[kBatch];
#pragma unroll
        for (int i = 0; i < kBatch; ++i)
          if (r0 + i < p.R) {
            x[i] = __ldcg(reinterpret_cast<const float4*>(s + (int64_t)(r0 + i) * kTile));
            l[i] = __ldcg(lse2 + r0 + i);
          }
#pragma unroll
        for (int i = 0; i < kBatch; ++i)
          if (r0 + i < p.R) {
            const float v[4] = {x[i].x, x[i].y, x[i].z, x[i].w};
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if (v[e] != -INFINITY) sum[e] += ex2(fmaf(v[e], p.c2, -l[i]));
          }
      }
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (j + e < n) w[e] = had[e] + sum[e];
    }
  }
}

// ---- host ---------------------------------------------------------------------
PFN_cuTensorMapEncodeTiled_v12000 get_encode() {
  static const PFN_cuTensorMapEncodeTiled_v12000 fn = []() -> PFN_cuTensorMapEncodeTiled_v12000 {
    void* f = nullptr;
    cudaDriverEntryPointQueryResult q;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &f, 12000, cudaEnableDefault, &q) != cudaSuccess ||
        q != cudaDriverEntryPointSuccess)
      return nullptr;
    return reinterpret_cast<PFN_cuTensorMapEncodeTiled_v12000>(f);
  }();
  return fn;
}

// Rows of D 16-bit elements over three outer dimensions, in boxes of 64 elements
// x `box`, zero past the extents.  A dimension of size 1 has no stride.
bool encode(CUtensorMap* map, bool bf16, const void* base, int D, const int64_t (&n)[3], const int64_t (&stride)[3],
            const int (&box)[3]) {
  const auto enc = get_encode();
  if (!enc) return false;
  cuuint64_t dims[4] = {(cuuint64_t)D}, bytes[3];
  cuuint32_t boxes[4] = {64}, ones[4] = {1, 1, 1, 1};
  for (int i = 0; i < 3; ++i) {
    dims[i + 1] = (cuuint64_t)n[i];
    bytes[i] = (cuuint64_t)(n[i] > 1 ? 2 * stride[i] : 2 * (int64_t)D);
    boxes[i + 1] = (cuuint32_t)box[i];
  }
  return enc(map, bf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 4,
             const_cast<void*>(base), dims, bytes, boxes, ones, CU_TENSOR_MAP_INTERLEAVE_NONE,
             CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
             CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// The same for a cache [batch][entry][head][D], in boxes of a tile of entries;
// with rows of two whole blocks of 64 elements the block is a dimension (after
// the entries), and a box has both.
bool encode_kv(CUtensorMap* map, bool bf16, const void* base, int D, const int64_t (&n)[3], const int64_t (&stride)[3]) {
  if (D != 128) return encode(map, bf16, base, D, n, stride, {kTile, 1, 1});
  const auto enc = get_encode();
  if (!enc) return false;
  const auto bytes = [&](int i) { return (cuuint64_t)(n[i] > 1 ? 2 * stride[i] : 2 * (int64_t)D); };
  const cuuint64_t dims[5] = {64, (cuuint64_t)n[0], 2, (cuuint64_t)n[1], (cuuint64_t)n[2]};
  const cuuint64_t strides[4] = {bytes(0), 128, bytes(1), bytes(2)};
  const cuuint32_t box[5] = {64, kTile, 2, 1, 1}, ones[5] = {1, 1, 1, 1, 1};
  return enc(map, bf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 5,
             const_cast<void*>(base), dims, strides, box, ones, CU_TENSOR_MAP_INTERLEAVE_NONE,
             CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
             CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int DK>
constexpr size_t attend_smem() {
  return kQBytes<DK> + (size_t)(kStagesK<DK> + kStagesV<DK>) * kTileBytes<DK> + (kOnes<DK> ? kBlock : 0) +
         (2 * kStagesK<DK> + 2 * kStagesV<DK> + 11) * 8 + 8 + 32 + (kGroups + 1) * 4;
}

static_assert(2 * (attend_smem<128>() + 1024) <= 228 * 1024 && 2 * (attend_smem<64>() + 1024) <= 228 * 1024, "two CTAs per SM");

template <int DK, bool BF16>
cudaError_t launch_attend_t(const AttnParams& p, const AttnMaps& maps, int dev, cudaStream_t s) {
  static PerDevice attr;
  cudaError_t e = attr.once(dev, []() {
    return cudaFuncSetAttribute(attend_kernel<DK, BF16>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                (int)attend_smem<DK>());
  });
  if (e != cudaSuccess) return e;
  e = launch_pdl(attend_kernel<DK, BF16>, dim3((unsigned)p.grid), dim3(kAttThreads), attend_smem<DK>(), s, maps, p);
  if (e != cudaSuccess) return e;
  const int64_t rows = (int64_t)p.c.B * p.Hkv * p.R;
  // Warps per row by the rows, and by the partial results that a row has if every
  // own cache is full.  us a call with 8 / 2 / 1: 64 chats (768 rows of 3 results)
  // 32.2 / 27.3 / 28.1, 19 sequences of 6 tokens (1824 of 15) 119 / 110 / 113, a
  // document (192 of 71) 54 / 59 / 66, 30 sequences of one token (240 of 147) 25 / 34 /
  // 50; 32 drafting sequences (3840 of 5) with 2 / 1 51.1 / 49.7, 128 (10240) 162 / 144;
  // many rows with 1 / a half: 128 drafting sequences 141 / 138, 128 of 196 entries 49.6 /
  // 47.1.
  const int64_t nt = p.nt_prefix + p.nt_cap;
  const int64_t tiles = p.Hkv * ((int64_t)p.rows.prefix_units * p.nt_prefix + (int64_t)p.c.B * p.rows.own_units * p.nt_cap);
  if (rows <= p.grid || (rows <= 2048 && p.grid * nt >= 24 * tiles))
    e = launch_pdl(combine_kernel<DK, BF16, 8, 8>, dim3((unsigned)rows), dim3(256), 0, s, p);
  else if (rows <= 2048)
    e = launch_pdl(combine_kernel<DK, BF16, 4, 2>, dim3((unsigned)((rows + 1) / 2)), dim3(128), 0, s, p);
  else
    e = launch_pdl(combine_kernel<DK, BF16, 4, 1>, dim3((unsigned)((rows + 7) / 8)), dim3(128), 0, s, p);
  if (e != cudaSuccess || !p.c.weights) return e;
  return launch_pdl(weights_kernel, dim3((unsigned)ceil_div(p.capacity, kWeightEntries), (unsigned)min(p.c.B * p.Hkv, 65535)),
                    dim3(kWeightThreads), 0, s, p);
}

Rows rows_of(int B, int T, int G) {
  Rows r;
  r.heads = min(G, kRows);
  r.head_tiles = ceil_div(G, kRows);
  r.tokens = r.head_tiles > 1 ? 1 : min(T, kRows / G);
  r.per_seq = ceil_div(T, r.tokens) * r.head_tiles;
  r.seqs = r.per_seq > 1 ? 1 : min(B, kRows / (T * G));
  r.own_units = r.per_seq;
  r.prefix_units = ceil_div(B, r.seqs) * r.per_seq;
  r.own_rows = r.heads * r.tokens;
  r.prefix_rows = r.own_rows * r.seqs;
  return r;
}

size_t round256(size_t n) { return (n + 255) / 256 * 256; }

// The workspace's parts, for calls of B sequences and T query tokens.
struct Parts {
  size_t units, lse2, p_ml, p_o, o_ml, o_o, scores, end;
};
Parts parts_of(const CacheShape& s, int B, int T, int grid) {
  const int G = s.Hq / s.Hkv, R = T * G, DK = s.D <= 64 ? 64 : 128;
  const Rows r = rows_of(B, T, G);
  const size_t p_slots = (size_t)grid + (size_t)s.Hkv * r.prefix_units;
  const size_t o_rows = ((size_t)grid + (size_t)B * s.Hkv * r.own_units) * r.own_rows;
  Parts w;
  w.units = 0;
  w.lse2 = round256(((size_t)s.Hkv * r.prefix_units + (size_t)B * s.Hkv * r.own_units) * 8);
  w.p_ml = w.lse2 + round256((size_t)B * s.Hkv * R * 4);
  w.p_o = w.p_ml + p_slots * kRows * 16;
  w.o_ml = w.p_o + p_slots * kRows * DK * 4;
  w.o_o = w.o_ml + round256(o_rows * 16);
  w.scores = w.o_o + round256(o_rows * DK * 4);
  w.end = w.scores + (s.weights ? (size_t)B * s.Hkv * ceil_div(s.capacity, kTile) * R * kTile * 4 : 0);
  return w;
}

}  // namespace

CacheWorkspace cache_workspace(const CacheShape& s, int sms) {
  CacheWorkspace w;
  // (the rows of a unit, and with them its parts, do not only grow with T)
  size_t most = 0;
  for (int T = 1; T <= s.max_T; ++T) most = max(most, parts_of(s, s.max_batch, T, 2 * sms).end);
  w.moves = round256(most);
  w.counts = w.moves + round256((size_t)s.max_batch * s.Hkv * (s.capacity / 2) * 8);
  w.bytes = w.counts + (size_t)s.max_batch * s.Hkv * 4;
  return w;
}

int64_t attend_tiles(const CacheShape& s, const sp_attend& c) {
  const Rows r = rows_of(c.B, c.T, s.Hq / s.Hkv);
  return s.Hkv * ((int64_t)r.prefix_units * ceil_div(c.prefix_len, kTile) +
                  (int64_t)c.B * r.own_units * ceil_div(s.capacity, kTile));
}

cudaError_t launch_attend(const CacheShape& s, const sp_attend& c, uint8_t* ws, int* err, int fault,
                          cudaStream_t stream) {
  int dev = 0, sms = 0;
  const cudaError_t e = current_device(&dev, &sms);
  if (e != cudaSuccess) return e;
  AttnParams p;
  p.c = c;
  p.Hq = s.Hq;
  p.Hkv = s.Hkv;
  p.G = s.Hq / s.Hkv;
  p.D = s.D;
  p.capacity = s.capacity;
  p.R = c.T * p.G;
  p.rows = rows_of(c.B, c.T, p.G);
  // A unit costs its rows' copy and its result about what three or four tiles do,
  // and own tiles come from memory where the prefix's are found in L2.  us a call
  // with (4, 6, 4, 6) / (8, 6, 8, 7) / these: 128 drafting sequences on 16384 entries
  // 158 / 150 / 146, 32 with 64-wide heads 56 / 52 / 50, 64 chats 39 / 36 / 35, 34
  // sequences of 18 to 54 entries on 73566 42 / 35 / 30.
  p.costs = Costs{24, 6, 20, 7};
  p.nt_prefix = ceil_div(c.prefix_len, kTile);
  p.nt_cap = ceil_div(s.capacity, kTile);
  p.c2 = c.scale * kLog2e;
  p.whole_rows = s.D == 128;
  p.err = err;
  p.fault = fault;
  p.limit = fault == kFaultStall ? kStallWaitCycles : kWaitLimitCycles;
  p.grid = 2 * sms;
  const Parts w = parts_of(s, c.B, c.T, p.grid);
  p.unit_ctas = reinterpret_cast<int2*>(ws + w.units);
  p.lse2 = reinterpret_cast<float*>(ws + w.lse2);
  p.p_ml = reinterpret_cast<float4*>(ws + w.p_ml);
  p.p_o = reinterpret_cast<float*>(ws + w.p_o);
  p.o_ml = reinterpret_cast<float4*>(ws + w.o_ml);
  p.o_o = reinterpret_cast<float*>(ws + w.o_o);
  p.scores = c.weights ? reinterpret_cast<float*>(ws + w.scores) : nullptr;
  const bool bf16 = s.dtype == SP_BF16;
  const Rows& r = p.rows;
  AttnMaps maps;
  const int64_t nq[3] = {s.Hq, c.T, c.B}, sq[3] = {c.q_head, c.q_token, c.q_batch};
  const int64_t nk[3] = {s.capacity, s.Hkv, c.B};
  if (!encode(&maps.q, bf16, c.q, s.D, nq, sq, {r.heads, r.tokens, 1}) ||
      !encode(&maps.pq, bf16, c.q, s.D, nq, sq, {r.heads, r.tokens, r.seqs}) ||
      !encode_kv(&maps.k, bf16, c.k, s.D, nk, {c.k_entry, c.k_head, c.k_batch}) ||
      !encode_kv(&maps.v, bf16, c.v, s.D, nk, {c.v_entry, c.v_head, c.v_batch}))
    return cudaErrorInvalidValue;
  if (c.prefix_len == 0) {
    maps.pk = maps.k;                      // (read by nothing)
    maps.pv = maps.v;
  } else {
    const int64_t np[3] = {c.prefix_len, s.Hkv, 1};
    if (!encode_kv(&maps.pk, bf16, c.prefix_k, s.D, np, {c.pk_entry, c.pk_head, 0}) ||
        !encode_kv(&maps.pv, bf16, c.prefix_v, s.D, np, {c.pv_entry, c.pv_head, 0}))
      return cudaErrorInvalidValue;
  }
  if (s.D <= 64)
    return bf16 ? launch_attend_t<64, true>(p, maps, dev, stream)
                : launch_attend_t<64, false>(p, maps, dev, stream);
  return bf16 ? launch_attend_t<128, true>(p, maps, dev, stream)
              : launch_attend_t<128, false>(p, maps, dev, stream);
}

}  // namespace sp
