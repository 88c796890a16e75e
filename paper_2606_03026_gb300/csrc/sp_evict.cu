// sp_evict.cu -- eviction from the sequences' own caches by accumulated
// attention weight (see spike_proj_cache_evict).  Of the n entries of one
// sequence and K/V head the `budget` first in the order (newest, weight
// descending, slot ascending) are kept; the kept ones from slot `budget` on
// move into the slots below it that others leave, so that no row is read and
// written in one call and nothing moves that can stay.
//
// One CTA per (sequence, head), or a thread-block cluster where there are few of
// them and their caches are long; its CTAs take contiguous ranges of slots, their
// warps contiguous spans.  The order's place of each entry is one 32-bit key:
// the weight's bits made monotone, above them NaN, above all the newest entries.
// The budget-th largest key is found by digits of 11, 11 and 10 bits, high ones
// first, from histograms that the CTAs of the cluster add up (the first one
// while the keys are made), and ends where every entry that shares the digits
// found is kept; ties at a whole key go by slot.  A CTA that is alone ranks the
// entries of the digits found one against another instead, once they are few.
// Then each warp turns its span into words of kept entries, and counts and
// ranks of the slots that are left and of the entries that move make a list of
// moves.  Few moves are made at once, in pieces of 16 bytes; many by a second
// kernel, whose CTAs take 64 moves each, whatever head they are of.
//
// Weights and pos have to be read once (8 bytes an entry), and what moves copied
// once.  Cutting 16 prompts of 3000 to 16384 entries, 8 heads each, to 4096 reads and
// writes 150 MB, 22 us of memory, in 40 us (replayed from a graph): about 24 us in
// move_kernel, whose rows of 128 bytes lie scattered, and before it the selection, in a
// CTA a chain of latencies (keys 5 us, digits 3.5, kept words and list 4).  64 sequences
// of 2048 to 2056 entries take 7.1 us, one of 1029 4.8: start, keys, one digit, one
// ranking.  The second kernel's grid goes by the moves that budget and capacity allow: up
// to 8 of 8200 entries of 512 heads leave in 26 us where the capacity is 8200, and in 102
// where it is 16384.
#include <math.h>

#include "sp_cache.h"
#include "sp_ptx.cuh"

namespace sp {
namespace {

constexpr int kEvBins = 2048;
constexpr int kCopies = 8;                 // pieces that a thread has on their way
constexpr int kFewMoves = 64;              // of a head, made by the kernel that finds them
constexpr int kMoveBlock = 64;             // of a CTA of the other kernel
constexpr int kMoveThreads = 256;
// Entries ranked one against another at most, in a histogram's place (64 / 256 / 1024:
// 16 prompts of up to 16384 cut to 4096 41.0 / 40.9 / 49.1 us a call, 64 heads of
// 10000 entries 23.2 / 21.3 / 21.3).
constexpr int kRanked = 256;
constexpr int kKeysAhead = 8;              // weights and pos of a thread on their way
constexpr int kEvMaxCluster = 8;
constexpr int kEvCached = 16 * 1024;       // keys of a CTA held in shared memory

struct EvictParams {
  sp_evict c;
  int32_t Hkv, capacity, cached;           // keys that fit in shared memory
  int32_t row16, row16_log2;               // 16-byte pieces of a K or V row; its logarithm, -1 if it is none
  int32_t* moves;                          // [B][Hkv][2][most_moves]: from, to
  int32_t* counts;                         // [B][Hkv], where a second kernel makes the moves; else null
  int32_t most_moves;                      // that a head can have
};

__device__ __forceinline__ uint32_t key_of(float w, int pos, int64_t newest) {
  if (pos >= newest) return 0xffffffffu;
  if (w != w) return 0xff800001u;          // above +infinity (0xff800000)
  const uint32_t u = __float_as_uint(w + 0.f);            // -0 as +0
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

__device__ __forceinline__ uint32_t ld_cluster(uint32_t addr) {
  uint32_t v;
  asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(addr) : "memory");
  return v;
}

__device__ __forceinline__ uint2 ld_cluster2(uint32_t addr) {
  uint2 v;
  asm volatile("ld.shared::cluster.v2.u32 {%0, %1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(addr) : "memory");
  return v;
}

// Of what every warp has left in its element of `of`: the sum over the warps before this one
// and that over all of them.
template <int WARPS> __device__ __forceinline__ uint2 over_warps(const uint32_t* of, int warp, int lane) {
  const uint32_t v = lane < WARPS ? of[lane] : 0u;
  return make_uint2(__reduce_add_sync(0xffffffffu, lane < warp ? v : 0u), __reduce_add_sync(0xffffffffu, v));
}

struct Counts {                            // of one CTA, read by its cluster
  uint32_t ties, holes, moved;
};

// What a move takes along: weight and pos of `count` moves, then the pieces of
// their K and V rows; thread `at` of `stride`, COPIES pieces on their way each.
template <int COPIES, typename Move>
__device__ __forceinline__ void make_moves(const EvictParams& p, int b, int h, uint32_t count, uint32_t at, uint32_t stride,
                                           Move move) {
  const sp_evict& c = p.c;
  const float* wt = c.weights + b * c.in_batch + h * c.in_head;
  const int* ps = c.pos + b * c.in_batch + h * c.in_head;
  float* wt_out = c.weights_out + b * c.out_batch + h * c.out_head;
  int* ps_out = c.pos_out + b * c.out_batch + h * c.out_head;
  uint16_t* K = static_cast<uint16_t*>(c.k) + b * c.k_batch + h * c.k_head;
  uint16_t* V = static_cast<uint16_t*>(c.v) + b * c.v_batch + h * c.v_head;
  for (uint32_t i = at; i < count; i += stride) {
    const int2 m = move(i);
    wt_out[m.y] = __ldg(wt + m.x);
    ps_out[m.y] = __ldg(ps + m.x);
  }
  // (a head has fewer than 2^23 moves of at most 32 pieces)
  const uint32_t pieces = 2 * p.row16, total = count * pieces;
  for (uint32_t e0 = at; e0 < total; e0 += COPIES * stride) {
    uint4 x[COPIES];
    uint16_t* to[COPIES];
#pragma unroll
    for (int i = 0; i < COPIES; ++i) {
      const uint32_t e = e0 + i * stride;
      to[i] = nullptr;
      if (e < total) {
        const uint32_t mv = p.row16_log2 >= 0 ? e >> (p.row16_log2 + 1) : e / pieces;
        uint32_t piece = e - mv * pieces;
        const bool is_v = piece >= (uint32_t)p.row16;
        if (is_v) piece -= p.row16;
        const int2 m = move(mv);
        uint16_t* X = (is_v ? V : K) + 8 * piece;
        const int64_t ent = is_v ? c.v_entry : c.k_entry;
        x[i] = __ldcg(reinterpret_cast<const uint4*>(X + m.x * ent));
        to[i] = X + m.y * ent;
      }
    }
#pragma unroll
    for (int i = 0; i < COPIES; ++i)
      if (to[i]) *reinterpret_cast<uint4*>(to[i]) = x[i];
  }
}

// NT threads, 1024 / NT CTAs per SM.
template <int NT>
__global__ void __launch_bounds__(NT, 1024 / NT) evict_kernel(const __grid_constant__ EvictParams p) {
  constexpr int kWarps = NT / 32, kPer = kEvBins / NT;     // bins of a thread
  extern __shared__ uint32_t s_keys[];
  __shared__ __align__(16) uint32_t s_hist[2][kEvBins];
  __shared__ uint32_t s_warp[3][kWarps], s_pick[3], s_ranked;
  __shared__ Counts s_counts;
  const sp_evict& c = p.c;
  const int t = threadIdx.x, warp = t >> 5, lane = t & 31;
  uint32_t rank, ranks;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
  asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(ranks));
  const int bh = blockIdx.x / ranks, b = bh / p.Hkv, h = bh % p.Hkv;
  for (int i = t; i < kEvBins; i += NT) s_hist[0][i] = 0;
  if (t == 0) s_ranked = 0;
  pdl_launch_dependents();
  pdl_wait();
  const int n = min(max(__ldg(c.lens + b), 0), p.capacity);
  const int64_t newest = (int64_t)__ldg(c.now + b) - c.recent;
  const float* wt = c.weights + b * c.in_batch + h * c.in_head;
  const int* ps = c.pos + b * c.in_batch + h * c.in_head;
  float* wt_out = c.weights_out + b * c.out_batch + h * c.out_head;
  int* ps_out = c.pos_out + b * c.out_batch + h * c.out_head;
  if (h == 0 && rank == 0 && t == 0) c.lens_out[b] = min(n, c.budget);
  const bool stay = n <= c.budget || c.budget == 0;        // nothing moves
  if (p.counts && rank == 0 && t == 0 && stay) p.counts[bh] = 0;
  if (c.budget == 0) return;
  const int per = ceil_div(n, (int)ranks), j0 = min((int)rank * per, n), j1 = min(j0 + per, n);
  const int span = ceil_div(ceil_div(per, kWarps), 32) * 32;
  const int w0 = min(j0 + warp * span, j1), w1 = min(w0 + span, j1);
  __syncthreads();                         // (the histogram is zero)
  // Weight and pos below the budget go out as they are (those of slots that
  // are left are written again with the moves); all of them make keys.
  for (int i = w0 + lane; i < w1; i += 32 * kKeysAhead) {
    float w[kKeysAhead];
    int q[kKeysAhead];
#pragma unroll
    for (int e = 0; e < kKeysAhead; ++e)
      if (i + 32 * e < w1) {
        w[e] = __ldg(wt + i + 32 * e);
        q[e] = __ldg(ps + i + 32 * e);
      }
#pragma unroll
    for (int e = 0; e < kKeysAhead; ++e) {
      const int j = i + 32 * e;
      if (j < w1) {
        const uint32_t k = key_of(w[e], q[e], newest);
        if (j < c.budget) {
          wt_out[j] = w[e];
          ps_out[j] = q[e];
        }
        if (!stay) {
          if (j - j0 < p.cached) s_keys[j - j0] = k;
          atomicAdd(&s_hist[0][k >> 21], 1u);
        }
      }
    }
  }
  if (stay) return;
  const auto key = [&](int j) {
    return j - j0 < p.cached ? s_keys[j - j0] : key_of(__ldg(wt + j), __ldg(ps + j), newest);
  };

  // The budget-th largest key: `top` its digits found so far, `need` how many
  // of the entries with these digits are kept.
  uint32_t top = 0, need = c.budget;
  int shift = 21;
  bool ties = true;
  for (int pass = 0;; ++pass) {
    const uint32_t* hist = s_hist[pass & 1];
    if (ranks > 1) cluster_sync(); else __syncthreads();
    // thread i has the kPer bins below kEvBins - kPer i: entries in them and in
    // higher bins
    const int bin = kEvBins - kPer * (t + 1);
    uint32_t in[kPer] = {}, mine = 0;
    if (ranks > 1) {
#pragma unroll
      for (uint32_t r = 0; r < kEvMaxCluster; ++r)
#pragma unroll
        for (int i = 0; i < kPer / 2; ++i)
          if (r < ranks) {
            const uint2 g = ld_cluster2(cluster_addr(&hist[bin + 2 * i], r));
            in[2 * i] += g.x, in[2 * i + 1] += g.y;
          }
    } else {
#pragma unroll
      for (int i = 0; i < kPer; ++i) in[i] = hist[bin + i];
    }
#pragma unroll
    for (int i = 0; i < kPer; ++i) mine += in[i];
    uint32_t incl = mine;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const uint32_t y = __shfl_up_sync(0xffffffffu, incl, d);
      if (lane >= d) incl += y;
    }
    if (lane == 31) s_warp[0][warp] = incl;
    // the next pass's histogram (that of two passes ago, which every CTA has read)
    for (int i = t; i < kEvBins; i += NT) s_hist[(pass + 1) & 1][i] = 0;
    __syncthreads();
    incl += over_warps<kWarps>(s_warp[0], warp, lane).x;
    if (incl >= need && incl - mine < need) {
      uint32_t over = incl - mine;         // entries in higher bins
      bool found = false;
#pragma unroll
      for (int i = kPer - 1; i >= 0; --i) {
        if (!found && over + in[i] >= need) {
          found = true;
          s_pick[0] = bin + i;
          s_pick[1] = need - over;
          s_pick[2] = in[i];
        }
        over += in[i];
      }
    }
    __syncthreads();
    top = (pass == 0 ? 0u : top << (pass == 1 ? 11 : 10)) | s_pick[0];
    need = s_pick[1];
    const uint32_t share = s_pick[2];      // entries with these digits
    ties = need != share;                  // else all of them are kept
    if (!ties || pass == 2) break;
    if (ranks == 1 && share <= kRanked && n <= p.cached && top < 0xffffffffu >> shift) {
      // few: by key, then slot; the kept ones get a key above the digits, the others 0
      unsigned long long* few = reinterpret_cast<unsigned long long*>(s_hist[(pass + 1) & 1]);
      for (int i = w0 + lane; i < w1; i += 32) {
        const uint32_t k = s_keys[i];
        if (k >> shift == top) few[atomicAdd(&s_ranked, 1u)] = (unsigned long long)k << 32 | (uint32_t)~i;
      }
      __syncthreads();
      for (uint32_t i = t; i < share; i += NT) {
        const unsigned long long x = few[i];
        uint32_t above = 0;
#pragma unroll 4
        for (uint32_t e = 0; e < share; ++e) above += few[e] > x;
        s_keys[~(uint32_t)x] = above < need ? (top + 1) << shift : 0u;
      }
      __syncthreads();
      ties = false;
      break;
    }
    const int next = pass == 0 ? 10 : 0;
    for (int i = w0 + lane; i < w1; i += 32) {
      const uint32_t k = key(i);
      if (k >> shift == top) atomicAdd(&s_hist[(pass + 1) & 1][(k >> next) & (pass == 0 ? 2047u : 1023u)], 1u);
    }
    shift = next;
  }

  // Ties at the key go by slot: those before this warp's span.
  uint32_t tie_at = 0;
  if (ties) {
    uint32_t cnt = 0;
    for (int i = w0; i < w1; i += 32) cnt += __popc(__ballot_sync(0xffffffffu, i + lane < w1 && key(i + lane) == top));
    if (lane == 0) s_warp[0][warp] = cnt;
    __syncthreads();
    const uint2 warps = over_warps<kWarps>(s_warp[0], warp, lane);
    tie_at = warps.x;
    if (ranks > 1) {
      if (t == 0) s_counts.ties = warps.y;
      cluster_sync();
      for (uint32_t r = 0; r < rank; ++r) tie_at += ld_cluster(cluster_addr(&s_counts.ties, r));
    }
  }
  // 32 words of the span: lane i's has a bit for each of the entries from
  // base + 32 i on that are kept.
  const auto kept_words = [&](int base, uint32_t& tie) {
    uint32_t mine = 0;
    const int words = min(32, ceil_div(w1 - base, 32));
    if (!ties && w1 - j0 <= p.cached) {
#pragma unroll 4
      for (int i = 0; i < words; ++i) {
        const int j = base + 32 * i + lane;
        const uint32_t kept = __ballot_sync(0xffffffffu, j < w1 && s_keys[j - j0] >> shift >= top);
        if (lane == i) mine = kept;
      }
      return mine;
    }
    for (int i = 0; i < words; ++i) {
      const int j = base + 32 * i + lane;
      const bool in = j < w1;
      const uint32_t d = in ? key(j) >> shift : 0u;
      uint32_t kept = __ballot_sync(0xffffffffu, in && (d > top || (!ties && d == top)));
      if (ties) {
        uint32_t eq = __ballot_sync(0xffffffffu, in && d == top);
        tie += __popc(eq);
        for (uint32_t cut = tie > need ? tie - need : 0u; cut > 0 && eq; --cut) eq &= ~(0x80000000u >> __clz(eq));
        kept |= eq;
      }
      if (lane == i) mine = kept;
    }
    return mine;
  };
  const auto low = [](int bits) { return bits >= 32 ? 0xffffffffu : bits <= 0 ? 0u : (1u << bits) - 1u; };
  // Slots below the budget that are left, and kept entries behind it.
  uint32_t holes = 0, moved = 0, tie = tie_at, word = 0;
  for (int base = w0; base < w1; base += 1024) {
    word = kept_words(base, tie);
    const int at = base + 32 * lane;
    const uint32_t there = low(w1 - at), below = low(c.budget - at);
    holes += __popc(~word & there & below);
    moved += __popc(word & there & ~below);
  }
  holes = __reduce_add_sync(0xffffffffu, holes);
  moved = __reduce_add_sync(0xffffffffu, moved);
  if (lane == 0) {
    s_warp[1][warp] = holes;
    s_warp[2][warp] = moved;
  }
  __syncthreads();
  const uint2 warp_holes = over_warps<kWarps>(s_warp[1], warp, lane), warp_moved = over_warps<kWarps>(s_warp[2], warp, lane);
  uint32_t hole_at = warp_holes.x, moved_at = warp_moved.x;
  uint32_t total = warp_moved.y;
  if (ranks > 1) {
    if (t == 0) {
      s_counts.holes = warp_holes.y;
      s_counts.moved = warp_moved.y;
    }
    cluster_sync();
    total = 0;
    for (uint32_t r = 0; r < ranks; ++r) {
      const uint32_t m = ld_cluster(cluster_addr(&s_counts.moved, r));
      if (r < rank) {
        hole_at += ld_cluster(cluster_addr(&s_counts.holes, r));
        moved_at += m;
      }
      total += m;
    }
  }
  // The list of moves: in shared memory where this CTA makes them itself, alone.
  const bool here = ranks == 1 && !p.counts;
  int32_t* from = here ? reinterpret_cast<int32_t*>(s_hist[0]) : p.moves + (int64_t)bh * 2 * p.most_moves;
  int32_t* to = from + (here ? kFewMoves : p.most_moves);
  const bool whole = w1 - w0 <= 1024;      // `word` is still the span's
  tie = tie_at;
  for (int base = w0; base < w1; base += 1024) {
    if (!whole) {
      word = kept_words(base, tie);
    }
    const int at = base + 32 * lane;
    const uint32_t there = low(w1 - at), below = low(c.budget - at);
    const uint32_t hole = ~word & there & below, move = word & there & ~below, before = (1u << lane) - 1u;
    const int words = min(32, ceil_div(w1 - base, 32));
#pragma unroll 4
    for (int i = 0; i < words; ++i) {
      const uint32_t hi = __shfl_sync(0xffffffffu, hole, i), mi = __shfl_sync(0xffffffffu, move, i);
      const int j = base + 32 * i + lane;
      if (hi >> lane & 1u) to[hole_at + __popc(hi & before)] = j;
      if (mi >> lane & 1u) from[moved_at + __popc(mi & before)] = j;
      hole_at += __popc(hi);
      moved_at += __popc(mi);
    }
  }
  if (p.counts) {
    if (rank == 0 && t == 0) p.counts[bh] = total;
    if (ranks > 1) cluster_sync();         // no CTA leaves while its counts may be read
    return;
  }
  if (here) {
    const int32_t* list = reinterpret_cast<const int32_t*>(s_hist[0]);
    __syncthreads();
    make_moves<kCopies>(p, b, h, total, t, NT, [&](uint32_t i) { return make_int2(list[i], list[kFewMoves + i]); });
  } else {
    cluster_sync();
    make_moves<kCopies>(p, b, h, total, rank * NT + t, ranks * NT,
                        [&](uint32_t i) { return make_int2(__ldcg(from + i), __ldcg(to + i)); });
  }
}

// CTA (i, bh): moves kMoveBlock i .. of the list of head bh.
__global__ void __launch_bounds__(kMoveThreads, 5) move_kernel(const __grid_constant__ EvictParams p) {
  __shared__ int2 s_moves[kMoveBlock];
  pdl_launch_dependents();
  pdl_wait();
  const uint32_t heads = p.c.B * p.Hkv, bh = blockIdx.x % heads, first = blockIdx.x / heads * kMoveBlock;
  const uint32_t total = __ldcg(p.counts + bh);
  if (first >= total) return;
  const uint32_t count = min((uint32_t)kMoveBlock, total - first);
  if (threadIdx.x < count) {
    const int32_t* from = p.moves + (int64_t)bh * 2 * p.most_moves + first + threadIdx.x;
    s_moves[threadIdx.x] = make_int2(__ldcg(from), __ldcg(from + p.most_moves));
  }
  __syncthreads();
  make_moves<4>(p, bh / p.Hkv, bh % p.Hkv, count, threadIdx.x, kMoveThreads, [&](uint32_t i) { return s_moves[i]; });
}

template <int NT>
cudaError_t launch_evict_t(EvictParams p, int dev, int cluster, cudaStream_t stream) {
  static PerDevice set;
  const cudaError_t e = set.once(dev, []() {
    return cudaFuncSetAttribute(evict_kernel<NT>, cudaFuncAttributeMaxDynamicSharedMemorySize, kEvCached * 4);
  });
  if (e != cudaSuccess) return e;
  p.cached = min(ceil_div(p.capacity, cluster), kEvCached);
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(p.c.B * p.Hkv * cluster), 1, 1);
  cfg.blockDim = dim3(NT, 1, 1);
  cfg.dynamicSmemBytes = (size_t)p.cached * 4;
  cfg.stream = stream;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = cluster;
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  return cudaLaunchKernelEx(&cfg, evict_kernel<NT>, p);
}

}  // namespace

cudaError_t launch_evict(const CacheShape& s, const sp_evict& c, uint8_t* ws, cudaStream_t stream) {
  int dev = 0, sms = 0;
  const cudaError_t e = current_device(&dev, &sms);
  if (e != cudaSuccess) return e;
  EvictParams p;
  p.c = c;
  p.Hkv = s.Hkv;
  p.capacity = s.capacity;
  p.row16 = s.D / 8;
  p.row16_log2 = -1;
  for (int i = 0; i < 8; ++i)
    if (p.row16 == 1 << i) p.row16_log2 = i;
  p.moves = reinterpret_cast<int32_t*>(ws + cache_workspace(s, sms).moves);
  const int heads = c.B * s.Hkv;
  // (n - budget entries go, budget stay: no more moves than the fewer of them)
  p.most_moves = max(0, min(c.budget, s.capacity - c.budget));
  p.counts = p.most_moves > kFewMoves ? reinterpret_cast<int32_t*>(ws + cache_workspace(s, sms).counts) : nullptr;
  // Clusters where four CTAs would find an SM each per head, and 8192 entries:
  // us a call with 1 / 2 / 4 / 8 CTAs: 1 head of 40000 entries 64 / 32 / 15.1 / 15.7,
  // 16 heads of 20000 40 / 29 / 27.8 / 46; beyond, the adding up of histograms costs
  // more than it saves (64 heads of 10000 18.1 / 19.4 / 28).
  // Threads by what fits the SMs in one wave, no more than the entries need: 256 / 512 /
  // 1024: 4 heads of 1029 entries 5.0 / 5.0 / 5.4, 256 heads of 2056 8.9 / 7.3 / 12, 128
  // heads of 16384 54 / 44 / 41.7, 1024 heads of 2000 17.7 / 26 / 44.
  int cluster = 1;
  while (cluster < kEvMaxCluster && 4 * cluster * heads <= sms && s.capacity >= 8192 * cluster) cluster *= 2;
  int nt = heads * cluster > 2 * sms ? 256 : heads * cluster > sms || s.capacity <= 4096 * cluster ? 512 : 1024;
  const cudaError_t r = nt == 1024 ? launch_evict_t<1024>(p, dev, cluster, stream)
                        : nt == 512 ? launch_evict_t<512>(p, dev, cluster, stream)
                                    : launch_evict_t<256>(p, dev, cluster, stream);
  if (r != cudaSuccess || !p.counts) return r;
  const int64_t blocks = (int64_t)heads * ceil_div(p.most_moves, kMoveBlock);
  return launch_pdl(move_kernel, dim3((unsigned)blocks), dim3(kMoveThreads), 0, stream, p);
}

}  // namespace sp
