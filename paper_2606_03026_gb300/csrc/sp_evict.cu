// sp_evict.cu -- eviction from the sequences' own caches by accumulated
// attention weight (see spike_proj_cache_evict).  Of the n entries of one
// sequence and K/V head the `budget` first in the order (newest, weight
// descending, slot ascending) are kept; the kept ones from slot `budget` on
// move into the slots below it that others leave, so that no row is read and
// written in one call and nothing moves that can stay.
//
// One thread-block cluster per (sequence, head); its CTAs take contiguous
// ranges of slots, their warps contiguous spans.  The order's place of each
// entry is one 32-bit key: the weight's bits made monotone, above them NaN,
// above all the newest entries.  The budget-th largest key is found by digits,
// high ones first, from histograms that the CTAs of the cluster add up; ties at
// it go by slot.  Then counts and ranks of the slots that are left and of the
// entries that move make a list of moves, and the cluster's warps share it.
#include <math.h>

#include "sp_cache.h"
#include "sp_ptx.cuh"

namespace sp {
namespace {

constexpr int kEvThreads = 512;
constexpr int kEvWarps = kEvThreads / 32;
constexpr int kEvBits = 8;
constexpr int kEvBins = 1 << kEvBits;
constexpr int kEvMaxCluster = 8;
constexpr int kEvCached = 20 * 1024;       // keys of a CTA held in shared memory

struct EvictParams {
  sp_evict c;
  int32_t Hkv, capacity, row16, cached;    // 16-byte pieces of a K or V row; keys that fit in shared memory
  int2* moves;                             // [B][Hkv][capacity / 2 + 1]
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

struct Counts {                            // of one CTA, read by its cluster
  uint32_t ties, holes, moved;
};

__global__ void __launch_bounds__(kEvThreads) evict_kernel(const __grid_constant__ EvictParams p) {
  extern __shared__ uint32_t s_keys[];
  __shared__ uint32_t s_hist[2][kEvBins], s_warp[3][kEvWarps], s_pick[3];
  __shared__ Counts s_counts;
  const sp_evict& c = p.c;
  const int t = threadIdx.x, warp = t >> 5, lane = t & 31;
  uint32_t rank, ranks;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
  asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(ranks));
  const int bh = blockIdx.x / ranks, b = bh / p.Hkv, h = bh % p.Hkv;
  pdl_launch_dependents();
  pdl_wait();
  const int n = min(max(__ldg(c.lens + b), 0), p.capacity);
  const float* wt = c.weights + b * c.in_batch + h * c.in_head;
  const int* ps = c.pos + b * c.in_batch + h * c.in_head;
  float* wt_out = c.weights_out + b * c.out_batch + h * c.out_head;
  int* ps_out = c.pos_out + b * c.out_batch + h * c.out_head;
  if (h == 0 && rank == 0 && t == 0) c.lens_out[b] = min(n, c.budget);
  if (n <= c.budget) {
    for (int j = rank * kEvThreads + t; j < n; j += ranks * kEvThreads) {
      wt_out[j] = __ldg(wt + j);
      ps_out[j] = __ldg(ps + j);
    }
    return;
  }
  if (c.budget == 0) return;

  const int64_t newest = (int64_t)__ldg(c.now + b) - c.recent;
  const int per = ceil_div(n, (int)ranks), j0 = min((int)rank * per, n), j1 = min(j0 + per, n);
  const int span = ceil_div(ceil_div(per, kEvWarps), 32) * 32;
  const int w0 = min(j0 + warp * span, j1), w1 = min(w0 + span, j1);
  for (int i = t; i < min(j1 - j0, p.cached); i += kEvThreads) s_keys[i] = key_of(__ldg(wt + j0 + i), __ldg(ps + j0 + i), newest);
  const auto key = [&](int j) {
    return j - j0 < p.cached ? s_keys[j - j0] : key_of(__ldg(wt + j), __ldg(ps + j), newest);
  };

  // The budget-th largest key: `top` its digits found so far, `need` how many
  // of the entries with these digits are kept.
  uint32_t top = 0, need = c.budget;
  int shift = 32, pass = 0;
  bool ties = true;
  while (shift > 0) {
    shift -= kEvBits;
    uint32_t* hist = s_hist[pass & 1];
    for (int i = t; i < kEvBins; i += kEvThreads) hist[i] = 0;
    __syncthreads();
    for (int i = w0 + lane; i < w1; i += 32) {
      const uint32_t k = key(i);
      if (pass == 0 || (k >> (shift + kEvBits)) == top) atomicAdd(&hist[(k >> shift) & (kEvBins - 1)], 1u);
    }
    if (ranks > 1) cluster_sync(); else __syncthreads();
    // thread i has bin kEvBins - 1 - i: entries in it and in higher bins
    uint32_t mine = 0, incl = 0;
    if (t < kEvBins) {
      if (ranks > 1)
        for (uint32_t r = 0; r < ranks; ++r) mine += ld_cluster(cluster_addr(&hist[kEvBins - 1 - t], r));
      else
        mine = hist[kEvBins - 1 - t];
      incl = mine;
#pragma unroll
      for (int d = 1; d < 32; d <<= 1) {
        const uint32_t y = __shfl_up_sync(0xffffffffu, incl, d);
        if (lane >= d) incl += y;
      }
      if (lane == 31) s_warp[0][warp] = incl;
    }
    __syncthreads();
    if (t < kEvBins) {
      for (int w = 0; w < warp; ++w) incl += s_warp[0][w];
      if (incl >= need && incl - mine < need) {
        s_pick[0] = kEvBins - 1 - t;
        s_pick[1] = need - (incl - mine);
        s_pick[2] = mine;
      }
    }
    __syncthreads();
    top = top << kEvBits | s_pick[0];
    need = s_pick[1];
    ++pass;
    if (need == s_pick[2]) {               // every entry with these digits is kept
      ties = false;
      break;
    }
  }

  // Ties at the key go by slot: those before this warp's span.
  uint32_t tie_at = 0;
  if (ties) {
    uint32_t cnt = 0;
    for (int i = w0; i < w1; i += 32) cnt += __popc(__ballot_sync(0xffffffffu, i + lane < w1 && key(i + lane) == top));
    if (lane == 0) s_warp[0][warp] = cnt;
    __syncthreads();
    uint32_t all = 0;
    for (int w = 0; w < kEvWarps; ++w) {
      if (w < warp) tie_at += s_warp[0][w];
      all += s_warp[0][w];
    }
    if (ranks > 1) {
      if (t == 0) s_counts.ties = all;
      cluster_sync();
      for (uint32_t r = 0; r < rank; ++r) tie_at += ld_cluster(cluster_addr(&s_counts.ties, r));
    }
  }
  const auto kept_of = [&](int j, uint32_t& tie) {     // (every lane of the warp together)
    const bool in = j < w1;
    const uint32_t k = in ? key(j) : 0u, d = shift < 32 ? k >> shift : 0u;
    bool kept = in && d > top;
    if (!ties) return kept || (in && d == top);
    const uint32_t eq = __ballot_sync(0xffffffffu, in && d == top);
    if (in && d == top) kept = tie + __popc(eq & ((1u << lane) - 1u)) < need;
    tie += __popc(eq);
    return kept;
  };
  // Slots below the budget that are left, and kept entries behind it.
  uint32_t holes = 0, moved = 0, tie = tie_at;
  for (int i = w0; i < w1; i += 32) {
    const int j = i + lane;
    const bool kept = kept_of(j, tie);
    holes += __popc(__ballot_sync(0xffffffffu, j < w1 && j < c.budget && !kept));
    moved += __popc(__ballot_sync(0xffffffffu, j < w1 && j >= c.budget && kept));
  }
  if (lane == 0) {
    s_warp[1][warp] = holes;
    s_warp[2][warp] = moved;
  }
  __syncthreads();
  uint32_t hole_at = 0, moved_at = 0, all_moved = 0, all_holes = 0;
  for (int w = 0; w < kEvWarps; ++w) {
    if (w < warp) {
      hole_at += s_warp[1][w];
      moved_at += s_warp[2][w];
    }
    all_holes += s_warp[1][w];
    all_moved += s_warp[2][w];
  }
  uint32_t total = all_moved;
  if (ranks > 1) {
    if (t == 0) {
      s_counts.holes = all_holes;
      s_counts.moved = all_moved;
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
  // The list of moves (from, to), and what stays in place.
  int2* moves = p.moves + (int64_t)bh * (p.capacity / 2 + 1);
  tie = tie_at;
  for (int i = w0; i < w1; i += 32) {
    const int j = i + lane;
    const bool kept = kept_of(j, tie), in = j < w1, below = j < c.budget;
    const uint32_t mh = __ballot_sync(0xffffffffu, in && below && !kept);
    const uint32_t mm = __ballot_sync(0xffffffffu, in && !below && kept);
    const uint32_t lower = (1u << lane) - 1u;
    if (in && below && !kept) moves[hole_at + __popc(mh & lower)].y = j;
    if (in && !below && kept) moves[moved_at + __popc(mm & lower)].x = j;
    if (in && below && kept) {
      wt_out[j] = __ldg(wt + j);
      ps_out[j] = __ldg(ps + j);
    }
    hole_at += __popc(mh);
    moved_at += __popc(mm);
  }
  if (ranks > 1) cluster_sync(); else __syncthreads();
  const int64_t kb = b * c.k_batch + h * c.k_head, vb = b * c.v_batch + h * c.v_head;
  uint16_t* K = static_cast<uint16_t*>(c.k) + kb;
  uint16_t* V = static_cast<uint16_t*>(c.v) + vb;
  for (uint32_t i = rank * kEvWarps + warp; i < total; i += ranks * kEvWarps) {
    const int2 m = __ldcg(moves + i);
    for (int e = lane; e < 2 * p.row16; e += 32) {
      const bool is_v = e >= p.row16;
      const int at = 8 * (is_v ? e - p.row16 : e);
      uint16_t* X = is_v ? V : K;
      const int64_t ent = is_v ? c.v_entry : c.k_entry;
      *reinterpret_cast<uint4*>(X + m.y * ent + at) = __ldcg(reinterpret_cast<const uint4*>(X + m.x * ent + at));
    }
    if (lane == 0) {
      wt_out[m.y] = __ldg(wt + m.x);
      ps_out[m.y] = __ldg(ps + m.x);
    }
  }
  if (ranks > 1) cluster_sync();           // no CTA leaves while its counts may be read
}

}  // namespace

cudaError_t launch_evict(const CacheShape& s, const sp_evict& c, uint8_t* ws, cudaStream_t stream) {
  static PerDevice attr_set;
  int dev = 0, sms = 0;
  cudaError_t e = current_device(&dev, &sms);
  if (e != cudaSuccess) return e;
  e = attr_set.once(dev, []() {
    return cudaFuncSetAttribute(evict_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kEvCached * 4);
  });
  if (e != cudaSuccess) return e;
  int cluster = kEvMaxCluster;
  while (cluster > 1 && (c.B * s.Hkv * cluster > 2 * sms || s.capacity < 2048 * cluster)) cluster /= 2;
  EvictParams p;
  p.c = c;
  p.Hkv = s.Hkv;
  p.capacity = s.capacity;
  p.row16 = s.D / 8;
  p.cached = min(ceil_div(s.capacity, cluster), kEvCached);
  p.moves = reinterpret_cast<int2*>(ws + cache_workspace(s, sms).moves);
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(c.B * s.Hkv * cluster), 1, 1);
  cfg.blockDim = dim3(kEvThreads, 1, 1);
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
  return cudaLaunchKernelEx(&cfg, evict_kernel, p);
}

}  // namespace sp
