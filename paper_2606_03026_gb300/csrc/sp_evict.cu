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
// of 11, 11 and 10 bits, high ones first, from histograms that the CTAs of the
// cluster add up (the first one while the keys are made), and ends where every
// entry that shares the digits found is kept; ties at a whole key go by slot.
// Then counts and ranks of the slots that are left and of the entries that move
// make a list of moves, and the cluster's threads copy its rows in pieces of 16
// bytes, kCopies of them on their way per thread.
#include <math.h>

#include "sp_cache.h"
#include "sp_ptx.cuh"

namespace sp {
namespace {

constexpr int kEvThreads = 256;
constexpr int kEvWarps = kEvThreads / 32;
constexpr int kEvBins = 2048;
constexpr int kEvPer = kEvBins / kEvThreads;       // bins of a thread
constexpr int kCopies = 8;
constexpr int kEvMaxCluster = 8;
constexpr int kEvCached = 16 * 1024;       // keys of a CTA held in shared memory

struct EvictParams {
  sp_evict c;
  int32_t Hkv, capacity, cached;           // keys that fit in shared memory
  int32_t row16, row16_log2;               // 16-byte pieces of a K or V row; its logarithm, -1 if it is none
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

__device__ __forceinline__ uint4 ld_cluster4(uint32_t addr) {
  uint4 v;
  asm volatile("ld.shared::cluster.v4.u32 {%0, %1, %2, %3}, [%4];"
               : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
               : "r"(addr)
               : "memory");
  return v;
}

struct Counts {                            // of one CTA, read by its cluster
  uint32_t ties, holes, moved;
};

__global__ void __launch_bounds__(kEvThreads) evict_kernel(const __grid_constant__ EvictParams p) {
  extern __shared__ uint32_t s_keys[];
  __shared__ __align__(16) uint32_t s_hist[2][kEvBins];
  __shared__ uint32_t s_warp[3][kEvWarps], s_pick[3];
  __shared__ Counts s_counts;
  const sp_evict& c = p.c;
  const int t = threadIdx.x, warp = t >> 5, lane = t & 31;
  uint32_t rank, ranks;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
  asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(ranks));
  const int bh = blockIdx.x / ranks, b = bh / p.Hkv, h = bh % p.Hkv;
  for (int i = t; i < kEvBins; i += kEvThreads) s_hist[0][i] = 0;
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
  const auto key = [&](int j) {
    return j - j0 < p.cached ? s_keys[j - j0] : key_of(__ldg(wt + j), __ldg(ps + j), newest);
  };
  __syncthreads();                         // (the histogram is zero)
  for (int i = w0 + lane; i < w1; i += 32 * 4) {
    float w[4];
    int q[4];
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (i + 32 * e < w1) {
        w[e] = __ldg(wt + i + 32 * e);
        q[e] = __ldg(ps + i + 32 * e);
      }
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (i + 32 * e < w1) {
        const uint32_t k = key_of(w[e], q[e], newest);
        if (i + 32 * e - j0 < p.cached) s_keys[i + 32 * e - j0] = k;
        atomicAdd(&s_hist[0][k >> 21], 1u);
      }
  }

  // The budget-th largest key: `top` its digits found so far, `need` how many
  // of the entries with these digits are kept.
  uint32_t top = 0, need = c.budget;
  int shift = 21;
  bool ties = true;
  for (int pass = 0;; ++pass) {
    const uint32_t* hist = s_hist[pass & 1];
    if (ranks > 1) cluster_sync(); else __syncthreads();
    // thread i has the kEvPer bins below kEvBins - kEvPer i: entries in them
    // and in higher bins
    const int bin = kEvBins - kEvPer * (t + 1);
    uint32_t in[kEvPer] = {}, mine = 0;
    for (uint32_t r = 0; r < ranks; ++r) {
#pragma unroll
      for (int i = 0; i < kEvPer / 4; ++i) {
        const uint4 g = ranks > 1 ? ld_cluster4(cluster_addr(&hist[bin + 4 * i], r))
                                  : *reinterpret_cast<const uint4*>(&hist[bin + 4 * i]);
        in[4 * i] += g.x, in[4 * i + 1] += g.y, in[4 * i + 2] += g.z, in[4 * i + 3] += g.w;
      }
    }
#pragma unroll
    for (int i = 0; i < kEvPer; ++i) mine += in[i];
    uint32_t incl = mine;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const uint32_t y = __shfl_up_sync(0xffffffffu, incl, d);
      if (lane >= d) incl += y;
    }
    if (lane == 31) s_warp[0][warp] = incl;
    // the next pass's histogram (that of two passes ago, which every CTA has read)
    for (int i = t; i < kEvBins; i += kEvThreads) s_hist[(pass + 1) & 1][i] = 0;
    __syncthreads();
    for (int w = 0; w < warp; ++w) incl += s_warp[0][w];
    if (incl >= need && incl - mine < need) {
      uint32_t over = incl - mine;         // entries in higher bins
      bool found = false;
#pragma unroll
      for (int i = kEvPer - 1; i >= 0; --i) {
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
    ties = need != s_pick[2];              // else every entry with these digits is kept
    if (!ties || pass == 2) break;
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
    const uint32_t d = in ? key(j) >> shift : 0u;
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
  const uint32_t stride = ranks * kEvThreads, at = rank * kEvThreads + t;
  for (uint32_t i = at; i < total; i += stride) {
    const int2 m = __ldcg(moves + i);
    wt_out[m.y] = __ldg(wt + m.x);
    ps_out[m.y] = __ldg(ps + m.x);
  }
  // (move, piece) pairs: the K row's pieces, then the V row's
  const uint32_t pieces = 2 * p.row16;
  for (uint64_t e0 = at; e0 < (uint64_t)total * pieces; e0 += (uint64_t)kCopies * stride) {
    uint4 x[kCopies];
    uint16_t* to[kCopies];
#pragma unroll
    for (int i = 0; i < kCopies; ++i) {
      const uint64_t e = e0 + (uint64_t)i * stride;
      to[i] = nullptr;
      if (e < (uint64_t)total * pieces) {
        const uint32_t mv = p.row16_log2 >= 0 ? (uint32_t)(e >> (p.row16_log2 + 1)) : (uint32_t)(e / pieces);
        uint32_t piece = (uint32_t)(e - (uint64_t)mv * pieces);
        const bool is_v = piece >= (uint32_t)p.row16;
        if (is_v) piece -= p.row16;
        const int2 m = __ldcg(moves + mv);
        uint16_t* X = (is_v ? V : K) + 8 * piece;
        const int64_t ent = is_v ? c.v_entry : c.k_entry;
        x[i] = __ldcg(reinterpret_cast<const uint4*>(X + m.x * ent));
        to[i] = X + m.y * ent;
      }
    }
#pragma unroll
    for (int i = 0; i < kCopies; ++i)
      if (to[i]) *reinterpret_cast<uint4*>(to[i]) = x[i];
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
  while (cluster > 1 && (c.B * s.Hkv * cluster > 4 * sms || s.capacity < 2048 * cluster)) cluster /= 2;
  EvictParams p;
  p.c = c;
  p.Hkv = s.Hkv;
  p.capacity = s.capacity;
  p.row16 = s.D / 8;
  p.row16_log2 = -1;
  for (int i = 0; i < 8; ++i)
    if (p.row16 == 1 << i) p.row16_log2 = i;
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
