// sp_verify.cu -- verification of drafted tokens (see spike_proj_verify):
//
//   n     = drafts kept before the first with u_t q_t(x_t) >= p_t(x_t)
//   r_v   = max(p_n(v) - q_n(v), 0)     (p_n alone when every draft is kept)
//   w_v   = rint(min(r_v, 1) 2^36), S = sum w, c = floor(U S / 2^24)
//   token = first v whose running sum of w passes c
//
// The sums are whole numbers in 64 bits, so that they may be split anywhere.
// One thread-block cluster per sequence: its CTAs take contiguous slices of the
// row, their warps contiguous spans of the slice.  A warp streams its span of
// both rows through a ring in shared memory of its own, in pieces of 512 entries
// (bulk copies: all that the ring holds is on its way, 64 KB per CTA), and keeps
// the sums of up to kGroups groups of pieces.  Copies are of whole 16 bytes within
// the row; up to three entries at either end of it are read by themselves, so that
// nothing beside a row is touched.  The spans' sums meet in shared
// memory, the slices' in every CTA's (distributed shared memory).  The CTA whose
// slice the running sum passes c in reads the one group where it does again,
// every thread a few entries of it.
//
// The row of p and the row of q that the token is drawn from have to be read once
// (8 V bytes a sequence; the drafts' own entries are a few sectors), which is what
// bounds it for many sequences: 64 of 57344 entries (25 MB, 3.6 us of memory) take
// 9.6 us (replayed from a graph), 200 of 50001 (65 MB, 9.6 us) 19.7, of which about 5 are the start, the two
// dependent reads that find the row, and the end; 200 CTAs also leave SMs with one
// where others have two.  One sequence takes 5.5 us, all of it latency, in a
// cluster of 16 CTAs.  Rings: 1 row piece of 1024 entries, 6 of 256 and 3 of 512 were
// measured slower (200 sequences 26, 28 and 19.4 us).
#include <math.h>

#include "sp_cache.h"
#include "sp_ptx.cuh"

namespace sp {
namespace {

constexpr int kVerThreads = 256;
constexpr int kVerWarps = kVerThreads / 32;
constexpr int kVerMaxCluster = 16;
constexpr int kVerPerSm = 2;               // CTAs that an SM holds
constexpr int kPiece = 512;                // entries of a bulk copy
constexpr int kPieceBytes = 4 * kPiece + 32;   // and what lies around them in its 16-byte pieces
constexpr int kRing = 2;                   // pieces of each row per warp
constexpr int kGroups = 64;
constexpr size_t kVerSmem = (size_t)kVerWarps * kRing * 2 * kPieceBytes;

struct VerifyParams {
  sp_verify c;
  int32_t slice, span;      // entries of a CTA and of a warp
  int32_t per_group;        // pieces of a group
};

__device__ __forceinline__ float unit(float u) { return fminf(fmaxf(u, 0.f), 0x1.fffffep-1f); }
__device__ __forceinline__ unsigned long long whole(float r) {
  return r > 0.f ? __float2ull_rn(fminf(r, 1.f) * 0x1p36f) : 0ull;
}

// Sum of the whole numbers of entries v0 .. v1 of a warp, the groups' into
// `groups`.  it: pieces that have gone through the ring before; copies: every
// copy so far has arrived.
__device__ __forceinline__ unsigned long long sum_span(const float* pr, const float* qr, int V, int v0, int v1,
                                                       int per_group, uint8_t* ring, uint64_t* full, int& it, bool& copies,
                                                       unsigned long long* groups) {
  const int lane = threadIdx.x & 31;
  const int pieces = ceil_div(max(v1 - v0, 0), kPiece);
  // where the rows begin in their first 16 bytes, and those
  const int p_skip = (int)(reinterpret_cast<uintptr_t>(pr) & 15), q_skip = qr ? (int)(reinterpret_cast<uintptr_t>(qr) & 15) : p_skip;
  const uint8_t *p16 = reinterpret_cast<const uint8_t*>(pr) - p_skip, *q16 = reinterpret_cast<const uint8_t*>(qr) - q_skip;
  // the first piece's 16 bytes, and what a whole one takes
  const int p_base = (p_skip + 4 * v0) & ~15, q_base = (q_skip + 4 * v0) & ~15;
  const int p_bytes = 4 * kPiece + ((p_skip + 4 * v0) & 15 ? 16 : 0), q_bytes = 4 * kPiece + ((q_skip + 4 * v0) & 15 ? 16 : 0);
  const auto fetch = [&](int i, int st) {
    if (lane != 0) return;
    const int v = v0 + i * kPiece, n = min(kPiece, v1 - v);
    uint8_t* to = ring + st * 2 * kPieceBytes;
    if (n == kPiece && v >= 4 && v + kPiece <= V - 4) {
      mbar_arrive_expect_tx(&full[st], p_bytes + (qr ? q_bytes : 0));
      bulk_load(to, p16 + p_base + 4 * kPiece * i, p_bytes, &full[st]);
      if (qr) bulk_load(to + kPieceBytes, q16 + q_base + 4 * kPiece * i, q_bytes, &full[st]);
      return;
    }
    const RowCopy x = row_copy(p_skip, V, v, n);
    RowCopy y = row_copy(q_skip, V, v, n);
    if (!qr) y.bytes = 0;
    mbar_arrive_expect_tx(&full[st], max(x.bytes, 0) + max(y.bytes, 0));
    if (x.bytes > 0) bulk_load(to + (x.from - x.base), p16 + x.from, x.bytes, &full[st]);
    if (y.bytes > 0) bulk_load(to + kPieceBytes + (y.from - y.base), q16 + y.from, y.bytes, &full[st]);
  };
  const auto arrived = [&](int st, uint32_t parity) {
    return __all_sync(0xffffffffu, mbar_try_wait(&full[st], parity) || mbar_wait(&full[st], parity)) != 0;
  };
  // The entries at the rows' ends that are not copied: a lane each, read here and
  // put where the copy would have left them.
  const RowEnds ends = row_ends(p_skip, q_skip, V);
  const int end = lane < ends.lead ? lane : lane >= 32 - ends.trail ? V - 32 + lane : -1;
  float p_end = 0.f, q_end = 0.f;
  if (end >= v0 && end < v1) {
    p_end = __ldg(pr + end);
    if (qr) q_end = __ldg(qr + end);
  }
  const auto use = [&](int i, int st, bool here) {
    const int v = v0 + i * kPiece, n = min(kPiece, v1 - v);
    float* x = reinterpret_cast<float*>(ring + st * 2 * kPieceBytes + ((p_skip + 4 * v) & 15));
    float* y = reinterpret_cast<float*>(ring + st * 2 * kPieceBytes + kPieceBytes + ((q_skip + 4 * v) & 15));
    unsigned long long sum = 0;
    if (!here) {                           // a copy has not arrived in time: the rows themselves
      for (int e = lane; e < n; e += 32) sum += whole(qr ? __ldg(pr + v + e) - __ldg(qr + v + e) : __ldg(pr + v + e));
      return sum;
    }
    if (v < ends.lead || v + n > V - ends.trail) {
      if (end >= v && end < v + n) {
        x[end - v] = p_end;
        y[end - v] = q_end;
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");     // (before another copy there)
      }
      __syncwarp();
    }
    // nearly every number fits 32 bits, whose conversion is several times faster
    float most = 0.f;
    if (n == kPiece) {
#pragma unroll
      for (int e = 0; e < kPiece / 32; ++e) {
        const float r = fmaxf(x[lane + 32 * e] - (qr ? y[lane + 32 * e] : 0.f), 0.f) * 0x1p36f;
        most = fmaxf(most, r);
        sum += __float2uint_rn(r);
      }
    } else {
      most = INFINITY;
    }
    if (most >= 0x1p31f) {
      sum = 0;
      for (int e = lane; e < n; e += 32) sum += whole(x[e] - (qr ? y[e] : 0.f));
    }
    __syncwarp();
    return sum;
  };
  unsigned long long all = 0, group = 0;
  const auto then = [&](int i, unsigned long long sum) {
#pragma unroll
    for (int d = 16; d >= 1; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
    all += sum;
    group += sum;
    if (i % per_group == per_group - 1 || i == pieces - 1) {
      if (lane == 0) groups[i / per_group] = group;
      group = 0;
    }
  };
  copies = walk_ring<kRing>(it, pieces, copies, fetch, arrived, use, then);
  it += pieces;
  return all;
}

__global__ void __launch_bounds__(kVerThreads, kVerPerSm) verify_kernel(const __grid_constant__ VerifyParams p) {
  extern __shared__ __align__(128) uint8_t s_ring[];
  __shared__ __align__(8) uint64_t s_full[kVerWarps][kRing];
  __shared__ int s_bad[2];
  __shared__ unsigned long long s_warp[kVerWarps], s_cta[2][kVerMaxCluster], s_scan[kVerWarps];
  __shared__ unsigned long long s_group[kVerWarps][kGroups];
  const sp_verify& c = p.c;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  uint32_t rank, ranks;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
  asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(ranks));
  const int b = blockIdx.x / ranks;
  if (lane == 0) {
    for (int i = 0; i < kRing; ++i) mbar_init(&s_full[warp][i], 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  __syncwarp();
  int it = 0;
  bool copies = true;
  asm volatile("barrier.cluster.arrive.release;" ::: "memory");
  pdl_launch_dependents();
  pdl_wait();

  // the first draft that is not kept
  const float us = unit(__ldg(c.u_sample + b));
  const int nd = c.n_draft ? min(max(__ldg(c.n_draft + b), 0), c.T) : c.T;
  int x = -1;
  if (warp < 2) {
    const int t = threadIdx.x;
    bool ok = false;
    if (t < c.T) {
      x = __ldg(c.draft + b * c.ld_draft + t);
      const float u = unit(__ldg(c.u + b * c.ld_u + t));
      if (x >= 0 && x < c.V)
        ok = __fmul_rn(u, __ldg(c.q + b * c.q_batch + t * c.q_row + x)) < __ldg(c.p + b * c.p_batch + t * c.p_row + x);
    }
    const uint32_t bad = __ballot_sync(0xffffffffu, !ok);
    if (lane == 0) s_bad[warp] = bad ? 32 * warp + __ffs(bad) - 1 : 64;
  }
  __syncthreads();
  const int n = min(min(s_bad[0], s_bad[1]), nd);
  const float* pr = c.p + b * c.p_batch + n * c.p_row;
  const float* qr = n < nd ? c.q + b * c.q_batch + n * c.q_row : nullptr;
  const int v0 = min((int)rank * p.slice + warp * p.span, c.V);
  const int v1 = min(min(v0 + p.span, (int)(rank + 1) * p.slice), c.V);
  asm volatile("barrier.cluster.wait.acquire;" ::: "memory");   // every CTA of the cluster is running
  for (int pass = 0;; ++pass) {
    const unsigned long long sum =
        sum_span(pr, qr, c.V, v0, v1, p.per_group, s_ring + (size_t)warp * kRing * 2 * kPieceBytes, s_full[warp], it, copies,
                 s_group[warp]);
    if (lane == 0) s_warp[warp] = sum;
    __syncthreads();
    if (threadIdx.x < ranks) {
      unsigned long long all = 0;
      for (int w = 0; w < kVerWarps; ++w) all += s_warp[w];
      asm volatile("st.shared::cluster.u64 [%0], %1;" ::"r"(cluster_addr(&s_cta[pass][rank], threadIdx.x)), "l"(all)
                   : "memory");
    }
    cluster_sync();
    // (every CTA has read the drafts and their number, whose places these may be)
    if (pass == 0 && rank == 0 && threadIdx.x <= c.T) {
      if ((int)threadIdx.x != n) c.tokens[b * c.ld_tokens + threadIdx.x] = (int)threadIdx.x < n ? x : -1;
      if (threadIdx.x == 0) c.n_accept[b] = n;
    }
    unsigned long long before = 0, S = 0;
    for (uint32_t r = 0; r < ranks; ++r) {
      if (r < rank) before += s_cta[pass][r];
      S += s_cta[pass][r];
    }
    if (S == 0) {
      if (pass == 0 && qr) {
        qr = nullptr;              // p alone
        continue;
      }
      if (rank == 0 && threadIdx.x == 0) c.tokens[b * c.ld_tokens + n] = -1;
      return;
    }
    const unsigned long long at = __umul64hi((unsigned long long)(us * 0x1p24f) << 40, S);
    if (at < before || at - before >= s_cta[pass][rank]) return;
    // the group of pieces in which the running sum passes c (the whole CTA is here)
    int w = 0, g = 0;
    while (at - before >= s_warp[w]) before += s_warp[w++];
    while (at - before >= s_group[w][g]) before += s_group[w][g++];
    const int w0 = (int)rank * p.slice + w * p.span + g * p.per_group * kPiece;
    const int w1 = min(min(w0 + p.per_group * kPiece, (int)rank * p.slice + (w + 1) * p.span), min((int)(rank + 1) * p.slice, c.V));
    const int each = p.per_group * kPiece / kVerThreads, i0 = w0 + (int)threadIdx.x * each, i1 = min(i0 + each, w1);
    unsigned long long mine = 0;
    for (int i = i0; i < i1; ++i) mine += whole(qr ? __ldg(pr + i) - __ldg(qr + i) : __ldg(pr + i));
    unsigned long long run = mine;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const unsigned long long y = __shfl_up_sync(0xffffffffu, run, d);
      if (lane >= d) run += y;
    }
    if (lane == 31) s_scan[warp] = run;
    __syncthreads();
    run += before - mine;                  // sum of all entries before this thread's
    for (int i = 0; i < warp; ++i) run += s_scan[i];
    if (run <= at && at - run < mine) {
      for (int i = i0;; ++i) {
        const unsigned long long x = whole(qr ? __ldg(pr + i) - __ldg(qr + i) : __ldg(pr + i));
        if (at - run < x) {
          c.tokens[b * c.ld_tokens + n] = i;
          break;
        }
        run += x;
      }
    }
    return;
  }
}

}  // namespace

cudaError_t launch_verify(const sp_verify& c, cudaStream_t stream) {
  int dev = 0, sms = 0;
  cudaError_t e = current_device(&dev, &sms);
  if (e != cudaSuccess) return e;
  static PerDevice set;
  e = set.once(dev, []() {
    const cudaError_t e = cudaFuncSetAttribute(verify_kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
    return e != cudaSuccess ? e : cudaFuncSetAttribute(verify_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kVerSmem);
  });
  if (e != cudaSuccess) return e;
  int cluster = kVerMaxCluster;
  while (cluster > 1 && (c.B * cluster > kVerPerSm * sms || c.V < 1024 * cluster)) cluster /= 2;
  VerifyParams p;
  p.c = c;
  p.slice = ceil_div(c.V, cluster);
  p.span = ceil_div(ceil_div(p.slice, kVerWarps), 64) * 64;
  p.per_group = ceil_div(ceil_div(p.span, kPiece), kGroups);
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(c.B * cluster), 1, 1);
  cfg.blockDim = dim3(kVerThreads, 1, 1);
  cfg.dynamicSmemBytes = kVerSmem;
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
  return cudaLaunchKernelEx(&cfg, verify_kernel, p);
}

}  // namespace sp
