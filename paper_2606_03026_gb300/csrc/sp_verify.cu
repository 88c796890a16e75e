// sp_verify.cu -- verification of drafted tokens (see spike_proj_verify):
//
//   n     = drafts kept before the first with u_t q_t(x_t) >= p_t(x_t)
//   r_v   = max(p_n(v) - q_n(v), 0)     (p_n alone when every draft is kept)
//   w_v   = rint(min(r_v, 1) 2^36), S = sum w, c = floor(U S / 2^24)
//   token = first v whose running sum of w passes c
//
// The sums are whole numbers in 64 bits, so that they may be split anywhere.
// One thread-block cluster per sequence: its CTAs take contiguous slices of the
// row, their warps contiguous spans of the slice.  The spans' sums meet in
// shared memory, the slices' in every CTA's (distributed shared memory), and
// the one warp whose span the running sum passes c in reads that span again.
#include <math.h>

#include "sp_cache.h"
#include "sp_ptx.cuh"

namespace sp {
namespace {

constexpr int kVerThreads = 512;
constexpr int kVerWarps = kVerThreads / 32;
constexpr int kVerMaxCluster = 16;

struct VerifyParams {
  sp_verify c;
  int32_t slice, span;      // entries of a CTA and of a warp
};

__device__ __forceinline__ float unit(float u) { return fminf(fmaxf(u, 0.f), 0x1.fffffep-1f); }
__device__ __forceinline__ unsigned long long whole(float r) {
  return r > 0.f ? __float2ull_rn(fminf(r, 1.f) * 0x1p36f) : 0ull;
}

__global__ void __launch_bounds__(kVerThreads) verify_kernel(const __grid_constant__ VerifyParams p) {
  __shared__ int s_bad[2];
  __shared__ unsigned long long s_warp[kVerWarps], s_cta[2][kVerMaxCluster];
  const sp_verify& c = p.c;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  uint32_t rank, ranks;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
  asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(ranks));
  const int b = blockIdx.x / ranks;
  asm volatile("barrier.cluster.arrive.release;" ::: "memory");
  pdl_launch_dependents();
  pdl_wait();

  // the first draft that is not kept
  const int nd = c.n_draft ? min(max(__ldg(c.n_draft + b), 0), c.T) : c.T;
  if (warp < 2) {
    const int t = threadIdx.x;
    bool ok = false;
    if (t < nd) {
      const int x = __ldg(c.draft + b * c.ld_draft + t);
      if (x >= 0 && x < c.V)
        ok = __fmul_rn(unit(__ldg(c.u + b * c.ld_u + t)), __ldg(c.q + b * c.q_batch + t * c.q_row + x)) <
             __ldg(c.p + b * c.p_batch + t * c.p_row + x);
    }
    const uint32_t bad = __ballot_sync(0xffffffffu, !ok);
    if (lane == 0) s_bad[warp] = bad ? 32 * warp + __ffs(bad) - 1 : 64;
  }
  __syncthreads();
  const int n = min(min(s_bad[0], s_bad[1]), nd);
  if (rank == 0 && threadIdx.x <= c.T) {
    const int t = threadIdx.x;
    if (t < n) c.tokens[b * c.ld_tokens + t] = __ldg(c.draft + b * c.ld_draft + t);
    if (t > n) c.tokens[b * c.ld_tokens + t] = -1;
    if (t == 0) c.n_accept[b] = n;
  }

  const float* pr = c.p + b * c.p_batch + n * c.p_row;
  const float* qr = n < nd ? c.q + b * c.q_batch + n * c.q_row : nullptr;
  const int v0 = min((int)rank * p.slice + warp * p.span, c.V);
  const int v1 = min(min(v0 + p.span, (int)(rank + 1) * p.slice), c.V);
  asm volatile("barrier.cluster.wait.acquire;" ::: "memory");   // every CTA of the cluster is running
  for (int pass = 0;; ++pass) {
    unsigned long long sum = 0;
    for (int v = v0 + lane; v < v1; v += 32) sum += whole(qr ? __ldg(pr + v) - __ldg(qr + v) : __ldg(pr + v));
#pragma unroll
    for (int d = 16; d >= 1; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
    if (lane == 0) s_warp[warp] = sum;
    __syncthreads();
    if (threadIdx.x < ranks) {
      unsigned long long all = 0;
      for (int w = 0; w < kVerWarps; ++w) all += s_warp[w];
      asm volatile("st.shared::cluster.u64 [%0], %1;" ::"r"(cluster_addr(&s_cta[pass][rank], threadIdx.x)), "l"(all)
                   : "memory");
    }
    cluster_sync();
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
    const unsigned long long at = __umul64hi((unsigned long long)(unit(__ldg(c.u_sample + b)) * 0x1p24f) << 40, S);
    for (int w = 0; w < warp; ++w) before += s_warp[w];
    if (at < before || at - before >= s_warp[warp]) return;
    for (int v = v0; v < v1; v += 32) {
      const int i = v + lane;
      unsigned long long x = i < v1 ? whole(qr ? __ldg(pr + i) - __ldg(qr + i) : __ldg(pr + i)) : 0ull;
#pragma unroll
      for (int d = 1; d < 32; d <<= 1) {
        const unsigned long long y = __shfl_up_sync(0xffffffffu, x, d);
        if (lane >= d) x += y;
      }
      const uint32_t past = __ballot_sync(0xffffffffu, before + x > at);
      if (past) {
        if (lane == 0) c.tokens[b * c.ld_tokens + n] = v + __ffs(past) - 1;
        return;
      }
      before += __shfl_sync(0xffffffffu, x, 31);
    }
    return;
  }
}

}  // namespace

cudaError_t launch_verify(const sp_verify& c, cudaStream_t stream) {
  int dev = 0, sms = 0;
  cudaError_t e = current_device(&dev, &sms);
  if (e != cudaSuccess) return e;
  int cluster = 8;
  while (cluster > 1 && (c.B * cluster > 2 * sms || c.V < 1024 * cluster)) cluster /= 2;
  VerifyParams p;
  p.c = c;
  p.slice = ceil_div(c.V, cluster);
  p.span = ceil_div(ceil_div(p.slice, kVerWarps), 32) * 32;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(c.B * cluster), 1, 1);
  cfg.blockDim = dim3(kVerThreads, 1, 1);
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
