// sp_attn.cu -- attention of a batch whose sequences share a prefix (see
// spike_proj_cache_attend): a query row r of sequence b sees the P entries of
// the prefix and its own entries,
//
//   s_j = scale q_r . k_j,   out_r = sum_j e^{s_j - lse_r} v_j,
//   weights[b][h][j] += sum over the rows of e^{s_j - lse_r}  (own entries)
//
// One CTA of four warps per query row: each warp takes every fourth entry with
// a running maximum and sum, the lanes holding D, and the four are merged.  A
// second kernel recomputes the scores of the own entries for the weights.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <math.h>

#include "sp_cache.h"
#include "sp_ptx.cuh"

namespace sp {
namespace {

constexpr int kWarps = 4;

struct AttnParams {
  sp_attend c;
  int32_t Hq, Hkv, G, D, capacity;
  float* lse;               // [B][T][Hq]
};

template <typename T16> __device__ __forceinline__ float to_f32(T16 x);
template <> __device__ __forceinline__ float to_f32(__nv_bfloat16 x) { return __bfloat162float(x); }
template <> __device__ __forceinline__ float to_f32(__half x) { return __half2float(x); }
template <typename T16> __device__ __forceinline__ T16 from_f32(float x);
template <> __device__ __forceinline__ __nv_bfloat16 from_f32(float x) { return __float2bfloat16_rn(x); }
template <> __device__ __forceinline__ __half from_f32(float x) { return __float2half_rn(x); }

// Elements lane, lane + 32, ... of a row of D.
template <typename T16>
__device__ __forceinline__ void load_row(const void* base, int64_t at, int D, int lane, float (&x)[4]) {
  const T16* p = static_cast<const T16*>(base) + at;
#pragma unroll
  for (int i = 0; i < 4; ++i) x[i] = lane + 32 * i < D ? to_f32(p[lane + 32 * i]) : 0.f;
}
__device__ __forceinline__ float dot(const float (&a)[4], const float (&b)[4]) {
  float s = 0.f;
#pragma unroll
  for (int i = 0; i < 4; ++i) s = fmaf(a[i], b[i], s);
#pragma unroll
  for (int d = 16; d >= 1; d >>= 1) s += __shfl_xor_sync(0xffffffffu, s, d);
  return s;
}
__device__ __forceinline__ int used(const AttnParams& p, int b) {
  return min(max(__ldg(p.c.lens + b), 0), p.capacity);
}

template <typename T16>
__global__ void __launch_bounds__(32 * kWarps) attend_kernel(const __grid_constant__ AttnParams p) {
  pdl_launch_dependents();
  pdl_wait();
  const sp_attend& c = p.c;
  const int row = blockIdx.x, hq = row % p.Hq, t = row / p.Hq % c.T, b = row / p.Hq / c.T;
  const int h = hq / p.G, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int own = max(0, used(p, b) - (c.T - 1 - t));
  float q[4], o[4] = {}, m = -INFINITY, l = 0.f;
  load_row<T16>(c.q, b * c.q_batch + t * c.q_token + hq * c.q_head, p.D, lane, q);
  for (int j = warp; j < c.prefix_len + own; j += kWarps) {
    float k[4], v[4];
    if (j < c.prefix_len) {
      load_row<T16>(c.prefix_k, (int64_t)j * c.pk_entry + h * c.pk_head, p.D, lane, k);
      load_row<T16>(c.prefix_v, (int64_t)j * c.pv_entry + h * c.pv_head, p.D, lane, v);
    } else {
      const int64_t i = j - c.prefix_len;
      load_row<T16>(c.k, b * c.k_batch + i * c.k_entry + h * c.k_head, p.D, lane, k);
      load_row<T16>(c.v, b * c.v_batch + i * c.v_entry + h * c.v_head, p.D, lane, v);
    }
    const float s = dot(q, k) * c.scale;
    const float mn = fmaxf(m, s), base = mn == -INFINITY ? 0.f : mn;
    const float a = m == -INFINITY ? 0.f : expf(m - base), e = expf(s - base);
    m = mn;
    l = l * a + e;
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] = o[i] * a + e * v[i];
  }
  __shared__ float s_m[kWarps], s_l[kWarps], s_o[kWarps][SPIKE_PROJ_CACHE_MAX_D];
#pragma unroll
  for (int i = 0; i < 4; ++i) s_o[warp][lane + 32 * i] = o[i];
  if (lane == 0) {
    s_m[warp] = m;
    s_l[warp] = l;
  }
  __syncthreads();
  float M = -INFINITY, L = 0.f, x = 0.f;
  for (int w = 0; w < kWarps; ++w) M = fmaxf(M, s_m[w]);
  for (int w = 0; w < kWarps; ++w) {
    const float a = s_m[w] == -INFINITY ? (s_l[w] == 0.f ? 0.f : 1.f) : expf(s_m[w] - M);
    L += a * s_l[w];
    if (a != 0.f) x += a * s_o[w][threadIdx.x];
  }
  if (threadIdx.x < p.D)
    static_cast<T16*>(c.out)[b * c.out_batch + t * c.out_token + hq * c.out_head + threadIdx.x] =
        from_f32<T16>(L == 0.f ? 0.f : x / L);
  if (threadIdx.x == 0) {
    const float lse = L == 0.f ? -INFINITY : (M == -INFINITY ? 0.f : M) + logf(L);
    p.lse[row] = lse;
    if (c.lse) c.lse[row] = lse;
  }
}

template <typename T16>
__global__ void __launch_bounds__(32 * kWarps) weights_kernel(const __grid_constant__ AttnParams p) {
  pdl_launch_dependents();
  pdl_wait();
  const sp_attend& c = p.c;
  const int b = blockIdx.y / p.Hkv, h = blockIdx.y % p.Hkv, lane = threadIdx.x & 31;
  const int n = used(p, b);
  for (int j = blockIdx.x * kWarps + (threadIdx.x >> 5); j < n; j += gridDim.x * kWarps) {
    float k[4], q[4], sum = 0.f;
    load_row<T16>(c.k, b * c.k_batch + (int64_t)j * c.k_entry + h * c.k_head, p.D, lane, k);
    for (int r = 0; r < c.T * p.G; ++r) {
      const int t = r / p.G, hq = h * p.G + r % p.G;
      if (j >= n - (c.T - 1 - t)) continue;
      load_row<T16>(c.q, b * c.q_batch + t * c.q_token + hq * c.q_head, p.D, lane, q);
      const float lse = p.lse[((int64_t)b * c.T + t) * p.Hq + hq];
      if (lse != -INFINITY) sum += expf(dot(q, k) * c.scale - lse);
    }
    if (lane == 0) c.weights[b * c.weights_batch + h * c.weights_head + j] += sum;
  }
}

template <typename T16>
cudaError_t launch_t(const AttnParams& p, cudaStream_t s) {
  cudaError_t e = launch_pdl(attend_kernel<T16>, dim3(p.c.B * p.c.T * p.Hq), dim3(32 * kWarps), 0, s, p);
  if (e != cudaSuccess || !p.c.weights) return e;
  const int blocks = min(ceil_div(p.capacity, kWarps), 256);
  return launch_pdl(weights_kernel<T16>, dim3(blocks, p.c.B * p.Hkv), dim3(32 * kWarps), 0, s, p);
}

}  // namespace

CacheWorkspace cache_workspace(const CacheShape& s, int) {
  CacheWorkspace w;
  w.lse = 0;
  w.moves = ((size_t)s.max_batch * s.max_T * s.Hq * 4 + 255) / 256 * 256;
  w.bytes = w.moves + (size_t)s.max_batch * s.Hkv * (s.capacity / 2 + 1) * 8;
  return w;
}

cudaError_t launch_attend(const CacheShape& s, const sp_attend& c, uint8_t* ws, int*, cudaStream_t stream) {
  AttnParams p;
  p.c = c;
  p.Hq = s.Hq;
  p.Hkv = s.Hkv;
  p.G = s.Hq / s.Hkv;
  p.D = s.D;
  p.capacity = s.capacity;
  p.lse = reinterpret_cast<float*>(ws + cache_workspace(s, 0).lse);
  return s.dtype == SP_BF16 ? launch_t<__nv_bfloat16>(p, stream) : launch_t<__half>(p, stream);
}

}  // namespace sp
