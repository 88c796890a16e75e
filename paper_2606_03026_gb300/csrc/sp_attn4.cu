// sp_attn4.cu -- attention over a KV cache held in 4 bits (see
// spike_proj_cache4_attend):
//
//   s_j = scale q . k_j,   lse = ln sum_j e^{s_j},   out = sum_j e^{s_j - lse} v_j
//
// for R = T x G query rows of a K/V head (G query heads share it), joined with the
// attention of the same rows over other entries where that is given.
//
// Codes become half precision in registers, where both products take them from:
// a code times its scale is exact there.  Queries are half precision too, each row
// times a power of two that brings its largest element to 2^14 .. 2^15, so that
// bf16's range fits (what is lost lies 2^-39 below the row's largest).  Entries are
// the rows of the matrix instructions (m16n8k16), query rows their 8 columns: for
// few rows an instruction is full of entries.  The order of the elements of a row
// in an instruction's sum, and of the entries in the other's, is free, so that a
// thread takes whole pieces of a row, with one or two scales each:
//   S^T = K Q^T   thread (g, t): entry of row g, elements t DK/4 .. (t + 1) DK/4
//   O^T = V^T P^T thread (g, t): elements g DK/8 .. (g + 1) DK/8 of entries
//                 t, t + 4, t + 8, t + 12
// P^T comes from S^T by transposing 8 x 8 blocks between the threads.
//
// Work: the entries of all (sequence, K/V head, up to 32 rows) are one line of
// tiles of 16, which the CTAs share out evenly, whatever the lengths (which only
// the device knows).  A warp takes every eighth tile of its CTA's, through a ring
// of its own in shared memory (cp.async), with its own running maximum and sums;
// the warps' results are merged at the end of a CTA's tiles of a unit.  Where a
// unit is of several CTAs, each leaves its result in the workspace, and the one
// that comes last merges them, in the order of the tiles.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <math.h>

#include "sp_cache4.cuh"
#include "sp_ptx.cuh"

namespace sp {
namespace {

constexpr int kWarps = 8, kThreads = 32 * kWarps;
constexpr int kTile = 16;                  // entries of a tile
constexpr int kMaxRows = 32;               // of a unit
constexpr int kMaxSeqs = SPIKE_PROJ_CACHE_MAX_B;
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
// The reference of the exponentials follows the running maximum only when that has
// grown by more than 2^kLag; it lies kLift below, so that half precision's
// subnormals are 2^-34 of the largest probability.
constexpr float kLag = 4.f, kLift = 10.f;
constexpr int kStart = 8;                  // cost of a unit beside its tiles
constexpr uint32_t kOnes = 0x3c003c00u;

template <int DK> constexpr int kRowBytes = DK / 2;
template <int DK> constexpr int kStageBytes = 2 * kTile * kRowBytes<DK> + 2 * kTile * 8;
// Rings take what a warp's result does in the merge, at the least.
template <int DK, int NT> constexpr int kStages = NT <= 2 ? 4 : DK == 128 ? 8 : 8;
template <int DK, int NT> constexpr int kWarpBytes = kStages<DK, NT> * kStageBytes<DK> > 8 * NT * DK * 4
                                                         ? kStages<DK, NT> * kStageBytes<DK>
                                                         : 8 * NT * DK * 4;

struct Params {
  sp_attend4 c;
  int32_t Hkv, G, D, capacity, R;
  int32_t blocks, block_rows;              // units of a (sequence, K/V head); rows of one
  int32_t bf16;
  float c2;                                // scale * log2 e
  uint32_t* tickets;                       // [grid], zero between calls
  float4* slot_ml;                         // [2 grid][32]: reference, sum, sum of the rounded
  float* slot_o;                           // [2 grid][32][DK]
};

// Dynamic shared memory: the warps' rings, and what the merge keeps of them.
template <int DK, int NT> constexpr size_t smem_bytes() {
  return (size_t)kWarps * kWarpBytes<DK, NT> + (NT > 1 ? NT * (DK / 16) * 32 * 8 : 0);
}

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ uint32_t pack_half2(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
__device__ __forceinline__ uint32_t transpose8(uint32_t x) {
  uint32_t r;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(x));
  return r;
}
__device__ __forceinline__ void mma(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
template <int BYTES>
__device__ __forceinline__ void copy_async(uint32_t to, const uint8_t* from) {
  if constexpr (BYTES == 16)
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(from) : "memory");
  else
    asm volatile("cp.async.ca.shared.global [%0], [%1], 8;" ::"r"(to), "l"(from) : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void copy_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

__device__ __forceinline__ float2 to_float(bool bf16, uint32_t x) {
  if (bf16) return make_float2(__uint_as_float(x << 16), __uint_as_float(x & 0xffff0000u));
  return __half22float2(*reinterpret_cast<const __half2*>(&x));
}
__device__ __forceinline__ uint32_t from_float(bool bf16, float lo, float hi) {
  uint32_t r;
  if (bf16) asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  else r = pack_half2(lo, hi);
  return r;
}

// Entry of row i < 16 of an instruction's K operand, and with it of element i of
// the sum over entries: thread t's elements 2t, 2t + 1, 2t + 8, 2t + 9 are the
// entries t, t + 4, t + 8, t + 12.
__device__ __forceinline__ int entry_of(int i) { return (i & 8) | (i & 1) << 2 | (i & 7) >> 1; }
// Where 16 bytes (8 where rows are 32 bytes) of an entry lie in a tile of the ring,
// so that neither operand's loads meet in a bank.
template <int DK> __device__ __forceinline__ int place_of(int entry, int byte) {
  if constexpr (DK == 128) {
    const int row = entry ^ (entry >> 2 & 1);
    return row * 64 + (byte ^ (row >> 1 & 1) << 5);
  } else {
    const int row = entry ^ (entry & 4) >> 1;
    return row * 32 + byte;
  }
}

// ---- the line of tiles --------------------------------------------------------
struct Line {
  int64_t all;
  int ctas;
  __device__ __forceinline__ int64_t first(int c) const { return c * all / ctas; }
  __device__ __forceinline__ int owner(int64_t at) const { return (int)(((at + 1) * ctas - 1) / all); }
};
__device__ __forceinline__ int used(const Params& p, int b) { return min(max(__ldg(p.c.lens + b), 0), p.capacity); }

// A row's results of several parts, as they are merged.
struct RowSum {
  float m, l, r;                           // reference, sum, sum of the rounded probabilities
};

template <int DK, int NT>
__global__ void __launch_bounds__(kThreads, NT <= 2 ? 2 : 1) attend4_kernel(const __grid_constant__ Params p) {
  constexpr int KS = DK / 16;              // steps of S's sum, m-tiles of O
  constexpr int RB = kRowBytes<DK>, NS = kStages<DK, NT>;
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ int64_t s_before[kMaxSeqs + 1];
  __shared__ int64_t s_scan[kWarps];
  __shared__ float s_m[kWarps][8 * NT], s_l[kWarps][8 * NT], s_r[kWarps][8 * NT];
  __shared__ uint32_t s_poison[8 * NT];
  __shared__ int s_last;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, t = lane & 3;
  uint8_t* ring = smem + warp * kWarpBytes<DK, NT>;
  uint2* s_q = reinterpret_cast<uint2*>(smem + kWarps * kWarpBytes<DK, NT>);     // [NT][KS][32]
  pdl_launch_dependents();
  pdl_wait();

  // cost of the units of all sequences before each
  const int per_seq = p.Hkv * p.blocks;
  {
    const int per = (p.c.B + kThreads - 1) / kThreads;
    int64_t sum = 0;
    for (int i = 0; i < per; ++i) {
      const int b = tid * per + i;
      if (b < p.c.B) sum += (int64_t)per_seq * (kStart + ceil_div(used(p, b), kTile));
    }
    int64_t up = sum;
#pragma unroll
    for (int d = 1; d < 32; d *= 2) {
      const int64_t x = __shfl_up_sync(0xffffffffu, up, d);
      if (lane >= d) up += x;
    }
    if (lane == 31) s_scan[warp] = up;
    __syncthreads();
    int64_t before = up - sum;
    for (int w = 0; w < warp; ++w) before += s_scan[w];
    for (int i = 0; i < per; ++i) {
      const int b = tid * per + i;
      if (b < p.c.B) {
        s_before[b] = before;
        before += (int64_t)per_seq * (kStart + ceil_div(used(p, b), kTile));
        if (b == p.c.B - 1) s_before[p.c.B] = before;
      }
    }
    __syncthreads();
  }
  Line line;
  line.all = s_before[p.c.B];
  // (a tile for each warp at least)
  line.ctas = (int)min((int64_t)gridDim.x, max((int64_t)1, line.all / (kStart + kWarps)));
  const int cta = blockIdx.x;
  if (cta >= line.ctas) return;
  const int64_t begin = line.first(cta), end = line.first(cta + 1);

  for (int64_t x = begin; x < end;) {
    int b = 0;
    for (int hi = p.c.B; hi - b > 1;) {
      const int mid = (b + hi) >> 1;
      if (s_before[mid] <= x) b = mid; else hi = mid;
    }
    const int n = used(p, b), nt = ceil_div(n, kTile), cost = kStart + nt;
    const int u = (int)((x - s_before[b]) / cost);
    const int64_t at = s_before[b] + (int64_t)u * cost, next = at + cost;
    const int h = u / p.blocks, block = u - h * p.blocks;
    const int j0 = (int)max((int64_t)0, x - at - kStart);
    const int j1 = (int)max((int64_t)0, min(end, next) - at - kStart);
    const bool initial = x == begin;
    x = next;
    if (j1 <= j0 && (nt > 0 || j0 > 0 || (initial && at != begin))) continue;
    const int row0 = block * p.block_rows, rows = min(p.block_rows, p.R - row0);

    // ---- the query rows ---------------------------------------------------------
    if (tid < 8 * NT) s_poison[tid] = 0;
    uint2 q[KS];                           // of one n-tile
    float c2[NT][2];                       // of the rows 2t, 2t + 1 of each n-tile
    int far[NT][2];                        // entries that they see
    __syncthreads();
#pragma unroll
    for (int i = 0; i < NT; ++i) {
      const int r = i * 8 + g;
      uint2 raw[KS];
      uint32_t top = 0;
#pragma unroll
      for (int j = 0; j < KS; ++j) raw[j] = make_uint2(0, 0);
      if (r < rows) {
        const int tok = (row0 + r) / p.G, hq = h * p.G + (row0 + r) - tok * p.G;
        const uint16_t* from = static_cast<const uint16_t*>(p.c.q) + b * p.c.q_batch + tok * p.c.q_token + hq * p.c.q_head;
#pragma unroll
        for (int j = 0; j < KS; ++j) {
          const int d = t * (DK / 4) + 4 * j;
          if (d < p.D) raw[j] = __ldg(reinterpret_cast<const uint2*>(from + d));
          // (the largest that is finite)
          const uint32_t w[2] = {raw[j].x & 0x7fff7fffu, raw[j].y & 0x7fff7fffu};
          const uint32_t inf = p.bf16 ? 0x7f807f80u : 0x7c007c00u;
#pragma unroll
          for (int e = 0; e < 2; ++e) top = __vmaxu2(top, w[e] & ~__vcmpgeu2(w[e], inf));
        }
      }
      top = max(top & 0xffffu, top >> 16);
      top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
      top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
      // 2^e that brings the largest to 2^14 .. 2^15 (bf16 only)
      int e = 0;
      if (p.bf16) e = min(14 - ((int)(top >> 7) - 127), 100);
      const float up = __int_as_float((e + 127) << 23);
#pragma unroll
      for (int j = 0; j < KS; ++j) {
        const float2 lo = to_float(p.bf16, raw[j].x), hi = to_float(p.bf16, raw[j].y);
        const uint2 x = make_uint2(pack_half2(lo.x * up, lo.y * up), pack_half2(hi.x * up, hi.y * up));
        if (NT == 1) q[j] = x;
        else if (warp == 0) s_q[(i * KS + j) * 32 + lane] = x;
      }
      // (lane 4 r has row r's)
      const float down = p.c2 * __int_as_float((127 - e) << 23);
#pragma unroll
      for (int e2 = 0; e2 < 2; ++e2) {
        c2[i][e2] = __shfl_sync(0xffffffffu, down, 4 * (2 * t + e2));
        const int r2 = i * 8 + 2 * t + e2;
        far[i][e2] = r2 < rows ? n - (p.c.causal ? p.c.T - 1 - (row0 + r2) / p.G : 0) : n;
      }
    }
    if (NT > 1) __syncthreads();
    const int all_see = n - (p.c.causal ? p.c.T - 1 : 0);

    // ---- a warp's tiles ---------------------------------------------------------
    const sp_kv4 &k4 = p.c.k4, &v4 = p.c.v4;
    const uint8_t* kc = k4.codes + b * k4.batch + h * k4.head;
    const uint8_t* vc = v4.codes + b * v4.batch + h * v4.head;
    // scales: lane l has those of entry l of a tile's keys, l - 16 of its values
    const sp_kv4& mine4 = lane < 16 ? k4 : v4;
    const uint8_t* sc = mine4.scales + b * mine4.scales_batch + h * mine4.scales_head;
    const int64_t sc_entry = mine4.scales_entry;
    const int groups = p.D / 16;
    const auto fetch_codes = [&](int tile, int stage) {
      const uint32_t to = smem_u32(ring) + stage * kStageBytes<DK>;
      const int nbytes = p.D / 2;
      if (nbytes % 16 == 0) {
        constexpr int C = RB / 16;         // of a row
#pragma unroll
        for (int i = 0; i < kTile * C / 32; ++i) {
          const int e = (i * 32 + lane) / C, byte = (i * 32 + lane) % C * 16;
          const int64_t entry = (int64_t)tile * kTile + e;
          if (entry < n && byte < nbytes) {
            copy_async<16>(to + place_of<DK>(e, byte), kc + entry * k4.entry + byte);
            copy_async<16>(to + kTile * RB + place_of<DK>(e, byte), vc + entry * v4.entry + byte);
          }
        }
      } else {
        constexpr int C = RB / 8;
#pragma unroll
        for (int i = 0; i < kTile * C / 32; ++i) {
          const int e = (i * 32 + lane) / C, byte = (i * 32 + lane) % C * 8;
          const int64_t entry = (int64_t)tile * kTile + e;
          if (entry < n && byte < nbytes) {
            copy_async<8>(to + place_of<DK>(e, byte), kc + entry * k4.entry + byte);
            copy_async<8>(to + kTile * RB + place_of<DK>(e, byte), vc + entry * v4.entry + byte);
          }
        }
      }
    };
    const auto fetch_scales = [&](int tile) {
      uint2 s = make_uint2(0, 0);
      const int64_t entry = (int64_t)tile * kTile + (lane & 15);
      if (tile < j1 && entry < n) {
        const uint8_t* from = sc + entry * sc_entry;
        if (groups == 8) s = __ldg(reinterpret_cast<const uint2*>(from));
        else if (groups == 4) s.x = __ldg(reinterpret_cast<const uint32_t*>(from));
        else
          for (int i = 0; i < groups; ++i) {
            const uint32_t x = __ldg(from + i);
            if (i < 4) s.x |= x << (8 * i); else s.y |= x << (8 * i - 32);
          }
      }
      return s;
    };
    // A NaN scale of a value must not meet a probability of 0 of a row that does not
    // see its entry: it becomes 0, and the rows that do see it remember the group.
    const auto store_scales = [&](int tile, int stage, uint2 s) {
      if (lane >= 16) {
        const uint32_t bad[2] = {__vcmpgeu4(s.x, 0xf9f9f9f9u), __vcmpgeu4(s.y, 0xf9f9f9f9u)};
        if (bad[0] | bad[1]) {
          s.x &= ~bad[0];
          s.y &= ~bad[1];
          uint32_t mask = 0;
          for (int i = 0; i < 8; ++i) mask |= (bad[i / 4] >> (8 * (i % 4)) & 1u) << i;
          const int entry = tile * kTile + (lane & 15);
          for (int r = 0; r < rows; ++r)
            if (entry < n - (p.c.causal ? p.c.T - 1 - (row0 + r) / p.G : 0)) atomicOr(&s_poison[r], mask);
        }
      }
      *reinterpret_cast<uint2*>(ring + stage * kStageBytes<DK> + 2 * kTile * RB + lane * 8) = s;
    };

    float o[NT][KS][4], sum_r[NT][4], m[NT][2], l[NT][2];
#pragma unroll
    for (int i = 0; i < NT; ++i) {
#pragma unroll
      for (int j = 0; j < KS; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[i][j][e] = 0.f;
#pragma unroll
      for (int e = 0; e < 4; ++e) sum_r[i][e] = 0.f;
      m[i][0] = m[i][1] = -INFINITY;
      l[i][0] = l[i][1] = 0.f;
    }
    const int mine = max(0, ceil_div(j1 - j0 - warp, kWarps));
    uint2 scales = fetch_scales(j0 + warp);
#pragma unroll
    for (int i = 0; i < NS - 1; ++i) {
      if (i < mine) fetch_codes(j0 + warp + i * kWarps, i);
      copy_commit();
    }
    for (int it = 0; it < mine; ++it) {
      const int tile = j0 + warp + it * kWarps, stage = it % NS;
      store_scales(tile, stage, scales);
      scales = fetch_scales(tile + kWarps);
      copy_wait<NS - 2>();
      __syncwarp();
      // (the place of the tile before, which every lane has left)
      if (it + NS - 1 < mine) fetch_codes(tile + (NS - 1) * kWarps, (it + NS - 1) % NS);
      copy_commit();
      const uint8_t* place = ring + stage * kStageBytes<DK>;
      const uint8_t* place_s = place + 2 * kTile * RB;

      // S^T = K Q^T
      float s[NT][4];
#pragma unroll
      for (int i = 0; i < NT; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) s[i][e] = 0.f;
      {
        constexpr int W = DK / 32;         // words of an entry: four code pairs each
        uint32_t w[2][W], sc2[2][W / 2];
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          const int e = entry_of(g + 8 * half);
          const uint8_t* from = place + place_of<DK>(e, t * (RB / 4));
          if constexpr (DK == 128) {
            const uint4 x = *reinterpret_cast<const uint4*>(from);
            w[half][0] = x.x, w[half][1] = x.y, w[half][2] = x.z, w[half][3] = x.w;
            const uint32_t y = *reinterpret_cast<const uint16_t*>(place_s + e * 8 + 2 * t);
            sc2[half][0] = scale_half2(y & 0xffu);
            sc2[half][1] = scale_half2(y >> 8);
          } else {
            const uint2 x = *reinterpret_cast<const uint2*>(from);
            w[half][0] = x.x, w[half][1] = x.y;
            sc2[half][0] = scale_half2(place_s[e * 8 + t]);
          }
        }
#pragma unroll
        for (int i = 0; i < W; ++i) {
          uint32_t lo[4], hi[4];
          codes_to_half(w[0][i], lo);
          codes_to_half(w[1][i], hi);
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            lo[k] = mul_half2(lo[k], sc2[0][i / 2]);
            hi[k] = mul_half2(hi[k], sc2[1][i / 2]);
          }
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            const uint32_t a[4] = {lo[2 * k], hi[2 * k], lo[2 * k + 1], hi[2 * k + 1]};
#pragma unroll
            for (int c = 0; c < NT; ++c) {
              const uint2 qq = NT == 1 ? q[2 * i + k] : s_q[(c * KS + 2 * i + k) * 32 + lane];
              mma(s[c], a, qq.x, qq.y);
            }
          }
        }
      }
      // probabilities
#pragma unroll
      for (int i = 0; i < NT; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) s[i][e] *= c2[i][e & 1];
      const int e0 = tile * kTile + entry_of(g);                 // of s[.][0 .. 1]; e0 + 8 of the others
      if (tile * kTile + kTile > all_see) {
#pragma unroll
        for (int i = 0; i < NT; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (e0 + (e >> 1) * 8 >= far[i][e & 1]) s[i][e] = -INFINITY;
      }
      uint32_t pb[NT][2];
      bool grow = false;
      float top[NT][2];
#pragma unroll
      for (int i = 0; i < NT; ++i)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          top[i][e] = fmaxf(s[i][e], s[i][e + 2]);
          grow |= top[i][e] > m[i][e] + kLag;
        }
      if (__any_sync(0xffffffffu, grow)) {
#pragma unroll
        for (int i = 0; i < NT; ++i) {
          float a[2];
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            float x = top[i][e];
#pragma unroll
            for (int d = 4; d < 32; d *= 2) x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, d));
            a[e] = 1.f;
            if (x > m[i][e] + kLag) {
              a[e] = ex2(m[i][e] - x);     // 0 at the first
              m[i][e] = x;
            }
            l[i][e] *= a[e];
          }
#pragma unroll
          for (int e = 0; e < 4; ++e) sum_r[i][e] *= a[e & 1];
#pragma unroll
          for (int j = 0; j < KS; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) o[i][j][e] *= a[e & 1];
        }
      }
#pragma unroll
      for (int i = 0; i < NT; ++i) {
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const float base = m[i][e] == -INFINITY ? 0.f : m[i][e] - kLift;
          s[i][e] = ex2(s[i][e] - base);
          s[i][e + 2] = ex2(s[i][e + 2] - base);
          l[i][e] += s[i][e] + s[i][e + 2];
        }
        pb[i][0] = transpose8(pack_half2(s[i][0], s[i][1]));
        pb[i][1] = transpose8(pack_half2(s[i][2], s[i][3]));
      }
      // O^T += V^T P^T
      {
        uint32_t w[4][KS / 4], sb[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int e = t + 4 * i;
          const uint8_t* from = place + kTile * RB + place_of<DK>(e, g * (RB / 8));
          if constexpr (DK == 128) {
            const uint2 x = *reinterpret_cast<const uint2*>(from);
            w[i][0] = x.x, w[i][1] = x.y;
            sb[i] = place_s[(16 + e) * 8 + g];
          } else {
            w[i][0] = *reinterpret_cast<const uint32_t*>(from);
            sb[i] = place_s[(16 + e) * 8 + g / 2];
          }
        }
        const uint32_t s01 = sb[0] << 7 | sb[1] << 23, s23 = sb[2] << 7 | sb[3] << 23;
#pragma unroll
        for (int i = 0; i < KS / 4; ++i) {
          uint32_t y[4][4];
#pragma unroll
          for (int k = 0; k < 4; ++k) codes_to_half(w[k][i], y[k]);
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const uint32_t a[4] = {mul_half2(__byte_perm(y[0][k], y[1][k], 0x5410), s01),
                                   mul_half2(__byte_perm(y[0][k], y[1][k], 0x7632), s01),
                                   mul_half2(__byte_perm(y[2][k], y[3][k], 0x5410), s23),
                                   mul_half2(__byte_perm(y[2][k], y[3][k], 0x7632), s23)};
#pragma unroll
            for (int c = 0; c < NT; ++c) mma(o[c][4 * i + k], a, pb[c][0], pb[c][1]);
          }
        }
        const uint32_t ones[4] = {kOnes, kOnes, kOnes, kOnes};
#pragma unroll
        for (int c = 0; c < NT; ++c) mma(sum_r[c], ones, pb[c][0], pb[c][1]);
      }
      __syncwarp();
    }
    copy_wait<0>();
    __syncwarp();

    // ---- the warps' results, one after the other --------------------------------
    float* ow = reinterpret_cast<float*>(ring);                  // [8 NT][DK]
#pragma unroll
    for (int i = 0; i < NT; ++i) {
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        float x = l[i][e];
#pragma unroll
        for (int d = 4; d < 32; d *= 2) x += __shfl_xor_sync(0xffffffffu, x, d);
        const int r = i * 8 + 2 * t + e;
        if (g == 0) {
          s_m[warp][r] = m[i][e];
          s_l[warp][r] = x;
          s_r[warp][r] = sum_r[i][e];
        }
#pragma unroll
        for (int j = 0; j < KS; ++j)
          *reinterpret_cast<float2*>(ow + r * DK + g * (DK / 8) + 2 * j) = make_float2(o[i][j][e], o[i][j][e + 2]);
      }
    }
    __syncthreads();

    const int c_first = nt > 0 ? line.owner(at + kStart) : cta, c_last = nt > 0 ? line.owner(at + kStart + nt - 1) : cta;
    // The sum over the warps: thread = (row, 4 elements).  (A NaN stays.)
    const auto over_warps = [&](int r, int d, RowSum& a) {
      a.m = -INFINITY;
#pragma unroll
      for (int w = 0; w < kWarps; ++w) a.m = fmaxf(a.m, s_m[w][r]);
      a.l = a.r = 0.f;
      float4 o4 = make_float4(0.f, 0.f, 0.f, 0.f);
      const float base = a.m == -INFINITY ? 0.f : a.m;
#pragma unroll
      for (int w = 0; w < kWarps; ++w) {
        const float f = ex2(s_m[w][r] - base);
        const float4 x = *reinterpret_cast<const float4*>(smem + w * kWarpBytes<DK, NT> + (r * DK + d) * 4);
        a.l = fmaf(f, s_l[w][r], a.l);
        a.r = fmaf(f, s_r[w][r], a.r);
        o4.x = fmaf(f, x.x, o4.x), o4.y = fmaf(f, x.y, o4.y), o4.z = fmaf(f, x.z, o4.z), o4.w = fmaf(f, x.w, o4.w);
      }
      return o4;
    };
    const auto finish = [&](int r, int d, RowSum a, float4 o4) {
      const int tok = (row0 + r) / p.G, hq = h * p.G + (row0 + r) - tok * p.G;
      const int64_t row = ((int64_t)b * p.c.T + tok) * p.Hkv * p.G + hq;
      float base = a.m - kLift;
      if (p.c.other_out) {
        const float other = p.c.other_lse[row] * kLog2e;
        if (!(other == -INFINITY)) {
          const float to = fmaxf(base, other);
          const float f = a.m == -INFINITY ? 0.f : ex2(base - to), fo = ex2(other - to);
          float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
          if (d < p.D) {
            const uint2 raw = *reinterpret_cast<const uint2*>(static_cast<const uint16_t*>(p.c.other_out) + b * p.c.other_batch +
                                                              tok * p.c.other_token + hq * p.c.other_head + d);
            const float2 lo = to_float(p.bf16, raw.x), hi = to_float(p.bf16, raw.y);
            x = make_float4(lo.x, lo.y, hi.x, hi.y);
          }
          o4.x = fmaf(fo, x.x, f * o4.x), o4.y = fmaf(fo, x.y, f * o4.y);
          o4.z = fmaf(fo, x.z, f * o4.z), o4.w = fmaf(fo, x.w, f * o4.w);
          a.l = fmaf(a.l, f, fo);
          a.r = fmaf(a.r, f, fo);
          a.m = 0.f;
          base = to;
        }
      }
      const bool empty = a.l == 0.f;
      const float inv = empty ? 0.f : 1.f / a.r;
      if (d < p.D) {
        uint2 w = make_uint2(0u, 0u);
        if (!empty) w = make_uint2(from_float(p.bf16, o4.x * inv, o4.y * inv), from_float(p.bf16, o4.z * inv, o4.w * inv));
        *reinterpret_cast<uint2*>(static_cast<uint16_t*>(p.c.out) + b * p.c.out_batch + tok * p.c.out_token +
                                  hq * p.c.out_head + d) = w;
      }
      if (d == 0 && p.c.lse) p.c.lse[row] = empty ? -INFINITY : (base + log2f(a.l)) * kLn2;
    };
    const auto poison = [&](int r, int d, float4& o4) {
      if (s_poison[r] >> (d / 16) & 1u) o4 = make_float4(NAN, NAN, NAN, NAN);
    };
    if (c_first == c_last) {
      for (int i = tid; i < rows * (DK / 4); i += kThreads) {
        const int r = i / (DK / 4), d = i % (DK / 4) * 4;
        RowSum a;
        float4 o4 = over_warps(r, d, a);
        poison(r, d, o4);
        finish(r, d, a, o4);
      }
      __syncthreads();
      continue;
    }
    {
      const int64_t slot = 2 * (int64_t)cta + (initial ? 0 : 1);
      for (int i = tid; i < rows * (DK / 4); i += kThreads) {
        const int r = i / (DK / 4), d = i % (DK / 4) * 4;
        RowSum a;
        float4 o4 = over_warps(r, d, a);
        poison(r, d, o4);
        if (d == 0) p.slot_ml[slot * kMaxRows + r] = make_float4(a.m, a.l, a.r, 0.f);
        *reinterpret_cast<float4*>(p.slot_o + (slot * kMaxRows + r) * DK + d) = o4;
      }
    }
    __threadfence();
    __syncthreads();
    if (tid == 0) {
      const uint32_t before = atomicAdd(p.tickets + c_first, 1u);
      s_last = before == (uint32_t)(c_last - c_first);
      if (s_last) p.tickets[c_first] = 0;
    }
    __syncthreads();
    if (!s_last) continue;
    __threadfence();
    // Warp w sums every eighth of the unit's results, row by row; the warps' sums are
    // then merged as those of their tiles were.
    const int first_slot = line.first(c_first) >= at ? 2 * c_first : 2 * c_first + 1;
    for (int r = 0; r < rows; ++r) {
      RowSum a{-INFINITY, 0.f, 0.f};
      float4 o4 = make_float4(0.f, 0.f, 0.f, 0.f);
      for (int c0 = c_first + warp; c0 <= c_last; c0 += kWarps * 4) {
        float4 ml[4], x[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int c = c0 + i * kWarps;
          ml[i] = make_float4(-INFINITY, 0.f, 0.f, 0.f);
          x[i] = make_float4(0.f, 0.f, 0.f, 0.f);
          if (c <= c_last) {
            const int64_t slot = c == c_first ? first_slot : 2 * (int64_t)c;
            ml[i] = __ldcg(p.slot_ml + slot * kMaxRows + r);
            if (lane < DK / 4) x[i] = __ldcg(reinterpret_cast<const float4*>(p.slot_o + (slot * kMaxRows + r) * DK + 4 * lane));
          }
        }
        float to = a.m;
#pragma unroll
        for (int i = 0; i < 4; ++i) to = fmaxf(to, ml[i].x);
        const float base = to == -INFINITY ? 0.f : to, f0 = ex2(a.m - base);
        a.m = to;
        a.l *= f0, a.r *= f0;
        o4.x *= f0, o4.y *= f0, o4.z *= f0, o4.w *= f0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float f = ex2(ml[i].x - base);
          a.l = fmaf(f, ml[i].y, a.l);
          a.r = fmaf(f, ml[i].z, a.r);
          o4.x = fmaf(f, x[i].x, o4.x), o4.y = fmaf(f, x[i].y, o4.y), o4.z = fmaf(f, x[i].z, o4.z), o4.w = fmaf(f, x[i].w, o4.w);
        }
      }
      if (lane < DK / 4) *reinterpret_cast<float4*>(ow + r * DK + 4 * lane) = o4;
      if (lane == 0) {
        s_m[warp][r] = a.m;
        s_l[warp][r] = a.l;
        s_r[warp][r] = a.r;
      }
    }
    __syncthreads();
    for (int i = tid; i < rows * (DK / 4); i += kThreads) {
      const int r = i / (DK / 4), d = i % (DK / 4) * 4;
      RowSum a;
      const float4 o4 = over_warps(r, d, a);
      finish(r, d, a, o4);
    }
    __syncthreads();
  }
}

// ---- host ---------------------------------------------------------------------
int ctas_per_sm(int NT) { return NT <= 2 ? 2 : 1; }
int n_tiles(int rows) { return (rows + 7) / 8; }
size_t round256(size_t n) { return (n + 255) / 256 * 256; }

template <int DK, int NT>
cudaError_t launch_t(const Params& p, int dev, int sms, cudaStream_t s) {
  static PerDevice attr;
  const cudaError_t e = attr.once(dev, []() {
    return cudaFuncSetAttribute(attend4_kernel<DK, NT>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem_bytes<DK, NT>());
  });
  if (e != cudaSuccess) return e;
  return launch_pdl(attend4_kernel<DK, NT>, dim3((unsigned)(sms * ctas_per_sm(NT))), dim3(kThreads), smem_bytes<DK, NT>(), s, p);
}

}  // namespace

Cache4Workspace cache4_workspace(const Cache4Shape& s, int sms) {
  const size_t grid = 2 * (size_t)sms, DK = s.D <= 64 ? 64 : 128;
  Cache4Workspace w;
  w.tickets = 0;
  w.slots = round256(grid * 4);
  w.bytes = w.slots + 2 * grid * kMaxRows * (16 + DK * 4);
  return w;
}

cudaError_t launch_attend4(const Cache4Shape& s, const sp_attend4& c, uint8_t* ws, cudaStream_t stream) {
  int dev = 0, sms = 0;
  const cudaError_t e = current_device(&dev, &sms);
  if (e != cudaSuccess) return e;
  Params p;
  p.c = c;
  p.Hkv = s.Hkv;
  p.G = s.Hq / s.Hkv;
  p.D = s.D;
  p.capacity = s.capacity;
  p.R = c.T * p.G;
  p.blocks = row_blocks4(p.R);
  p.block_rows = ceil_div(p.R, p.blocks);
  p.bf16 = s.dtype == SP_BF16;
  p.c2 = c.scale * kLog2e;
  const Cache4Workspace w = cache4_workspace(s, sms);
  p.tickets = reinterpret_cast<uint32_t*>(ws + w.tickets);
  p.slot_ml = reinterpret_cast<float4*>(ws + w.slots);
  p.slot_o = reinterpret_cast<float*>(ws + w.slots + 4 * (size_t)sms * kMaxRows * 16);
  const int NT = n_tiles(p.block_rows);
  if (s.D <= 64) {
    switch (NT) {
      case 1: return launch_t<64, 1>(p, dev, sms, stream);
      case 2: return launch_t<64, 2>(p, dev, sms, stream);
      case 3: return launch_t<64, 3>(p, dev, sms, stream);
      default: return launch_t<64, 4>(p, dev, sms, stream);
    }
  }
  switch (NT) {
    case 1: return launch_t<128, 1>(p, dev, sms, stream);
    case 2: return launch_t<128, 2>(p, dev, sms, stream);
    case 3: return launch_t<128, 3>(p, dev, sms, stream);
    default: return launch_t<128, 4>(p, dev, sms, stream);
  }
}

}  // namespace sp
