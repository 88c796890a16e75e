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
// attend_kernel: units of (128 rows, K/V head) x all their entries, cut into
// tiles of 128 entries.  The tiles of all units, the prefix's first, are one
// line that two CTAs per SM share out evenly, whatever the lengths (which only
// the device knows); a CTA's run of tiles within a unit is a segment, which
// leaves its sum over V, its maximum and its sum of exponentials in a slot of
// the workspace.  Per CTA (192 threads):
//   warps 0-3   the softmax, thread = row = tensor-memory lane: they write the
//               segment's query rows to shared memory in the 128-byte swizzle
//               that the MMA reads, and per tile read the 128 scores of their
//               row, keep the running maximum and sum, and put the
//               probabilities, rounded to the type, back over the scores.
//   warp 4      TMA: K and V tiles into a ring.
//   warp 5      one thread issues S = Q K^T and O += P V (tcgen05, M = 128, P
//               from tensor memory, V as an N-major operand).
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
// combine_kernel: one or four warps per query row merge its segments' slots and
// these last entries.  weights_kernel: the weights, from the scores of the own
// entries that attend_kernel left in the workspace and the rows' lse.
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cudaTypedefs.h>

#include <math.h>

#include "sp_cache.h"
#include "sp_ptx.cuh"

namespace sp {
namespace {

constexpr int kTile = 128;                 // entries of a tile, rows of a unit
constexpr int kAttThreads = 192;
constexpr int kTmemCols = 256;             // S and P: 0 .. 127, O: 128 .. 255
constexpr uint32_t kTmemO = 128;
constexpr int kBlockBytes = kTile * 128;   // 64 elements of 128 entries
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

template <int DK> constexpr int kStages = DK == 64 ? 2 : 1;
template <int DK> constexpr int kTileBytes = DK / 64 * kBlockBytes;

struct AttnParams {
  sp_attend c;
  int32_t Hq, Hkv, G, D, capacity;
  int32_t R, Rm, mt_own, mt_prefix, nt_prefix, nt_cap;   // Rm: rows of an own slot
  float c2;                 // scale * log2 e
  int* err;
  int32_t* sched;           // [B + 1]: own tiles before each sequence; [B] all of them
  float4* p_ml;             // prefix slots: [slot][128] reference, sum, sum of the rounded
  float* p_o;               //               [slot][128][DK]
  float4* o_ml;             // own slots: [slot][Rm], [slot][Rm][DK]
  float* o_o;
  float* scores;            // [B][Hkv][nt_cap][R][128], or null
  float* lse2;              // [B][Hkv][R], base 2; +infinity where a row sees nothing
};

// ---- the line of tiles -------------------------------------------------------
__device__ __forceinline__ int used(const AttnParams& p, int b) {
  return min(max(__ldg(p.c.lens + b), 0), p.capacity);
}
// Own entries of a sequence that every query token sees, and their tiles.
__device__ __forceinline__ int seen_by_all(const AttnParams& p, int b) { return max(0, used(p, b) - (p.c.T - 1)); }

struct Line {
  int prefix;               // tiles of the prefix units
  int64_t all;              // tiles
  int ctas;                 // that have any
  // CTA c has tiles first(c) .. first(c + 1)
  __device__ __forceinline__ int64_t first(int c) const { return c * all / ctas; }
  // the CTA of a tile
  __device__ __forceinline__ int cta(int64_t tile) const { return (int)(((tile + 1) * ctas - 1) / all); }
};
__device__ __forceinline__ Line line_of(const AttnParams& p, int own_tiles, int grid) {
  Line l;
  l.prefix = p.Hkv * p.mt_prefix * p.nt_prefix;
  l.all = (int64_t)l.prefix + own_tiles;
  l.ctas = (int)min((int64_t)grid, l.all);
  return l;
}

struct Segment {
  bool prefix;
  int b, h, m;              // sequence (own), head, row tile
  int j0, count;            // tiles
  int seen;                 // entries of the unit
  int rows;                 // of the unit
  int64_t slot;
};
// The segment at tile x of a CTA whose tiles end at `end`.
__device__ __forceinline__ Segment segment_at(const AttnParams& p, const Line& l, const int* off, int64_t x,
                                              int64_t end, int cta) {
  Segment s;
  s.prefix = x < l.prefix;
  if (s.prefix) {
    const int u = (int)x / p.nt_prefix;
    s.j0 = (int)x - u * p.nt_prefix;
    s.count = (int)min((int64_t)(p.nt_prefix - s.j0), end - x);
    s.b = 0;
    s.h = u / p.mt_prefix;
    s.m = u - s.h * p.mt_prefix;
    s.seen = p.c.prefix_len;
    s.rows = min(kTile, p.c.B * p.R - s.m * kTile);
    s.slot = cta + u;
    return s;
  }
  const int y = (int)(x - l.prefix);
  int lo = 0, hi = p.c.B;                  // off[lo] <= y < off[hi]
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (off[mid] <= y) lo = mid; else hi = mid;
  }
  s.b = lo;
  const int nt = (off[lo + 1] - off[lo]) / (p.Hkv * p.mt_own);
  const int u = (y - off[lo]) / nt;
  s.j0 = y - off[lo] - u * nt;
  s.count = (int)min((int64_t)(nt - s.j0), end - x);
  s.h = u / p.mt_own;
  s.m = u - s.h * p.mt_own;
  s.seen = seen_by_all(p, lo);
  s.rows = min(kTile, p.R - s.m * kTile);
  s.slot = cta + (int64_t)lo * p.Hkv * p.mt_own + u;
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
// of N kBlockBytes on.
__device__ __forceinline__ uint64_t n_major_desc(const void* p) {
  uint64_t d = smem_desc(p, 1024, kSwizzle128);
  d &= ~((uint64_t)0x3FFF << 16);
  return d | (uint64_t)(kBlockBytes >> 4) << 16;
}

template <int DK, bool BF16>
__global__ void __launch_bounds__(kAttThreads, 2)
attend_kernel(const __grid_constant__ CUtensorMap map_pk, const __grid_constant__ CUtensorMap map_pv,
              const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v,
              const __grid_constant__ AttnParams p) {
  constexpr int NS = kStages<DK>, kBytes = kTileBytes<DK>;
  constexpr uint32_t kType = BF16 ? 1u << 7 | 1u << 10 : 0u;
  constexpr uint32_t kIdescS = 1u << 4 | kType | (uint32_t)(kTile >> 3) << 17 | (uint32_t)(kTile >> 4) << 24;
  constexpr uint32_t kIdescO = 1u << 4 | kType | 1u << 16 | (uint32_t)(DK >> 3) << 17 | (uint32_t)(kTile >> 4) << 24;
  constexpr float kLag = BF16 ? 8.f : 4.f, kLift = BF16 ? 0.f : 10.f;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  uint8_t* sQ = smem;
  uint8_t* sK = sQ + kBytes;
  uint8_t* sV = sK + NS * kBytes;
  uint64_t* bars = reinterpret_cast<uint64_t*>(sV + NS * kBytes);
  uint64_t *k_full = bars, *k_empty = bars + NS, *v_full = bars + 2 * NS, *v_empty = bars + 3 * NS;
  uint64_t *q_full = bars + 4 * NS, *s_full = q_full + 1, *p_full = q_full + 2, *o_full = q_full + 3,
           *o_empty = q_full + 4, *done = q_full + 5;
  uint32_t* s_tmem = reinterpret_cast<uint32_t*>(done + 1);
  volatile int* s_abort = reinterpret_cast<volatile int*>(s_tmem + 1);
  int* s_sum = reinterpret_cast<int*>(s_tmem + 2);         // [8]
  int* s_off = s_sum + 8;                                  // [B + 1]

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    for (int i = 0; i < NS; ++i) {
      mbar_init(&k_full[i], 1);
      mbar_init(&k_empty[i], 1);
      mbar_init(&v_full[i], 1);
      mbar_init(&v_empty[i], 1);
    }
    mbar_init(q_full, 4);
    mbar_init(s_full, 1);
    mbar_init(p_full, 4);
    mbar_init(o_full, 1);
    mbar_init(o_empty, 4);
    mbar_init(done, 1);
    *s_abort = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    tma_prefetch_desc(&map_pk);
    tma_prefetch_desc(&map_pv);
    tma_prefetch_desc(&map_k);
    tma_prefetch_desc(&map_v);
  }
  if (warp == 5) tmem_alloc(s_tmem, kTmemCols);
  pdl_launch_dependents();
  pdl_wait();

  // own tiles before each sequence: every CTA adds them up for itself
  {
    const int per = ceil_div(p.c.B, kAttThreads), b0 = threadIdx.x * per, b1 = min(b0 + per, p.c.B);
    int sum = 0;
    for (int b = b0; b < b1; ++b) sum += ceil_div(seen_by_all(p, b), kTile) * p.Hkv * p.mt_own;
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
    for (int b = b0; b < b1; ++b) {
      s_off[b] = at;
      if (blockIdx.x == 0) p.sched[b] = at;
      at += ceil_div(seen_by_all(p, b), kTile) * p.Hkv * p.mt_own;
    }
    if (b0 < p.c.B && b1 == p.c.B) {
      s_off[p.c.B] = at;
      if (blockIdx.x == 0) p.sched[p.c.B] = at;
    }
    __syncthreads();
  }
  const uint32_t tmem = *s_tmem;
  const Line line = line_of(p, s_off[p.c.B], gridDim.x);
  const int cta = blockIdx.x;
  const int64_t x0 = cta < line.ctas ? line.first(cta) : 0, x1 = cta < line.ctas ? line.first(cta + 1) : 0;

  if (warp == 4) {
    // ------------------------------ TMA -----------------------------------------
    if (lane == 0) {
      int it = 0;
      for (int64_t x = x0; x < x1 && !*s_abort;) {
        const Segment s = segment_at(p, line, s_off, x, x1, cta);
        const CUtensorMap* mk = s.prefix ? &map_pk : &map_k;
        const CUtensorMap* mv = s.prefix ? &map_pv : &map_v;
        for (int j = 0; j < s.count && !*s_abort; ++j, ++it) {
          const int st = it % NS;
          const uint32_t ph = (it / NS) & 1;
          bool ok = mbar_wait_sleep(&k_empty[st], ph ^ 1u);
          if (ok) {
            mbar_arrive_expect_tx(&k_full[st], kBytes);
            for (int i = 0; i < DK / 64; ++i)
              tma_load_4d(sK + st * kBytes + i * kBlockBytes, mk, &k_full[st], 64 * i, (s.j0 + j) * kTile, s.h, s.b);
            ok = mbar_wait_sleep(&v_empty[st], ph ^ 1u);
            if (ok) {
              mbar_arrive_expect_tx(&v_full[st], kBytes);
              for (int i = 0; i < DK / 64; ++i)
                tma_load_4d(sV + st * kBytes + i * kBlockBytes, mv, &v_full[st], 64 * i, (s.j0 + j) * kTile, s.h, s.b);
            } else {
              mbar_wait(&k_full[st], ph);  // no copy is in flight at the end
            }
          }
          if (!ok) {
            *s_abort = 1;
            atomicExch(p.err, kErrMbarTimeout);
            break;
          }
        }
        x += s.count;
      }
      // the last copies have landed
      for (int i = max(0, it - NS); i < it; ++i) {
        mbar_wait(&k_full[i % NS], (i / NS) & 1);
        mbar_wait(&v_full[i % NS], (i / NS) & 1);
      }
    }
  } else if (warp == 5) {
    // ------------------------------ MMA -----------------------------------------
    if (lane == 0) {
      int it = 0, seg = 0;
      bool ok = true;
      const uint64_t qd = smem_desc(sQ, 1024, kSwizzle128);
      for (int64_t x = x0; x < x1 && ok; ++seg) {
        const Segment s = segment_at(p, line, s_off, x, x1, cta);
        ok = mbar_wait(q_full, seg & 1);
        for (int j = 0; j < s.count && ok; ++j, ++it) {
          const int st = it % NS;
          const uint32_t ph = (it / NS) & 1;
          ok = mbar_wait(&k_full[st], ph) && !*s_abort;
          if (!ok) break;
          tc_fence_after();
          const uint64_t kd = smem_desc(sK + st * kBytes, 1024, kSwizzle128);
#pragma unroll
          for (int k = 0; k < DK / 16; ++k)
            mma_f16(tmem, qd + (k / 4) * (kBlockBytes >> 4) + (k % 4) * 2, kd + (k / 4) * (kBlockBytes >> 4) + (k % 4) * 2,
                    kIdescS, k > 0);
          mma_commit(s_full);
          mma_commit(&k_empty[st]);
          ok = mbar_wait(p_full, it & 1) && mbar_wait(&v_full[st], ph) && (j > 0 || mbar_wait(o_empty, (seg & 1) ^ 1u)) &&
               !*s_abort;
          if (!ok) break;
          tc_fence_after();
          const uint64_t vd = n_major_desc(sV + st * kBytes);
#pragma unroll
          for (int k = 0; k < kTile / 16; ++k)
            mma_f16_ta(tmem + kTmemO, tmem + 8 * k, vd + k * (2048 >> 4), kIdescO, j > 0 || k > 0);
          mma_commit(&v_empty[st]);
        }
        if (ok) mma_commit(o_full);
        x += s.count;
      }
      if (!ok) {
        *s_abort = 1;
        atomicExch(p.err, kErrMbarTimeout);
      }
      mma_commit(done);                    // every MMA has retired
      mbar_wait(done, 0);
    }
  } else {
    // ------------------------------ softmax -------------------------------------
    const int row = threadIdx.x;
    const uint32_t t_row = tmem + ((uint32_t)(warp * 32) << 16);
    int it = 0, seg = 0;
    bool ok = true;
    for (int64_t x = x0; x < x1 && ok; ++seg) {
      const Segment s = segment_at(p, line, s_off, x, x1, cta);
      const bool work = warp * 32 < s.rows, mine = row < s.rows;
      // the segment's query rows (the tile's other rows hold what they hold)
      int b = s.b, rr = s.m * kTile + row;
      if (s.prefix) {
        b = rr / p.R;
        rr -= b * p.R;
      }
      {
        const int t = rr / p.G;
        const int64_t at = mine ? b * p.c.q_batch + t * p.c.q_token + (int64_t)(s.h * p.G + rr - t * p.G) * p.c.q_head : 0;
        constexpr int kPieces = DK / 8, kRows = 32 / kPieces;
        const int piece = lane % kPieces;
        const bool real = piece * 8 < p.D;
#pragma unroll 4
        for (int r = lane / kPieces; r < 32; r += kRows) {
          const int64_t from = __shfl_sync(0xffffffffu, at, r);
          const int tr = warp * 32 + r;
          if (tr < s.rows) {
            uint4 v = make_uint4(0u, 0u, 0u, 0u);
            if (real) v = __ldg(reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(p.c.q) + from) + piece);
            *reinterpret_cast<uint4*>(sQ + (piece / 8) * kBlockBytes + tr * 128 + (((piece % 8) ^ (tr & 7)) << 4)) = v;
          }
        }
        fence_async_shared();
        __syncwarp();
        if (lane == 0) mbar_arrive(q_full);
      }
      float m = -INFINITY, ref = 0.f, l = 0.f, rl = 0.f;
      for (int j = 0; j < s.count; ++j, ++it) {
        const int nv = min(kTile, s.seen - (s.j0 + j) * kTile);
        ok = __all_sync(0xffffffffu, mbar_wait(s_full, it & 1) && !*s_abort);
        if (!ok) break;
        tc_fence_after();
        if (work) {
          uint32_t v[4][32];
#pragma unroll
          for (int i = 0; i < 4; ++i) tmem_ld32_issue(t_row + 32 * i, v[i]);
          tmem_ld_wait();
#pragma unroll
          for (int i = 0; i < 4; ++i) reg_pin(v[i]);
          if (!s.prefix && p.scores && mine) {
            float4* dst = reinterpret_cast<float4*>(
                p.scores + ((((int64_t)s.b * p.Hkv + s.h) * p.nt_cap + s.j0 + j) * p.R + rr) * kTile);
#pragma unroll
            for (int i = 0; i < 32; ++i)
              dst[i] = make_float4(__uint_as_float(v[i / 8][i % 8 * 4]), __uint_as_float(v[i / 8][i % 8 * 4 + 1]),
                                   __uint_as_float(v[i / 8][i % 8 * 4 + 2]), __uint_as_float(v[i / 8][i % 8 * 4 + 3]));
          }
          if (nv < kTile) {
#pragma unroll
            for (int i = 0; i < 128; ++i)
              if (i >= nv) v[i / 32][i % 32] = 0xff800000u;
          }
          float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
          for (int i = 0; i < 128; ++i) mx[i % 4] = fmaxf(mx[i % 4], __uint_as_float(v[i / 32][i % 32]));
          const float top = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3])) * p.c2;
          const bool grow = top > m + kLag;
          if (__any_sync(0xffffffffu, grow)) {
            float a = 1.f;
            if (grow) {
              a = ex2(m - top);            // 0 at the first
              m = top;
              ref = top - kLift;
            }
            l *= a;
            rl *= a;
            if (j > 0) {
#pragma unroll
              for (int i = 0; i < DK / 16; ++i) {
                uint32_t o[16];
                tmem_ld16(t_row + kTmemO + 16 * i, o);
                reg_pin(o);
#pragma unroll
                for (int e = 0; e < 16; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * a);
                tmem_st16_issue(t_row + kTmemO + 16 * i, o);
              }
            }
          }
          f32x2 sum[2] = {}, rsum[2] = {};
          const f32x2 c2 = pair(p.c2, p.c2), base = pair(-ref, -ref);
#pragma unroll
          for (int h2 = 0; h2 < 2; ++h2) {
            uint32_t pk[32];
#pragma unroll
            for (int i = 0; i < 32; ++i) {
              const int e = 64 * h2 + 2 * i;
              const float2 x = halves(fma2(
                  pair(__uint_as_float(v[e / 32][e % 32]), __uint_as_float(v[e / 32][e % 32 + 1])), c2, base));
              const float2 y = make_float2(ex2(x.x), ex2(x.y));
              pk[i] = pack2<BF16>(y.x, y.y);
              const float2 r = unpack2<BF16>(pk[i]);
              sum[i % 2] = add2(sum[i % 2], pair(y.x, y.y));
              rsum[i % 2] = add2(rsum[i % 2], pair(r.x, r.y));
            }
            tmem_st32_issue(t_row + 32 * h2, pk);
          }
          const float2 ls = halves(add2(sum[0], sum[1])), lr = halves(add2(rsum[0], rsum[1]));
          l += ls.x + ls.y;
          rl += lr.x + lr.y;
          tmem_st_wait();
        }
        if (!s.prefix && nv < kTile) {
          // entries past those in use hold anything: their values become 0
          const int st = it % NS;
          ok = __all_sync(0xffffffffu, mbar_wait(&v_full[st], (it / NS) & 1));
          if (!ok) break;
          if (row >= nv) {
#pragma unroll
            for (int i = 0; i < DK / 64; ++i)
#pragma unroll
              for (int e = 0; e < 8; ++e)
                *reinterpret_cast<uint4*>(sV + st * kBytes + i * kBlockBytes + row * 128 + 16 * e) =
                    make_uint4(0u, 0u, 0u, 0u);
          }
          fence_async_shared();
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(p_full);
      }
      if (!ok) break;
      ok = __all_sync(0xffffffffu, mbar_wait(o_full, seg & 1) && !*s_abort);
      if (!ok) break;
      tc_fence_after();
      if (work) {
        float* o = s.prefix ? p.p_o + (s.slot * kTile + row) * DK : p.o_o + (s.slot * p.Rm + row) * DK;
        if (mine) (s.prefix ? p.p_ml + s.slot * kTile : p.o_ml + s.slot * p.Rm)[row] = make_float4(ref, l, rl, 0.f);
#pragma unroll
        for (int i = 0; i < DK / 32; ++i) {
          uint32_t v[32];
          tmem_ld32(t_row + kTmemO + 32 * i, v);
          reg_pin(v);
          if (mine) {
#pragma unroll
            for (int e = 0; e < 8; ++e)
              reinterpret_cast<uint4*>(o)[8 * i + e] = make_uint4(v[4 * e], v[4 * e + 1], v[4 * e + 2], v[4 * e + 3]);
          }
        }
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(o_empty);
      x += s.count;
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
// A lane has DK / 32 elements of a row: lane * DK / 32 ...
template <int DK, bool BF16>
__device__ __forceinline__ void load_row(const void* base, int64_t at, int D, int lane, float (&x)[DK / 32]) {
  constexpr int E = DK / 32;
  const uint16_t* p = static_cast<const uint16_t*>(base) + at + lane * E;
  uint32_t w[E / 2];
#pragma unroll
  for (int i = 0; i < E / 2; ++i) w[i] = 0u;
  if (lane * E < D) {                      // (D is a multiple of 8)
    if constexpr (E == 4) {
      const uint2 u = __ldg(reinterpret_cast<const uint2*>(p));
      w[0] = u.x;
      w[1] = u.y;
    } else {
      w[0] = __ldg(reinterpret_cast<const uint32_t*>(p));
    }
  }
#pragma unroll
  for (int i = 0; i < E / 2; ++i) {
    const float2 f = unpack2<BF16>(w[i]);
    x[2 * i] = f.x;
    x[2 * i + 1] = f.y;
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

constexpr int kCombWarps = 4;

template <int DK, bool BF16, int WPR>      // WPR warps per query row
__global__ void __launch_bounds__(32 * kCombWarps) combine_kernel(const __grid_constant__ AttnParams p, int grid) {
  constexpr int E = DK / 32;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, sub = warp % WPR;
  pdl_launch_dependents();
  pdl_wait();
  const int64_t id = (int64_t)blockIdx.x * (kCombWarps / WPR) + warp / WPR;     // (b, h, row)
  const bool real = id < (int64_t)p.c.B * p.Hkv * p.R;
  Part<E> a;
  a.m = -INFINITY;
  a.l = a.r = 0.f;
#pragma unroll
  for (int i = 0; i < E; ++i) a.o[i] = 0.f;
  int b = 0, h = 0, rr = 0;
  if (real) {
    rr = (int)(id % p.R);
    h = (int)(id / p.R % p.Hkv);
    b = (int)(id / p.R / p.Hkv);
    const Line line = line_of(p, __ldg(p.sched + p.c.B), grid);
    // slots of the row: those of the prefix unit, then those of the own unit
    int np = 0, no = 0;
    int64_t sp0 = 0, so0 = 0;
    int rp = 0, ro = 0;
    if (p.nt_prefix > 0) {
      const int64_t at = (int64_t)b * p.R + rr;
      const int m = (int)(at / kTile), u = h * p.mt_prefix + m;
      rp = (int)(at % kTile);
      const int64_t t0 = (int64_t)u * p.nt_prefix;
      const int c0 = line.cta(t0), c1 = line.cta(t0 + p.nt_prefix - 1);
      sp0 = c0 + u;
      np = c1 - c0 + 1;
    }
    const int own0 = __ldg(p.sched + b), nt = (__ldg(p.sched + b + 1) - own0) / (p.Hkv * p.mt_own);
    if (nt > 0) {
      const int u = h * p.mt_own + rr / kTile;
      ro = rr % kTile;
      const int64_t t0 = line.prefix + own0 + (int64_t)u * nt;
      const int c0 = line.cta(t0), c1 = line.cta(t0 + nt - 1);
      so0 = c0 + (int64_t)b * p.Hkv * p.mt_own + u;
      no = c1 - c0 + 1;
    }
    for (int s0 = 32 * sub; s0 < np + no; s0 += 32 * WPR) {
      const int s = s0 + lane;
      float4 ml = make_float4(0.f, 0.f, 0.f, 0.f);
      if (s < np) ml = __ldcg(p.p_ml + (sp0 + s) * kTile + rp);
      else if (s < np + no) ml = __ldcg(p.o_ml + (so0 + s - np) * p.Rm + ro);
      float m = ml.y == 0.f ? -INFINITY : ml.x;             // (a NaN sum stays in)
      float top = m;
#pragma unroll
      for (int d = 16; d >= 1; d >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
      if (top == -INFINITY) continue;
      if (top > a.m) a.rebase(top);
      const float w = m == -INFINITY ? 0.f : ex2(m - a.m);
      float l = m == -INFINITY ? 0.f : w * ml.y, r = m == -INFINITY ? 0.f : w * ml.z;
#pragma unroll
      for (int d = 16; d >= 1; d >>= 1) {
        l += __shfl_xor_sync(0xffffffffu, l, d);
        r += __shfl_xor_sync(0xffffffffu, r, d);
      }
      a.l += l;
      a.r += r;
      const int n = min(32, np + no - s0);
#pragma unroll 4
      for (int i = 0; i < n; ++i) {
        const float wi = __shfl_sync(0xffffffffu, w, i);
        const int si = s0 + i;
        const float* src = si < np ? p.p_o + ((sp0 + si) * kTile + rp) * DK : p.o_o + ((so0 + si - np) * p.Rm + ro) * DK;
        float o[E];
        if constexpr (E == 4) {
          const float4 f = __ldcg(reinterpret_cast<const float4*>(src) + lane);
          o[0] = f.x, o[1] = f.y, o[2] = f.z, o[3] = f.w;
        } else {
          const float2 f = __ldcg(reinterpret_cast<const float2*>(src) + lane);
          o[0] = f.x, o[1] = f.y;
        }
        if (wi != 0.f) {
#pragma unroll
          for (int e = 0; e < E; ++e) a.o[e] = fmaf(wi, o[e], a.o[e]);
        }
      }
    }
    // the last T - 1 own entries, of which this row sees the first few
    if (sub == 0 && p.c.T > 1) {
      const int t = rr / p.G, hq = h * p.G + rr % p.G, n = used(p, b), j0 = max(0, n - (p.c.T - 1));
      const int far = n - (p.c.T - 1 - t);
      float q[E];
      load_row<DK, BF16>(p.c.q, b * p.c.q_batch + t * p.c.q_token + hq * p.c.q_head, p.D, lane, q);
      for (int j = j0; j < n; ++j) {
        float s = -INFINITY;
        if (j < far) {
          float k[E], v[E];
          load_row<DK, BF16>(p.c.k, b * p.c.k_batch + j * p.c.k_entry + h * p.c.k_head, p.D, lane, k);
          load_row<DK, BF16>(p.c.v, b * p.c.v_batch + j * p.c.v_entry + h * p.c.v_head, p.D, lane, v);
          s = 0.f;
#pragma unroll
          for (int e = 0; e < E; ++e) s = fmaf(q[e], k[e], s);
#pragma unroll
          for (int d = 16; d >= 1; d >>= 1) s += __shfl_xor_sync(0xffffffffu, s, d);
          const float x = s * p.c2;
          if (x > a.m) a.rebase(x);
          const float w = ex2(fmaf(s, p.c2, a.m == -INFINITY ? 0.f : -a.m));
          a.l += w;
          a.r += w;
#pragma unroll
          for (int e = 0; e < E; ++e) a.o[e] = fmaf(w, v[e], a.o[e]);
          if (a.m == -INFINITY && w != 0.f) a.m = 0.f;      // (a NaN score)
        }
        if (p.scores && lane == 0)
          p.scores[((((int64_t)b * p.Hkv + h) * p.nt_cap + j / kTile) * p.R + rr) * kTile + j % kTile] = s;
      }
    }
  }
  if constexpr (WPR > 1) {
    __shared__ float s_ml[kCombWarps][3], s_o[kCombWarps][DK];
#pragma unroll
    for (int e = 0; e < E; ++e) s_o[warp][lane * E + e] = a.o[e];
    if (lane == 0) {
      s_ml[warp][0] = a.m;
      s_ml[warp][1] = a.l;
      s_ml[warp][2] = a.r;
    }
    __syncthreads();
    if (sub != 0) return;
#pragma unroll
    for (int w = 1; w < WPR; ++w) {
      const float m = s_ml[warp + w][0];
      if (m == -INFINITY) continue;
      if (m > a.m) a.rebase(m);
      const float x = ex2(m - a.m);
      a.l = fmaf(x, s_ml[warp + w][1], a.l);
      a.r = fmaf(x, s_ml[warp + w][2], a.r);
#pragma unroll
      for (int e = 0; e < E; ++e) a.o[e] = fmaf(x, s_o[warp + w][lane * E + e], a.o[e]);
    }
  }
  if (!real) return;
  const int t = rr / p.G, hq = h * p.G + rr % p.G;
  const bool empty = a.l == 0.f;
  const float inv = empty ? 0.f : 1.f / a.r;
  if (lane * E < p.D) {
    uint16_t* out = static_cast<uint16_t*>(p.c.out) + b * p.c.out_batch + t * p.c.out_token + hq * p.c.out_head + lane * E;
    uint32_t w[E / 2];
#pragma unroll
    for (int i = 0; i < E / 2; ++i)
      w[i] = empty ? 0u : pack2<BF16>(a.o[2 * i] * inv, a.o[2 * i + 1] * inv);
    if constexpr (E == 4) *reinterpret_cast<uint2*>(out) = make_uint2(w[0], w[1]);
    else *reinterpret_cast<uint32_t*>(out) = w[0];
  }
  if (lane == 0) {
    const float l2 = a.m + log2f(a.l);
    if (p.c.lse) p.c.lse[((int64_t)b * p.c.T + t) * p.Hq + hq] = empty ? -INFINITY : l2 * kLn2;
    if (p.scores) p.lse2[id] = empty ? INFINITY : l2;
  }
}

// One warp per 32 entries of a tile: the rows' scores of an entry, added up.
__global__ void __launch_bounds__(kTile) weights_kernel(const __grid_constant__ AttnParams p) {
  pdl_launch_dependents();
  pdl_wait();
  const int b = blockIdx.y / p.Hkv, h = blockIdx.y % p.Hkv, n = used(p, b);
  const float* lse2 = p.lse2 + (int64_t)blockIdx.y * p.R;
  for (int tile = blockIdx.x; tile * kTile < n; tile += gridDim.x) {
    const int j = tile * kTile + threadIdx.x;
    if (j >= n) return;
    const float* s = p.scores + ((int64_t)blockIdx.y * p.nt_cap + tile) * p.R * kTile + threadIdx.x;
    float* w = p.c.weights + b * p.c.weights_batch + h * p.c.weights_head + j;
    float sum = 0.f;
#pragma unroll 4
    for (int r = 0; r < p.R; ++r) {
      const float x = __ldcg(s + (int64_t)r * kTile);
      if (x != -INFINITY) sum += ex2(fmaf(x, p.c2, -__ldcg(lse2 + r)));
    }
    *w += sum;
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

// [batch][entry][head][D] of 16-bit elements in boxes of 64 elements x 128
// entries, zero past the extents.  A dimension of size 1 has no stride.
bool encode_kv(CUtensorMap* map, bool bf16, const void* base, int D, int64_t entries, int64_t heads, int64_t batch,
               int64_t s_entry, int64_t s_head, int64_t s_batch) {
  const auto enc = get_encode();
  if (!enc) return false;
  const auto bytes = [&](int64_t n, int64_t stride) { return (cuuint64_t)(n > 1 ? 2 * stride : 2 * (int64_t)D); };
  const cuuint64_t dims[4] = {(cuuint64_t)D, (cuuint64_t)entries, (cuuint64_t)heads, (cuuint64_t)batch};
  const cuuint64_t strides[3] = {bytes(entries, s_entry), bytes(heads, s_head), bytes(batch, s_batch)};
  const cuuint32_t box[4] = {64, kTile, 1, 1}, ones[4] = {1, 1, 1, 1};
  return enc(map, bf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 4,
             const_cast<void*>(base), dims, strides, box, ones, CU_TENSOR_MAP_INTERLEAVE_NONE,
             CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
             CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int DK>
size_t attend_smem(int B) {
  return 1024 + (size_t)(1 + 2 * kStages<DK>) * kTileBytes<DK> + (4 * kStages<DK> + 6) * 8 + 8 + 32 + (size_t)(B + 1) * 4;
}

template <int DK, bool BF16>
cudaError_t launch_attend_t(const AttnParams& p, const CUtensorMap (&maps)[4], int dev, int grid, cudaStream_t s) {
  static PerDevice attr;
  cudaError_t e = attr.once(dev, []() {
    return cudaFuncSetAttribute(attend_kernel<DK, BF16>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                (int)attend_smem<DK>(SPIKE_PROJ_CACHE_MAX_B));
  });
  if (e != cudaSuccess) return e;
  e = launch_pdl(attend_kernel<DK, BF16>, dim3(grid), dim3(kAttThreads), attend_smem<DK>(p.c.B), s, maps[0], maps[1],
                 maps[2], maps[3], p);
  if (e != cudaSuccess) return e;
  const int64_t rows = (int64_t)p.c.B * p.Hkv * p.R;
  if (rows <= 2048)
    e = launch_pdl(combine_kernel<DK, BF16, 4>, dim3((unsigned)rows), dim3(32 * kCombWarps), 0, s, p, grid);
  else
    e = launch_pdl(combine_kernel<DK, BF16, 1>, dim3((unsigned)((rows + 3) / 4)), dim3(32 * kCombWarps), 0, s, p, grid);
  if (e != cudaSuccess || !p.c.weights) return e;
  return launch_pdl(weights_kernel, dim3((unsigned)min(p.nt_cap, 65535), (unsigned)(p.c.B * p.Hkv)), dim3(kTile), 0, s, p);
}

size_t round256(size_t n) { return (n + 255) / 256 * 256; }

// The workspace's parts, for calls of B sequences and T query tokens.
struct Parts {
  size_t sched, lse2, p_ml, p_o, o_ml, o_o, scores, end;
};
Parts parts_of(const CacheShape& s, int B, int T, int grid) {
  const int R = T * (s.Hq / s.Hkv), Rm = min(R, kTile), DK = s.D <= 64 ? 64 : 128;
  const size_t p_slots = (size_t)grid + (size_t)s.Hkv * ceil_div(B * R, kTile);
  const size_t o_slots = (size_t)grid + (size_t)B * s.Hkv * ceil_div(R, kTile);
  Parts w;
  w.sched = 0;
  w.lse2 = round256((size_t)(B + 1) * 4);
  w.p_ml = w.lse2 + round256((size_t)B * s.Hkv * R * 4);
  w.p_o = w.p_ml + p_slots * kTile * 16;
  w.o_ml = w.p_o + p_slots * kTile * DK * 4;
  w.o_o = w.o_ml + round256(o_slots * Rm * 16);
  w.scores = w.o_o + round256(o_slots * Rm * DK * 4);
  w.end = w.scores + (s.weights ? (size_t)B * s.Hkv * ceil_div(s.capacity, kTile) * R * kTile * 4 : 0);
  return w;
}

}  // namespace

CacheWorkspace cache_workspace(const CacheShape& s, int sms) {
  CacheWorkspace w;
  w.moves = round256(parts_of(s, s.max_batch, s.max_T, 2 * sms).end);
  w.bytes = w.moves + (size_t)s.max_batch * s.Hkv * (s.capacity / 2 + 1) * 8;
  return w;
}

cudaError_t launch_attend(const CacheShape& s, const sp_attend& c, uint8_t* ws, int* err, cudaStream_t stream) {
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
  p.Rm = min(p.R, kTile);
  p.mt_own = ceil_div(p.R, kTile);
  p.mt_prefix = ceil_div(c.B * p.R, kTile);
  p.nt_prefix = ceil_div(c.prefix_len, kTile);
  p.nt_cap = ceil_div(s.capacity, kTile);
  p.c2 = c.scale * kLog2e;
  p.err = err;
  const int grid = 2 * sms;
  const Parts w = parts_of(s, c.B, c.T, grid);
  p.sched = reinterpret_cast<int32_t*>(ws + w.sched);
  p.lse2 = reinterpret_cast<float*>(ws + w.lse2);
  p.p_ml = reinterpret_cast<float4*>(ws + w.p_ml);
  p.p_o = reinterpret_cast<float*>(ws + w.p_o);
  p.o_ml = reinterpret_cast<float4*>(ws + w.o_ml);
  p.o_o = reinterpret_cast<float*>(ws + w.o_o);
  p.scores = c.weights ? reinterpret_cast<float*>(ws + w.scores) : nullptr;
  const bool bf16 = s.dtype == SP_BF16;
  CUtensorMap maps[4];
  if (!encode_kv(&maps[2], bf16, c.k, s.D, s.capacity, s.Hkv, c.B, c.k_entry, c.k_head, c.k_batch) ||
      !encode_kv(&maps[3], bf16, c.v, s.D, s.capacity, s.Hkv, c.B, c.v_entry, c.v_head, c.v_batch))
    return cudaErrorInvalidValue;
  if (c.prefix_len == 0) {
    maps[0] = maps[2];                     // (read by nothing)
    maps[1] = maps[3];
  } else if (!encode_kv(&maps[0], bf16, c.prefix_k, s.D, c.prefix_len, s.Hkv, 1, c.pk_entry, c.pk_head, 0) ||
             !encode_kv(&maps[1], bf16, c.prefix_v, s.D, c.prefix_len, s.Hkv, 1, c.pv_entry, c.pv_head, 0)) {
    return cudaErrorInvalidValue;
  }
  if (s.D <= 64)
    return bf16 ? launch_attend_t<64, true>(p, maps, dev, grid, stream)
                : launch_attend_t<64, false>(p, maps, dev, grid, stream);
  return bf16 ? launch_attend_t<128, true>(p, maps, dev, grid, stream)
              : launch_attend_t<128, false>(p, maps, dev, grid, stream);
}

}  // namespace sp
