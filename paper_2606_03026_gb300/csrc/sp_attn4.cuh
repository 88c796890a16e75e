// sp_attn4.cuh -- what the kernels of attention over a cache held in 4 bits have in
// common (see sp_attn4.cu): the form of the operands, the line of tiles that the work
// is shared out on, query rows, and a row's end.
#pragma once

#include <cuda_fp16.h>

#include <math.h>

#include "sp_cache4.cuh"
#include "sp_ptx.cuh"

namespace sp {

struct Attend4Params {
  sp_attend4 c;
  int32_t Hkv, G, D, capacity, R;
  int32_t blocks, block_rows;              // units of a (sequence, K/V head); rows of one
  Divide by_blocks, by_G;
  int32_t side;                            // workers that walk side by side, each in units of its own
  int32_t on_line;                         // places of a sequence's units on the line: Hkv blocks / side
  Divide by_side;
  int32_t workers, slot_rows;              // two slots a worker; rows of one
  int32_t bf16;
  float c2;                                // scale * log2 e is c2 2^c2_power, 1 <= c2 <= 2
  int32_t c2_power;
  int* err;
  int fault;                               // kFaultStall: the first keys are never there (tests of the error path)
  long long limit;                         // cycles that a wait takes at most
  int2* units;                             // [B][Hkv][blocks]: slot of the first part (-1: whole), worker of the last
  float4* slot_ml;                         // [2 workers][slot_rows]: reference, sum, sum of the rounded
  float* slot_o;                           // [2 workers][slot_rows][DK]
};

// Units of more rows than one warp takes, a CTA each (sp_attn4_rows.cu).
cudaError_t launch_attend4_rows(const Attend4Params& p, int dev, int sms, cudaStream_t s);

namespace {

constexpr int kWarps = kWarps4, kThreads = 32 * kWarps;
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
// The reference of the exponentials follows the running maximum only when that has
// grown by more than 2^kLag; it lies kLift below, so that half precision's
// subnormals are 2^-34 of the largest probability.  (As much as half precision holds, 2^15.75 <
// 65504: of activations as projections give them 7 % of the tiles of 32 rows move it; with
// kLag = 4 the calls of 64 rows a head took 47.3 us, not 46.4.)
constexpr float kLag = 5.75f, kLift = 10.f;
constexpr int kLeast = 4;                  // cost that is worth a worker
constexpr uint32_t kOnes = 0x3c003c00u;
template <int DK> constexpr int kRowBytes = DK / 2;

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
  else if constexpr (BYTES == 8)
    asm volatile("cp.async.ca.shared.global [%0], [%1], 8;" ::"r"(to), "l"(from) : "memory");
  else
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(to), "l"(from) : "memory");
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
  uint32_t all, workers, each, more;       // the first `more` workers have each + 1 of it, the others each
  Line() = default;
  __device__ __forceinline__ Line(uint32_t all, uint32_t most) : all(all) {
    workers = min(most, max(1u, all / kLeast));
    each = all / workers;
    more = all - each * workers;
  }
  __device__ __forceinline__ uint32_t first(uint32_t w) const { return w * each + min(w, more); }
  __device__ __forceinline__ uint32_t owner(uint32_t at) const {
    const uint32_t long_ones = more * (each + 1);
    return at < long_ones ? at / (each + 1) : more + (at - long_ones) / each;
  }
};
__device__ __forceinline__ int used(const Attend4Params& p, int b) { return min(max(p.c.lens[b], 0), p.capacity); }

// The number of the worker that has place `at` of a unit's line, beside worker `me`.
__device__ __forceinline__ int worker_of(const Attend4Params& p, const Line& line, uint32_t at, int me) {
  uint32_t which = 0;
  if (p.side > 1) p.by_side(me, &which);
  return (int)(line.owner(at) * p.side + which);
}

// A worker's (a warp, or a CTA) way along the line: unit (b, u), its entries, its tiles j .. j1 of the
// worker's.  A unit takes START + nt on the line from `at` on; tile j is at + START + j,
// and belongs to the worker whose part of the line that is in (a unit without tiles to
// the one that `at` is in).
template <int TILE, int START>
struct Cursor {
  int b, u, n, nt, j, j1;
  uint32_t at;
  __device__ __forceinline__ void settle(uint32_t begin, uint32_t end) {
    nt = ceil_div(n, TILE);
    j = begin > at + START ? (int)(begin - at - START) : 0;
    j1 = end > at + START ? min(nt, (int)(end - at - START)) : 0;
  }
  __device__ __forceinline__ void next(const Attend4Params& p, uint32_t begin, uint32_t end) {
    at += START + nt;
    u += p.side;
    if (u >= p.Hkv * p.blocks) {
      u -= p.Hkv * p.blocks;
      ++b;
    }
    if (at < end) {
      n = used(p, b);
      settle(begin, end);
    } else {
      j = j1 = 0;
    }
  }
};

// Where worker `me` of at most `most` begins; all threads of a CTA take part.  before:
// room in shared memory for SPIKE_PROJ_CACHE_MAX_B + 1 words, free again afterwards.  (Up to
// 128 sequences a warp adds the costs up by itself, which waits for no other: 64 chats
// 30.9 -> 29.4 us, 32 drafting sequences 35.4 -> 33.9.)
template <int TILE, int START>
struct Start {
  Line line;
  uint32_t begin, end;
  Cursor<TILE, START> cur;
};
template <int TILE, int START, int THREADS>
__device__ __forceinline__ Start<TILE, START> start_of(const Attend4Params& p, uint32_t* before, int me, uint32_t most) {
  __shared__ uint32_t s_scan[THREADS / 32];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const uint32_t per_seq = p.on_line;
  Start<TILE, START> s;
  uint32_t which = 0;                      // of those that walk side by side
  if (p.side > 1) {
    me = p.by_side(me, &which);
    most = p.by_side(most);
  }
  const auto set_off = [&](int b, uint32_t at, int n) {
    const uint32_t cost = START + ceil_div(n, TILE);
    s.cur.b = b;
    const uint32_t u = (s.begin - at) / cost;
    s.cur.u = (int)(u * p.side + which);
    s.cur.at = at + u * cost;
    s.cur.n = n;
    s.cur.settle(s.begin, s.end);
  };
  constexpr int kFew = 4;
  if (p.c.B <= 32 * kFew) {
    // A warp by itself: lane l has sequences kFew l and on.
    int n[kFew];
    uint32_t cost[kFew], sum = 0;
#pragma unroll
    for (int i = 0; i < kFew; ++i) n[i] = lane * kFew + i < p.c.B ? used(p, lane * kFew + i) : 0;
#pragma unroll
    for (int i = 0; i < kFew; ++i) {
      cost[i] = lane * kFew + i < p.c.B ? per_seq * (START + ceil_div(n[i], TILE)) : 0;
      sum += cost[i];
    }
    uint32_t up = sum;
#pragma unroll
    for (int d = 1; d < 32; d *= 2) {
      const uint32_t x = __shfl_up_sync(0xffffffffu, up, d);
      if (lane >= d) up += x;
    }
    s.line = Line(__shfl_sync(0xffffffffu, up, 31), most);
    s.begin = s.line.first(min((uint32_t)me, s.line.workers));
    s.end = s.line.first(min((uint32_t)me + 1, s.line.workers));
    // the lane, and its sequence, that the worker begins in
    uint32_t at = up - sum;
    const int of = min(31 - __clz((int)__ballot_sync(0xffffffffu, at <= s.begin)), (p.c.B - 1) / kFew);
    int b = lane * kFew, length = n[0];
#pragma unroll
    for (int i = 1; i < kFew; ++i) {
      const bool on = b == lane * kFew + i - 1 && at + cost[i - 1] <= s.begin && b + 1 < p.c.B;
      at = on ? at + cost[i - 1] : at;
      b = on ? b + 1 : b;
      length = on ? n[i] : length;
    }
    set_off(__shfl_sync(0xffffffffu, b, of), __shfl_sync(0xffffffffu, at, of), __shfl_sync(0xffffffffu, length, of));
    return s;
  }
  const uint32_t per = (p.c.B + THREADS - 1) / THREADS;
  uint32_t sum = 0;
  for (uint32_t i = 0; i < per; ++i) {
    const int b = tid * per + i;
    if (b < p.c.B) sum += per_seq * (START + ceil_div(used(p, b), TILE));
  }
  uint32_t up = sum;
#pragma unroll
  for (int d = 1; d < 32; d *= 2) {
    const uint32_t x = __shfl_up_sync(0xffffffffu, up, d);
    if (lane >= d) up += x;
  }
  if (lane == 31) s_scan[warp] = up;
  __syncthreads();
  uint32_t x = up - sum;
  for (int w = 0; w < warp; ++w) x += s_scan[w];
  for (uint32_t i = 0; i < per; ++i) {
    const int b = tid * per + i;
    if (b < p.c.B) {
      before[b] = x;
      x += per_seq * (START + ceil_div(used(p, b), TILE));
      if (b == p.c.B - 1) before[p.c.B] = x;
    }
  }
  __syncthreads();
  s.line = Line(before[p.c.B], most);
  s.begin = s.line.first(min((uint32_t)me, s.line.workers));
  s.end = s.line.first(min((uint32_t)me + 1, s.line.workers));
  int lo = 0;
  for (int hi = p.c.B; hi - lo > 1;) {
    const int mid = (lo + hi) >> 1;
    if (before[mid] <= s.begin) lo = mid; else hi = mid;
  }
  set_off(lo, before[lo], used(p, lo));
  __syncthreads();
  return s;
}

// ---- query rows -----------------------------------------------------------------
// Elements t DK/4 .. (t + 1) DK/4 of row r of a K/V head (`there`: there is one), for the
// four lanes t of the row together.
template <int DK>
__device__ __forceinline__ void load_query(const Attend4Params& p, int b, int h, int r, bool there, int t,
                                           uint2 (&x)[DK / 16]) {
#pragma unroll
  for (int j = 0; j < DK / 16; ++j) x[j] = make_uint2(0, 0);
  if (there) {
    uint32_t in_head;
    const int tok = p.by_G(r, &in_head);
    const uint16_t* from = static_cast<const uint16_t*>(p.c.q) + b * p.c.q_batch + tok * p.c.q_token +
                           (int64_t)(h * p.G + in_head) * p.c.q_head + t * (DK / 4);
#pragma unroll
    for (int j = 0; j < DK / 16; ++j)
      if (t * (DK / 4) + 4 * j < p.D) x[j] = *reinterpret_cast<const uint2*>(from + 4 * j);
  }
}
// The size of queries.  A row of bf16 is brought to half precision times 2^e, which puts its
// largest finite element at 2^14 .. 2^15.  e is at most 126, as far as a factor of FP32 goes: of
// a row below 2^-112 nothing is lost there, as bf16's numbers are multiples of 2^-133.
__device__ __forceinline__ float power_of_two(int e) { return __int_as_float((e + 127) << 23); }
__device__ __forceinline__ int lift_of(uint32_t top) { return min(14 - ((int)(top >> 7) - 127), 126); }  // bits of that element
// What the matrix instructions' scores s of such a row are multiplied by, scale log2 e 2^-e =
// c2 2^power: `by`, within 2^-126 .. 2^127, times `more`.  by is not 0, so that masked scores stay
// -infinity, nor infinite, times which a difference of 0 were a NaN.  Weights do not change by these
// limits: s is below 2^39, and a multiple of 2^-42 (2^-24 of queries, 2^-18 of keys), so that
// where `more` is not 1 scores are equal or more than 2^83 apart.  An lse does: see finish().
struct RowFactor {
  float by, more;
};
__device__ __forceinline__ RowFactor factor_of(const Attend4Params& p, int e) {
  const int power = p.c2_power - e, some = min(max(power, -126), 126);
  return RowFactor{p.c2 * power_of_two(some), power_of_two(max(power - some, 0))};
}

// These as the instructions take them, in half precision.  Returns what the row's scores are to
// be multiplied by.
template <int DK>
__device__ __forceinline__ float make_query(const Attend4Params& p, uint2 (&x)[DK / 16]) {
  constexpr int KS = DK / 16;
  int e = 0;
  if (p.bf16) {
    const auto largest = [&](bool all) {
      uint32_t top = 0;
#pragma unroll
      for (int j = 0; j < KS; ++j) {
        const uint32_t y[2] = {x[j].x & 0x7fff7fffu, x[j].y & 0x7fff7fffu};
#pragma unroll
        for (int i = 0; i < 2; ++i) top = __vmaxu2(top, all ? y[i] : y[i] & ~__vcmpgeu2(y[i], 0x7f807f80u));
      }
      top = max(top & 0xffffu, top >> 16);
      top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
      return max(top, __shfl_xor_sync(0xffffffffu, top, 2));
    };
    uint32_t top = largest(true);
    if (__any_sync(0xffffffffu, top >= 0x7f80u)) top = largest(false);
    e = lift_of(top);
    const float up = power_of_two(e);
#pragma unroll
    for (int j = 0; j < KS; ++j) {
      const float2 lo = to_float(true, x[j].x), hi = to_float(true, x[j].y);
      x[j] = make_uint2(pack_half2(lo.x * up, lo.y * up), pack_half2(hi.x * up, hi.y * up));
    }
  }
  return factor_of(p, e).by;
}

// A row's scales on their way: what a load brings is not looked at before value(), so
// that nothing waits for it.  PLAIN: rows of DK elements.
template <int DK, bool PLAIN>
struct ScaleRow {
  uint32_t b[PLAIN ? DK / 64 : DK / 16];
  __device__ __forceinline__ void load(const uint8_t* from, int groups, bool there) {
    if constexpr (PLAIN) {
#pragma unroll
      for (int i = 0; i < DK / 64; ++i) b[i] = 0;
      if (!there) return;
      if constexpr (DK == 128) {
        const uint2 x = *reinterpret_cast<const uint2*>(from);
        b[0] = x.x, b[DK / 64 - 1] = x.y;
      } else {
        b[0] = *reinterpret_cast<const uint32_t*>(from);
      }
    } else {
      const bool even = groups % 2 == 0;
#pragma unroll
      for (int i = 0; i < DK / 16; ++i) {
        b[i] = 0;
        if (even) {
          if (2 * i < groups && there) b[i] = reinterpret_cast<const uint16_t*>(from)[i];
        } else if (i < groups && there) {
          b[i] = from[i];
        }
      }
    }
  }
  // all of them (8 at most), bytes
  __device__ __forceinline__ uint2 value(int groups) const {
    if constexpr (PLAIN) {
      return make_uint2(b[0], DK == 128 ? b[DK / 64 - 1] : 0u);
    } else if constexpr (DK == 64) {
      return make_uint2(groups % 2 == 0 ? b[0] | b[1] << 16 : b[0] | b[1] << 8 | b[2] << 16, 0u);
    } else {
      if (groups % 2 == 0) return make_uint2(b[0] | b[1] << 16, b[2] | b[3] << 16);
      return make_uint2(b[0] | b[1] << 8 | b[2] << 16 | b[3] << 24, b[4] | b[5] << 8 | b[6] << 16);
    }
  }
};
// The bytes of a row's scales that are NaN (exponent 31), their upper bits.
__device__ __forceinline__ uint32_t nan_scales(uint32_t x) { return ((x & 0x78787878u) + 0x08080808u) & x & 0x80808080u; }
__device__ __forceinline__ uint32_t groups_of(const uint32_t (&bad)[2]) {
  uint32_t mask = 0;
  for (int i = 0; i < 8; ++i) mask |= (bad[i / 4] >> (8 * (i % 4) + 7) & 1u) << i;
  return mask;
}

// The lse (base 2) of the attention over other entries that row r of a K/V head is
// joined with.  It may lie where the row's lse goes, so that all of a row's threads
// have it before one of them stores that.
__device__ __forceinline__ float other_of(const Attend4Params& p, int b, int h, int r) {
  if (!p.c.other_out) return -INFINITY;
  uint32_t in_head;
  const int tok = p.by_G(r, &in_head);
  return p.c.other_lse[((int64_t)b * p.c.T + tok) * p.Hkv * p.G + h * p.G + in_head] * kLog2e;
}
// N values of a row from element d on, out of the sums o with reference `base`, sums l
// and r: joined with other attention, divided, rounded, stored.
template <int N>
__device__ __forceinline__ void finish(const Attend4Params& p, int b, int h, int r, int d, float base, float l, float r_sum,
                                       float (&o)[N], float other, bool first) {
  uint32_t in_head;
  const int tok = p.by_G(r, &in_head), hq = h * p.G + in_head;
  if (fabsf(base) >= 0x1p64f && base != -INFINITY) {           // (where more may not be 1: at 2^83 and above)
    const uint16_t* q = static_cast<const uint16_t*>(p.c.q) + b * p.c.q_batch + tok * p.c.q_token + hq * p.c.q_head;
    uint32_t top = 0;
#pragma unroll 1
    for (int i = 0; i < p.D; ++i) {
      const uint32_t x = q[i] & 0x7fffu;
      if (x < 0x7f80u) top = max(top, x);
    }
    base *= factor_of(p, p.bf16 ? lift_of(top) : 0).more;
    if (base == -INFINITY) l = 0.f;        // (scores below FP32's range)
  }
  if (!(other == -INFINITY)) {
    const float to = fmaxf(base, other);
    // (what the rounding of probabilities did to their sum must not change the parts' weights)
    const float f = base == -INFINITY ? 0.f : ex2(base - to), fo = ex2(other - to), fr = l == 0.f ? 0.f : f * (l / r_sum);
    const uint16_t* from = static_cast<const uint16_t*>(p.c.other_out) + b * p.c.other_batch + tok * p.c.other_token +
                           hq * p.c.other_head + d;
#pragma unroll
    for (int i = 0; i < N; i += 4)
      if (d + i < p.D) {
        const uint2 raw = *reinterpret_cast<const uint2*>(from + i);
        const float2 lo = to_float(p.bf16, raw.x), hi = to_float(p.bf16, raw.y);
        o[i] = fmaf(fo, lo.x, fr * o[i]), o[i + 1] = fmaf(fo, lo.y, fr * o[i + 1]);
        o[i + 2] = fmaf(fo, hi.x, fr * o[i + 2]), o[i + 3] = fmaf(fo, hi.y, fr * o[i + 3]);
      }
    l = fmaf(l, f, fo);
    r_sum = l;
    base = to;
  }
  const bool empty = l == 0.f;
  const float inv = empty ? 0.f : 1.f / r_sum;
  uint16_t* out = static_cast<uint16_t*>(p.c.out) + b * p.c.out_batch + tok * p.c.out_token + hq * p.c.out_head + d;
  uint32_t w[N / 2];
#pragma unroll
  for (int i = 0; i < N / 2; ++i) w[i] = empty ? 0u : from_float(p.bf16, o[2 * i] * inv, o[2 * i + 1] * inv);
  if constexpr (N % 8 == 0) {
#pragma unroll
    for (int i = 0; i < N; i += 8)
      if (d + i < p.D) *reinterpret_cast<uint4*>(out + i) = make_uint4(w[i / 2], w[i / 2 + 1], w[i / 2 + 2], w[i / 2 + 3]);
  } else {
#pragma unroll
    for (int i = 0; i < N; i += 4)
      if (d + i < p.D) *reinterpret_cast<uint2*>(out + i) = make_uint2(w[i / 2], w[i / 2 + 1]);
  }
  if (first && p.c.lse) p.c.lse[((int64_t)b * p.c.T + tok) * p.Hkv * p.G + hq] = empty ? -INFINITY : (base + log2f(l)) * kLn2;
}

}  // namespace
}  // namespace sp
