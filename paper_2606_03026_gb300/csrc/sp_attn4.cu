// sp_attn4.cu -- attention over a KV cache held in 4 bits (see
// spike_proj_cache4_attend):
//
//   s_j = scale q . k_j,   lse = ln sum_j e^{s_j},   out = sum_j e^{s_j - lse} v_j
//
// for R = T x G query rows of a K/V head (G query heads share it), joined with the
// attention of the same rows over other entries where that is given.
//
// Codes become half precision in registers, where both products take them from:
// a code times its scale is exact there.  Queries are half precision too, each row of
// bf16 times a power of two that brings its largest element to 2^14 .. 2^15, so that
// its range fits (what is lost lies 2^-39 below the row's largest).  Entries are
// the rows of the matrix instructions (m16n8k16), query rows their 8 columns: for
// few rows an instruction is full of entries.  The order of the elements of a row
// in an instruction's sum, and of the entries in the other's, is free, so that a
// thread takes whole pieces of a row, with one or two scales each:
//   S^T = K Q^T   thread (g, t): entry of row g, elements t DK/4 .. (t + 1) DK/4
//   O^T = V^T P^T thread (g, t): elements g DK/8 .. (g + 1) DK/8 of entries
//                 t, t + 4, t + 8, t + 12
// P^T comes from S^T by transposing 8 x 8 blocks between the threads.
//
// Work: the entries of all units (sequence, K/V head, up to 8 or 16 rows) are one line of
// tiles of 32, which all warps share out evenly, whatever the lengths (which only
// the device knows).  A warp works by itself: its tiles come through a ring of its
// own in shared memory (cp.async), unit after unit without a pause, and it keeps
// its own maximum and sums.  A unit that one warp has the whole of is written out
// by it; of others each warp leaves its part in the workspace, and merge4_kernel
// adds them up, in the order of the tiles.  (Warps, not CTAs, so that no barrier stands
// between a tile and the next: with tiles shared by a CTA's warps only one CTA had room
// on an SM, and 64 chats took 59 us.)
//
// What bounds it: for long caches memory.  64 sequences of 4096 to 16384 entries, 32/8
// heads of 128, 756 MB: 130 us, 5.8 TB/s (87 % of a copy's rate); at the same time 61 % of the
// issue slots, as 16 entries of a head take about 310 warp instructions (64 conversions of
// code pairs, 64 products with scales, 17 of the matrix unit), which is what bounds 16 rows
// (two walks over the same entries, 245 us).  For short ones the start (places on the line
// 1.6 us, first tiles there at 5 to 9) and the merge with its launch (4): 64 chats of 2048
// entries on average, 76 MB, 27 us.
#include <cmath>
#include <type_traits>

#include "sp_attn4.cuh"

namespace sp {
namespace {

using Params = Attend4Params;
constexpr int kTile = 32, kSubs = kTile / 16;   // entries of a tile, instructions that they are the rows of
constexpr int kStart = 2;                  // cost of a unit beside its tiles
constexpr int kSmallTiles = 24;            // of a cache whose units are CTAs' by themselves

template <int DK> constexpr int kStageBytes = 2 * kTile * kRowBytes<DK> + 2 * kTile * 8;
template <int DK> constexpr int kStages = DK == 64 ? 4 : 3;
template <int DK, int NT> constexpr int kQueryBytes = NT > 1 ? NT * (DK / 16) * 32 * 8 : 0;
template <int DK, int NT> constexpr int kWarpBytes = kStages<DK> * kStageBytes<DK> + kQueryBytes<DK, NT>;
static_assert(attend4_blocks(1, true) * (kWarps * kWarpBytes<128, 1> + 1280) <= 228 * 1024 &&
              attend4_blocks(2, true) * (kWarps * kWarpBytes<64, 2> + 1280) <= 228 * 1024, "shared memory of an SM");
static_assert(kWarps * kWarpBytes<64, 1> >= (SPIKE_PROJ_CACHE_MAX_B + 1) * 4, "room for the costs before each sequence");

// From shared memory, in order with the waits for its copies.
__device__ __forceinline__ uint4 shared16(uint32_t at) {
  uint4 x;
  asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(x.x), "=r"(x.y), "=r"(x.z), "=r"(x.w) : "r"(at));
  return x;
}
__device__ __forceinline__ uint2 shared8(uint32_t at) {
  uint2 x;
  asm volatile("ld.shared.v2.b32 {%0, %1}, [%2];" : "=r"(x.x), "=r"(x.y) : "r"(at));
  return x;
}
__device__ __forceinline__ uint32_t shared4(uint32_t at) {
  uint32_t x;
  asm volatile("ld.shared.b32 %0, [%1];" : "=r"(x) : "r"(at));
  return x;
}
__device__ __forceinline__ uint32_t shared2(uint32_t at) {
  uint32_t x;
  asm volatile("{\n\t.reg .u16 h;\n\tld.shared.u16 h, [%1];\n\tcvt.u32.u16 %0, h;\n\t}" : "=r"(x) : "r"(at));
  return x;
}
__device__ __forceinline__ uint32_t shared1(uint32_t at) {
  uint32_t x;
  asm volatile("{\n\t.reg .u16 h;\n\tld.shared.u8 h, [%1];\n\tcvt.u32.u16 %0, h;\n\t}" : "=r"(x) : "r"(at));
  return x;
}

// A row's sums over parts of a unit, by a warp: parts i0, i0 + STEP, .. of `count`, in the
// slots slot_of(i), row `in` of each.  A lane has E consecutive elements.
template <int DK>
struct RowSum {
  static constexpr int E = DK / 32;
  float m = -INFINITY, l = 0.f, r = 0.f, o[E] = {};
};
template <int DK, int STEP, int BATCH, typename SlotOf>
__device__ __forceinline__ RowSum<DK> sum_parts(const Params& p, int in, int i0, int count, SlotOf slot_of) {
  constexpr int E = DK / 32;
  const int lane = threadIdx.x & 31;
  RowSum<DK> a;
  for (; i0 < count; i0 += 32 * STEP) {
    // lane j: part i0 + j STEP
    const int mine = i0 + lane * STEP, some = min(32, (count - i0 + STEP - 1) / STEP);
    float4 ml = make_float4(-INFINITY, 0.f, 0.f, 0.f);
    if (mine < count) ml = __ldcg(p.slot_ml + slot_of(mine) * p.slot_rows + in);
    float x[BATCH][E];
    const auto load = [&](int j0) {
#pragma unroll
      for (int j = 0; j < BATCH; ++j)
        if (j0 + j < some) {
          const float* from = p.slot_o + (slot_of(i0 + (j0 + j) * STEP) * p.slot_rows + in) * DK + lane * E;
          if constexpr (E == 4) {
            const float4 y = __ldcg(reinterpret_cast<const float4*>(from));
            x[j][0] = y.x, x[j][1] = y.y, x[j][2] = y.z, x[j][3] = y.w;
          } else {
            const float2 y = __ldcg(reinterpret_cast<const float2*>(from));
            x[j][0] = y.x, x[j][1] = y.y;
          }
        }
    };
    load(0);
    float top = ml.x;
#pragma unroll
    for (int d = 1; d < 32; d *= 2) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
    const float to = fmaxf(a.m, top), base = to == -INFINITY ? 0.f : to, f = ex2(a.m - base), w = ex2(ml.x - base);
    float ls = w * ml.y, rr = w * ml.z;
#pragma unroll
    for (int d = 1; d < 32; d *= 2) {
      ls += __shfl_xor_sync(0xffffffffu, ls, d);
      rr += __shfl_xor_sync(0xffffffffu, rr, d);
    }
    a.m = to;
    a.l = fmaf(a.l, f, ls);
    a.r = fmaf(a.r, f, rr);
#pragma unroll
    for (int e = 0; e < E; ++e) a.o[e] *= f;
    for (int j0 = 0; j0 < some; j0 += BATCH) {
      if (j0 > 0) load(j0);
#pragma unroll
      for (int j = 0; j < BATCH; ++j) {
        // (a part without weight too: what it has of NaN stays)
        const float wj = __shfl_sync(0xffffffffu, w, j0 + j);
        if (j0 + j < some)
#pragma unroll
          for (int e = 0; e < E; ++e) a.o[e] = fmaf(wj, x[j][e], a.o[e]);
      }
    }
  }
  return a;
}
template <int DK>
__device__ __forceinline__ void finish_row(const Params& p, int b, int h, int r, RowSum<DK>& a, float other) {
  const int lane = threadIdx.x & 31;
  __syncwarp();
  if constexpr (DK == 128) {
    finish<4>(p, b, h, r, lane * 4, a.m, a.l, a.r, a.o, other, lane == 0);
  } else {
    // two lanes' elements in one of them
    float v[4] = {a.o[0], a.o[1], __shfl_down_sync(0xffffffffu, a.o[0], 1), __shfl_down_sync(0xffffffffu, a.o[1], 1)};
    if (lane % 2 == 0) finish<4>(p, b, h, r, lane * 2, a.m, a.l, a.r, v, other, lane == 0);
  }
}

// PLAIN: heads of DK elements; else of fewer, whose rows are not of whole 16 bytes.
// SMALL: a unit is a CTA's, whose warps share its tiles out and merge their parts.
template <int DK, int NT, bool PLAIN, bool SMALL>
__global__ void __launch_bounds__(kThreads, attend4_blocks(NT, PLAIN)) attend4_kernel(const __grid_constant__ Params p) {
  constexpr int KS = DK / 16;              // steps of S's sum, m-tiles of O
  constexpr int RB = kRowBytes<DK>, NS = kStages<DK>;
  constexpr int SB = NT == 1 ? kSubs : 1;  // instructions' entries between two looks at the maximum
  extern __shared__ __align__(128) uint8_t smem[];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, t = lane & 3;
  uint8_t* ring = smem + warp * kWarpBytes<DK, NT>;
  uint2* s_q = reinterpret_cast<uint2*>(ring + NS * kStageBytes<DK>);            // [NT][KS][32]
  pdl_launch_dependents();
  pdl_wait();

  const int me = blockIdx.x * kWarps + warp;
  Line line;
  uint32_t begin = 0, end = 1;
  Cursor<kTile, kStart> cur;
  if constexpr (SMALL) {
    const int per_seq = p.Hkv * p.blocks;
    cur.b = blockIdx.x / per_seq;
    cur.u = blockIdx.x - cur.b * per_seq;
    cur.at = 0;
    cur.n = used(p, cur.b);
    cur.nt = ceil_div(cur.n, kTile);
    cur.j = cur.nt * warp / kWarps;
    cur.j1 = cur.nt * (warp + 1) / kWarps;
    if (cur.j == cur.j1 && (cur.nt > 0 || warp > 0)) end = 0;  // (without entries: warp 0's)
  } else {
    const Start<kTile, kStart> start = start_of<kTile, kStart, kThreads>(p, reinterpret_cast<uint32_t*>(smem), me, gridDim.x * kWarps);
    line = start.line;
    begin = start.begin;
    end = start.end;
    cur = start.cur;
    if (begin >= end) return;
  }
  [[maybe_unused]] const Cursor<kTile, kStart> unit = cur;       // (SMALL)

  // ---- tiles on their way ---------------------------------------------------------
  const sp_kv4 &k4 = p.c.k4, &v4 = p.c.v4;
  const int nbytes = PLAIN ? RB : p.D / 2, groups = PLAIN ? DK / 16 : p.D / 16;
  Cursor<kTile, kStart> f = cur;                          // of the tile to be fetched
  // A lane copies 16 bytes of every kCopyRows-th entry of a tile, from copy_row on.
  // Scales: lane l has those of entry l.
  constexpr int C = RB / 16, kCopyRows = 32 / C;
  const int copy_row = lane / C, copy_byte = lane % C * 16;
  const uint32_t ring_u32 = smem_u32(ring), copy_to = ring_u32 + place_of<DK>(copy_row, copy_byte);
  const uint8_t *kp, *vp, *ks, *vs;
  const auto enter_unit = [&]() {
    while (f.j >= f.j1 && f.at < end) f.next(p, begin, end);
    if (f.at >= end) return;
    const int h = p.by_blocks(f.u);
    const int64_t e = (int64_t)f.j * kTile;
    kp = k4.codes + f.b * k4.batch + h * k4.head + (e + copy_row) * k4.entry + copy_byte;
    vp = v4.codes + f.b * v4.batch + h * v4.head + (e + copy_row) * v4.entry + copy_byte;
    ks = k4.scales + f.b * k4.scales_batch + h * k4.scales_head + (e + lane) * k4.scales_entry;
    vs = v4.scales + f.b * v4.scales_batch + h * v4.scales_head + (e + lane) * v4.scales_entry;
  };
  ScaleRow<DK, PLAIN> k_scales, v_scales;  // of the tile fetched last
  // Rows of a head one after the other.
  const bool lined = PLAIN && k4.entry == RB && v4.entry == RB;
  const auto fetch = [&](int stage) {
    if (f.j < f.j1) {
      const uint32_t to = copy_to + stage * kStageBytes<DK>;
      const int left = f.n - f.j * kTile;  // entries from the tile's first on
      if (lined && left >= kTile) {
#pragma unroll
        for (int i = 0; i < kTile / kCopyRows; ++i) {
          copy_async<16>(to + i * kCopyRows * RB, kp + i * kCopyRows * RB);
          copy_async<16>(to + (kTile + i * kCopyRows) * RB, vp + i * kCopyRows * RB);
        }
      } else if (PLAIN || nbytes % 16 == 0) {
        const uint8_t *kr = kp, *vr = vp;
#pragma unroll
        for (int i = 0; i < kTile / kCopyRows; ++i) {
          if (copy_row + i * kCopyRows < left && (PLAIN || copy_byte < nbytes)) {
            copy_async<16>(to + i * kCopyRows * RB, kr);
            copy_async<16>(to + (kTile + i * kCopyRows) * RB, vr);
          }
          kr += kCopyRows * k4.entry;
          vr += kCopyRows * v4.entry;
        }
      } else {
        // 8 bytes of every kRows8-th entry
        constexpr int C8 = RB / 8, kRows8 = 32 / C8;
        const int row = lane / C8, byte = lane % C8 * 8;
        const uint8_t* kr = kp + (row - copy_row) * k4.entry + (byte - copy_byte);
        const uint8_t* vr = vp + (row - copy_row) * v4.entry + (byte - copy_byte);
        const uint32_t to8 = ring_u32 + stage * kStageBytes<DK>;
#pragma unroll
        for (int i = 0; i < kTile / kRows8; ++i) {
          if (row + i * kRows8 < left && byte < nbytes) {
            copy_async<8>(to8 + place_of<DK>(row + i * kRows8, byte), kr);
            copy_async<8>(to8 + kTile * RB + place_of<DK>(row + i * kRows8, byte), vr);
          }
          kr += kRows8 * k4.entry;
          vr += kRows8 * v4.entry;
        }
      }
      k_scales.load(ks, groups, lane < left);
      v_scales.load(vs, groups, lane < left);
      if (++f.j < f.j1) {
        kp += kTile * k4.entry;
        vp += kTile * v4.entry;
        ks += kTile * k4.scales_entry;
        vs += kTile * v4.scales_entry;
      } else {
        enter_unit();
      }
    }
    copy_commit();
  };
  const auto store_scales = [&](int stage, const ScaleRow<DK, PLAIN>& k, const ScaleRow<DK, PLAIN>& v) {
    uint8_t* to = ring + stage * kStageBytes<DK> + 2 * kTile * RB + lane * 8;
    *reinterpret_cast<uint2*>(to) = k.value(groups);
    *reinterpret_cast<uint2*>(to + kTile * 8) = v.value(groups);
  };
  k_scales.load(nullptr, groups, false);
  v_scales = k_scales;
  // the first unit's queries before its tiles, which would hold them up
  const auto skipped = [&]() { return cur.j >= cur.j1 && (cur.nt > 0 || cur.at < begin); };
  uint2 x[NT][KS];
  const auto load_queries = [&]() {
    const int h = p.by_blocks(cur.u), row0 = (cur.u - h * p.blocks) * p.block_rows, rows = min(p.block_rows, p.R - row0);
#pragma unroll
    for (int i = 0; i < NT; ++i) load_query<DK>(p, cur.b, h, row0 + i * 8 + g, i * 8 + g < rows, t, x[i]);
  };
  while (cur.at < end && skipped()) cur.next(p, begin, end);
  if (cur.at < end) load_queries();
  enter_unit();
  ScaleRow<DK, PLAIN> k_first[NS - 1], v_first[NS - 1];        // (stored when the queries are there)
#pragma unroll
  for (int i = 0; i < NS - 1; ++i) {
    fetch(i);
    k_first[i] = k_scales, v_first[i] = v_scales;
  }
  bool first_unit = true;
  // Where a lane's operands and scales lie in a tile.  (Kept: the compiler would rather
  // make them anew for every tile.)
  uint32_t k_off = place_of<DK>(entry_of(g), t * (RB / 4)), ks_off = 2 * kTile * RB + entry_of(g) * 8 + t * (DK / 64);
  uint32_t v_off = kTile * RB + place_of<DK>(t, g * (RB / 8)), v4_off = kTile * RB + place_of<DK>(t + 4, g * (RB / 8));
  uint32_t vs_off = 2 * kTile * RB + (kTile + t) * 8 + (DK == 128 ? g : g / 2);
  asm volatile("" : "+r"(k_off), "+r"(ks_off), "+r"(v_off), "+r"(v4_off), "+r"(vs_off));
  int stage = 0, ahead = NS - 1;           // places in the ring: of the tile, of the tile to be fetched

  for (; cur.at < end; cur.next(p, begin, end)) {
    const int b = cur.b, n = cur.n, nt = cur.nt, h = p.by_blocks(cur.u), block = cur.u - h * p.blocks;
    if (skipped()) continue;
    if (!first_unit) load_queries();
    const int row0 = block * p.block_rows, rows = min(p.block_rows, p.R - row0);

    // ---- the query rows ---------------------------------------------------------
    uint2 q[KS];                           // of one n-tile
    float c2[NT][2];                       // of the rows 2t, 2t + 1 of each n-tile
    int far[NT][2];                        // entries that they see
#pragma unroll
    for (int i = 0; i < NT; ++i) {
      const float by = make_query<DK>(p, x[i]);
#pragma unroll
      for (int j = 0; j < KS; ++j) {
        if (NT == 1) q[j] = x[i][j];
        else s_q[(i * KS + j) * 32 + lane] = x[i][j];
      }
      // (lane 4 r has row r's)
#pragma unroll
      for (int e2 = 0; e2 < 2; ++e2) {
        c2[i][e2] = __shfl_sync(0xffffffffu, by, 4 * (2 * t + e2));
        const int r2 = i * 8 + 2 * t + e2;
        far[i][e2] = r2 < rows && p.c.causal ? n - (p.c.T - 1 - (int)p.by_G(row0 + r2)) : n;
      }
    }
    const int all_see = n - (p.c.causal ? p.c.T - 1 : 0);
    if (first_unit) {
#pragma unroll
      for (int i = 0; i < NS - 2; ++i) store_scales(i, k_first[i], v_first[i]);
      first_unit = false;
    }
    uint32_t poison = 0;                   // lane r: groups of which row r sees a NaN value

    // ---- the unit's tiles -------------------------------------------------------
    float o[NT][KS][4], sum_r[NT][4];
    f32x2 l[NT], minus_m[NT];              // of the rows 2t, 2t + 1: sums, the maximum that the reference has
    float lag[NT][2];                      // from how far above it on that follows: kLag, at first from anywhere
#pragma unroll
    for (int i = 0; i < NT; ++i) {
#pragma unroll
      for (int j = 0; j < KS; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[i][j][e] = 0.f;
#pragma unroll
      for (int e = 0; e < 4; ++e) sum_r[i][e] = 0.f;
      lag[i][0] = lag[i][1] = -INFINITY;
      l[i] = minus_m[i] = pair(0.f, 0.f);
    }
#pragma unroll 1
    for (int tile = cur.j; tile < cur.j1; ++tile) {
      // (the place before this one's that is to be fetched to)
      store_scales(ahead == 0 ? NS - 1 : ahead - 1, k_scales, v_scales);
      copy_wait<NS - 2>();
      __syncwarp();
      // (the place of the tile before, which every lane has left)
      fetch(ahead);
      const uint32_t place = ring_u32 + stage * kStageBytes<DK>;
      uint8_t* place_s = ring + stage * kStageBytes<DK> + 2 * kTile * RB;
      stage = stage + 1 == NS ? 0 : stage + 1;
      ahead = ahead + 1 == NS ? 0 : ahead + 1;
      // A NaN scale (exponent 31) of a value must not meet a probability of 0 of a row
      // that does not see its entry: it becomes 0, and the rows that do see it
      // remember the group.  (Where all rows see all entries it makes them NaN itself.)
      if (tile * kTile + kTile > all_see) {
        uint2* at = reinterpret_cast<uint2*>(place_s + (kTile + lane) * 8);
        const uint2 x = *at;
        const uint32_t bad[2] = {nan_scales(x.x), nan_scales(x.y)};
        if (__any_sync(0xffffffffu, bad[0] | bad[1])) {
          *at = make_uint2(x.x & ~(bad[0] / 128 * 255), x.y & ~(bad[1] / 128 * 255));
          const int my_far = lane >= rows ? 0 : p.c.causal ? n - (p.c.T - 1 - (int)p.by_G(row0 + lane)) : n;
          const uint32_t mask = groups_of(bad);
          for (int e = 0; e < kTile; ++e) {
            const uint32_t m = __shfl_sync(0xffffffffu, mask, e);
            if (tile * kTile + e < my_far) poison |= m;
          }
          __syncwarp();
        }
      }
#pragma unroll 1
      for (int sub0 = 0; sub0 < kSubs; sub0 += SB) {
      // S^T = K Q^T
      float s[SB][NT][4];
#pragma unroll
      for (int sub = 0; sub < SB; ++sub) {
#pragma unroll
        for (int i = 0; i < NT; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e) s[sub][i][e] = 0.f;
        constexpr int W = DK / 32;         // words of an entry: four code pairs each
        uint32_t w[2][W], sc2[2];
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          const int below = 16 * (sub0 + sub) + 8 * half;
          if constexpr (DK == 128) {
            const uint4 x = shared16(place + k_off + below * RB);
            w[half][0] = x.x, w[half][1] = x.y, w[half][2] = x.z, w[half][3] = x.w;
            sc2[half] = scales_half2(shared2(place + ks_off + below * 8));
          } else {
            const uint2 x = shared8(place + k_off + below * RB);
            w[half][0] = x.x, w[half][1] = x.y;
            sc2[half] = shared1(place + ks_off + below * 8) << 7;
          }
        }
#pragma unroll
        for (int i = 0; i < W; ++i) {
          uint32_t lo[4], hi[4];
          codes_to_half(w[0][i], lo);
          codes_to_half(w[1][i], hi);
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            lo[k] = i < 2 ? mul_half2_by<0>(lo[k], sc2[0]) : mul_half2_by<1>(lo[k], sc2[0]);
            hi[k] = i < 2 ? mul_half2_by<0>(hi[k], sc2[1]) : mul_half2_by<1>(hi[k], sc2[1]);
          }
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            const uint32_t a[4] = {lo[2 * k], hi[2 * k], lo[2 * k + 1], hi[2 * k + 1]};
#pragma unroll
            for (int c = 0; c < NT; ++c) {
              const uint2 qq = NT == 1 ? q[2 * i + k] : s_q[(c * KS + 2 * i + k) * 32 + lane];
              mma(s[sub][c], a, qq.x, qq.y);
            }
          }
        }
      }
      // probabilities
      if (tile * kTile + 16 * (sub0 + SB) > all_see) {
        const int e0 = tile * kTile + entry_of(g);               // of s[0][.][0 .. 1]; e0 + 8 of the others
#pragma unroll
        for (int sub = 0; sub < SB; ++sub)
#pragma unroll
          for (int i = 0; i < NT; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if (e0 + 16 * (sub0 + sub) + (e >> 1) * 8 >= far[i][e & 1]) s[sub][i][e] = -INFINITY;
      }
      bool grow = false;
      float top[NT][2];
#pragma unroll
      for (int i = 0; i < NT; ++i)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          top[i][e] = fmaxf(s[0][i][e], s[0][i][e + 2]);
#pragma unroll
          for (int sub = 1; sub < SB; ++sub) top[i][e] = fmaxf(top[i][e], fmaxf(s[sub][i][e], s[sub][i][e + 2]));
          grow |= (top[i][e] + (e ? halves(minus_m[i]).y : halves(minus_m[i]).x)) * c2[i][e] > lag[i][e];
        }
      if (__any_sync(0xffffffffu, grow)) {
#pragma unroll
        for (int i = 0; i < NT; ++i) {
          float a[2], m[2] = {halves(minus_m[i]).x, halves(minus_m[i]).y};
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            float x = top[i][e];
#pragma unroll
            for (int d = 4; d < 32; d *= 2) x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, d));
            a[e] = 1.f;
            const float by = (x + m[e]) * c2[i][e];
            if (by > lag[i][e]) {
              a[e] = lag[i][e] == -INFINITY ? 0.f : ex2(-by);
              lag[i][e] = kLag;
              m[e] = -x;
            }
          }
          minus_m[i] = pair(m[0], m[1]);
          l[i] = fma2(l[i], pair(a[0], a[1]), pair(0.f, 0.f));
#pragma unroll
          for (int e = 0; e < 4; ++e) sum_r[i][e] *= a[e & 1];
#pragma unroll
          for (int j = 0; j < KS; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) o[i][j][e] *= a[e & 1];
        }
      }
      uint32_t pb[SB][NT][2];
#pragma unroll
      for (int i = 0; i < NT; ++i) {
        const f32x2 by = pair(c2[i][0], c2[i][1]), lift = pair(kLift, kLift);
        f32x2 sum[2 * SB];
#pragma unroll
        for (int sub = 0; sub < SB; ++sub)
#pragma unroll
          for (int half = 0; half < 2; ++half) {
            // (the difference first, which is exact near the maximum: of large scores the product
            // is off by more than half precision has room for)
            const float2 x = halves(fma2(add2(pair(s[sub][i][2 * half], s[sub][i][2 * half + 1]), minus_m[i]), by, lift));
            const float2 y = make_float2(ex2(x.x), ex2(x.y));
            sum[2 * sub + half] = pair(y.x, y.y);
            pb[sub][i][half] = transpose8(pack_half2(y.x, y.y));
          }
#pragma unroll
        for (int d = SB; d > 0; d /= 2)
#pragma unroll
          for (int j = 0; j < d; ++j) sum[j] = add2(sum[j], sum[j + d]);
        l[i] = add2(l[i], sum[0]);
      }
      // O^T += V^T P^T
#pragma unroll
      for (int sub = 0; sub < SB; ++sub) {
        uint32_t w[4][KS / 4], sb[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int below = 16 * (sub0 + sub) + 8 * (i >> 1);
          const uint32_t from = place + (i & 1 ? v4_off : v_off) + below * RB;
          if constexpr (DK == 128) {
            const uint2 x = shared8(from);
            w[i][0] = x.x, w[i][1] = x.y;
          } else {
            w[i][0] = shared4(from);
          }
          sb[i] = shared1(place + vs_off + (16 * (sub0 + sub) + 4 * i) * 8);
        }
        const uint32_t s01 = sb[0] << 7 | sb[1] << 23, s23 = sb[2] << 7 | sb[3] << 23;
#pragma unroll
        for (int i = 0; i < KS / 4; ++i) {
          // pairs of entries instead of pairs of elements: even elements, odd ones
          uint32_t y[4][4];
          constexpr uint32_t low = 0x0f0f0f0fu;
          codes_to_half(select_bits<low>(w[0][i], w[1][i] << 4), y[0]);
          codes_to_half(select_bits<low>(w[0][i] >> 4, w[1][i]), y[1]);
          codes_to_half(select_bits<low>(w[2][i], w[3][i] << 4), y[2]);
          codes_to_half(select_bits<low>(w[2][i] >> 4, w[3][i]), y[3]);
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const uint32_t a[4] = {mul_half2(y[0][k], s01), mul_half2(y[1][k], s01), mul_half2(y[2][k], s23),
                                   mul_half2(y[3][k], s23)};
#pragma unroll
            for (int c = 0; c < NT; ++c) mma(o[c][4 * i + k], a, pb[sub][c][0], pb[sub][c][1]);
          }
        }
        const uint32_t ones[4] = {kOnes, kOnes, kOnes, kOnes};
#pragma unroll
        for (int c = 0; c < NT; ++c) mma(sum_r[c], ones, pb[sub][c][0], pb[sub][c][1]);
      }
      }
      __syncwarp();
    }

    // ---- what the warp has of the unit ------------------------------------------
    const bool begins = cur.j == 0, whole = begins && cur.j1 == nt;
    const int64_t slot = 2 * (int64_t)me + (cur.at >= begin ? 1 : 0);            // (begun before, or here)
    if (!SMALL && lane == 0 && begins)
      p.units[(int64_t)b * p.Hkv * p.blocks + cur.u] = make_int2(whole ? -1 : (int)slot, whole ? me : worker_of(p, line, cur.at + kStart + nt - 1, me));
    const bool poisoned = __any_sync(0xffffffffu, poison != 0);
    float other[NT][2];
#pragma unroll
    for (int i = 0; i < NT; ++i)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int r = i * 8 + 2 * t + e;
        other[i][e] = whole && r < rows ? other_of(p, b, h, row0 + r) : -INFINITY;
      }
    __syncwarp();
#pragma unroll
    for (int i = 0; i < NT; ++i) {
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        float x = e ? halves(l[i]).y : halves(l[i]).x;
#pragma unroll
        for (int d = 4; d < 32; d *= 2) x += __shfl_xor_sync(0xffffffffu, x, d);
        const int r = i * 8 + 2 * t + e;
        float v[DK / 8];
#pragma unroll
        for (int j = 0; j < KS; ++j) v[2 * j] = o[i][j][e], v[2 * j + 1] = o[i][j][e + 2];
        if (poisoned) {
          const uint32_t bits = __shfl_sync(0xffffffffu, poison, r);
          if (bits >> (g * (DK / 8) / 16) & 1u)
#pragma unroll
            for (int j = 0; j < DK / 8; ++j) v[j] = NAN;
        }
        const float ref = lag[i][e] == -INFINITY ? -INFINITY : fmaf(-(e ? halves(minus_m[i]).y : halves(minus_m[i]).x), c2[i][e], -kLift);
        if (r < rows) {
          if (whole) {
            finish<DK / 8>(p, b, h, row0 + r, g * (DK / 8), ref, x, sum_r[i][e], v, other[i][e], g == 0);
          } else {
            if (g == 0) p.slot_ml[slot * p.slot_rows + r] = make_float4(ref, x, sum_r[i][e], 0.f);
            float* to = p.slot_o + (slot * p.slot_rows + r) * DK + g * (DK / 8);
#pragma unroll
            for (int j = 0; j < DK / 8; j += 4) *reinterpret_cast<float4*>(to + j) = make_float4(v[j], v[j + 1], v[j + 2], v[j + 3]);
          }
        }
      }
    }
    __syncwarp();                          // (the queries' place)
  }
  copy_wait<0>();
  if constexpr (SMALL) {
    __syncthreads();
    const int parts = min(unit.nt, kWarps);
    if (parts > 1) {
      const int h = p.by_blocks(unit.u), row0 = (unit.u - h * p.blocks) * p.block_rows, rows = min(p.block_rows, p.R - row0);
      // the i-th warp that has tiles
      const auto warp_of = [&](int i) { return unit.nt >= kWarps ? i : (kWarps * (i + 1) + unit.nt - 1) / unit.nt - 1; };
      for (int r = warp; r < rows; r += kWarps) {
        const float other = other_of(p, unit.b, h, row0 + r);
        RowSum<DK> a = sum_parts<DK, 1, kWarps>(p, r, 0, parts,
                                                [&](int i) { return 2 * ((int64_t)blockIdx.x * kWarps + warp_of(i)) + 1; });
        finish_row<DK>(p, unit.b, h, row0 + r, a, other);
      }
    }
  }
}

// Rows of units that several workers have parts of: WPR warps a row.
//
// It does not let the next kernel in before it ends: its blocks beside the next call's break an
// SM's registers into pieces, the last of four CTAs of attend4_kernel finds no room, and
// begins when others end (chats 38.7 us instead of 31, drafts 46 instead of 38).
template <int DK, int WPR>
__global__ void __launch_bounds__(32 * WPR) merge4_kernel(const __grid_constant__ Params p) {
  constexpr int E = DK / 32;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  pdl_wait();
  const int64_t id = blockIdx.x;           // (sequence, K/V head, row)
  const int64_t bh = id / p.R;
  const int r = (int)(id - bh * p.R), block = r / p.block_rows, in = r - block * p.block_rows;
  const int b = (int)(bh / p.Hkv), h = (int)(bh - (int64_t)b * p.Hkv);
  const int2 unit = __ldcg(p.units + bh * p.blocks + block);
  if (unit.x < 0 || !parts_within(unit.x, unit.y, p.workers)) return;
  const float other = other_of(p, b, h, r);
  const int first = unit.x >> 1, parts = (int)p.by_side(max(0, unit.y - first)) + 1;
  RowSum<DK> a = sum_parts<DK, WPR, 8>(p, in, warp, parts,
                                       [&](int i) { return i == 0 ? (int64_t)unit.x : 2 * (first + (int64_t)i * p.side); });
  if constexpr (WPR > 1) {
    __shared__ float s_ml[WPR][3], s_o[WPR][DK];
#pragma unroll
    for (int e = 0; e < E; ++e) s_o[warp][lane * E + e] = a.o[e];
    if (lane == 0) {
      s_ml[warp][0] = a.m;
      s_ml[warp][1] = a.l;
      s_ml[warp][2] = a.r;
    }
    __syncthreads();
    if (warp > 0) return;
    float to = a.m;
    for (int w = 1; w < WPR; ++w) to = fmaxf(to, s_ml[w][0]);
    const float base = to == -INFINITY ? 0.f : to, f = ex2(a.m - base);
    a.l *= f, a.r *= f;
#pragma unroll
    for (int e = 0; e < E; ++e) a.o[e] *= f;
    for (int w = 1; w < WPR; ++w) {
      const float x = ex2(s_ml[w][0] - base);
      a.l = fmaf(x, s_ml[w][1], a.l);
      a.r = fmaf(x, s_ml[w][2], a.r);
#pragma unroll
      for (int e = 0; e < E; ++e) a.o[e] = fmaf(x, s_o[w][lane * E + e], a.o[e]);
    }
    a.m = to;
  }
  finish_row<DK>(p, b, h, r, a, other);
}

// ---- host ---------------------------------------------------------------------
template <int DK, int WPR>
cudaError_t launch_merge(const Params& p, cudaStream_t s) {
  return launch_pdl(merge4_kernel<DK, WPR>, dim3((unsigned)((int64_t)p.c.B * p.Hkv * p.R)), dim3(32 * WPR), 0, s, p);
}

template <int DK, int NT, bool PLAIN, bool SMALL>
cudaError_t launch_t(const Params& p, int dev, int grid, cudaStream_t s) {
  static PerDevice attr;
  constexpr size_t bytes = (size_t)kWarps * kWarpBytes<DK, NT>;
  const cudaError_t e = attr.once(dev, []() {
    return cudaFuncSetAttribute(attend4_kernel<DK, NT, PLAIN, SMALL>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
  });
  if (e != cudaSuccess) return e;
  return launch_pdl(attend4_kernel<DK, NT, PLAIN, SMALL>, dim3((unsigned)grid), dim3(kThreads), bytes, s, p);
}

}  // namespace

int64_t attend4_tiles(const Cache4Shape& s, const sp_attend4& c) {
  return (int64_t)c.B * s.Hkv * plan4_of(c.T * (s.Hq / s.Hkv), s.D, 1).blocks * (kStart + ceil_div(s.capacity, kTile));
}

cudaError_t launch_attend4(const Cache4Shape& s, const sp_attend4& c, uint8_t* ws, size_t slots, int* err, int fault,
                           cudaStream_t stream) {
  int dev = 0, sms = 0;
  cudaError_t e = current_device(&dev, &sms);
  if (e != cudaSuccess) return e;
  Params p;
  p.c = c;
  p.Hkv = s.Hkv;
  p.G = s.Hq / s.Hkv;
  p.D = s.D;
  p.capacity = s.capacity;
  p.R = c.T * p.G;
  const Plan4 plan = plan4_of(p.R, s.D, sms);
  p.blocks = plan.blocks;
  p.block_rows = plan.rows;
  p.by_blocks = Divide(p.blocks);
  p.by_G = Divide(p.G);
  // The units of the same entries' query rows walk side by side, and where an entry's heads lie
  // side by side theirs too: memory's 64 bytes that several heads' scales are in are then in
  // the L2 (64 sequences of 4096 to 16384 entries, 8 heads: 136 us instead of 262, 113 by
  // bytes; 64 chats, 4 heads: 27.2 instead of 29.9).  Not where more than a tenth of the workers
  // would be left over.
  const bool adjacent = c.k4.head < c.k4.entry && c.v4.head < c.v4.entry;
  const auto fits = [&](int side) { return plan.workers % side * 10 <= plan.workers; };
  p.side = adjacent && fits(s.Hkv * p.blocks) ? s.Hkv * p.blocks : fits(p.blocks) ? p.blocks : 1;
  p.on_line = s.Hkv * p.blocks / p.side;
  p.by_side = Divide(p.side);
  p.bf16 = s.dtype == SP_BF16;
  // (the product in 64 bits, whose range no scale leaves)
  p.c2 = 2.f * (float)std::frexp((double)c.scale * (double)kLog2e, &p.c2_power);
  --p.c2_power;
  p.err = err;
  p.fault = fault;
  p.limit = fault == kFaultStall ? kStallWaitCycles : kWaitLimitCycles;
  p.workers = plan.workers;
  p.slot_rows = 8 * plan.NT;
  const Slots4 at = slots4_of(plan);
  p.units = reinterpret_cast<int2*>(ws);
  p.slot_ml = reinterpret_cast<float4*>(ws + slots + at.ml);
  p.slot_o = reinterpret_cast<float*>(ws + slots + at.o);
  const int64_t units = (int64_t)c.B * s.Hkv * plan.blocks;
  // Units that a CTA has by itself need neither the line nor the merge of another
  // kernel (one sequence, 4 heads, 60 of 512 entries: 4.6 us instead of 8.0).
  // Above 768 entries a CTA is too little for a unit: with 1024 entries 64 sequences take
  // 15.7 us instead of 14.2, with 2048 one takes 17.9 instead of 11.5.
  const bool small = !plan.by_ctas && s.capacity <= kSmallTiles * kTile && units * kWarps <= plan.workers;
  const int grid = small ? (int)units : plan.workers / kWarps;
  const bool wide = plan.wide, plain = plan.plain;
  const auto launch = [&](auto is_small) {
    constexpr bool S = decltype(is_small)::value;
    return wide             ? (plain ? launch_t<128, 1, true, S>(p, dev, grid, stream) : launch_t<128, 1, false, S>(p, dev, grid, stream))
           : plan.NT == 1 ? (plain ? launch_t<64, 1, true, S>(p, dev, grid, stream) : launch_t<64, 1, false, S>(p, dev, grid, stream))
           : plain        ? launch_t<64, 2, true, S>(p, dev, grid, stream)
                          : launch_t<64, 2, false, S>(p, dev, grid, stream);
  };
  if (small) return launch(std::true_type());
  e = plan.by_ctas ? launch_attend4_rows(p, dev, sms, stream) : launch(std::false_type());
  if (e != cudaSuccess) return e;
  // Warps a row by its parts, if all sequences are of a length.  1, 8 and 32 of them, us of
  // the call: 608 parts (one sequence of 65536 entries) 55, 25, 22; 152 parts 48, 38, 38; 38
  // parts (16 sequences of 8192) 27.4, 25.0, 29.6; 28 parts (8 of 8192, 15 rows) 26.9, 27.2, 44;
  // 9 parts (64 of 8192) 62, 64, 76.
  const int64_t parts = plan.workers / units;
  const auto merge = [&](auto wpr) {
    constexpr int W = decltype(wpr)::value;
    return wide ? launch_merge<128, W>(p, stream) : launch_merge<64, W>(p, stream);
  };
  return parts >= 128  ? merge(std::integral_constant<int, 32>())
         : parts >= 16 ? merge(std::integral_constant<int, 8>())
                       : merge(std::integral_constant<int, 1>());
}

}  // namespace sp
