// sp_attn4_rows.cu -- attention over a cache held in 4 bits for units of many query
// rows (see sp_attn4.cu for the operands and for the line that the work is on): what
// codes cost to be made half precision is shared by up to 64 rows, so the four warps
// of a CTA work on one unit together, in tiles of 64 entries.
//
//   S^T = K Q^T   warp w: entries 16 w .. 16 w + 15, all rows
//   P^T           from each warp's registers through shared memory to all warps
//   O^T = V^T P^T warp w: the w-th quarter of the elements, all entries
//
// so that no code is decoded twice, and a warp holds O of a quarter of the elements
// only.  The reference of a row's exponentials is the CTA's; it is looked at after
// the probabilities are made, at the barrier that hands them over, and they are made
// again in the few tiles where it has to change.
#include "sp_attn4.cuh"

namespace sp {
namespace {

using Params = Attend4Params;
constexpr int kTile = 64;
constexpr float kNone = 1.7e38f;           // negative reference of a row without a score yet: any score is above it

constexpr int ctas_per_sm(int NT) { return NT <= 4 ? 4 : 3; }
template <int DK> constexpr int kStageBytes = 2 * kTile * kRowBytes<DK> + 2 * kTile * 8;
constexpr int kStages = 3;
template <int DK, int NT> constexpr int kQueryBytes = NT * (DK / 32) * 32 * 16;
template <int NT> constexpr int kProbBytes = kWarps * (NT / 2) * 32 * 16;
template <int DK, int NT> constexpr int kSmem = kStages * kStageBytes<DK> + kQueryBytes<DK, NT> + kProbBytes<NT>;
static_assert(3 * (kSmem<128, 8> + 5 * 1024) <= 228 * 1024 && 4 * (kSmem<128, 4> + 3 * 1024) <= 228 * 1024, "shared memory of an SM");
static_assert(kSmem<64, 2> >= (SPIKE_PROJ_CACHE_MAX_B + 1) * 4, "room for the costs before each sequence");

template <int DK, int NT>
__global__ void __launch_bounds__(kThreads, ctas_per_sm(NT)) attend4_rows_kernel(const __grid_constant__ Params p) {
  constexpr int KS = DK / 16, RB = kRowBytes<DK>, NS = kStages;
  constexpr int MT = DK / 64;              // m-tiles of O of a warp
  constexpr int OWN = (NT + 3) / 4;        // n-tiles whose rounded probabilities a warp adds up: warp, warp + 4
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ float4 s_row[NT][4];          // rows 2t, 2t + 1 of n-tile i: factors of scores, negative references
  __shared__ int2 s_far[NT][4];            // entries that they see
  __shared__ float s_top[kWarps][8 * NT], s_sum[8 * NT];       // (tops of a tile, sums of a unit)
  __shared__ uint32_t s_poison[8 * NT];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, t = lane & 3;
  uint4* s_q = reinterpret_cast<uint4*>(smem + NS * kStageBytes<DK>);            // [NT][KS / 2][32]
  uint4* s_p = reinterpret_cast<uint4*>(smem + NS * kStageBytes<DK> + kQueryBytes<DK, NT>);      // [4][NT / 2][32]
  pdl_launch_dependents();
  pdl_wait();

  const int me = blockIdx.x;
  const Start<kTile> start = start_of<kTile>(p, reinterpret_cast<uint32_t*>(smem), me, gridDim.x);
  const Line line = start.line;
  const uint32_t begin = start.begin, end = start.end;
  __syncthreads();
  if (begin >= end) return;
  Cursor<kTile> cur = start.cur;

  // ---- tiles on their way ---------------------------------------------------------
  const sp_kv4 &k4 = p.c.k4, &v4 = p.c.v4;
  const int nbytes = p.D / 2, groups = p.D / 16;
  Cursor<kTile> f = cur;                   // of the tile to be fetched
  // A thread copies 16 bytes of every kCopyRows-th entry of a tile, from copy_row on.
  // Scales: thread i has those of key i, i - 64 of its values.
  constexpr int C = RB / 16, kCopyRows = kThreads / C;
  const int copy_row = tid / C, copy_byte = tid % C * 16;
  const uint32_t ring_u32 = smem_u32(smem), copy_to = ring_u32 + place_of<DK>(copy_row, copy_byte);
  const sp_kv4& scale4 = tid < kTile ? k4 : v4;
  const uint8_t *kp = nullptr, *vp = nullptr, *sc = nullptr;
  const auto enter_unit = [&]() {
    while (f.j >= f.j1 && f.at < end) f.next(p, begin, end);
    if (f.at >= end) return;
    const int h = p.by_blocks(f.u);
    const int64_t e = (int64_t)f.j * kTile;
    kp = k4.codes + f.b * k4.batch + h * k4.head + (e + copy_row) * k4.entry + copy_byte;
    vp = v4.codes + f.b * v4.batch + h * v4.head + (e + copy_row) * v4.entry + copy_byte;
    sc = scale4.scales + f.b * scale4.scales_batch + h * scale4.scales_head + (e + tid % kTile) * scale4.scales_entry;
  };
  uint2 scales = make_uint2(0, 0);         // of the tile fetched last
  const auto fetch = [&](int stage) {
    if (f.j < f.j1) {
      const uint32_t to = copy_to + stage * kStageBytes<DK>;
      const int left = f.n - f.j * kTile;  // entries from the tile's first on
      if (nbytes % 16 == 0) {
        const uint8_t *kr = kp, *vr = vp;
        if (copy_byte < nbytes) {
#pragma unroll
          for (int i = 0; i < kTile / kCopyRows; ++i) {
            if (copy_row + i * kCopyRows < left) {
              copy_async<16>(to + i * kCopyRows * RB, kr);
              copy_async<16>(to + (kTile + i * kCopyRows) * RB, vr);
            }
            kr += kCopyRows * k4.entry;
            vr += kCopyRows * v4.entry;
          }
        }
      } else {
        constexpr int C8 = RB / 8;
        const uint8_t* kc = kp - copy_row * k4.entry - copy_byte;
        const uint8_t* vc = vp - copy_row * v4.entry - copy_byte;
        const uint32_t to8 = ring_u32 + stage * kStageBytes<DK>;
#pragma unroll 2
        for (int i = 0; i < kTile * C8 / kThreads; ++i) {
          const int e = (i * kThreads + tid) / C8, byte = (i * kThreads + tid) % C8 * 8;
          if (e < left && byte < nbytes) {
            copy_async<8>(to8 + place_of<DK>(e, byte), kc + e * k4.entry + byte);
            copy_async<8>(to8 + kTile * RB + place_of<DK>(e, byte), vc + e * v4.entry + byte);
          }
        }
      }
      scales = make_uint2(0, 0);
      if (tid % kTile < left) scales = row_scales(sc, groups);
      if (++f.j < f.j1) {
        kp += kTile * k4.entry;
        vp += kTile * v4.entry;
        sc += kTile * scale4.scales_entry;
      } else {
        enter_unit();
      }
    }
    copy_commit();
  };
  const auto store_scales = [&](int stage, uint2 x) {
    *reinterpret_cast<uint2*>(smem + stage * kStageBytes<DK> + 2 * kTile * RB + tid * 8) = x;
  };
  enter_unit();
  uint2 first_scales[NS - 1];              // (stored when the queries are there)
#pragma unroll
  for (int i = 0; i < NS - 1; ++i) {
    fetch(i);
    first_scales[i] = scales;
  }
  bool first_unit = true;
  int stage = 0, ahead = NS - 1;           // places in the ring: of the tile, of the tile to be fetched

  for (; cur.at < end; cur.next(p, begin, end)) {
    const int b = cur.b, n = cur.n, nt = cur.nt, h = p.by_blocks(cur.u), block = cur.u - h * p.blocks;
    if (cur.j >= cur.j1 && (nt > 0 || cur.at < begin)) continue;
    const int row0 = block * p.block_rows, rows = min(p.block_rows, p.R - row0);

    // ---- the query rows ---------------------------------------------------------
    __syncthreads();                       // (the unit before has left its place)
    if (tid < 8 * NT) s_poison[tid] = 0;
    for (int i = warp; i < NT; i += kWarps) {
      const int r = i * 8 + g;
      uint2 x[KS];
      const float down = load_query<DK>(p, b, h, row0 + r, r < rows, t, x);
#pragma unroll
      for (int j = 0; j < KS / 2; ++j)
        s_q[(i * (KS / 2) + j) * 32 + lane] = make_uint4(x[2 * j].x, x[2 * j].y, x[2 * j + 1].x, x[2 * j + 1].y);
      if (t == 0) {
        float* row = reinterpret_cast<float*>(&s_row[i][g >> 1]) + (g & 1);
        row[0] = down;
        row[2] = kNone;
        reinterpret_cast<int*>(&s_far[i][g >> 1])[g & 1] = r < rows && p.c.causal ? n - (p.c.T - 1 - (int)p.by_G(row0 + r)) : n;
      }
    }
    if (first_unit) {
#pragma unroll
      for (int i = 0; i < NS - 2; ++i) store_scales(i, first_scales[i]);
      first_unit = false;
    }
    const int all_see = n - (p.c.causal ? p.c.T - 1 : 0);

    // ---- the unit's tiles -------------------------------------------------------
    float o[MT][NT][4], sum_r[OWN][4];
    f32x2 l[NT];
#pragma unroll
    for (int i = 0; i < NT; ++i) {
#pragma unroll
      for (int j = 0; j < MT; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[j][i][e] = 0.f;
      l[i] = pair(0.f, 0.f);
    }
#pragma unroll
    for (int i = 0; i < OWN; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) sum_r[i][e] = 0.f;
#pragma unroll 1
    for (int tile = cur.j; tile < cur.j1; ++tile) {
      // (the place before this one's that is to be fetched to)
      store_scales(ahead == 0 ? NS - 1 : ahead - 1, scales);
      copy_wait<NS - 2>();
      __syncthreads();
      // (the place of the tile before, which every warp has left)
      fetch(ahead);
      uint8_t* place = smem + stage * kStageBytes<DK>;
      uint8_t* place_s = place + 2 * kTile * RB;
      stage = stage + 1 == NS ? 0 : stage + 1;
      ahead = ahead + 1 == NS ? 0 : ahead + 1;
      // A NaN scale of a value must not meet a probability of 0 of a row that does not
      // see its entry: it becomes 0 (before the next barrier, behind which it is read),
      // and the rows that do see it remember the group.
      if (tid >= kTile) {
        uint2* at = reinterpret_cast<uint2*>(place_s + tid * 8);
        const uint2 x = *at;
        const uint32_t bad[2] = {nan_scales(x.x), nan_scales(x.y)};
        if (bad[0] | bad[1]) {
          *at = make_uint2(x.x & ~(bad[0] / 128 * 255), x.y & ~(bad[1] / 128 * 255));
          const uint32_t mask = groups_of(bad);
          for (int r = 0; r < rows; ++r)
            if (tile * kTile + tid - kTile < reinterpret_cast<const int*>(&s_far[r >> 3][(r & 7) >> 1])[r & 1])
              atomicOr(&s_poison[r], mask);
        }
      }

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
          const uint8_t* from = place + place_of<DK>(entry_of(g), t * (RB / 4)) + (16 * warp + 8 * half) * RB;
          const uint8_t* from_s = place_s + (16 * warp + entry_of(g) + 8 * half) * 8;
          if constexpr (DK == 128) {
            const uint4 x = *reinterpret_cast<const uint4*>(from);
            w[half][0] = x.x, w[half][1] = x.y, w[half][2] = x.z, w[half][3] = x.w;
            const uint32_t y = *reinterpret_cast<const uint16_t*>(from_s + 2 * t);
            sc2[half][0] = scale_half2(y & 0xffu);
            sc2[half][1] = scale_half2(y >> 8);
          } else {
            const uint2 x = *reinterpret_cast<const uint2*>(from);
            w[half][0] = x.x, w[half][1] = x.y;
            sc2[half][0] = scale_half2(from_s[t]);
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
          const uint32_t a0[4] = {lo[0], hi[0], lo[1], hi[1]}, a1[4] = {lo[2], hi[2], lo[3], hi[3]};
#pragma unroll
          for (int c = 0; c < NT; ++c) {
            const uint4 qq = s_q[(c * (KS / 2) + i) * 32 + lane];
            mma(s[c], a0, qq.x, qq.y);
            mma(s[c], a1, qq.z, qq.w);
          }
        }
      }
      // probabilities
      if (tile * kTile + 16 * (warp + 1) > all_see) {
        const int e0 = tile * kTile + 16 * warp + entry_of(g);   // of s[.][0 .. 1]; e0 + 8 of the others
#pragma unroll
        for (int i = 0; i < NT; ++i) {
          const int2 far = s_far[i][t];
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (e0 + (e >> 1) * 8 >= (e & 1 ? far.y : far.x)) s[i][e] = -INFINITY;
        }
      }
      f32x2 sum[NT];
      const auto make = [&](int i, uint32_t (&pb)[2], f32x2 by, f32x2 nb) {
        f32x2 y[2];
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          const float2 x = halves(fma2(pair(s[i][2 * half], s[i][2 * half + 1]), by, nb));
          const float2 z = make_float2(ex2(x.x), ex2(x.y));
          y[half] = pair(z.x, z.y);
          pb[half] = transpose8(pack_half2(z.x, z.y));
        }
        sum[i] = add2(y[0], y[1]);
        return fmaxf(halves(sum[i]).x, halves(sum[i]).y);
      };
      float most = 0.f;                    // (of two probabilities: none of them above is too large for half precision)
#pragma unroll
      for (int i = 0; i < NT; i += 2) {
        const float4 r0 = s_row[i][t], r1 = s_row[i + 1][t];
        uint32_t a[2], c[2];
        most = fmaxf(most, make(i, a, pair(r0.x, r0.y), pair(r0.z, r0.w)));
        most = fmaxf(most, make(i + 1, c, pair(r1.x, r1.y), pair(r1.z, r1.w)));
        s_p[(warp * (NT / 2) + i / 2) * 32 + lane] = make_uint4(a[0], a[1], c[0], c[1]);
      }
      if (__syncthreads_or(most > 16384.f)) {
#pragma unroll
        for (int i = 0; i < NT; ++i) {
          const float4 row = s_row[i][t];
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            float x = fmaxf(s[i][e], s[i][e + 2]) * (e ? row.y : row.x);
#pragma unroll
            for (int d = 4; d < 32; d *= 2) x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, d));
            if (g == 0) s_top[warp][i * 8 + 2 * t + e] = x;
          }
        }
        __syncthreads();
        float nb[NT][2];
#pragma unroll
        for (int i = 0; i < NT; ++i) {
          const float4 row = s_row[i][t];
          float a[2];
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const int r = i * 8 + 2 * t + e;
            const float x = fmaxf(fmaxf(s_top[0][r], s_top[1][r]), fmaxf(s_top[2][r], s_top[3][r])), had = e ? row.w : row.z;
            nb[i][e] = had;
            a[e] = 1.f;
            if (x + had > kLift + kLag - 1.f) {
              nb[i][e] = kLift - x;
              a[e] = ex2(nb[i][e] - had);  // 0 at the first
            }
          }
          l[i] = mul2(l[i], pair(a[0], a[1]));
#pragma unroll
          for (int e = 0; e < 4; ++e) {
#pragma unroll
            for (int j = 0; j < MT; ++j) o[j][i][e] *= a[e & 1];
            if (i % 4 == warp) sum_r[i / 4][e] *= a[e & 1];
          }
          uint32_t pb[2];
          make(i, pb, pair(row.x, row.y), pair(nb[i][0], nb[i][1]));
          *(reinterpret_cast<uint2*>(s_p + (warp * (NT / 2) + i / 2) * 32 + lane) + i % 2) = make_uint2(pb[0], pb[1]);
        }
        __syncthreads();
        // (read again behind the next tile's barrier)
#pragma unroll
        for (int i = 0; i < NT; ++i)
          if (i % 4 == warp && g == 0) {
            s_row[i][t].z = nb[i][0];
            s_row[i][t].w = nb[i][1];
          }
      }
#pragma unroll
      for (int i = 0; i < NT; ++i) l[i] = add2(l[i], sum[i]);
      // O^T += V^T P^T: elements 32 warp + 4 g .. + 3 (16 warp + 2 g, + 1 of 64)
      const uint32_t ones[4] = {kOnes, kOnes, kOnes, kOnes};
      constexpr uint32_t low = 0x0f0f0f0fu;
      const auto products = [&](int k, const uint32_t (&a)[MT][4]) {
#pragma unroll
        for (int i = 0; i < NT; i += 2) {
          const uint4 pb = s_p[(k * (NT / 2) + i / 2) * 32 + lane];
#pragma unroll
          for (int j = 0; j < MT; ++j) {
            mma(o[j][i], a[j], pb.x, pb.y);
            mma(o[j][i + 1], a[j], pb.z, pb.w);
          }
          if (i % 4 == (warp & 2)) {       // n-tiles warp, warp + 4
            if (warp & 1) mma(sum_r[i / 4], ones, pb.z, pb.w);
            else mma(sum_r[i / 4], ones, pb.x, pb.y);
          }
        }
      };
      if constexpr (DK == 128) {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          uint32_t w[4], sb[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            w[i] = *reinterpret_cast<const uint16_t*>(place + place_of<DK>(t + 4 * (i & 1), 16 * warp + 2 * g) +
                                                      (kTile + 16 * k + 8 * (i >> 1)) * RB);
            sb[i] = place_s[(kTile + 16 * k + t + 4 * i) * 8 + 2 * warp + (g >> 2)];
          }
          const uint32_t s01 = sb[0] << 7 | sb[1] << 23, s23 = sb[2] << 7 | sb[3] << 23;
          // entries t and t + 8 in one word, t + 4 and t + 12 in the other; pairs of entries
          const uint32_t x = w[0] | w[2] << 16, z = w[1] | w[3] << 16;
          uint32_t even[4], odd[4];        // elements 0, 2 (and 1, 3) of t, t + 4; of t + 8, t + 12
          codes_to_half((x & low) | (z << 4 & ~low), even);
          codes_to_half((x >> 4 & low) | (z & ~low), odd);
          uint32_t a[MT][4];
#pragma unroll
          for (int j = 0; j < MT; ++j) {
            a[j][0] = mul_half2(even[j], s01);
            a[j][1] = mul_half2(odd[j], s01);
            a[j][2] = mul_half2(even[2 + j], s23);
            a[j][3] = mul_half2(odd[2 + j], s23);
          }
          products(k, a);
        }
      } else {
#pragma unroll
        for (int k = 0; k < 4; k += 2) {
          uint32_t x = 0, z = 0, sb[8];
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const uint32_t w = place[place_of<DK>(t + 4 * (i & 1), 8 * warp + g) + (kTile + 16 * k + 8 * (i >> 1)) * RB];
            if (i & 1) z |= w << (8 * (i >> 1)); else x |= w << (8 * (i >> 1));
            sb[i] = place_s[(kTile + 16 * k + t + 4 * i) * 8 + warp];
          }
          uint32_t even[4], odd[4];
          codes_to_half((x & low) | (z << 4 & ~low), even);
          codes_to_half((x >> 4 & low) | (z & ~low), odd);
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const uint32_t s01 = sb[4 * i] << 7 | sb[4 * i + 1] << 23, s23 = sb[4 * i + 2] << 7 | sb[4 * i + 3] << 23;
            const uint32_t a[MT][4] = {{mul_half2(even[2 * i], s01), mul_half2(odd[2 * i], s01),
                                        mul_half2(even[2 * i + 1], s23), mul_half2(odd[2 * i + 1], s23)}};
            products(k + i, a);
          }
        }
      }
    }

    // ---- what the CTA has of the unit -------------------------------------------
    const bool begins = cur.j == 0, whole = begins && cur.j1 == nt;
    const int64_t slot = 2 * (int64_t)me + (cur.at >= begin ? 1 : 0);            // (begun before, or here)
    if (tid == 0 && begins)
      p.units[(int64_t)b * p.Hkv * p.blocks + cur.u] =
          make_int2(whole ? -1 : (int)slot, whole ? me : line.owner(cur.at + kStart + nt - 1));
    __syncthreads();                       // (tops were read, references written)
#pragma unroll
    for (int i = 0; i < NT; ++i) {
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        float x = e ? halves(l[i]).y : halves(l[i]).x;
#pragma unroll
        for (int d = 4; d < 32; d *= 2) x += __shfl_xor_sync(0xffffffffu, x, d);
        if (g == 0) {
          s_top[warp][i * 8 + 2 * t + e] = x;
          if (i % 4 == warp) s_sum[i * 8 + 2 * t + e] = sum_r[i / 4][e];
        }
      }
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < NT; ++i) {
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int r = i * 8 + 2 * t + e;
        const float had = e ? s_row[i][t].w : s_row[i][t].z, ref = had == kNone ? -INFINITY : -had;
        const float sum = (s_top[0][r] + s_top[1][r]) + (s_top[2][r] + s_top[3][r]), rounded = s_sum[r];
        float v[4];
        int d;
        if constexpr (DK == 128) {
          d = 32 * warp + 4 * g;
          v[0] = o[0][i][e], v[1] = o[0][i][e + 2], v[2] = o[MT - 1][i][e], v[3] = o[MT - 1][i][e + 2];
        } else {                           // two lanes' elements in one of them
          d = 16 * warp + 2 * g;
          v[0] = o[0][i][e], v[1] = o[0][i][e + 2];
          v[2] = __shfl_down_sync(0xffffffffu, v[0], 4);
          v[3] = __shfl_down_sync(0xffffffffu, v[1], 4);
        }
        if (s_poison[r] >> (d / 16) & 1u) v[0] = v[1] = v[2] = v[3] = NAN;
        if (r < rows && (DK == 128 || g % 2 == 0)) {
          if (whole) {
            finish<4>(p, b, h, row0 + r, d, ref, sum, rounded, v, d == 0);
          } else {
            if (d == 0) p.slot_ml[slot * p.slot_rows + r] = make_float4(ref, sum, rounded, 0.f);
            *reinterpret_cast<float4*>(p.slot_o + (slot * p.slot_rows + r) * DK + d) = make_float4(v[0], v[1], v[2], v[3]);
          }
        }
      }
    }
  }
  copy_wait<0>();
}

template <int DK, int NT>
cudaError_t launch_t(const Params& p, int dev, int sms, cudaStream_t s) {
  static PerDevice attr;
  const cudaError_t e = attr.once(dev, []() {
    return cudaFuncSetAttribute(attend4_rows_kernel<DK, NT>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem<DK, NT>);
  });
  if (e != cudaSuccess) return e;
  return launch_pdl(attend4_rows_kernel<DK, NT>, dim3((unsigned)rows4_workers(NT, sms)), dim3(kThreads), kSmem<DK, NT>, s, p);
}

}  // namespace

int rows4_workers(int NT, int sms) { return sms * ctas_per_sm(NT); }

cudaError_t launch_attend4_rows(const Attend4Params& p, int dev, int sms, cudaStream_t s) {
  const int NT = p.slot_rows / 8;
  if (p.D <= 64) return NT == 2   ? launch_t<64, 2>(p, dev, sms, s)
                        : NT == 4 ? launch_t<64, 4>(p, dev, sms, s)
                        : NT == 6 ? launch_t<64, 6>(p, dev, sms, s)
                                  : launch_t<64, 8>(p, dev, sms, s);
  return NT == 2   ? launch_t<128, 2>(p, dev, sms, s)
         : NT == 4 ? launch_t<128, 4>(p, dev, sms, s)
         : NT == 6 ? launch_t<128, 6>(p, dev, sms, s)
                   : launch_t<128, 8>(p, dev, sms, s);
}

}  // namespace sp
