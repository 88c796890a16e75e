// sp_attn4_rows.cu -- attention over a cache held in 4 bits for units of many query
// rows (see sp_attn4.cu for the form of the cache, and for the line that the work is
// on).  What codes cost to be made half precision is shared by up to 96 rows, and the
// products are tcgen05's (M = 128, query rows are the lanes of tensor memory).
//
// A CTA (256 threads, two per SM) walks its tiles of 64 entries:
//   warps 4-7   decode, two the keys and two the values: a thread makes an entry half
//               precision, into rings in shared memory; the codes of the next two tiles
//               are on their way meanwhile (cp.async, each warp its own)
//   warps 0-2   the softmax, thread = row: per tile they read the 64 scores of their
//               row, keep the running maximum and sums, and put the probabilities,
//               rounded to half precision, back over the scores; at the end of a
//               unit's tiles they read O.  At its beginning they make its queries.
//   warp 3      S = Q K^T one tile ahead of O += P V (P from tensor memory, V as an
//               N-major operand)
// (96 rows, not the 128 of the MMA, so that 8 warps do, with 128 registers a thread:
// with a ninth and 96 the loops spilled and a tile took twice as long.)
// A row's queries are times a power of two, and its scores are masked, by its thread.
//
// What bounds it: for half of its time, by the bytes that the code moves, shared memory.  A tile of
// 128-wide heads moves 114 KB in it (codes in and out 18, half precision in 32, operands 64, of
// which half are the 128 rows of Q that the MMA reads again for each tile): 890 cycles at 128 bytes;
// with two CTAs an SM a tile takes 1950, for 16 rows as for 64.  16 sequences of 3500 entries, 64/8
// heads, 8 tokens, 69 MB: 48.5 us, of which 6.4 until the first scores (places 2.2, queries 3,
// product 1), 24 the tiles, 2 a unit's end, 9 the merge of 8192 rows.
#include "sp_attn4.cuh"

namespace sp {
namespace {

using Params = Attend4Params;
constexpr int kTile = 64, kUnitStart = 6;
constexpr int kRows = 128, kRowWarps = kRowsMost4 / 32;        // of the MMA; warps that query rows are the lanes of
constexpr int kRowThreads = 256;
constexpr int kRing = 2;                   // tiles of K in half precision
template <int DK> constexpr int kRingV = DK == 128 ? 1 : 2;    // and of V: what there is room for
constexpr int kRaw = 3;                    // tiles of codes and scales, as they are held
constexpr int kTmemCols = 256;             // S and P: 0 .. 63 and 64 .. 127, O from 128 on
constexpr uint32_t kTmemO = 128;
constexpr int kQBlock = kRows * 128;       // 64 elements of 128 rows
constexpr int kBlock = kTile * 128;        // 64 elements of a tile's entries
template <int DK> constexpr int kQBytes = DK / 64 * kQBlock;
template <int DK> constexpr int kTileBytes = DK / 64 * kBlock;
template <int DK> constexpr int kRawBytes = 32 * (kRowBytes<DK> + 8);   // of a warp: 32 entries
template <int DK> constexpr int kSmem = 1024 + kQBytes<DK> + (kRing + kRingV<DK>) * kTileBytes<DK> + 4 * kRaw * kRawBytes<DK>;
static_assert(2 * (kSmem<128> + 4 * 1024) <= 228 * 1024, "two CTAs per SM");
static_assert(kRing * kTileBytes<64> >= (SPIKE_PROJ_CACHE_MAX_B + 1) * 4, "room for the costs before each sequence");

// Bounded wait; false too when another warp of the CTA has given up.
__device__ __forceinline__ bool wait(const Params& p, uint64_t* bar, uint32_t parity, const volatile int* stop) {
  if (mbar_try_wait(bar, parity)) return true;
  const long long t0 = clock64();
  do {
    if (mbar_try_wait(bar, parity)) return true;
  } while (!*stop && clock64() - t0 < p.limit);
  return false;
}
__device__ __forceinline__ bool all(bool x) { return __all_sync(0xffffffffu, x) != 0; }
// a += the lower half of x, b += the upper one.
__device__ __forceinline__ void add_halves(uint32_t x, float& a, float& b) {
  asm("{\n\t.reg .b16 l, h;\n\tmov.b32 {l, h}, %2;\n\tadd.rn.f32.f16 %0, l, %0;\n\tadd.rn.f32.f16 %1, h, %1;\n\t}"
      : "+f"(a), "+f"(b)
      : "r"(x));
}

struct Bars {
  uint64_t k_full[kRing], k_empty[kRing], v_full[2], v_empty[2], s_full[2], p_full[2];
  uint64_t q_full, o_full, o_empty, done;
};

// PLAIN: heads of DK elements; else of fewer, whose rows are not of whole 16 bytes.
template <int DK, bool PLAIN>
__global__ void __launch_bounds__(kRowThreads, 2) attend4_rows_kernel(const __grid_constant__ Params p) {
  constexpr uint32_t kIdescS = 1u << 4 | (uint32_t)(kTile >> 3) << 17 | (uint32_t)(kRows >> 4) << 24;
  constexpr uint32_t kIdescO = 1u << 4 | 1u << 16 | (uint32_t)(DK >> 3) << 17 | (uint32_t)(kRows >> 4) << 24;
  extern __shared__ uint8_t smem_base[];
  uint8_t* smem = smem_base + (-smem_u32(smem_base) & 1023u);  // (swizzled operands begin on 1024 bytes)
  __shared__ Bars bars;
  __shared__ uint32_t s_tmem;
  __shared__ volatile int s_abort;
  // groups of which a row sees a NaN value, by unit (values are decoded up to two
  // units ahead of the one whose O is read)
  __shared__ uint32_t s_poison[4][kRows];
  uint8_t* sQ = smem;
  uint8_t* sK = sQ + kQBytes<DK>;
  uint8_t* sV = sK + kRing * kTileBytes<DK>;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  if (tid == 0) {
    for (int i = 0; i < 2; ++i) {
      mbar_init(&bars.k_full[i], 2);
      mbar_init(&bars.k_empty[i], 1);
      mbar_init(&bars.v_full[i], 2);
      mbar_init(&bars.v_empty[i], 1);
      mbar_init(&bars.s_full[i], 1);
      mbar_init(&bars.p_full[i], kRowWarps);
    }
    mbar_init(&bars.q_full, kRowWarps);
    mbar_init(&bars.o_full, 1);
    mbar_init(&bars.o_empty, kRowWarps);
    mbar_init(&bars.done, 1);
    s_abort = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  for (int i = tid; i < 4 * kRows; i += kRowThreads) s_poison[i / kRows][i % kRows] = 0;
  if (warp == 0) tmem_alloc(&s_tmem, kTmemCols);
  pdl_launch_dependents();
  pdl_wait();

  const int me = blockIdx.x;
  tc_fence_before();
  const Start<kTile, kUnitStart> start =
      start_of<kTile, kUnitStart, kRowThreads>(p, reinterpret_cast<uint32_t*>(sK), me, gridDim.x);
  __syncthreads();
  tc_fence_after();
  const Line line = start.line;
  const uint32_t begin = start.begin, end = start.end, tmem = s_tmem;
  // The first rows are those of warps 0 and 1, or, in the CTA that has the SM's other half of
  // tensor memory, of warps 2 and 3: its softmax is at work where the first CTA's is not.
  const int turn = tmem / kTmemCols % 2 * 2, lw = warp < 4 ? (warp + turn) & 3 : warp;
  Cursor<kTile, kUnitStart> cur = start.cur;
  const volatile int* stop = &s_abort;
  bool ok = true;
  // A unit that the CTA has no tile of: of no concern, but for one without entries,
  // whose rows warps 0 to 3 write out.
  const auto skip = [&]() { return cur.j >= cur.j1; };

  if (warp >= 4) {
    // ------------------------------ decode ------------------------------------------
    // Warps 4 and 5 have the keys of a tile's entries 0 .. 31 and 32 .. 63, warps 6 and
    // 7 the values; thread = entry, but for the copies.
    constexpr int RB = kRowBytes<DK>, C = RB / 16, kCopyRows = 32 / C;
    const bool keys = warp < 6;
    const int e0 = (warp & 1) * 32, e = e0 + lane, nbytes = PLAIN ? RB : p.D / 2, groups = PLAIN ? DK / 16 : p.D / 16;
    const sp_kv4 held = keys ? p.c.k4 : p.c.v4;
    const uint32_t raw_u32 = smem_u32(sV + kRingV<DK> * kTileBytes<DK>) + (warp - 4) * (kRaw * kRawBytes<DK>);
    // 16 bytes of a row: so that neither the copies' rows nor a row's reads meet in a bank
    const auto raw_at = [&](int row, int chunk) { return row * RB + (chunk ^ (DK == 128 ? row >> 1 & 3 : row >> 2 & 1)) * 16; };
    const int copy_row = lane / C, copy_byte = lane % C * 16;
    // f: the tile that is copied, kRaw - 1 before cur, the one that is decoded
    Cursor<kTile, kUnitStart> f = cur;
    const uint8_t *code = nullptr, *scale = nullptr;
    const auto settle = [&](Cursor<kTile, kUnitStart>& c) {    // at a tile, or at the end
      while (c.at < end && c.j >= c.j1) c.next(p, begin, end);
    };
    const auto enter = [&]() {
      settle(f);
      if (f.at >= end) return;
      const int h = p.by_blocks(f.u);
      const int64_t entry = (int64_t)f.j * kTile + e0;
      code = held.codes + f.b * held.batch + (entry + copy_row) * held.entry + h * held.head + copy_byte;
      scale = held.scales + f.b * held.scales_batch + (entry + lane) * held.scales_entry + h * held.scales_head;
    };
    ScaleRow<DK, PLAIN> scales;            // of the tile copied last
    scales.load(nullptr, groups, false);
    const bool lined = PLAIN && held.entry == RB;              // rows of a head one after the other
    const auto fetch = [&](int stage) {    // and on
      if (f.at < end) {
        const uint32_t to = raw_u32 + stage * kRawBytes<DK>;
        const int left = f.n - f.j * kTile - e0;
        if (lined && left >= 32) {
#pragma unroll
          for (int i = 0; i < 32 / kCopyRows; ++i)
            copy_async<16>(to + raw_at(copy_row + i * kCopyRows, lane % C), code + i * kCopyRows * RB);
        } else if (PLAIN || nbytes % 16 == 0) {
          const uint8_t* from = code;
#pragma unroll
          for (int i = 0; i < 32 / kCopyRows; ++i) {
            const int row = copy_row + i * kCopyRows;
            if (row < left && (PLAIN || copy_byte < nbytes)) copy_async<16>(to + raw_at(row, lane % C), from);
            from += kCopyRows * held.entry;
          }
        } else {
          // 8 bytes of every kRows8-th entry
          constexpr int C8 = RB / 8, kRows8 = 32 / C8;
          const int row8 = lane / C8, byte = lane % C8 * 8;
          const uint8_t* from = code + (row8 - copy_row) * held.entry + (byte - copy_byte);
#pragma unroll
          for (int i = 0; i < 32 / kRows8; ++i) {
            const int row = row8 + i * kRows8;
            if (row < left && byte < nbytes) copy_async<8>(to + raw_at(row, byte >> 4) + (byte & 8), from);
            from += kRows8 * held.entry;
          }
        }
        scales.load(scale, groups, lane < left);
        code += kTile * held.entry;
        scale += kTile * held.scales_entry;
        if (++f.j >= f.j1) enter();
      }
      copy_commit();
    };
    const auto store_scales = [&](int stage, uint2 x) {
      asm volatile("st.shared.v2.b32 [%0], {%1, %2};" ::"r"(raw_u32 + stage * kRawBytes<DK> + 32 * RB + lane * 8), "r"(x.x), "r"(x.y)
                   : "memory");
    };
    // A thread's entry to its row of a tile, 16 bytes at a time (swizzled as the MMA reads
    // them).  (Codes of entries that are not there are anything, their scales 0.)
    const auto decode = [&](int stage, uint2 x, uint8_t* tile) {
      const uint32_t to = smem_u32(tile) + e * 128 + (e & 7) * 16;
      uint32_t w[C][4];                    // (all loads before the stores: these are not moved past each other)
#pragma unroll
      for (int c = 0; c < C; ++c)
        asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];"
                     : "=r"(w[c][0]), "=r"(w[c][1]), "=r"(w[c][2]), "=r"(w[c][3])
                     : "r"(raw_u32 + stage * kRawBytes<DK> + raw_at(lane, c)));
#pragma unroll
      for (int c = 0; c < C; ++c) {
        const uint32_t s = scales_half2((c < 2 ? x.x : x.y) >> c % 2 * 16);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          uint32_t h[4];
          codes_to_half(w[c][i], h);
#pragma unroll
          for (int k = 0; k < 4; ++k) h[k] = i < 2 ? mul_half2_by<0>(h[k], s) : mul_half2_by<1>(h[k], s);
          asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"((to ^ (c % 2 * 4 + i) * 16) + c / 2 * kBlock),
                       "r"(h[0]), "r"(h[1]), "r"(h[2]), "r"(h[3]));
        }
      }
    };
    settle(cur);
    enter();
    {
      ScaleRow<DK, PLAIN> x[kRaw - 1];
#pragma unroll
      for (int i = 0; i < kRaw - 1; ++i) {
        fetch(i);
        x[i] = scales;
      }
#pragma unroll
      for (int i = 0; i < kRaw - 2; ++i) store_scales(i, x[i].value(groups));
    }
    uint64_t *full = keys ? bars.k_full : bars.v_full, *empty = keys ? bars.k_empty : bars.v_empty;
    uint8_t* tiles = keys ? sK : sV;
    const int ring = keys ? kRing : kRingV<DK>;
    int seg = 0, raw = 0, st = 0;
    uint32_t free = 1;                     // parity of a place's release
    for (int it = 0; cur.at < end; ++it) {
      const int ahead = raw == 0 ? kRaw - 1 : raw - 1;
      store_scales(ahead == 0 ? kRaw - 1 : ahead - 1, scales.value(groups));
      copy_wait<kRaw - 2>();
      __syncwarp();
      fetch(ahead);                        // (the place of the tile before, which every lane has left)
      uint2 x;
      asm volatile("ld.shared.v2.b32 {%0, %1}, [%2];"
                   : "=r"(x.x), "=r"(x.y)
                   : "r"(raw_u32 + raw * kRawBytes<DK> + 32 * RB + lane * 8));
      // A NaN scale of a value must not meet a probability of 0 of a row that does not
      // see its entry: it becomes 0, and the rows that do see it remember the group.
      const uint32_t bad[2] = {keys ? 0u : nan_scales(x.x), keys ? 0u : nan_scales(x.y)};
      if (bad[0] | bad[1]) {
        x.x &= ~(bad[0] / 128 * 255);
        x.y &= ~(bad[1] / 128 * 255);
        const uint32_t mask = groups_of(bad);
        const int row0 = (cur.u - p.by_blocks(cur.u) * p.blocks) * p.block_rows, rows = min(p.block_rows, p.R - row0);
        for (int r = 0; r < rows; ++r)
          if (cur.j * kTile + e < (p.c.causal ? cur.n - (p.c.T - 1 - (int)p.by_G(row0 + r)) : cur.n))
            atomicOr(&s_poison[seg & 3][r], mask);
      }
      ok = all(wait(p, &empty[st], free, stop));
      if (!ok) break;
      decode(raw, x, tiles + st * kTileBytes<DK>);
      fence_async_shared();
      __syncwarp();
      if (lane == 0 && !(p.fault == kFaultStall && it == 0 && keys)) mbar_arrive(&full[st]);
      raw = raw + 1 == kRaw ? 0 : raw + 1;
      if (++st == ring) {
        st = 0;
        free ^= 1;
      }
      if (++cur.j >= cur.j1) {
        settle(cur);
        ++seg;
      }
    }
    copy_wait<0>();
  } else if (lw == 3) {
    // ------------------------------ products ----------------------------------------
    int it = 0, seg = 0;
    const uint32_t one = elect_one();
    const auto scores = [&](int i) {
      const int st = i % kRing;
      if (!all(wait(p, &bars.k_full[st], i / kRing & 1, stop))) return false;
      tc_fence_after();
      const uint64_t qd = smem_desc(sQ, 1024, kSwizzle128), kd = smem_desc(sK + st * kTileBytes<DK>, 1024, kSwizzle128);
#pragma unroll
      for (int k = 0; k < DK / 16; ++k)
        mma_f16_if(one, tmem + (i & 1) * kTile, qd + (k / 4) * (kQBlock >> 4) + (k % 4) * 2,
                   kd + (k / 4) * (kBlock >> 4) + (k % 4) * 2, kIdescS, k > 0);
      mma_commit_if(one, &bars.s_full[i & 1]);
      mma_commit_if(one, &bars.k_empty[st]);
      return true;
    };
    const auto values = [&](int i, bool first, bool last) {
      const int st = i % kRingV<DK>;
      if (!all(wait(p, &bars.p_full[i & 1], i >> 1 & 1, stop) && wait(p, &bars.v_full[st], i / kRingV<DK> & 1, stop) &&
               (!first || wait(p, &bars.o_empty, (seg & 1) ^ 1u, stop))))
        return false;
      tc_fence_after();
      const uint64_t vd = n_major_desc(sV + st * kTileBytes<DK>, kBlock);
#pragma unroll
      for (int k = 0; k < kTile / 16; ++k)
        mma_f16_ta_if(one, tmem + kTmemO, tmem + (i & 1) * kTile + 8 * k, vd + k * (2048 >> 4), kIdescO, !first || k > 0);
      mma_commit_if(one, &bars.v_empty[st]);
      if (last) mma_commit_if(one, &bars.o_full);
      return true;
    };
    for (; ok && cur.at < end; cur.next(p, begin, end)) {
      if (cur.j >= cur.j1) continue;
      const int count = cur.j1 - cur.j;
      // (the buffer of tile i + 1 is that of tile i - 1, whose product with V, issued
      // before, reads the probabilities there first)
      ok = all(wait(p, &bars.q_full, seg & 1, stop)) && scores(it);
      for (int j = 0; j < count && ok; ++j, ++it)
        ok = (j + 1 == count || scores(it + 1)) && values(it, j == 0, j + 1 == count);
      ++seg;
    }
    mma_commit_if(one, &bars.done);        // every MMA has retired
    const volatile int never = 0;
    wait(p, &bars.done, 0, &never);
  } else {
    // ------------------------------ softmax -----------------------------------------
    const uint32_t lanes = tmem + ((uint32_t)(warp * 32) << 16);
    const int row = lw * 32 + lane;        // of the unit's; warp * 32 + lane: of the MMAs'
    int it = 0, seg = 0;
    for (; ok && cur.at < end; cur.next(p, begin, end)) {
      const bool empty = cur.nt == 0 && cur.at >= begin;
      if (skip() && !empty) continue;
      const int b = cur.b, n = cur.n, h = p.by_blocks(cur.u), block = cur.u - h * p.blocks;
      const int row0 = block * p.block_rows, rows = min(p.block_rows, p.R - row0), r = row0 + row;
      const bool mine = row < rows, work = lw * 32 < rows;
      const int tok = p.by_G(mine ? r : 0);
      int2* const unit = p.units + (int64_t)b * p.Hkv * p.blocks + cur.u;
      if (empty) {
        if (row == 0) *unit = make_int2(-1, me);
        const float other = mine ? other_of(p, b, h, r) : 0.f;
        for (int d = 0; d < DK && mine; d += 16) {
          float none[16] = {};
          finish<16>(p, b, h, r, d, -INFINITY, 0.f, 0.f, none, other, d == 0);
        }
        continue;
      }
      // The thread's row of queries (the tiles before have been multiplied: their scores
      // were here).  A row a thread, not a row by several: the loads touch more lines, but
      // a warp has a third of the instructions, and it has them to itself.
      int e = 0;                           // (see factor_of)
      if (work) {
        uint32_t in;
        const int token = p.by_G(mine ? r : 0, &in);
        const uint4* from = reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(p.c.q) + b * p.c.q_batch +
                                                           token * p.c.q_token + (int64_t)(h * p.G + in) * p.c.q_head);
        const int chunks = !mine ? 0 : PLAIN ? DK / 8 : p.D / 8, at = warp * 32 + lane;
        uint4 x[DK / 8];
#pragma unroll
        for (int i = 0; i < DK / 8; ++i) x[i] = i < chunks ? from[i] : make_uint4(0, 0, 0, 0);
        float by = 1.f;
        if (p.bf16) {
          const auto largest = [&](bool finite) {
            uint32_t most[2] = {0, 0};
#pragma unroll
            for (int i = 0; i < DK / 8; ++i) {
              const uint32_t w[4] = {x[i].x, x[i].y, x[i].z, x[i].w};
#pragma unroll
              for (int j = 0; j < 4; ++j) {
                const uint32_t y = w[j] & 0x7fff7fffu;
                most[j % 2] = __vmaxu2(most[j % 2], finite ? y & ~__vcmpgeu2(y, 0x7f807f80u) : y);
              }
            }
            most[0] = __vmaxu2(most[0], most[1]);
            return max(most[0] & 0xffffu, most[0] >> 16);
          };
          uint32_t most = largest(false);
          if (most >= 0x7f80u) most = largest(true);
          e = lift_of(most);
          by = power_of_two(e);
        }
        const f32x2 by2 = pair(by, by);
#pragma unroll
        for (int i = 0; i < DK / 8; ++i) {
          uint32_t w[4] = {x[i].x, x[i].y, x[i].z, x[i].w};
          if (p.bf16) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              const float2 y = to_float(true, w[j]), z = halves(mul2(pair(y.x, y.y), by2));
              w[j] = pack_half2(z.x, z.y);
            }
          }
          *reinterpret_cast<uint4*>(sQ + (i >> 3) * kQBlock + at * 128 + ((i ^ at) & 7) * 16) = make_uint4(w[0], w[1], w[2], w[3]);
        }
        fence_async_shared();
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(&bars.q_full);
      const float c2 = factor_of(p, e).by;
      const int far = p.c.causal ? n - (p.c.T - 1 - tok) : n;  // entries that the row sees
      // how far above the maximum that the reference has it follows (at first from anywhere), that maximum; sums
      float lag = -INFINITY, m = 0.f, l = 0.f, rl = 0.f;
      for (int j = cur.j; j < cur.j1; ++j, ++it) {
        ok = all(wait(p, &bars.s_full[it & 1], it >> 1 & 1, stop));
        if (!ok) break;
        tc_fence_after();
        if (work) {
          const uint32_t s_buf = lanes + (it & 1) * kTile, o_buf = lanes + kTmemO;
          uint32_t v[2][32];
          tmem_ld32_issue(s_buf, v[0]);
          tmem_ld32_issue(s_buf + 32, v[1]);
          tmem_ld_wait();
          reg_pin(v[0]);
          reg_pin(v[1]);
          const int nv = far - j * kTile;
          if (__any_sync(0xffffffffu, nv < kTile)) {
#pragma unroll
            for (int i = 0; i < kTile; ++i)
              if (i >= nv) v[i / 32][i % 32] = 0xff800000u;
          }
          float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
          for (int i = 0; i < kTile; ++i) mx[i % 4] = fmaxf(mx[i % 4], __uint_as_float(v[i / 32][i % 32]));
          const float top = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3])), above = (top - m) * c2;
          const bool grow = above > lag;
          if (__any_sync(0xffffffffu, grow)) {
            float a = 1.f;
            if (grow) {
              a = lag == -INFINITY ? 0.f : ex2(-above);
              lag = kLag;
              m = top;
            }
            l *= a;
            rl *= a;
            if (j > cur.j) {
              ok = all(wait(p, &bars.v_empty[(it - 1) % kRingV<DK>], (it - 1) / kRingV<DK> & 1, stop));
              if (!ok) break;
              tc_fence_after();
#pragma unroll 1                           // (rare, and registers are short)
              for (int i = 0; i < DK / 16; ++i) {
                uint32_t o[16];
                tmem_ld16_issue(o_buf + 16 * i, o);
                tmem_ld_wait();
                reg_pin(o);
#pragma unroll
                for (int x = 0; x < 16; ++x) o[x] = __float_as_uint(__uint_as_float(o[x]) * a);
                tmem_st16_issue(o_buf + 16 * i, o);
              }
            }
          }
          f32x2 sum[2] = {pair(0.f, 0.f), pair(0.f, 0.f)};
          float rsum[4] = {};
          const f32x2 by = pair(c2, c2), minus_m = pair(-m, -m), lift = pair(kLift, kLift);
#pragma unroll
          for (int g = 0; g < 2; ++g) {
            uint32_t pk[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) {
              // (the difference first: see attend4_kernel)
              const float2 x =
                  halves(fma2(add2(pair(__uint_as_float(v[g][2 * i]), __uint_as_float(v[g][2 * i + 1])), minus_m), by, lift));
              const float2 y = make_float2(ex2(x.x), ex2(x.y));
              pk[i] = pack_half2(y.x, y.y);
              sum[i % 2] = add2(sum[i % 2], pair(y.x, y.y));
              add_halves(pk[i], rsum[i % 2 * 2], rsum[i % 2 * 2 + 1]);
            }
            tmem_st16_issue(s_buf + 16 * g, pk);
          }
          const float2 ls = halves(add2(sum[0], sum[1]));
          l += ls.x + ls.y;
          rl += (rsum[0] + rsum[1]) + (rsum[2] + rsum[3]);
          tmem_st_wait();
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&bars.p_full[it & 1]);
      }
      if (!ok) break;
      const bool begins = cur.j == 0, whole = begins && cur.j1 == cur.nt;
      const int64_t slot = 2 * (int64_t)me + (cur.at >= begin ? 1 : 0);          // (begun before, or here)
      if (row == 0 && begins)
        *unit = make_int2(whole ? -1 : (int)slot, whole ? me : worker_of(p, line, cur.at + kUnitStart + cur.nt - 1, me));
      ok = all(wait(p, &bars.o_full, seg & 1, stop));
      if (!ok) break;
      tc_fence_after();
      if (work) {
        const uint32_t poison = s_poison[seg & 3][row];
        s_poison[seg & 3][row] = 0;
        const float base = lag == -INFINITY ? -INFINITY : fmaf(m, c2, -kLift);
        const float other = mine && whole ? other_of(p, b, h, r) : -INFINITY;
        float* to = p.slot_o + (slot * p.slot_rows + row) * DK;
        if (mine && !whole) p.slot_ml[slot * p.slot_rows + row] = make_float4(base, l, rl, 0.f);
        if (whole || __any_sync(0xffffffffu, poison != 0)) {
#pragma unroll 1
          for (int i = 0; i < DK / 16; ++i) {
            uint32_t raw[16];
            tmem_ld16_issue(lanes + kTmemO + 16 * i, raw);
            tmem_ld_wait();
            reg_pin(raw);
            float o[16];
#pragma unroll
            for (int x = 0; x < 16; ++x) o[x] = poison >> i & 1u ? NAN : __uint_as_float(raw[x]);
            if (mine) {
              if (whole) {
                finish<16>(p, b, h, r, 16 * i, base, l, rl, o, other, i == 0);
              } else {
#pragma unroll
                for (int x = 0; x < 16; x += 4) *reinterpret_cast<float4*>(to + 16 * i + x) = make_float4(o[x], o[x + 1], o[x + 2], o[x + 3]);
              }
            }
          }
        } else {
#pragma unroll
          for (int i = 0; i < DK; i += 32) {
            uint32_t o[32];
            tmem_ld32_issue(lanes + kTmemO + i, o);
            tmem_ld_wait();
            reg_pin(o);
            if (mine)
#pragma unroll
              for (int x = 0; x < 32; x += 4) *reinterpret_cast<uint4*>(to + i + x) = make_uint4(o[x], o[x + 1], o[x + 2], o[x + 3]);
          }
        }
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(&bars.o_empty);
      ++seg;
    }
  }
  if (!ok) {
    s_abort = 1;
    if (lane == 0) atomicExch(p.err, kErrMbarTimeout);
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp == 0) tmem_dealloc(tmem, kTmemCols);
}

template <int DK, bool PLAIN>
cudaError_t launch_t(const Params& p, int dev, int sms, cudaStream_t s) {
  static PerDevice attr;
  const cudaError_t e = attr.once(dev, []() {
    return cudaFuncSetAttribute(attend4_rows_kernel<DK, PLAIN>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem<DK>);
  });
  if (e != cudaSuccess) return e;
  return launch_pdl(attend4_rows_kernel<DK, PLAIN>, dim3((unsigned)rows4_workers(sms)), dim3(kRowThreads), kSmem<DK>, s, p);
}

}  // namespace

cudaError_t launch_attend4_rows(const Attend4Params& p, int dev, int sms, cudaStream_t s) {
  if (p.D <= 64) return p.D == 64 ? launch_t<64, true>(p, dev, sms, s) : launch_t<64, false>(p, dev, sms, s);
  return p.D == 128 ? launch_t<128, true>(p, dev, sms, s) : launch_t<128, false>(p, dev, sms, s);
}

}  // namespace sp
