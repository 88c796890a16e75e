// sp_cache.h -- launch wrappers of the operators around a KV cache: attention
// over a shared prefix and own caches, eviction, and draft verification.
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

#include "sp_internal.h"

namespace sp {

// What a cache handle is made for, and the workspace that its calls share.
struct CacheShape {
  int32_t max_batch, max_T, Hq, Hkv, D, capacity, dtype;
  bool weights;
};

// Workspace of a handle (bytes from the start of one allocation).
struct CacheWorkspace {
  size_t bytes;
  size_t moves, counts;                    // of evictions: lists of slot pairs per head, their lengths
};
CacheWorkspace cache_workspace(const CacheShape& s, int sms);

// The partial results of a unit of query rows, as the merge finds them: one of each
// of the CTAs first .. last that the attention kernel noted down.  Where it gave
// up on a wait the note may be anything, so that both are taken into 0 .. grid - 1
// and a reversed pair holds none.
struct Results {
  int32_t first, last;
  __host__ __device__ int32_t count() const { return last < first ? 0 : last - first + 1; }
};
inline __host__ __device__ int32_t within(int32_t cta, int32_t grid) { return cta < 0 ? 0 : cta < grid ? cta : grid - 1; }
inline __host__ __device__ Results noted_results(int32_t first, int32_t last, int32_t grid) {
  return Results{within(first, grid), within(last, grid)};
}
// Part `sub` of `parts` of n >= 0 things: begin .. end (none where end <= begin).
struct Share {
  int32_t begin, end;
};
inline __host__ __device__ Share share_of(int32_t n, int32_t sub, int32_t parts) {
  const int32_t each = (int32_t)((uint32_t)(n + parts - 1) / (uint32_t)parts), begin = sub * each;
  return Share{begin, begin + each < n ? begin + each : n};
}

// Pieces of a row through a ring of RING places, one warp.  it: pieces that have
// gone through the ring before; copies: every copy so far has arrived in time.
// fetch(i, place) copies piece i there, arrived(place, parity) waits (within a
// limit) for it, use(i, place, here) takes it from there, or from the row itself
// where a copy has not come, then(i, x) is given what use returned after the
// place has its next copy.  Returns `copies`.  When a wait has run out, all that
// is still on its way is waited for once more, as nothing may land in the memory
// of a CTA that has left.
#ifdef __CUDACC__
#define SP_WARP __device__ __forceinline__
#else
#define SP_WARP inline                     // (a test's simulation)
#endif
template <int RING, typename Fetch, typename Arrived, typename Use, typename Then>
SP_WARP bool walk_ring(int it, int pieces, bool copies, Fetch fetch, Arrived arrived, Use use, Then then) {
  if (copies)
    for (int i = 0; i < RING && i < pieces; ++i) fetch(i, (it + i) % RING);
  for (int i = 0; i < pieces; ++i) {
    const int place = (it + i) % RING;
    if (copies && !arrived(place, (uint32_t)((it + i) / RING & 1))) {
      copies = false;
      for (int j = i; j < i + RING && j < pieces; ++j) arrived((it + j) % RING, (uint32_t)((it + j) / RING & 1));
    }
    const auto x = use(i, place, copies);
    if (copies && i + RING < pieces) fetch(i + RING, place);
    then(i, x);
  }
  return copies;
}

// A row of V 32-bit entries (V < 2^26) that begins `skip` bytes (0, 4, 8 or 12) into
// 16 is copied in whole 16-byte pieces that lie within it: all but up to three
// entries at each end.  A bulk copy of entries v .. v + n - 1 and what lies around
// them up to these boundaries, in bytes from where the row's first 16 begin: `bytes`
// (<= 0: nothing) from `from` on, for a place that begins with the 16 bytes at `base`.
struct RowCopy {
  int32_t base, from, bytes;
};
inline __host__ __device__ RowCopy row_copy(int32_t skip, int32_t V, int32_t v, int32_t n) {
  const int32_t base = (skip + 4 * v) & ~15, from = base == 0 && skip ? 16 : base;
  const int32_t to = (skip + 4 * (v + n) + 15) & ~15, last = (skip + 4 * V) & ~15;
  return RowCopy{base, from, (to < last ? to : last) - from};
}
// Entries at the ends of two rows that are not copied in one of them at least (of
// one row: give it twice); lead + trail <= V.
struct RowEnds {
  int32_t lead, trail;
};
inline __host__ __device__ RowEnds row_ends(int32_t skip_p, int32_t skip_q, int32_t V) {
  const int32_t lead_p = (16 - skip_p) / 4 & 3, lead_q = (16 - skip_q) / 4 & 3;
  const int32_t trail_p = (skip_p / 4 + V) & 3, trail_q = (skip_q / 4 + V) & 3;
  int32_t lead = lead_p > lead_q ? lead_p : lead_q, trail = trail_p > trail_q ? trail_p : trail_q;
  lead = lead < V ? lead : V;
  return RowEnds{lead, trail < V - lead ? trail : V - lead};
}

// Tiles of entries that a call has at most (its launch counts them in 32 bits).
int64_t attend_tiles(const CacheShape& s, const sp_attend& c);
cudaError_t launch_attend(const CacheShape& s, const sp_attend& c, uint8_t* ws, int* err, int fault,
                          cudaStream_t stream);
cudaError_t launch_evict(const CacheShape& s, const sp_evict& c, uint8_t* ws, cudaStream_t stream);
cudaError_t launch_verify(const sp_verify& c, cudaStream_t stream);

}  // namespace sp
