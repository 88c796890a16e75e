// Index arithmetic that the cache kernels share with the host, for tests of it
// without a GPU.
#include <vector>

#include "sp_cache.h"

extern "C" {
// count results from CTA first on; returns the part sub of `parts` of n of them
void arith_results(int32_t first, int32_t last, int32_t grid, int32_t* from, int32_t* count) {
  const sp::Results r = sp::noted_results(first, last, grid);
  *from = r.first;
  *count = r.count();
}
void arith_share(int32_t n, int32_t sub, int32_t parts, int32_t* begin, int32_t* end) {
  const sp::Share s = sp::share_of(n, sub, parts);
  *begin = s.begin;
  *end = s.end;
}

void arith_row_copy(int32_t skip, int32_t V, int32_t v, int32_t n, int32_t* copy) {
  const sp::RowCopy c = sp::row_copy(skip, V, v, n);
  copy[0] = c.base;
  copy[1] = c.from;
  copy[2] = c.bytes;
}
void arith_row_ends(int32_t skip_p, int32_t skip_q, int32_t V, int32_t* lead, int32_t* trail) {
  const sp::RowEnds e = sp::row_ends(skip_p, skip_q, V);
  *lead = e.lead;
  *trail = e.trail;
}

// The walk of rows of pieces[0 .. rows - 1] pieces through a ring of two places
// whose copies behave as how[] says, one after another: 0 it arrives at once, 1
// after the time of a wait that runs out, 2 never.  Returns 0 where every piece was
// used once, from the ring where and only where its own copy was there, no place
// had two copies on their way, and at the end none that would ever arrive was;
// else the number of the rule that was broken.
int arith_ring(int rows, const int* pieces, const int* how) {
  constexpr int kRing = 2;
  struct Place {
    int filled = 0, on_way = -1, holds = -1;        // phases completed; copies, by number
  } ring[kRing];
  std::vector<int> since;                           // of each copy
  int it = 0, broken = 0, now = 0;                  // now: waits that have run out
  bool copies = true;
  for (int r = 0; r < rows; ++r) {
    int next = 0, first = (int)since.size();
    const auto fetch = [&](int i, int place) {
      if (ring[place].on_way >= 0) broken = 1;
      if (i != (int)since.size() - first) broken = 2;
      ring[place].on_way = (int)since.size();
      since.push_back(now);
    };
    const auto arrived = [&](int place, uint32_t parity) {
      Place& p = ring[place];
      if ((uint32_t)(p.filled & 1) != parity) return true;      // that phase is over
      if (p.on_way < 0) {
        broken = 3;                                 // waits for nothing
        return false;
      }
      const int c = p.on_way;
      if (how[c] == 2 || now < since[c] + how[c]) {
        ++now;
        return false;
      }
      p.holds = c;
      p.on_way = -1;
      ++p.filled;
      return true;
    };
    const auto use = [&](int i, int place, bool here) {
      if (i != next++) broken = 4;
      if (here && ring[place].holds != first + i) broken = 5;
      return i;
    };
    const auto then = [&](int i, int x) {
      if (x != i) broken = 6;
    };
    copies = sp::walk_ring<kRing>(it, pieces[r], copies, fetch, arrived, use, then);
    if (next != pieces[r]) broken = 7;
    it += pieces[r];
  }
  for (const Place& p : ring)
    if (p.on_way >= 0 && how[p.on_way] != 2) broken = 8;
  return broken;
}
}
