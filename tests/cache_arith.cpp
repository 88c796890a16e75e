// Index arithmetic that the cache kernels share with the host, for tests of it
// without a GPU.
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
}
