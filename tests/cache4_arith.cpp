// Index arithmetic that the kernels of the 4-bit cache share with the host, for tests
// of it without a GPU.
#include <algorithm>

#include "sp_cache4.cuh"

extern "C" {
// Workers of the plan for R query rows of a K/V head.
int arith4_workers(int R, int D, int sms) { return sp::plan4_of(R, D, sms).workers; }

// The merge of R rows of a K/V head, where `side` workers walk beside each other, over the
// parts that a note gives: how many there are (0: the note is not followed), and where in the workspace of a handle for
// up to max_T tokens the first byte that is read lies, and the first behind the last one;
// at[2], end[2]: of references and sums, of elements.  Returns the workspace's bytes.
int64_t arith4_merge(int max_T, int Hq, int Hkv, int D, int sms, int R, int side, int32_t slot, int32_t last, int32_t* parts,
                     int64_t* at, int64_t* end) {
  const sp::Cache4Workspace w = sp::cache4_workspace(sp::Cache4Shape{max_T, Hq, Hkv, D, 1 << 20, 0}, sms);
  const sp::Plan4 plan = sp::plan4_of(R, D, sms);
  const sp::Slots4 slots = sp::slots4_of(plan);
  const int64_t rows = 8 * plan.NT, row_bytes[2] = {16, (plan.wide ? 128 : 64) * 4}, base[2] = {(int64_t)slots.ml, (int64_t)slots.o};
  *parts = sp::parts_within(slot, last, plan.workers) ? std::max(0, last - (slot >> 1)) / side + 1 : 0;
  for (int k = 0; k < 2; ++k)
    for (int i = 0; i < *parts; ++i) {
      const int64_t s = i == 0 ? slot : 2 * ((slot >> 1) + (int64_t)i * side);
      const int64_t from = w.slots + base[k] + s * rows * row_bytes[k], to = from + rows * row_bytes[k];
      at[k] = i == 0 || from < at[k] ? from : at[k];
      end[k] = i == 0 || to > end[k] ? to : end[k];
    }
  return (int64_t)w.bytes;
}
// Where the two kinds of data of R rows begin in that workspace, and end.
void arith4_slots(int max_T, int Hq, int Hkv, int D, int sms, int R, int64_t* at) {
  const sp::Cache4Workspace w = sp::cache4_workspace(sp::Cache4Shape{max_T, Hq, Hkv, D, 1 << 20, 0}, sms);
  const sp::Slots4 slots = sp::slots4_of(sp::plan4_of(R, D, sms));
  at[0] = w.slots + slots.ml;
  at[1] = w.slots + slots.o;
  at[2] = w.slots + slots.end;
}
}
