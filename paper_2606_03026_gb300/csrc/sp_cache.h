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

// Tiles of entries that a call has at most (its launch counts them in 32 bits).
int64_t attend_tiles(const CacheShape& s, const sp_attend& c);
cudaError_t launch_attend(const CacheShape& s, const sp_attend& c, uint8_t* ws, int* err,
                          cudaStream_t stream);
cudaError_t launch_evict(const CacheShape& s, const sp_evict& c, uint8_t* ws, cudaStream_t stream);
cudaError_t launch_verify(const sp_verify& c, cudaStream_t stream);

}  // namespace sp
