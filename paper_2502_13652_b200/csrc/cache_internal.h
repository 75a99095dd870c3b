// What the calls on a paged key/value cache share (cache_pages.cu, verify_attention.cu).  See include/c2t.h.
#pragma once
#include "c2t_internal.h"

namespace c2t {

// the host's checks of a cache description: C2T_OK or the code that a call returns
int check_cache(const c2t_cache *c);

inline bool vector_aligned(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }
inline bool vector_stride(int64_t elements) { return elements % 8 == 0; }      // elements of 16 bits

#ifdef __CUDACC__
__device__ __forceinline__ void cache_fault(const c2t_cache &c, int b, uint32_t bits) {
  if (c.status_dev) atomicOr(c.status_dev + b, bits);
}

// pages that slot b holds, whatever its word says
__device__ __forceinline__ int held_pages(const c2t_cache &c, int b) {
  const int n = c.held_dev[b];
  return n < 0 ? 0 : n > c.max_pages ? c.max_pages : n;
}
#endif

}  // namespace c2t
