// Places in a pool of pages, for host and device code.
#pragma once

#include <stddef.h>
#include <stdint.h>

#include <hip/hip_runtime.h>

namespace adapld {

__host__ __device__ inline int log2_pow2(int x) {
  int s = 0;
  while ((1 << s) < x) ++s;
  return s;
}

// Row index of (page, kv head, offset in the page) in arrays [n_pages, Hkv,
// page_size, ...].  64-bit: a pool may hold more than 2^31 rows.
__host__ __device__ inline size_t pool_row(int page, int g, int off, int Hkv, int page_shift) {
  return ((((size_t)page * Hkv + g) << page_shift) + off);
}

// A page id from a table, inside the pool whatever the table holds.
__host__ __device__ inline int page_in_pool(int page, int n_pages) {
  return page < 0 ? 0 : page >= n_pages ? n_pages - 1 : page;
}

}  // namespace adapld
