// Layout of the paged 4-bit K/V cache, for host and device code.
//
// A row is one token of one kv head: kKv4RowBytes bytes of E2M1 codes (two
// dimensions a byte, the even one in the low half) and kKv4Scales exponent
// bytes (bias 127), one for each ADAPLD_KV4_GROUP dimensions.  The rows of a
// (page, kv head) are contiguous, codes and scales in arrays of their own, so
// a tile of keys is read in long lines and a row's codes stay 16-byte aligned.
#pragma once

#include <stddef.h>
#include <stdint.h>

#include "adapld.h"

namespace adapld {

constexpr int kKv4RowBytes = ADAPLD_HEAD_DIM / 2;                   // 64
constexpr int kKv4Scales = ADAPLD_HEAD_DIM / ADAPLD_KV4_GROUP;      // 4

__host__ __device__ inline int log2_pow2(int x) {
  int s = 0;
  while ((1 << s) < x) ++s;
  return s;
}

// Row index of (page, kv head, offset in the page); times kKv4RowBytes or
// kKv4Scales the byte offset of its codes or scales.  64-bit: a pool may hold
// more than 2^31 rows.
__host__ __device__ inline size_t kv4_row(int page, int g, int off, int Hkv, int page_shift) {
  return ((((size_t)page * Hkv + g) << page_shift) + off);
}

// Blocks of the slot map's own launch for N slots of a sequence.  N may be
// INT32_MAX, so the sum is formed in 64 bits.
constexpr int kKv4SlotThreads = 256;
constexpr int kKv4SlotsPerBlock = 4 * kKv4SlotThreads;
constexpr unsigned kv4_slot_blocks(int N) {
  return (unsigned)(((int64_t)N + kKv4SlotsPerBlock - 1) / kKv4SlotsPerBlock);
}

// A page id from a table, inside the pool whatever the table holds.
__host__ __device__ inline int kv4_page_in_pool(int page, int n_pages) {
  return page < 0 ? 0 : page >= n_pages ? n_pages - 1 : page;
}

}  // namespace adapld
