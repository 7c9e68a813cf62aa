// Layout of the paged 8-bit K/V cache, for host and device code.
//
// A row is one token of one kv head: ADAPLD_HEAD_DIM E4M3 codes of a byte each.  The
// rows of a (page, kv head) are contiguous, and every ADAPLD_KV8_BLOCK of them share
// an exponent byte e (bias 127): a value is E4M3 * 2^(e - 127), exact in bf16 for e
// in kKv8MinExp..kKv8MaxExp (2^-9 * 2^(e - 127) is a normal bf16, 448 * 2^(e - 127) a
// finite one).
#pragma once

#include "adapld.h"
#include "paged.h"

namespace adapld {

constexpr int kKv8RowBytes = ADAPLD_HEAD_DIM;
constexpr int kKv8BlockShift = 4;
static_assert(1 << kKv8BlockShift == ADAPLD_KV8_BLOCK, "tokens of a block");
constexpr int kKv8MinExp = 10, kKv8MaxExp = 246;

// Blocks that N tokens behind any position can touch.
constexpr int64_t kv8_blocks_touched(int64_t N) { return (N + ADAPLD_KV8_BLOCK - 2) / ADAPLD_KV8_BLOCK + 1; }

}  // namespace adapld
