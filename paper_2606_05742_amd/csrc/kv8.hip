// The rows of the paged 8-bit K/V cache: new tokens quantised into its blocks.  The
// attention that reads it is in kv8_verify.hip.
#include <hip/hip_runtime.h>

#include "adapld_internal.h"
#include "device_utils.h"
#include "kv8.h"
#include "kv8_device.h"

namespace adapld {
namespace {

// A wave takes one (sequence, block, kv head): its 16 rows in four rounds of four,
// a row 16 lanes of 8 dimensions (16 bytes of bf16, 8 of codes), K and V.  The new
// rows decide how far the block's exponent has to rise; the rows of older tokens are
// read only then, and rounded again to the new step (exactly, but for values below
// 2^-6 of the new scale, whose last bits E4M3 no longer holds).  Few rows take a
// launch and three round trips to memory (lengths, page, rows with the scale): 13 accepted
// nodes of 16 sequences 4.6 us.  Prompts are bound by HBM.
constexpr int kAppendThreads = 256;
constexpr int kAppendWaves = kAppendThreads / kWave;
// A bf16 magnitude's bits: below, 448 times the largest scale holds it.
constexpr uint32_t kPlainBelow = (uint32_t)(kKv8MaxExp + 8) << 7;

struct AppendArgs {
  const uint16_t* x[2];   // K and V rows
  const int32_t* rows;
  const int32_t* lens_old;
  const int32_t* lens_new;
  const int32_t* page_table;
  int B, n_src, N, Hkv, page_shift, n_pages, max_pages;
  uint32_t blocks;        // of a sequence
  uint8_t* codes[2];
  uint8_t* scales[2];
};

// STREAM: the source rows are loaded with the non-temporal hint.
template <bool STREAM>
__global__ __launch_bounds__(kAppendThreads) void kv8_append_kernel(const AppendArgs a) {
  // B * blocks * Hkv fits 31 bits by the host's check
  const uint32_t job = blockIdx.x * kAppendWaves + __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const uint32_t sb = job / (uint32_t)a.Hkv;
  const int g = (int)(job - sb * (uint32_t)a.Hkv);
  const int b = (int)(sb / a.blocks);
  if (b >= a.B) return;
  const int capacity = a.max_pages << a.page_shift;   // fits 31 bits by the host's check
  const int old = min(max(a.lens_old[b], 0), capacity);
  const int end = (int)min((int64_t)min(max(a.lens_new[b], 0), capacity), (int64_t)old + a.N);
  const int64_t start64 = (int64_t)((old >> kKv8BlockShift) + (int)(sb - (uint32_t)b * a.blocks)) << kKv8BlockShift;
  if (start64 >= end || end <= old) return;
  const int start = (int)start64;
  const int page = a.page_table[(size_t)b * a.max_pages + (start >> a.page_shift)];
  if (page < 0 || page >= a.n_pages) return;
  const size_t row0 = pool_row(page, g, start & ((1 << a.page_shift) - 1), a.Hkv, a.page_shift);
  const int part = lane_id() % kKv8RowLanes, sub = lane_id() / kKv8RowLanes;

  uint4 x[2][4];
#pragma unroll
  for (int t = 0; t < 4; ++t) {
    const int i = start + 4 * t + sub - old;
    int src = -1;
    if (i >= 0 && i < end - old) src = a.rows ? a.rows[(size_t)b * a.N + i] : i;
#pragma unroll
    for (int n = 0; n < 2; ++n) {
      x[n][t] = make_uint4(0, 0, 0, 0);   // a source row outside [0, n_src) is stored as zeros
      if (src >= 0 && src < a.n_src) {
        typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
        const u32x4_t* const p = reinterpret_cast<const u32x4_t*>(
            a.x[n] + (((size_t)b * a.n_src + src) * a.Hkv + g) * ADAPLD_HEAD_DIM + part * 8);
        if constexpr (STREAM) x[n][t] = __builtin_bit_cast(uint4, __builtin_nontemporal_load(p));
        else x[n][t] = __builtin_bit_cast(uint4, *p);
      }
    }
  }
#pragma unroll
  for (int n = 0; n < 2; ++n) {
    uint32_t m = 0;
#pragma unroll
    for (int t = 0; t < 4; ++t) m = kv8_max2(m, kv8_amax2(x[n][t]));
    m = kv8_wave_max(kv8_halves_max(m));
    // infinities, NaN and values near the largest take the longer way
    const bool any = m >= kPlainBelow;
    if (any) {
      m = 0;
#pragma unroll
      for (int t = 0; t < 4; ++t) m = max(m, kv8_finite_amax(x[n][t]));
      m = kv8_wave_max(m);
    }
    int e = kv8_exponent(m);
    uint8_t* const scale = a.scales[n] + (row0 >> kKv8BlockShift);
    const bool held = start < old;
    const int before = held ? *scale : 0;
    e = max(e, before);
    if (lane_id() == 0 && e != before) *scale = (uint8_t)e;
    const bool again = held && e != before;
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      const int r = 4 * t + sub;
      uint2* const at = reinterpret_cast<uint2*>(a.codes[n] + (row0 + r) * kKv8RowBytes + part * 8);
      if (start + r >= old) {
        if (start + r < end) *at = any ? kv8_quantise(x[n][t], e) : kv8_round(x[n][t], kv8_scale(e));
      } else if (again) {
        *at = kv8_rescale(*at, before, e);
      }
    }
  }
}

}  // namespace

hipError_t launch_kv8_append(const uint16_t* k_new, const uint16_t* v_new, const int32_t* rows, const int32_t* lens_old,
                             const int32_t* lens_new, const int32_t* page_table, int B, int n_src, int N, int Hkv,
                             int page_size, int n_pages, int max_pages, uint8_t* k_codes, uint8_t* k_scales,
                             uint8_t* v_codes, uint8_t* v_scales, hipStream_t stream) {
  AppendArgs a{};
  a.x[0] = k_new; a.x[1] = v_new; a.rows = rows; a.lens_old = lens_old; a.lens_new = lens_new;
  a.page_table = page_table;
  a.B = B; a.n_src = n_src; a.N = N; a.Hkv = Hkv; a.page_shift = log2_pow2(page_size);
  a.n_pages = n_pages; a.max_pages = max_pages;
  a.blocks = (uint32_t)kv8_blocks_touched(N);
  a.codes[0] = k_codes; a.codes[1] = v_codes; a.scales[0] = k_scales; a.scales[1] = v_scales;
  const int64_t jobs = (int64_t)B * a.blocks * Hkv;
  const dim3 grid((unsigned)((jobs + kAppendWaves - 1) / kAppendWaves));
  // Prompts beyond what the L2s hold (32 MiB) are streamed, us a call plain / non-temporal:
  // 16 x 2048 rows of 8 heads (180 MB in and out) 39.5 / 33.3, 5.4 TB/s; fewer rows come
  // from the caches (accepted nodes of 16 sequences 4.6 / 4.8, three round trips to memory).
  constexpr size_t kPlainBytes = (size_t)32 << 20;
  if ((size_t)B * N * Hkv * ADAPLD_HEAD_DIM * 4 > kPlainBytes)
    hipLaunchKernelGGL(kv8_append_kernel<true>, grid, dim3(kAppendThreads), 0, stream, a);
  else
    hipLaunchKernelGGL(kv8_append_kernel<false>, grid, dim3(kAppendThreads), 0, stream, a);
  return hipGetLastError();
}

}  // namespace adapld
