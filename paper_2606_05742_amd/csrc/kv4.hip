// The paged 4-bit K/V cache: its pages (page map) and its rows (append and
// gather).  The attention that reads it is in kv4_verify.hip.
#include <hip/hip_runtime.h>

#include "adapld_internal.h"
#include "device_utils.h"
#include "kv4.h"

namespace adapld {
namespace {

// ------------------------------------------------------------------- page map
//
// Workgroup 0 keeps the state: it takes the sequences in index order, kMapThreads
// at a time, and has one prefix sum for the pages given back and one for the
// pages asked for.  The moved pages of such a group are then laid end to end
// over the threads (each finds its sequence in the prefix sums by bisection), so
// one long prompt does not make one thread walk its pages.  Everything is given
// back before anything is handed out: the stack's height after the first pass
// decides who is served, and the second pass may pop what the first has pushed.
//
// The slots of a batch that is one such group are filled in the same launch by
// the other workgroups, which repeat the prefix sums and work out the page of a
// new token from what workgroup 0 does not write: the old count, the stack below
// it and the table entries that were held before the call.  Larger batches, and
// calls that update the count in place, leave few slots to workgroup 0 and take a
// second launch for many.
constexpr int kMapThreads = 1024;
constexpr int kMapWaves = kMapThreads / kWave;
enum SlotsBy { kSlotsByFirst, kSlotsByOthers, kSlotsLater };

struct MapArgs {
  const int32_t* lens_old;
  const int32_t* lens_new;
  int B, page_shift, max_pages, n_pages, N;
  int32_t* page_table;   // read and written by one launch: never through the scalar cache
  int32_t* free_pages;
  const int32_t* free_count;
  int32_t* free_count_out;
  int32_t* slot_map;
  int32_t* granted;
};

// Lengths in [0, max_pages << page_shift], which fits 31 bits by the host's check.
__device__ __forceinline__ int clamp_len(int len, const MapArgs& a) {
  return min(max(len, 0), a.max_pages << a.page_shift);
}
__device__ __forceinline__ int pages_of(int len, int shift) {
  return (int)(((int64_t)len + (1 << shift) - 1) >> shift);
}

// Inclusive prefix sum over the workgroup; `total` is the sum.
__device__ __forceinline__ int block_incl_scan(int v, int* s_wave, int& total) {
  const int lane = lane_id(), wave = threadIdx.x / kWave;
  const int in = wave_incl_scan_i32(v);
  if (lane == kWave - 1) s_wave[wave] = in;
  __syncthreads();
  int before = 0, sum = 0;
#pragma unroll
  for (int w = 0; w < kMapWaves; ++w) {
    const int t = s_wave[w];
    before += w < wave ? t : 0;
    sum += t;
  }
  __syncthreads();
  total = sum;
  return in + before;
}

// The first index whose inclusive prefix sum exceeds p (p below the total).
__device__ __forceinline__ int find_in_prefix(const int* s_incl, int p) {
  int lo = 0;
#pragma unroll
  for (int step = kMapThreads / 2; step > 0; step >>= 1)
    if (s_incl[lo + step - 1] <= p) lo += step;
  return lo;
}

__device__ __forceinline__ int slot_in_page(const MapArgs& a, int page, int pos) {
  if (page < 0 || page >= a.n_pages) return -1;
  return (page << a.page_shift) + (pos & ((1 << a.page_shift) - 1));
}
__device__ __forceinline__ int slot_at(const MapArgs& a, int b, int pos) {
  return slot_in_page(a, a.page_table[(size_t)b * a.max_pages + (pos >> a.page_shift)], pos);
}

// Slots of a batch of at most kMapThreads sequences, beside workgroup 0.
__device__ void fill_slots_beside(const MapArgs& a, int* s_back, int* s_need, int* s_wave, int* s_first) {
  const int tid = threadIdx.x, shift = a.page_shift;
  int back = 0, need = 0;
  if (tid < a.B) {
    const int held = pages_of(clamp_len(a.lens_old[tid], a), shift);
    const int want = pages_of(clamp_len(a.lens_new[tid], a), shift);
    back = max(held - want, 0);
    need = max(want - held, 0);
    s_first[tid] = want;
  }
  const int start = min(max(a.free_count[0], 0), a.n_pages);
  int total;
  s_back[tid] = block_incl_scan(back, s_wave, total);
  const int height = (int)min<int64_t>((int64_t)start + total, a.n_pages);
  s_need[tid] = block_incl_scan(need, s_wave, total);
  __syncthreads();
  // The batch's slots end to end over the workgroups; B * N fits 31 bits by the
  // host's check, so one more round fits 32.
  const uint32_t end = (uint32_t)a.B * (uint32_t)a.N, step = (gridDim.x - 1) * kMapThreads;
  for (uint32_t at_slot = (blockIdx.x - 1) * kMapThreads + tid; at_slot < end; at_slot += step) {
    const int b = (int)(at_slot / (uint32_t)a.N), i = (int)(at_slot - (uint32_t)b * (uint32_t)a.N);
    const int o = clamp_len(a.lens_old[b], a), n = clamp_len(a.lens_new[b], a);
    const int before = b > 0 ? s_need[b - 1] : 0;
    const bool granted = s_need[b] <= height || s_need[b] == before;
    int slot = -1;
    if (granted && i < n - o) {
      const int held = pages_of(o, shift);
      const int pos = o + i, at = pos >> shift;
      int page;
      if (at < held) {
        page = a.page_table[(size_t)b * a.max_pages + at];
      } else {
        const int from = height - 1 - (before + at - held);   // its place on the stack
        if (from < start) {
          page = a.free_pages[from];
        } else {   // given back by this call
          const int p = from - start, seq = find_in_prefix(s_back, p);
          page = a.page_table[(size_t)seq * a.max_pages + s_first[seq] + p - (seq > 0 ? s_back[seq - 1] : 0)];
        }
      }
      slot = slot_in_page(a, page, pos);
    }
    a.slot_map[at_slot] = slot;
  }
}

__global__ __launch_bounds__(kMapThreads) void page_map_kernel(const MapArgs a, SlotsBy slots) {
  __shared__ int s_incl[kMapThreads];
  __shared__ int s_first[kMapThreads];   // first page index of the sequence's moved pages
  __shared__ int s_need[kMapThreads];
  __shared__ int s_wave[kMapWaves];
  if (blockIdx.x > 0) {
    fill_slots_beside(a, s_incl, s_need, s_wave, s_first);
    return;
  }
  const int tid = threadIdx.x;
  const int shift = a.page_shift;
  const int start = min(max(a.free_count[0], 0), a.n_pages);

  int64_t back = 0;   // pages given back so far
  for (int b0 = 0; b0 < a.B; b0 += kMapThreads) {
    const int b = b0 + tid;
    int n = 0, first = 0;
    if (b < a.B) {
      const int held = pages_of(clamp_len(a.lens_old[b], a), shift);
      const int want = pages_of(clamp_len(a.lens_new[b], a), shift);
      n = max(held - want, 0);
      first = want;
    }
    int total;
    const int incl = block_incl_scan(n, s_wave, total);
    s_incl[tid] = incl;
    s_first[tid] = first;
    __syncthreads();
    for (int p = tid; p < total; p += kMapThreads) {
      const int i = find_in_prefix(s_incl, p);
      const int j = p - (i > 0 ? s_incl[i - 1] : 0);
      const int64_t at = start + back + p;
      // a count that does not fit the pool (pages given back twice) drops the rest
      if (at < a.n_pages) a.free_pages[at] = a.page_table[(size_t)(b0 + i) * a.max_pages + s_first[i] + j];
    }
    back += total;
    __syncthreads();
  }

  const int height = (int)min<int64_t>(start + back, a.n_pages);
  int64_t asked = 0;   // pages asked for so far, served or not
  int left = height;
  for (int b0 = 0; b0 < a.B; b0 += kMapThreads) {
    const int b = b0 + tid;
    int need = 0, held = 0;
    if (b < a.B) {
      held = pages_of(clamp_len(a.lens_old[b], a), shift);
      need = max(pages_of(clamp_len(a.lens_new[b], a), shift) - held, 0);
    }
    int total;
    const int incl = block_incl_scan(need, s_wave, total);
    const bool ok = asked + incl <= height || need == 0;
    if (b < a.B) a.granted[b] = ok;
    s_incl[tid] = incl;
    s_first[tid] = held;
    // Sequences are served while their running sum fits, so the pages handed
    // out here are the first `served` of the group's.
    const int fits = (int)wave_max_i32(ok && need > 0 ? incl : 0);
    __syncthreads();
    if (lane_id() == 0) s_wave[tid / kWave] = fits;
    __syncthreads();
    int served = 0;
#pragma unroll
    for (int w = 0; w < kMapWaves; ++w) served = max(served, s_wave[w]);
    for (int p = tid; p < served; p += kMapThreads) {
      const int i = find_in_prefix(s_incl, p);
      const int j = p - (i > 0 ? s_incl[i - 1] : 0);
      a.page_table[(size_t)(b0 + i) * a.max_pages + s_first[i] + j] = a.free_pages[height - 1 - (asked + p)];
    }
    left -= served;
    asked += total;
    __syncthreads();
  }
  if (tid == 0) a.free_count_out[0] = left;

  if (slots != kSlotsByFirst) return;
  __syncthreads();
  for (int idx = tid; idx < a.B * a.N; idx += kMapThreads) {
    const int b = idx / a.N, i = idx - b * a.N;
    const int o = clamp_len(a.lens_old[b], a), n = clamp_len(a.lens_new[b], a);
    a.slot_map[idx] = a.granted[b] && i < n - o ? slot_at(a, b, o + i) : -1;
  }
}

// Slots of a larger batch, after the pages.
__global__ __launch_bounds__(kKv4SlotThreads) void slot_map_kernel(const MapArgs a) {
  const int b = blockIdx.y;
  const int o = clamp_len(a.lens_old[b], a), n = clamp_len(a.lens_new[b], a);
  const bool ok = a.granted[b] != 0;
#pragma unroll
  for (int k = 0; k < kKv4SlotsPerBlock / kKv4SlotThreads; ++k) {
    const int i = blockIdx.x * kKv4SlotsPerBlock + k * kKv4SlotThreads + threadIdx.x;
    if (i < a.N) a.slot_map[(size_t)b * a.N + i] = ok && i < n - o ? slot_at(a, b, o + i) : -1;
  }
}

// --------------------------------------------------------------- append, gather
//
// 16 lanes take one row (token, kv head): a lane 8 dimensions of K and of V, so
// loads are 16 bytes a lane and the row's codes leave as one 64-byte line.
// Four lanes share a scale.
constexpr int kRowThreads = 256;
constexpr int kRowLanes = ADAPLD_HEAD_DIM / 8;

struct RowArgs {
  const uint16_t* k_new;   // append: source rows
  const uint16_t* v_new;
  const int32_t* rows;
  uint16_t* k_out;         // gather: destination rows
  uint16_t* v_out;
  const int32_t* slot_map;
  int B, n_src, N, Hkv, page_shift, n_pages;
  uint8_t* k_codes;
  uint8_t* k_scales;
  uint8_t* v_codes;
  uint8_t* v_scales;
};

// The 8 values of x (bf16) as codes, and the exponent byte of their group of
// four lanes.  The scale X is the smallest power of two with amax < 7 X: then
// no value is off by more than X, the half step below 8 X that saturating at
// 6 X also costs at most.  On the bits of a bf16 amax this is adding 0x20 (a
// quarter of the mantissa, so 1.75 carries into the exponent) and taking 2
// from the exponent; 1..252 keeps X normal and 6 X finite in bf16.  Values are
// rounded to the nearest E2M1, ties to even, once.
__device__ __forceinline__ uint32_t quantise8(uint4 x, uint32_t& exponent) {
  const uint32_t w[4] = {x.x, x.y, x.z, x.w};
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) m = max(m, max(w[i] & 0x7fffu, (w[i] >> 16) & 0x7fffu));
  m = max(m, xor_lanes_u32<1>(m));
  m = max(m, xor_lanes_u32<2>(m));
  const int e = min(max((int)((m + 0x20u) >> 7) - 2, 1), 252);
  exponent = (uint32_t)e;
  const float X = __uint_as_float((uint32_t)e << 23);
  uint32_t c = 0;
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2_t, w[0]), X, 0);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2_t, w[1]), X, 1);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2_t, w[2]), X, 2);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2_t, w[3]), X, 3);
  return c;
}

__device__ __forceinline__ uint4 dequantise8(uint32_t c, uint32_t exponent) {
  const float X = __uint_as_float(exponent << 23);
  uint4 r;
  r.x = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, X, 0));
  r.y = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, X, 1));
  r.z = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, X, 2));
  r.w = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, X, 3));
  return r;
}

// The row of this lane's 16: (token t of B * N, kv head g); false past the end.
struct RowAt {
  uint32_t t;
  int g, slot;
};
__device__ __forceinline__ bool row_of_thread(const RowArgs& a, RowAt& r) {
  // B * N * Hkv fits 31 bits by the host's check
  const uint32_t row = blockIdx.x * (kRowThreads / kRowLanes) + threadIdx.x / kRowLanes;
  r.t = row / (uint32_t)a.Hkv;
  r.g = (int)(row - r.t * (uint32_t)a.Hkv);
  if (r.t >= (uint32_t)a.B * (uint32_t)a.N) return false;
  r.slot = a.slot_map[r.t];
  return r.slot >= 0 && (r.slot >> a.page_shift) < a.n_pages;
}
__device__ __forceinline__ size_t row_in_pool(const RowArgs& a, const RowAt& r) {
  return kv4_row(r.slot >> a.page_shift, r.g, r.slot & ((1 << a.page_shift) - 1), a.Hkv, a.page_shift);
}

__global__ __launch_bounds__(kRowThreads) void kv4_append_kernel(const RowArgs a) {
  RowAt r;
  if (!row_of_thread(a, r)) return;   // the 16 lanes of a row leave together
  const uint32_t b = r.t / (uint32_t)a.N;
  const int src = a.rows ? a.rows[r.t] : (int)(r.t - b * a.N);
  if (src < 0 || src >= a.n_src) return;
  const int part = threadIdx.x % kRowLanes;
  const size_t from = (((size_t)b * a.n_src + src) * a.Hkv + r.g) * ADAPLD_HEAD_DIM + part * 8;
  const uint4 kx = *reinterpret_cast<const uint4*>(a.k_new + from);
  const uint4 vx = *reinterpret_cast<const uint4*>(a.v_new + from);
  uint32_t ke, ve;
  const uint32_t kc = quantise8(kx, ke), vc = quantise8(vx, ve);
  const size_t to = row_in_pool(a, r);
  *reinterpret_cast<uint32_t*>(a.k_codes + to * kKv4RowBytes + part * 4) = kc;
  *reinterpret_cast<uint32_t*>(a.v_codes + to * kKv4RowBytes + part * 4) = vc;
  if (part % 4 == 0) {
    a.k_scales[to * kKv4Scales + part / 4] = (uint8_t)ke;
    a.v_scales[to * kKv4Scales + part / 4] = (uint8_t)ve;
  }
}

// STREAM: the rows are stored with the non-temporal hint.
template <bool STREAM>
__global__ __launch_bounds__(kRowThreads) void kv4_gather_kernel(const RowArgs a) {
  RowAt r;
  if (!row_of_thread(a, r)) return;
  const int part = threadIdx.x % kRowLanes;
  const size_t from = row_in_pool(a, r);
  const uint32_t kc = *reinterpret_cast<const uint32_t*>(a.k_codes + from * kKv4RowBytes + part * 4);
  const uint32_t vc = *reinterpret_cast<const uint32_t*>(a.v_codes + from * kKv4RowBytes + part * 4);
  const uint32_t ke = a.k_scales[from * kKv4Scales + part / 4];
  const uint32_t ve = a.v_scales[from * kKv4Scales + part / 4];
  const size_t to = ((size_t)r.t * a.Hkv + r.g) * ADAPLD_HEAD_DIM + part * 8;
  typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
  const u32x4_t kx = __builtin_bit_cast(u32x4_t, dequantise8(kc, ke));
  const u32x4_t vx = __builtin_bit_cast(u32x4_t, dequantise8(vc, ve));
  u32x4_t* const k_to = reinterpret_cast<u32x4_t*>(a.k_out + to);
  u32x4_t* const v_to = reinterpret_cast<u32x4_t*>(a.v_out + to);
  if constexpr (STREAM) {
    __builtin_nontemporal_store(kx, k_to);
    __builtin_nontemporal_store(vx, v_to);
  } else {
    *k_to = kx;
    *v_to = vx;
  }
}

}  // namespace

hipError_t launch_kv4_page_map(const int32_t* lens_old, const int32_t* lens_new, int B, int page_size, int max_pages,
                               int n_pages, int N, int32_t* page_table, int32_t* free_pages,
                               const int32_t* free_count, int32_t* free_count_out, int32_t* slot_map,
                               int32_t* granted, hipStream_t stream) {
  MapArgs a{};
  a.lens_old = lens_old; a.lens_new = lens_new;
  a.B = B; a.page_shift = log2_pow2(page_size); a.max_pages = max_pages; a.n_pages = n_pages; a.N = N;
  a.page_table = page_table; a.free_pages = free_pages; a.free_count = free_count;
  a.free_count_out = free_count_out; a.slot_map = slot_map; a.granted = granted;
  // us a call inside a graph, slots by the other workgroups / by the first: 16 x 13
  // slots 4.2 / 4.5, 64 x 64 4.2 / 5.9, 16 x 2048 5.0 / 18.  In place, by a second
  // launch / by the first: 16 x 13 5.6 / 4.1, 64 x 64 5.8 / 5.0, 64 x 128 5.6 / 6.1.
  constexpr int kFewSlots = 4 * kMapThreads;
  constexpr int64_t kOthersMax = 2 * 256 - 1;   // two workgroups a CU; they take the slots in turn
  const int64_t total = (int64_t)B * N;
  const SlotsBy slots = N == 0                                               ? kSlotsByFirst
                        : B <= kMapThreads && free_count_out != free_count ? kSlotsByOthers
                        : total <= kFewSlots                               ? kSlotsByFirst
                                                                           : kSlotsLater;
  const int64_t groups = (total + kMapThreads - 1) / kMapThreads;
  const unsigned others = slots == kSlotsByOthers ? (unsigned)(groups < kOthersMax ? groups : kOthersMax) : 0u;
  hipLaunchKernelGGL(page_map_kernel, dim3(1 + others), dim3(kMapThreads), 0, stream, a, slots);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || slots != kSlotsLater) return e;
  hipLaunchKernelGGL(slot_map_kernel, dim3(kv4_slot_blocks(N), B), dim3(kKv4SlotThreads), 0, stream, a);
  return hipGetLastError();
}

namespace {
inline unsigned row_blocks(int B, int N, int Hkv) {
  return (unsigned)(((int64_t)B * N * Hkv * kRowLanes + kRowThreads - 1) / kRowThreads);
}
}  // namespace

hipError_t launch_kv4_append(const uint16_t* k_new, const uint16_t* v_new, const int32_t* rows,
                             const int32_t* slot_map, int B, int n_src, int N, int Hkv, int page_size, int n_pages,
                             uint8_t* k_codes, uint8_t* k_scales, uint8_t* v_codes, uint8_t* v_scales,
                             hipStream_t stream) {
  RowArgs a{};
  a.k_new = k_new; a.v_new = v_new; a.rows = rows; a.slot_map = slot_map;
  a.B = B; a.n_src = n_src; a.N = N; a.Hkv = Hkv; a.page_shift = log2_pow2(page_size); a.n_pages = n_pages;
  a.k_codes = k_codes; a.k_scales = k_scales; a.v_codes = v_codes; a.v_scales = v_scales;
  hipLaunchKernelGGL(kv4_append_kernel, dim3(row_blocks(B, N, Hkv)), dim3(kRowThreads), 0, stream, a);
  return hipGetLastError();
}

hipError_t launch_kv4_gather(const uint8_t* k_codes, const uint8_t* k_scales, const uint8_t* v_codes,
                             const uint8_t* v_scales, const int32_t* slot_map, int B, int N, int Hkv, int page_size,
                             int n_pages, uint16_t* k_out, uint16_t* v_out, hipStream_t stream) {
  RowArgs a{};
  a.k_out = k_out; a.v_out = v_out; a.slot_map = slot_map;
  a.B = B; a.N = N; a.Hkv = Hkv; a.page_shift = log2_pow2(page_size); a.n_pages = n_pages;
  a.k_codes = const_cast<uint8_t*>(k_codes); a.k_scales = const_cast<uint8_t*>(k_scales);
  a.v_codes = const_cast<uint8_t*>(v_codes); a.v_scales = const_cast<uint8_t*>(v_scales);
  // Rows beyond what the L2s hold (32 MiB) are streamed, us a call plain / non-
  // temporal: 16 x 2048 rows of 8 heads (128 MiB) 35.9 / 28.0, 5 x 6007 of 4 (59
  // MiB) 15.1 / 14.2; a consumer finds fewer ones in the caches.
  constexpr size_t kPlainBytes = (size_t)32 << 20;
  const dim3 grid(row_blocks(B, N, Hkv));
  if ((size_t)B * N * Hkv * ADAPLD_HEAD_DIM * 4 > kPlainBytes)
    hipLaunchKernelGGL(kv4_gather_kernel<true>, grid, dim3(kRowThreads), 0, stream, a);
  else
    hipLaunchKernelGGL(kv4_gather_kernel<false>, grid, dim3(kRowThreads), 0, stream, a);
  return hipGetLastError();
}

}  // namespace adapld
