// Eviction from the paged 8-bit cache by accumulated attention weight.
//
// Two launches: one workgroup a (sequence, kv head) finds which tokens stay and which
// of them move where, then a wave a block of the kept slots moves the rows.  Rows move
// only from slots >= budget to free slots below it, so no row is read that the launch
// writes, and nothing moves that can stay.
#include "adapld_internal.h"
#include "kv8_device.h"

namespace adapld {
namespace {

constexpr int kSelectThreads = 1024;
constexpr int kSelectWaves = kSelectThreads / kWave;
constexpr int kBins = 2048;
constexpr int kMoveThreads = 256;
constexpr int kMoveWaves = kMoveThreads / kWave;

// Workspace of a (sequence, kv head): src[budget], the slot that each kept slot takes
// its token from; free[most], the freed slots in ascending order; moved, their number.
struct EvictWs {
  int32_t* src;
  int32_t* free;
  int32_t* moved;
};
__host__ __device__ inline int evict_most(int L_max, int budget) { return L_max - budget < budget ? L_max - budget : budget; }
__device__ __forceinline__ EvictWs evict_ws(const EvictCall& c, size_t pair, size_t pairs) {
  int32_t* const base = static_cast<int32_t*>(c.ws);
  const size_t most = evict_most(c.L_max, c.budget);
  return {base + pair * c.budget, base + pairs * c.budget + pair * most, base + pairs * (c.budget + most) + pair};
}

// A float's bits as an unsigned number of the same order.
__device__ __forceinline__ uint32_t ordered_bits(float w) {
  const uint32_t u = __float_as_uint(w);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// Exclusive prefix sum over the workgroup; `total` is the sum.
__device__ __forceinline__ int block_excl_scan(int v, int* s_wave, int& total) {
  const int in = wave_incl_scan_i32(v);
  if (lane_id() == kWave - 1) s_wave[threadIdx.x / kWave] = in;
  __syncthreads();
  int before = 0, sum = 0;
#pragma unroll
  for (int w = 0; w < kSelectWaves; ++w) {
    before += w < (int)(threadIdx.x / kWave) ? s_wave[w] : 0;
    sum += s_wave[w];
  }
  __syncthreads();
  total = sum;
  return in - v + before;
}

__global__ __launch_bounds__(kSelectThreads) void kv8_evict_select_kernel(const EvictCall c) {
  __shared__ int s_hist[kBins];
  __shared__ int s_wave[kSelectWaves];
  __shared__ int s_pick[3];
  const int pair = blockIdx.x, tid = threadIdx.x;
  const int b = pair / c.Hkv;
  const int L = min(max(c.lens[b], 0), c.L_max);
  const float* const w_in = c.weights + (size_t)pair * c.stride;
  const int32_t* const p_in = c.positions + (size_t)pair * c.stride;
  float* const w_out = c.weights_out + (size_t)pair * c.stride;
  int32_t* const p_out = c.positions_out + (size_t)pair * c.stride;
  if (L <= c.budget) {
    for (int j = tid; j < L; j += kSelectThreads) {
      w_out[j] = w_in[j];
      p_out[j] = p_in[j];
    }
    if (tid == 0 && c.L_max > c.budget) *evict_ws(c, pair, gridDim.x).moved = 0;
    if (tid == 0 && c.L_max <= c.budget && pair == b * c.Hkv) c.lens_out[b] = L;
    return;
  }
  const EvictWs ws = evict_ws(c, pair, gridDim.x);
  const int64_t since = (int64_t)c.next_position[b] - c.recent;

  // The protected tokens stay, and of the others as many as there is room for; where
  // they alone are too many, as many of them.
  int mine = 0, protects;
  for (int j = tid; j < L; j += kSelectThreads) mine += p_in[j] >= since;
  block_excl_scan(mine, s_wave, protects);
  const bool among = protects >= c.budget;   // the choice is among the protected ones
  int want = among ? c.budget : c.budget - protects;

  // The want-th largest weight of those, by digits of 11, 11 and 10 bits.
  uint32_t found = 0, known = 0;   // its leading bits, and which those are
  int equal = 0;
#pragma unroll
  for (int pass = 0; pass < 3; ++pass) {
    const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, bins = pass == 2 ? kBins / 2 : kBins;
    for (int i = tid; i < kBins; i += kSelectThreads) s_hist[i] = 0;
    __syncthreads();
    for (int j = tid; j < L; j += kSelectThreads) {
      const uint32_t key = ordered_bits(w_in[j]);
      if ((p_in[j] >= since) == among && (key & known) == found) atomicAdd(&s_hist[(key >> shift) & (bins - 1)], 1);
    }
    __syncthreads();
    // two bins a thread, the largest first
    const int hi = kBins - 1 - 2 * tid;
    const int n1 = s_hist[hi], n0 = s_hist[hi - 1];
    int total;
    const int above = block_excl_scan(n1 + n0, s_wave, total);
    if (above < want && above + n1 + n0 >= want) {
      const bool first = above + n1 >= want;
      s_pick[0] = first ? hi : hi - 1;
      s_pick[1] = want - (first ? above : above + n1);
      s_pick[2] = first ? n1 : n0;
    }
    __syncthreads();
    found |= (uint32_t)s_pick[0] << shift;
    known |= (uint32_t)(bins - 1) << shift;
    want = s_pick[1];
    equal = s_pick[2];
    __syncthreads();
  }

  // In order of slots: the first `want` of the equal ones stay.
  int equals = 0, frees = 0, moves = 0;   // so far
  for (int j0 = 0; j0 < L; j0 += kSelectThreads) {
    const int j = j0 + tid;
    const bool in = j < L;
    const float w = in ? w_in[j] : 0.f;
    const int p = in ? p_in[j] : 0;
    const uint32_t key = ordered_bits(w);
    const bool chosen = in && (p >= since) == among;
    bool kept = in && (chosen ? key > found : !among);
    int total;
    if (want == equal) {
      kept |= chosen && key == found;
    } else {
      const bool eq = chosen && key == found;
      const int rank = equals + block_excl_scan(eq, s_wave, total);
      kept |= eq && rank < want;
      equals += total;
    }
    const bool frees_slot = in && !kept && j < c.budget, moves_row = kept && j >= c.budget;
    const int at = block_excl_scan((frees_slot ? 1 : 0) + (moves_row ? 1 << 16 : 0), s_wave, total);
    if (frees_slot) ws.free[frees + (at & 0xffff)] = j;
    if (kept && j < c.budget) {
      ws.src[j] = j;
      w_out[j] = w;
      p_out[j] = p;
    }
    __syncthreads();
    if (moves_row) {
      const int to = ws.free[moves + (at >> 16)];
      ws.src[to] = j;
      w_out[to] = w;
      p_out[to] = p;
    }
    frees += total & 0xffff;
    moves += total >> 16;
  }
  if (tid == 0) *ws.moved = moves;
}

// A wave takes one block of the kept slots, 16 lanes a row, four rows at a time.
__global__ __launch_bounds__(kMoveThreads) void kv8_evict_move_kernel(const EvictCall c, int blocks, int page_shift) {
  const uint32_t job = blockIdx.x * kMoveWaves + __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const uint32_t pairs = (uint32_t)c.B * c.Hkv;
  const uint32_t pair = job / (uint32_t)blocks;
  if (pair >= pairs) return;
  const int block = (int)(job - pair * (uint32_t)blocks);
  const int b = (int)(pair / (uint32_t)c.Hkv), g = (int)(pair - (uint32_t)b * c.Hkv);
  const int lane = lane_id();
  if (block == 0 && g == 0 && lane == 0) c.lens_out[b] = min(min(max(c.lens[b], 0), c.L_max), c.budget);
  const EvictWs ws = evict_ws(c, pair, pairs);
  if (*ws.moved == 0) return;
  const int slot0 = block << kKv8BlockShift, row = lane % ADAPLD_KV8_BLOCK;
  const int src = ws.src[slot0 + row];
  if (!__any(src != slot0 + row)) return;
  const int32_t* const table = c.page_table + (size_t)b * c.max_pages;
  const int mask = (1 << page_shift) - 1;
  const int page = table[slot0 >> page_shift];
  if (page < 0 || page >= c.n_pages) return;
  const size_t to = pool_row(page, g, slot0 & mask, c.Hkv, page_shift);
  const size_t from = pool_row(page_in_pool(table[src >> page_shift], c.n_pages), g, src & mask, c.Hkv, page_shift);
  const int part = lane % kKv8RowLanes, sub = lane / kKv8RowLanes;
#pragma unroll
  for (int n = 0; n < 2; ++n) {
    const int e = c.scales[n][from >> kKv8BlockShift];
    const int most = wave_max_i32(e);
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      const int r = 4 * t + sub;
      const size_t from_r = __shfl(from, r, kWave);
      const int e_r = __shfl(e, r, kWave);
      if (from_r != to + r || e_r != most)
        *reinterpret_cast<uint2*>(c.codes[n] + (to + r) * kKv8RowBytes + part * 8) = kv8_rescale(
            *reinterpret_cast<const uint2*>(c.codes[n] + from_r * kKv8RowBytes + part * 8), e_r, most);
    }
    if (lane == 0) c.scales[n][to >> kKv8BlockShift] = (uint8_t)most;
  }
}

}  // namespace

size_t evict_ws_bytes(int B, int Hkv, int L_max, int budget) {
  if (L_max <= budget) return 0;
  return ((size_t)B * Hkv * (budget + evict_most(L_max, budget) + 1) * sizeof(int32_t) + 15) / 16 * 16;
}

hipError_t launch_kv8_evict(const EvictCall& c, hipStream_t stream) {
  hipLaunchKernelGGL(kv8_evict_select_kernel, dim3((unsigned)c.B * c.Hkv), dim3(kSelectThreads), 0, stream, c);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || c.L_max <= c.budget) return e;
  const int blocks = c.budget >> kKv8BlockShift;
  const int64_t jobs = (int64_t)c.B * c.Hkv * blocks;
  hipLaunchKernelGGL(kv8_evict_move_kernel, dim3((unsigned)((jobs + kMoveWaves - 1) / kMoveWaves)), dim3(kMoveThreads),
                     0, stream, c, blocks, log2_pow2(c.page_size));
  return hipGetLastError();
}

}  // namespace adapld
