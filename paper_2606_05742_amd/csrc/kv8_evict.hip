// Eviction from the paged 8-bit cache by accumulated attention weight.
//
// One workgroup a (sequence, kv head) finds which tokens stay and which of them move
// where, then a wave a block of the kept slots moves the rows: in the same launch where
// few can move, else in a second one over all CUs.  Rows move only from slots >= budget
// to free slots below it, so no row is read that a launch writes, and nothing moves that
// can stay.
//
// The weights are ranked by digits of 11, 11 and 10 bits from the top, a histogram in LDS
// each, until all equal ones stay; a thread holds its slots' weights and positions in
// registers throughout, up to 16384 slots.
//
// Where it stands: 128 kv heads, 2065 tokens to 2048, 12 us: launch and loads 3, a digit
// 1.2, the ranks 2, the moves 3.5, one after the other, half of the CUs busy; 75 tokens to
// 32 of 8 heads 9.  With more slots, 17 of which go, in one launch too: 8209 23, and beyond
// the registers, with the weights read again for each step, 16401 43, 32785 70.  8192 tokens
// at most to 2048: selection 14 and moves 24 (some 91 MB, 3.7 TB/s in the latter; without the
// rows' reads 17, without their writes 18.5, without the scales 19).  One, two or four blocks
// a wave, and a head's blocks on one XCD, made no difference.
#include <type_traits>

#include "adapld_internal.h"
#include "kv8_device.h"

namespace adapld {
namespace {

constexpr int kSelectThreads = 1024;
constexpr int kSelectWaves = kSelectThreads / kWave;
constexpr int kBins = 2048;
constexpr int kCopies = 4;             // of a histogram: weights crowd in few bins
constexpr int kFewMoves = 64;          // moved beside the selection
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

// A float's bits as an unsigned number of the same order, and back.
__device__ __forceinline__ uint32_t ordered_bits(float w) {
  const uint32_t u = __float_as_uint(w);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float weight_of(uint32_t key) { return __uint_as_float(key & 0x80000000u ? key ^ 0x80000000u : ~key); }

// The sum of the first n counts of the waves, on every lane.
__device__ __forceinline__ int sum_of_waves(const int* counts, int n) {
  static_assert(kSelectWaves == 16, "a row of lanes");
  int v = lane_id() % 16 < n ? counts[lane_id() % 16] : 0;
  v += __builtin_amdgcn_mov_dpp(v, 0x128, 0xf, 0xf, false);   // row_ror:8, 4, 2, 1
  v += __builtin_amdgcn_mov_dpp(v, 0x124, 0xf, 0xf, false);
  v += __builtin_amdgcn_mov_dpp(v, 0x122, 0xf, 0xf, false);
  v += __builtin_amdgcn_mov_dpp(v, 0x121, 0xf, 0xf, false);
  return __builtin_amdgcn_readfirstlane(v);
}

// One block of kept slots takes its rows: lane r < 16 (and those 16, 32, 48 behind it)
// gives the slot that row r comes from, the row itself where it stays.  16 lanes a row,
// four rows at a time.  Rows of a smaller scale than the largest are rounded again.
// EAGER: rows that stay are read with the others, not when their scale asks for it.
template <bool EAGER>
__device__ __forceinline__ void move_block(const EvictCall& c, int b, int g, int slot0, int src, int page_shift) {
  const int lane = lane_id(), part = lane % kKv8RowLanes, sub = lane / kKv8RowLanes;
  const int32_t* const table = c.page_table + (size_t)b * c.max_pages;
  const int mask = (1 << page_shift) - 1;
  const int page = table[slot0 >> page_shift], from_page = table[src >> page_shift];
  if (page < 0 || page >= c.n_pages) return;
  const size_t to = pool_row(page, g, slot0 & mask, c.Hkv, page_shift);
  const size_t from = pool_row(page_in_pool(from_page, c.n_pages), g, src & mask, c.Hkv, page_shift);
  const int e[2] = {c.scales[0][from >> kKv8BlockShift], c.scales[1][from >> kKv8BlockShift]};
  uint2 x[2][4];
  size_t from_r[4];
#pragma unroll
  for (int t = 0; t < 4; ++t) {
    from_r[t] = __shfl(from, 4 * t + sub, kWave);
#pragma unroll
    for (int n = 0; n < 2; ++n) {
      x[n][t] = make_uint2(0, 0);
      if (EAGER || from_r[t] != to + 4 * t + sub) x[n][t] = *reinterpret_cast<const uint2*>(c.codes[n] + from_r[t] * kKv8RowBytes + part * 8);
    }
  }
#pragma unroll
  for (int n = 0; n < 2; ++n) {
    const int most = wave_max_i32(e[n]);
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      const int r = 4 * t + sub, e_r = __shfl(e[n], r, kWave);
      const bool comes = from_r[t] != to + r;
      uint2* const at = reinterpret_cast<uint2*>(c.codes[n] + (to + r) * kKv8RowBytes + part * 8);
      if (e_r != most) *at = kv8_rescale(EAGER || comes ? x[n][t] : *at, e_r, most);
      else if (comes) *at = x[n][t];
    }
    if (lane == 0) c.scales[n][to >> kKv8BlockShift] = (uint8_t)most;
  }
}

// A thread holds R slots, 1024 apart; R * 1024 slots at a time where there are more.
// FEW: at most kFewMoves rows move; they move here, and nothing is kept in the
// workspace.
template <int R, bool FEW>
__global__ __launch_bounds__(kSelectThreads) void kv8_evict_select_kernel(const EvictCall c, int page_shift) {
  __shared__ __attribute__((aligned(16))) int s_hist[2][kCopies][kBins];
  __shared__ int s_wave[kSelectWaves], s_protects[kSelectWaves];
  __shared__ int s_count[R][kSelectWaves];
  __shared__ int s_pick[3];
  __shared__ int s_free[FEW ? kFewMoves : 1], s_from[FEW ? kFewMoves : 1];
  const int pair = blockIdx.x, tid = threadIdx.x, lane = lane_id();
  const int wave = __builtin_amdgcn_readfirstlane(tid / kWave);
  const int b = pair / c.Hkv;
  const int L = min(max(c.lens[b], 0), c.L_max);
  const float* const w_in = c.weights + (size_t)pair * c.stride;
  const int32_t* const p_in = c.positions + (size_t)pair * c.stride;
  float* const w_out = c.weights_out + (size_t)pair * c.stride;
  int32_t* const p_out = c.positions_out + (size_t)pair * c.stride;
  const bool first_head = pair == b * c.Hkv;
  if (L <= c.budget) {
    for (int j = tid; j < L; j += kSelectThreads) {
      w_out[j] = w_in[j];
      p_out[j] = p_in[j];
    }
    if (tid == 0) {
      if (!FEW && c.L_max > c.budget) *evict_ws(c, pair, gridDim.x).moved = 0;
      else if (first_head) c.lens_out[b] = L;
    }
    return;
  }
  const int since = (int)max((int64_t)c.next_position[b] - c.recent, (int64_t)INT32_MIN);

  constexpr int kChunk = R * kSelectThreads;
  uint32_t key[R];
  int pos[R];
  const bool resident = L <= kChunk;
  auto load = [&](int j0) {
#pragma unroll
    for (int i = 0; i < R; ++i) {
      const int j = min(j0 + i * kSelectThreads + tid, L - 1);
      key[i] = ordered_bits(w_in[j]);
      pos[i] = p_in[j];
    }
  };
  // Whether any lane of the wave has an i-th slot.
  auto live = [&](int j0, int i) { return j0 + i * kSelectThreads + wave * kWave < L; };
  // f(slot, i) for the thread's slots.
  auto each = [&](bool reload, auto&& f) {
    for (int j0 = 0; j0 < L; j0 += kChunk) {
      if (reload) load(j0);
#pragma unroll
      for (int i = 0; i < R; ++i) {
        if (!live(j0, i)) break;
        const int j = j0 + i * kSelectThreads + tid;
        if (j < L) f(j, i);
      }
    }
  };

  // The protected tokens stay, and of the others as many as there is room for; where
  // they alone are too many, as many of them.  The want-th largest weight of those, by
  // digits of 11, 11 and 10 bits: the first one's histogram is made for both kinds,
  // before it is known which is asked for.
  if (resident) load(0);
  for (int i = tid; i < 2 * kCopies * kBins / 4; i += kSelectThreads) reinterpret_cast<int4*>(s_hist)[i] = make_int4(0, 0, 0, 0);
  __syncthreads();
  bool among = false;   // the choice is among the protected ones
  int want = 0;
  uint32_t found = 0, known = 0;   // its leading bits, and which those are
  int equal = 0;
#pragma unroll
  for (int pass = 0; pass < 3; ++pass) {
    const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0;
    const uint32_t digit = pass == 2 ? kBins / 2 - 1 : kBins - 1;
    int mine = 0;
    each(!resident, [&](int, int i) {
      const bool kept = pos[i] >= since;
      mine += kept;
      if (pass == 0 || (kept == among && (key[i] & known) == found))
        atomicAdd(&s_hist[pass == 0 && kept][tid % kCopies][(key[i] >> shift) & digit], 1);
    });
    if (pass == 0) {
      mine = wave_incl_scan_i32(mine);
      if (lane == kWave - 1) s_protects[wave] = mine;
    }
    __syncthreads();
    if (pass == 0) {
      const int protects = sum_of_waves(s_protects, kSelectWaves);
      among = protects >= c.budget;
      want = among ? c.budget : c.budget - protects;
    }
    // two bins a thread, the largest first; the first kind's are cleared for the next pass
    const int hi = kBins - 1 - 2 * tid;
    int n1 = 0, n0 = 0;
#pragma unroll
    for (int k = 0; k < kCopies; ++k) {
      const int2 n = *reinterpret_cast<const int2*>(&s_hist[pass == 0 && among][k][hi - 1]);
      n0 += n.x;
      n1 += n.y;
      *reinterpret_cast<int2*>(&s_hist[0][k][hi - 1]) = make_int2(0, 0);
    }
    const int in = wave_incl_scan_i32(n1 + n0);
    if (lane == kWave - 1) s_wave[wave] = in;
    __syncthreads();
    const int above = in - n1 - n0 + sum_of_waves(s_wave, wave);
    if (above < want && above + n1 + n0 >= want) {
      const bool first = above + n1 >= want;
      s_pick[0] = first ? hi : hi - 1;
      s_pick[1] = want - (first ? above : above + n1);
      s_pick[2] = first ? n1 : n0;
    }
    __syncthreads();
    found |= (uint32_t)s_pick[0] << shift;
    known |= digit << shift;
    want = s_pick[1];
    equal = s_pick[2];
    if (want == equal) break;   // all of them stay: the other digits do not matter
  }

  // In order of slots: the first `want` of the equal ones stay.  A slot's rank is the
  // number of marked ones before it: of earlier waves' by counts, of its own by ballot.
  const EvictWs ws = FEW ? EvictWs{} : evict_ws(c, pair, gridDim.x);
  // Exclusive prefix sums of s_count in order; two counts of 16 bits an entry.
  auto scan_counts = [&](int& total) {
    __syncthreads();
    constexpr int kEach = (R * kSelectWaves + kWave - 1) / kWave;
    int* const flat = &s_count[0][0];
    if (wave == 0) {
      int v[kEach], sum = 0;
#pragma unroll
      for (int k = 0; k < kEach; ++k) {
        const int at = lane * kEach + k;
        v[k] = at < R * kSelectWaves ? flat[at] : 0;
        sum += v[k];
      }
      int before = wave_incl_scan_i32(sum);
      if (lane == kWave - 1) s_pick[0] = before;
      before -= sum;
#pragma unroll
      for (int k = 0; k < kEach; ++k) {
        if (lane * kEach + k < R * kSelectWaves) flat[lane * kEach + k] = before;
        before += v[k];
      }
    }
    __syncthreads();
    total = s_pick[0];
  };
  int equals = 0, frees = 0, moves = 0;   // so far
  for (int j0 = 0; j0 < L; j0 += kChunk) {
    if (!resident) load(j0);
    uint32_t kept = 0;   // bit i: the thread's i-th slot stays
    if (want == equal) {
#pragma unroll
      for (int i = 0; i < R; ++i) {
        if (!live(j0, i)) break;
        const bool chosen = (pos[i] >= since) == among;
        if (chosen ? key[i] >= found : !among) kept |= 1u << i;
      }
    } else {
      uint32_t ranks[R];
#pragma unroll
      for (int i = 0; i < R; ++i) {
        ranks[i] = ~0u;
        if (!live(j0, i)) {
          if (lane == 0) s_count[i][wave] = 0;
          continue;
        }
        const int j = j0 + i * kSelectThreads + tid;
        const bool eq = j < L && (pos[i] >= since) == among && key[i] == found;
        const uint64_t m = __ballot(eq);
        ranks[i] = eq ? (uint32_t)__popcll(m & lanes_below()) : ~0u;
        if (lane == 0) s_count[i][wave] = __popcll(m);
      }
      int total;
      scan_counts(total);
#pragma unroll
      for (int i = 0; i < R; ++i) {
        if (!live(j0, i)) break;
        const bool chosen = (pos[i] >= since) == among;
        bool stays = chosen ? key[i] > found : !among;
        if (ranks[i] != ~0u) stays = equals + s_count[i][wave] + (int)ranks[i] < want;
        if (stays) kept |= 1u << i;
      }
      equals += total;
      __syncthreads();
    }
    // the slots that become free below the budget, and the rows that move from behind it
    int at[R];
#pragma unroll
    for (int i = 0; i < R; ++i) {
      at[i] = 0;
      if (!live(j0, i)) {
        if (lane == 0) s_count[i][wave] = 0;
        continue;
      }
      const int j = j0 + i * kSelectThreads + tid;
      const bool in = j < L, stays = kept >> i & 1;
      const uint64_t f = __ballot(in && !stays && j < c.budget), m = __ballot(in && stays && j >= c.budget);
      at[i] = (j < c.budget ? __popcll(f & lanes_below()) : __popcll(m & lanes_below()));
      if (lane == 0) s_count[i][wave] = __popcll(f) | __popcll(m) << 16;
    }
    int total;
    scan_counts(total);
#pragma unroll
    for (int i = 0; i < R; ++i) {
      if (!live(j0, i)) break;
      const int j = j0 + i * kSelectThreads + tid;
      if (j >= L) continue;
      const int before = s_count[i][wave];
      if (j < c.budget) {
        if (kept >> i & 1) {
          if (!FEW) ws.src[j] = j;
          w_out[j] = weight_of(key[i]);
          p_out[j] = pos[i];
        } else {
          const int k = frees + (before & 0xffff) + at[i];
          if (FEW) s_free[k] = j;
          else ws.free[k] = j;
        }
      }
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < R; ++i) {
      if (!live(j0, i)) break;
      const int j = j0 + i * kSelectThreads + tid;
      if (j >= L || j < c.budget || !(kept >> i & 1)) continue;
      const int k = moves + (s_count[i][wave] >> 16) + at[i];
      const int to = FEW ? s_free[k] : ws.free[k];
      if (FEW) s_from[k] = j;
      else ws.src[to] = j;
      w_out[to] = weight_of(key[i]);
      p_out[to] = pos[i];
    }
    frees += total & 0xffff;
    moves += total >> 16;
    __syncthreads();
  }
  if constexpr (!FEW) {
    if (tid == 0) *ws.moved = moves;
  } else {
    if (tid == 0 && first_head) c.lens_out[b] = c.budget;
    const int g = pair - b * c.Hkv, row = lane % ADAPLD_KV8_BLOCK;
    for (int k = wave; k < moves; k += kSelectWaves) {
      const int block = s_free[k] >> kKv8BlockShift;
      if (k > 0 && s_free[k - 1] >> kKv8BlockShift == block) continue;   // another wave's block
      int src = (block << kKv8BlockShift) + row;
      for (int m = k; m < moves && s_free[m] >> kKv8BlockShift == block; ++m)
        if (s_free[m] % ADAPLD_KV8_BLOCK == row) src = s_from[m];
      move_block<true>(c, b, g, block << kKv8BlockShift, src, page_shift);
    }
  }
}

// A wave takes one block of the kept slots.
__global__ __launch_bounds__(kMoveThreads) void kv8_evict_move_kernel(const EvictCall c, int blocks, int page_shift) {
  const uint32_t job = blockIdx.x * kMoveWaves + __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const uint32_t pairs = (uint32_t)c.B * c.Hkv;
  const uint32_t pair = job / (uint32_t)blocks;
  if (pair >= pairs) return;
  const int block = (int)(job - pair * (uint32_t)blocks);
  const int b = (int)(pair / (uint32_t)c.Hkv), g = (int)(pair - (uint32_t)b * c.Hkv);
  if (block == 0 && g == 0 && lane_id() == 0) c.lens_out[b] = min(min(max(c.lens[b], 0), c.L_max), c.budget);
  const EvictWs ws = evict_ws(c, pair, pairs);
  const int slot0 = block << kKv8BlockShift, row = lane_id() % ADAPLD_KV8_BLOCK;
  const int moved = *ws.moved, src = ws.src[slot0 + row];
  // without moves src holds anything
  if (moved == 0 || !__any(src != slot0 + row)) return;
  move_block<false>(c, b, g, slot0, src, page_shift);
}

}  // namespace

size_t evict_ws_bytes(int B, int Hkv, int L_max, int budget) {
  if (L_max <= budget) return 0;
  return ((size_t)B * Hkv * (budget + evict_most(L_max, budget) + 1) * sizeof(int32_t) + 15) / 16 * 16;
}

hipError_t launch_kv8_evict(const EvictCall& c, hipStream_t stream) {
  const int page_shift = log2_pow2(c.page_size);
  // Where few rows can move, a launch less.  (lens_out may be lens: the heads of a
  // sequence all read it, so then only a second launch can write it.)
  const bool few = c.L_max > c.budget && evict_most(c.L_max, c.budget) <= kFewMoves && c.lens_out != c.lens;
  auto select = [&](auto r) {
    constexpr int R = decltype(r)::value;
    const dim3 grid((unsigned)c.B * c.Hkv);
    if (few) hipLaunchKernelGGL((kv8_evict_select_kernel<R, true>), grid, dim3(kSelectThreads), 0, stream, c, page_shift);
    else hipLaunchKernelGGL((kv8_evict_select_kernel<R, false>), grid, dim3(kSelectThreads), 0, stream, c, page_shift);
  };
  if (c.L_max <= 4 * kSelectThreads) select(std::integral_constant<int, 4>{});
  else if (c.L_max <= 8 * kSelectThreads) select(std::integral_constant<int, 8>{});
  else select(std::integral_constant<int, 16>{});
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || c.L_max <= c.budget || few) return e;
  const int blocks = c.budget >> kKv8BlockShift;
  const int64_t jobs = (int64_t)c.B * c.Hkv * blocks;
  hipLaunchKernelGGL(kv8_evict_move_kernel, dim3((unsigned)((jobs + kMoveWaves - 1) / kMoveWaves)), dim3(kMoveThreads),
                     0, stream, c, blocks, page_shift);
  return hipGetLastError();
}

}  // namespace adapld
