// The attention weight that each cached token gets from new rows, over the paged 8-bit
// cache: a pass over its keys alone, with the log-sum-exp that the attention left.
//
// For one sequence and kv head the n * G new query rows are stacked as row = i * G +
// head.  The codes become bf16 operands in registers (exact), the logits fp32 sums of
// matrix products, and a weight 2^(s scale log2(e) - lse log2(e)).  One wave (or one
// workgroup's waves in a fixed order) sums up all that a key gets: no atomics, and the order
// of a sum is fixed by the call's sizes.  Those choose one of the kernels below, which take a
// key's rows in different orders, so L_max, B, N and the heads can change a sum's last bits;
// what the other sequences of a batch hold does not.
//
// Where it stands: single tokens, 32 x 8192 keys of 8 heads, read 286 MB in 54 us, 5.3
// TB/s.  196 rows (28 new ones, 28 heads over 4), 16 x 8192 keys 38 us, 0.69 PFLOP/s; 1792
// rows, 4 x 4096 keys 40 us, 0.75 PFLOP/s, the exponentials beside the products; 4 x 6007
// at most, two thirds of it tokens, 63 us, in part-filled rounds of workgroups over the
// CUs.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "adapld_internal.h"
#include "kv8_device.h"

namespace adapld {
namespace {

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef float f32x16_t __attribute__((ext_vector_type(16)));
typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));

constexpr int kD = ADAPLD_HEAD_DIM;
constexpr float kLog2e = 1.4426950408889634f;

struct WeightsArgs {
  AttnWeightsCall c;
  int G, page_shift, nsplit, chunk;   // keys of a workgroup
  float sl2;
};

// Stacked row r of at most N * G: its new row i, the place of its query among the
// sequence's, and its log-sum-exp in units of log2, infinite where the row gives nothing
// (but for what the lengths say, which these loads do not wait for).
struct RowAt {
  int i, place;
  float lse2;
};
__device__ __forceinline__ RowAt row_at(const WeightsArgs& a, int b, int g, int r) {
  const AttnWeightsCall& c = a.c;
  const int most = c.N * a.G, rr = min(r, most - 1), i = rr / a.G, h = g * a.G + (rr - i * a.G);
  const int u = c.rows ? c.rows[(size_t)b * c.N + i] : i;
  const bool in = u >= 0 && u < c.T_max;
  const float lse = c.lse[((size_t)b * c.Hq + h) * c.T_max + (in ? u : 0)];
  return {i, (in ? u : 0) * c.Hq + h, in && r < most && lse > -INFINITY ? lse * kLog2e : INFINITY};
}

__device__ __forceinline__ bf16x8_t operand(uint32_t lo, uint32_t hi, float X) {
  return __builtin_bit_cast(bf16x8_t, kv8_values(make_uint2(lo, hi), X));
}
__device__ __forceinline__ u32x4_t load16(const uint8_t* p) { return *reinterpret_cast<const u32x4_t*>(p); }
__device__ __forceinline__ float add_lane_xor32(float v) {
  const auto t = __builtin_amdgcn_permlane32_swap(__float_as_int(v), __float_as_int(v), false, false);
  return __int_as_float(t[0]) + __int_as_float(t[1]);
}
__device__ __forceinline__ float add_lane_xor16(float v) {
  const auto t = __builtin_amdgcn_permlane16_swap(__float_as_int(v), __float_as_int(v), false, false);
  return __int_as_float(t[0]) + __int_as_float(t[1]);
}

// ------------------------------------------------------------- up to 64 rows
//
// One pass over the keys: a wave takes steps of 32, alone, the queries stay in its
// registers.  On v_mfma_f32_16x16x32_bf16 with the rows as A and 16 keys as B a lane
// has 4 rows of one key, so a key's sum is its lane's own but for two exchanges.
// Codes of three steps are in flight.
constexpr int kNarrowThreads = 256;
constexpr int kNarrowWaves = kNarrowThreads / kWave;
constexpr int kStep = 32;
constexpr int kMaxSteps = 16;   // of a wave
static_assert(kMaxSteps <= kWave, "a lane for each step's page ids");

template <int RB>
__global__ __launch_bounds__(kNarrowThreads, RB == 1 ? 4 : RB == 2 ? 3 : 2) void kv8_weights_narrow_kernel(const WeightsArgs a) {
  const AttnWeightsCall& c = a.c;
  const int bg = blockIdx.x / a.nsplit, split = blockIdx.x - bg * a.nsplit;
  const int b = bg / c.Hkv, g = bg - b * c.Hkv;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int lane = lane_id(), col = lane & 15, quad = lane >> 4;
  const int c0 = split * a.chunk;
  // Lane j holds the page ids of the two halves of the wave's step j (kMaxSteps at most).
  const int32_t* const table = c.page_table + (size_t)b * c.max_pages;
  int ids[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int pos = c0 + (wave + lane * kNarrowWaves) * kStep + 16 * i;
    ids[i] = page_in_pool(table[min(pos >> a.page_shift, c.max_pages - 1)], c.n_pages);
  }
  const RowAt mine = row_at(a, b, g, lane);   // lane r looks row r up for all
  const int old = min(max(c.lens_old[b], 0), c.L_max);
  const int n = min(max(min(max(c.lens_new[b], 0), c.L_max) - old, 0), c.N);
  const int c1 = min(c0 + a.chunk, old + n);
  if (c0 + wave * kStep >= c1) return;
  const int steps = (c1 - c0 + kStep - 1) / kStep;
  const float* const w_in = c.weights + (size_t)bg * c.stride;
  float* const w_out = c.weights_out + (size_t)bg * c.stride;

  struct Raw {
    u32x4_t k[2][2];
    uint32_t e[2];
    float w;   // of key k0 + lane, lanes 0..31
  };
  // Step s; behind the wave's last step a line of that one, so that the number of loads in
  // flight does not depend on a branch.
  const int last = wave + (steps - 1 - wave) / kNarrowWaves * kNarrowWaves;
  auto load = [&](int s, Raw& r) {
    const bool used = s <= last;
    s = min(s, last);
    const int k0 = c0 + s * kStep, at = (s - wave) / kNarrowWaves, part = used ? quad : 0;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      // Keys behind the last read the last one again; their sums are not stored.
      int pos = k0 + 16 * i;
      uint32_t key = used ? col : 0;
      int page = __builtin_amdgcn_readlane(ids[i], at);
      if (pos + 16 > c1) {
        if (pos >= c1) {
          page = __builtin_amdgcn_readlane(ids[0], at);
          pos = k0;
        }
        key = min((int)key, c1 - 1 - pos);
      }
      const size_t row = pool_row(page, g, pos & ((1 << a.page_shift) - 1), c.Hkv, a.page_shift);
      const uint8_t* const p = c.k_codes + row * kKv8RowBytes;
      r.k[i][0] = load16(p + key * kKv8RowBytes + part * 16);
      r.k[i][1] = load16(p + key * kKv8RowBytes + part * 16 + 64);
      r.e[i] = c.k_scales[row >> kKv8BlockShift];
    }
    r.w = w_in[min(k0 + (lane & 31), max(old - 1, 0))];
  };
  Raw r[3];
  load(wave, r[0]);
  load(wave + kNarrowWaves, r[1]);
  load(wave + 2 * kNarrowWaves, r[2]);

  const float my_lse2 = lane < n * a.G ? mine.lse2 : INFINITY;
  const int my_place = my_lse2 < INFINITY ? mine.place : -1;
  const bool none = !__any(my_lse2 < INFINITY);   // then nothing is known of the keys
  bf16x8_t q[RB][4];
  float lse2[RB][4];
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    const int place = __shfl(my_place, 16 * rb + col, kWave);
    const uint4* const p = reinterpret_cast<const uint4*>(c.q + ((size_t)b * c.T_max * c.Hq + max(place, 0)) * kD);
#pragma unroll
    for (int j = 0; j < 4; ++j)   // a row that gives nothing must not bring a NaN
      q[rb][j] = __builtin_bit_cast(bf16x8_t, place >= 0 ? p[8 * (j >> 1) + 2 * quad + (j & 1)] : make_uint4(0, 0, 0, 0));
#pragma unroll
    for (int t = 0; t < 4; ++t) lse2[rb][t] = __shfl(my_lse2, 16 * rb + 4 * quad + t, kWave);
  }

  auto step = [&](int s, Raw& x) {
    const int k0 = c0 + s * kStep;
    const bool plain = k0 + kStep <= old;
    float sum[2];
    const float w = x.w;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const float X = kv8_scale((int)x.e[i]);
      bf16x8_t k[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) k[j] = operand(x.k[i][j >> 1][2 * (j & 1)], x.k[i][j >> 1][2 * (j & 1) + 1], X);
      f32x4_t z[RB];
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) {
        z[rb] = f32x4_t{};
#pragma unroll
        for (int j = 0; j < 4; ++j) z[rb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(q[rb][j], k[j], z[rb], 0, 0, 0);
      }
      float p[4] = {};
#pragma unroll
      for (int rb = 0; rb < RB; ++rb)
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          float e = __builtin_amdgcn_exp2f(fmaf(z[rb][t], a.sl2, -lse2[rb][t]));
          // A new row sees no later one, and one that gives nothing none of the new ones: where
          // no other row sees them they may be NaN.  All rows see the older ones.
          if (!plain) {
            const int last_seen = old + __shfl(mine.i, 16 * rb + 4 * quad + t, kWave);   // by all lanes
            e = lse2[rb][t] < INFINITY && k0 + 16 * i + col <= last_seen ? e : 0.f;
          }
          p[t] += e;
        }
      sum[i] = (p[0] + p[1]) + (p[2] + p[3]);
    }
    load(s + 3 * kNarrowWaves, x);
    // lanes 0..15 and 16..31 take the sums of either half
    const float v0 = add_lane_xor32(add_lane_xor16(sum[0])), v1 = add_lane_xor32(add_lane_xor16(sum[1]));
    const float v = none ? 0.f : quad & 1 ? v1 : v0;
    const int key = k0 + lane;
    if (lane < kStep && key < c1) {
      w_out[key] = key < old ? w + v : v;
      if (key >= old) c.positions[(size_t)bg * c.stride + key] = c.first_position[b] + (key - old);
    }
  };
  int s = wave;
  for (; s + 2 * kNarrowWaves < steps; s += 3 * kNarrowWaves) {
    step(s, r[0]);
    step(s + kNarrowWaves, r[1]);
    step(s + 2 * kNarrowWaves, r[2]);
  }
  if (s < steps) step(s, r[0]);
  if (s + kNarrowWaves < steps) step(s + kNarrowWaves, r[1]);
}

// ---------------------------------------------------------- more than 64 rows
//
// A wave keeps 64 keys as A operands in registers and the rows pass by, 32 a block on
// v_mfma_f32_32x32x16_bf16: a lane then has one row, so one log-sum-exp, and 32 sums
// of keys that stay its own until the end.  Of a workgroup's 8 waves 8 / KG share the
// keys, each with every (8 / KG)-th block of rows.  A round is a block for each of
// them; rounds come straight to a ring of four in LDS, two ahead, and the exponentials
// of one round run beside the products of the next.
constexpr int kWideKeys = 64;            // of a wave
constexpr int kRowBytes = kD * 2;
constexpr int kStages = 4;               // rounds in the ring
constexpr int kMaxRows = 2048;           // rows whose places and log-sum-exps LDS holds at a time

// Physical 16-byte chunk of logical chunk ch in row r: lanes that read one chunk of 16
// consecutive rows hit every bank once.
__device__ __forceinline__ int swizzled(int r, int ch) { return r * kRowBytes + ((ch ^ (r & 15)) << 4); }

// Four weights of 64 keys and 32 rows, value n4 of 8: to the sums of the lane's keys; rows
// see the first `sees` + 1 keys, or with `plain` all.
template <class PLAIN>
__device__ __forceinline__ void add4(const WeightsArgs& a, float (&sum)[2][16], const f32x16_t (&z)[2], int n4, float lse2,
                                     int sees, PLAIN) {
  const int m = n4 / 4;
#pragma unroll
  for (int t = 4 * (n4 % 4); t < 4 * (n4 % 4) + 4; ++t) {
    const float w = __builtin_amdgcn_exp2f(fmaf(z[m][t], a.sl2, -lse2));
    if constexpr (PLAIN::value) sum[m][t] += w;
    else sum[m][t] += 32 * m + 8 * (t >> 2) + (t & 3) <= sees ? w : 0.f;
  }
}

// Sums over the 32 lanes of a half: out[key] of the 64 keys.  Values 16 lanes apart and 8
// apart are added in pairs, each half of the lanes keeping one.
__device__ __forceinline__ void sums_of_keys(const float (&sum)[2][16], float* out) {
  const int lane = lane_id(), half = lane >> 5;
#pragma unroll
  for (int m = 0; m < 2; ++m)
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      float h[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {   // values t + 4 i and t + 4 i + 8, the latter where bit 4 of the lane is set
        const auto w = __builtin_amdgcn_permlane16_swap(__float_as_int(sum[m][t + 4 * i]), __float_as_int(sum[m][t + 4 * i + 8]), false, false);
        h[i] = __int_as_float(w[0]) + __int_as_float(w[1]);
      }
      const bool up = lane & 8;       // h[1] where bit 3 is set
      float v = (up ? h[1] : h[0]) + dpp_f32<0x128>(up ? h[0] : h[1]);   // row_ror:8
      v += dpp_f32<0x141>(v);             // row_half_mirror
      v += dpp_f32<0xb1>(v);              // quad_perm 1 0 3 2
      v += dpp_f32<0x4e>(v);              // quad_perm 2 3 0 1
      const int value = t + 4 * ((lane >> 3) & 1) + 8 * ((lane >> 4) & 1);
      if ((lane & 7) == 0) out[32 * m + 8 * (value >> 2) + (value & 3) + 4 * half] = v;
    }
}

template <int KG, int kParts>
__global__ __launch_bounds__(KG * kParts * kWave, 2) void kv8_weights_wide_kernel(const WeightsArgs a) {
  constexpr int kWideThreads = KG * kParts * kWave;
  constexpr int kRows = 32 * kParts;               // rows of a round
  constexpr int kLoads = 8 / KG;                   // of a wave for a round
  __shared__ __attribute__((aligned(1024))) uint8_t s_rows[kStages][kRows * kRowBytes];
  __shared__ int s_at[kMaxRows];       // query of a row, in rows of q behind the sequence's first; -1: it gives nothing
  __shared__ float s_lse2[kMaxRows];
  // The last key that a row sees; -1 where it gives nothing: new keys that no other row sees
  // may be NaN.
  __shared__ int s_last[kMaxRows];
  __shared__ int s_any;
  const AttnWeightsCall& c = a.c;
  const int bg = blockIdx.x / a.nsplit, split = blockIdx.x - bg * a.nsplit;
  const int b = bg / c.Hkv, g = bg - b * c.Hkv;
  const int tid = threadIdx.x;
  const int wave = __builtin_amdgcn_readfirstlane(tid / kWave);
  const int kg = wave % KG, part = wave / KG;
  const int lane = lane_id(), col = lane & 31, half = lane >> 5;
  const int old = min(max(c.lens_old[b], 0), c.L_max);
  const int n = min(max(min(max(c.lens_new[b], 0), c.L_max) - old, 0), c.N);
  const int end = old + n, c0 = split * (KG * kWideKeys);
  if (c0 >= end) return;
  const int k0 = c0 + kg * kWideKeys;
  const int rows = n * a.G;

  // Keys: lane (half, col) the dimensions [64 * half, +64) of keys col and 32 + col;
  // keys behind the last read the last one again, their sums are not stored.
  u32x4_t codes[2][4];
  uint32_t exponent[2];
#pragma unroll
  for (int m = 0; m < 2; ++m) {
    const int j = min(k0 + 32 * m + col, end - 1);
    const int page = page_in_pool(c.page_table[(size_t)b * c.max_pages + (j >> a.page_shift)], c.n_pages);
    const size_t row = pool_row(page, g, j & ((1 << a.page_shift) - 1), c.Hkv, a.page_shift);
    const u32x4_t* p = reinterpret_cast<const u32x4_t*>(c.k_codes + row * kKv8RowBytes + 64 * half);
#pragma unroll
    for (int i = 0; i < 4; ++i) codes[m][i] = p[i];
    exponent[m] = c.k_scales[row >> kKv8BlockShift];
  }

  float sum[2][16] = {};
  bf16x8_t kf[2][8];
  const uint16_t* const q0 = c.q + (size_t)b * c.T_max * c.Hq * kD;
  for (int first = 0; first < rows; first += kMaxRows) {
    const int some = min(rows - first, kMaxRows), rounds = (some + kRows - 1) / kRows;
    if (tid == 0) s_any = -1;
    __syncthreads();
    // all in flight together
    RowAt x[kMaxRows / kWideThreads];
#pragma unroll
    for (int i = 0; i < kMaxRows / kWideThreads; ++i) x[i] = row_at(a, b, g, first + min(tid + i * kWideThreads, some - 1));
#pragma unroll
    for (int i = 0; i < kMaxRows / kWideThreads; ++i) {
      const int r = tid + i * kWideThreads;
      if (r < rounds * kRows) {
        const bool gives = first + r < rows && x[i].lse2 < INFINITY;
        s_at[r] = gives ? x[i].place : -1;
        s_lse2[r] = gives ? x[i].lse2 : INFINITY;
        s_last[r] = gives ? old + x[i].i : -1;
        if (gives) s_any = x[i].place;
      }
    }
    __syncthreads();
    // A row that gives nothing takes the place of one that does, with an infinite log-sum-
    // exp: what its own place in q holds may be no number.
    const int any = s_any;
    // A wave brings kLoads KiB of a round, four rows a load; behind the last round that
    // one again, so that the number of loads in flight is the same in every round.
    // Places are read from LDS a round before they are used.
    const int r4 = wave * kLoads * 4;
    int at[kLoads];
    auto places = [&](int round) {
#pragma unroll
      for (int i = 0; i < kLoads; ++i) at[i] = s_at[min(round, rounds - 1) * kRows + r4 + 4 * i + lane / 16];
    };
    auto load = [&](int round) {
      const uint32_t to = lds_addr(s_rows[round % kStages]) + r4 * kRowBytes;
#pragma unroll
      for (int i = 0; i < kLoads; ++i)
        dma16(q0 + (size_t)(at[i] < 0 ? any : at[i]) * kD + ((lane ^ (r4 + 4 * i + lane / 16)) & 15) * 8,
              __builtin_amdgcn_readfirstlane(to + 4 * i * kRowBytes));
    };
#pragma unroll
    for (int i = 0; i + 1 < kStages; ++i) {
      places(i);
      if (any >= 0) load(i);
    }
    places(kStages - 1);
    if (first == 0) {
#pragma unroll
      for (int m = 0; m < 2; ++m)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float X = kv8_scale((int)exponent[m]);
          kf[m][2 * i] = operand(codes[m][i][0], codes[m][i][1], X);
          kf[m][2 * i + 1] = operand(codes[m][i][2], codes[m][i][3], X);
        }
    }
    if (any < 0) continue;
    // Eight chunks of a round: two products and four exponentials of the round before,
    // kept together by scheduling barriers (left alone, the compiler sets the products
    // behind each other, every one behind its operand's way through LDS).
    auto operand_of = [&](int round, int d) {
      return *reinterpret_cast<const bf16x8_t*>(s_rows[round % kStages] + 32 * part * kRowBytes + swizzled(col, 8 * half + d));
    };
    // With NEXT the products of the next round, with ADD the exponentials of this one.
    auto round_of = [&](int i, f32x16_t (&z)[2], f32x16_t (&z_next)[2], auto plain, auto NEXT, auto ADD) {
      constexpr bool kNext = decltype(NEXT)::value, kAdd = decltype(ADD)::value;
      bf16x8_t q[8];
      if constexpr (kNext) {
#pragma unroll
        for (int d = 0; d < 3; ++d) q[d] = operand_of(i + 1, d);
        z_next[0] = z_next[1] = f32x16_t{};
      }
      const int r = i * kRows + 32 * part + col;
      float lse2 = 0.f;
      int sees = 0;
      if constexpr (kAdd) {
        lse2 = s_lse2[r];
        // the last key that the row sees, counted from the lane's first
        if constexpr (!decltype(plain)::value) sees = s_last[r] - k0 - 4 * half;
      }
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int d = 0; d < 8; ++d) {
        if constexpr (kNext) {
          if (d + 3 < 8) q[d + 3] = operand_of(i + 1, d + 3);
#pragma unroll
          for (int m = 0; m < 2; ++m) z_next[m] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[m][d], q[d], z_next[m], 0, 0, 0);
        }
        if constexpr (kAdd) add4(a, sum, z, d, lse2, sees, plain);
        __builtin_amdgcn_sched_barrier(0);
      }
    };
    auto run = [&](auto plain) {
      using Yes = std::true_type;
      using No = std::false_type;
      f32x16_t za[2], zb[2];
      waitcnt_vm<(kStages - 2) * kLoads>();
      __syncthreads();
      round_of(-1, zb, za, plain, Yes{}, No{});
      waitcnt_vm<(kStages - 3) * kLoads>();
      __syncthreads();
      // Round i + 1, whose products are formed, has landed; round i + kStages - 1 takes the
      // place of round i - 1.
      auto body = [&](int i, f32x16_t (&z)[2], f32x16_t (&z_next)[2]) {
        load(i + kStages - 1);
        places(i + kStages);
        round_of(i, z, z_next, plain, Yes{}, Yes{});
        waitcnt_vm<(kStages - 3) * kLoads>();
        __syncthreads();
      };
      int i = 0;
      for (; i + 2 < rounds; i += 2) {
        body(i, za, zb);
        body(i + 1, zb, za);
      }
      if (i + 1 < rounds) {
        body(i, za, zb);
        round_of(i + 1, zb, za, plain, No{}, Yes{});
      } else {
        round_of(i, za, zb, plain, No{}, Yes{});
      }
    };
    if (k0 + kWideKeys <= old + 1) run(std::true_type{});   // every row sees all the wave's keys
    else run(std::false_type{});
    waitcnt_vm<0>();
  }
  float* const s_sum = reinterpret_cast<float*>(s_rows);   // [waves][64 keys]
  __syncthreads();
  sums_of_keys(sum, s_sum + wave * kWideKeys);
  __syncthreads();
  const int key = c0 + tid;
  if (tid < KG * kWideKeys && key < end) {
    float v = s_sum[tid];
#pragma unroll
    for (int p = 1; p < kParts; ++p) v += s_sum[p * KG * kWideKeys + tid];
    const size_t at = (size_t)bg * c.stride + key;
    c.weights_out[at] = key < old ? c.weights[at] + v : v;
    if (key >= old) c.positions[at] = c.first_position[b] + (key - old);
  }
}

// ----------------------------------------------------- 65 to 256 rows, many keys
//
// So few rows fit LDS together with the codes of the keys to come, so a workgroup brings
// them once and its waves take blocks of 64 keys, alone, without a barrier: as above a
// block is A operands in registers and the rows pass by, 32 at a time, the exponentials
// of 32 beside the products of the next.  The codes of a wave's next block come straight
// from memory to LDS meanwhile.
constexpr int kMidThreads = 512;
constexpr int kMidWaves = kMidThreads / kWave;
constexpr int kMidRows = 256;
constexpr int kMidBlocks = 16;   // of a workgroup, at most

__global__ __launch_bounds__(kMidThreads, 2) void kv8_weights_mid_kernel(const WeightsArgs a) {
  __shared__ __attribute__((aligned(1024))) uint8_t s_rows[kMidRows * kRowBytes];
  __shared__ __attribute__((aligned(1024))) uint8_t s_codes[kMidWaves][kWideKeys * kKv8RowBytes];
  __shared__ int s_at[kMidRows];       // as in the wide kernel
  __shared__ float s_lse2[kMidRows];
  __shared__ int s_last[kMidRows];
  __shared__ float s_sum[kMidWaves][kWideKeys];
  __shared__ int s_any;
  const AttnWeightsCall& c = a.c;
  const int bg = blockIdx.x / a.nsplit, split = blockIdx.x - bg * a.nsplit;
  const int b = bg / c.Hkv, g = bg - b * c.Hkv;
  const int tid = threadIdx.x;
  const int wave = __builtin_amdgcn_readfirstlane(tid / kWave);
  const int lane = lane_id(), col = lane & 31, half = lane >> 5;
  const RowAt mine = row_at(a, b, g, tid % kMidRows);
  const int old = min(max(c.lens_old[b], 0), c.L_max);
  const int n = min(max(min(max(c.lens_new[b], 0), c.L_max) - old, 0), c.N);
  const int end = old + n, chunk0 = split * a.chunk, c1 = min(chunk0 + a.chunk, end);
  if (chunk0 >= end) return;
  const int rows = n * a.G, blocks = (rows + 31) / 32;
  const float* const w_in = c.weights + (size_t)bg * c.stride;
  float* const w_out = c.weights_out + (size_t)bg * c.stride;

  // Of the wave's block at k0: lane j the page of key j, the codes to LDS (chunk p of key
  // j lies at p ^ (j & 7)), the scales of the lane's two keys, the older weight of key
  // `lane`.  Keys behind the last read the last one again; their sums are not stored.
  const int32_t* const table = c.page_table + (size_t)b * c.max_pages;
  auto pages_of = [&](int k0) { return page_in_pool(table[min(k0 + lane, end - 1) >> a.page_shift], c.n_pages); };
  uint32_t exponent[2];
  float w;
  auto load_keys = [&](int k0, int pages) {
    auto row_of = [&](int key) {
      return pool_row(__shfl(pages, key, kWave), g, min(k0 + key, end - 1) & ((1 << a.page_shift) - 1), c.Hkv, a.page_shift);
    };
    const uint32_t to = lds_addr(s_codes[wave]);
#pragma unroll
    for (int i = 0; i < 8; ++i)
      dma16(c.k_codes + row_of(8 * i + lane / 8) * kKv8RowBytes + ((lane ^ (lane / 8)) & 7) * 16,
            __builtin_amdgcn_readfirstlane(to + i * 1024));
#pragma unroll
    for (int m = 0; m < 2; ++m) exponent[m] = c.k_scales[row_of(32 * m + col) >> kKv8BlockShift];
    w = w_in[min(k0 + lane, max(old - 1, 0))];
  };
  int k0 = chunk0 + wave * kWideKeys;
  constexpr int kNext = kMidWaves * kWideKeys;
  int pages = pages_of(k0);
  load_keys(k0, pages);
  pages = pages_of(k0 + kNext);

  if (tid == 0) s_any = -1;
  __syncthreads();
  if (tid < blocks * 32) {
    const bool gives = tid < rows && mine.lse2 < INFINITY;
    s_at[tid] = gives ? mine.place : -1;
    s_lse2[tid] = gives ? mine.lse2 : INFINITY;
    s_last[tid] = gives ? old + mine.i : -1;
    if (gives) s_any = mine.place;
  }
  __syncthreads();
  const int any = s_any;
  if (any >= 0) {
    const uint16_t* const q0 = c.q + (size_t)b * c.T_max * c.Hq * kD;
    for (int i = 0; i < blocks; ++i) {
      const int r4 = 32 * i + 4 * wave, row = r4 + lane / 16, at = s_at[row];
      dma16(q0 + (size_t)(at < 0 ? any : at) * kD + ((lane ^ row) & 15) * 8,
            __builtin_amdgcn_readfirstlane(lds_addr(s_rows) + r4 * kRowBytes));
    }
  }
  waitcnt_vm<0>();
  __syncthreads();

  for (; k0 < c1; k0 += kNext) {
    waitcnt_vm<0>();
    asm volatile("" ::: "memory");   // the codes have landed
    bf16x8_t kf[2][8];
#pragma unroll
    for (int m = 0; m < 2; ++m) {
      const float X = kv8_scale((int)exponent[m]);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const u32x4_t x = *reinterpret_cast<const u32x4_t*>(s_codes[wave] + (32 * m + col) * kKv8RowBytes +
                                                            (((4 * half + i) ^ col) & 7) * 16);
        kf[m][2 * i] = operand(x[0], x[1], X);
        kf[m][2 * i + 1] = operand(x[2], x[3], X);
      }
    }
    const float before = w;
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // and are read
    if (k0 + kNext < c1) {
      load_keys(k0 + kNext, pages);
      pages = pages_of(k0 + 2 * kNext);
    }
    float sum[2][16] = {};
    // As in the wide kernel: eight chunks, products and exponentials in turn.
    auto round_of = [&](int i, f32x16_t (&z)[2], f32x16_t (&z_next)[2], auto plain, auto NEXT, auto ADD) {
      constexpr bool kNextRows = decltype(NEXT)::value, kAdd = decltype(ADD)::value;
      bf16x8_t q[8];
      auto operand_of = [&](int d) {
        return *reinterpret_cast<const bf16x8_t*>(s_rows + 32 * (i + 1) * kRowBytes + swizzled(col, 8 * half + d));
      };
      if constexpr (kNextRows) {
#pragma unroll
        for (int d = 0; d < 3; ++d) q[d] = operand_of(d);
        z_next[0] = z_next[1] = f32x16_t{};
      }
      float lse2 = 0.f;
      int sees = 0;
      if constexpr (kAdd) {
        lse2 = s_lse2[32 * i + col];
        // as in the wide kernel
        if constexpr (!decltype(plain)::value) sees = s_last[32 * i + col] - k0 - 4 * half;
      }
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int d = 0; d < 8; ++d) {
        if constexpr (kNextRows) {
          if (d + 3 < 8) q[d + 3] = operand_of(d + 3);
#pragma unroll
          for (int m = 0; m < 2; ++m) z_next[m] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[m][d], q[d], z_next[m], 0, 0, 0);
        }
        if constexpr (kAdd) add4(a, sum, z, d, lse2, sees, plain);
        __builtin_amdgcn_sched_barrier(0);
      }
    };
    auto run = [&](auto plain) {
      using Yes = std::true_type;
      using No = std::false_type;
      f32x16_t za[2], zb[2];
      round_of(-1, zb, za, plain, Yes{}, No{});
      int i = 0;
      for (; i + 2 < blocks; i += 2) {
        round_of(i, za, zb, plain, Yes{}, Yes{});
        round_of(i + 1, zb, za, plain, Yes{}, Yes{});
      }
      if (i + 1 < blocks) {
        round_of(i, za, zb, plain, Yes{}, Yes{});
        round_of(i + 1, zb, za, plain, No{}, Yes{});
      } else {
        round_of(i, za, zb, plain, No{}, Yes{});
      }
    };
    if (any >= 0) {
      if (k0 + kWideKeys <= old + 1) run(std::true_type{});   // every row sees all the wave's keys
      else run(std::false_type{});
    }
    sums_of_keys(sum, s_sum[wave]);
    __builtin_amdgcn_wave_barrier();
    const int key = k0 + lane;
    if (key < c1) {
      const float v = s_sum[wave][lane];
      w_out[key] = key < old ? before + v : v;
      if (key >= old) c.positions[(size_t)bg * c.stride + key] = c.first_position[b] + (key - old);
    }
    __builtin_amdgcn_wave_barrier();
  }
}

}  // namespace

hipError_t launch_kv8_attn_weights(const AttnWeightsCall& c, hipStream_t stream) {
  WeightsArgs a{};
  a.c = c;
  a.G = c.Hq / c.Hkv;
  a.page_shift = log2_pow2(c.page_size);
  a.sl2 = c.scale * kLog2e;
  const int64_t pairs = (int64_t)c.B * c.Hkv;
  const int64_t rows = (int64_t)c.N * a.G;
  if (rows > 64) {
    // In us, 256 workgroups at a time.  One of 256 keys passes 64 rows a round, one of 128
    // keys 128 rows; a round takes 1.2 to 1.3, the rest 4.  us a call, 256 / 128 keys: 4 x
    // 4096 keys of 4 heads, 256 rows of 7 heads 41.2 / 49.9, 32 of them 13.2 / 18.8; 4 x
    // 2048, 256 rows 37.3 / 27.3, 32 13.2 / 10.0.
    auto times = [&](int keys) { return std::ceil((double)(pairs * ((c.L_max + keys - 1) / keys)) / 256); };
    auto cost = [&](int keys, int round) { return 3 + times(keys) * (4 + 1.25 * (double)((rows + round - 1) / round)); };
    // Up to 256 rows in LDS with blocks of 512 keys in turn.  us a call, so / as above: 16 x
    // 8192 keys of 4 heads, 196 rows 38 / 72; 32 x 4096 of 8, 80 rows 45 / 116; 13 x 2000 of
    // 16, 100 rows 27 / 54; 2 x 4096 of 4, 196 rows 11.8 / 10.2.
    constexpr int kBlock = kMidWaves * kWideKeys;
    int blocks = 0;   // of a workgroup, best
    double least = std::min(cost(256, 64), cost(128, 128));
    for (int p = 1; p <= kMidBlocks && rows <= kMidRows; ++p) {
      const double t = 2.5 + times(p * kBlock) * (2.2 + p * (0.3 + 0.97 * (double)((rows + 31) / 32)));
      if (t < least) {
        least = t;
        blocks = p;
      }
    }
    if (blocks > 0) {
      a.chunk = blocks * kBlock;
      a.nsplit = (c.L_max + a.chunk - 1) / a.chunk;
      hipLaunchKernelGGL(kv8_weights_mid_kernel, dim3((unsigned)(pairs * a.nsplit)), dim3(kMidThreads), 0, stream, a);
      return hipGetLastError();
    }
    auto wide = [&](auto KG, auto parts) {
      constexpr int kg = decltype(KG)::value, kp = decltype(parts)::value;
      a.chunk = kg * kWideKeys;
      a.nsplit = (c.L_max + a.chunk - 1) / a.chunk;
      hipLaunchKernelGGL((kv8_weights_wide_kernel<kg, kp>), dim3((unsigned)(pairs * a.nsplit)), dim3(kg * kp * kWave), 0,
                         stream, a);
    };
    using Two = std::integral_constant<int, 2>;
    using Four = std::integral_constant<int, 4>;
    if (cost(256, 64) <= cost(128, 128)) wide(Four{}, Two{});
    else wide(Two{}, Four{});
    return hipGetLastError();
  }
  // Steps of a wave by the least estimated time in us: at least a wave's own latency, start
  // and steps, and at least what all workgroups take, `at_once` of them at a time.  us a
  // call at the choice / with steps for 1024 workgroups, 8 at most: single tokens of 32
  // heads over 8, 32 x 8192 56.7 / 57.8, 4 x 12000 14.4 / 16.0, 13 x 4087 14.9 / 18.0; 28
  // rows, 13 x 4087 12.8 / 17.1; 42 rows, 13 x 4087 16.1 / 25.0; 52 rows, 32 x 4087 36.7 /
  // 47.2.  Over 80 sizes it is 2 % behind the best number of steps on average (15 on these
  // sizes by the other rule).
  struct Cost {
    double start, step, base, group, group_step;
    int at_once, most;
  };
  static const Cost costs[] = {{4.0, 0.65, 2.3, 2.2, 1.75, 1024, 8},        // up to 16 rows
                               {4.7, 0.95, 3.3, 2.5, 1.7, 768, kMaxSteps},   // 32
                               {5.7, 1.2, 5.6, 2.9, 1.9, 512, kMaxSteps}};   // 64
  const Cost& k = costs[rows <= 16 ? 0 : rows <= 32 ? 1 : 2];
  constexpr int kUnit = kNarrowWaves * kStep;
  const int units = (c.L_max + kUnit - 1) / kUnit;
  int per = 1;
  double least = 0.0;
  for (int p = 1; p <= k.most; ++p) {
    const double groups = (double)(pairs * ((units + p - 1) / p));
    const double t = std::max(k.start + k.step * p, k.base + groups / k.at_once * (k.group + k.group_step * p));
    if (p == 1 || t < least) {
      least = t;
      per = p;
    }
  }
  a.chunk = per * kUnit;
  a.nsplit = (units + per - 1) / per;
  auto narrow = [&](auto rb) {
    constexpr int RB = decltype(rb)::value;
    hipLaunchKernelGGL(kv8_weights_narrow_kernel<RB>, dim3((unsigned)(pairs * a.nsplit)), dim3(kNarrowThreads), 0, stream, a);
  };
  if (rows <= 16) narrow(std::integral_constant<int, 1>{});
  else if (rows <= 32) narrow(std::integral_constant<int, 2>{});
  else narrow(std::integral_constant<int, 4>{});
  return hipGetLastError();
}

}  // namespace adapld
