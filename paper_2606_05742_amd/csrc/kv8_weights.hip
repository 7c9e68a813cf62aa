// The attention weight that each cached token gets from new rows, over the paged 8-bit
// cache: a pass over its keys alone, with the log-sum-exp that the attention left.
//
// For one sequence and kv head the n * G new query rows are stacked as row = i * G +
// head.  The codes become bf16 operands in registers (exact), the logits fp32 sums of
// matrix products, and a weight 2^(s scale log2(e) - lse log2(e)).  One wave (or one
// workgroup's waves in a fixed order) sums up all that a key gets, so the order of a
// sum does not depend on the launch.
#include <algorithm>
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

// The stacked row's query, or none: rows behind the last, and those whose entry of
// `rows` is no query.
struct RowAt {
  int i, h, u;
  bool in;
};
__device__ __forceinline__ RowAt row_at(const WeightsArgs& a, int b, int g, int n, int r) {
  RowAt x;
  const int rows = n * a.G, rr = max(min(r, rows - 1), 0);
  x.i = rr / a.G;
  x.h = g * a.G + (rr - x.i * a.G);
  x.u = a.c.rows ? a.c.rows[(size_t)b * a.c.N + x.i] : x.i;
  x.in = r < rows && x.u >= 0 && x.u < a.c.T_max;
  x.u = x.in ? x.u : 0;
  return x;
}
// Its log-sum-exp in units of log2; infinite where the row gives nothing.
__device__ __forceinline__ float lse2_of(const WeightsArgs& a, int b, const RowAt& x) {
  const float lse = a.c.lse[((size_t)b * a.c.Hq + x.h) * a.c.T_max + x.u];
  return x.in && lse > -INFINITY ? lse * kLog2e : INFINITY;
}
__device__ __forceinline__ const uint16_t* query_of(const WeightsArgs& a, int b, const RowAt& x) {
  return a.c.q + (((size_t)b * a.c.T_max + x.u) * a.c.Hq + x.h) * kD;
}

__device__ __forceinline__ bf16x8_t operand(uint32_t lo, uint32_t hi, float X) {
  return __builtin_bit_cast(bf16x8_t, kv8_values(make_uint2(lo, hi), X));
}
template <bool STREAM>
__device__ __forceinline__ u32x4_t load16(const uint8_t* p) {
  const u32x4_t* q = reinterpret_cast<const u32x4_t*>(p);
  if constexpr (STREAM) return __builtin_nontemporal_load(q);
  else return *q;
}
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
// Codes of two steps are in flight.
constexpr int kNarrowThreads = 256;
constexpr int kNarrowWaves = kNarrowThreads / kWave;
constexpr int kStep = 32;

template <int RB, bool STREAM>
__global__ __launch_bounds__(kNarrowThreads) void kv8_weights_narrow_kernel(const WeightsArgs a) {
  const AttnWeightsCall& c = a.c;
  const int bg = blockIdx.x / a.nsplit, split = blockIdx.x - bg * a.nsplit;
  const int b = bg / c.Hkv, g = bg - b * c.Hkv;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int lane = lane_id(), col = lane & 15, quad = lane >> 4;
  const int c0 = split * a.chunk;
  // Lane j holds the page ids of the two halves of the wave's step first + j.
  const int32_t* const table = c.page_table + (size_t)b * c.max_pages;
  int ids[2];
  auto load_ids = [&](int first) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int pos = c0 + (wave + (first + lane) * kNarrowWaves) * kStep + 16 * i;
      ids[i] = page_in_pool(table[min(pos >> a.page_shift, c.max_pages - 1)], c.n_pages);
    }
  };
  load_ids(0);
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
  auto load = [&](int s, Raw& r) {
    const int k0 = c0 + s * kStep, at = ((s - wave) / kNarrowWaves) & 63;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      // Keys behind the last read the last one again; their sums are not stored.
      int pos = k0 + 16 * i;
      uint32_t key = col;
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
      r.k[i][0] = load16<STREAM>(p + key * kKv8RowBytes + quad * 16);
      r.k[i][1] = load16<STREAM>(p + key * kKv8RowBytes + quad * 16 + 64);
      r.e[i] = c.k_scales[row >> kKv8BlockShift];
    }
    r.w = w_in[min(k0 + (lane & 31), max(old - 1, 0))];
  };
  // Codes of the second next step; behind the wave's last step that one again, so that
  // the number of loads in flight does not depend on a branch.
  const int last = wave + (steps - 1 - wave) / kNarrowWaves * kNarrowWaves;
  auto load_later = [&](int s, Raw& r) {
    const int later = min(s + 2 * kNarrowWaves, last);
    if ((later - wave) / kNarrowWaves % 64 == 0) load_ids((later - wave) / kNarrowWaves);
    load(later, r);
  };
  Raw r[2];
  load(wave, r[0]);
  load(min(wave + kNarrowWaves, last), r[1]);

  bf16x8_t q[RB][4];
  float lse2[RB][4];
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    const RowAt x = row_at(a, b, g, n, 16 * rb + col);
    const uint4* const p = reinterpret_cast<const uint4*>(query_of(a, b, x));
#pragma unroll
    for (int j = 0; j < 4; ++j)   // a row that is none must not bring a NaN
      q[rb][j] = __builtin_bit_cast(bf16x8_t, x.in ? p[8 * (j >> 1) + 2 * quad + (j & 1)] : make_uint4(0, 0, 0, 0));
#pragma unroll
    for (int t = 0; t < 4; ++t) lse2[rb][t] = lse2_of(a, b, row_at(a, b, g, n, 16 * rb + 4 * quad + t));
  }

  auto step = [&](int s, Raw& x) {
    const int k0 = c0 + s * kStep;
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
          if (k0 + kStep > old)   // a new row sees no later one
            e = k0 + 16 * i + col <= old + (16 * rb + 4 * quad + t) / a.G ? e : 0.f;
          p[t] += e;
        }
      sum[i] = (p[0] + p[1]) + (p[2] + p[3]);
    }
    load_later(s, x);
    // lanes 0..15 and 16..31 take the sums of either half
    const float v0 = add_lane_xor32(add_lane_xor16(sum[0])), v1 = add_lane_xor32(add_lane_xor16(sum[1]));
    const float v = n == 0 ? 0.f : quad & 1 ? v1 : v0;   // without rows nothing is known of the keys
    const int key = k0 + lane;
    if (lane < kStep && key < c1) {
      w_out[key] = key < old ? w + v : v;
      if (key >= old) c.positions[(size_t)bg * c.stride + key] = c.first_position[b] + (key - old);
    }
  };
  int s = wave;
  for (; s + kNarrowWaves < steps; s += 2 * kNarrowWaves) {
    step(s, r[0]);
    step(s + kNarrowWaves, r[1]);
  }
  if (s < steps) step(s, r[0]);
}

// ---------------------------------------------------------- more than 64 rows
//
// A wave keeps 64 keys as A operands in registers and the rows pass by, 32 a block on
// v_mfma_f32_32x32x16_bf16: a lane then has one row, so one log-sum-exp, and 32 sums
// of keys that stay its own until the end.  Of a workgroup's 8 waves two share the
// keys, each with every other block of rows; blocks come through LDS, the next pair
// while the current one is multiplied.
constexpr int kWideThreads = 512;
constexpr int kWideKeys = 64;                         // of a wave
constexpr int kWideGroups = kWideThreads / kWave / 2; // of waves with the same keys
constexpr int kRowsBytes = 32 * kD * 2;               // a block of rows in LDS

// Physical 16-byte chunk of logical chunk ch in row r: lanes that read one chunk of 16
// consecutive rows hit every bank once.
__device__ __forceinline__ int swizzled(int r, int ch) { return (r << 8) + ((ch ^ (r & 15)) << 4); }

__global__ __launch_bounds__(kWideThreads, 2) void kv8_weights_wide_kernel(const WeightsArgs a) {
  __shared__ __attribute__((aligned(1024))) uint8_t s_rows[2][2][kRowsBytes];
  __shared__ float s_lse2[2][2][32];
  const AttnWeightsCall& c = a.c;
  const int bg = blockIdx.x / a.nsplit, split = blockIdx.x - bg * a.nsplit;
  const int b = bg / c.Hkv, g = bg - b * c.Hkv;
  const int tid = threadIdx.x;
  const int wave = __builtin_amdgcn_readfirstlane(tid / kWave);
  const int kg = wave % kWideGroups, part = wave / kWideGroups;
  const int lane = lane_id(), col = lane & 31, half = lane >> 5;
  const int old = min(max(c.lens_old[b], 0), c.L_max);
  const int n = min(max(min(max(c.lens_new[b], 0), c.L_max) - old, 0), c.N);
  const int end = old + n, c0 = split * (kWideGroups * kWideKeys);
  if (c0 >= end) return;
  const int k0 = c0 + kg * kWideKeys;
  const int rows = n * a.G;

  // Keys: lane (half, col) the dimensions [64 * half, +64) of keys col and 32 + col;
  // keys behind the last read the last one again, their sums are not stored.
  bf16x8_t kf[2][8];
#pragma unroll
  for (int m = 0; m < 2; ++m) {
    const int j = min(k0 + 32 * m + col, end - 1);
    const int page = page_in_pool(c.page_table[(size_t)b * c.max_pages + (j >> a.page_shift)], c.n_pages);
    const size_t row = pool_row(page, g, j & ((1 << a.page_shift) - 1), c.Hkv, a.page_shift);
    const float X = kv8_scale(c.k_scales[row >> kKv8BlockShift]);
    const u32x4_t* p = reinterpret_cast<const u32x4_t*>(c.k_codes + row * kKv8RowBytes + 64 * half);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const u32x4_t w = p[i];
      kf[m][2 * i] = operand(w[0], w[1], X);
      kf[m][2 * i + 1] = operand(w[2], w[3], X);
    }
  }

  // Loader: 512 threads bring 64 rows, a thread two 16-byte chunks of one row.
  const int lrow = tid >> 3, lch = tid & 7;
  uint4 next[2];
  float next_lse2 = 0.f;
  auto fetch = [&](int r0) {
    const RowAt x = row_at(a, b, g, n, r0 + lrow);
    const uint4* const p = reinterpret_cast<const uint4*>(query_of(a, b, x));
    next[0] = x.in ? p[lch] : make_uint4(0, 0, 0, 0);   // a row that is none must not bring a NaN
    next[1] = x.in ? p[lch + 8] : make_uint4(0, 0, 0, 0);
    if (lch == 0) next_lse2 = lse2_of(a, b, x);
  };
  auto store = [&](int buf) {
    uint8_t* const p = s_rows[buf][lrow >> 5];
    *reinterpret_cast<uint4*>(p + swizzled(lrow & 31, lch)) = next[0];
    *reinterpret_cast<uint4*>(p + swizzled(lrow & 31, lch + 8)) = next[1];
    if (lch == 0) s_lse2[buf][lrow >> 5][lrow & 31] = next_lse2;
  };
  fetch(0);
  store(0);
  __syncthreads();
  float sum[2][16] = {};
  const bool plain = k0 + kWideKeys <= old + 1;   // every row sees all the wave's keys
  int buf = 0;
  for (int r0 = 0; r0 < rows; r0 += 64, buf ^= 1) {
    if (r0 + 64 < rows) fetch(r0 + 64);
    const uint8_t* const p = s_rows[buf][part];
    const float lse2 = s_lse2[buf][part][col];
    f32x16_t z[2] = {};
#pragma unroll
    for (int d = 0; d < 8; ++d) {
      const bf16x8_t q = *reinterpret_cast<const bf16x8_t*>(p + swizzled(col, 8 * half + d));
#pragma unroll
      for (int m = 0; m < 2; ++m) z[m] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[m][d], q, z[m], 0, 0, 0);
    }
    if (plain) {
#pragma unroll
      for (int m = 0; m < 2; ++m)
#pragma unroll
        for (int t = 0; t < 16; ++t) sum[m][t] += __builtin_amdgcn_exp2f(fmaf(z[m][t], a.sl2, -lse2));
    } else {
      const int sees = old + (r0 + 32 * part + col) / a.G;
#pragma unroll
      for (int m = 0; m < 2; ++m)
#pragma unroll
        for (int t = 0; t < 16; ++t) {
          const float e = __builtin_amdgcn_exp2f(fmaf(z[m][t], a.sl2, -lse2));
          sum[m][t] += k0 + 32 * m + 8 * (t >> 2) + (t & 3) + 4 * half <= sees ? e : 0.f;
        }
    }
    if (r0 + 64 < rows) store(buf ^ 1);
    __syncthreads();
  }
  // Sums over the 32 lanes of a half, then of the two waves of the same keys.
  float* const s_sum = reinterpret_cast<float*>(s_rows);   // [waves][64 keys]
  __syncthreads();
#pragma unroll
  for (int m = 0; m < 2; ++m)
#pragma unroll
    for (int t = 0; t < 16; ++t) {
      float v = sum[m][t];
      v += __shfl_xor(v, 16, kWave);
      v += __shfl_xor(v, 8, kWave);
      v += __shfl_xor(v, 4, kWave);
      v += __shfl_xor(v, 2, kWave);
      v += __shfl_xor(v, 1, kWave);
      if (col == t) s_sum[wave * kWideKeys + 32 * m + 8 * (t >> 2) + (t & 3) + 4 * half] = v;
    }
  __syncthreads();
  if (tid < kWideGroups * kWideKeys) {
    const int key = c0 + tid;
    if (key < end) {
      const float v = s_sum[tid] + s_sum[kWideGroups * kWideKeys + tid];
      const size_t at = (size_t)bg * c.stride + key;
      c.weights_out[at] = key < old ? c.weights[at] + v : v;
      if (key >= old) c.positions[at] = c.first_position[b] + (key - old);
    }
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
    a.chunk = kWideGroups * kWideKeys;
    a.nsplit = (c.L_max + a.chunk - 1) / a.chunk;
    hipLaunchKernelGGL(kv8_weights_wide_kernel, dim3((unsigned)(pairs * a.nsplit)), dim3(kWideThreads), 0, stream, a);
    return hipGetLastError();
  }
  // Steps of a wave: up to 16, fewer while there are not 1024 workgroups.
  constexpr int kUnit = kNarrowWaves * kStep;
  const int units = (c.L_max + kUnit - 1) / kUnit;
  const int per = (int)std::min<int64_t>(16, std::max<int64_t>(1, pairs * units / 1024));
  a.chunk = per * kUnit;
  a.nsplit = (units + per - 1) / per;
  constexpr size_t kPlainBytes = (size_t)64 << 20;
  const bool stream_k = (size_t)pairs * c.L_max * kKv8RowBytes >= kPlainBytes;
  auto narrow = [&](auto rb) {
    constexpr int RB = decltype(rb)::value;
    const dim3 grid((unsigned)(pairs * a.nsplit));
    if (stream_k) hipLaunchKernelGGL((kv8_weights_narrow_kernel<RB, true>), grid, dim3(kNarrowThreads), 0, stream, a);
    else hipLaunchKernelGGL((kv8_weights_narrow_kernel<RB, false>), grid, dim3(kNarrowThreads), 0, stream, a);
  };
  if (rows <= 16) narrow(std::integral_constant<int, 1>{});
  else if (rows <= 32) narrow(std::integral_constant<int, 2>{});
  else narrow(std::integral_constant<int, 4>{});
  return hipGetLastError();
}

}  // namespace adapld
