// The norm of query and key heads and their rotation by position, in one pass.
//
// 16 lanes take a head of a token, a lane 8 dimensions in two runs of 4 that hold the
// pairs it turns: neighbouring runs where pairs are (2i, 2i + 1), runs rot / 2 apart where
// they are (i, i + rot / 2).  So each angle is worked out once.  A wave takes one token and
// up to 4 * H of its heads, whose angles and weights are the same, with all their loads in
// flight before the first is used.
//
// Rows are read and written once, so the call is bound by HBM: 4 x 6007 tokens (a fifth of
// them padding), 28 heads over 4, 309 MB, 65 to 68 us, 4.6 to 4.8 TB/s where a copy moves
// 5.1.  A tree's few rows (16 x 52 tokens, 40 heads, 13.5 MB: 6.8 us) wait for memory once.
//
// An angle is the fraction of a turn frac(p * f) with f in units of 2^-64: the low 64
// bits of an integer product, exact for every position.  Its upper 32 bits go to the
// sine and cosine instructions, which take turns; they are off by 2^-22.9 at most
// (measured over 2^20 angles), against the 2^-9 of the output's rounding.
#include <hip/hip_runtime.h>

#include <type_traits>

#include "adapld_internal.h"
#include "device_utils.h"

namespace adapld {
namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / kWave;
constexpr int kLanes = ADAPLD_HEAD_DIM / 8;   // of a head
constexpr int kGroups = kWave / kLanes;       // heads of a wave at a time

// The sum over 16 lanes: rotations by 8, 4, 2 and 1.
__device__ __forceinline__ float sum16(float v) {
  v += dpp_f32<0x128>(v);
  v += dpp_f32<0x124>(v);
  v += dpp_f32<0x122>(v);
  return v + dpp_f32<0x121>(v);
}

__device__ __forceinline__ void unpack4(uint2 w, float* x) {
  x[0] = bf16_lo(w.x);
  x[1] = bf16_hi(w.x);
  x[2] = bf16_lo(w.y);
  x[3] = bf16_hi(w.y);
}

// Two fp32 values as bf16 (nearest, ties to even; infinities and NaN stay).
__device__ __forceinline__ uint32_t pack2(float a, float b) {
  typedef float f32x2_t __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2_t){a, b}, bf16x2_t));
}

// The angle p * f in turns, in [-1/2, 1/2).
__device__ __forceinline__ float turns(int64_t p, uint64_t f) {
  return (float)(int32_t)(uint32_t)(((uint64_t)p * f) >> 32) * 0x1p-32f;
}

typedef uint32_t u32x2_t __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
template <bool STREAM, class V>
__device__ __forceinline__ V load(const V* p) {
  if constexpr (STREAM) return __builtin_nontemporal_load(p);
  else return *p;
}
template <bool STREAM, class V>
__device__ __forceinline__ void store(V* p, V v) {
  if constexpr (STREAM) __builtin_nontemporal_store(v, p);
  else *p = v;
}

// Where the other half of a pair is: kBeside it (16 bytes a lane, both runs); rot_dim / 2
// on, kApart (8 bytes a run); or, where that is a power of two of lanes, so many on: then
// those lanes read 16 bytes each and exchange a run, before and after (14298 tokens of 64
// heads, 16 of 128 dimensions rotated 101 -> 87 us against 8 bytes a run).
constexpr int kBeside = 0, kApart = -1;

// What the lane X further on or back has.
template <int X>
__device__ __forceinline__ uint32_t of_lane_xor(uint32_t v) {
  static_assert(X == 1 || X == 2 || X == 4 || X == 8, "within a head's lanes");
  auto dpp = [](uint32_t x, auto ctrl) {
    return (uint32_t)__builtin_amdgcn_mov_dpp((int)x, decltype(ctrl)::value, 0xf, 0xf, false);
  };
  if constexpr (X == 1) return dpp(v, std::integral_constant<int, 0xb1>{});        // quad_perm 1 0 3 2
  else if constexpr (X == 2) return dpp(v, std::integral_constant<int, 0x4e>{});   // quad_perm 2 3 0 1
  else if constexpr (X == 4)                                                       // row_half_mirror, quad_perm 3 2 1 0
    return dpp(dpp(v, std::integral_constant<int, 0x141>{}), std::integral_constant<int, 0x1b>{});
  else return dpp(v, std::integral_constant<int, 0x128>{});                        // row_ror:8
}
template <int X>
__device__ __forceinline__ uint2 of_lane_xor(uint2 v) {
  return make_uint2(of_lane_xor<X>(v.x), of_lane_xor<X>(v.y));
}

// STREAM: for many rows; they are loaded and stored with the non-temporal hint, and
// not before it is known that the token counts.
template <int PAIRS, int H, bool STREAM>
__global__ __launch_bounds__(kThreads) void qk_norm_rope_kernel(const NormRopeCall c, int parts) {
  // B * T * parts fits 31 bits by the host's check
  const uint32_t job = blockIdx.x * kWaves + __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const uint32_t tok = job / (uint32_t)parts;
  const int b = (int)(tok / (uint32_t)c.T), u = (int)(tok - (uint32_t)b * c.T);
  if (b >= c.B) return;
  const int heads = c.Hq + c.Hkv, first = (int)(job - tok * (uint32_t)parts) * (kGroups * H);
  const int part = threadIdx.x % kLanes, group = lane_id() / kLanes;
  // the lane's two runs
  const bool rotated = part < c.rot_dim / 8;
  const bool low = !(part & PAIRS);
  const int run0 = PAIRS == kBeside || !rotated ? 8 * part : PAIRS == kApart ? 4 * part : low ? 8 * part : 8 * (part - PAIRS) + 4;
  const int run1 = PAIRS == kBeside || !rotated ? run0 + 4 : run0 + c.rot_dim / 2;
  const int freq0 = PAIRS == kBeside ? 4 * part : run0;

  const int count = c.counts ? c.counts[b] : c.T;
  const int base = c.base[b], offset = c.offsets ? c.offsets[(size_t)b * c.T + u] : u;
  if (STREAM && u >= count) return;
  uint2 x[H][2];
#pragma unroll
  for (int i = 0; i < H; ++i) {
    const int h = min(first + kGroups * i + group, heads - 1), side = h >= c.Hq;
    const uint16_t* const p = c.x[side] + b * c.batch[side] + u * c.token[side] + (size_t)(side ? h - c.Hq : h) * ADAPLD_HEAD_DIM;
    if constexpr (PAIRS != kApart) {
      const u32x4_t v = load<STREAM>(reinterpret_cast<const u32x4_t*>(p + 8 * part));
      x[i][0] = make_uint2(v[0], v[1]);
      x[i][1] = make_uint2(v[2], v[3]);
    } else {
      const u32x2_t v0 = load<STREAM>(reinterpret_cast<const u32x2_t*>(p + run0)), v1 = load<STREAM>(reinterpret_cast<const u32x2_t*>(p + run1));
      x[i][0] = make_uint2(v0[0], v0[1]);
      x[i][1] = make_uint2(v1[0], v1[1]);
    }
  }
  uint2 wr[2][2];
#pragma unroll
  for (int side = 0; side < 2; ++side) {
    if (c.weight[side]) {
      wr[side][0] = *reinterpret_cast<const uint2*>(c.weight[side] + run0);
      wr[side][1] = *reinterpret_cast<const uint2*>(c.weight[side] + run1);
    }
  }
  uint64_t f[4];
  if (rotated) {
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = c.freqs[freq0 + i];
  }
  if (u >= count) return;
  float w[2][8];
#pragma unroll
  for (int side = 0; side < 2; ++side) {
    unpack4(wr[side][0], w[side]);
    unpack4(wr[side][1], w[side] + 4);
  }
  float cs[4], sn[4];
  if (rotated) {
    const int64_t p = (int64_t)base + offset;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float t = turns(p, f[i]);
      cs[i] = __builtin_amdgcn_cosf(t);
      sn[i] = __builtin_amdgcn_sinf(t);
    }
  }
#pragma unroll
  for (int i = 0; i < H; ++i) {
    const int h = first + kGroups * i + group, side = h >= c.Hq;
    if (h >= heads) return;   // the 16 lanes of a head leave together
    if constexpr (PAIRS > 0) {
      const uint2 other = of_lane_xor<PAIRS>(low ? x[i][1] : x[i][0]);
      if (rotated && low) x[i][1] = other;
      if (rotated && !low) x[i][0] = other;
    }
    float y[8];
    unpack4(x[i][0], y);
    unpack4(x[i][1], y + 4);
    if (c.weight[side]) {
      float ss = 0.f;
#pragma unroll
      for (int k = 0; k < 8; ++k) ss = fmaf(y[k], y[k], ss);
      const float r = rsqrtf(fmaf(sum16(ss), 1.f / ADAPLD_HEAD_DIM, c.eps));
#pragma unroll
      for (int k = 0; k < 8; ++k) y[k] = y[k] * r * (side ? w[1][k] : w[0][k]);
    }
    if (rotated) {
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int lo = PAIRS == kBeside ? 2 * k : k, hi = PAIRS == kBeside ? 2 * k + 1 : k + 4;
        const float a = y[lo], z = y[hi];
        y[lo] = a * cs[k] - z * sn[k];
        y[hi] = z * cs[k] + a * sn[k];
      }
    }
    uint16_t* const to = c.out[side] + ((size_t)tok * (side ? c.Hkv : c.Hq) + (side ? h - c.Hq : h)) * ADAPLD_HEAD_DIM;
    uint2 r0 = make_uint2(pack2(y[0], y[1]), pack2(y[2], y[3])), r1 = make_uint2(pack2(y[4], y[5]), pack2(y[6], y[7]));
    if constexpr (PAIRS > 0) {
      const uint2 other = of_lane_xor<PAIRS>(low ? r1 : r0);
      if (rotated && low) r1 = other;
      if (rotated && !low) r0 = other;
    }
    if constexpr (PAIRS != kApart) {
      store<STREAM>(reinterpret_cast<u32x4_t*>(to + 8 * part), (u32x4_t){r0.x, r0.y, r1.x, r1.y});
    } else {
      store<STREAM>(reinterpret_cast<u32x2_t*>(to + run0), (u32x2_t){r0.x, r0.y});
      store<STREAM>(reinterpret_cast<u32x2_t*>(to + run1), (u32x2_t){r1.x, r1.y});
    }
  }
}

}  // namespace

hipError_t launch_qk_norm_rope(const NormRopeCall& c, hipStream_t stream) {
  const int64_t tokens = (int64_t)c.B * c.T;
  const int heads = c.Hq + c.Hkv;
  auto go = [&](auto h, auto st) {
    constexpr int H = decltype(h)::value;
    constexpr bool STREAM = decltype(st)::value;
    const int parts = (heads + kGroups * H - 1) / (kGroups * H);
    const dim3 grid((unsigned)((tokens * parts + kWaves - 1) / kWaves));
    auto launch = [&](auto pairs) {
      hipLaunchKernelGGL((qk_norm_rope_kernel<decltype(pairs)::value, H, STREAM>), grid, dim3(kThreads), 0, stream, c, parts);
    };
    if (c.interleaved) return launch(std::integral_constant<int, kBeside>{});
    switch (c.rot_dim) {
      case 16: return launch(std::integral_constant<int, 1>{});
      case 32: return launch(std::integral_constant<int, 2>{});
      case 64: return launch(std::integral_constant<int, 4>{});
      case 128: return launch(std::integral_constant<int, 8>{});
      default: return launch(std::integral_constant<int, kApart>{});
    }
  };
  using One = std::integral_constant<int, 1>;
  using Two = std::integral_constant<int, 2>;
  using Four = std::integral_constant<int, 4>;
  const int64_t rows = tokens * heads;
  // us a call, 4 / 8 / 16 heads a wave, the largest streamed: 1 token of 40 heads 2.7 / 3.0
  // / 3.9; 832 7.2 / 6.8 / 7.6; 2800 14.8 / 12.6 / 13.5; 24028 of 32 112 / 90 / 79, streamed
  // - / 78 / 68 (pairs beside each other 98 / 83 / 76, - / 73 / 65: 4.8 TB/s, where a copy
  // moves 5.1).  8 heads plain / 16 streamed: 190080 rows 23.7 / 24.4, 240000 33.3 / 31.2.
  if (rows <= 8192) go(One{}, std::false_type{});
  else if (rows <= 3 << 16) go(Two{}, std::false_type{});
  else go(Four{}, std::true_type{});
  return hipGetLastError();
}

}  // namespace adapld
