// Values of the 8-bit cache in registers: 8 dimensions of a row are a lane's 16 bytes
// of bf16 or 8 bytes of codes, a row is 16 lanes.
#pragma once

#include "device_utils.h"
#include "kv8.h"

namespace adapld {

constexpr int kKv8RowLanes = ADAPLD_HEAD_DIM / 8;

// The largest magnitude of 8 bf16 values as bits, infinities and NaN left out.
__device__ __forceinline__ uint32_t kv8_amax(uint4 x) {
  const uint32_t w[4] = {x.x, x.y, x.z, x.w};
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t lo = w[i] & 0x7fffu, hi = (w[i] >> 16) & 0x7fffu;
    m = max(m, max(lo < 0x7f80u ? lo : 0u, hi < 0x7f80u ? hi : 0u));
  }
  return m;
}
__device__ __forceinline__ uint32_t kv8_wave_max(uint32_t m) { return (uint32_t)wave_max_i32((int)m); }

// The exponent byte of the least scale X with amax <= 448 X = 1.75 * 2^8 X.  On the
// bits of a bf16 amax: a fraction above .75 (0x60) carries into the exponent.
__device__ __forceinline__ int kv8_exponent(uint32_t amax) {
  return min(max((int)((amax + 0x1fu) >> 7) - 8, kKv8MinExp), kKv8MaxExp);
}
__device__ __forceinline__ float kv8_scale(int e) { return __uint_as_float((uint32_t)e << 23); }

typedef short kv8_s16x2_t __attribute__((ext_vector_type(2)));

// 8 bf16 values as codes: rounded once, to the nearest, ties to even; magnitudes above
// 448 X (infinities, and what 2^(kKv8MaxExp - 127) does not reach) as 448 X, NaN as
// 0x7f (the conversion gives 0xff, whatever the NaN's sign).
__device__ __forceinline__ uint32_t kv8_plain_nan(uint32_t c) {
  return c & ~(((c & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u);
}
__device__ __forceinline__ uint2 kv8_quantise(uint4 x, int e) {
  const float X = kv8_scale(e);
  const uint32_t most = (uint32_t)(e + 8) << 7 | 0x60u;
  uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t lo = w[i] & 0x7fffu, hi = (w[i] >> 16) & 0x7fffu;
    const uint32_t lo2 = lo <= 0x7f80u ? min(lo, most) : lo, hi2 = hi <= 0x7f80u ? min(hi, most) : hi;
    w[i] = (w[i] & 0x80008000u) | lo2 | (hi2 << 16);
  }
  kv8_s16x2_t a{}, b{};
  a = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(a, __builtin_bit_cast(bf16x2_t, w[0]), X, false);
  a = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(a, __builtin_bit_cast(bf16x2_t, w[1]), X, true);
  b = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(b, __builtin_bit_cast(bf16x2_t, w[2]), X, false);
  b = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(b, __builtin_bit_cast(bf16x2_t, w[3]), X, true);
  return make_uint2(kv8_plain_nan(__builtin_bit_cast(uint32_t, a)), kv8_plain_nan(__builtin_bit_cast(uint32_t, b)));
}

// 8 codes as bf16 values, exact.
__device__ __forceinline__ uint4 kv8_values(uint2 c, float X) {
  uint4 r;
  r.x = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c.x, X, false));
  r.y = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c.x, X, true));
  r.z = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c.y, X, false));
  r.w = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c.y, X, true));
  return r;
}

// Codes of exponent `from` at exponent `to` >= from.
__device__ __forceinline__ uint2 kv8_rescale(uint2 c, int from, int to) {
  return kv8_quantise(kv8_values(c, kv8_scale(from)), to);
}

}  // namespace adapld
