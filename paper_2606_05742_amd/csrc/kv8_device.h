// Values of the 8-bit cache in registers: 8 dimensions of a row are a lane's 16 bytes
// of bf16 or 8 bytes of codes, a row is 16 lanes.
#pragma once

#include "device_utils.h"
#include "kv8.h"

namespace adapld {

constexpr int kKv8RowLanes = ADAPLD_HEAD_DIM / 8;

// The largest magnitude of 8 bf16 values as bits.
typedef uint16_t kv8_u16x2_t __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t kv8_max2(uint32_t a, uint32_t b) {
  return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(kv8_u16x2_t, a), __builtin_bit_cast(kv8_u16x2_t, b)));
}
__device__ __forceinline__ uint32_t kv8_amax2(uint4 x) {   // of either half of the words
  const uint32_t m = 0x7fff7fffu;
  return kv8_max2(kv8_max2(x.x & m, x.y & m), kv8_max2(x.z & m, x.w & m));
}
__device__ __forceinline__ uint32_t kv8_halves_max(uint32_t m) { return max(m & 0xffffu, m >> 16); }
// The same with infinities and NaN left out.
__device__ __forceinline__ uint32_t kv8_finite_amax(uint4 x) {
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

// 8 bf16 values of magnitudes up to 448 X as codes: rounded once, to the nearest, ties
// to even.
__device__ __forceinline__ uint2 kv8_round(uint4 x, float X) {
  kv8_s16x2_t a{}, b{};
  a = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(a, __builtin_bit_cast(bf16x2_t, x.x), X, false);
  a = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(a, __builtin_bit_cast(bf16x2_t, x.y), X, true);
  b = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(b, __builtin_bit_cast(bf16x2_t, x.z), X, false);
  b = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(b, __builtin_bit_cast(bf16x2_t, x.w), X, true);
  return make_uint2(__builtin_bit_cast(uint32_t, a), __builtin_bit_cast(uint32_t, b));
}
// Any 8 values: magnitudes above 448 X (infinities, and what 2^(kKv8MaxExp - 127) does
// not reach) as 448 X, NaN as 0x7f (the conversion gives 0xff, whatever the NaN's sign).
__device__ __forceinline__ uint32_t kv8_plain_nan(uint32_t c) {
  return c & ~(((c & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u);
}
__device__ __forceinline__ uint2 kv8_quantise(uint4 x, int e) {
  const uint32_t most = (uint32_t)(e + 8) << 7 | 0x60u;
  uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t lo = w[i] & 0x7fffu, hi = (w[i] >> 16) & 0x7fffu;
    const uint32_t lo2 = lo <= 0x7f80u ? min(lo, most) : lo, hi2 = hi <= 0x7f80u ? min(hi, most) : hi;
    w[i] = (w[i] & 0x80008000u) | lo2 | (hi2 << 16);
  }
  const uint2 c = kv8_round(make_uint4(w[0], w[1], w[2], w[3]), kv8_scale(e));
  return make_uint2(kv8_plain_nan(c.x), kv8_plain_nan(c.y));
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
