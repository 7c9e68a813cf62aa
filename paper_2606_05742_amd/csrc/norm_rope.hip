// The norm of query and key heads and their rotation by position, in one pass.
//
// 16 lanes take a head of a token: a lane 8 dimensions (16 bytes).  The sum of squares
// is four exchanges within the 16 lanes.  The other half of a pair (i, i + rot / 2) is
// rot / 16 lanes away and comes by one exchange of the lane's packed 16 bytes;
// neighbouring pairs are a lane's own.
//
// An angle is the fraction of a turn frac(p * f) with f in units of 2^-64: the low 64
// bits of an integer product, exact for every position.  Its upper 32 bits go to the
// sine and cosine instructions, which take turns; they are off by 2^-22.9 at most
// (measured over 2^20 angles), against the 2^-9 of the output's rounding.
#include <hip/hip_runtime.h>

#include "adapld_internal.h"
#include "device_utils.h"

namespace adapld {
namespace {

constexpr int kThreads = 256;
constexpr int kLanes = ADAPLD_HEAD_DIM / 8;   // of a head

__device__ __forceinline__ float sum16(float v) {
  v += __shfl_xor(v, 8, kWave);
  v += __shfl_xor(v, 4, kWave);
  v += __shfl_xor(v, 2, kWave);
  return v + __shfl_xor(v, 1, kWave);
}

__device__ __forceinline__ void unpack8(uint4 w, float (&x)[8]) {
  const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = bf16_lo(u[i]);
    x[2 * i + 1] = bf16_hi(u[i]);
  }
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

template <bool INTERLEAVED>
__global__ __launch_bounds__(kThreads) void qk_norm_rope_kernel(const NormRopeCall c) {
  const int heads = c.Hq + c.Hkv;
  // B * T * heads fits 31 bits by the host's check
  const uint32_t row = blockIdx.x * (kThreads / kLanes) + threadIdx.x / kLanes;
  const uint32_t tok = row / (uint32_t)heads;
  int h = (int)(row - tok * (uint32_t)heads);
  const int b = (int)(tok / (uint32_t)c.T), u = (int)(tok - (uint32_t)b * c.T);
  if (b >= c.B) return;   // the 16 lanes of a head leave together
  if (c.counts && u >= c.counts[b]) return;
  const int side = h >= c.Hq;
  if (side) h -= c.Hq;
  const int part = threadIdx.x % kLanes, d0 = 8 * part;
  const uint4 raw = *reinterpret_cast<const uint4*>(c.x[side] + b * c.batch[side] + u * c.token[side] +
                                                    h * ADAPLD_HEAD_DIM + d0);
  const int half = c.rot_dim / 2;
  const bool rotated = d0 < c.rot_dim;
  float y[8];
  unpack8(raw, y);
  float r = 1.f;
  const uint16_t* const weight = c.weight[side];
  if (weight) {
    float ss = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) ss = fmaf(y[i], y[i], ss);
    r = rsqrtf(fmaf(sum16(ss), 1.f / ADAPLD_HEAD_DIM, c.eps));
    float w[8];
    unpack8(*reinterpret_cast<const uint4*>(weight + d0), w);
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = y[i] * r * w[i];
  }
  const int64_t p = (int64_t)c.base[b] + (c.offsets ? c.offsets[(size_t)b * c.T + u] : u);
  if constexpr (INTERLEAVED) {
    if (rotated) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float t = turns(p, c.freqs[d0 / 2 + i]);
        const float cs = __builtin_amdgcn_cosf(t), sn = __builtin_amdgcn_sinf(t);
        const float a = y[2 * i], z = y[2 * i + 1];
        y[2 * i] = a * cs - z * sn;
        y[2 * i + 1] = z * cs + a * sn;
      }
    }
  } else {
    // The other half: its values are raw * r * weight as here.
    const bool first = d0 < half;
    const int mate = rotated ? (first ? part + half / 8 : part - half / 8) : part;
    const int src = (lane_id() & ~(kLanes - 1)) + mate;
    uint4 o;
    o.x = __shfl(raw.x, src, kWave);
    o.y = __shfl(raw.y, src, kWave);
    o.z = __shfl(raw.z, src, kWave);
    o.w = __shfl(raw.w, src, kWave);
    if (rotated) {
      float z[8];
      unpack8(o, z);
      if (weight) {
        float w[8];
        unpack8(*reinterpret_cast<const uint4*>(weight + 8 * mate), w);
#pragma unroll
        for (int i = 0; i < 8; ++i) z[i] = z[i] * r * w[i];
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float t = turns(p, c.freqs[(first ? d0 : d0 - half) + i]);
        const float cs = __builtin_amdgcn_cosf(t), sn = __builtin_amdgcn_sinf(t);
        y[i] = first ? y[i] * cs - z[i] * sn : y[i] * cs + z[i] * sn;
      }
    }
  }
  uint4 out;
  out.x = pack2(y[0], y[1]);
  out.y = pack2(y[2], y[3]);
  out.z = pack2(y[4], y[5]);
  out.w = pack2(y[6], y[7]);
  *reinterpret_cast<uint4*>(c.out[side] + ((size_t)tok * (side ? c.Hkv : c.Hq) + h) * ADAPLD_HEAD_DIM + d0) = out;
}

}  // namespace

hipError_t launch_qk_norm_rope(const NormRopeCall& c, hipStream_t stream) {
  const int64_t rows = (int64_t)c.B * c.T * (c.Hq + c.Hkv);
  const dim3 grid((unsigned)((rows * kLanes + kThreads - 1) / kThreads));
  if (c.interleaved)
    hipLaunchKernelGGL(qk_norm_rope_kernel<true>, grid, dim3(kThreads), 0, stream, c);
  else
    hipLaunchKernelGGL(qk_norm_rope_kernel<false>, grid, dim3(kThreads), 0, stream, c);
  return hipGetLastError();
}

}  // namespace adapld
