// The attention weight that each cached token gets from new rows, over the paged 8-bit
// cache: a pass over its keys alone, with the log-sum-exp that the attention left.
#include "adapld_internal.h"
#include "kv8_device.h"

namespace adapld {
namespace {

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef float f32x16_t __attribute__((ext_vector_type(16)));

constexpr int kD = ADAPLD_HEAD_DIM;
constexpr int kThreads = 256;
constexpr int kWaves = kThreads / kWave;
constexpr int kStep = 32;   // keys of a wave
constexpr float kLog2e = 1.4426950408889634f;

// A wave takes 32 keys of one (sequence, kv head): their codes become bf16 A fragments
// in registers (exact), and blocks of 32 of the n * G stacked rows (row = i * G + head)
// pass by as B operands.  S^T = K Q^T on v_mfma_f32_32x32x16_bf16 leaves a lane one row
// and 16 keys, so the weights of a row need one log-sum-exp a lane, and the sums over
// rows are the lane's own until the end, when 32 lanes add up.  One wave alone has a
// key, so the order of a sum does not depend on the launch.
__global__ __launch_bounds__(kThreads) void kv8_weights_kernel(const AttnWeightsCall c, int chunks, int page_shift) {
  const int bg = blockIdx.x / chunks;
  const int b = bg / c.Hkv, g = bg - b * c.Hkv;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int lane = lane_id(), col = lane & 31, half = lane >> 5;
  const int old = min(max(c.lens_old[b], 0), c.L_max);
  const int n = min(max(min(max(c.lens_new[b], 0), c.L_max) - old, 0), c.N);
  const int end = old + n;
  const int64_t k0_64 = ((int64_t)(blockIdx.x - bg * chunks) * kWaves + wave) * kStep;
  if (k0_64 >= end) return;
  const int k0 = (int)k0_64;
  const int G = c.Hq / c.Hkv, rows = n * G;

  // Keys: lane (half, col) the dimensions [64 * half, +64) of key col; keys behind the
  // last read the last one again, their sums are not stored.
  bf16x8_t kf[8];
  {
    const int j = min(k0 + col, end - 1);
    const int page = page_in_pool(c.page_table[(size_t)b * c.max_pages + (j >> page_shift)], c.n_pages);
    const size_t row = pool_row(page, g, j & ((1 << page_shift) - 1), c.Hkv, page_shift);
    const float X = kv8_scale(c.k_scales[row >> kKv8BlockShift]);
    const uint4* p = reinterpret_cast<const uint4*>(c.k_codes + row * kKv8RowBytes + 64 * half);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint4 w = p[i];
      kf[2 * i] = __builtin_bit_cast(bf16x8_t, kv8_values(make_uint2(w.x, w.y), X));
      kf[2 * i + 1] = __builtin_bit_cast(bf16x8_t, kv8_values(make_uint2(w.z, w.w), X));
    }
  }
  const float sl2 = c.scale * kLog2e;
  float sum[16] = {};
  for (int r0 = 0; r0 < rows; r0 += 32) {
    const int r = min(r0 + col, rows - 1);
    const int i = r / G, h = g * G + (r - i * G);
    const int u = c.rows ? c.rows[(size_t)b * c.N + i] : i;
    const bool in = r0 + col < rows && u >= 0 && u < c.T_max;
    const int uu = in ? u : 0;
    const uint16_t* qp = c.q + (((size_t)b * c.T_max + uu) * c.Hq + h) * kD + 64 * half;
    const float lse = c.lse[((size_t)b * c.Hq + h) * c.T_max + uu];
    // a row that gives nothing: its weights are 2^-inf
    const float lse2 = in && lse > -INFINITY ? lse * kLog2e : INFINITY;
    f32x16_t s = f32x16_t{};
#pragma unroll
    for (int d = 0; d < 8; ++d)
      s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[d], __builtin_bit_cast(bf16x8_t, reinterpret_cast<const uint4*>(qp)[d]),
                                                  s, 0, 0, 0);
#pragma unroll
    for (int t = 0; t < 16; ++t) {
      const int key = k0 + 8 * (t >> 2) + (t & 3) + 4 * half;
      const float w = __builtin_amdgcn_exp2f(fmaf(s[t], sl2, -lse2));
      sum[t] += key <= old + i ? w : 0.f;
    }
  }
#pragma unroll
  for (int t = 0; t < 16; ++t) {
    float v = sum[t];
    v += __shfl_xor(v, 16, kWave);
    v += __shfl_xor(v, 8, kWave);
    v += __shfl_xor(v, 4, kWave);
    v += __shfl_xor(v, 2, kWave);
    v += __shfl_xor(v, 1, kWave);
    const int key = k0 + 8 * (t >> 2) + (t & 3) + 4 * half;
    if (col == t && key < end) {
      const size_t at = (size_t)bg * c.stride + key;
      c.weights_out[at] = key < old ? c.weights[at] + v : v;
      if (key >= old) c.positions[at] = c.first_position[b] + (key - old);
    }
  }
}

}  // namespace

hipError_t launch_kv8_attn_weights(const AttnWeightsCall& c, hipStream_t stream) {
  const int chunks = (c.L_max + kWaves * kStep - 1) / (kWaves * kStep);
  hipLaunchKernelGGL(kv8_weights_kernel, dim3((unsigned)((int64_t)c.B * c.Hkv * chunks)), dim3(kThreads), 0, stream, c,
                     chunks, log2_pow2(c.page_size));
  return hipGetLastError();
}

}  // namespace adapld
