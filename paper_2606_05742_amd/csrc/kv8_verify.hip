// Tree-masked verify attention over the paged 8-bit K/V cache: the kernels of
// paged_verify.h for rows of E4M3 codes with a scale for each 16 tokens.
#include "kv8_device.h"
#include "paged_verify.h"

namespace adapld {
namespace {

// A part is two runs of 16 dimensions, 64 apart, so that a load of four lanes reads
// 64 bytes of a row in one piece.  The scale is that of the 16 keys that a load
// brings: the same for all its lanes.
struct Kv8Format {
  static constexpr int kLoads = 2, kCodeBytes = kKv8RowBytes;
  // Two loads share a line, which the non-temporal hint lets go between them: us a call,
  // plain / with it, single tokens, 32 x 8192 keys of 8 heads 93.6 / 103.9, 4 x 30000 51.5
  // / 58.1; 8 nodes, 16 x 4096 36.3 / 38.9.
  static constexpr size_t kStreamBytes = 0;
  static __device__ __forceinline__ uint32_t code_at(uint32_t key, int part, int i) { return key * kKv8RowBytes + i * 64 + part * 16; }
  static __device__ __forceinline__ int chunk(int part, int j) { return 8 * (j >> 1) + 2 * part + (j & 1); }
  static __device__ __forceinline__ uint32_t load_scale(const uint8_t* scales, size_t row, uint32_t, int) {
    return scales[row >> kKv8BlockShift];
  }
  static __device__ __forceinline__ uint4 dequant(const u32x4_t (&v)[2], int j, float X) {
    return kv8_values(make_uint2(v[j >> 1][2 * (j & 1)], v[j >> 1][2 * (j & 1) + 1]), X);
  }
};

}  // namespace

VerifyPagedPlan plan_verify_kv8(int B, int L_max, int T_max, int Hq, int Hkv) {
  static const PagedShape shapes[] = {{16, true, kWaves * kStep, 5.5, 1.3, 1.3},
                                      {32, true, kWaves * kStep, 5.5, 2.0, 2.0},
                                      {64, true, kWaves / 2 * kStep, 5.5, 1.7, 1.7},
                                      {128, false, kKeyTile, 10.0, 1.12, 1.12},
                                      {256, false, kKeyTile, 10.0, 1.9, 1.12}};
  return plan_paged(shapes, B, L_max, T_max, Hq, Hkv);
}

size_t verify_kv8_ws_bytes(const VerifyPagedPlan& p, int B, int Hkv) { return paged_ws_bytes(p, B, Hkv); }

hipError_t launch_tree_verify_attn_kv8(const VerifyPagedCall& c, const VerifyPagedPlan& p, hipStream_t stream) {
  return launch_paged<Kv8Format>(c, p, stream);
}

}  // namespace adapld
