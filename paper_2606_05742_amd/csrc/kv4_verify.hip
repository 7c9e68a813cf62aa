// Tree-masked verify attention over the paged 4-bit K/V cache: the kernels of
// paged_verify.h for rows of E2M1 codes with a scale for each 32 dimensions.
//
// v_cvt_scalef32_pk_bf16_fp4 converts two codes in 6 to 8 cycles of a wave, exactly
// (E2M1 times a power of two).  The matrix instructions that take 4-bit operands
// beside 8-bit ones would save K's conversion, but drop products below 2^-13 of the
// largest in a sum (measured), so they are not used.
//
// Where it stands (us a call, bytes and flops of the definition): single tokens,
// 32 sequences x 8192 keys, 32 heads over 8: 46, 6.2 TB/s, HBM bound (a copy
// moves 4.8, the fastest reads here 6.0 to 6.5); chains of 16 nodes, 32 x 4096: 53,
// two row blocks convert the same codes; 16 x 8192, 52 nodes: 126 to 137 by the box,
// 0.82 to 0.89 PFLOP/s, and 8 x 32768, 64 over 8, 72 nodes: 611 to 658, 0.94 to 1.01,
// of the 1.14 of a large library product: the matrix products (48 % of the cycles),
// the exponentials and the conversions share two waves a SIMD.
#include "kv4.h"
#include "paged_verify.h"

namespace adapld {
namespace {

// A part is a group of 32 dimensions: 16 bytes of codes and a scale of its own.
struct Kv4Format {
  static constexpr int kLoads = 1, kCodeBytes = kKv4RowBytes;
  static constexpr int kSmallFrom = 0;
  // A model's layers each bring their own cache, so a call finds its codes in
  // HBM; where one wave reads each of them, large ones are streamed past the
  // caches.  us a call over rotating caches, plain / non-temporal: single tokens,
  // 32 x 8192 keys of 8 kv heads (256 MiB of codes) 58.5 / 54.5, 4 x 30000 (117)
  // 35.4 / 32.5; 8 nodes, 16 x 4096 (64) 29.4 / 27.9; 8 x 2048 (16) 12.9 / 12.9.
  // Called again on the same cache, plain loads find it in the last-level cache:
  // 49.4 / 54.4, 29.4 / 30.8, 25.4 / 27.3, 10.8 / 11.3; so small ones load plainly.
  // Two row blocks read the codes twice: chains of 16 nodes, 32 x 4096 62.5 / 63.5.
  static constexpr size_t kStreamBytes = (size_t)64 << 20;
  static __device__ __forceinline__ uint32_t code_at(uint32_t key, int part, int) { return key * kKv4RowBytes + part * 16; }
  static __device__ __forceinline__ int chunk(int part, int j) { return 4 * part + j; }
  static __device__ __forceinline__ uint32_t load_scale(const uint8_t* scales, size_t row, uint32_t key, int part) {
    return (scales + row * kKv4Scales)[key * kKv4Scales + part];
  }
  static __device__ __forceinline__ uint4 dequant(const u32x4_t (&v)[1], int j, float X) {
    const uint32_t c = v[0][j];
    uint4 r;
    r.x = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, X, 0));
    r.y = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, X, 1));
    r.z = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, X, 2));
    r.w = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, X, 3));
    return r;
  }
};

}  // namespace

VerifyPagedPlan plan_verify_kv4(int B, int L_max, int T_max, int Hq, int Hkv) {
  // The constants (us) were fitted before the kernels' last
  // steps and read up to 36 % high; what counts is the order of the candidates,
  // which holds.  us a call inside a graph over three sets of inputs, at the choice
  // / at others: 16 x 8192 keys, 32 heads over 8, 52 nodes 256 rows in 2 splits 133
  // to 138 / 128 rows unsplit 141, in 2 154; 8 x 32768, 64 over 8, 72 nodes 256 rows
  // in 4 616 / 128 in 4 675; 4 x 2048, 40 over 8, 136 nodes 128 unsplit 46 / 256 in 2
  // 48; 1 x 4096, 32 over 8, 44 nodes 128 in 13 20.8 / in 16 20.8, in 11 20.2; 24 x
  // 6007 at most, 28 over 4, 35 nodes 256 in 2 89 / in 3 96, 128 unsplit 98; single
  // tokens, 4 x 30000, 64 over 8 in 8 29 / in 6 32; 8 x 2048, 32 over 8 in 4 11.2 /
  // in 2 12.0.
  // Up to 64 rows the narrow shape that just holds them, us at it / at the next
  // larger one (as above): single tokens 32 x 8192 47 to 49 / 53, 1 x 4096 9.7 /
  // 10.5 (4 rows); 32 rows, 16 x 4096 24.2 / 30.5; 64 rows, 32 x 4096 56 / 76, 4 x
  // 4096 19.1 / 21.1.
  static const PagedShape shapes[] = {{16, true, kWaves * kStep, 5.5, 1.3, 1.3},
                          {32, true, kWaves * kStep, 5.5, 2.0, 2.0},
                          {64, true, kWaves / 2 * kStep, 5.5, 1.7, 1.7},
                          {128, false, kKeyTile, 10.0, 1.12, 1.12},
                          {256, false, kKeyTile, 10.0, 1.9, 1.12}};
  return plan_paged(shapes, B, L_max, T_max, Hq, Hkv);
}

size_t verify_kv4_ws_bytes(const VerifyPagedPlan& p, int B, int Hkv) { return paged_ws_bytes(p, B, Hkv); }

hipError_t launch_tree_verify_attn_kv4(const VerifyPagedCall& c, const VerifyPagedPlan& p, hipStream_t stream) {
  return launch_paged<Kv4Format>(c, p, stream);
}

}  // namespace adapld
