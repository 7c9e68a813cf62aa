// Tree-masked verify attention over the paged 8-bit K/V cache: the kernels of
// paged_verify.h for rows of E4M3 codes with a scale for each 16 tokens.
//
// Where it stands, us a call: single tokens, 32 x 8192 keys of 8 heads, 93 (538 MB, 5.8
// TB/s: the reads).  16 x 8192, 52 nodes, 32 heads over 8, 142 (0.79 PFLOP/s, of which the
// merge 9), some 8 % behind 4-bit rows: twice the bytes and the same products beside the
// same vector instructions.  Left out there one at a time (of 146): the codes' loads 123,
// the exponentials 133, the conversions 146.  Four tiles of codes in flight, and products
// and exponentials in chunks kept apart by scheduling barriers, changed nothing.  One
// sequence, 32 heads, 517 keys: 9.2, of which 4.7 a launch with a step of keys; a CU
// brings the rest at 31 bytes a ns.
#include "kv8_device.h"
#include "paged_verify.h"

namespace adapld {
namespace {

// A part is two runs of 16 dimensions, 64 apart, so that a load of four lanes reads
// 64 bytes of a row in one piece.  The scale is that of the 16 keys that a load
// brings: the same for all its lanes.
struct Kv8Format {
  static constexpr int kLoads = 2, kCodeBytes = kKv8RowBytes;
  // Where there are more workgroups than CUs, two share one.  us a call, 4 / 8 waves: 64 x
  // 4096 keys of 8 heads, single tokens 93.9 / 97.2; 48 x 4096 76.4 / 81.7; 16 x 300 of 32
  // heads 12.9 / 15.5; 64 x 517 of 8, 8 nodes 21.0 / 25.8; 45 x 130 of 32, 56 rows 54.1 /
  // 67.0.  With no more they are the same or slower: 1 x 517 of 32 10.1 / 9.3, 32 x 4096, 64
  // rows 86.6 / 81.7.
  static constexpr int kSmallFrom = 256;
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

// What the constants were fitted to, us a call in a graph at the choice / at others, 32
// heads over 8 unless said: single tokens, 1 x 517 keys unsplit 9.1 / in 3 9.2 (and a
// launch more for the host); 1 x 1024 in 4 9.1 / unsplit 12.6; 8 x 1024 in 4 11.0 /
// unsplit 13.6; 1 x 8192 in 16 14.1 / in 32 15.4; 16 x 8192 in 2 53 / unsplit 66, in 4
// 57.  8 nodes: 1 x 768 in 3 12.9 / unsplit 15.5; 16 nodes: 1 x 384 in 3 12.7 / unsplit
// 15.8, 1 x 4096 in 16 18.2 / in 32 20.8.  Over 175 sizes the choice is 0.5 % behind the
// best on average (16 at most); over 87 of tiles 1.5 (13).  Tiles, with the 4-bit cache's constants: 16 x 8192, 52
// nodes 256 rows in 2 143 / in 4 156, 128 rows unsplit 164; 24 x 6007 at most, 28 over 4,
// 35 nodes 256 in 2 93 / in 3 100, 128 unsplit 103; 1 x 4096 128 in 13 25.9 / in 8 24.6.
VerifyPagedPlan plan_verify_kv8(int B, int L_max, int T_max, int Hq, int Hkv) {
  static const PagedShape shapes[] = {{16, true, kWaves * kStep, 5.3, 1.75, 1.75, 2.7, 0.2, true},
                                      {32, true, kWaves * kStep, 8.9, 1.8, 1.8, 2.7, 0.2, true},
                                      {64, true, kWaves / 2 * kStep, 10.4, 1.77, 1.77, 2.5, 0.25, true},
                                      {128, false, kKeyTile, 10.0, 1.12, 1.12},
                                      {256, false, kKeyTile, 10.0, 1.9, 1.12}};
  return plan_paged(shapes, B, L_max, T_max, Hq, Hkv);
}

size_t verify_kv8_ws_bytes(const VerifyPagedPlan& p, int B, int Hkv) { return paged_ws_bytes(p, B, Hkv); }

hipError_t launch_tree_verify_attn_kv8(const VerifyPagedCall& c, const VerifyPagedPlan& p, hipStream_t stream) {
  return launch_paged<Kv8Format>(c, p, stream);
}

}  // namespace adapld
