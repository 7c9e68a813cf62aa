// Tree-masked verify attention over the paged 4-bit K/V cache (Sec. 3.6: all
// draft paths are scored in one target forward with tree attention).
//
// For one sequence and kv head the T*G query rows (node u, query head g*G + i) are
// stacked as row = u*G + i, so the G heads that share a kv head share every byte
// of the cache.  A workgroup of 8 waves takes a number of rows and one split of
// the context; the last split also takes the tree's keys, which are bf16.  Two
// kernels share the work by the number of rows: up to 64 rows a pass of
// independent waves (kv4_narrow_kernel), above a pipeline over tiles of 64 keys
// (kv4_verify_kernel).  Both convert the codes to bf16 (exact: E2M1 times a power
// of two; v_cvt_scalef32_pk_bf16_fp4, two values in 6 to 8 cycles of a wave) and
// multiply on bf16 matrix products with fp32 sums.  The matrix instructions that
// take 4-bit operands beside 8-bit ones would save K's conversion, but drop
// products below 2^-13 of the largest in a sum (measured), so they are not used.
//
// Where it stands (us a call, bytes and flops of the definition): single tokens,
// 32 sequences x 8192 keys, 32 heads over 8: 46, 6.2 TB/s, HBM bound (a copy
// moves 4.8, the fastest reads here 6.0 to 6.5); chains of 16 nodes, 32 x 4096: 53,
// two row blocks convert the same codes; 16 x 8192, 52 nodes: 126 to 137 by the box,
// 0.82 to 0.89 PFLOP/s, and 8 x 32768, 64 over 8, 72 nodes: 611 to 658, 0.94 to 1.01,
// of the 1.14 of a large library product: the matrix products (48 % of the cycles),
// the exponentials and the conversions share two waves a SIMD.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "adapld_internal.h"
#include "device_utils.h"
#include "kv4.h"

namespace adapld {
namespace {

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef float f32x2_t __attribute__((ext_vector_type(2)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef float f32x16_t __attribute__((ext_vector_type(16)));
typedef short s16x4_t __attribute__((ext_vector_type(4)));
typedef short s16x8_t __attribute__((ext_vector_type(8)));
typedef __attribute__((address_space(3))) s16x4_t lds_s16x4_t;
typedef __attribute__((address_space(3))) uint8_t lds_u8;
typedef __attribute__((address_space(3))) bf16x8_t lds_bf16x8_t;

constexpr int kD = ADAPLD_HEAD_DIM;
constexpr int kRowBytes = kD * 2;                 // one bf16 row in LDS
constexpr int kTileBytes = kKeyTile * kRowBytes;  // 16 KiB for K (and for V)
constexpr int kStages = 4;                        // ring of tiles, a power of two
constexpr int kVRegion = kStages * kTileBytes;    // the V tiles behind the K tiles
constexpr int kWaves = 8;
constexpr int kThreads = kWaves * kWave;
constexpr int kMaskWords = (ADAPLD_MAX_TREE_NODES + 63) / 64;
constexpr int kMaxChunk = 32768;                  // keys of one split, less the tree's: about 1 ms of a workgroup
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

// Weights are taken relative to a reference: a maximum of the row's logits seen
// so far (log2 units) plus a margin.  The maximum may lag: a step that looks for it
// moves it where it is more than kRescaleSlack behind, the others where a lane's
// weights of the step (16 at most) sum up to more than 2^kLag times the weight of
// the maximum.  The margin keeps a row's sum of weights below 1 even if all n of
// its keys are at that limit (8 at least share a lane's sum), so that no sum of
// weights times values leaves fp32's range, whatever finite values V holds, and no
// partial output or merge does: 2^margin is at least 2^kLag * n.  Weights of less
// than 2^(margin - 126) times the row's largest (2^-100 for 8192 keys) are zero, and
// products of a weight and a value below 2^-126 may be.
constexpr float kRescaleSlack = 8.0f;
constexpr int kLag = 12;   // log2(16) + kRescaleSlack: where the second rule asks, the first moves
inline int weight_margin(int L_max, int T_max) { return kLag + 1 + log2_pow2(std::max(L_max, T_max)); }

struct Kv4Args {
  VerifyKv4Call c;
  int G, rows_max, nw, nsplit, chunk, rowgroups, page_shift;
  int margin;          // weight_margin(L_max, T_max)
  float weight_limit;  // 2^(kLag - margin)
  float scale_log2;
  float* ws_o;     // [B*Hkv][nsplit][rows_max][D]  partial outputs O/l
  float2* ws_ml;   // [B*Hkv][nsplit][rows_max]     (reference in log2 units, sum)
};

// Physical 16-byte chunk of logical chunk c in key row r is c ^ swz(r).  LDS has 64
// four-byte banks for reads (a 256-byte row once around); 16-byte writes go by
// 8 lanes over 32 of them.  With r = r3 r2 r1 r0 the swizzle is (r1, r0, r1 ^ r3,
// r2): a bijection on 16 rows (K fragments: 16 lanes read one chunk of 16 rows),
// its low three bits one on every aligned 8 (the loader: 8 lanes write one chunk
// of 8 rows), its high two on every aligned 4 (transposed V reads: 32 lanes cover
// 64 bytes of 4 rows).  All three are free of bank conflicts.
__device__ __forceinline__ int swz(int r) {
  return ((r & 3) << 2) | ((((r >> 1) ^ (r >> 3)) & 1) << 1) | ((r >> 2) & 1);
}
// The same for transposed reads in which 32 lanes cover 32 bytes of 8 rows:
// (r2, r1, r0, r2 ^ r3), its high three bits a bijection on every aligned 8.
__device__ __forceinline__ int swz16(int r) { return ((r & 7) << 1) | (((r >> 2) ^ (r >> 3)) & 1); }

__device__ __forceinline__ bf16x8_t as_bf16x8(uint4 v) { return __builtin_bit_cast(bf16x8_t, v); }

// 8 codes with their scale as 8 bf16 values.
__device__ __forceinline__ uint4 dequant8(uint32_t c, float X) {
  uint4 r;
  r.x = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, X, 0));
  r.y = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, X, 1));
  r.z = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, X, 2));
  r.w = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, X, 3));
  return r;
}

// 16 bytes of codes; STREAM for data that nothing reads again.
typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
template <bool STREAM>
__device__ __forceinline__ uint4 load_codes(const uint8_t* p) {
  const u32x4_t* q = reinterpret_cast<const u32x4_t*>(p);
  u32x4_t v;
  if constexpr (STREAM) v = __builtin_nontemporal_load(q);
  else v = *q;
  return make_uint4(v[0], v[1], v[2], v[3]);
}

// ------------------------------------------------- one 32-row block's softmax
//
// S^T = K Q^T on v_mfma_f32_32x32x16_bf16 (A = 32 keys, B = 32 query rows)
// leaves a lane one query row (lane & 31) and 16 keys of it: value r is key
// 8*(r/4) + 4*(lane/32) + r%4.  So the online softmax is lane-local but for
// one exchange with the other half of the wave, and P^T goes straight back as
// the B operand of O^T = V^T P^T.
struct Block {
  float m, l;              // reference (log2 units) and this lane's share of the sum
  f32x16_t o[kD / 32];     // O^T: value r is dim 32*db + 8*(r/4) + 4*(lane/32) + r%4
};

__device__ __forceinline__ void block_init(Block& x) {
  x.m = -INFINITY;
  x.l = 0.f;
#pragma unroll
  for (int db = 0; db < kD / 32; ++db) x.o[db] = f32x16_t{};
}

// Keys at or past n (of 32) out, and with TREE those whose mask bit is 0.
template <bool TREE>
__device__ __forceinline__ void mask_keys(f32x16_t& s, int n, uint32_t bits) {
  const int k0 = 4 * (lane_id() >> 5);
#pragma unroll
  for (int r = 0; r < 16; ++r) {
    const int key = 8 * (r >> 2) + (r & 3) + k0;
    s[r] = key < n && (!TREE || ((bits >> key) & 1u)) ? s[r] : -INFINITY;
  }
}

// The softmax of 32 keys in pieces.  Logits, the reference (in log2 units), the
// sum and O are fp32; the weights are rounded to bf16 once, as the operand of P V
// (relative 2^-8, the size of the output's own rounding), and summed before that.
// P^T comes in the order of the B operand.
__device__ __forceinline__ float row_max(const f32x16_t& s) {
  float mx = fmaxf(fmaxf(s[0], s[1]), s[2]);
#pragma unroll
  for (int r = 3; r < 15; r += 2) mx = fmaxf(fmaxf(mx, s[r]), s[r + 1]);
  mx = fmaxf(mx, s[15]);
  const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_int(mx), __float_as_int(mx), false, false);
  return fmaxf(__int_as_float(sw[0]), __int_as_float(sw[1]));
}
__device__ __forceinline__ void rescale_to(Block& x, float mt) {
  const float m_new = fmaxf(x.m, mt);
  const float alpha = m_new == x.m ? 1.f : __builtin_amdgcn_exp2f(x.m - m_new);
  x.m = m_new;
  x.l *= alpha;
#pragma unroll
  for (int db = 0; db < kD / 32; ++db) x.o[db] *= alpha;
}
// The exponentials of values [8*s2, +8), added to psum.
__device__ __forceinline__ void exp_part(const f32x16_t& s, int s2, float sl2, float m_use, bf16x8_t& pb, float& psum) {
#pragma unroll
  for (int i = 0; i < 8; i += 2) {
    const float e0 = __builtin_amdgcn_exp2f(fmaf(s[8 * s2 + i], sl2, -m_use));
    const float e1 = __builtin_amdgcn_exp2f(fmaf(s[8 * s2 + i + 1], sl2, -m_use));
    psum += e0 + e1;
    const bf16x2_t pk = __builtin_convertvector((f32x2_t){e0, e1}, bf16x2_t);
    pb[i] = pk[0];
    pb[i + 1] = pk[1];
  }
}
// The reference that a step's own maximum gives (scale > 0, so the max commutes
// with scaling).
__device__ __forceinline__ float reference_of(float mx, float sl2, float margin) { return fmaf(mx, sl2, margin); }
__device__ __forceinline__ void softmax_step(const f32x16_t& s, float sl2, float margin, Block& x, bf16x8_t (&pb)[2]) {
  const float mt = reference_of(row_max(s), sl2, margin);
  if (__ballot(mt > x.m + kRescaleSlack)) rescale_to(x, mt);
  const float m_use = x.m == -INFINITY ? 0.f : x.m;
  float psum = 0.f;
  exp_part(s, 0, sl2, m_use, pb[0], psum);
  exp_part(s, 1, sl2, m_use, pb[1], psum);
  x.l += psum;
}

// Natural logarithm of the sum of exponentials that a reference and a sum of
// weights (> 0) stand for.
__device__ __forceinline__ float lse_of(const Kv4Args& a, float m, float l) {
  return (m - (float)a.margin + log2f(ldexpf(l, a.margin))) * kLn2;
}

// Four dimensions (chunk ch of 32) of a finished row: to the output, or to the
// partial outputs of a split context.  v is the unnormalised output, ml its
// reference and sum; 32 lanes store a row.
__device__ __forceinline__ void store_row(const Kv4Args& a, int b, int g, int split, int qr, int ch, float2 ml,
                                          float4 v) {
  const VerifyKv4Call& c = a.c;
  const float inv = ml.y > 0.f ? 1.f / ml.y : 0.f;   // a row without any key: 0
  v = make_float4(v.x * inv, v.y * inv, v.z * inv, v.w * inv);
  if (a.nsplit == 1) {
    const int u = qr / a.G, h = g * a.G + (qr - u * a.G);
    uint2 pk;
    pk.x = f32_to_bf16_bits(v.x) | (f32_to_bf16_bits(v.y) << 16);
    pk.y = f32_to_bf16_bits(v.z) | (f32_to_bf16_bits(v.w) << 16);
    *reinterpret_cast<uint2*>(c.out + (((size_t)b * c.T_max + u) * c.Hq + h) * kD + 4 * ch) = pk;
    if (ch == 0 && c.lse)
      c.lse[((size_t)b * c.Hq + h) * c.T_max + u] = ml.y > 0.f ? lse_of(a, ml.x, ml.y) : -INFINITY;
  } else {
    const size_t at = (((size_t)b * c.Hkv + g) * a.nsplit + split) * a.rows_max + qr;
    *reinterpret_cast<float4*>(a.ws_o + at * kD + 4 * ch) = v;
    if (ch == 0) a.ws_ml[at] = ml;
  }
}

// V^T fragment of 16 keys x 32 dims from row-major bf16 rows: each 16-lane
// group reads 4 keys x 16 dims transposed, in the key order of P^T.
__device__ __forceinline__ bf16x8_t v_fragment(const lds_u8* rows, int lo_ofs, int hi_ofs) {
  const s16x4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_t*)(rows + lo_ofs));
  const s16x4_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_t*)(rows + hi_ofs));
  const s16x8_t vv = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
  return __builtin_bit_cast(bf16x8_t, vv);
}
// Byte offsets of a lane's two reads for dims [32*db, +32): keys vkey and vkey + 8.
__device__ __forceinline__ void v_offsets(int (&vofs)[2][kD / 32]) {
  const int lane = lane_id();
  const int vkey = 4 * (lane >> 5) + ((lane & 15) >> 2);
  const int vdim = (lane & 16) + 4 * (lane & 3);
#pragma unroll
  for (int db = 0; db < kD / 32; ++db) {
    const int c = (db * 32 + vdim) >> 3;
    vofs[0][db] = vkey * kRowBytes + ((c ^ swz(vkey)) << 4) + (vdim & 7) * 2;
    vofs[1][db] = (vkey + 8) * kRowBytes + ((c ^ swz(vkey + 8)) << 4) + (vdim & 7) * 2;
  }
}

// ------------------------------------------------------------ more than 64 rows
//
// R 32-row blocks per workgroup; with R = 8 every wave owns one and takes both
// 32-key halves of each tile, with R = 4 two waves share one and take a half
// each.  Tiles of 64 keys are converted once per workgroup, by all its waves, into
// a ring of 4 bf16 stages in LDS (128 KiB): while tile t is computed, tile t + 1 is
// written and the codes of t + 2 and t + 3 are in flight in registers (10 of
// them, against 128 KiB of LDS for bf16 tiles).  One barrier a tile publishes the
// next tile and frees the one before.  The loop is software-pipelined over half
// tiles: the products P V of half h - 1 and S of half h + 1 are issued beside the
// exponentials of half h, with every LDS address a lane offset plus an immediate
// (the loop is unrolled over the ring).
//
// A tile takes 1.9 us with R = 8 and 1.1 with R = 4, all CUs busy; a SIMD's share
// is 64 products (1.0 us) and some 2200 cycles of vector instructions, of which
// the exponentials are 1000 and the conversions 450.  What did not help, us a call
// before / after: matrix products at a raised wave priority 141 / 149 (16 x 8192,
// 52 nodes), the exponentials 141 / 148, the two waves of a SIMD in turn 141 / 146;
// one product to four vector instructions by scheduling groups 141 / 146; V
// fragments requested a half ahead 141 / 142; the tree's tiles first 22.5 / 23.3 (1
// x 4096, 44 nodes); results written through LDS in whole lines 49 / 51 (4 x 2048,
// 136 nodes; stored by all eight waves, equal: they leave at 5.4 TB/s either way).
template <int R>
__global__ __launch_bounds__(kThreads, 1) void kv4_verify_kernel(const Kv4Args a) {
  static_assert(R == 8 || R == 4, "one or two waves per row block");
  constexpr int KH = kWaves / R;
  constexpr int HP = 2 / KH;   // 32-key halves of a tile that one wave takes
  __shared__ __attribute__((aligned(1024))) uint8_t smem[2 * kVRegion];
  __shared__ uint64_t s_mask[ADAPLD_MAX_TREE_NODES * kMaskWords];
  const VerifyKv4Call& c = a.c;

  // ---- the workgroup's job: the row groups of one (sequence, kv head, split)
  // have consecutive slots on one XCD, so its L2 serves the second reader.
  const int slot = blockIdx.x >> 3;
  const int unit = (slot / a.rowgroups) * 8 + (blockIdx.x & 7);   // = bg * nsplit + split
  const int rg = slot % a.rowgroups;
  const int bg = unit / a.nsplit, split = unit - bg * a.nsplit;
  const int b = bg / c.Hkv, g = bg - b * c.Hkv;
  if (b >= c.B) return;
  const int G = a.G;
  const int row_base = rg * (R * 32);
  const int tid = threadIdx.x;
  const int lane = lane_id();
  const int wave = __builtin_amdgcn_readfirstlane(tid / kWave);
  const int wrow = wave % R, kh = wave / R;
  const int col = lane & 31, half = lane >> 5;

  // ---- one memory round trip for everything that no other load decides: the
  // lengths, the page ids of a full split, the queries of a full tree and its
  // mask (what lies behind the sequence's own length and nodes goes unused).
  const int c0 = split * a.chunk;
  // loader: waves 0-3 bring K, waves 4-7 V; a lane one group of 32 dimensions (16
  // bytes of codes) of one key.  A wave's 16 keys never cross a page: lane j
  // holds their page id of tile first + j, and an address is a scalar base plus a
  // fixed lane offset.
  const bool is_v = wave >= 4;
  const int lkey = 16 * (wave & 3) + (lane & 15), lgrp = lane >> 4;
  const int32_t* const table = c.page_table + (size_t)b * c.max_pages;
  int ids;
  auto load_ids = [&](int first) {
    const int pos = c0 + (first + lane) * kKeyTile + 16 * (wave & 3);
    ids = kv4_page_in_pool(table[min(pos >> a.page_shift, c.max_pages - 1)], c.n_pages);
  };
  load_ids(0);
  const int nodes = c.node_count[b], len = c.lens[b];
  // Query fragments (B operand): lane holds dims [16*ds + 8*half, +8) of its row.
  const int qr = row_base + wrow * 32 + col;
  const int u = qr < a.rows_max ? qr / G : 0;
  const int h = g * G + (qr < a.rows_max ? qr - u * G : 0);
  bf16x8_t qf[kD / 16];
  {
    const uint16_t* qp = c.q + (((size_t)b * c.T_max + u) * c.Hq + h) * kD + 8 * half;
#pragma unroll
    for (int ds = 0; ds < kD / 16; ++ds) qf[ds] = as_bf16x8(*reinterpret_cast<const uint4*>(qp + 16 * ds));
  }
  const bool do_tree = split == a.nsplit - 1 && c.k_tree;
  if (do_tree)
    for (int i = tid; i < c.T_max * a.nw; i += kThreads) s_mask[i] = c.tree_mask[(size_t)b * c.T_max * a.nw + i];
  const int T = min(max(nodes, 0), c.T_max);
  const int L = min(max(len, 0), c.L_max);
  const int rows = T * G;
  if (row_base >= rows) return;
  const bool valid = qr < rows;
  const int c1 = min(c0 + a.chunk, L);
  const int n_ctx = c1 > c0 ? (c1 - c0 + kKeyTile - 1) / kKeyTile : 0;
  const int n_tiles = n_ctx + (do_tree ? (T + kKeyTile - 1) / kKeyTile : 0);

  const uint8_t* const codes = is_v ? c.v_codes : c.k_codes;
  const uint8_t* const scales = is_v ? c.v_scales : c.k_scales;
  uint8_t* const lrow = smem + (is_v ? kVRegion : 0) + lkey * kRowBytes;
  int lpos[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) lpos[j] = ((4 * lgrp + j) ^ swz(lkey)) << 4;

  struct Codes {
    uint4 c;
    uint32_t e;
  };
  auto load = [&](int t, Codes& x) {
    if (t > 0 && t % 64 == 0) load_ids(t);
    // Keys behind the last read the last one again; their logits are masked.
    int pos = c0 + t * kKeyTile + 16 * (wave & 3);
    uint32_t key = lane & 15;
    int page = __builtin_amdgcn_readlane(ids, t & 63);
    if (pos + 16 > c1) {
      const int last = c1 - 1;
      if (pos > last) {   // none of the wave's keys: the tile's first page holds one of the context
        pos = c0 + t * kKeyTile;
        page = kv4_page_in_pool(table[pos >> a.page_shift], c.n_pages);
        key = 0;
      }
      key = min((int)key, last - pos);
    }
    const size_t row = kv4_row(page, g, pos & ((1 << a.page_shift) - 1), c.Hkv, a.page_shift);
    x.c = *reinterpret_cast<const uint4*>(codes + row * kKv4RowBytes + (key * kKv4RowBytes + lgrp * 16));
    x.e = (scales + row * kKv4Scales)[key * kKv4Scales + lgrp];
  };
  auto store = [&](int t, const Codes& x) {
    uint8_t* p = lrow + (t % kStages) * kTileBytes;
    const float X = __uint_as_float(x.e << 23);
    const uint32_t w[4] = {x.c.x, x.c.y, x.c.z, x.c.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) *reinterpret_cast<uint4*>(p + lpos[j]) = dequant8(w[j], X);
  };
  auto store_tree = [&](int t) {
    const int v = min((t - n_ctx) * kKeyTile + lkey, T - 1);
    const uint4* src = reinterpret_cast<const uint4*>((is_v ? c.v_tree : c.k_tree) +
                                                      (((size_t)b * c.T_max + v) * c.Hkv + g) * kD + lgrp * 32);
    uint8_t* p = lrow + (t % kStages) * kTileBytes;
#pragma unroll
    for (int j = 0; j < 4; ++j) *reinterpret_cast<uint4*>(p + lpos[j]) = src[j];
  };
  // Tile t + 1 to its stage while tile t is computed; the codes of tiles t + 2
  // and t + 3 are in flight, those of even tiles in `even`.
  Codes even{}, odd{};
  auto advance = [&](int t, Codes& x) {
    if (t + 1 < n_ctx) {
      store(t + 1, x);
      if (t + 3 < n_ctx) load(t + 3, x);
    } else if (t + 1 < n_tiles) {
      store_tree(t + 1);
    }
  };
  auto advance_any = [&](int t) {
    if (t & 1) advance(t, even);
    else advance(t, odd);
  };
  // The same where tile t has no masked key.  Behind the context its last tile
  // is loaded again, so that the number of loads in flight does not depend on
  // a branch (the wait for a tile's codes would then be one for all).
  auto advance_plain = [&](int t, Codes& x) {
    if (t + 1 < n_ctx) store(t + 1, x);
    else if (t + 1 < n_tiles) store_tree(t + 1);
    load(min(t + 3, n_ctx - 1), x);
  };

  // ---- LDS offsets of the fragments within a stage (kh: the wave's half)
  const int half_off = (KH == 2 ? kh : 0) * 32 * kRowBytes;
  int kofs[kD / 16];
#pragma unroll
  for (int ds = 0; ds < kD / 16; ++ds)
    kofs[ds] = half_off + col * kRowBytes + (((2 * ds + half) ^ swz(col)) << 4);
  int vofs[2][kD / 32];
  v_offsets(vofs);
#pragma unroll
  for (int db = 0; db < kD / 32; ++db) {
    vofs[0][db] += half_off + kVRegion;
    vofs[1][db] += half_off + kVRegion;
  }

  Block x;
  block_init(x);
  const float sl2 = a.scale_log2, margin = (float)a.margin;

  // The wave's half h lies in tile h / HP; with KH = 1 it covers keys
  // [32*(h&1), +32) of that tile, with KH = 2 the wave's own half.  hs is h,
  // or in the unrolled loop h modulo the ring's period, a constant: every LDS
  // address is then a lane offset plus an immediate.
  constexpr int kPeriod = HP * kStages;
  auto base_of = [&](int hs) {
    return (const lds_u8*)smem + ((hs / HP) % kStages) * kTileBytes + (HP == 2 ? (hs & 1) : 0) * 32 * kRowBytes;
  };
  auto qk = [&](int hs, f32x16_t& s) {
    const lds_u8* base = base_of(hs);
    s = f32x16_t{};
#pragma unroll
    for (int ds = 0; ds < kD / 16; ++ds) {
      const bf16x8_t ka = *reinterpret_cast<const lds_bf16x8_t*>(base + kofs[ds]);
      s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ka, qf[ds], s, 0, 0, 0);
    }
  };
  auto pv = [&](int hs, const bf16x8_t (&pb)[2]) {
    const lds_u8* base = base_of(hs);
#pragma unroll
    for (int s2 = 0; s2 < 2; ++s2)
#pragma unroll
      for (int db = 0; db < kD / 32; ++db)
        x.o[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
            v_fragment(base + 16 * s2 * kRowBytes, vofs[0][db], vofs[1][db]), pb[s2], x.o[db], 0, 0, 0);
  };
  auto mask = [&](int h, f32x16_t& s) {
    const int t = h / HP, kb = 32 * (HP == 2 ? (h & 1) : kh);   // first key of the half
    if (t >= n_ctx) {
      const int k0 = (t - n_ctx) * kKeyTile;
      const uint64_t mword = valid ? s_mask[u * a.nw + (k0 >> 6)] : 0ull;
      mask_keys<true>(s, T - k0 - kb, (uint32_t)(mword >> kb));
    } else {
      mask_keys<false>(s, c1 - c0 - t * kKeyTile - kb, 0u);
    }
  };
  // Publishes the tile that was written since the last one; the stage of the
  // tile before the current one is free after it.  Loads stay in flight.
  auto tile_barrier = [&]() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); };

  if (n_ctx > 0) {
    load(0, even);
    if (n_ctx > 1) load(1, odd);
    store(0, even);
    if (n_ctx > 2) load(2, even);
  } else if (n_tiles > 0) {
    store_tree(0);
  }
  tile_barrier();
#pragma unroll
  for (int ds = 0; ds < kD / 16; ++ds)   // here, so that the first codes do not wait for the queries
    if (!valid) qf[ds] = as_bf16x8(make_uint4(0, 0, 0, 0));

  const int H = HP * n_tiles;
  const int n_plain = max(c1 - c0, 0) / kKeyTile;   // leading context tiles with no masked key
  const int H_plain = HP * n_plain;
  // A wave whose row block holds no valid row brings its share of every tile,
  // takes every barrier, and does no math.
  if (row_base + wrow * 32 >= rows) {
    for (int t = 0; t + 1 < n_tiles; ++t) {
      advance_any(t);
      tile_barrier();
    }
  } else if (H > 0) {
    f32x16_t s_cur, s_nxt;
    bf16x8_t pb[2];
    qk(0, s_cur);
    if (H_plain == 0) mask(0, s_cur);
    advance_any(0);
    if (HP == 1 && H > 1) tile_barrier();   // half 1 is in tile 1
    qk(1, s_nxt);
    softmax_step(s_cur, sl2, margin, x, pb);
    s_cur = s_nxt;
    // Half h: its softmax runs beside the products of P V of half h - 1 and of
    // S of half h + 1.  (Past the last half qk reads a stale stage; unused.)
    auto body = [&](int h, bool masked) {
      if (h % HP == 0) advance_any(h / HP);
      pv(h - 1, pb);
      if (masked) mask(h, s_cur);
      if (h % HP == HP - 1 && h + 1 < H) tile_barrier();
      qk(h + 1, s_nxt);
      softmax_step(s_cur, sl2, margin, x, pb);
      s_cur = s_nxt;
    };
    auto body_c = [&](auto J, int h) {
      constexpr int j = decltype(J)::value;
      pv((j + kPeriod - 1) % kPeriod, pb);
      if constexpr (j % HP == 0) {
        if constexpr ((j / HP) & 1) advance_plain(h / HP, even);
        else advance_plain(h / HP, odd);
      }
      // The exponentials use the reference as it stands, eight products on
      // either side of the tile barrier beside half of them each.  A weight's
      // scale costs no accuracy, so the max is not even looked for unless a lane's
      // weights of the half pass the limit: then the half is done again with the
      // reference moved.
      float psum = 0.f;
      bf16x8_t pn[2];
      exp_part(s_cur, 0, sl2, x.m, pn[0], psum);
      // Empty asm statements that consume the values pin each part to its side
      // of the barrier; otherwise both sink below the check.
      asm volatile("" ::"v"(pn[0]), "v"(psum));
      if (j % HP == HP - 1 && h + 1 < H) tile_barrier();
      qk((j + 1) % kPeriod, s_nxt);
      exp_part(s_cur, 1, sl2, x.m, pn[1], psum);
      asm volatile("" ::"v"(pn[1]), "v"(psum));
      if (__ballot(psum > a.weight_limit)) {
        rescale_to(x, reference_of(row_max(s_cur), sl2, margin));
        psum = 0.f;
        exp_part(s_cur, 0, sl2, x.m, pn[0], psum);
        exp_part(s_cur, 1, sl2, x.m, pn[1], psum);
      }
      x.l += psum;
      pb[0] = pn[0];
      pb[1] = pn[1];
      s_cur = s_nxt;
    };
    int h = 1;
    if constexpr (kPeriod == 8) {
      for (; h + 8 <= H_plain; h += 8) {   // h = 1 (mod 8) here
        body_c(std::integral_constant<int, 1>{}, h);
        body_c(std::integral_constant<int, 2>{}, h + 1);
        body_c(std::integral_constant<int, 3>{}, h + 2);
        body_c(std::integral_constant<int, 4>{}, h + 3);
        body_c(std::integral_constant<int, 5>{}, h + 4);
        body_c(std::integral_constant<int, 6>{}, h + 5);
        body_c(std::integral_constant<int, 7>{}, h + 6);
        body_c(std::integral_constant<int, 0>{}, h + 7);
      }
    } else {
      static_assert(kPeriod == 4, "one or two halves per tile, four stages");
      for (; h + 4 <= H_plain; h += 4) {   // h = 1 (mod 4) here
        body_c(std::integral_constant<int, 1>{}, h);
        body_c(std::integral_constant<int, 2>{}, h + 1);
        body_c(std::integral_constant<int, 3>{}, h + 2);
        body_c(std::integral_constant<int, 0>{}, h + 3);
      }
    }
    for (; h < H; ++h) body(h, h >= H_plain);
    pv(H - 1, pb);
  }

  // ---- epilogue: lane holds dims db*32 + 8*(r/4) + 4*half + r%4 of its query row
  float l_tot = x.l + __shfl_xor(x.l, 32, kWave);
  if constexpr (KH == 2) {
    // The wave with the other half of the keys hands its state over; each
    // state is relative to its own reference, the merged one to M.
    float4* xo = reinterpret_cast<float4*>(smem);                        // [R][16][64]
    float2* xml = reinterpret_cast<float2*>(s_mask);                     // [R][64]
    static_assert(R * 16 * 64 * 16 <= 2 * kVRegion && R * 64 <= ADAPLD_MAX_TREE_NODES * kMaskWords,
                  "the handed-over states fit");
    __syncthreads();   // no wave reads the ring or the mask any more
    if (kh == 1) {
#pragma unroll
      for (int db = 0; db < kD / 32; ++db)
#pragma unroll
        for (int r4 = 0; r4 < 4; ++r4)
          xo[(wrow * 16 + db * 4 + r4) * 64 + lane] =
              make_float4(x.o[db][4 * r4], x.o[db][4 * r4 + 1], x.o[db][4 * r4 + 2], x.o[db][4 * r4 + 3]);
      xml[wrow * 64 + lane] = make_float2(x.m, l_tot);
    }
    __syncthreads();
    if (kh == 1) return;
    const float2 ml = xml[wrow * 64 + lane];
    const float M = fmaxf(x.m, ml.x);
    const float a0 = x.m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(x.m - M);
    const float a1 = ml.x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(ml.x - M);
#pragma unroll
    for (int db = 0; db < kD / 32; ++db)
#pragma unroll
      for (int r4 = 0; r4 < 4; ++r4) {
        const float4 v = xo[(wrow * 16 + db * 4 + r4) * 64 + lane];
        x.o[db][4 * r4 + 0] = fmaf(a1, v.x, a0 * x.o[db][4 * r4 + 0]);
        x.o[db][4 * r4 + 1] = fmaf(a1, v.y, a0 * x.o[db][4 * r4 + 1]);
        x.o[db][4 * r4 + 2] = fmaf(a1, v.z, a0 * x.o[db][4 * r4 + 2]);
        x.o[db][4 * r4 + 3] = fmaf(a1, v.w, a0 * x.o[db][4 * r4 + 3]);
      }
    l_tot = fmaf(a0, l_tot, a1 * ml.y);
    x.m = M;
  }
  if (!valid) return;
  const float inv = l_tot > 0.f ? 1.f / l_tot : 0.f;   // a row without any key: 0
  if (a.nsplit == 1) {
    uint16_t* op = c.out + (((size_t)b * c.T_max + u) * c.Hq + h) * kD;
#pragma unroll
    for (int db = 0; db < kD / 32; ++db)
#pragma unroll
      for (int r4 = 0; r4 < 4; ++r4) {
        uint2 pk;
        pk.x = f32_to_bf16_bits(x.o[db][4 * r4 + 0] * inv) | (f32_to_bf16_bits(x.o[db][4 * r4 + 1] * inv) << 16);
        pk.y = f32_to_bf16_bits(x.o[db][4 * r4 + 2] * inv) | (f32_to_bf16_bits(x.o[db][4 * r4 + 3] * inv) << 16);
        *reinterpret_cast<uint2*>(op + db * 32 + 8 * r4 + 4 * half) = pk;
      }
    if (half == 0 && c.lse)
      c.lse[((size_t)b * c.Hq + h) * c.T_max + u] = l_tot > 0.f ? lse_of(a, x.m, l_tot) : -INFINITY;
  } else {
    const size_t at = ((size_t)bg * a.nsplit + split) * a.rows_max + qr;
    float* wp = a.ws_o + at * kD;
#pragma unroll
    for (int db = 0; db < kD / 32; ++db)
#pragma unroll
      for (int r4 = 0; r4 < 4; ++r4)
        *reinterpret_cast<float4*>(wp + db * 32 + 8 * r4 + 4 * half) =
            make_float4(x.o[db][4 * r4] * inv, x.o[db][4 * r4 + 1] * inv, x.o[db][4 * r4 + 2] * inv, x.o[db][4 * r4 + 3] * inv);
    if (half == 0) a.ws_ml[at] = make_float2(x.m, l_tot);
  }
}

// ------------------------------------------------------------- up to 64 rows
//
// With few rows (single tokens, one copied chain) the call is one pass over the
// cache, so waves share no keys: of the 8 waves, 8 / RB take the 32-key steps of
// the split in turn for each of RB row blocks, alone, without a barrier.  16
// rows run on 16x16x32 products, 32 and 64 in blocks of 32 on 32x32x16 ones.
//
// Lane (quad, col) brings group `quad` (16 bytes of codes, one scale) of keys col
// and 16 + col.  K codes become A fragments in registers: the order of the
// dimensions in the products is free, so a group is four fragments, and Q is
// loaded in the same order.  V codes become bf16 rows in LDS that the wave has
// for itself, from which they are read transposed.  16 keys never cross a page,
// so their page id is a scalar (a lane of a register holds it for each of the
// next 64 steps) and every address a scalar base plus a fixed lane offset.
//
// Codes of two steps are in flight, and the conversion and products S of one
// step run beside the softmax and products O of the step before it (two V
// buffers): the products then hide behind the conversions and exponentials of
// the same wave.  At the end the waves' states are merged through LDS.
constexpr int kStep = 32;
constexpr int kVBuffer = kStep * kRowBytes;   // 8 KiB

// A block of 16 rows on v_mfma_f32_16x16x32_bf16: a lane owns row `col` and the
// keys 16*i + 4*quad + r (value r of tile i), again in the order of P's operand.
struct Rows16 {
  static constexpr int kRows = 16;
  struct Logits {
    f32x4_t v[2];
  };
  typedef bf16x8_t Weights;
  float m, l;
  f32x4_t o[kD / 16];   // value r is dim 16*db + 4*quad + r
  bf16x8_t q[4];
  int vofs[kD / 16];

  __device__ __forceinline__ void init() {
    m = -INFINITY;
    l = 0.f;
    const int col = lane_id() & 15, key = 4 * (lane_id() >> 4) + (col >> 2);
#pragma unroll
    for (int db = 0; db < kD / 16; ++db) {
      o[db] = f32x4_t{};
      // 4 keys x 16 dims by each 16 lanes; the next 16 keys lie 16 rows on,
      // where the swizzle repeats
      vofs[db] = key * kRowBytes + (((2 * db + ((col & 3) >> 1)) ^ swizzle(key)) << 4) + (col & 1) * 8;
    }
  }
  static __device__ __forceinline__ int swizzle(int r) { return swz16(r); }
  static __device__ __forceinline__ int row() { return lane_id() & 15; }
  static __device__ __forceinline__ bool first_of_row() { return lane_id() < 16; }
  __device__ __forceinline__ void load_q(const uint16_t* p) {
#pragma unroll
    for (int j = 0; j < 4; ++j)
      q[j] = as_bf16x8(*reinterpret_cast<const uint4*>(p + 32 * (lane_id() >> 4) + 8 * j));
  }
  __device__ __forceinline__ void clear_q() {
#pragma unroll
    for (int j = 0; j < 4; ++j) q[j] = as_bf16x8(make_uint4(0, 0, 0, 0));
  }
  // Codes as loaded are in order: part i is group quad of key 16*i + col.
  static __device__ __forceinline__ void order_codes(uint4 (&)[2], uint32_t (&)[2]) {}
  static __device__ __forceinline__ int key_of(int i) { return 16 * i + (lane_id() & 15); }
  static __device__ __forceinline__ int dim_of(int) { return 32 * (lane_id() >> 4); }

  template <class K>
  __device__ __forceinline__ void products_s(K&& ka, Logits& s) const {
    s.v[0] = s.v[1] = f32x4_t{};
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int i = 0; i < 2; ++i) s.v[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ka(i, j), q[j], s.v[i], 0, 0, 0);
  }
  template <bool TREE>
  static __device__ __forceinline__ void mask(Logits& s, int n, uint32_t bits) {
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int key = 16 * i + 4 * (lane_id() >> 4) + r;
        s.v[i][r] = key < n && (!TREE || ((bits >> key) & 1u)) ? s.v[i][r] : -INFINITY;
      }
  }
  __device__ __forceinline__ void move_reference(const Logits& s, float sl2, float margin) {
    float mx = fmaxf(fmaxf(s.v[0][0], s.v[0][1]), s.v[0][2]);
    mx = fmaxf(fmaxf(mx, s.v[0][3]), s.v[1][0]);
    mx = fmaxf(fmaxf(mx, s.v[1][1]), s.v[1][2]);
    mx = fmaxf(mx, s.v[1][3]);
    const auto w32 = __builtin_amdgcn_permlane32_swap(__float_as_int(mx), __float_as_int(mx), false, false);
    mx = fmaxf(__int_as_float(w32[0]), __int_as_float(w32[1]));
    const auto w16 = __builtin_amdgcn_permlane16_swap(__float_as_int(mx), __float_as_int(mx), false, false);
    mx = fmaxf(__int_as_float(w16[0]), __int_as_float(w16[1]));
    const float mt = reference_of(mx, sl2, margin);
    if (__ballot(mt > m + kRescaleSlack)) {
      const float m_new = fmaxf(m, mt);
      const float alpha = m_new == m ? 1.f : __builtin_amdgcn_exp2f(m - m_new);
      m = m_new;
      l *= alpha;
#pragma unroll
      for (int db = 0; db < kD / 16; ++db) o[db] *= alpha;
    }
  }
  // The weights of a step relative to m_use; returns the lane's sum.
  static __device__ __forceinline__ float weights(const Logits& s, float sl2, float m_use, Weights& p) {
    float psum = 0.f;
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int r = 0; r < 4; r += 2) {
        const float e0 = __builtin_amdgcn_exp2f(fmaf(s.v[i][r], sl2, -m_use));
        const float e1 = __builtin_amdgcn_exp2f(fmaf(s.v[i][r + 1], sl2, -m_use));
        psum += e0 + e1;
        const bf16x2_t pk = __builtin_convertvector((f32x2_t){e0, e1}, bf16x2_t);
        p[4 * i + r] = pk[0];
        p[4 * i + r + 1] = pk[1];
      }
    return psum;
  }
  __device__ __forceinline__ void add(float psum) { l += psum; }
  struct VAhead {};
  static __device__ __forceinline__ void read_v(const lds_u8*, VAhead&) {}
  static __device__ __forceinline__ void interleave() {}
  __device__ __forceinline__ void products_o(const lds_u8* v, const VAhead&, const Weights& p) {
#pragma unroll
    for (int db = 0; db < kD / 16; ++db)
      o[db] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v_fragment(v, vofs[db], vofs[db] + 16 * kRowBytes), p, o[db], 0,
                                                      0, 0);
  }
  __device__ __forceinline__ float reference() const { return m; }
  __device__ __forceinline__ float total() const {
    const float t = l + __shfl_xor(l, 32, kWave);
    return t + __shfl_xor(t, 16, kWave);
  }
  // The lane's chunks of four dimensions, for the merge.
  template <class F>
  __device__ __forceinline__ void chunks(F&& f) const {
#pragma unroll
    for (int db = 0; db < kD / 16; ++db) f(4 * db + (lane_id() >> 4), o[db]);
  }
};

// A block of 32 rows (Block above).
struct Rows32 {
  static constexpr int kRows = 32;
  struct Logits {
    f32x16_t v;
  };
  struct Weights {
    bf16x8_t v[2];
  };
  Block x;
  bf16x8_t q[2][4];
  int vofs[2][kD / 32];

  __device__ __forceinline__ void init() {
    block_init(x);
    v_offsets(vofs);
  }
  static __device__ __forceinline__ int swizzle(int r) { return swz(r); }
  static __device__ __forceinline__ int row() { return lane_id() & 31; }
  static __device__ __forceinline__ bool first_of_row() { return lane_id() < 32; }
  // Part i of a key is its group 2 * (lane / 32) + i.
  static __device__ __forceinline__ int key_of(int) { return lane_id() & 31; }
  static __device__ __forceinline__ int dim_of(int i) { return 64 * (lane_id() >> 5) + 32 * i; }
  __device__ __forceinline__ void load_q(const uint16_t* p) {
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) q[i][j] = as_bf16x8(*reinterpret_cast<const uint4*>(p + dim_of(i) + 8 * j));
  }
  __device__ __forceinline__ void clear_q() {
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) q[i][j] = as_bf16x8(make_uint4(0, 0, 0, 0));
  }
  // From group `quad` of keys col and 16 + col to groups 2 * half + {0, 1} of key
  // lane & 31: lanes 16 apart exchange one of their two.
  static __device__ __forceinline__ void order_codes(uint4 (&k)[2], uint32_t (&e)[2]) {
    uint32_t p[5] = {k[0].x, k[0].y, k[0].z, k[0].w, e[0]}, q[5] = {k[1].x, k[1].y, k[1].z, k[1].w, e[1]};
#pragma unroll
    for (int w = 0; w < 5; ++w) {
      const auto t = __builtin_amdgcn_permlane16_swap(p[w], q[w], false, false);
      p[w] = t[0];
      q[w] = t[1];
    }
    k[0] = make_uint4(p[0], p[1], p[2], p[3]);
    k[1] = make_uint4(q[0], q[1], q[2], q[3]);
    e[0] = p[4];
    e[1] = q[4];
  }
  template <class K>
  __device__ __forceinline__ void products_s(K&& ka, Logits& s) const {
    s.v = f32x16_t{};
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) s.v = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ka(i, j), q[i][j], s.v, 0, 0, 0);
  }
  template <bool TREE>
  static __device__ __forceinline__ void mask(Logits& s, int n, uint32_t bits) {
    mask_keys<TREE>(s.v, n, bits);
  }
  __device__ __forceinline__ void move_reference(const Logits& s, float sl2, float margin) {
    const float mt = reference_of(row_max(s.v), sl2, margin);
    if (__ballot(mt > x.m + kRescaleSlack)) rescale_to(x, mt);
  }
  static __device__ __forceinline__ float weights(const Logits& s, float sl2, float m_use, Weights& p) {
    float psum = 0.f;
    exp_part(s.v, 0, sl2, m_use, p.v[0], psum);
    exp_part(s.v, 1, sl2, m_use, p.v[1], psum);
    return psum;
  }
  __device__ __forceinline__ void add(float psum) { x.l += psum; }
  // The V fragments of the first 16 keys are requested before the exponentials,
  // which hide their way through LDS.
  typedef bf16x8_t VAhead[kD / 32];
  __device__ __forceinline__ void read_v(const lds_u8* v, VAhead& f) const {
#pragma unroll
    for (int db = 0; db < kD / 32; ++db) f[db] = v_fragment(v, vofs[0][db], vofs[1][db]);
  }
  __device__ __forceinline__ void products_o(const lds_u8* v, const VAhead& f, const Weights& p) {
    VAhead g;
    read_v(v + 16 * kRowBytes, g);
#pragma unroll
    for (int db = 0; db < kD / 32; ++db)
      x.o[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f[db], p.v[0], x.o[db], 0, 0, 0);
#pragma unroll
    for (int db = 0; db < kD / 32; ++db)
      x.o[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(g[db], p.v[1], x.o[db], 0, 0, 0);
  }
  // One product to five vector instructions, so that the 16 products of a step
  // spread over its conversions (chains of 16 nodes, 32 x 4096 keys: 61.3 -> 58.6
  // us with the fragments ahead; the 16-row block does not gain).
  static __device__ __forceinline__ void interleave() {
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);
      __builtin_amdgcn_sched_group_barrier(0x2, 5, 0);
    }
  }
  __device__ __forceinline__ float reference() const { return x.m; }
  __device__ __forceinline__ float total() const { return x.l + __shfl_xor(x.l, 32, kWave); }
  template <class F>
  __device__ __forceinline__ void chunks(F&& f) const {
#pragma unroll
    for (int db = 0; db < kD / 32; ++db)
#pragma unroll
      for (int r4 = 0; r4 < 4; ++r4) {
        const f32x4_t v = {x.o[db][4 * r4], x.o[db][4 * r4 + 1], x.o[db][4 * r4 + 2], x.o[db][4 * r4 + 3]};
        f(8 * db + 2 * r4 + (lane_id() >> 5), v);
      }
  }
};

// STREAM: the codes are loaded with the non-temporal hint.
template <class ROWS, int RB, bool STREAM>
__global__ __launch_bounds__(kThreads) void kv4_narrow_kernel(const Kv4Args a) {
  constexpr int kSlices = kWaves / RB;   // waves that share a row block's keys
  __shared__ __attribute__((aligned(1024))) uint8_t smem[kWaves * 2 * kVBuffer];
  __shared__ float2 s_ml[kWaves][ROWS::kRows];
  const VerifyKv4Call& c = a.c;
  const int bg = blockIdx.x / a.nsplit, split = blockIdx.x - bg * a.nsplit;
  const int b = bg / c.Hkv, g = bg - b * c.Hkv;
  const int G = a.G;
  const int tid = threadIdx.x;
  const int lane = lane_id();
  const int wave = __builtin_amdgcn_readfirstlane(tid / kWave);
  const int slice = wave / RB, row0 = wave % RB * ROWS::kRows;
  const int col = lane & 15, quad = lane >> 4;
  const int c0 = split * a.chunk;
  const bool do_tree = split == a.nsplit - 1 && c.k_tree;

  // One memory round trip for everything that no other load decides: the
  // lengths, page ids, the queries of a full tree and its mask (what lies
  // behind the sequence's own length and nodes goes unused).  Lane j holds the
  // page ids of the two halves of the wave's step first + j.
  const int32_t* const table = c.page_table + (size_t)b * c.max_pages;
  int ids[2];
  auto load_ids = [&](int first) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int pos = c0 + (slice + (first + lane) * kSlices) * kStep + 16 * i;
      ids[i] = kv4_page_in_pool(table[min(pos >> a.page_shift, c.max_pages - 1)], c.n_pages);
    }
  };
  load_ids(0);
  const int T = min(max(c.node_count[b], 0), c.T_max);
  const int L = min(max(c.lens[b], 0), c.L_max);
  const int rows = T * G;
  const int qr = row0 + ROWS::row();
  const int qu = qr < a.rows_max ? qr / G : 0;
  const int qh = g * G + (qr < a.rows_max ? qr - qu * G : 0);
  ROWS x;
  x.load_q(c.q + (((size_t)b * c.T_max + qu) * c.Hq + qh) * kD);
  // at most 64 rows, so at most 64 nodes and one mask word
  const uint64_t sees = do_tree ? c.tree_mask[(size_t)b * c.T_max + qu] : 0ull;
  if (rows == 0) return;
  const int c1 = min(c0 + a.chunk, L);
  const int n_ctx = c1 > c0 ? (c1 - c0 + kStep - 1) / kStep : 0;

  x.init();
  const float sl2 = a.scale_log2, margin = (float)a.margin;
  uint8_t* const vrows = smem + wave * 2 * kVBuffer;
  int vpos[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) vpos[j] = col * kRowBytes + (((4 * quad + j) ^ ROWS::swizzle(col)) << 4);

  struct Raw {
    uint4 k[2], v[2];
    uint32_t ke[2], ve[2];
  };
  auto load = [&](int s, Raw& r) {
    const int k0 = c0 + s * kStep, at = ((s - slice) / kSlices) & 63;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      // Keys behind the last read the last one again; their logits are masked.
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
      const size_t row = kv4_row(page, g, pos & ((1 << a.page_shift) - 1), c.Hkv, a.page_shift);
      const uint32_t code_at = key * kKv4RowBytes + quad * 16, scale_at = key * kKv4Scales + quad;
      r.k[i] = load_codes<STREAM>(c.k_codes + row * kKv4RowBytes + code_at);
      r.v[i] = load_codes<STREAM>(c.v_codes + row * kKv4RowBytes + code_at);
      r.ke[i] = (c.k_scales + row * kKv4Scales)[scale_at];
      r.ve[i] = (c.v_scales + row * kKv4Scales)[scale_at];
    }
  };
  // Codes of step s + 2 * kSlices, once r's are used; behind the wave's last step
  // that one again, so that the number of loads in flight does not depend on
  // a branch (the wait for a step's codes would then be one for all).
  const int last = slice + (n_ctx - 1 - slice) / kSlices * kSlices;
  auto load_later = [&](int s, Raw& r) {
    const int later = min(s + 2 * kSlices, last);
    if ((later - slice) / kSlices % 64 == 0) load_ids((later - slice) / kSlices);
    load(later, r);
  };
  // V rows of a context step to buffer `buf`, and its S.
  auto begin_ctx = [&](Raw& r, int buf, typename ROWS::Logits& s) {
    uint8_t* const vb = vrows + buf * kVBuffer;
    ROWS::order_codes(r.k, r.ke);
    const float KX[2] = {__uint_as_float(r.ke[0] << 23), __uint_as_float(r.ke[1] << 23)};
    x.products_s(
        [&](int i, int j) {
          const uint32_t w[4] = {r.k[i].x, r.k[i].y, r.k[i].z, r.k[i].w};
          return as_bf16x8(dequant8(w[j], KX[i]));
        },
        s);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const float X = __uint_as_float(r.ve[i] << 23);
      const uint32_t w[4] = {r.v[i].x, r.v[i].y, r.v[i].z, r.v[i].w};
#pragma unroll
      for (int j = 0; j < 4; ++j)
        *reinterpret_cast<uint4*>(vb + 16 * i * kRowBytes + vpos[j]) = dequant8(w[j], X);
    }
  };

  {
    Raw r[2];
    typename ROWS::Logits s_cur, s_nxt;
    typename ROWS::Weights p;
    // The tree's keys come first: their rows need no page ids, so they bridge the
    // wait for the first codes.  Its (at most two) steps go to the last slices,
    // which have no more context steps than the others.
    const int tree0 = (kSlices - 1 - slice) * kStep;
    const bool has_tree = do_tree && tree0 < T;
    u32x4_t tk[2][4] = {}, tv[2][4] = {};
    if (has_tree) {
      auto row = [&](const uint16_t* p, int key) {
        return p + (((size_t)b * c.T_max + min(tree0 + key, T - 1)) * c.Hkv + g) * kD;
      };
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const u32x4_t* ks = reinterpret_cast<const u32x4_t*>(row(c.k_tree, ROWS::key_of(i)) + ROWS::dim_of(i));
        const u32x4_t* vs = reinterpret_cast<const u32x4_t*>(row(c.v_tree, col + 16 * i) + 32 * quad);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          tk[i][j] = ks[j];
          tv[i][j] = vs[j];
        }
      }
    }
    int s = slice;
    if (s < n_ctx) {
      load(s, r[0]);
      if (s + kSlices < n_ctx) load(s + kSlices, r[1]);
    }
    if (qr >= rows) x.clear_q();   // here, so that the first codes do not wait for the queries
    if (has_tree) {
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) *reinterpret_cast<u32x4_t*>(vrows + 16 * i * kRowBytes + vpos[j]) = tv[i][j];
      x.products_s([&](int i, int j) { return __builtin_bit_cast(bf16x8_t, tk[i][j]); }, s_cur);
      ROWS::template mask<true>(s_cur, T - tree0, (uint32_t)(sees >> tree0));
      x.move_reference(s_cur, sl2, margin);
      const float m = x.reference();
      x.add(ROWS::weights(s_cur, sl2, m == -INFINITY ? 0.f : m, p));
      typename ROWS::VAhead f;
      x.read_v((const lds_u8*)vrows, f);
      x.products_o((const lds_u8*)vrows, f, p);
    }
    if (s < n_ctx) {
      begin_ctx(r[0], 0, s_cur);
      x.move_reference(s_cur, sl2, margin);   // a first max (keys behind the last repeat it)
    }
    auto ctx_pair = [&](int at, Raw& rn, int buf) {   // step `at` beside the start of the next, both of the context
      const lds_u8* const v = (const lds_u8*)vrows + buf * kVBuffer;
      typename ROWS::VAhead f;
      x.read_v(v, f);
      // as in the tile kernel, the max is looked for when the weights grow
      float psum = ROWS::weights(s_cur, sl2, x.reference(), p);
      if (__ballot(psum > a.weight_limit)) {
        x.move_reference(s_cur, sl2, margin);
        psum = ROWS::weights(s_cur, sl2, x.reference(), p);
      }
      x.add(psum);
      x.products_o(v, f, p);
      begin_ctx(rn, buf ^ 1, s_nxt);
      ROWS::interleave();
      s_cur = s_nxt;
      load_later(at + kSlices, rn);
    };
    // the next two steps are of the context, so this one and the next are full
    if (s + 2 * kSlices < n_ctx) load_later(s, r[0]);
    for (; s + 2 * kSlices < n_ctx; s += 2 * kSlices) {
      // Of a SIMD's two waves the older one wins every tie and would end early,
      // with the loads of half the waves left for the rest: 32 x 8192, single tokens,
      // 42 us against 48.  So the younger goes first in every other step (47.5 ->
      // 46.8 us a call; chains of 16 nodes, 32 x 4096, 55.2 -> 54.3).
      if (wave >= kWaves / 2) __builtin_amdgcn_s_setprio(1);
      ctx_pair(s, r[1], 0);
      __builtin_amdgcn_s_setprio(0);
      ctx_pair(s + kSlices, r[0], 1);
    }
    for (int buf = 0; s < n_ctx; s += kSlices, buf ^= 1) {   // at most two steps
      if (c1 - c0 - s * kStep < kStep) ROWS::template mask<false>(s_cur, c1 - c0 - s * kStep, 0u);
      x.move_reference(s_cur, sl2, margin);
      x.add(ROWS::weights(s_cur, sl2, x.reference(), p));
      typename ROWS::VAhead f;
      x.read_v((const lds_u8*)vrows + buf * kVBuffer, f);
      x.products_o((const lds_u8*)vrows + buf * kVBuffer, f, p);
      if (s + kSlices < n_ctx) begin_ctx(r[1], buf ^ 1, s_cur);
    }
  }

  // ---- merge: every wave leaves its output where its V rows were, [row][dim]
  // with 16-byte chunks swizzled by the row, and each row is summed relative to
  // its waves' common max.
  constexpr int kMergeRows = 2 * kVBuffer / (kD * 4);   // rows of a wave's part
  static_assert(ROWS::kRows <= kMergeRows, "a wave's rows fit its own V buffers");
  float4* const xo = reinterpret_cast<float4*>(smem);   // [kWaves][kMergeRows][32]
  {
    const float l = x.total();
    const int r = ROWS::row();
    if (ROWS::first_of_row()) s_ml[wave][r] = make_float2(x.reference(), l);
    x.chunks([&](int ch, f32x4_t v) {
      xo[(wave * kMergeRows + r) * 32 + (ch ^ (r & 15))] = make_float4(v[0], v[1], v[2], v[3]);
    });
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < RB * ROWS::kRows / 16; ++i) {
    const int out_row = 16 * i + (tid >> 5), ch = tid & 31;
    if (out_row >= rows) break;
    const int rb = out_row / ROWS::kRows, r = out_row % ROWS::kRows;
    float2 ml[kSlices];
    float M = -INFINITY, l = 0.f;
#pragma unroll
    for (int w = 0; w < kSlices; ++w) {
      ml[w] = s_ml[w * RB + rb][r];
      M = fmaxf(M, ml[w].x);
    }
    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int w = 0; w < kSlices; ++w) {
      const float f = ml[w].x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(ml[w].x - M);
      const float4 y = xo[((w * RB + rb) * kMergeRows + r) * 32 + (ch ^ (r & 15))];
      l = fmaf(ml[w].y, f, l);
      v.x = fmaf(y.x, f, v.x);
      v.y = fmaf(y.y, f, v.y);
      v.z = fmaf(y.z, f, v.z);
      v.w = fmaf(y.w, f, v.w);
    }
    store_row(a, b, g, split, out_row, ch, make_float2(M, l), v);
  }
}

// Merge the splits: a row is 32 lanes of four dimensions.  Split s carries
// O_s/l_s with weight l_s 2^(m_s - M).
constexpr int kCombineThreads = 256;
constexpr int kCombineRows = kCombineThreads / 32;
template <int GROUP>
__global__ __launch_bounds__(kCombineThreads) void kv4_combine_kernel(const Kv4Args a) {
  const VerifyKv4Call& c = a.c;
  const uint32_t row = blockIdx.x * kCombineRows + threadIdx.x / 32;
  const uint32_t bg = row / (uint32_t)a.rows_max;
  const int qr = (int)(row - bg * (uint32_t)a.rows_max);
  const int b = (int)(bg / (uint32_t)c.Hkv);
  if (b >= c.B) return;
  const int nodes = c.node_count[b];
  const int dim = (threadIdx.x & 31) * 4;
  const size_t row0 = (size_t)bg * a.nsplit * a.rows_max + qr;
  // In index order, GROUP splits' loads in flight at a time.
  float M = -INFINITY, den = 0.f;
  float4 num = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int s0 = 0; s0 < a.nsplit; s0 += GROUP) {
    float2 ml[GROUP];
    float4 v[GROUP];
#pragma unroll
    for (int j = 0; j < GROUP; ++j) {
      const bool in = s0 + j < a.nsplit;
      const size_t at = row0 + (size_t)(s0 + j) * a.rows_max;
      ml[j] = in ? a.ws_ml[at] : make_float2(-INFINITY, 0.f);
      v[j] = in ? *reinterpret_cast<const float4*>(a.ws_o + at * kD + dim) : make_float4(0.f, 0.f, 0.f, 0.f);
    }
#pragma unroll
    for (int j = 0; j < GROUP; ++j) {
      if (ml[j].y > 0.f) {
        const float m_new = fmaxf(M, ml[j].x);
        const float keep = exp2f(M - m_new);   // 0 while nothing has been merged
        const float w = ml[j].y * exp2f(ml[j].x - m_new);
        num.x = fmaf(num.x, keep, w * v[j].x);
        num.y = fmaf(num.y, keep, w * v[j].y);
        num.z = fmaf(num.z, keep, w * v[j].z);
        num.w = fmaf(num.w, keep, w * v[j].w);
        den = fmaf(den, keep, w);
        M = m_new;
      }
    }
  }
  // rows past the tree are dropped only here, so the node count shares the
  // partials' memory round trip
  if (qr >= min(max(nodes, 0), c.T_max) * a.G) return;
  const int g = (int)bg - b * c.Hkv;
  const int u = qr / a.G;
  const int h = g * a.G + (qr - u * a.G);
  const float inv = den > 0.f ? 1.f / den : 0.f;
  uint2 pk;
  pk.x = f32_to_bf16_bits(num.x * inv) | (f32_to_bf16_bits(num.y * inv) << 16);
  pk.y = f32_to_bf16_bits(num.z * inv) | (f32_to_bf16_bits(num.w * inv) << 16);
  *reinterpret_cast<uint2*>(c.out + (((size_t)b * c.T_max + u) * c.Hq + h) * kD + dim) = pk;
  if (dim == 0 && c.lse)
    c.lse[((size_t)b * c.Hq + h) * c.T_max + u] = den > 0.f ? lse_of(a, M, den) : -INFINITY;
}

}  // namespace

VerifyKv4Plan plan_verify_kv4(int B, int L_max, int T_max, int Hq, int Hkv) {
  // The shape and the number of context splits with the least estimated time.
  // A workgroup (one a CU) takes a start-up and a time per unit of keys, which
  // for the 256-row shape depends on whether some SIMD has two row blocks; a
  // call takes its rounds of workgroups over the 256 CUs at their mean time, at
  // least the longest one's; a split context also the second launch and the
  // partials' traffic.  The constants (us) were fitted before the kernels' last
  // steps and read up to 36 % high; what counts is the order of the candidates,
  // which holds.  us a call inside a graph over three sets of inputs, at the choice
  // / at others: 16 x 8192 keys, 32 heads over 8, 52 nodes 256 rows in 2 splits 133
  // to 138 / 128 rows unsplit 141, in 2 154; 8 x 32768, 64 over 8, 72 nodes 256 rows
  // in 4 616 / 128 in 4 675; 4 x 2048, 40 over 8, 136 nodes 128 unsplit 46 / 256 in 2
  // 48; 1 x 4096, 32 over 8, 44 nodes 128 in 13 20.8 / in 16 20.8, in 11 20.2; 24 x
  // 6007 at most, 28 over 4, 35 nodes 256 in 2 89 / in 3 96, 128 unsplit 98; single
  // tokens, 4 x 30000, 64 over 8 in 8 29 / in 6 32; 8 x 2048, 32 over 8 in 4 11.2 /
  // in 2 12.0.
  constexpr int kCUs = 256;
  constexpr double kCombine = 5.0, kPartialBytesPerUs = 6e6;
  struct Shape {
    int rows;       // stacked rows per workgroup
    bool narrow;    // up to 64 rows: the shape that just holds them
    int unit;       // keys of a step of the workgroup
    double start, per_unit, per_unit_half;   // the latter where at most half the rows live
  };
  // Up to 64 rows the narrow shape that just holds them, us at it / at the next
  // larger one (as above): single tokens 32 x 8192 47 to 49 / 53, 1 x 4096 9.7 /
  // 10.5 (4 rows); 32 rows, 16 x 4096 24.2 / 30.5; 64 rows, 32 x 4096 56 / 76, 4 x
  // 4096 19.1 / 21.1.
  const Shape shapes[] = {{16, true, kWaves * kStep, 5.5, 1.3, 1.3},
                          {32, true, kWaves * kStep, 5.5, 2.0, 2.0},
                          {64, true, kWaves / 2 * kStep, 5.5, 1.7, 1.7},
                          {128, false, kKeyTile, 10.0, 1.12, 1.12},
                          {256, false, kKeyTile, 10.0, 1.9, 1.12}};
  const int rows_max = T_max * (Hq / Hkv);
  const int64_t pairs = (int64_t)B * Hkv;
  VerifyKv4Plan best{};
  double best_cost = 0.0;
  for (const Shape& s : shapes) {
    if (s.narrow ? rows_max > s.rows || (s.rows > 16 && rows_max <= s.rows / 2) : rows_max <= 64) continue;
    const int rowgroups = (rows_max + s.rows - 1) / s.rows;
    const bool half_last = rows_max - (rowgroups - 1) * s.rows <= s.rows / 2;
    const double longest = rowgroups == 1 && half_last ? s.per_unit_half : s.per_unit;
    const double mean = ((rowgroups - 1) * s.per_unit + (half_last ? s.per_unit_half : s.per_unit)) / rowgroups;
    const int tree = (T_max + s.unit - 1) / s.unit;
    const int units = (L_max + s.unit - 1) / s.unit;   // L_max is at most 2^30
    const int least = (int)(((int64_t)units * s.unit + kMaxChunk - 1) / kMaxChunk);
    const int most = std::max(least, std::min(64, units));
    // Of the tile shapes the last split's units include the tree's (1 x 4096, 44
    // nodes: 13 splits of 5 tiles 21.6, 16 of 4 and one more 21.9).  Of the narrow
    // ones two waves take the tree beside the others' context (counted the same
    // way, single tokens, 1 x 4096, 11.6 -> 12.7).
    const int beside = s.narrow ? tree : 0;
    for (int want = least; want <= most; ++want) {
      const int per = (units + tree - beside + want - 1) / want;   // units of a split
      const int nsplit = (units + per - 1) / per;
      if (nsplit != want && want > least) continue;   // the same split as a smaller count
      const int64_t wgs = pairs * rowgroups * nsplit;
      const double rounds = (double)((wgs + kCUs - 1) / kCUs);
      double cost = std::max(rounds * (s.start + mean * (per + beside)), s.start + longest * (per + beside));
      if (nsplit > 1)
        cost += kCombine + (double)(pairs * nsplit) * rows_max * 2 * (kD * 4 + 8) / kPartialBytesPerUs;
      if (best.rows == 0 || cost < best_cost) {
        best_cost = cost;
        best = VerifyKv4Plan{rows_max, s.rows, rowgroups, nsplit, per * s.unit};
      }
    }
  }
  return best;
}

size_t verify_kv4_ws_bytes(const VerifyKv4Plan& p, int B, int Hkv) {
  if (p.nsplit <= 1) return 0;
  return (size_t)B * Hkv * p.nsplit * p.rows_max * (kD * sizeof(float) + sizeof(float2));
}

hipError_t launch_tree_verify_attn_kv4(const VerifyKv4Call& c, const VerifyKv4Plan& p, hipStream_t stream) {
  Kv4Args a{};
  a.c = c;
  a.G = c.Hq / c.Hkv; a.rows_max = p.rows_max; a.nw = (c.T_max + 63) / 64;
  a.nsplit = p.nsplit; a.chunk = p.chunk; a.rowgroups = p.rowgroups; a.page_shift = log2_pow2(c.page_size);
  a.margin = weight_margin(c.L_max, c.T_max);
  a.weight_limit = std::ldexp(1.f, kLag - a.margin);
  a.scale_log2 = c.scale * kLog2e;
  const size_t slots = (size_t)c.B * c.Hkv * p.nsplit * p.rows_max;
  a.ws_o = static_cast<float*>(c.ws);
  a.ws_ml = c.ws ? reinterpret_cast<float2*>(static_cast<float*>(c.ws) + slots * kD) : nullptr;
  const int units = c.B * c.Hkv * p.nsplit;
  const dim3 grid((unsigned)((units + 7) / 8 * 8 * p.rowgroups));
  // A model's layers each bring their own cache, so a call finds its codes in
  // HBM; where one wave reads each of them, large ones are streamed past the
  // caches.  us a call over rotating caches, plain / non-temporal: single tokens,
  // 32 x 8192 keys of 8 kv heads (256 MiB of codes) 58.5 / 54.5, 4 x 30000 (117)
  // 35.4 / 32.5; 8 nodes, 16 x 4096 (64) 29.4 / 27.9; 8 x 2048 (16) 12.9 / 12.9.
  // Called again on the same cache, plain loads find it in the last-level cache:
  // 49.4 / 54.4, 29.4 / 30.8, 25.4 / 27.3, 10.8 / 11.3; so small ones load plainly.
  // Two row blocks read the codes twice: chains of 16 nodes, 32 x 4096 62.5 / 63.5.
  constexpr size_t kPlainBytes = (size_t)64 << 20;
  const bool stream_kv = (size_t)c.B * c.L_max * c.Hkv * 2 * kKv4RowBytes >= kPlainBytes;
  auto narrow = [&](auto rows, auto rb, auto st) {
    hipLaunchKernelGGL((kv4_narrow_kernel<decltype(rows), decltype(rb)::value, decltype(st)::value>),
                       dim3((unsigned)units), dim3(kThreads), 0, stream, a);
  };
  using One = std::integral_constant<int, 1>;
  using Two = std::integral_constant<int, 2>;
  switch (p.rows) {
    case 16:
      if (stream_kv) narrow(Rows16{}, One{}, std::true_type{});
      else narrow(Rows16{}, One{}, std::false_type{});
      break;
    case 32:
      if (stream_kv) narrow(Rows32{}, One{}, std::true_type{});
      else narrow(Rows32{}, One{}, std::false_type{});
      break;
    case 64: narrow(Rows32{}, Two{}, std::false_type{}); break;
    case 128: hipLaunchKernelGGL(kv4_verify_kernel<4>, grid, dim3(kThreads), 0, stream, a); break;
    default: hipLaunchKernelGGL(kv4_verify_kernel<8>, grid, dim3(kThreads), 0, stream, a); break;
  }
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || p.nsplit == 1) return e;
  const unsigned n_rows = (unsigned)c.B * c.Hkv * p.rows_max;
  const dim3 merge_grid((n_rows + kCombineRows - 1) / kCombineRows);
  // us a call, eight / four at a time: 2 splits 140.9 / 139.6 and 94.0 / 92.8 (registers
  // that no split fills cost waves), 16 splits 11.8 / 12.2 (more round trips).
  if (p.nsplit <= 4)
    hipLaunchKernelGGL(kv4_combine_kernel<4>, merge_grid, dim3(kCombineThreads), 0, stream, a);
  else
    hipLaunchKernelGGL(kv4_combine_kernel<8>, merge_grid, dim3(kCombineThreads), 0, stream, a);
  return hipGetLastError();
}

}  // namespace adapld
