/*
 * adapld_kv8.h -- the paged 8-bit K/V cache of libadapld and the operators
 * around it: the norm and rotation of the queries and keys that enter it, its
 * rows, the verify attention over it (Sec. 3.6), the weight its tokens gather
 * and the eviction of those with the least.  Included by adapld.h, whose
 * conventions hold.
 */
#ifndef ADAPLD_KV8_H
#define ADAPLD_KV8_H

#include <stddef.h>
#include <stdint.h>

#include <hip/hip_runtime_api.h>

#ifdef __cplusplus
extern "C" {
#endif

/* Operation id for adapld_workspace_bytes. */
#define ADAPLD_OP_TREE_VERIFY_ATTN_KV8 10

/*
 * adapld_qk_norm_rope -- the norm of every query and key head and the rotation
 * by its token's position, in one pass: what makes the q and k_tree of the
 * verify attention, and the keys that enter a cache, from a projection's rows.
 *
 * For token u of sequence b (u < counts[b], clamped on the device to [0, T]) and
 * each head x of its q and k:
 *   y = x * w / sqrt(mean(x^2) + eps)      (y = x without that weight)
 * then, for pair i < rot_dim / 2 of dimensions (i, i + rot_dim / 2), or (2i, 2i +
 * 1) with interleaved = 1, turned by a = 2 pi * frac(p * freqs[i] / 2^64):
 *   (y1, y2) -> (y1 cos a - y2 sin a, y2 cos a + y1 sin a)
 * with the position p = base[b] + offsets[b, u], or base[b] + u without offsets
 * (the sum in 64 bits; p may be negative).  The other dimensions are y.  p * freqs
 * is exact modulo one turn, however far the position.  All of it is computed in
 * fp32 and rounded to bf16 once (a mean of squares that leaves fp32's range, as with
 * magnitudes above 2^60, or below 2^-60 where eps is 0, makes no norm).  A row's
 * infinities and NaN stay in it.
 *
 *   q, k        bf16, token u of sequence b at q + b * q_batch + u * q_token (in
 *               elements, multiples of 8): its heads [Hq, D] or [Hkv, D], dense
 *   q_weight, k_weight  bf16 [D], or NULL: no norm of that side
 *   freqs       uint64 [rot_dim / 2]: turns per position in units of 2^-64 (a
 *               negative frequency modulo 2^64); may be NULL if rot_dim is 0
 *   base        int32 [B]
 *   offsets     int32 [B, T] or NULL      e.g. a tree's node_depth
 *   counts      int32 [B] or NULL (T)     e.g. node_count
 *   rot_dim     0..D, a multiple of 16
 *   q_out       bf16 [B, T, Hq, D]  (out) rows u >= counts[b] are not written
 *   k_out       bf16 [B, T, Hkv, D] (out)
 * q_out may be q itself and k_out k, where those are dense; no other overlap.
 *
 * Errors: NULL_ARG; INVALID_ARG for B < 0, T, Hq, Hkv < 1, rot_dim outside 0..D or
 * no multiple of 16, interleaved outside {0, 1}, eps not finite or < 0, strides
 * that are negative or no multiples of 8, misaligned pointers (8 bytes for
 * freqs); UNSUPPORTED for D != 128, B * T * (Hq + Hkv) > 2^28 - 16 or B * T *
 * ceil((Hq + Hkv) / 16) > 2^26 - 4.
 */
int adapld_qk_norm_rope(const uint16_t* q, const uint16_t* k, int64_t q_batch, int64_t q_token, int64_t k_batch,
                        int64_t k_token, const uint16_t* q_weight, const uint16_t* k_weight, const uint64_t* freqs,
                        const int32_t* base, const int32_t* offsets, const int32_t* counts, int B, int T, int Hq,
                        int Hkv, int D, int rot_dim, int interleaved, float eps, uint16_t* q_out, uint16_t* k_out,
                        hipStream_t stream);

/*
 * Paged 8-bit K/V cache -- the context's K/V of the verify attention in pages
 * of a pool, at 256 bytes and an eighth per token and kv head.
 *
 * A row is one token of one kv head, for K and for V: 128 codes of 8 bits
 * (E4M3: sign, 4 bits of exponent with bias 7, 3 of fraction; no infinities,
 * 0x7f and 0xff are NaN).  The ADAPLD_KV8_BLOCK tokens of an aligned block of a
 * page share one scale byte e for each kv head, K and V apart; a value is E4M3 *
 * 2^(e - 127), exact in bf16.  e is 10..246 (adapld_kv8_append writes no other
 * byte; a block with another one reads as unspecified values).
 *
 *   k_codes, v_codes    uint8 [n_pages, Hkv, page_size, D], 16-byte aligned
 *   k_scales, v_scales  uint8 [n_pages, Hkv, page_size / ADAPLD_KV8_BLOCK]
 *   page_table          int32 [B, max_pages]: page i of sequence b holds its
 *                       positions [i * page_size, (i + 1) * page_size)
 *   page_size           16, 32, 64, 128 or 256 tokens
 * Pages, their stack and adapld_kv4_page_map are those of the 4-bit cache.
 */
#define ADAPLD_KV8_BLOCK 16

/*
 * adapld_kv8_append -- quantises new tokens' rows of K/V into the cache.
 *
 * Sequence b goes from lens_old[b] to lens_new[b] tokens (each clamped on the
 * device to [0, max_pages * page_size]; at most N are added, none if lens_new is
 * not larger).  Position lens_old[b] + i gets the Hkv rows k_new[b, r], v_new[b, r],
 * r = rows[b, i] (i itself if `rows` is NULL); for an r outside [0, n_src) zeros.
 *
 * For each block that gets rows, kv head, and K and V apart: amax is the largest
 * finite magnitude of the new rows; the least e in 10..246 with amax <= 448 *
 * 2^(e - 127) is needed.  A block whose first position is at or behind
 * lens_old[b] takes that e.  One that held tokens keeps its own or, if that is
 * less, takes the needed one, and its older rows are rounded again to the new
 * scale: exactly, but for values below 2^-6 of it.  Values are rounded once, to
 * the nearest E4M3 with ties to even; infinities and finite values above 448 *
 * 2^119 are stored as the largest value, a NaN as 0x7f, and neither changes
 * another value.
 * A block that gets rows belongs to one sequence: its page is in the table of no
 * other sequence of the call.  A block of a page id outside the pool is skipped.
 * Rows at or behind the new length are left as they are.
 *
 *   k_new, v_new  bf16 [B, n_src, Hkv, D]   the layout of k_tree, v_tree
 *   rows          int32 [B, N] or NULL      e.g. accept_nodes (NULL: N <= n_src)
 *   lens_old, lens_new  int32 [B]
 *
 * Errors: NULL_ARG; INVALID_ARG for B < 0, n_src, N, Hkv, n_pages, max_pages < 1,
 * a page_size other than the five, N > n_src without rows or misaligned pointers;
 * UNSUPPORTED for D != 128, n_pages * page_size or max_pages * page_size >
 * INT32_MAX, or more than 2^26 - 4 blocks of a kv head.
 */
int adapld_kv8_append(const uint16_t* k_new, const uint16_t* v_new, const int32_t* rows, const int32_t* lens_old,
                      const int32_t* lens_new, const int32_t* page_table, int B, int n_src, int N, int Hkv, int D,
                      int page_size, int n_pages, int max_pages, uint8_t* k_codes, uint8_t* k_scales,
                      uint8_t* v_codes, uint8_t* v_scales, hipStream_t stream);

/*
 * adapld_tree_verify_attn_kv8 -- adapld_tree_verify_attn with the context's K/V in
 * the paged 8-bit cache.
 *
 * Everything is as in adapld_tree_verify_attn_kv4 (arguments, single tokens without
 * a tree, rows without any key, which entries and rows may hold anything, what has
 * to be finite, how weights are rounded, limits and errors), but for the cache's
 * format; the workspace is that of ADAPLD_OP_TREE_VERIFY_ATTN_KV8.  Where a sequence's
 * kv head holds a NaN below its length, the results of that head are unspecified, and
 * no other's.
 */
int adapld_tree_verify_attn_kv8(const uint16_t* q, const uint8_t* k_codes, const uint8_t* k_scales,
                                const uint8_t* v_codes, const uint8_t* v_scales, const int32_t* page_table,
                                const uint16_t* k_tree, const uint16_t* v_tree, const int32_t* lens,
                                const int32_t* node_count, const uint64_t* tree_mask, int B, int L_max, int T_max,
                                int Hq, int Hkv, int D, int page_size, int n_pages, int max_pages, float scale,
                                uint16_t* out, float* lse, void* ws, size_t ws_bytes, hipStream_t stream);

/*
 * Eviction by accumulated attention weight.  A caller that bounds the cache keeps
 * for every (sequence, kv head) the weight that each cached token has got from the
 * rows so far and the token's position:
 *   weights     fp32  [B, Hkv, stride]   finite, not negative
 *   positions   int32 [B, Hkv, stride]
 * entry j belongs to the row of that kv head at position j of the page table (its
 * slot); after an eviction the kv heads of a sequence hold different tokens in the
 * same slot, and a token's place is no longer its position (rotations take the
 * position, see adapld_qk_norm_rope).  An iteration: append and attention as above,
 * adapld_kv8_attn_weights for the rows that were kept, adapld_kv8_evict, and
 * adapld_kv4_page_map from the old to the new lengths for the pages given back.
 */

/*
 * adapld_kv8_attn_weights -- adds the attention weight that new rows give.
 *
 * Sequence b holds lens_new[b] tokens (clamped on the device to [0, L_max]), the last
 * n = min(lens_new - lens_old, N) (0 if negative) of them those of the new rows: row
 * i < n has query u = rows[b, i] (i itself if `rows` is NULL) and sees the slots j <=
 * lens_old[b] + i.  For every slot j < lens_old[b] + n and kv head g:
 *   weights_out[b, g, j] = (weights[b, g, j] if j < lens_old[b], else 0)
 *     + sum over the rows i that see j, and over the Hq / Hkv heads h of g, of
 *       exp(scale * q[b, u, h] . k[b, g, j] - lse[b, h, u])
 * and positions[b, g, lens_old[b] + i] = first_position[b] + i.  Other entries are
 * left as they are.  A row whose u is outside [0, T_max) and a head whose lse is -inf
 * (a row without any key) or NaN give nothing, whatever q holds there.
 *
 *   q           bf16 [B, T_max, Hq, D]  as the attention took it
 *   lse         fp32 [B, Hq, T_max]     as the attention wrote it
 *   rows        int32 [B, N] or NULL    e.g. accept_nodes (NULL: N <= T_max)
 *   k_codes, k_scales, page_table       the cache, with the new rows' keys
 *   lens_old, lens_new, first_position  int32 [B]
 *   L_max       an upper bound of the lengths, at most max_pages * page_size and
 *               at most stride
 *   weights_out fp32 [B, Hkv, stride] (out); weights itself, or no overlap
 * Sums are fp32, in an order that the sizes fix.  For the rows and heads that give, q,
 * the keys that they see and scale * q.k * log2(e) are finite; a key that only others
 * see may be a NaN, and gets nothing.
 *
 * Errors: NULL_ARG; INVALID_ARG for B < 0, Hq % Hkv != 0, non-positive sizes, N > T_max
 * without rows, L_max > max_pages * page_size or stride, a page_size other than the
 * five, scale as in the attention, or misaligned pointers; UNSUPPORTED for D != 128,
 * T_max or N > ADAPLD_MAX_TREE_NODES, n_pages * page_size or max_pages * page_size >
 * INT32_MAX, L_max > 2^30, B * max(T_max, N) * Hq > 2^27 - 8, or B * Hkv * (L_max / 128 +
 * 1) > 2^23 - 1.
 */
int adapld_kv8_attn_weights(const uint16_t* q, const float* lse, const int32_t* rows, const uint8_t* k_codes,
                            const uint8_t* k_scales, const int32_t* page_table, const int32_t* lens_old,
                            const int32_t* lens_new, const int32_t* first_position, int B, int L_max, int T_max,
                            int N, int Hq, int Hkv, int D, int page_size, int n_pages, int max_pages, int stride,
                            float scale, const float* weights, float* weights_out, int32_t* positions,
                            hipStream_t stream);

/*
 * adapld_kv8_evict -- keeps `budget` tokens of every kv head.
 *
 * For each sequence b with L = lens[b] tokens (clamped on the device to [0, L_max])
 * and kv head: where L > budget, the tokens are ranked, those with positions[j] >=
 * next_position[b] - recent (in 64 bits) before the others, then by weight, largest
 * first, then by slot, lowest first; the first `budget` stay.  Those of them in
 * slots >= budget move into the slots < budget that the others leave, both in
 * ascending order of slots, with their rows of K and V, weight and position; the
 * rest stay where they are.  A block of the cache that rows move into takes the
 * largest scale of the rows that it then holds, and rows of smaller scales are
 * rounded again to it (exactly, but for values below 2^-6 of the scale).
 * lens_out[b] = min(L, budget), and weights_out and positions_out hold the entries
 * of the slots below that; other entries are left as they are, and so are the
 * cache's rows at or behind it.  (Made again with the same weights, positions and
 * lens, the call leaves the same cache.)
 *
 *   budget      a multiple of ADAPLD_KV8_BLOCK, >= ADAPLD_KV8_BLOCK
 *   recent      >= 0
 *   weights_out, positions_out  weights and positions themselves, or no overlap
 *   lens_out    int32 [B] (out); lens itself, or no overlap
 *   L_max       an upper bound of the lengths, at most max_pages * page_size and
 *               at most stride
 *   ws          adapld_kv8_evict_workspace_bytes(B, Hkv, L_max, budget) bytes (may
 *               be NULL if 0), 16-byte aligned
 * The pages of slots below min(L, budget) are in the table of no other sequence.  A
 * page id outside the pool is read as the nearest page, and never written.
 * Weights are compared as numbers, -0 before 0 as the smaller, a NaN by its sign as
 * the largest or the smallest.
 *
 * Errors: NULL_ARG; INVALID_ARG for B < 0, non-positive sizes, a budget as above,
 * recent < 0, L_max > max_pages * page_size or stride, a page_size other than the
 * five, or misaligned pointers; UNSUPPORTED for D != 128, n_pages * page_size or
 * max_pages * page_size > INT32_MAX, L_max > 2^30, B * Hkv > 2^22 - 1, or (where
 * L_max > budget) more than 2^26 - 4 blocks to keep of a kv head; WORKSPACE_TOO_SMALL.
 */
size_t adapld_kv8_evict_workspace_bytes(int B, int Hkv, int L_max, int budget);
int adapld_kv8_evict(const float* weights, const int32_t* positions, const int32_t* lens,
                     const int32_t* next_position, const int32_t* page_table, int B, int L_max, int budget, int recent,
                     int Hkv, int D, int page_size, int n_pages, int max_pages, int stride, uint8_t* k_codes,
                     uint8_t* k_scales, uint8_t* v_codes, uint8_t* v_scales, float* weights_out,
                     int32_t* positions_out, int32_t* lens_out, void* ws, size_t ws_bytes, hipStream_t stream);

#ifdef __cplusplus
}
#endif

#endif /* ADAPLD_KV8_H */
