/*
 * mg_kv4.h -- C ABI of the 4-bit key/value cache in libmg.so (MI355X / gfx950):
 * tokens written into it, attention that reads it, tokens evicted from it by
 * the attention weight they have gathered, and rows read back.
 *
 * Values.  A token's K row (and V row) of one head is held in groups of
 * g = min(d, 64) channels, each as 4-bit codes with a scale and a minimum:
 *
 *   min   = bf16(min x)                         (nearest even)
 *   scale = bf16((max x - min x) / 15)          (f32 difference and quotient)
 *   code  = clamp(round((x - min) / scale), 0, 15)   (nearest even; 0 where
 *                                                     the scale is 0; bf16 x:
 *                                                     the difference in f32)
 *   value = scale * code + min                  (what the cache stands for)
 *
 * A scale below 2^-126 is taken as 0.  A group that holds an infinity or NaN,
 * or whose scale or minimum is not finite, stands for NaN in all its channels.
 *
 * Layout of a cache of B sequences, H heads and room for L tokens each: four
 * regions, each starting on a 256-byte boundary; Lp = L rounded up to 32:
 *   K words   u32 [B][H][Lp][d/8]     channel c of a token: nibble c%8 (bits
 *             4(c%8)..+3) of word (c/8 % 4) * (d/32) + c/32 of its row
 *   V words   u32 [B][H][Lp/8][d]     token t: nibble t%8 of the words of row
 *             t/8; channel c at word 16 w (b / w) + w (c%16) + b % w with
 *             b = c/16 and w = min(4, d/16)
 *   K groups  u32 [B][H][Lp][max(1, d/64)]    scale's bf16 bits in the upper
 *   V groups  u32 [B][H][Lp][max(1, d/64)]    half, the minimum's in the lower
 * K's order gives a lane of a 16x16x32 matrix product its operand words in one
 * load, V's packs the eight tokens such a lane contracts over into one word.
 * A cache needs no initialization: nothing beyond the lengths given is used.
 *
 * Weights.  `weight` is f32 [B][H][L], one running sum a token: the attention
 * probabilities that query rows gave it.
 *
 * Contracts: MG_CONTRACT_FAST_BF16 (K, V, Q, O bf16) and MG_CONTRACT_STRICT_F32
 * (all f32).  Codes are exact matrix operands in every form but one, and scores are
 * exact products summed in f32.  What is rounded to f16 on the way:
 *   strict  Q, and a probability times a V scale, as two f16 parts (within 2^-23 of
 *           the f32 value)
 *   bf16    a probability times a V scale, once (2^-11); Q is exact
 *   bf16, 128 query rows a cache head and more (2^25 pairs of a row and a token, and
 *           more)  probabilities and V's values scale * code + min, each once (2^-11)
 * f16 has no more range than that: Q's rows are scaled by a power of two, and values
 * below 2^-29 (strict: 2^-17) of the row's largest are off by up to 2^-39 of it.  What
 * it means for O stands at mg_attn_fwd_kv4.  MG_CONTRACT_ACCELERATED gives exactly the
 * strict results.  LSE, weights and the workspace are f32.
 *
 * Ownership, asynchrony, errors: as for mg_attn.h.  The caller owns every
 * buffer; nothing is allocated; calls enqueue on `stream` and return;
 * arguments are checked on the host before anything is enqueued.  Pointers
 * are 16-byte aligned device memory except int32 and weight arrays (4-byte).
 * Lengths in device arrays are clamped on the device.  Outputs must not alias
 * inputs except where said.  No atomics on results: they are bitwise
 * reproducible.  Calls on one cache must be ordered by the caller (one stream,
 * or events).
 *
 * Sizes: d in {32, 64, 128}; L and n at most 2^24, B*H at most 2^19, B*H*L (L
 * rounded up to 32) at most 2^30, B*H*n at most 2^28, B*Hq*Lq*d below 2^31.
 */
#ifndef MG_KV4_H
#define MG_KV4_H

#include <stddef.h>
#include <stdint.h>

#include "mg_attn.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Bytes of a cache; 0 for sizes below 1 or that no cache has (above). */
size_t mg_kv4_cache_bytes(int B, int H, int L, int d);

/*
 * Write new tokens.  K, V [B][H][n][d]; row j < count[b] (NULL: all n) becomes
 * token start[b] + j (start NULL: 0) of sequence b.  Rows that would land
 * outside [0, L) are dropped, other tokens are left as they were.  `weight`
 * (may be NULL) is set to 0 for the tokens written.
 */
mg_status_t mg_kv4_append(const void *K, const void *V, void *cache, float *weight,
                          const int32_t *start, const int32_t *count,
                          int B, int H, int n, int L, int d,
                          mg_contract_t contract, hipStream_t stream);

/*
 * Read tokens back as the values they stand for, rounded to the contract's
 * type: K, V [B][H][n][d], row j < count[b] from token start[b] + j.  Rows
 * behind count[b] or from outside [0, L) are left as they were.
 */
mg_status_t mg_kv4_read(const void *cache, void *K, void *V,
                        const int32_t *start, const int32_t *count,
                        int B, int H, int n, int L, int d,
                        mg_contract_t contract, hipStream_t stream);

/*
 * Attention of Lq query rows a head over the cache.  Q, O [B][Hq][Lq][d], LSE
 * [B][Hq][Lq]; Hq is a multiple of H and query head hq reads cache head
 * hq / (Hq / H).  Sequence b holds key_len[b] tokens (NULL: L) and has
 * q_len[b] query rows (NULL: Lq).  Row i sees token j when
 *
 *   i < q_len[b]  and  j < key_len[b]  and
 *   (!causal or j <= i + key_len[b] - q_len[b])
 *
 * (its rows are the sequence's last tokens).  Rows that see nothing, rows at
 * or behind q_len[b] among them (whatever these hold), get O = 0 and LSE =
 * -inf.  With `weight` (may be NULL), weight[b][h][j] grows by the probabilities
 * that all rows of h's query heads give token j < key_len[b].
 *
 * In range are: |V| below 2^96 and |scale| * max |Q| * max |K| below 2^110, of the
 * tokens and of the query rows that share them; Q, K and scale may have any size
 * beside that (a scale whose product with log2 e is infinite is refused; one below
 * 2^-126 loses bits).  Beyond it results may be infinite or NaN.
 *
 * Beside errors relative to sum p |v|, O has absolute ones, from f16's range.  With the
 * largest V scale s that a row sees and its n tokens: up to 15 n 2^-35 s (strict 8 n).
 * With many bf16 rows (above): up to 2^-22 of the largest |v| that it sees, and n 2^-35
 * of it.  So a row's outputs lose bits where a token it sees has V above 2^25 times
 * (strict: 2^13) that of those that matter, whatever its own probability.  Tokens that a
 * row does not see have no part in it.  In any case: up to 2^-110.
 *
 * Sums are f32, in chains of at most 2^18 tokens (more where the workspace would pass
 * 8 GiB): terms that are all alike may drift by some 2^-11 of their sum in one.
 */
mg_status_t mg_attn_fwd_kv4(const void *Q, const void *cache, void *O, float *LSE,
                            float *weight, const int32_t *key_len, const int32_t *q_len,
                            int B, int Hq, int H, int Lq, int L, int d, int causal, float scale,
                            mg_contract_t contract,
                            void *workspace, size_t workspace_bytes, hipStream_t stream);

/*
 * Bytes of workspace for it: partial outputs of the key splits that small
 * grids and caches above 2^18 tokens are cut into and, when weights are
 * gathered, for at most 16 rows a cache head (Hq/H * Lq) their scores, for more
 * the sums of the shares that their rows are cut into.  0 also for invalid
 * arguments.
 */
size_t mg_attn_fwd_kv4_workspace_bytes(int B, int Hq, int H, int Lq, int L, int d, int weights,
                                       mg_contract_t contract);

/*
 * Cut sequences to at most `keep` tokens.  Where n = key_len[b] (NULL: L) is
 * above keep, every head keeps the last `recent` tokens (0 <= recent <= keep)
 * and, of the others, the keep - recent with the largest weight (equal weights:
 * the lower index; NaN counts as below everything), in their order.  Their rows and
 * weights move to the front of out_cache and out_weight, which are either
 * `cache` and `weight` themselves (in place) or buffers that do not overlap
 * them; what lies behind the kept tokens is left as it was.
 *   index   int32 [B][H][keep]: where each kept token was; -1 behind the last
 *   new_len int32 [B]: min(n, keep); may be key_len itself
 */
mg_status_t mg_kv4_evict(const void *cache, const float *weight,
                         void *out_cache, float *out_weight,
                         int32_t *index, int32_t *new_len, const int32_t *key_len,
                         int B, int H, int L, int d, int keep, int recent, hipStream_t stream);

#ifdef __cplusplus
}
#endif

#endif /* MG_KV4_H */
