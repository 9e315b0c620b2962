/*
 * mg_paged.h -- C ABI of the paged key/value cache in libmg.so (MI355X /
 * gfx950): sequences brought to new lengths (block tables and slots), rows
 * written through the slots, attention of new tokens over the pages, and the
 * same over pages that a cheap score selects for each query row.
 *
 * Layout.  K and V live in two pools of N pages, [N][H][page][d], rows bf16 or
 * f32 as the contract says; page is 16, 32, 64, 128 or 256 tokens.  `table` is
 * int32 [B][P]: token j of sequence b is row j % page of page table[b][j / page].
 * Its slot is table[b][j / page] * page + j % page.  Several tables may name one
 * page.  Entries behind a sequence's last page are not read; tokens of a page
 * whose entry is not in [0, N) are not seen.  `bounds` (only for the selection)
 * is [N][H][2][d] of the pools' type: the smallest, then the largest K of every
 * page and channel.  Pools and bounds need no initialization.
 *
 * A step of a served batch, which one graph may capture:
 *   mg_paged_resize    lengths + 1: pages given back and taken, slots of the rows
 *   mg_paged_append    the step's K and V rows into their slots
 *   mg_attn_fwd_paged  attention over the pages, or
 *   mg_paged_select    the pages worth reading, and
 *   mg_attn_fwd_paged_sparse   attention over those
 *
 * Contracts: MG_CONTRACT_FAST_BF16 (K, V, Q, O and bounds bf16) and
 * MG_CONTRACT_STRICT_F32 (all f32); MG_CONTRACT_ACCELERATED gives exactly the
 * strict results.  Scores and outputs are sums of exact products in f32; with
 * bf16 a probability enters as two bf16 parts (within 2^-15 of its f32 value),
 * and O is rounded once.  LSE and the workspace are f32.  Sums are in chains of
 * at most 2^18 tokens.
 *
 * In range are sums of |Q K| below 2^127, with any scale (one whose product with
 * log2 e is infinite is refused), and n tokens of |V| below 2^127 / n (2^103 at any
 * length), as a row's weights, of which the largest is 1, are added before they are
 * divided.  Beyond that results may be infinite or NaN.
 *
 * Ownership, asynchrony, errors: as for mg_attn.h.  The caller owns every
 * buffer; nothing is allocated; calls enqueue on `stream` and return; arguments
 * are checked on the host before anything is enqueued.  Rows, pools and
 * workspaces are 16-byte aligned device memory, int32 arrays 4-byte.  Lengths
 * in device arrays are clamped on the device.  Outputs must not alias inputs
 * except where said.  No atomics on results: they are bitwise reproducible.
 * Calls on one pool must be ordered by the caller, and calls that may run at
 * the same time need workspaces of their own.
 *
 * Sizes: d in {32, 64, 128}; N*page below 2^31; P*page at most 2^24 and B*P*page
 * at most 2^35; B at most 2^16 and B*H*Lq at most 2^19; H*page*d below 2^28;
 * B*Hq*Lq*d below 2^31.  Attention that would need 2^24 workgroups is refused.
 */
#ifndef MG_PAGED_H
#define MG_PAGED_H

#include <stddef.h>
#include <stdint.h>

#include "mg_attn.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * Bring sequences from key_len[b] to want[b] tokens.  `free_pages` is a stack,
 * int32 [N], of which the first free_count[0] entries are the pages nobody
 * holds.
 *
 *   want <  key_len (0: the sequence ends): its last pages(key_len) - pages(want)
 *           table entries go on the stack, in order, where pages(n) is n / page
 *           rounded up; sequence after sequence.  (Pages that several tables
 *           name would be given back several times: leave them out of it.)
 *   want >  key_len: want - key_len rows follow those of the sequences before
 *           it: row offset[b] + j is to become token key_len[b] + j.  What pages
 *           it needs are taken from the top of the stack, after all that were
 *           given back, sequence after sequence.  It stays as it is, without
 *           slots, where want is above P*page, its rows reach behind T, or it
 *           needs pages and these, with those that the growing sequences before
 *           it need, are more than there are.
 *
 *   new_len   int32 [B]: want, or key_len where it stays; may be key_len itself
 *   new_count int32 [1]: pages left on the stack; may be free_count itself
 *   slot      int32 [T]: of every row; -1 for rows without one
 *   offset    int32 [B+1]: where a sequence's rows begin, T at most
 *   table     entries of new pages are written, others left as they were
 *
 * Lengths are clamped to [0, P*page], want to 0 and above, free_count to [0, N];
 * pages given back beyond N are lost.  B*P below 2^31, T at most 2^28.
 */
mg_status_t mg_paged_resize(const int32_t *key_len, const int32_t *want, int32_t *table,
                            int32_t *free_pages, const int32_t *free_count,
                            int32_t *new_len, int32_t *new_count, int32_t *slot, int32_t *offset,
                            int B, int page, int P, int N, int T,
                            void *workspace, size_t workspace_bytes, hipStream_t stream);
size_t mg_paged_resize_workspace_bytes(int B, int T);

/*
 * Write rows.  K, V [T][H][d]: row t goes to slot[t] of the pools Kp, Vp, or
 * nowhere where that is outside [0, N*page).  `bounds` (may be NULL): a page
 * whose first row is written holds the bounds of what this call writes to it,
 * others gone on with those and what they were.  (So they cover every token that
 * a page holds, and may cover ones that a sequence has since lost.)  NaN is left
 * out (of a channel that is NaN in all rows nothing is left: lo is the type's
 * largest value, hi the lowest, which the next rows go on from), infinities count
 * as the type's largest value.
 *
 * A slot must not occur twice in a call, and the rows of one page must follow
 * each other in `slot`, without a row of another page or one without a slot
 * between them, with rising slots, as mg_paged_resize gives them (slots may be
 * left out): otherwise which row a slot holds is not defined, nor what bounds its
 * page has.
 * T*H at most 2^28.
 */
mg_status_t mg_paged_append(const void *K, const void *V, void *Kp, void *Vp, void *bounds,
                            const int32_t *slot, int T, int H, int d, int page, int N,
                            mg_contract_t contract, hipStream_t stream);

/*
 * Attention of Lq query rows a head, the last tokens of their sequences, over
 * the pages.  Q, O [B][Hq][Lq][d], LSE [B][Hq][Lq]; Hq is a multiple of H and
 * query head hq reads cache head hq / (Hq / H).  Sequence b holds key_len[b]
 * tokens (at most P*page) and has q_len[b] query rows (NULL: Lq).  Row i sees
 * token j when
 *
 *   i < q_len[b]  and  j < key_len[b]  and
 *   (!causal or j <= i + key_len[b] - q_len[b])
 *
 * Rows that see nothing, rows at or behind q_len[b] among them (whatever these
 * hold), get O = 0 and LSE = -inf.  Tokens that a row does not see have no part
 * in it, whatever their slots hold.
 *
 * Made for one new token or a few: up to 128 of the rows that share a cache head
 * (Hq/H * Lq) are worked on at once, and the cache is read anew for the next 128.
 */
mg_status_t mg_attn_fwd_paged(const void *Q, const void *Kp, const void *Vp, void *O, float *LSE,
                              const int32_t *table, const int32_t *key_len, const int32_t *q_len,
                              int B, int Hq, int H, int Lq, int d, int page, int P, int N,
                              int causal, float scale, mg_contract_t contract,
                              void *workspace, size_t workspace_bytes, hipStream_t stream);

/*
 * Bytes of workspace for it: partial outputs of the stretches that sequences are
 * cut into.  0 also for invalid arguments.
 */
size_t mg_attn_fwd_paged_workspace_bytes(int B, int Hq, int H, int Lq, int d, int page, int P,
                                         mg_contract_t contract);

/*
 * For every query row and cache head, at most `keep` pages.  Of the m pages that
 * hold what row i sees (above), all where m <= keep; otherwise the first `first`,
 * the last `recent` and, of the others, the keep - first - recent with the
 * largest score (equal scores: the lower index; NaN counts as below everything).
 * A page's score is the largest that its bounds allow a row of the group to give
 * one of its tokens (scale > 0):
 *
 *   max over the group's heads g of  sum_c (max(Q[g][c], 0) hi[c] + min(Q[g][c], 0) lo[c])
 *
 * each sum in 64 bits, rounded to f32.  (A channel that is NaN in all of a page's
 * tokens, whose lo is the type's largest value and hi the lowest, takes the page
 * behind the others where Q[g][c] is not 0: its tokens' scores are NaN.  Bounds are
 * finite, as mg_paged_append leaves them: a sum in which 0 meets an infinite one is
 * NaN.  A page without an entry in [0, N) counts as NaN.)
 *   index  int32 [B][H][Lq][keep]: pages j / page, ascending; -1 behind the last
 * B*H*Lq*P and B*H*Lq*keep at most 2^29.
 */
mg_status_t mg_paged_select(const void *Q, const void *bounds, const int32_t *table,
                            const int32_t *key_len, const int32_t *q_len, int32_t *index,
                            int B, int Hq, int H, int Lq, int d, int page, int P, int N,
                            int causal, int keep, int first, int recent, mg_contract_t contract,
                            void *workspace, size_t workspace_bytes, hipStream_t stream);

/* Bytes of workspace for it: the scores.  0 also for invalid arguments. */
size_t mg_paged_select_workspace_bytes(int B, int Hq, int H, int Lq, int d, int page, int P,
                                       mg_contract_t contract);

/*
 * mg_attn_fwd_paged where row i of cache head h sees, of its tokens, those of
 * the pages index[b][h][i][0..keep) only.  The list ascends: an entry that is not
 * above the one before it (a repeated one) and one outside [0, P) are skipped.
 * keep*page at most 2^24.
 */
mg_status_t mg_attn_fwd_paged_sparse(const void *Q, const void *Kp, const void *Vp, void *O,
                                     float *LSE, const int32_t *table, const int32_t *index,
                                     const int32_t *key_len, const int32_t *q_len,
                                     int B, int Hq, int H, int Lq, int d, int page, int P, int N,
                                     int causal, int keep, float scale, mg_contract_t contract,
                                     void *workspace, size_t workspace_bytes, hipStream_t stream);
size_t mg_attn_fwd_paged_sparse_workspace_bytes(int B, int Hq, int H, int Lq, int d,
                                                int page, int keep, mg_contract_t contract);

#ifdef __cplusplus
}
#endif

#endif /* MG_PAGED_H */
