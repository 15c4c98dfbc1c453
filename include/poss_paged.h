/*
 * poss_paged.h -- paged key/value caches, rotary positions, beam selection and token scores of the PosS library.
 *
 * The calls of poss.h work on one contiguous cache per sequence.  These work on a batch of sequences of any lengths
 * whose caches lie in pages of one pool, pages that sequences may share: tree-masked attention of all sequences in
 * one call (the verification phase of Section 2.1 for a batch; one row per sequence is plain decoding), the commit of
 * all sequences' accepted paths, forking / reordering / growing / freeing of sequences, and the selection step of a
 * beam search whose states those sequences are.  The paper has no counterpart for the pages and the beams.
 *
 * Conventions (beside those of poss.h)
 *   - Pool: kv_pages [n_layers][n_pages][2][n_kv_heads][page_slots][head_dim], contiguous, 16-byte aligned; the 2 are
 *     keys and values.  A page holds page_slots consecutive slots of one sequence, in every layer.
 *   - tables int32[batch][max_pages]: entry i of a sequence's row names the page of its slots [i * page_slots,
 *     (i + 1) * page_slots); entries behind the last page are negative.
 *   - Lengths, tables and row counts are read on the device when the kernels run: a captured graph can be replayed
 *     with new ones.
 *   - No context and no state: scratch comes from the caller, needs no initial value, and may be used again by the
 *     next call in stream order.  Calls that share scratch must not overlap on the GPU.
 *   - status (may be NULL) int32[1] on the device, sticky: a call raises it to POSS_E_INVALID when a length, a row
 *     count or a needed page is out of range, to POSS_E_TIMEOUT when a bounded wait ran out, and never lowers it.
 *     What is out of range is never followed: see each call.
 */
#ifndef POSS_PAGED_H
#define POSS_PAGED_H

#include "poss.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct {
  int n_layers, n_pages, n_kv_heads;
  int page_slots;    /* 1 .. POSS_MAX_PAGE_SLOTS */
  int head_dim;      /* 32, 64 or 128 */
  int dtype;         /* POSS_FP32 | POSS_BF16 */
} poss_page_pool;

enum { POSS_MAX_PAGE_SLOTS = 1024,
       POSS_MAX_PAGED_BATCH = 1024,     /* sequences of one call */
       POSS_MAX_ROTARY_DIM = 512 };     /* elements of a head that turn */

/* Writes the keys and values of every sequence's new rows into its pages of layer `layer`: row r of sequence b goes to
 * slot prefix_len[b] + r.  k, v [batch][rows][n_kv_heads][head_dim] (already rotated), consecutive rows ld_kv elements
 * apart (>= n_kv_heads * head_dim, a multiple of 16 bytes; sequences rows * ld_kv apart).  n_rows int32[batch] (NULL:
 * `rows` each): rows behind a sequence's n_rows are not read and write nothing.  1 <= rows <= 65535 (a prompt's chunk
 * as well as a tree).  The slots must lie in pages that no other sequence holds.  A row whose page is missing or whose
 * sequence has lengths out of range is not written (status).  Errors: INVALID, SHAPE, CAPACITY. */
POSS_API int poss_pages_append(const poss_page_pool* pool, int layer, void* kv_pages, const int32_t* tables,
                      int max_pages, int batch, int rows, const void* k, const void* v, int64_t ld_kv,
                      const int32_t* prefix_len, const int32_t* n_rows, int32_t* status, poss_stream stream);

/* ---- rotary positions
 * Pairs (u, v) of the first rot_dim (even) elements of a head turn: (u cos a - v sin a, v cos a + u sin a) * magnitude, a =
 * position * freq[i] radians for pair i < rot_dim / 2.  interleaved 0: pair i is elements i and rot_dim / 2 + i; else elements 2i and
 * 2i + 1.  Elements from rot_dim on stay as they are (magnitude does not touch them).  freq double[rot_dim / 2] on the device.
 * Any position, far and negative ones too (the latter turn back), is as exact as a near one: angles are reduced in 64 bits; cosine and
 * sine are fp32, the result is rounded once to its type.  rot_dim <= POSS_MAX_ROTARY_DIM. */

/* Frequencies of the usual schemes, on the HOST: h_freq double[rot_dim / 2], freq[i] = theta^(-2i / rot_dim), theta > 1, and for
 * contexts that are `factor` (>= 1) times longer than the original one of original_len tokens
 *   LINEAR  all divided by factor
 *   BASE    theta multiplied by factor^(rot_dim / (rot_dim - 2)) (rot_dim >= 4): the fastest stays, the slowest is divided by factor
 *   BANDS   pairs that make more than `high` turns over original_len stay, those with less than `low` are divided by factor, between
 *           them the kept share rises with the turns
 *   RAMP    the same bounds, but the kept share falls with the pair's index, between the pairs (rounded outwards) that make `high` and
 *           `low` turns
 * low, high, original_len are used by the last two (0 < low < high).  Such models often want a magnitude too (0.1 ln factor + 1).
 * Errors: INVALID, CAPACITY. */
enum { POSS_ROTARY_PLAIN = 0, POSS_ROTARY_LINEAR = 1, POSS_ROTARY_BASE = 2, POSS_ROTARY_BANDS = 3, POSS_ROTARY_RAMP = 4 };
POSS_API int poss_rotary_frequencies(double* h_freq, int rot_dim, double theta, int scaling, double factor, double low, double high,
                            double original_len);

/* Turns n rows of `heads` heads: x, out [n][heads][head_dim], consecutive rows ld_x / ld_out elements apart (>= heads * head_dim, a
 * multiple of 16 bytes), 16-byte aligned; head_dim a multiple of 16 bytes (else SHAPE), n below 2^31.  positions int32[n].  out may be
 * x (in place, ld_out = ld_x), else they do not overlap.  Errors: INVALID, SHAPE, CAPACITY. */
POSS_API int poss_rotary(const void* x, int64_t ld_x, void* out, int64_t ld_out, int dtype, int64_t n, int heads, int head_dim,
                const int32_t* positions, const double* freq, int rot_dim, int interleaved, float magnitude, poss_stream stream);

/* poss_pages_append of rows that are not rotated yet, and the rotation of their queries, in one launch: k turned into the pages, v as
 * it is, q [batch][rows][n_q_heads][head_dim] turned into out_q of the same shape (rows ld_q and ld_out_q elements apart; out_q may be
 * q; n_q_heads 0: no queries).  positions int32[batch][rows]; NULL: the slot that the row goes to.  (A tree's row sits at its prefix plus
 * its depth; after an eviction positions go on where they were and slots do not.)  out_q overlaps neither k nor v: in place, and with
 * rows ld_kv apart like theirs (a projection of all three), rows may lie between one another, but no element is of two; elsewhere it lies
 * before or behind them.  kv_pages overlaps none of the four.  All else as poss_pages_append; the queries of a row
 * whose page is missing are turned all the same, rows behind n_rows leave out_q as it was.  Errors: INVALID, SHAPE, CAPACITY. */
POSS_API int poss_pages_append_rotary(const poss_page_pool* pool, int layer, void* kv_pages, const int32_t* tables, int max_pages,
                             int batch, int rows, const void* k, const void* v, int64_t ld_kv, int n_q_heads, const void* q,
                             int64_t ld_q, void* out_q, int64_t ld_out_q, const int32_t* prefix_len, const int32_t* n_rows,
                             const int32_t* positions, const double* freq, int rot_dim, int interleaved, float magnitude,
                             int32_t* status, poss_stream stream);

/* Scratch of poss_paged_tree_attention, in bytes (0: arguments out of range).  It grows with batch, rows and
 * max_pages, so one made for the largest call serves the smaller ones. */
POSS_API size_t poss_paged_attention_workspace_bytes(const poss_page_pool* pool, int batch, int rows, int n_q_heads,
                                            int max_pages);

/* Tree-masked attention of a batch of sequences over layer `layer` of the pool, the paged form of poss_tree_attention
 * (Section 2.1, the verification phase; rows = 1: one token per sequence).
 * q [batch][rows][n_q_heads][head_dim], consecutive rows ld_q elements apart (>= n_q_heads * head_dim, a multiple of
 * 16 bytes; sequences rows * ld_q apart); out [batch][rows][n_q_heads][head_dim], contiguous.  The rows' own keys and
 * values are already in the pages (poss_pages_append).  Row r of sequence b sees slots [0, prefix_len[b]) and slot
 * prefix_len[b] + j for every bit j < n_rows[b] of anc_mask[b][r] (uint64[batch][rows][ceil(rows/64)]); query head h
 * reads KV head h / (n_q_heads / n_kv_heads).  prefix_len int32[batch]; n_rows int32[batch], 0 .. rows (NULL: `rows`
 * each).  Output rows behind n_rows[b] are left as they were; a row that sees nothing becomes zeros.  What is not seen
 * has no influence, whatever it holds (infinities and NaN too).  A missing page's slots count as unseen, a sequence
 * with lengths out of range has no rows (status).
 * out must not overlap q.  rows <= POSS_MAX_ROWS.  bf16 with head dimension 64 or 128, a page size of 16, 32, 64, 128 or
 * 256 slots, at most 128 query heads per KV head (G) and a positive scale runs on the tensor cores.  There the
 * probabilities enter the second product as the sum of two bf16 (2^-15 relative), sums and the output's accumulation are
 * fp32, scores times scale must stay below 2^29 in size (else the row is not finite), and batch * n_kv_heads *
 * ceil(rows / (2 * floor(128 / G))) * ceil(max_pages * page_slots / 64) must be below 2^31 (else CAPACITY).  How the keys
 * are cut, and so the last bits of a result, depends on the whole batch's lengths; equal calls give equal bits.
 * Errors: INVALID, SHAPE, CAPACITY, WORKSPACE (too small, not 256-byte aligned), CUDA. */
POSS_API int poss_paged_tree_attention(const poss_page_pool* pool, int layer, const void* kv_pages, const int32_t* tables,
                              int max_pages, int batch, int rows, int n_q_heads, const void* q, int64_t ld_q,
                              const int32_t* prefix_len, const int32_t* n_rows, const uint64_t* anc_mask, float scale,
                              void* out, void* workspace, size_t workspace_bytes, int32_t* status,
                              poss_stream stream);

/* ---- caches that are kept short by the attention that their slots draw
 * mass float[n_layers][batch][n_kv_heads][mass_slots], mass_slots >= max_pages * page_slots, belongs to the sequences of a batch (not to
 * pages: sequences that share pages weigh their slots each by itself; a forked sequence starts with a copy of its parent's). */

/* poss_paged_tree_attention, which also adds up the weight that each slot draws in this layer: with P the probabilities of the rows of
 * sequence b and the query heads of KV head h,
 *   W[s] = sum over rows r < n_rows[b] and those heads of row_weights[b][r] * P[s],
 *   mass[layer][b][h][s] += W[s] for s < prefix_len[b],  = W[s] for the rows' own slots prefix_len[b] <= s < prefix_len[b] + n_rows[b].
 * (The rows' slots are new: what mass held there is of no account.)  All other entries, and those of a sequence without rows, are left
 * as they were; an unseen slot draws nothing, a missing page's slots neither.  row_weights float[batch][rows] (NULL: 1 each), such as a
 * tree's draft probabilities; those behind n_rows are not read.  Terms are added in fp32, in one order: equal calls give equal bits.
 * 2^x is off by 2^-22, the maxima and sums are the attention's own.  mass must not overlap q, out or row_weights.  Scratch: calls of few
 * rows, and all off the tensor cores, keep their scores there (4 bytes per row, query head and slot that max_pages has room for, whatever the
 * lengths; where that passes 2^29 bytes none are kept and the keys are read again), so that one made for several shapes takes the greatest
 * of their sizes, which need not be that of the most rows.  All else, errors too, as poss_paged_tree_attention. */
POSS_API size_t poss_paged_attention_mass_workspace_bytes(const poss_page_pool* pool, int batch, int rows, int n_q_heads,
                                                 int max_pages);
POSS_API int poss_paged_tree_attention_mass(const poss_page_pool* pool, int layer, const void* kv_pages, float* mass,
                                   int64_t mass_slots, const int32_t* tables, int max_pages, int batch, int rows, int n_q_heads,
                                   const void* q, int64_t ld_q, const int32_t* prefix_len, const int32_t* n_rows,
                                   const uint64_t* anc_mask, const float* row_weights, float scale, void* out, void* workspace,
                                   size_t workspace_bytes, int32_t* status, poss_stream stream);

/* Cuts sequences down to their budgets: of the first seq_len[b] slots (int32[batch]) of sequence b, keep[b] (int32[batch]) stay, in
 * every layer and KV head its own: the first `first`, the last `recent`, and of those between the ones of greatest mass, ties to the
 * lower slot (-0 equals 0, NaN is below all).  They move to slots 0 .. keep[b] - 1 in their order, keys and values, and their masses to
 * out_mass (same shape; may be mass).  A sequence with seq_len[b] <= keep[b] keeps its slots (its masses are copied).  out_len int32
 * [batch] = slots that stay.  Slots and out_mass entries behind them are left as they were; poss_pages_remap gives surplus pages back.
 * Keys stay rotated as they are: positions of later rows go on.  The pages of places `first` to keep[b] - 1 are written: no other
 * sequence may hold them, none of the same call either, and a table names a page once.  poss_pages_evict takes the caller's word for it;
 * poss_pages_evict_refs looks it up in refs int32[n_pages], the holders of every page as poss_pages_remap counts them (NULL: the caller's
 * word): a sequence that would write to a page of more than one holder (a fork, a pinned prefix behind `first`) keeps its slots, as one
 * without a page that it needs.  (Forks and prefixes that are to be cut all the same: let `first` reach to the end of the shared pages, or
 * cut them before they are shared.)  A sequence with seq_len out of range, keep[b] < 0 or, where slots have to go, keep[b] < first + recent, or without
 * a page that it needs, keeps its slots and gets out_len = seq_len (status; its out_mass entries are left as they were).
 * out_mass equals mass or does not overlap it, nor refs; out_len overlaps no input.  Errors: INVALID, SHAPE, CAPACITY, WORKSPACE. */
POSS_API size_t poss_pages_evict_workspace_bytes(const poss_page_pool* pool, int batch, int max_pages);
POSS_API int poss_pages_evict(const poss_page_pool* pool, void* kv_pages, const int32_t* tables, int max_pages, int batch,
                     const float* mass, float* out_mass, int64_t mass_slots, const int32_t* seq_len, const int32_t* keep, int first,
                     int recent, int32_t* out_len, void* workspace, size_t workspace_bytes, int32_t* status, poss_stream stream);
POSS_API int poss_pages_evict_refs(const poss_page_pool* pool, void* kv_pages, const int32_t* tables, int max_pages, int batch,
                          const int32_t* refs, const float* mass, float* out_mass, int64_t mass_slots, const int32_t* seq_len,
                          const int32_t* keep, int first, int recent, int32_t* out_len, void* workspace, size_t workspace_bytes,
                          int32_t* status, poss_stream stream);

/* poss_pages_compact whose accepted slots take their masses with them: mass[..][prefix_len[b] + k] = mass[..][prefix_len[b] +
 * path[b][k]] for k = 1 .. n_accepted[b], in every layer and KV head.  (What lies behind is set by the attention that follows.) */
POSS_API int poss_pages_compact_mass(const poss_page_pool* pool, void* kv_pages, float* mass, int64_t mass_slots,
                            const int32_t* tables, int max_pages, int batch, const int32_t* prefix_len, const int32_t* path,
                            const int32_t* n_accepted, int32_t* out_len, int32_t* status, poss_stream stream);

/* Commit of a round for a batch (the paged form of poss_kv_compact): in every layer sequence b's slot prefix_len[b] +
 * path[b][k] moves to prefix_len[b] + k for k = 1 .. n_accepted[b]; out_len[b] (int32[batch]) = prefix_len[b] +
 * n_accepted[b] + 1, the slots committed then (the tree's root among them).  path int32[batch][POSS_MAX_DEPTH + 1],
 * n_accepted int32[batch]: the outputs of poss_verify_accept / poss_verify_sample, one row per sequence; path[b][k] is
 * increasing in k.  The slots must lie in pages that no other sequence holds; out_len must not overlap an input.
 * A sequence with a length, an n_accepted (0 .. POSS_MAX_DEPTH) or a path out of order or range, or without a page that it needs, keeps its slots and gets
 * out_len = prefix_len (status).  Surplus pages stay in the table: poss_pages_remap gives them back. */
POSS_API int poss_pages_compact(const poss_page_pool* pool, void* kv_pages, const int32_t* tables, int max_pages, int batch,
                       const int32_t* prefix_len, const int32_t* path, const int32_t* n_accepted, int32_t* out_len,
                       int32_t* status, poss_stream stream);

/* Scratch of poss_pages_remap and poss_pages_remap_fresh, in bytes (0: arguments out of range). */
POSS_API size_t poss_pages_remap_workspace_bytes(const poss_page_pool* pool, int n_before, int n_after, int max_pages);

/* Replaces the n_before sequences of a table by n_after new ones: reordering and forking (several sequences with one
 * parent), growing, cutting and freeing in one step.  New sequence i continues old sequence parents[i] (int32[n_after];
 * negative: starts empty; NULL: i itself, and n_after = n_before): it keeps the parent's first seq_len[parents[i]]
 * slots (int32[n_before]) and gets room for room[i] more (int32[n_after], NULL: none).  out_len[i] = slots kept.
 * refs int32[n_pages] counts the holders of every page: each old sequence gives up its pages, each new one holds the
 * ceil((kept + room) / page_slots) pages that it needs.  Pages full of kept slots are shared.  A page that the new
 * sequence will write (its kept slots' last, partly filled one and those behind) has to be its own: the new sequences
 * take these in order, and one that meets a page with other holders left takes a fresh page instead, with the kept
 * slots copied in all layers; needed pages that the parent lacks are fresh too.  Fresh pages are the lowest-numbered
 * ones without a holder (those given up by this very call included), in order of sequence and place.
 * out_tables int32[n_after][max_pages], out_refs int32[n_pages], out_len and out_free must not overlap the inputs nor each
 * other.  out_free int32[1] =
 * pages without a holder afterwards.  If fewer pages are free than needed, out_free is minus the number that is
 * missing, out_refs equals refs, out_tables, out_len and the pool are left as they were.
 * A parent >= n_before, a length or room out of range or beyond max_pages, or a table entry >= n_pages: that sequence
 * starts empty without room, that entry counts as absent (status).  Holders outside the table (a pinned prefix) are
 * counted in refs and keep their pages.
 * Errors: INVALID, SHAPE, CAPACITY, WORKSPACE, CUDA. */
POSS_API int poss_pages_remap(const poss_page_pool* pool, void* kv_pages, const int32_t* tables, int32_t* out_tables,
                     int max_pages, int n_before, int n_after, const int32_t* seq_len, const int32_t* refs,
                     int32_t* out_refs, const int32_t* parents, const int32_t* room, int32_t* out_len,
                     int32_t* out_free, void* workspace, size_t workspace_bytes, int32_t* status,
                     poss_stream stream);

/* poss_pages_remap into outputs that hold nothing yet: if fewer pages are free than needed, every entry of out_tables
 * becomes -1 and every length 0 instead of being left, so that what follows before out_free has been read finds no page
 * to write to.  (The old tables go on with refs, which out_refs equals then.)  All else, errors too, is the same. */
POSS_API int poss_pages_remap_fresh(const poss_page_pool* pool, void* kv_pages, const int32_t* tables,
                     int32_t* out_tables, int max_pages, int n_before, int n_after, const int32_t* seq_len,
                     const int32_t* refs, int32_t* out_refs, const int32_t* parents, const int32_t* room,
                     int32_t* out_len, int32_t* out_free, void* workspace, size_t workspace_bytes, int32_t* status,
                     poss_stream stream);

/* Scratch of poss_beam_select, in bytes (0: arguments out of range). */
POSS_API size_t poss_beam_select_workspace_bytes(int batch, int beams, int vocab);

/* One selection step of a beam search over `batch` groups of `beams` beams: of all continuations (beam, token) of a
 * group the `beams` best by scores[beam] + log_softmax(logits[beam])[token], best first; ties go to the lower beam,
 * then the lower token.  logits [batch][beams][vocab] of type dtype (POSS_FP32 | POSS_BF16), 16-byte aligned; scores
 * float[batch][beams], cumulative log-probabilities.  finished int32[batch][beams] (NULL: none is): a finished beam's
 * only continuation is (beam, eos) at its score as it is, its logits are not read.  A logit that is not finite bans
 * its token; a beam whose score is not finite has no continuation (a search starts with scores 0, -inf, -inf, ...).
 * out_tokens, out_parents, out_finished int32[batch][beams], out_scores float[batch][beams]: the token, the global
 * index group * beams + beam of the beam that it continues (parents for poss_pages_remap), whether it is finished now
 * (its beam was, or the token is eos; eos < 0: only the former), the new score.  With fewer continuations than beams the
 * rest is token -1, parent -1, score -inf, finished 1.  Scores are compared in 64 bits; the sum of exponentials is a sum of fp32 terms.
 * out_scores may be scores and out_finished finished (in place); the outputs overlap no input and no other output else.
 * 1 <= beams <= POSS_MAX_TOPK, eos < vocab (with `finished` given, eos >= 0).  Errors: INVALID, CAPACITY, WORKSPACE. */
POSS_API int poss_beam_select(const void* logits, int dtype, int batch, int beams, int vocab, const float* scores,
                     const int32_t* finished, int eos, int32_t* out_tokens, int32_t* out_parents, float* out_scores,
                     int32_t* out_finished, void* workspace, size_t workspace_bytes, poss_stream stream);

/* Log-probabilities of given tokens, and of each row its entropy and best tokens: what a server answers beside tokens, or scores a
 * prompt with.  p = softmax(logits[r] / temperature), temperature > 0; a logit that is not finite bans its token (p = 0).
 * logits [rows][vocab] of type dtype (POSS_FP32 | POSS_BF16), rows ld >= vocab elements apart, any alignment of their type.
 *   out_logp float[n_tokens]: of token tokens[i] (int32) in row token_rows[i] (int32; NULL: row i, n_tokens <= rows).  In a draft tree
 *     tokens are the nodes' and token_rows their parents: the target's log-probability of every node.  A token or row below 0 is
 *     none (a tree's root): 0; one that is banned, >= vocab or >= rows: -inf.  n_tokens may be 0.
 *   out_lse float[rows] (may be NULL): log of the sum of e^(logit / temperature), -inf where all are banned.
 *   out_entropy float[rows] (may be NULL): - sum p ln p, 0 where all are banned.
 *   out_top_tokens int32, out_top_logp float [rows][topk], topk 0 .. POSS_MAX_TOPK: the greatest logits, ties to the lower token, with
 *     their log-probabilities; behind the last token that is not banned -1 and -inf.
 * Logits of any finite size are safe.  Log-probabilities are never above 0.  Sums are fp32; an entropy is a difference of numbers up to some
 * 20.  Every row looks through all of token_rows: 2048 tokens over 2048 rows cost 4 us, 32768 tokens 85.  Without rows n_tokens is 0.  The
 * outputs overlap neither the inputs nor each other.  No scratch.  Errors: INVALID, CAPACITY. */
POSS_API int poss_token_logprobs(const void* logits, int64_t ld, int dtype, int rows, int vocab, float temperature,
                        const int32_t* tokens, const int32_t* token_rows, int n_tokens, float* out_logp, float* out_lse,
                        float* out_entropy, int topk, int32_t* out_top_tokens, float* out_top_logp, poss_stream stream);

#ifdef __cplusplus
}
#endif
#endif /* POSS_PAGED_H */
