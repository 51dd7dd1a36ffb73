/*
 * opw_prefix.h -- C ABI of decode attention for a batch whose sequences share prefixes.
 *
 * Samples of one prompt, beams, and requests behind one system prompt name the same pages in the first entries of their page-table
 * rows (opw_kv_fork makes such rows).  opw_decode_attention reads those pages once per sequence; the call below reads them once per
 * GROUP of sequences, for the queries of all of them together, and each sequence's other pages as before.
 *
 * Conventions as in opw_draft.h: plain C, status codes, DEVICE pointers are caller-owned memory on the stage's device, calls only
 * enqueue on the stream and may be made while another device is current; page ids, starts and lengths that are out of range are masked
 * out or cut off and recorded as OPW_ERR_BAD_PAGE in the stage's status word.  The kernels are launched with programmatic stream
 * serialisation (OPW_FLAG_NO_PDL at stage creation switches it off); the obligation stated at opw_decode_attention holds for kv_lens,
 * group_starts, prefix_lens and the page table.
 */
#ifndef OPW_PREFIX_H_
#define OPW_PREFIX_H_

#include "opw_attn.h"

#ifdef __cplusplus
extern "C" {
#endif

#define OPW_PREFIX_MAX_BATCH 2048
#define OPW_PREFIX_MAX_GROUPS 1024

typedef struct opw_prefix_attn opw_prefix_attn_t; /* opaque handle (host memory only) */

/* Scratch bytes of one handle (0 on invalid arguments and for stages that opw_prefix_attn_create does not take). */
size_t opw_prefix_attn_workspace_bytes(const opw_attn_stage_t *stage);

/*
 * Binds the operator to a stage (all of its layers).  flags must be 0; workspace: DEVICE, 256-byte aligned, caller-owned.  The calls of
 * one handle use its workspace one after the other: calls (or captured graphs) that may overlap on the device need a handle each.
 * The stage must outlive the handle.  A stage whose tables hold more than INT32_MAX - 128 tokens per sequence is refused
 * (OPW_ERR_UNSUPPORTED).
 */
opw_status_t opw_prefix_attn_create(opw_attn_stage_t *stage, uint32_t flags, void *workspace, size_t workspace_bytes,
                                    opw_prefix_attn_t **out);
opw_status_t opw_prefix_attn_destroy(opw_prefix_attn_t *prefix); /* NULL is accepted */

/*
 * out and lse as opw_decode_attention computes them from q, kv_lens and page_table, provided that the sequences of a group hold the same
 * pages where they say so: for group g < groups, the rows group_starts[g] .. group_starts[g + 1] - 1 name, in their first
 * prefix_lens[g] / page_size entries (whole pages only), the same pages as far as their own kv_lens reach.  Only the entries of the group's
 * longest row (the first of those) are read there, on a window layer from the first key on that any row of the group sees: that row has to hold
 * them all.  A group of one row, or with a prefix of less than a page, is fine and shares nothing;
 * rows may be shorter than their group's prefix, or inactive (kv_lens <= 0: out = 0, lse = -inf).  A group may be empty, so that a captured step can
 * have as many as it may ever need.
 * On a window layer each row sees the last W keys of its own, in the prefix and behind it.
 * Cached rows that a sequence does not see do not touch its result, whatever they hold (NaN and infinities included).  Scores, maxima, sums
 * and the accumulated output are fp32; the weights are rounded to bf16 for the product with V, not for the sum, as in opw_tree_attention; the
 * output is rounded to bf16 once.
 *   q, out     : DEVICE bf16 [batch, Hq, D], 16-byte aligned; out and lse must not overlap each other or any of the inputs
 *   kv_lens    : DEVICE int32 [batch]; beyond the table they are cut off and recorded
 *   group_starts : DEVICE int32 [groups + 1], from 0 to batch, not descending.  Other starts share nothing (the result is the same) and
 *                are recorded
 *   prefix_lens  : DEVICE int32 [groups]; negative ones count as 0
 *   page_table : DEVICE int32 [batch, max_pages_per_seq]; entries wholly before the windows of all of a group's rows are never read
 *   lse        : DEVICE float [batch, Hq] or NULL
 * groups >= 1.  batch <= max_batch, batch <= OPW_PREFIX_MAX_BATCH and groups <= OPW_PREFIX_MAX_GROUPS (OPW_ERR_CAPACITY).  Enqueues two
 * kernels.  How the keys are split depends on batch, groups, starts, lengths and the window only, never on page ids, and the result does
 * not vary from run to run.
 */
opw_status_t opw_prefix_attention(opw_prefix_attn_t *prefix, int32_t layer, int32_t batch, int32_t groups, const void *q,
                                  const int32_t *kv_lens, const int32_t *group_starts, const int32_t *prefix_lens,
                                  const int32_t *page_table, void *out, float *lse, void *cuda_stream);

#ifdef __cplusplus
}
#endif
#endif /* OPW_PREFIX_H_ */
