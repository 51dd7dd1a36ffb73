/*
 * opw_draft.h -- C ABI of the operators that verify drafted tokens on the attention stage.
 *
 * A server that drafts several tokens ahead and verifies them in one pass sends the stage, per
 * sequence, not one query but the queries of a whole TREE of drafted tokens (a chain is the
 * simplest one): node i of the tree continues the committed context by the path from the root
 * to i, and attends to the context and to its own ancestors.  One step of one layer is
 *     opw_rope_append      rotate the nodes' queries and keys, append keys and values to the
 *                          cache, node i of sequence b in slot ctx[b] + i
 *     opw_tree_attention   every node against the context and the nodes its mask names
 * and, once the step's logits have decided which path is accepted,
 *     opw_kv_commit        move the accepted nodes' cached rows together, in slots ctx[b],
 *                          ctx[b] + 1, ..., of all layers that share a page table
 * after which the sequence is an ordinary one again (opw_decode_step may follow).
 * opw_rope_append also takes prompts into the cache: its rows are any tokens of any sequences.
 *
 * These calls are no plan items and no part of opw_decode_step_host or of the attention module (opw_afd.h); a caller who wants
 * one submission per step captures them into a CUDA graph of its own.  Layers with recurrent state (opw_linear_attn.h) have no
 * form for drafted tokens: their state cannot be advanced along a tree nor taken back, so that in a hybrid stack these calls
 * serve the attention layers only.
 *
 * Conventions as in opw_attn.h: plain C, status codes, DEVICE pointers are caller-owned memory
 * on the stage's device, calls only enqueue on the stream and never synchronise.  The calls may
 * be made while another device is current.  Page ids and positions that are out of range are
 * skipped or masked out and recorded as OPW_ERR_BAD_PAGE in the stage's status word
 * (opw_attn_stage_poll_error).  The kernels are launched with programmatic stream serialisation
 * like the stage's own (OPW_FLAG_NO_PDL at stage creation switches it off), and the obligation
 * stated at opw_decode_attention holds for ctx_lens, tree_lens, tree_mask, positions and the page
 * table of opw_tree_attention; opw_kv_commit, which writes lengths, never releases its dependents
 * early.
 */
#ifndef OPW_DRAFT_H_
#define OPW_DRAFT_H_

#include "opw_attn.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ------------------------------------------------------------------------------------------
 * Rotary encoding and append
 * ------------------------------------------------------------------------------------------ */

#define OPW_ROPE_HALF 0        /* pair i is (x_i, x_{i + r/2}), r = rotary_dim */
#define OPW_ROPE_INTERLEAVED 1 /* pair i is (x_{2i}, x_{2i + 1}) */

/* How the frequencies are changed for contexts longer than the model was trained on; f_i = theta^(-2i/r):
 *   PLAIN   f_i
 *   LINEAR  f_i / factor
 *   NTK     theta replaced by theta * factor^(r / (r - 2))   (r > 2)
 *   BANDS   by the number of turns t_i = original_context * f_i / (2 pi): f_i / factor below `low`,
 *           f_i above `high`, linear in t_i between   (low 0 -> 1, high 0 -> 4)
 *   YARN    f_i / factor * w_i + f_i * (1 - w_i), w_i rising linearly in i from 0 to 1 between the
 *           (rounded) indices whose pair makes `high` and `low` turns over original_context
 *           (low 0 -> 1, high 0 -> 32); the amplitude defaults to 1 + 0.1 ln(factor) */
#define OPW_ROPE_PLAIN 0
#define OPW_ROPE_LINEAR 1
#define OPW_ROPE_NTK 2
#define OPW_ROPE_BANDS 3
#define OPW_ROPE_YARN 4

typedef struct {
  uint32_t struct_size;     /* sizeof(opw_rope_config_t) */
  int32_t rotary_dim;       /* r: even, 2..256; the head's first r elements are rotated, the rest pass */
  int32_t scaling;          /* OPW_ROPE_PLAIN .. OPW_ROPE_YARN */
  int32_t reserved;         /* must be 0 */
  double theta;             /* > 1 (e.g. 10000) */
  double factor;            /* >= 1; read unless PLAIN */
  double original_context;  /* > 0; read by BANDS and YARN */
  double low, high;         /* 0 -> the defaults above; 0 < low < high */
  double amplitude;         /* factor on the rotated values; 0 -> 1, or YARN's default */
} opw_rope_config_t;

/*
 * Host helper: fills table_host, rotary_dim / 2 + 1 doubles: the turns per position f_i / (2 pi) of each
 * pair, then the amplitude.  The caller copies it to the device once and hands it to opw_rope_append.
 * In 64 bits because position * f_i is: a 32-bit angle is off by 1e-7 of itself, 0.1 radians at a position of 1e6.
 */
opw_status_t opw_rope_table(const opw_rope_config_t *cfg, double *table_host);

/*
 * For every token row r < rows with seq[r] >= 0: rotates the heads of q[r] and k[r] at positions[r],
 *     pair (a, b) -> amplitude * (a cos - b sin, b cos + a sin),   angle = positions[r] * f_i,
 * stores the rotated queries to q_out[r] and appends the rotated keys and the values to slot slots[r] of
 * sequence seq[r]'s cache (page_table row seq[r]).  Angles are reduced in 64 bits, the rotation is fp32,
 * rounded to bf16 once.  Rows with seq[r] < 0 are padding: nothing is read or written for them.  A slot
 * outside the table or a bad page id skips that row's append (its query is still rotated); so does a
 * seq[r] >= num_rows.  Two rows of one call must not name the same (seq, slot).
 *   rotary_dim, layout : as in the table; rotary_dim <= head_dim.  OPW_ROPE_HALF or OPW_ROPE_INTERLEAVED
 *   table      : DEVICE double [rotary_dim / 2 + 1] from opw_rope_table, 8-byte aligned
 *   q, k, v    : DEVICE bf16; row r of q starts at q + r * q_stride and holds [Hq, D] (k, v: [Hkv, D]).  Strides in
 *                elements, multiples of 8, at least a row's length (views into one packed projection are fine);
 *                16-byte aligned
 *   q_out      : DEVICE bf16 [rows, Hq, D], 16-byte aligned; may be q itself if q_stride == Hq * D, must not
 *                overlap q in any other way, nor any other input; q == q_out == NULL: keys and values only
 *   seq, slots, positions : DEVICE int32 [rows]
 *   page_table : DEVICE int32 [num_rows, max_pages_per_seq], num_rows >= 1
 */
opw_status_t opw_rope_append(opw_attn_stage_t *stage, int32_t layer, int32_t rows, int32_t rotary_dim, int32_t layout,
                             const double *table, const void *q, int64_t q_stride, const void *k, int64_t k_stride,
                             const void *v, int64_t v_stride, const int32_t *seq, const int32_t *slots,
                             const int32_t *positions, int32_t num_rows, const int32_t *page_table, void *q_out,
                             void *cuda_stream);

/* ------------------------------------------------------------------------------------------
 * Attention of a tree of drafted tokens
 * ------------------------------------------------------------------------------------------ */

#define OPW_TREE_MAX_NODES 64

typedef struct opw_tree_attn opw_tree_attn_t; /* opaque handle (host memory only) */

/*
 * Host helper for trees whose shape is fixed: parents[i] < i is node i's parent, -1 for a node that
 * continues the committed context directly.  mask[i] gets the bits of i and its ancestors, depth[i] (may
 * be NULL) their number less one, so that node i's position is ctx + depth[i].  INVALID_ARG if a parent
 * does not come before its child.  1 <= nodes <= OPW_TREE_MAX_NODES.
 */
opw_status_t opw_tree_mask(int32_t nodes, const int32_t *parents, uint64_t *mask, int32_t *depth);

/* Scratch bytes of one handle (0 on invalid arguments and for stages that opw_tree_attn_create does not take). */
size_t opw_tree_attn_workspace_bytes(const opw_attn_stage_t *stage, int32_t max_nodes);

/*
 * Binds tree attention to a stage (all of its layers).  max_nodes in 1..OPW_TREE_MAX_NODES; flags must be 0;
 * workspace: DEVICE, 256-byte aligned, caller-owned.  The calls of one handle use its workspace one after the
 * other: calls (or captured graphs) that may overlap on the device need a handle each.  The stage must outlive
 * the handle.  A stage whose tables hold more than INT32_MAX - 128 tokens per sequence is refused (OPW_ERR_UNSUPPORTED).
 */
opw_status_t opw_tree_attn_create(opw_attn_stage_t *stage, int32_t max_nodes, uint32_t flags, void *workspace,
                                  size_t workspace_bytes, opw_tree_attn_t **out);
opw_status_t opw_tree_attn_destroy(opw_tree_attn_t *tree); /* NULL is accepted */

/*
 * For every sequence b < batch with c = ctx_lens[b] >= 0 and t = tree_lens[b] > 0, node i < t and query head h:
 *     out[b,i,h,:] = sum_j softmax_j(scale * <q[b,i,h,:], K_j[h/G,:]>) V_j[h/G,:]      (lse as in opw_decode_attention)
 * over the cached rows j that node i sees:
 *     the context, j < c, and
 *     the drafted rows j = c + m, m < t, with bit m of tree_mask[b,i] set (its own bit is not implied),
 * on a window layer (window W) only those whose position is above p_i - W, where the position of context row j is j, that
 * of drafted row c + m is positions[b,m], and p_i = positions[b,i] (a position below c counts as c).  Cached
 * rows that a node does not see do not touch its result, whatever they hold (NaN and infinities included).  An infinite value that it
 * does see leaves an infinity or a NaN (either, where its weight is below what fp32 holds).
 * Scores, maxima, sums and the accumulated output are fp32.  The weights p_j = 2^(score - running maximum) are rounded to bf16 for the
 * product with V -- not for the sum -- as the decode kernels do, which moves an output by at most 2^-8 sum_j p_j |V_j| / sum_j p_j;
 * the output is rounded to bf16 once.
 * A node that sees nothing, nodes i >= t and inactive sequences (c < 0 or t <= 0) get out = 0, lse = -inf.
 * t > nodes, rows beyond the table and bad page ids are cut off or masked out and recorded as OPW_ERR_BAD_PAGE.
 *   nodes      : 1..max_nodes, the row stride of q, tree_mask, positions, out and lse
 *   q, out     : DEVICE bf16 [batch, nodes, Hq, D], 16-byte aligned; out and lse must not overlap each other or any of the inputs
 *   tree_mask  : DEVICE uint64 [batch, nodes], 8-byte aligned
 *   positions  : DEVICE int32 [batch, nodes]; read on window layers only
 *   ctx_lens, tree_lens : DEVICE int32 [batch]
 *   page_table : DEVICE int32 [batch, max_pages_per_seq]; entries wholly before the window are never read
 *   lse        : DEVICE float [batch, nodes, Hq] or NULL
 * batch <= max_batch and <= 4096 (OPW_ERR_CAPACITY).  Enqueues two kernels.  The split of the keys depends on the
 * lengths and the window only, never on page ids, and the result does not vary from run to run.
 */
opw_status_t opw_tree_attention(opw_tree_attn_t *tree, int32_t layer, int32_t batch, int32_t nodes, const void *q,
                                const uint64_t *tree_mask, const int32_t *positions, const int32_t *ctx_lens,
                                const int32_t *tree_lens, const int32_t *page_table, void *out, float *lse,
                                void *cuda_stream);

/* ------------------------------------------------------------------------------------------
 * The accepted path
 * ------------------------------------------------------------------------------------------ */

/*
 * For every sequence b < batch and every layer in layers[0..num_layers): with c = ctx_lens[b] >= 0 and
 * m = accepted_lens[b], cached row c + i takes what row c + accepted[b,i] held before the call, for i < m, bit for
 * bit, keys and values of all heads.  (A gather: accepted may name a row twice; an accepted path lists ascending
 * nodes.)  Rows from c + m on are left as they are.  new_lens[b] = c + m (c where c < 0; m < 0 counts as 0).  An accepted
 * node outside [0, nodes) or a bad page skips its row (a row that is in place already has its page looked at too), m > nodes is
 * cut to nodes; both are recorded.  new_lens counts skipped rows all the same.
 *   layers     : HOST int32 [num_layers], layers that share the page table, without repetition
 *   accepted   : DEVICE int32 [batch, nodes], 1 <= nodes <= OPW_TREE_MAX_NODES
 *   accepted_lens, ctx_lens : DEVICE int32 [batch]
 *   new_lens   : DEVICE int32 [batch] or NULL; must not overlap any of the inputs
 * Sequences must not share the pages of their drafted rows (they never do while only whole, full pages are shared).
 */
opw_status_t opw_kv_commit(opw_attn_stage_t *stage, const int32_t *layers, int32_t num_layers, int32_t batch, int32_t nodes,
                           const int32_t *accepted, const int32_t *accepted_lens, const int32_t *ctx_lens,
                           const int32_t *page_table, int32_t *new_lens, void *cuda_stream);

#ifdef __cplusplus
}
#endif
#endif /* OPW_DRAFT_H_ */
