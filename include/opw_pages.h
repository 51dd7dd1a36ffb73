/*
 * opw_pages.h -- C ABI for sharing and returning the pages of the stage's paged cache.
 *
 * Sequences with a common prefix (samples of one prompt, beams, a kept system prompt) need its pages only once: their
 * page-table rows name the same physical pages.  The state that goes with a page table is one reference count per
 * physical page, DEVICE int32 [num_pages], caller-owned: the number of page-table entries that name the page, 0 for a
 * free one.  A "table group" is the set of layers that share one page table; a stage whose layers all use one
 * table has one group.
 *
 * Conventions as in opw_attn.h; calls only enqueue, may be made while another device is current, and record page ids, rows and lengths
 * that are out of range as OPW_ERR_BAD_PAGE in the stage's status word.  None of these kernels releases its dependents
 * early, so that they may precede any step call that reads the table.  Counts are changed by integer atomics: results do
 * not depend on their order.
 */
#ifndef OPW_PAGES_H_
#define OPW_PAGES_H_

#include "opw_attn.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * Hands the first lens[f] tokens of table row src_rows[f] to table row dst_rows[f], for every f < n: with
 * w = lens[f] / page_size whole pages and rest = lens[f] % page_size,
 *     entries p < w of the child name the parent's pages, whose counts grow by one (an unmapped entry, < 0, stays -1),
 *     if rest > 0, entry w names new_pages[f], whose count becomes 1, and the first `rest` slots of the parent's page w
 *         are copied into it, in every layer of the group,
 *     entries behind are -1.
 * The child row must hold no pages (opw_kv_release first) and new_pages[f], where rest > 0, must be free: a count of 0, named by no
 * entry of the table.  Neither is checked.  Refused, skipped as a whole and recorded: a row outside
 * [0, num_rows), a dst row that is also a source or named twice, lens[f] < 0 or beyond the table, and, where rest > 0, a
 * parent without a page w, a new page outside the pool or named twice by forks that need one.
 *   layers     : HOST int32 [num_layers], the table group, without repetition
 *   src_rows, dst_rows, lens, new_pages : DEVICE int32 [n]
 *   page_table : DEVICE int32 [num_rows, max_pages_per_seq], changed in place
 *   refcounts  : DEVICE int32 [the smallest num_pages of the group], changed in place
 *   1 <= num_rows; n <= 65535 (OPW_ERR_CAPACITY)
 */
opw_status_t opw_kv_fork(opw_attn_stage_t *stage, const int32_t *layers, int32_t num_layers, int32_t n,
                         const int32_t *src_rows, const int32_t *dst_rows, const int32_t *lens, const int32_t *new_pages,
                         int32_t num_rows, int32_t *page_table, int32_t *refcounts, void *cuda_stream);

/*
 * Drops the pages of table rows[f] behind its first keep_lens[f] tokens (keep_lens NULL or negative: all of them): their
 * entries become -1 and their counts shrink by one.  A row named twice is dropped once, to one of its lengths' union (the
 * shortest).  A count that is already 0 stays 0 and is recorded.
 *   num_pages  : length of refcounts;  n <= 65535 (OPW_ERR_CAPACITY)
 */
opw_status_t opw_kv_release(opw_attn_stage_t *stage, int32_t n, const int32_t *rows, const int32_t *keep_lens,
                            int32_t num_rows, int32_t *page_table, int32_t *refcounts, int64_t num_pages, void *cuda_stream);

/*
 * The pages with a count of 0, in ascending order: *count gets their number, free_list its first
 * min(*count, max_list) of them; what lies behind is left as it is.
 *   refcounts  : DEVICE int32 [num_pages], num_pages <= INT32_MAX
 *   free_list  : DEVICE int32 [max_list];  count : DEVICE int32 [1]
 */
opw_status_t opw_kv_free_pages(opw_attn_stage_t *stage, const int32_t *refcounts, int64_t num_pages, int32_t *free_list,
                               int64_t max_list, int32_t *count, void *cuda_stream);

/*
 * Pages and places for the new tokens of n ragged requests, prompts and single tokens alike: request f adds new_tokens[f] = m tokens
 * behind the old_lens[f] = c that table row rows[f] holds.  What follows is all that opw_rope_append and opw_norm_rope_append need of
 * them when the requests' tokens lie one behind the other.
 *     row_starts[f] = sum of max(new_tokens[i], 0) over i < f, and row_starts[n] their total: the requests' rows
 *     entries p of the request's table row, c / page_size <= p < ceil((c + m) / page_size), that name no page (< 0) get one:
 *         the next of free_list, whose count becomes 1.  Pages are dealt in the order of the requests, and within one in that of
 *         its entries, from free_list[*free_begin] on; free_list and *free_count as opw_kv_free_pages leaves them
 *     new_lens[f] = c + m, and for the request's rows r: seq[r] = rows[f], slots[r] = c + (r - row_starts[f])
 * A request gets all that it needs or nothing: with nothing, new_lens[f] = c, its rows get seq[r] = slots[r] = -1 (padding for the calls
 * that follow), and its entries stay.  A request gets nothing
 *   - if it lacks pages, and they and those that the requests before it lack are more than the list has left: not an error;
 *   - if rows[f] < 0: not an error, the request is idle;
 *   - and is recorded, if rows[f] >= num_rows or is named by another request too, a length is negative, c + m is beyond the table, its rows end
 *     beyond max_rows, or (m > 0; the table is not looked at for less) the page that holds its last c % page_size tokens is missing, or one of
 *     the entries that its tokens go to names a page outside [0, num_pages) or one whose count is not 1 (its tokens would show up in
 *     other sequences).
 * Requests that are refused or idle take nothing from the list; those for whom it was too short come after all that were served
 * from it.  An id of the list that is out of range or not free (a list that is out of date) is not dealt: its entry stays as it
 * is, and it is recorded.  An id that the list names twice is dealt once and recorded; which of the two entries gets it may vary.
 *   rows, old_lens, new_tokens : DEVICE int32 [n]
 *   page_table : DEVICE int32 [num_rows, max_pages_per_seq];  refcounts : DEVICE int32 [num_pages]; both changed in place
 *   free_list  : DEVICE int32 [max_list];  free_count : DEVICE int32 [1]: the list's length is min(*free_count, max_list)
 *   free_begin : DEVICE int32 [1] or NULL (0; so is a negative one): where dealing begins
 *   free_end   : DEVICE int32 [1] or NULL: where it ended; may be free_begin, which makes that a cursor through one list
 *   row_starts : DEVICE int32 [n + 1] or NULL; starts beyond max_rows count as max_rows
 *   new_lens   : DEVICE int32 [n] or NULL
 *   seq, slots : DEVICE int32 [max_rows]; rows behind the last request's get -1, so that a captured step may have more rows than
 *                tokens.  max_rows = -1: NULL both, no rows are placed, and only rows beyond INT32_MAX are too many
 * What is written must not overlap what is read, nor each other.  n <= 8192 and num_rows <= 262144 (OPW_ERR_CAPACITY).
 */
opw_status_t opw_kv_extend(opw_attn_stage_t *stage, int32_t n, const int32_t *rows, const int32_t *old_lens, const int32_t *new_tokens,
                           int32_t num_rows, int32_t *page_table, int32_t *refcounts, int64_t num_pages, const int32_t *free_list,
                           int64_t max_list, const int32_t *free_count, const int32_t *free_begin, int32_t *free_end,
                           int32_t *row_starts, int32_t *new_lens, int32_t max_rows, int32_t *seq, int32_t *slots, void *cuda_stream);

#ifdef __cplusplus
}
#endif
#endif /* OPW_PAGES_H_ */
