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

#ifdef __cplusplus
}
#endif
#endif /* OPW_PAGES_H_ */
