/*
 * rocs_history.h - C ABI of librocs, part two: attention of a request's own
 * rows over its history, over packed K/V or over a cache that keeps the
 * histories' K/V in pages between calls, and the operators that keep the
 * pages of that cache. Conventions, types and error reporting are those of
 * rocs.h (device pointers, caller-owned memory, status codes, nothing is
 * synchronised or allocated).
 *
 * The mask and score rules of both attentions
 *   Request r has n_r = q_offsets[r+1] - q_offsets[r] query rows and a history
 *   of L_r keys; its query rows are the last n_r of the history: row i stands
 *   at position p = L_r - n_r + i (a row whose position is negative sees no
 *   key under the causal mask but the prefix). Head h reads K/V head
 *   h / (num_heads / kv_heads). For key j (0 <= j < L_r), in this order:
 *     s_j  = scale * <q, k_j>             scale <= 0: 1/sqrt(head_dim)
 *     s_j  = cap * tanh(s_j / cap)        cap > 0 only
 *     s_j -= slopes[h] * |p - j|          slopes non-NULL only
 *   key j is seen iff  (not causal, or j <= p, or j < prefix_lens[r])
 *                 and  (no documents, or q_docs[row] == kv_docs[key])
 *   out  = sum over seen j of softmax(s)_j * v_j.
 *   A row that sees no key (or whose seen scores are all -inf) is zero. Keys
 *   that a row does not see have no part in it, whatever they hold: infinities
 *   and NaN there do not reach the row.
 *   Infinities and NaN in V cost time (in q and K too, at head_dims that are
 *   not the kernels' own 64 and 128): a row whose tile meets one is formed again
 *   by a slow path, 200 to 600 times a long call's time where all rows do.
 *   Scores, softmax and sums are fp32; the bf16 kernels round the softmax
 *   weights to bf16 for the product with V and sum the rounded weights. Their
 *   cap adds an error of at most 2^-22 cap to a score for caps up to 128, and of
 *   2^-19 of the score itself for larger ones (which take more instructions).
 */
#ifndef ROCS_HISTORY_H
#define ROCS_HISTORY_H

#include "rocs.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * ---------------------------------------------------------------------------
 * rocs_history_attention: packed histories.
 *
 *   q            [N, num_heads, head_dim], rows q_row_stride elements apart
 *                (0: dense); the queries of request r are rows q_offsets[r] ..
 *   k, v         [num_kv_rows, kv_heads, head_dim], rows kv_row_stride
 *                elements apart (0: dense); request r's keys are rows
 *                kv_offsets[r] .. kv_offsets[r+1]-1. q, k and v may be column
 *                slices of one projection output.
 *   q_offsets, kv_offsets [R + 1] int32 (the same array for whole histories)
 *   prefix_lens  [R] int32 or NULL: the first prefix_lens[r] keys are seen by
 *                every row of r (causal only; values outside 0 .. L_r act as
 *                the nearest of the two)
 *   q_docs [N], kv_docs [num_kv_rows] int32, both or neither: a row sees only
 *                keys of its own document. Documents may come in any order;
 *                stretches of 64 keys without a document of the tile's rows
 *                are passed over, which is fast where documents are contiguous.
 *   slopes       [num_heads] fp32 or NULL;  cap 0 (none) or at least 1e-30
 *   causal       0 or 1
 *   max_kv_len   an upper bound on every L_r, known on the host, or 0 for
 *                num_kv_rows: it only decides how a long history is split over
 *                workgroups (the results' fp32 sums follow that split)
 *   out          [N, num_heads, head_dim], dense, not overlapping an input;
 *                rows past q_offsets[R] (a padded batch) stay as they are
 *   workspace    at least rocs_history_workspace_size(R, N, num_heads,
 *                kv_heads, head_dim, max_kv_len or num_kv_rows, dtype) bytes,
 *                256-byte aligned; may be NULL when that is 0. Scratch.
 *                That size is the one call's: fewer requests, rows or keys may
 *                need more (they are cut into more parts). One workspace for
 *                calls of many sizes takes the largest of theirs, or
 *                  4 (head_dim + 2) min(num_heads N P, C) + 512 bytes,
 *                  P = min(256, ceil(max_kv_len / 256)),
 *                  C = 524,288 (bf16 and head_dim a multiple of 8 up to 128)
 *                      or 8,192 (all others),
 *                which is enough for any number of requests and up to N rows
 *                and max_kv_len keys.
 *
 * Fast path (bf16 MFMA kernels): bf16, head_dim a multiple of 8 up to 128
 * (fastest at 64 and 128), strides multiples of 8 elements, pointers 16-byte
 * aligned. Other cases run a general kernel (fp32 matrix instructions),
 * head_dim up to 256. One kernel and one cut of the histories serve a whole
 * call, by the average rows of a request and the bound on the lengths: single
 * rows beside long chunks, or one very long history beside many short ones, are
 * faster as calls of their own.
 * Limits: N * num_heads <= 2^30, num_heads < 2^16, num_kv_rows <= 2^31 - 4096,
 * and fewer than 2^24 workgroups (of 128, 32 or, in the general kernel, 16 rows
 * of one request and K/V head, times the parts that histories are cut into).
 * ---------------------------------------------------------------------------
 */
size_t rocs_history_workspace_size(int64_t num_requests, int64_t num_rows, int32_t num_heads,
                                   int32_t kv_heads, int32_t head_dim, int64_t max_kv_len,
                                   int32_t dtype);

int32_t rocs_history_attention(const void* q, int64_t q_row_stride, const void* k, const void* v,
                               int64_t kv_row_stride, const int32_t* q_offsets,
                               const int32_t* kv_offsets, const int32_t* prefix_lens,
                               const int32_t* q_docs, const int32_t* kv_docs,
                               const float* slopes, int64_t num_requests, int64_t num_rows,
                               int64_t num_kv_rows, int32_t num_heads, int32_t kv_heads,
                               int32_t head_dim, float softmax_scale, float cap, int32_t causal,
                               int64_t max_kv_len, int32_t dtype, void* out, void* workspace,
                               size_t workspace_bytes, void* stream);

/*
 * ---------------------------------------------------------------------------
 * rocs_paged_attention: the same over a paged cache. Slot s of the cache holds
 * one history of kv_lens[s] rows: its key j is row j % page_size of page
 * page_table[s][j / page_size].
 *
 *   q            as above: one row a request for single events, any ragged
 *                number for chunks of new events (whose K/V are in the cache
 *                already: the rows stand at the history's end), or candidates
 *                with causal = 0
 *   k_pages, v_pages  row i of page p starts at p * page_stride + i *
 *                kv_row_stride elements and holds [kv_heads, head_dim]; K and
 *                V may be two column slices of one [pages, page_size, 2, ..]
 *                array. 0: dense rows, dense pages.
 *   page_table   [num_slots, table_width] int32
 *   kv_lens      [num_slots] int32 (a length outside 0 .. table_width *
 *                page_size acts as the nearest of the two)
 *   slots        [R] int32, the slot of each request, or NULL: request r is
 *                slot r (then R <= num_slots)
 *   max_kv_len   an upper bound on the lengths, or 0 for the table's width
 *   workspace    sized as above with min(max_kv_len, table_width * page_size)
 *                keys, or that product without a bound
 * Every other argument, the result and the limits are those of
 * rocs_history_attention, and table_width * page_size <= 2^31 - 4096. Page ids
 * and slots are device data: one outside its range is clamped into it (wrong
 * rows, never an access outside the pages).
 * Rows of a page past a history's end are not read.
 *
 * Fast path: as above, with page_size a multiple of 16.
 * ---------------------------------------------------------------------------
 */
int32_t rocs_paged_attention(const void* q, int64_t q_row_stride, const void* k_pages,
                             const void* v_pages, int64_t page_stride, int64_t kv_row_stride,
                             const int32_t* page_table, int64_t table_width,
                             const int32_t* kv_lens, const int32_t* slots, int64_t num_slots,
                             const int32_t* q_offsets, const int32_t* prefix_lens,
                             const float* slopes, int64_t num_requests, int64_t num_rows,
                             int64_t num_pages, int32_t page_size, int32_t num_heads,
                             int32_t kv_heads, int32_t head_dim, float softmax_scale, float cap,
                             int32_t causal, int64_t max_kv_len, int32_t dtype, void* out,
                             void* workspace, size_t workspace_bytes, void* stream);

/*
 * ---------------------------------------------------------------------------
 * The cache's pages. Its state is the caller's device memory:
 *
 *   pool        num_layers x num_pages pages of page_size rows of row_bytes
 *               bytes, dense (one table serves all layers of a model)
 *   page_table  [num_slots, table_width] int32; the entries past a slot's
 *               length are -1
 *   lens        [num_slots] int32, rows held
 *   refs        [num_pages] int32, the number of slots that hold the page;
 *               0: the page is free
 * and starts as page_table = -1, lens = 0, refs = 0. A page that is not full
 * belongs to one slot alone.
 *
 * Free pages are taken lowest index first, in the order of a call's entries,
 * so equal calls give equal tables. An operator that needs pages does all of
 * its work or none; it writes status[2]: {0, 0} when done, else
 *   ROCS_CACHE_NO_PAGES    status[1] = the pages that were missing
 *   ROCS_CACHE_TABLE_FULL  a slot would need more than table_width pages (in
 *                          reserve also one that holds more than that already)
 *   ROCS_CACHE_BAD_SLOT    a slot outside [0, num_slots), one named twice (as
 *                          an entry of reserve, or a child of fork), a child
 *                          that is not empty or that is a parent as well, a
 *                          slot with a negative length, a parent with more
 *                          rows than table_width pages hold
 * (the last cause in this list that holds). Nothing else is changed then.
 *
 * The lists of a call do not overlap the cache's arrays or its outputs.
 * Limits: num_slots <= 2^18, entries <= 2^30 (free: < 2^24); num_pages *
 * page_size and table_width * page_size < 2^31.
 * ---------------------------------------------------------------------------
 */
#define ROCS_CACHE_NO_PAGES 1
#define ROCS_CACHE_TABLE_FULL 2
#define ROCS_CACHE_BAD_SLOT 3

size_t rocs_cache_workspace_size(int64_t entries, int64_t num_pages);

/* Room for new rows: entry i adds row_offsets[i+1] - row_offsets[i] rows to
 * slot slots[i]. lens, page_table and refs follow; rows[m] (int32 [num_rows])
 * becomes the pool row (page * page_size + row in the page) of new row m, or
 * -1 where the call could not be done and for rows past row_offsets[entries]
 * (a batch padded to a fixed num_rows). workspace:
 * rocs_cache_workspace_size(entries, num_pages) bytes, 256-byte aligned. */
int32_t rocs_cache_reserve(const int32_t* slots, const int32_t* row_offsets, int64_t entries,
                           int64_t num_rows, int32_t* page_table, int64_t table_width,
                           int32_t* lens, int64_t num_slots, int32_t* refs, int64_t num_pages,
                           int32_t page_size, int32_t* rows, int32_t* status, void* workspace,
                           size_t workspace_bytes, void* stream);

/* Row m of x (x_row_stride bytes apart, row_bytes bytes) into row rows[m] of
 * one layer's pool of num_pool_rows rows. A row number outside the pool is
 * passed over; a pool row that is named twice holds any mix of the two. */
int32_t rocs_cache_write(const void* x, int64_t x_row_stride, const int32_t* rows,
                         int64_t num_rows, void* pool, int64_t num_pool_rows, int64_t row_bytes,
                         void* stream);

/* Child i (an empty slot) becomes a copy of slot parents[i]: it shares the
 * parent's full pages (refs + 1), and gets a copy, in every layer, of the
 * filled rows of a last page that is not full. workspace:
 * rocs_cache_workspace_size(entries, num_pages). */
int32_t rocs_cache_fork(const int32_t* parents, const int32_t* children, int64_t entries,
                        int32_t* page_table, int64_t table_width, int32_t* lens,
                        int64_t num_slots, int32_t* refs, int64_t num_pages, int32_t page_size,
                        void* pool, int64_t num_layers, int64_t row_bytes, int32_t* status,
                        void* workspace, size_t workspace_bytes, void* stream);

/* The slots' pages back (refs - 1), their table rows -1, their lengths 0. A
 * slot that is empty, named again or outside [0, num_slots) is passed over. */
int32_t rocs_cache_free(const int32_t* slots, int64_t entries, int32_t* page_table,
                        int64_t table_width, int32_t* lens, int64_t num_slots, int32_t* refs,
                        int64_t num_pages, int32_t page_size, void* stream);

/* Live pages together: with n live pages, those at index n and above move, in
 * order, into the free pages below n, in every layer; page_table and refs
 * follow. status becomes {0, n}: the pages from n on are free. workspace:
 * rocs_cache_workspace_size(0, num_pages). */
int32_t rocs_cache_compact(int32_t* page_table, int64_t table_width, int64_t num_slots,
                           int32_t* refs, int64_t num_pages, int32_t page_size, void* pool,
                           int64_t num_layers, int64_t row_bytes, int32_t* status,
                           void* workspace, size_t workspace_bytes, void* stream);

/* Page src_pages[i] of src_pool into page dst_pages[i] of dst_pool, in every
 * layer (the pools may be one, or of different page counts). A pair with an id
 * outside its pool is passed over. A page that is written twice in one call
 * holds any mix of its sources, other ones in other layers; so does a copy of a
 * page that the same call writes. page_bytes = page_size * row_bytes. */
int32_t rocs_cache_copy(const int32_t* src_pages, const int32_t* dst_pages, int64_t entries,
                        const void* src_pool, int64_t src_num_pages, void* dst_pool,
                        int64_t dst_num_pages, int64_t num_layers, int64_t page_bytes,
                        void* stream);

#ifdef __cplusplus
}
#endif

#endif /* ROCS_HISTORY_H */
