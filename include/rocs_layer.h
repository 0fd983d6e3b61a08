/*
 * rocs_layer.h - C ABI of librocs, part three: a history layer over a cache
 * held in 4 bits. A shared projection with the low-rank adapters of many
 * requests beside it, new rows into the cache's pages with the position
 * rotation on the way, and attention over pages in 4 bits. Conventions, types
 * and error reporting are those of rocs.h (device pointers, caller-owned
 * memory, status codes, nothing is synchronised or allocated); slots, pages,
 * offsets and the cache's bookkeeping are those of rocs_history.h.
 */
#ifndef ROCS_LAYER_H
#define ROCS_LAYER_H

#include "rocs_history.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * ---------------------------------------------------------------------------
 * rocs_adapter_linear: out[n] = act( W x[n] + bias + s_a B_a (A_a x[n]) ), with
 * a = adapter_ids[r] of the request r that owns row n. A request whose id is
 * outside [0, num_adapters) has no adapter.
 *
 *   x            [N, K], rows x_row_stride elements apart (0: dense)
 *   w            [D, K], dense (the paper's [out, in] orientation)
 *   a            [num_adapters, rank, K], b [num_adapters, D, rank], dense; may
 *                be NULL with num_adapters = 0
 *   scales       [num_adapters] fp32 or NULL (1)
 *   bias         [D] fp32 or NULL
 *   offsets      [R + 1] int32: request r owns rows offsets[r] .. offsets[r+1]-1
 *   adapter_ids  [R] int32
 *   out          [N, D], dense, not overlapping an input; rows past offsets[R]
 *                (a padded batch) stay as they are
 *   workspace    rocs_adapter_workspace_size(R, N, K, D, rank, dtype) bytes,
 *                256-byte aligned. Scratch.
 * Sums are fp32. On the fast path the scaled s_a A_a x[n] is rounded to bf16 once,
 * for its product with B_a on the matrix cores; the general kernel keeps it in fp32.
 *
 * Fast path (bf16 MFMA kernels): K, rank and x_row_stride multiples of 8, D a
 * multiple of 4, x, w, a and b 16-byte aligned, out 16-byte aligned. Other
 * cases run a general kernel (fp32 matrix instructions), projection and all, which
 * costs large calls dearly: 32,768 rows, 2,048 -> 2,048, take 280 us at rank 8 or
 * 16 and 7,450 or 7,820 at 4 or 12. Pad the adapters with zeros to a rank that is a
 * multiple of 8.
 * One kernel serves a call, chosen by its average rows a request: single rows beside
 * a long chunk are faster as a call of their own. Neighbouring rows with the same
 * adapter are fastest as one request (offsets here only say whose adapter a row has):
 * 24,000 rows, 512 -> 1,024, rank 16, of 64 adapters take 197 us as 12,000 requests in
 * any order, 122 in the adapters' order, 52 as one request an adapter.
 * An infinity or NaN in one request's rows or adapter does not reach another's; where
 * one stands in B, the rows that share its tiles of 32 are formed again by a slow path.
 * Limits: rank <= 256; K, D < 2^22; R + ceil(N / 32) < 2^23 and ceil(N / 128) *
 * ceil(D / 128) < 2^24.
 * ---------------------------------------------------------------------------
 */
size_t rocs_adapter_workspace_size(int64_t num_requests, int64_t num_rows, int64_t k, int64_t d_out,
                                   int32_t rank, int32_t dtype);

int32_t rocs_adapter_linear(const void* x, int64_t x_row_stride, const void* w, const void* a,
                            const void* b, const float* scales, const float* bias,
                            const int32_t* offsets, const int32_t* adapter_ids,
                            int64_t num_requests, int64_t num_rows, int64_t k, int64_t d_out,
                            int32_t rank, int64_t num_adapters, int32_t dtype, int32_t activation,
                            void* out, void* workspace, size_t workspace_bytes, void* stream);

/*
 * ---------------------------------------------------------------------------
 * The position rotation. Of a head's dims the first rot_dim (even) are rot_dim /
 * 2 pairs; pair i is dims (2 i, 2 i + 1) with interleaved = 1, dims (i, i +
 * rot_dim / 2) with 0. A row at position p has each pair turned by the angle t =
 * p * freqs[i] (radians), whose cosine and sine are formed in 64 bits and rounded
 * to fp32 once:
 *   (x, y) -> (x cos t - y sin t, x sin t + y cos t)      each operation in fp32
 * The other dims stay. rot_dim = 0: no rotation, freqs may be NULL.
 *
 * A row's position is positions[m] (int32 [num_rows]); or, with positions NULL,
 * the one that the attentions give it: request r's rows offsets[r] ..
 * offsets[r+1]-1 are the last rows of slot slots[r] (NULL: slot r), which holds
 * lens[slot] rows with them: p = lens - n_r + i. Slots outside [0, num_slots) are
 * clamped into it. Rows past offsets[R] are passed over. With positions,
 * offsets (and slots, lens) may be NULL, R and num_slots 0.
 *
 * rocs_rotate: x [num_rows, num_heads, head_dim] (rows x_row_stride elements
 * apart, 0: dense) turned into out (dense, not overlapping an input).
 *
 * rocs_cache_append: row m of k and v ([num_rows, kv_heads, head_dim], rows
 * kv_row_stride elements apart) into row rows[m] (from rocs_cache_reserve) of
 * one layer's pool of num_pool_rows rows, k turned; and, with q not NULL, the
 * same rows' queries q [num_rows, num_heads, head_dim] turned into q_out. A row
 * number outside the pool is passed over (its query is turned all the same); a
 * pool row that is named twice holds any mix of the two. form:
 *   ROCS_POOL_ROWS  a row is [2, kv_heads, head_dim] of dtype: K, then V
 *   ROCS_POOL_FP4   a row is rocs_fp4_row_bytes(kv_heads, head_dim) bytes, in 4
 *                   bits a value, see below; the pool 16-byte aligned
 * Limits: head_dim <= 256, num_heads, kv_heads < 2^16, num_rows < 2^24, num_rows *
 * heads <= 2^30 (of q, and of k with v), num_pool_rows < 2^31.
 *
 * The 4-bit form (OCP's MXFP4 element and scale). head_dim is a multiple of 32.
 * A block of 32 values of a head shares a scale byte E; a value is the sign and
 * one of 0, 0.5, 1, 1.5, 2, 3, 4, 6 (bit 3, bits 2-0), times 2^(E - 127). A row is
 *   K values  kv_heads * head_dim / 2 bytes, value 2 j in the low half of byte j
 *   V values  the same
 *   K scales  kv_heads * head_dim / 32 bytes, V scales the same
 * padded to a multiple of 16 bytes (padding is not written). Written rows have
 *   E - 127 = floor(log2 m) - 2, or 1 more where m / 2^that > 7, in -126 .. 125,
 * of the block's largest magnitude m; values are rounded to the nearest, ties to
 * the even code, magnitudes past 6 to 6. So for m from 3.5 * 2^-126 to 7 * 2^125 a
 * value is off by at most 2^(E - 127), at most m / 3.5. Past that, where E stays at
 * its limit: magnitudes above 6 * 2^125 become 6 * 2^125, less than 2^126 off (m / 4);
 * with a smaller m a value is off by at most 2^-127, and up to 2^-128 it becomes
 * zero. A block that holds an infinity or NaN gets E = 255 and reads as NaN, all of
 * it. (Bytes from elsewhere: E = 0 is 2^-127; 4 and 6 under E = 253, and 2 and more
 * under 254, pass the types' range and have no defined reading.)
 * ---------------------------------------------------------------------------
 */
#define ROCS_POOL_ROWS 0
#define ROCS_POOL_FP4 1

int32_t rocs_rotate(const void* x, int64_t x_row_stride, const float* freqs, int32_t rot_dim,
                    int32_t interleaved, const int32_t* positions, const int32_t* offsets,
                    const int32_t* slots, const int32_t* lens, int64_t num_requests,
                    int64_t num_slots, int64_t num_rows, int32_t num_heads, int32_t head_dim,
                    int32_t dtype, void* out, void* stream);

int32_t rocs_cache_append(const void* q, int64_t q_row_stride, const void* k, const void* v,
                          int64_t kv_row_stride, const int32_t* rows, const float* freqs,
                          int32_t rot_dim, int32_t interleaved, const int32_t* positions,
                          const int32_t* offsets, const int32_t* slots, const int32_t* lens,
                          int64_t num_requests, int64_t num_slots, int64_t num_rows,
                          int32_t num_heads, int32_t kv_heads, int32_t head_dim, int32_t dtype,
                          void* pool, int64_t num_pool_rows, int32_t form, void* q_out,
                          void* stream);

/* Bytes of a row of a 4-bit pool; 0 where head_dim is no multiple of 32. */
size_t rocs_fp4_row_bytes(int32_t kv_heads, int32_t head_dim);

/* Rows rows[m] of a 4-bit pool as values: out [num_rows, 2, kv_heads, head_dim]
 * (K, then V; dense; 16-byte aligned, as the pool is). A row number outside the
 * pool gives zeros. */
int32_t rocs_cache_read_fp4(const int32_t* rows, int64_t num_rows, const void* pool,
                            int64_t num_pool_rows, int32_t kv_heads, int32_t head_dim,
                            int32_t dtype, void* out, void* stream);

/*
 * ---------------------------------------------------------------------------
 * rocs_paged_attention_fp4: rocs_paged_attention over pages in the 4-bit form.
 *
 *   pages        num_pages pages of page_size rows of rocs_fp4_row_bytes(kv_heads,
 *                head_dim) bytes, dense, 16-byte aligned: one layer's pool
 *   dtype        of q and out
 *   workspace    rocs_paged_fp4_workspace_size(R, N, num_heads, kv_heads,
 *                head_dim, keys, dtype) bytes with keys = min(max_kv_len,
 *                table_width * page_size), or that product without a bound;
 *                256-byte aligned; may be NULL when that is 0. The bound for one
 *                workspace under calls of many sizes is that of
 *                rocs_history_attention with C = 524,288 for bf16 and head_dim
 *                up to 128.
 * Every other argument, the rules of masks and scores, the result and the
 * limits are those of rocs_paged_attention (workgroups have 128 or 16 rows), with
 * head_dim a multiple of 32 up to 256 and num_pages * page_size < 2^31. A key whose block's scale is 255 is NaN
 * to the rows that see it, and has no part in the others.
 *
 * Fast path (bf16 MFMA kernels): bf16, head_dim up to 128 (fastest at 64 and
 * 128), q's row stride a multiple of 8 elements, q and out 16-byte aligned, any
 * page size. Other cases run a general kernel.
 * ---------------------------------------------------------------------------
 */
size_t rocs_paged_fp4_workspace_size(int64_t num_requests, int64_t num_rows, int32_t num_heads,
                                     int32_t kv_heads, int32_t head_dim, int64_t max_kv_len,
                                     int32_t dtype);

int32_t rocs_paged_attention_fp4(const void* q, int64_t q_row_stride, const void* pages,
                                 const int32_t* page_table, int64_t table_width,
                                 const int32_t* kv_lens, const int32_t* slots, int64_t num_slots,
                                 const int32_t* q_offsets, const int32_t* prefix_lens,
                                 const float* slopes, int64_t num_requests, int64_t num_rows,
                                 int64_t num_pages, int32_t page_size, int32_t num_heads,
                                 int32_t kv_heads, int32_t head_dim, float softmax_scale, float cap,
                                 int32_t causal, int64_t max_kv_len, int32_t dtype, void* out,
                                 void* workspace, size_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* ROCS_LAYER_H */
