/*
 * spec_cache.h -- C ABI of the key/value cache around the verification step
 * (spec_verify.h) for AMD Instinct MI355X (gfx950).
 *
 * Speculative sampling (arXiv 2406.11016, Sec. 3.1) passes gamma drafted tokens
 * and the token before them through the target model in one go and then keeps
 * the first accepted_len of the drafts.  The target model's attention caches
 * keys and values, so each such step writes gamma + 1 entries a sequence, reads
 * everything cached so far, and keeps accepted_len + 1 of the new entries:
 *
 *   spec_cache_plan    which cache entries the next step's tokens get: advances
 *                      the sequences by what was verified, gives the pages of
 *                      ended sequences back, takes new ones, and writes the
 *                      block tables and the slot map, all on the GPU;
 *   spec_cache_append  writes new keys and values to the mapped slots;
 *   spec_cache_attend  attention of the new tokens to a prefix that the whole
 *                      batch shares and to each sequence's own entries;
 *   spec_cache_append4, spec_cache_read4, spec_cache_attend4
 *                      the same with a cache that is held in 4 bits, and its
 *                      entries back in 16 (below).
 *
 * Layout.  All tensors are row-major and live in device memory.
 *   k_cache, v_cache  [num_pages, kv_heads, page_size, head_dim]  16-bit; the
 *                     three inner dimensions are dense, pages lie page_stride
 *                     elements apart (so that K and V may alternate)
 *   block_table       [batch, max_pages] int32: the pages of each sequence in
 *                     the order of its tokens, -1 behind its last one
 *   lengths           [batch] int32: tokens of each sequence in the cache,
 *                     without the shared prefix
 *   slots             [batch, max_new] int32: page * page_size + place of each
 *                     new token, -1 behind a sequence's last one
 * A page holds page_size tokens, a power of two from 16 to 1024.  The tensors
 * of a step are padded to max_new tokens a sequence, as the ragged verification
 * calls' are; sequence b uses its first counts[b].
 *
 * Ownership, streams and errors are those of spec_verify.h: every pointer is
 * the caller's, nothing is allocated, a call enqueues its kernels on `stream`
 * (of the current device) and returns, SV_OK means "launched", and every call
 * may be captured into a HIP graph.  The functions keep no state of their own:
 * they are reentrant and thread-safe.  Calls that share tables, caches or a
 * workspace must be ordered.
 */
#ifndef SPEC_CACHE_H
#define SPEC_CACHE_H

#include "spec_verify.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Largest batch of one call. */
#define SV_CACHE_MAX_BATCH 4096
#define SV_CACHE_MAX_BATCH_D256 2048  /* spec_cache_attend at head_dim 256 (the batch's sums share the LDS) */
#define SV_CACHE4_MAX_BATCH_D256 1024 /* spec_cache_attend4 there */

/*
 * The tables of a batch.  num_pages is the number of pages of the caches;
 * free_pages is a stack of the free ones, its top at free_count[0] - 1.
 */
typedef struct sv_cache_tables {
    int32_t* lengths;      /* device [batch] */
    int32_t* counts;       /* device [batch]: the tokens that the last plan gave slots; -1: it could not */
    int32_t* held;         /* device [batch]: pages of each sequence */
    int32_t* block_table;  /* device [batch, max_pages] */
    int32_t* free_pages;   /* device [num_pages] */
    int32_t* free_count;   /* device [1] */
    int32_t batch, max_pages, num_pages, page_size;
} sv_cache_tables_t;

/*
 * Empty tables: no sequence holds a page, and the pages first_page ..
 * num_pages - 1 are free (the ones before them are the caller's, for a shared
 * prefix).  Pages are taken in ascending order.
 */
sv_status_t spec_cache_init(const sv_cache_tables_t* tables, int32_t first_page, hipStream_t stream);

/*
 * Plans the next step, for each sequence b:
 *   1. release[b] != 0: the sequence has ended; its pages go on the stack of
 *      free ones (in the order of b, then of the table) and it starts again
 *      with no tokens.
 *   2. Otherwise the tokens of the last plan that stay are kept: with
 *      accepted_len the last token and the accepted drafts, accepted_len[b] + 1
 *      of the counts[b] planned ones (none for the verification's sentinel -1),
 *      without it all of them.  Nothing is kept where the last plan gave no
 *      slots (counts[b] <= 0); accepted_len[b] is not looked at there.
 *   3. new_tokens[b] (0 .. max_new; without the array max_new) more tokens get
 *      slots behind them; where the sequence's pages do not suffice it takes
 *      new ones from the top of the stack, sequences in the order of b.
 * lengths, counts, held, block_table and the stack are updated, and
 *   slots      [batch, max_new]  is written whole;
 *   positions  [batch, max_new]  if not NULL: position_base + the token's place
 *                                in its sequence, -1 behind the last one.
 * A sequence that cannot be served gets counts[b] = -1 and no slots and takes no
 * pages: accepted_len[b] outside -1 .. counts[b] - 1 (nothing is kept then),
 * new_tokens[b] outside 0 .. max_new, more than max_pages pages, or no free
 * pages left: it is the first whose pages are not there, or comes after it and
 * needs a page too.  Sequences keep the pages of rejected tokens for the next
 * ones.  One launch, two for large batch * max_new.
 * accepted_len, new_tokens, release and positions may be NULL.
 */
sv_status_t spec_cache_plan(const sv_cache_tables_t* tables, const int32_t* accepted_len, const int32_t* new_tokens,
                            const int32_t* release, int32_t max_new, int32_t position_base, int32_t* slots,
                            int32_t* positions, hipStream_t stream);

/*
 * Writes new keys and values [batch, max_new, kv_heads, head_dim] to the cache
 * slots that `slots` names; tokens whose slot is outside 0 .. num_pages *
 * page_size - 1 (-1 among them) are not read.  No slot may be named twice.
 * Strides are in elements: of the batch, token and head dimension (head_dim is
 * dense).  head_dim is a multiple of 8; pointers are aligned to 16 bytes and
 * strides are multiples of 8 elements (SV_ERR_PARAM otherwise).
 */
typedef struct sv_cache_append_desc {
    const void* k;
    const void* v;
    int64_t k_stride[3], v_stride[3];
    void* k_cache;
    void* v_cache;
    int64_t page_stride;
    const int32_t* slots;
    sv_dtype_t dtype;  /* SV_F16 or SV_BF16 */
    int32_t batch, max_new, kv_heads, head_dim, num_pages, page_size;
} sv_cache_append_desc_t;

sv_status_t spec_cache_append(const sv_cache_append_desc_t* desc, hipStream_t stream);

/*
 * Attention of new tokens whose keys and values are in the cache already
 * (spec_cache_append).  Token i of sequence b sees the whole prefix (prefix_len
 * tokens in the pages of prefix_table) and the sequence's own tokens
 * 0 .. lengths[b] + i:
 *
 *   out[b, i, h] = sum_j w_j v_j / sum_j w_j,   w_j = exp(scale q[b, i, h] . k_j)
 *
 * with the keys and values of head h / (q_heads / kv_heads).  The tokens of the
 * whole batch share the reads of the prefix: it is read for tiles of up to 128
 * rows (token x head), not for sequences, and by neighbouring tiles through one
 * cache.  q and out [batch, max_new, q_heads, head_dim] do not overlap;
 * rows behind counts[b] are neither read nor written (all of them where
 * counts[b] <= 0; without `counts` every sequence has max_new).  Entries of the
 * cache that a token does not see have no influence on it, whatever their bits.
 *
 * Scores, statistics and sums are held in fp32; the weights are rounded to the
 * storage type for their product with the values (what is rounded off would take a
 * second product).  Weights below 2^-31 (fp16) or 2^-98 (bf16) of a row's largest
 * may count as 0 there, so an infinite value of such a key gives infinity or NaN;
 * so may, in bf16, products of such a relative weight and a value below 2^-98.
 *
 * Bad data found on the device makes the outputs of the sequence NaN: a page
 * outside 0 .. num_pages - 1 among those that the sequence needs (in the prefix:
 * of every sequence), lengths[b] < 0, counts[b] > max_new, or lengths[b] +
 * counts[b] > max_pages * page_size.
 *
 * head_dim is 64, 80, 96, 128 or 256 (for at most SV_CACHE_MAX_BATCH_D256
 * sequences); q_heads a multiple of kv_heads; scale between 1e-30 and 1e30.
 * Pointers are aligned to 16 bytes, strides (elements; batch, token, head) are
 * multiples of 8, and out's are not 0 where there is more than one element.
 * `workspace` holds
 * spec_cache_attend_workspace_bytes() bytes, aligned to 16, and needs no
 * initialisation.
 */
typedef struct sv_cache_attend_desc {
    const void* q;
    void* out;
    int64_t q_stride[3], out_stride[3];
    const void* k_cache;
    const void* v_cache;
    int64_t page_stride;
    const int32_t* block_table;
    const int32_t* lengths;
    const int32_t* counts;        /* may be NULL: max_new */
    const int32_t* prefix_table;  /* device, the prefix's pages; may be NULL if prefix_len is 0 */
    int32_t prefix_len;
    sv_dtype_t dtype;             /* SV_F16 or SV_BF16 */
    int32_t batch, max_new, q_heads, kv_heads, head_dim;
    int32_t max_pages, num_pages, page_size;
    float scale;
    void* workspace;
    size_t workspace_bytes;
} sv_cache_attend_desc_t;

sv_status_t spec_cache_attend(const sv_cache_attend_desc_t* desc, hipStream_t stream);

/* Bytes of workspace that such a call needs, with or without a prefix; 0 for invalid sizes. */
size_t spec_cache_attend_workspace_bytes(int32_t batch, int32_t max_new, int32_t q_heads, int32_t kv_heads,
                                         int32_t head_dim);

/*
 * Caches in 4 bits.  A value is held as an e2m1 number (0, 0.5, 1, 1.5, 2, 3, 4, 6
 * and their negatives: codes 0 to 7, and 8 to 15), and each block of 32 values of a
 * token and head (head_dim's last block may be shorter) shares a power of two,
 * whose exponent + 127 is a byte: 4.25 bits a value (4.3 at head_dim 80).  This is the block format of
 * the OCP microscaling specification (MXFP4), so the byte 255 makes its block NaN.
 *   k_cache, v_cache  [num_pages, kv_heads, page_size * row] bytes, with
 *                     row = head_dim / 2 + (head_dim + 31) / 32.  Of each page and
 *                     head first the codes [page_size, head_dim / 2], an even
 *                     value's in the low half of its byte, then the scales
 *                     [page_size, (head_dim + 31) / 32].  Pages lie page_stride
 *                     BYTES apart, a multiple of 16.
 * The tables, slots and plans are the same as those of caches in 16 bits.
 */

/*
 * spec_cache_append to such caches: each token's values are quantised as they
 * are written, by themselves, so nothing that was written before changes.  A
 * block's scale is the power of two that brings its largest magnitude into
 * 3.5 .. 7, but not below 2^-23 (fp16) or 2^-125 (bf16).  Values go to the nearest number
 * that the codes have, those in the middle of two to the even code, those beyond 6 to 6:
 * they move by at most a fifth of the block's largest magnitude, or a quarter of the
 * smallest scale where that is more.  With the greatest scale, 2^14 (fp16, a largest
 * magnitude of 57,344 or more) or 2^126 (bf16, 1.75 * 2^127 or more), 4 is no number of the
 * storage type, and those of 3.5 and more go to 3: they move by at most a quarter of the
 * largest.  So what is held of finite values are finite numbers of the storage type.
 * A block with an infinity or NaN reads as NaN.
 */
sv_status_t spec_cache_append4(const sv_cache_append_desc_t* desc, hipStream_t stream);

/*
 * Entries of such caches, in 16 bits: k and v [batch, max_new, kv_heads, head_dim]
 * of the tokens whose slots are named (they may be named more than once); rows
 * whose slot is outside 0 .. num_pages * page_size - 1 (-1 among them) are not
 * written.  What spec_cache_append4 wrote from the same type is returned exactly
 * as it is held.  Strides and alignment are those of spec_cache_append, and rows
 * do not lie on one another.
 */
typedef struct sv_cache_read_desc {
    void* k;
    void* v;
    int64_t k_stride[3], v_stride[3];
    const void* k_cache;
    const void* v_cache;
    int64_t page_stride;  /* bytes */
    const int32_t* slots;
    sv_dtype_t dtype;     /* SV_F16 or SV_BF16 */
    int32_t batch, max_new, kv_heads, head_dim, num_pages, page_size;
} sv_cache_read_desc_t;

sv_status_t spec_cache_read4(const sv_cache_read_desc_t* desc, hipStream_t stream);

/*
 * spec_cache_attend over such caches: the same attention, of the values that
 * spec_cache_read4 gives for `dtype`, with the same accuracy, limits and errors, but for at
 * most SV_CACHE4_MAX_BATCH_D256 sequences at head_dim 256.  (Values
 * that do not fit fp16, as bf16 may have written them, are infinite or lose
 * bits there.)  Without a prefix, for up to 48 rows (tokens x q_heads / kv_heads; 16 at
 * head_dim 256) and tables of up to 1,024 tokens a sequence, it is one launch, two otherwise:
 * a table no larger than the sequences need saves short ones 3 us.
 */
sv_status_t spec_cache_attend4(const sv_cache_attend_desc_t* desc, hipStream_t stream);

/* Bytes of workspace that such a call needs, with or without a prefix; 0 for invalid sizes. */
size_t spec_cache_attend4_workspace_bytes(int32_t batch, int32_t max_new, int32_t q_heads, int32_t kv_heads,
                                          int32_t head_dim);

#ifdef __cplusplus
}
#endif

#endif /* SPEC_CACHE_H */
