/*
 * sparse_attention.h -- C ABI of the attention half of a transformer block over kept rows (same library as sparse_block.h).
 *
 *   sparse_attn_plan / _run / _backward   attention over packed sequences of the kept rows, with gradients
 *   sparse_kv_write / _read               a paged cache of keys and values, as they are or in 8 bits, written and read back
 *   sparse_attn_decode                    single tokens against such a cache
 *
 * Conventions are those of sparse_block.h: mask byte != 0 keeps a row, a dropped row of a dense output holds +0.0, the library
 * allocates no device memory, argument checks come before the first HIP call, *_run, *_backward, *_write, *_read and *_decode only
 * enqueue work on hip_stream, and the same call gives the same bits.  Workspaces, o, its gradient, lse, caches, tables and lengths are
 * contiguous and aligned to 16 bytes; q, k, v and their gradients have a stride of their own from row to row (in entries, at least the
 * row's own length; so that they may be parts of one product's rows) and the alignment of an entry, 16-byte groups being the fast path.
 * Scores, softmax statistics and sums are floats; probabilities and the gradients of scores are rounded to the tensors' type, as
 * operands of the next product (to f16 where values are 8-bit codes of 16-bit types; SC_F16: gradients of scores beyond 65 504 are infinite and
 * below 2^-25 zero); every result is rounded once.
 */
#ifndef SPARSE_ATTENTION_H_
#define SPARSE_ATTENTION_H_

#include "sparse_block.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct {
  int32_t heads, kv_heads; /* query heads; key-value heads, a divisor of heads with heads / kv_heads <= 512.  Query head h reads key-value
                              head h / (heads / kv_heads) */
  int32_t d;               /* channels of a head, 1 .. 128 */
  int32_t dtype;           /* sc_dtype */
  int32_t causal;          /* 0/1: row i sees keys j <= i only */
  int32_t window;          /* 0, or row i sees keys with |i - j| < window only */
  float scale;             /* of q . k; > 0 and at most 2^127 */
} sc_attn_desc;

/* ---- attention over packed sequences ----------------------------------------------------------------------------------------------
 *   o_i = sum_j softmax_j(scale q_i . k_j) v_j      over the keys j of row i's sequence that it sees
 * Sequence s consists of the rows starts[s] .. starts[s + 1] - 1 (host memory, starts[0] = 0, ascending; empty sequences are allowed); of
 * these the kept ones count, if `rows` is not NULL, and are numbered without gaps (i and j above).  Rows from starts[seqs] on belong to
 * no sequence: they are neither read nor written.
 * The plan lays lists out in the caller's workspace, which has to stay as it is while the plan is used, and synchronises the stream.  After
 * sparse_rows_set_mask the row set needs a new plan: runs with the old one are refused (SC_ERR_MASK_COUNT).
 * q, o: [rows][heads][d], k, v: [rows][kv_heads][d], with row_format = SC_ROWS_COMPACT of the kept rows alone.
 * lse: float[kept][heads], log sum exp of the scores, for the backward pass; NULL in inference.  kept: of sparse_attn_info.
 * A row of q that is not finite loses its o and dq, one of do its dq, and no other row's; either loses dk and dv of the keys that it sees, and may
 * lose those of all keys of its sequence and key-value head.  A row of k or v that is not finite loses what is made of its sequence and key-value
 * head.  A row of q all of whose scores are -infinity gives zeros, has zeros for its gradient and adds nothing to dk and dv; one whose largest
 * score is beyond a float's range is NaN, as one that is not finite.  Scores and lse are floats, which limits probabilities: those of the gradients
 * are off by 2^-24 of lse's size relatively, and from scores of 2^24 on weights of f16 may leave its range.
 * rows * heads / kv_heads <= 2^30, rows * heads <= 2^36, (rows * heads / kv_heads / 128 + seqs) * kv_heads < 2^23 - 512. */
typedef struct sc_attn sc_attn;

/* Bytes for plans of up to `seqs` sequences of up to `rows` rows in all. */
sc_status sparse_attn_workspace_bytes(const sc_attn_desc* desc, int64_t seqs, int64_t rows, size_t* bytes);
sc_status sparse_attn_plan(const sc_attn_desc* desc, int64_t seqs, const int64_t* starts, const sc_rows* rows, void* workspace_dev,
                           size_t workspace_bytes, void* hip_stream, sc_attn** out);
/* end: starts[seqs]; kept: rows that belong to a sequence and are kept.  Any of the outputs may be NULL. */
sc_status sparse_attn_info(const sc_attn* plan, int64_t* end, int64_t* kept);
void sparse_attn_destroy(sc_attn* plan);

sc_status sparse_attn_run(const sc_attn* plan, const sc_rows* rows, int32_t row_format, const void* q_dev, int64_t q_stride,
                          const void* k_dev, int64_t k_stride, const void* v_dev, int64_t v_stride, void* o_dev, float* lse_dev,
                          void* hip_stream);
/* o and lse are those of the run, do_dev the gradient of o.  dq, dk, dv have the formats of q, k, v and strides of their own. */
sc_status sparse_attn_backward_workspace_bytes(const sc_attn* plan, size_t* bytes);
sc_status sparse_attn_backward(const sc_attn* plan, const sc_rows* rows, int32_t row_format, const void* q_dev, int64_t q_stride,
                               const void* k_dev, int64_t k_stride, const void* v_dev, int64_t v_stride, const void* o_dev,
                               const float* lse_dev, const void* do_dev, void* dq_dev, int64_t dq_stride, void* dk_dev,
                               int64_t dk_stride, void* dv_dev, int64_t dv_stride, void* workspace_dev, size_t workspace_bytes,
                               void* hip_stream);

/* ---- paged cache of keys and values -------------------------------------------------------------------------------------------------
 * k_pages, v_pages: [pages][kv_heads][page_rows][row], a row being d entries and zeros up to a whole 16-byte group.  Entries are of
 * the descriptor's type (bits = 0), or 8-bit codes -127 .. 127 (int8, bits = 8) with a float scale for every row and head,
 * k_scales, v_scales: [pages][kv_heads][page_rows]: x = code * scale, scale = max |x| / 127 (at least 2^-126), code the nearest whole
 * number to x / scale, ties to even.  A row that is not finite gets the scale NaN and reads as NaN.
 * slots: int64[rows], place page * page_rows + row of each row; a row whose slot is not in the cache (-1 for one) is not written, and
 * read as zeros.  The slots of one write differ (a place that is named twice holds a mixture of its rows afterwards).  rows * kv_heads <
 * 2^28 - 16. */
typedef struct {
  int32_t kv_heads, d;     /* d 1 .. 128 */
  int32_t page_rows;       /* rows of a page, a power of two, 1 .. 65 536 */
  int32_t pages;           /* pages * kv_heads * page_rows <= 2^31 - 1 */
  int32_t dtype;           /* sc_dtype of keys and values outside the cache */
  int32_t bits;            /* 0: as they are; 8 */
} sc_kv_desc;

/* Entries of a cache row: d rounded up to a whole 16-byte group. */
sc_status sparse_kv_row_entries(const sc_kv_desc* desc, int32_t* entries);
sc_status sparse_kv_write(const sc_kv_desc* desc, int64_t rows, const void* k_dev, int64_t k_stride, const void* v_dev, int64_t v_stride,
                          const int64_t* slots_dev, void* k_pages_dev, void* v_pages_dev, float* k_scales_dev, float* v_scales_dev,
                          void* hip_stream);
/* k, v: [rows][kv_heads][d], with strides of their own */
sc_status sparse_kv_read(const sc_kv_desc* desc, int64_t rows, const int64_t* slots_dev, const void* k_pages_dev, const void* v_pages_dev,
                         const float* k_scales_dev, const float* v_scales_dev, void* k_dev, int64_t k_stride, void* v_dev,
                         int64_t v_stride, void* hip_stream);

/* ---- single tokens against the cache ---------------------------------------------------------------------------------------------------
 * q, o: [rows][heads][d], contiguous.  Row r attends to the first lengths[r] rows of its sequence in the cache (its own token among
 * them, the last), of these to the last `window` ones if the descriptor has a window; `causal` has no meaning here.  Row j of the sequence
 * lies in page table[r][j / page_rows] (int32[rows][table_width]).  lengths[r] <= 0: o is zero; beyond table_width * page_rows: what the
 * table holds.  Rows of a page that is not in the cache are not there: no weight, nothing read.
 * What lies in the cache behind a sequence's length is not looked at, whatever it is.  A key or value that is not finite loses the heads
 * that read it in this row of q, and no other row; a score beyond a float's range is as above.  Against 8-bit codes a head's row of q in SC_BF16 is
 * taken in f16, in units of its largest entry: entries below 2^-28 of that lose digits.  rows * heads < 2^24, and so is the number of workgroups, which
 * the sequences' longest length that table_width allows multiplies. */
sc_status sparse_attn_decode_workspace_bytes(const sc_attn_desc* desc, const sc_kv_desc* cache, int64_t rows, int64_t table_width,
                                             size_t* bytes);
sc_status sparse_attn_decode(const sc_attn_desc* desc, const sc_kv_desc* cache, int64_t rows, const void* q_dev, const int32_t* table_dev,
                             int64_t table_width, const int32_t* lengths_dev, const void* k_pages_dev, const void* v_pages_dev,
                             const float* k_scales_dev, const float* v_scales_dev, void* o_dev, void* workspace_dev,
                             size_t workspace_bytes, void* hip_stream);

#ifdef __cplusplus
}
#endif

#endif /* SPARSE_ATTENTION_H_ */
