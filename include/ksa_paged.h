/*
 * ksa_paged.h -- C ABI of the paged KV cache: rows of K and V kept in pages that the sequences of a server share, as
 * bf16 or in 8 bits, and three operators over them: writing the rows of new tokens (quantised on the way), reading rows
 * back, and the attention of a run of new rows -- one token, a few drafted ones or a piece of a prompt -- over everything
 * cached before them and over each other.
 *
 * Rows.  A sequence's rows are those of Eq. 1: k text tokens, then the m summaries of their chunk, chunk after chunk.  Row a
 * belongs to chunk c = a / (k + m); with r = a mod (k + m) it is text token c k + r (r < k) or summary c m + (r - k).
 *
 * Pages.  kpages, vpages hold num_pages pages of page_rows rows for every KV head, element (page, head, row, d) at
 * page * page_stride + head * head_stride + row * row_stride + d.  Text tokens and summaries of a sequence lie in
 * pages of their own: text token x of sequence b in page text_table[b][x / page_rows], summary x in page
 * summ_table[b][x / page_rows], each at row x mod page_rows.  Pages may stand in any order, and sequences may share
 * pages that they only read.  An entry of -1 is a page given back: text that every window has left (Eq. 3) need not be kept.
 *
 * Formats.  KSA_KV_BF16: values as they are.  KSA_KV_E4M3: a row of a head (head_dim values) is held as e4m3 values
 * y and one byte e, standing for y * 2^(e - 127); e = 255 stands for a row of NaN.  kscale, vscale hold the bytes,
 * [num_pages, num_kv_heads, page_rows], contiguous.  ksa_paged_append picks the smallest power of two, from 2^-110 up, at
 * which the row's largest magnitude is within 448, and rounds to nearest even (a power of two, so that scaling rounds
 * nothing: a value of at least 2^-6 times the scale is off by at most 2^-4 of itself; at the largest scale, 2^120, values
 * go to 240 instead of 256, which bf16 does not hold).  A row that holds an infinity or a NaN is stored as zeros with
 * e = 255.
 *
 * Calls.  A call takes `batch` sequences; sequence b has `cached[b]` rows before the call and the packed rows
 * [cu_rows[b], cu_rows[b + 1]) of the call's tensors, its rows cached[b], cached[b] + 1, ...  Lengths and tables are read on
 * the device: a call recorded into a CUDA graph follows what stands there at each replay.  num_rows is the rows of the
 * tensors, all of them in memory; what stands in rows from cu_rows[batch] on does not matter (ksa_paged_append may load it), and
 * they are left as they were.  A sequence may have no rows.
 *
 * Tensors (DEVICE; bf16 unless said otherwise; 16-byte aligned, int32 and lse 4-byte; strides in elements, multiples of 8 for bf16 and of 16 for
 * e4m3, of pages and of what is written not 0; head_dim contiguous):
 *   q, out : [num_rows, num_q_heads, head_dim]     k, v : [num_rows, num_kv_heads, head_dim]
 *   lse    : fp32 [num_q_heads, num_rows], natural log of the softmax denominator
 *   text_table : int32 [batch, text_cols]   summ_table : int32 [batch, summ_cols]   cached : int32 [batch]
 *   cu_rows : int32 [batch + 1], ascending, from 0 to at most num_rows; a sequence has at most 2^30 rows
 * Nothing is allocated, nothing synchronises the host; calls on different streams are independent as far as their tensors
 * and workspaces are.
 *
 * What only the device can see is reported through ksa_last_device_status: a row that the call needs lies in no page
 * (an entry outside 0 .. num_pages - 1, or a column past the table): KSA_PAGED_STATUS_BAD_PAGE; cu_rows or cached that
 * are no such lengths: KSA_PAGED_STATUS_BAD_ROWS.  Nothing outside the given memory is touched then; a sequence with bad
 * lengths is skipped, the outputs of a sequence with a bad page are not valid.
 */
#ifndef KSA_PAGED_H
#define KSA_PAGED_H

#include "ksa.h"

#ifdef __cplusplus
extern "C" {
#endif

#define KSA_KV_BF16  0
#define KSA_KV_E4M3  1

/* ksa_paged_attn takes what it expects to be faster for the call's sizes: the kernel for few query rows (mma.sync) for all
 * sequences, or the one for many (tcgen05), beside it the former for sequences of few rows where there are several.  These hold it
 * to the first or the second; results differ by roundings (see ksa_paged_attn).  Not both. */
#define KSA_FLAG_PAGED_MMA_SYNC  0x20u
#define KSA_FLAG_PAGED_TCGEN05   0x40u

typedef struct {
    int32_t  struct_size;        /* sizeof(ksa_paged_params) */
    int32_t  batch;              /* sequences of the call, >= 1 */
    int32_t  num_rows;           /* rows of q / k / v / out, >= 0 */
    int32_t  chunk_len;          /* k >= 1 */
    int32_t  summaries_per_chunk;/* m >= 0 */
    int32_t  window_chunks;      /* C >= 0 */
    int32_t  num_q_heads, num_kv_heads;   /* group size num_q_heads / num_kv_heads <= 64 */
    int32_t  head_dim;           /* 64 or 128 */
    float    softmax_scale;
    uint32_t flags;              /* KSA_FLAG_SUMMARY_TEXT_ONLY, KSA_FLAG_PAGED_* */
    int32_t  kv_format;          /* KSA_KV_* */
    int32_t  page_rows;          /* 16, 32, 64 or 128 */
    int32_t  num_pages;          /* >= 1 */
    int32_t  text_cols, summ_cols;        /* columns of the tables; summ_cols may be 0 where m == 0 */
    int64_t  page_stride, head_stride, row_stride;    /* of kpages and vpages */
    int64_t  q_stride_tok, q_stride_head;
    int64_t  k_stride_tok, k_stride_head;
    int64_t  v_stride_tok, v_stride_head;
    int64_t  o_stride_tok, o_stride_head;
} ksa_paged_params;

/* The cache and the batch of a call (DEVICE pointers; kscale, vscale: KSA_KV_E4M3 only, else NULL). */
typedef struct {
    void* kpages; void* vpages; uint8_t* kscale; uint8_t* vscale;
    const int32_t* text_table; const int32_t* summ_table; const int32_t* cached; const int32_t* cu_rows;
} ksa_paged_kv;

/* Writes k, v of the call's rows into their pages.  No two rows of a call may fall on the same place of the pool. */
int ksa_paged_append(ksa_ctx* ctx, const ksa_paged_kv* kv, const void* k, const void* v, const ksa_paged_params* p, void* cuda_stream);
/* Reads the rows [cached[b], cached[b] + cu_rows[b + 1] - cu_rows[b]) of every sequence back into k, v, rounded once to
 * bf16 (exact for what ksa_paged_append wrote).  Rows of a page that was given back (entry -1) come as zeros. */
int ksa_paged_gather(ksa_ctx* ctx, const ksa_paged_kv* kv, void* k, void* v, const ksa_paged_params* p, void* cuda_stream);
/*
 * Attention of the call's rows, whose own K and V have been appended before: a text token i of chunk c sees the text
 * [max(0, c - C) k, i] and the summaries [0, max(0, c - C) m) (Eq. 3; C >= the number of chunks and m = 0: plain causal
 * attention), a summary the text of its own chunk and that chunk's summaries up to itself (text only under
 * KSA_FLAG_SUMMARY_TEXT_ONLY).  Query head h reads KV head h / (num_q_heads / num_kv_heads).  Pages that no row of a sequence
 * sees are not looked up.  What stands in rows that no row of the call sees -- behind the sequence, before its windows --
 * does not matter; rows that one of the call's rows sees must be finite (or NaN reaches rows of the same sequence that do
 * not see them, and LSEs too).  e4m3 pages hold no NaN codes (0x7f, 0xff): a row of NaN is said by its scale byte.
 *
 * Roundings: scores, maxima, sums and outputs are fp32 until the output's one rounding to bf16.  A probability is rounded before its
 * product with V, to bf16 (2^-8 of itself at most), or to f16 over e4m3 pages: the mma.sync kernel takes it times its value
 * row's scale and keeps what is above 2^-25 of the largest such product among the keys of a warp, the tcgen05 kernel what is above
 * 2^-36 of the largest probability (all of it where the scales of the value rows in view differ by more than 2^10).  q over e4m3
 * pages is f16 too, times a power of two for each row: exact down to 2^-22 of the row's largest value, off by 2^-33 of that at most below.
 */
int ksa_paged_attn(ksa_ctx* ctx, const ksa_paged_kv* kv, const void* q, void* out, float* lse, void* workspace, size_t workspace_bytes,
                   const ksa_paged_params* p, void* cuda_stream);
/* Bytes of DEVICE workspace, 256-byte aligned, with which ksa_paged_attn is faster for p: 0 but for calls of many rows a sequence
 * over an e4m3 cache (then room for the rows in view as bf16; of p the strides do not matter).  The workspace is scratch
 * for the length of the call, and other work must not use it meanwhile; without one (NULL, or smaller) the call works all the
 * same, and its results differ by roundings. */
int ksa_paged_workspace_bytes(const ksa_paged_params* p, size_t* bytes);

#define KSA_PAGED_STATUS_BAD_PAGE  103   /* a row that a call needs lies in no page of the pool */
#define KSA_PAGED_STATUS_BAD_ROWS  104   /* cu_rows or cached are no lengths */

#ifdef __cplusplus
}
#endif
#endif /* KSA_PAGED_H */
