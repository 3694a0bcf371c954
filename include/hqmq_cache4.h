/*
 * hqmq_cache4.h - C ABI of a paged KV cache held in 4 bits that grows token by token (the conventions of hqmq.h on
 * pointers, streams, buffers and return values hold here too): new rows of a ragged batch quantised into their
 * sequences' pages, rows read back, and causal attention over the pages for generation steps, drafts and prompts.
 *
 * Where the packed form of hqmq.h wants a whole batch of tokens (its thresholds are medians over one, its search walks
 * codebooks) and keeps less than 5 bits a number with outliers verbatim, this one quantises each token by itself as it
 * arrives, for fp16 and bf16 models.
 *
 * Format.  Each run of 32 channels of a token's K or V row (a group; the last one of a head may be shorter) is quantised
 * by itself.  Inputs are clamped to +-49152 (6 * 2^13) first; a NaN counts as 0.
 *   HQMQ_CACHE4_FLOAT  4.25 bits a number: a sign and one of 0, 0.5, 1, 1.5, 2, 3, 4, 6 (bit 3, bits 2..0), times 2^e with
 *                      e the least of -23 .. 13 for which the group's largest magnitude is at most 7 * 2^e, stored as the
 *                      byte e + 127; nearest value, ties to the even code.  Every value is an fp16 number.
 *   HQMQ_CACHE4_INT    5 bits a number: m + c s, c = 0 .. 15, with the fp16 numbers s = (max - min) / 15 (difference and
 *                      product with fp32(1/15) in fp32, then rounded) and m = min, stored in this order; c nearest to
 *                      (x - m) / s, ties to even, 0 where s is 0.  The value is m + c s rounded once to fp16.
 * With width the head dimension rounded up to a multiple of 32, above 128 of 64, and G = width / 32, a page of page_size
 * tokens (a power of two, 16 or more) lies as
 *   k_codes   uint8 [n_pages][H][page_size][width / 2]: channel 2 i in the low half of byte i, 2 i + 1 in the high half
 *   k_scales  [n_pages][H][page_size][G] bytes, or fp16 pairs
 *   v_codes   uint8 [n_pages][H][page_size / 4][2 * width]: the width in parts of 128, 64 or 32 channels, largest first; a
 *             part is [16][token % 4][4, 2 or 1 bytes], the 16 being consecutive runs of 8, 4 or 2 channels
 *   v_scales  [n_pages][H][page_size / 4][G][token % 4] bytes, or fp16 pairs
 * (an attention's operand layout, so that it reads V without exchanging values between lanes).
 *
 * The batch.  Sequence i has length_i tokens, the call's own rows included, token t in page block_table[i][t / page_size],
 * place t % page_size; its n_i rows are the rows starts[i] .. starts[i + 1] - 1 of the tensors passed, and row j of them
 * stands at position length_i - n_i + j.  Several sequences may share pages that are only read.
 *
 * None of the calls allocates or synchronises; all of them can be recorded into a graph (hqmq_init first).  Workspaces hold nothing between
 * calls; calls that may overlap need one each.
 */
#ifndef HQMQ_CACHE4_H
#define HQMQ_CACHE4_H

#include "hqmq.h"

#ifdef __cplusplus
extern "C" {
#endif

#define HQMQ_CACHE4_FLOAT 0
#define HQMQ_CACHE4_INT 1

/* Types of the rows passed. */
#define HQMQ_TYPE_FP16 0
#define HQMQ_TYPE_BF16 1

typedef struct hqmq_cache4_params {
    int32_t n_pages;   /* 1 or more; offsets into the cache are 64-bit                     */
    int32_t page_size; /* tokens of a page: a power of two, 16 .. 2^20                      */
    int32_t H;         /* kv heads, 1 .. 4096                                               */
    int32_t D;         /* head dimension, 1 .. 256                                          */
    int32_t format;    /* HQMQ_CACHE4_FLOAT or HQMQ_CACHE4_INT                              */
} hqmq_cache4_params;

/* HOST struct of DEVICE pointers, 16-byte aligned, of the sizes that hqmq_cache4_sizes gives.  They need no
 * initialisation. */
typedef struct hqmq_cache4_buffers {
    void *k_codes, *k_scales, *v_codes, *v_scales;
} hqmq_cache4_buffers;

/* A batch: HOST struct.
 *   block_table DEVICE, int32 [n_seqs][pages_per_seq]; entries behind a sequence's last page are not used.
 *   lengths     DEVICE, int32 [n_seqs]: negative ones count as 0, larger ones as pages_per_seq * page_size.  Rows are placed by what
 *               counts: of a sequence grown past its table's room the last places are written again, and what they held is lost.
 *               The table needs the page of a step's tokens before the step is enqueued.
 *   starts      DEVICE, int32 [n_seqs + 1], ascending, or NULL: every sequence has n_rows / n_seqs rows.  Rows outside
 *               starts[0] .. starts[n_seqs] - 1 are no sequence's: they are not read, nor written.
 *   max_rows, max_length   the largest number of rows and length of a sequence as far as the host knows them: they shape
 *               the launch and, through it, the order of sums; every row and token counts whatever they say.  max_rows is
 *               ignored where starts is NULL, and counts as n_rows / n_seqs, rounded up, where it is less.
 * A page number outside 0 .. n_pages - 1, and a position below 0 (more rows than tokens), are no tokens: write leaves
 * them out, read gives zeros, attend does not see them. */
typedef struct hqmq_cache4_batch {
    int32_t n_seqs;        /* 1 .. 65535 */
    int32_t pages_per_seq; /* pages_per_seq * page_size at most 2^30 */
    int32_t max_rows, max_length; /* 1 or more */
    const int32_t *block_table;
    const int32_t *lengths;
    const int32_t *starts;
} hqmq_cache4_batch;

/* Rows [n_rows][heads][D] with element strides, channels contiguous: HOST struct of a DEVICE pointer, aligned to 2 bytes.
 * Any alignment of 2 bytes does: rows are moved 8 channels at a time, at any address.  Strides are 0 .. 2^30.  The memory from the
 * first element to the last may hold anything of the caller's between the rows, but none of the cache. */
typedef struct hqmq_cache4_rows {
    void *data;
    int64_t stride_row, stride_head;
} hqmq_cache4_rows;

/* Bytes of k_codes (and v_codes) and of k_scales (and v_scales).  Errors: INVALID_ARG, UNSUPPORTED (D above 256, an unknown
 * format, more than 2^46 bytes). */
int32_t hqmq_cache4_sizes(const hqmq_cache4_params *params, uint64_t *code_bytes, uint64_t *scale_bytes);

/* Quantise n_rows rows of K and V (HQMQ_TYPE_*) into the pages of their sequences.  Every page that is written must be one
 * sequence's only, at one place of its table: of tokens that two of them hold in one place the result is a mixture.
 *   k, v  HOST.
 * Errors: INVALID_ARG, UNSUPPORTED, HIP. */
int32_t hqmq_cache4_write(const hqmq_cache4_params *params, const hqmq_cache4_buffers *cache, const hqmq_cache4_batch *batch,
                          int32_t n_rows, int32_t type, const hqmq_cache4_rows *k, const hqmq_cache4_rows *v, void *stream);

/* Read the rows of the batch's positions back: the same positions that hqmq_cache4_write writes for the same batch (whole
 * sequences: n_i = length_i).  bf16 rows hold the cache's values rounded once more, which HQMQ_CACHE4_FLOAT's never need.
 *   k, v  HOST; no element of both.  Beside each other in one memory (a fused projection's) they need the same strides.
 * Errors: INVALID_ARG, UNSUPPORTED, HIP. */
int32_t hqmq_cache4_read(const hqmq_cache4_params *params, const hqmq_cache4_buffers *cache, const hqmq_cache4_batch *batch,
                         int32_t n_rows, int32_t type, const hqmq_cache4_rows *k, const hqmq_cache4_rows *v, void *stream);

/* Causal attention of the batch's rows over their sequences' pages (which hold the rows' own tokens already): query head hq
 * of the row at position p reads kv head hq / (n_q_heads / H), tokens t <= p, with a window those of t > p - window:
 *     o = sum_t e^{s_t - M} V_t / sum_t e^{s_t - M},  s_t = scale <q, K_t>
 * over the fp16 values of the cache.  Products are accumulated in fp32, the softmax subtracts a running reference, the
 * result is rounded once.  Weights enter the products with V with 22 significant bits for fp16 rows, and with 11 for bf16
 * rows, whose results have 8, none finer than 2^-31 of the row's largest; their sum and lse are of the weights as fp32 has them.  Queries
 * of bf16 enter as fp16 behind a power of two per row, which rounds channels below 2^-28 of the row's largest.  Tokens that no row of a sequence sees (behind the last row, before the first one's window) may
 * hold anything, and their pages may be none, or another's.  A query that holds an infinity or a NaN gives NaN, in its own row.
 *   n_q_heads   a multiple of H, at most 65535.
 *   q, out      HOST; rows of type `type`, [n_rows][n_q_heads][D]; out may be q itself with the same strides, and may share no
 *               element with it otherwise (in one memory between each other they need the same strides).  A row that sees nothing gets zeros.
 *   scale       finite, at most 2^100 in magnitude; scale q_c and scores are to stay below 2^126 (behind it scores tie, or
 *               count as unseen).
 *   window      0: none; else the number of tokens that a row sees at most, its own included.
 *   lse_dev     DEVICE, out, fp32 [n_rows][n_q_heads] contiguous, or NULL: M + ln(sum of e^{s - M}), -infinity where a row
 *               sees nothing.
 *   workspace_dev  DEVICE, 256-byte aligned, hqmq_cache4_attend_workspace_bytes() of the same sizes; may be NULL if that
 *               is 0.
 * Errors: INVALID_ARG, UNSUPPORTED, BUFFER_TOO_SMALL, HIP. */
int32_t hqmq_cache4_attend(const hqmq_cache4_params *params, const hqmq_cache4_buffers *cache, const hqmq_cache4_batch *batch,
                           int32_t n_rows, int32_t n_q_heads, int32_t type, const hqmq_cache4_rows *q, float scale,
                           int32_t window, const hqmq_cache4_rows *out, float *lse_dev, void *workspace_dev,
                           uint64_t workspace_bytes, void *stream);

/* Workspace of hqmq_cache4_attend in bytes, by the sizes in params and batch (its pointers are not read, only whether starts
 * is NULL); 0 if none is needed, or if the arguments are invalid. */
uint64_t hqmq_cache4_attend_workspace_bytes(const hqmq_cache4_params *params, const hqmq_cache4_batch *batch, int32_t n_rows,
                                            int32_t n_q_heads, int32_t window);

#ifdef __cplusplus
}
#endif
#endif /* HQMQ_CACHE4_H */
