/*
 * hqmq_serve.h - C ABI for serving a batch from packed caches (the format of hqmq.h, whose conventions on
 * pointers, streams, buffers and return values hold here too): attention of many sequences over one packed
 * prefix, the attention weight that cached tokens accumulate, the choice of the tokens to keep when a cache
 * outgrows its budget, and the packed rows of those tokens moved into a cache of their own.
 *
 * How they go together, per layer and generation step:
 *     hqmq_attend_shared   prefix and own tokens of every sequence; returns lse, the logarithm of each query
 *                          head's softmax denominator over all that it read
 *     hqmq_attend_mass     with that lse: the weights' sums per cached token, added to the running sums
 *     hqmq_evict_select    when a cache is full: which tokens stay
 *     hqmq_evict_compact   K and V rows of these as packed tensors with T = n_keep, which every entry point takes
 *
 * None of the calls allocates or synchronises; all of them can be recorded into a graph (hqmq_init first).
 * Workspaces hold nothing between calls; calls that may overlap need one each.
 */
#ifndef HQMQ_SERVE_H
#define HQMQ_SERVE_H

#include "hqmq.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Most sequences (or query positions) that share a packed tensor in one call. */
#define HQMQ_MAX_SHARE 1024

/* The sequences' own packed tokens, for hqmq_attend_shared: K and V tensors with one batch entry per sequence, encoded
 * with the codebooks of the prefix.
 *   params      HOST; B = prefix B * n_share, H, D, S and b_r as the prefix's, T the padded number of tokens
 *               (strides are ignored).
 *   enc_k, enc_v, cap_k, cap_v   as enc / outlier_capacity of hqmq_decode.
 *   visible_dev DEVICE, int32 [B][n_q_heads]: query head hq of sequence n sees its own tokens t < visible (a ragged
 *               batch: the sequence's length), or NULL: all T.  Values above T mean T, negative ones 0. */
typedef struct hqmq_own_tokens {
    const hqmq_params *params;
    const hqmq_encoded *enc_k;
    const hqmq_encoded *enc_v;
    uint64_t cap_k, cap_v;
    const int32_t *visible_dev;
} hqmq_own_tokens;

/* Attention of the generation step for a batch whose sequences share prefixes: sequence n = b * n_share + m reads the
 * packed prefix b, which is reconstructed once for all n_share of them (up to 256 query rows n_share * n_q_heads / H of a kv
 * head; once more for every further 256), and then its own packed tokens:
 *     o = (sum_t e^{s_t - M} V_hat_t + sum_u e^{s'_u - M} V_hat'_u) / (the same sums without V),  s = scale <q, K_hat>
 * K_hat and V_hat are the fp16 tensors hqmq_decode returns (up to the last fp32 bit before that rounding).  Products
 * are accumulated in fp32, the softmax subtracts a running maximum, the result is rounded once to fp16.  The softmax weights
 * enter the products with V with 22 significant bits.
 *   params      HOST; the prefix tensors': B prefixes, H, T, D (64, 96 or 128), S, b_r (strides are ignored).
 *   n_share     1 .. HQMQ_MAX_SHARE sequences per prefix; several query positions of one sequence are sequences here.
 *   n_q_heads   a multiple of H, at most 16 * H; query head hq reads kv head hq / (n_q_heads / H).
 *   q_dev       DEVICE, fp16 [B * n_share][n_q_heads][D] contiguous, 16-byte aligned.
 *   scale       finite.
 *   enc_k .. sec_v_dev   as for hqmq_attend.
 *   visible_dev DEVICE, int32 [B * n_share][n_q_heads]: the head sees the prefix tokens t < visible (sequences that
 *               branch off a prompt tree, causal limits of a window), or NULL: all T.  Values above T mean T,
 *               negative ones 0.
 *   own         HOST, or NULL: no tokens besides the prefix.
 *   out_dev     DEVICE, out, fp16 as q_dev.  A head that sees nothing gets zeros.
 *               Tokens that no query head of their kv head sees (behind every limit) may hold anything, infinities and NaN
 *               among their payloads included.  A token's V that some of them see is multiplied by the others' weight of zero:
 *               it has to be finite for these to stay so.
 *   lse_dev     DEVICE, out, fp32 [B * n_share][n_q_heads], or NULL: M + ln(sum of e^{s - M}) over everything the
 *               head saw, -infinity where that is nothing.
 *   workspace_dev  DEVICE, 256-byte aligned, hqmq_attend_shared_workspace_bytes().
 * Errors: INVALID_ARG (null / misaligned pointer, bad n_q_heads or n_share, non-finite scale, own tokens of another
 * shape), UNSUPPORTED (as hqmq_attend; B * n_share * H at 2^18 or above, with own tokens above 65535), BUFFER_TOO_SMALL,
 * HIP. */
int32_t hqmq_attend_shared(const hqmq_params *params, int32_t n_share, int32_t n_q_heads, const void *q_dev, float scale,
                           const hqmq_encoded *enc_k, uint64_t cap_k, const float *sec_k_dev,
                           const hqmq_encoded *enc_v, uint64_t cap_v, const float *sec_v_dev,
                           const int32_t *visible_dev, const hqmq_own_tokens *own, void *out_dev, float *lse_dev,
                           void *workspace_dev, uint64_t workspace_bytes, void *stream);

/* Workspace of hqmq_attend_shared in bytes (0 if the arguments are invalid); own_params: of the own tokens, or NULL. */
uint64_t hqmq_attend_shared_workspace_bytes(const hqmq_params *params, int32_t n_share, int32_t n_q_heads,
                                            const hqmq_params *own_params);

/* The attention weight of every cached token, summed over the query heads that read its kv head and added to what
 * earlier steps left:
 *     mass_out[b][h][t] = decay * mass_in[b][h][t] + sum over (m, g) with t < visible of e^{scale <q, K_hat_t> - lse}
 * over the n_share sequences (or query positions: a window of a prompt's last tokens) m of batch entry b and the query
 * heads g of kv head h.  The sum runs in one fixed order in fp32: results are the same from call to call.
 *   params .. sec_k_dev   as for hqmq_attend_shared (n_share = 1: caches of their own).
 *   lse_dev     DEVICE, fp32 [B * n_share][n_q_heads]: as hqmq_attend_lse, hqmq_attend_masked or hqmq_attend_shared
 *               returned it; a head with -infinity (it saw nothing) adds nothing.
 *   visible_dev as for hqmq_attend_shared, or NULL.
 *   mass_in_dev DEVICE, fp32 [B][H][T]; not read, and may be NULL, if decay is 0.
 *   decay       finite.
 *   mass_out_dev  DEVICE, out, fp32 [B][H][T]; may be mass_in_dev itself.
 * Errors: as hqmq_attend_shared, but any B * n_share * H. */
int32_t hqmq_attend_mass(const hqmq_params *params, int32_t n_share, int32_t n_q_heads, const void *q_dev, float scale,
                         const hqmq_encoded *enc_k, uint64_t cap_k, const float *sec_k_dev, const float *lse_dev,
                         const int32_t *visible_dev, const float *mass_in_dev, float decay, float *mass_out_dev,
                         void *stream);

/* The tokens that a cache keeps: per (b, h), of the sequence's length tokens the first n_sink, the last n_recent and,
 * of those between, the ones of largest mass, n_keep in all; equal masses: the lower index first; a NaN counts as less
 * than any number.  A sequence of at most n_keep tokens keeps them all.
 *   B, H, T     of the mass; B may run over layers too.
 *   mass_dev    DEVICE, fp32 [B][H][T].
 *   length_dev  DEVICE, int32 [B]: tokens of each sequence (values above T mean T, negative ones 0), or NULL: T.
 *   n_sink, n_recent >= 0, n_sink + n_recent <= n_keep, 1 <= n_keep <= T.
 *   keep_dev    DEVICE, out, int32 [B][H][n_keep]: ascending token indices, -1 behind the last.
 *   n_kept_dev  DEVICE, out, int32 [B][H]: min(length, n_keep).
 *   kept_mass_dev  DEVICE, out, fp32 [B][H][n_keep]: their mass, 0 behind the last; or NULL.
 *   workspace_dev  DEVICE, 256-byte aligned, hqmq_evict_select_workspace_bytes() bytes; may be NULL if that is 0.
 * Errors: INVALID_ARG, UNSUPPORTED (B * H above 65535, T above 2^30, B * H * T at 2^32 or above), BUFFER_TOO_SMALL, HIP. */
int32_t hqmq_evict_select(int32_t B, int32_t H, int32_t T, const float *mass_dev, const int32_t *length_dev,
                          int32_t n_sink, int32_t n_recent, int32_t n_keep, int32_t *keep_dev, int32_t *n_kept_dev,
                          float *kept_mass_dev, void *workspace_dev, uint64_t workspace_bytes, void *stream);
uint64_t hqmq_evict_select_workspace_bytes(int32_t B, int32_t H, int32_t T, int32_t n_keep);

/* The rows keep[b][h][j] of n_tensors packed tensors of one shape (K and V of a layer, or of many) as packed tensors
 * [B, H, n_keep, D] of their own: codes, scales, flags and payloads moved as they are, offsets and counts made anew.
 * No arithmetic: a kept row decodes to what it decoded to before.  An index outside 0 .. T-1 (the -1 behind a short
 * sequence's tokens) gives a row that decodes to zeros (limit what attention sees by n_kept).  Indices may come in any
 * order and repeat.
 *   params      HOST; of the tensors given: B, H, T, D <= 128, S, b_r (strides are ignored).
 *   enc, outlier_capacity   HOST arrays of n_tensors, as for hqmq_decode_batch (n_outliers is not read; status is).
 *   keep_dev    HOST array of n_tensors DEVICE pointers to int32 [B][H][n_keep]; they may be equal.
 *   out, out_capacity   HOST arrays: the new tensors, sized by hqmq_sizes with T = n_keep, every pointer set; no buffer
 *               may be one of the tensors given, or used twice.  Entries of the outlier list behind the last are not
 *               written.  A payload that lies beyond the list of the tensor given moves as zeros.  If the new list is
 *               too short the surplus is dropped and status gets HQMQ_STATUS_OUTLIER_OVERFLOW; the status bits of the
 *               tensor given are kept.
 *   n_keep      1 .. 2^31 - 1, B * H * n_keep * 32 < 2^32.
 *   workspace_dev  DEVICE, 256-byte aligned, hqmq_evict_compact_workspace_bytes() bytes.
 * Errors: INVALID_ARG, UNSUPPORTED, BUFFER_TOO_SMALL, HIP. */
int32_t hqmq_evict_compact(const hqmq_params *params, int32_t n_keep, int32_t n_tensors, const hqmq_encoded *enc,
                           const uint64_t *outlier_capacity, const int32_t *const *keep_dev, const hqmq_encoded *out,
                           const uint64_t *out_capacity, void *workspace_dev, uint64_t workspace_bytes, void *stream);
uint64_t hqmq_evict_compact_workspace_bytes(const hqmq_params *params, int32_t n_keep, int32_t n_tensors);

#ifdef __cplusplus
}
#endif
#endif /* HQMQ_SERVE_H */
