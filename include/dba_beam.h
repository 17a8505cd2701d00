/*
 * libdba - what a beam-search decoder does next to the selection step, on AMD MI355X (gfx950), behind a C ABI:
 *
 *   dba_beam_select     the new beam from the decoder's logits (no constraints; dba_step of dba.h has those)
 *   dba_beam_reorder    decoder states follow the back-pointers
 *   dba_cache_append    new keys and values into a paged cache, rotated by their position on the way
 *   dba_tree_attend     attention of the nodes of a tree of hypotheses (or of drafted tokens) over that cache
 *
 * The cache of a sentence holds its shared prefix and, behind it, every token that any hypothesis has generated; what a
 * hypothesis sees of those is a row of mask bits (its ancestors).  So the cache never moves when the beam is
 * reordered: dba_beam_reorder moves the mask rows, and recurrent states where a decoder has them.
 *
 * Conventions are those of dba.h: "host" / "device" is said for every pointer, no device memory is allocated, work is
 * only enqueued on the stream given, every function returns DBA_OK or a negative code and none throws or aborts;
 * dba_last_error(NULL) gives the text of the calling thread's last failure.  There is no ctx: calls keep nothing, and any
 * number of them may run at once on streams of their own with workspaces of their own.  All may be captured into a
 * graph.  Formats are DBA_LOGP_F32 / F16 / BF16 of dba.h.  Strides are in elements unless said otherwise.
 */
#ifndef DBA_BEAM_H
#define DBA_BEAM_H

#include "dba.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * Selection over beams and vocabulary.  For every live row h of a sentence
 *     s(h, w) = score[h] + (logits[h, w] - log sum_u exp(logits[h, u])),
 * and the k_out greatest s of the sentence's k_in * V extensions become the new beam, best first; equal ones in the order
 * of h*V + w.  The scores are compared before they are rounded to fp32.  A completed hypothesis (DBA_FLAG_FINISHED)
 * has one extension: pad_id, at its own score.  Rows with DBA_FLAG_DEAD or a score of -inf offer nothing and their
 * logits are not looked at.  A logit of -inf is an extension that does not exist.  A row whose score or
 * normaliser is not finite (a NaN, a +inf, nothing but -inf) offers nothing.
 *
 *   B, k_in, k_out, V   sentences (1..65535), rows a sentence (1..64), slots of the new beam (1..64), vocabulary (1..2^24)
 *   eos_id, pad_id      different ids in [0, V); eos_id may be -1 (no hypothesis ever completes)
 *   logits_dev          device [B,k_in,V] of logits_format, aligned to the element size; sent_stride and row_stride
 *                       (>= V) between sentences and rows, last axis dense
 *   score_dev           device [B,k_in] fp32
 *   flags_dev           device [B,k_in] uint8 of DBA_FLAG_* bits; NULL: all rows are live
 *   out_token_dev, out_backptr_dev, out_score_dev, out_flags_dev
 *                       device [B,k_out] int32, int32, fp32, uint8 as dba_step writes them: an empty slot has pad_id,
 *                       -1, -inf, DBA_FLAG_DEAD.  None may be NULL, lie in an input or the workspace, or overlap another.
 *   workspace_dev       device, 256-byte aligned, at least dba_beam_select_workspace_bytes bytes; its content does not matter; no input lies in it
 */
DBA_API size_t dba_beam_select_workspace_bytes(int B, int k_in, int k_out, int V, int logits_format);
DBA_API int dba_beam_select(int B, int k_in, int k_out, int V, int eos_id, int pad_id, const void *logits_dev, int logits_format,
                            int64_t sent_stride, int64_t row_stride, const float *score_dev, const uint8_t *flags_dev,
                            int32_t *out_token_dev, int32_t *out_backptr_dev, float *out_score_dev, uint8_t *out_flags_dev,
                            void *workspace_dev, size_t workspace_bytes, void *hip_stream);

/*
 * One state of the hypotheses: for each of B sentences and k slots `segs` pieces of seg_bytes bytes.  Strides are in bytes.
 * E.g. of keys [B,k,heads,capacity,width] with t places in use: segs = heads, seg_bytes = t * width * element size, stride_seg =
 * capacity * width * element size.
 */
typedef struct dba_state {
    void *dst;             /* device */
    const void *src;       /* device; the same address as dst: in place (the strides are then the same too) */
    int64_t dst_sent, dst_row, dst_seg;
    int64_t src_sent, src_row, src_seg;
    int64_t segs, seg_bytes;
} dba_state;

/*
 * dst[b, h] = src[b, backptr[b, h]] for every state; a back-pointer outside [0, k) (an empty slot has -1) clears the row.
 * In place, rows that stay where they are are neither read nor written.  dst and src of one state are the same or have no byte in common,
 * pieces of dst do not overlap each other, and no state's dst has a byte in common with another state's dst or src: the states are
 * moved at the same time.  (Views of one tensor that interleave are apart.  Where they interleave in different strides, more than
 * 65536 times, they count as overlapping.)
 *   backptr_dev  device [B,k] int32 (as dba_step or dba_beam_select wrote it); must not lie in a dst
 *   states_host  host [n_states] (copied before the call returns)
 */
DBA_API int dba_beam_reorder(int B, int k, const int32_t *backptr_dev, const dba_state *states_host, int n_states, void *hip_stream);

/*
 * A paged cache: pools of pages of page_size tokens, and for each sentence the list of its pages.  Token t of sentence b
 * is at k + table[b*table_stride + t / page_size] * page_stride + (t % page_size) * token_stride + head * head_stride
 * (and in v alike).  A page number outside [0, n_pages) is a page that is not there: its tokens are not written and are seen by nobody.
 */
typedef struct dba_cache {
    void *k, *v;                     /* device, 16-byte aligned */
    const int32_t *table;            /* device [B, max_pages] */
    int64_t table_stride;
    int64_t page_stride, token_stride, head_stride;   /* multiples of 16 bytes; the D elements of a head are dense */
    int format;                      /* DBA_LOGP_* */
    int n_pages, page_size;          /* page_size: a power of two, at most 65536 */
    int max_pages;                   /* of a sentence: max_pages * page_size < 2^31 */
    int heads, head_dim;             /* head_dim: a multiple of 8, at most 256 */
} dba_cache;

/* Where a tensor [B, n, heads, head_dim] is: strides in elements, 16-byte aligned; the last axis is dense. */
typedef struct dba_heads {
    void *data;                      /* device */
    int64_t sent_stride, token_stride, head_stride;
} dba_heads;

/*
 * Tokens first[b] + i (0 <= i < min(n, count[b])) of sentence b's cache become k[b, i] and v[b, i], k rotated by its position:
 * pair j of the rot_dim first elements turns by the angle position * inv_freq[j], computed in 64 bits.  Pairs are
 * (j, j + rot_dim/2), or with interleaved != 0 (2j, 2j + 1).  Elements from rot_dim on are taken over as they are.  The rotation
 * is done in fp32 and rounded once.  Tokens outside [0, max_pages * page_size) or in a page that is not there are not written.
 *   k, v          the new tokens, heads as the cache's (they may lie in the pools, but not in places that this call writes)
 *   q, q_out      optional (both NULL or none): queries [B, n, q_heads, head_dim], rotated alike into q_out (which may be q, and else has no
 *                 byte in common with q, k and v); rows from count[b] on become 0
 *   first_dev     device [B] int32
 *   count_dev     device [B] int32; NULL: n everywhere
 *   position_dev  device [B, n] int32; NULL: first[b] + i
 *   inv_freq_dev  device [rot_dim / 2] fp32 (radians per position); rot_dim a multiple of 16, at most head_dim; 0: no rotation (NULL)
 */
DBA_API int dba_cache_append(int B, int n, const dba_cache *cache, const dba_heads *k, const dba_heads *v, int q_heads, const dba_heads *q,
                             const dba_heads *q_out, const int32_t *first_dev, const int32_t *count_dev, const int32_t *position_dev,
                             const float *inv_freq_dev, int rot_dim, int interleaved, void *hip_stream);

/*
 * out[b, i, h] = sum_t softmax_t(scale * q[b, i, h] . k[b, t, h / (q_heads / heads)]) v[b, t, ...] over the tokens t that node i
 * sees: the prefix[b] first ones of the sentence's cache and, of the tree[b] ones behind them, token j where bit j % 64 of
 * mask[b, i, j / 64] is set (bits from 64 * mask_words on count as not set); without a mask those with j <= tree[b] - n + i (the n queries are
 * the last n tokens of a chain).  A node that sees nothing gets 0 and a normaliser of -inf.
 *   q, out         [B, n, q_heads, head_dim]; q_heads a multiple of the cache's heads; n * q_heads <= 2^22, and B * heads times the
 *                  sixteens of n * q_heads / heads at most 2^28
 *                  out may be q, and else has no byte in common with it; nor has it, or out_lse_dev, with places that are read, with
 *                  each other or with the workspace
 *   prefix_dev, tree_dev   device [B] int32; negative ones count as 0; tree_dev may be NULL (0 everywhere)
 *   mask_dev       device [B, n, mask_words] uint64, or NULL
 *   max_len        no sentence sees tokens from max_len on (at most max_pages * page_size and 2^31 - 1024); the launch is laid out for it
 *   out_lse_dev    device [B, n, q_heads] fp32: log of the sum of the exponentials; may be NULL
 *   workspace_dev  device, 256-byte aligned, at least dba_tree_attend_workspace_bytes bytes (which may be 0)
 * What masked places, and places behind the end, hold never matters, NaN and infinities included.  Where a token is seen, an element of
 * its values that is not finite makes that element of the node's output an infinity or a NaN, whatever its weight, and a key that is
 * not finite may make all of them NaN.
 */
DBA_API size_t dba_tree_attend_workspace_bytes(int B, int n, int q_heads, const dba_cache *cache, int max_len);
DBA_API int dba_tree_attend(int B, int n, int q_heads, const dba_heads *q, const dba_cache *cache, const int32_t *prefix_dev,
                            const int32_t *tree_dev, const uint64_t *mask_dev, int mask_words, int max_len, float scale,
                            const dba_heads *out, float *out_lse_dev, void *workspace_dev, size_t workspace_bytes, void *hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* DBA_BEAM_H */
