/*
 * libspqt - a decoder's key/value cache in 8 bits: the append of new tokens, the attention that reads it, and the
 * eviction of what attention no longer weighs.  Between the GEMVs that make q, k and v and the one that takes the
 * attention's output.  All calls are DEVICE, async, and follow the conventions of spqt.h (status codes, streams, a workspace
 * for each stream); lengths stay on the device, so a decode step can be captured in a graph.
 *
 * A cache is a pool of pages.  A page holds 64 tokens of one layer for all its kv heads:
 *
 *   codes   uint8 [pages][kv_heads][2][64 * head_dim], code + 128 with codes from -127 to 127
 *             keys   (0): byte t * head_dim + d                    token t of the page, element d
 *             values (1): byte d * 64 + place(t),   place(t) = 16 * (t / 4 % 4) + 4 * (t / 16) + t % 4
 *   scales  float [pages][kv_heads][2], one for the keys and one for the values of a page and head
 *   weights float [pages][kv_heads][64] (optional): what every cached token has weighed in attention
 *   table   int32 [sequences][max_blocks]: page of tokens 64 b .. 64 b + 63 of sequence s; entries past a sequence's
 *             last block are not read
 *   lengths int32 [sequences]: tokens of every sequence INCLUDING those of the call: a caller adds a step's tokens to
 *             the lengths first, once for all layers
 *   tail    16 bit [sequences][kv_heads][2][64][head_dim]: the values that the codes of a sequence's last block were
 *             made from
 *
 * Quantization.  With a = the largest |x| of a block's tokens and one head, keys and values apart,
 *   scale(a) = the least fp32 number from a / 127 (2^-100 if that is more) on that has 12 significant bits, the last of them set
 *   code     = x / scale(a), rounded to the nearest integer
 * A 16-bit x has at most 11 significant bits, so x / scale is never half way between two integers and fp32 rounds it
 * as exact arithmetic does.  When a new token raises the scale of the open block, its older tokens are quantized again
 * from the tail: what a block holds depends on its tokens only, not on the calls in which they came.  A block that was
 * given an infinity or a NaN has the scale NaN, and every row that sees a token of it has NaN outputs.
 *
 * Lengths grow by the appended counts and fall by an eviction only.  An append keeps the open block's scale, and takes the
 * tail for the values of that block: after lengths that were merely set back it would requantize from tokens that are gone,
 * or from another block's.  To take tokens back (drafts that were rejected), put back what their append has changed behind
 * the tokens that stay, and then the lengths: the codes and scales of the page that was open, and the sequence's tail, as
 * they were before it.  Pages that the tokens have begun need nothing; an append to an empty block reads neither.
 *
 * Positions.  The call's row i (i < counts[s], or `rows` without counts) of sequence s is the token at position
 * lengths[s] - counts[s] + i.  Lengths outside 0 .. 64 * max_blocks and counts outside 0 .. rows are taken as the nearest
 * of these.  A table entry outside 0 .. pages - 1 is not followed: what would be written there is dropped, and what
 * would be read there is NaN.
 */
#ifndef SPQT_KV_H
#define SPQT_KV_H

#include "spqt.h"

#ifdef __cplusplus
extern "C" {
#endif

#define SPQT_KV_BLOCK 64      /* tokens of a page */
#define SPQT_KV_FP16 0
#define SPQT_KV_BF16 1
#define SPQT_KV_MAX_DIM 256

typedef struct {
    void *codes;            /* 16-byte aligned */
    float *scales;          /* 8-byte aligned */
    void *tail;             /* append and evict; 16-byte aligned */
    float *weights;         /* optional except for spqt_kv_evict; 16-byte aligned */
    const int32_t *table;
    const int32_t *lengths;
    int64_t pages;          /* 1 .. 2^31 - 1 */
    int sequences;          /* 1 .. 65535 */
    int max_blocks;         /* 1 .. 2^24 */
    int kv_heads;           /* 1 .. 16384 */
    int head_dim;           /* 64, 128, 192 or 256 */
    int type;               /* of the 16-bit tensors: SPQT_KV_FP16 or SPQT_KV_BF16 */
} spqt_kv_cache;

/* A 16-bit tensor [sequences][rows][heads][head_dim] with these strides in elements, all of them multiples of 8 and not
 * negative; the last dimension is dense and the first element 16-byte aligned. */
typedef struct {
    void *data;
    int64_t sequence, row, head;
} spqt_kv_rows;

/* Quantizes the new tokens' keys and values into the cache.  rows: the second extent of k and v; counts: int32 [sequences]
 * or NULL (all rows).  The weights of the new tokens, if the cache has weights, are set to 0. */
int spqt_kv_append(const spqt_kv_cache *cache, const spqt_kv_rows *k, const spqt_kv_rows *v, int rows, const int32_t *counts, void *stream);

/* The last counts[s] tokens of every sequence as 16-bit values, code * scale rounded to nearest (at most the type's
 * largest number); rows from counts[s] on, and rows before the sequence's first token, are set to 0. */
int spqt_kv_read(const spqt_kv_cache *cache, const spqt_kv_rows *k_out, const spqt_kv_rows *v_out, int rows, const int32_t *counts, void *stream);

/* Bytes of the workspace that spqt_kv_attention needs for up to this many rows, at any lengths. */
int spqt_kv_workspace_bytes(int sequences, int rows, int q_heads, int kv_heads, int head_dim, int max_blocks, size_t *out_bytes);

/* Attention of the call's rows over the cache.  Query head j reads kv head j / (q_heads / kv_heads), a quotient of at most
 * 2^20.  Row i at position p sees the tokens t <= p of its sequence, and with window > 0 only those with t > p - window.
 *   out  = sum over t of softmax(scale * q . k_t) v_t            16 bit (at most the type's largest number), strided as q
 *   lse  = ln sum over t of exp(scale * q . k_t)                 fp32 [sequences][rows][q_heads], optional
 * Sums and statistics are fp32; for the products with the values a probability has 22 bits, but no finer than about 2^-40 of the row's
 * largest product of a probability and its block's scale.
 * A row that sees nothing, and a row from counts[s] on, has out 0 and lse -infinity.
 * decay: with cache->weights, and lse given, every token t of the sequence gets
 *   weights = decay * weights + sum over the call's rows and the heads that read its kv head of its probability
 * (decay 0 does not read them).
 * out may be q, element for element, in calls without weights; with weights, whose queries are read once more after out is
 * written, it must not overlap q (SPQT_EINVAL where both begin at one address), and in any other way it never may.
 * workspace: workspace_bytes >= spqt_kv_workspace_bytes, 256-byte aligned, prepared once with spqt_workspace_init;
 * every call leaves what the next one relies on, so attention calls on one stream may share one, whatever their shapes.  Not
 * with GEMVs: these rely on all zeros, and an attention leaves its partial sums.  It raises the flag that makes them yield NaN
 * on its workspace until spqt_workspace_init, rather than take such a word for one of theirs. */
int spqt_kv_attention(const spqt_kv_cache *cache, const spqt_kv_rows *q, const spqt_kv_rows *out, float *lse, int rows, const int32_t *counts,
                      int q_heads, float scale, int window, float decay, void *workspace, size_t workspace_bytes, void *stream);

/* Cuts every sequence down to `keep` tokens, for each kv head its own: the last `recent` ones (0 <= recent <= keep), and of the
 * others those with the largest weights, the earlier one where two weigh the same (a NaN weighs most).  What is kept moves in
 * order to the pages of new_table: 16-bit values as spqt_kv_read gives them are quantized as spqt_kv_append does, the weights are
 * copied and those of the last page's free places set to 0.  A sequence of at most `keep` tokens is moved whole.
 *   new_table    int32 [sequences][new_blocks], new_blocks >= ceil(keep / 64); its pages differ from the sequences' pages.
 *   new_lengths  int32 [sequences], receives min(length, keep); not the cache's lengths.
 *   kept         int32 [sequences][kv_heads][keep], receives the kept tokens' positions in ascending order, then -1. */
int spqt_kv_evict(const spqt_kv_cache *cache, int keep, int recent, const int32_t *new_table, int new_blocks, int32_t *new_lengths, int32_t *kept,
                  void *stream);

/* The same for caches that are cut down again and again: codes times their scales are quantized as they are, not by way of 16-bit values.
 *   new scale = scale(the largest |code * scale| of a block's kept tokens),   new code = code * (scale / new scale), the quotient in fp32, rounded to
 *   the nearest integer, ties to even
 * A block whose tokens all stay keeps its scale and its codes for good.  By way of fp16, 127 * scale may be rounded up and ask for the next scale: such a
 * block grows by 0.03 % with every spqt_kv_evict on average (1 % after 50, 5 % at worst); by way of bf16, it does so once at most. */
int spqt_kv_evict_exact(const spqt_kv_cache *cache, int keep, int recent, const int32_t *new_table, int new_blocks, int32_t *new_lengths, int32_t *kept,
                        void *stream);

#ifdef __cplusplus
}
#endif
#endif
