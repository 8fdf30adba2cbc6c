/*
 * kvx_attend -- operators on a replica's paged KV cache (kv_cache of kvx.h), on AMD Instinct MI355X
 * (gfx950): what a replica computes on a cache that kv_load restored and kv_store will publish.
 *
 *   kv_append   the new tokens' K/V rows into the cache's pages (as they are, or as e4m3 with a scale)
 *   kv_attend   attention of the new tokens over their sequence's cached tokens, from one new token per
 *               sequence to the tail of a prompt behind a restored prefix, and the weight that every
 *               cached token received
 *   kv_keep     from accumulated weights: the tokens that a sequence keeps under a budget
 *   kv_compact  the kept tokens' rows into fresh pages
 *
 * Conventions are kvx.h's: a plain C ABI, explicit HOST and DEVICE pointers, streams as void*, a kv_status from
 * every entry point (kv_last_error has the reason), nothing enqueued when an argument is refused.  Each call works on
 * one layer of the cache, on the current device, which must be the cache's, and only enqueues kernels on `stream`: it
 * allocates nothing, never blocks the host, keeps nothing between calls and may be captured into a graph.  All reads
 * and writes of a call follow earlier work on `stream` and precede later work there; calls on different streams are
 * ordered by the caller where they share a written buffer (a cache, an output or a workspace).  DEVICE arrays are read
 * and written until the call's work has completed there.  Outputs overlap neither inputs nor the workspace, unless said.
 * Results do not depend on the order in which workgroups run: the same call gives the same bits.
 *
 * ---------------------------------------------------------------------------
 * A batch of sequences.  Sequence b has lens[b] tokens, its new ones among them: token t lies in block
 * block_tables[b*table_stride + t / BS] at slot t % BS of the layer's buffer.  Its new tokens are the rows
 * starts[b] .. starts[b+1] of the new tokens' arrays, and the last of its tokens: new row i of q is token
 * lens[b] - q + i (rows that would lie before token 0 have no place: they are not appended, and attend to nothing).
 * The host bounds (max_queries, max_len) size the launches; the numbers on the device may change between the replays
 * of a graph within them.
 *
 * What only the device can see is checked there and reported by kv_attend_async_error:
 *   KV_ASYNC_BAD_BLOCK  a block id outside [0, num_blocks): that page is neither read nor written, and its tokens
 *                       take part in nothing;
 *   KV_ASYNC_BAD_BATCH  a length outside [0, max_len], or rows outside [0, num_queries] or more than max_queries: the
 *                       sequence is left out, and nothing of its outputs is written; more kept tokens than the budget,
 *                       likewise.  A kept token outside its sequence's table: that row alone is not moved.
 * ---------------------------------------------------------------------------
 */
#ifndef KVX_ATTEND_H
#define KVX_ATTEND_H

#include "kvx.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Element types of rows and caches. */
#define KV_DTYPE_BF16 1
#define KV_DTYPE_F16 2
#define KV_DTYPE_E4M3 3  /* caches only: a value is the stored e4m3 (fn: no infinities) times k_scale or v_scale */

/* Async error bits, beside KV_ASYNC_BAD_BLOCK of kvx.h. */
#define KV_ASYNC_BAD_BATCH 2

/* Rows of new tokens, [tokens][heads][D]: element (t, h, d) at data + t*token_stride + h*head_stride + d
 * (strides in elements; a view of a wider projection's output needs no copy). */
typedef struct kv_rows {
    void *data;           /* DEVICE, 16-byte aligned */
    int64_t token_stride; /* both strides >= 0 and, over more than one token or head, multiples of 16 bytes */
    int64_t head_stride;
    int32_t heads;
    int32_t dtype;        /* KV_DTYPE_BF16 or KV_DTYPE_F16 */
} kv_rows;

typedef struct kv_batch {
    int32_t num_seqs;            /* sequences; 0 is a no-op */
    int32_t max_queries;         /* most new tokens of a sequence, >= 1 */
    int32_t num_queries;         /* rows of the new tokens' arrays */
    int32_t max_len;             /* most tokens of a sequence, at most table_len * BS */
    int32_t table_len;           /* entries of a sequence's block table that may be read */
    int32_t reserved;            /* must be 0 */
    int64_t table_stride;        /* entries between the tables of two sequences */
    const int32_t *block_tables; /* DEVICE int32[num_seqs][table_stride]; may be NULL where table_len is 0 */
    const int32_t *lens;         /* DEVICE int32[num_seqs] */
    const int32_t *starts;       /* DEVICE int32[num_seqs + 1]; NULL: one new token each, row b of sequence b */
} kv_batch;

/* Scores, in this order: s = scale * k_scale * (q . k); softcap > 0: s = softcap * tanh(s / softcap); slopes: s -=
 * slopes[query head] * (p - t), with p the query's own token and t the cached one.  Token t takes part where t <= p and,
 * with window > 0, p - t < window.  Zero-initialised fields take the documented defaults. */
typedef struct kv_attend_options {
    int32_t cache_dtype;      /* KV_DTYPE_*: what the cache's elements are (required; 1 byte: E4M3) */
    int32_t window;           /* 0 = none */
    float scale;              /* 0 = 1 / sqrt(D) */
    float softcap;            /* 0 = none */
    float k_scale, v_scale;   /* 0 = 1; E4M3 caches only */
    const float *slopes;      /* DEVICE float[query heads], or NULL */
    /* With weights_out: what each token t < lens[b] received, sum over the call's rows of its sequence and the query
     * heads of KV head h of exp(s - lse), is added to weights_in (NULL: to 0) and written to weights_out, both at
     * b*weights_seq_stride + h*weights_head_stride + t.  They may be the same array; tokens from lens[b] on are left
     * as they were. */
    const float *weights_in;  /* DEVICE */
    float *weights_out;       /* DEVICE, or NULL */
    int64_t weights_seq_stride, weights_head_stride;  /* elements; rows of max_len elements do not overlap */
    int32_t full_weights;     /* 1: exp(s) meets V as two numbers of q's type in every sequence (see kv_attend) */
    int32_t reserved;         /* must be 0 */
} kv_attend_options;

/*
 * kv_append -- write the new tokens' K and V rows into layer `layer` of the cache.  The rows' type is the cache's, or
 * for an E4M3 cache x is stored as e4m3(clamp(x / k_scale, -448, 448)) (K; V with v_scale), rounded to nearest even;
 * NaN stays NaN.  Every other byte of the cache is untouched.  Two sequences must not name the same page for new tokens
 * (precondition; otherwise the result depends on write order).
 * Errors: KV_EINVAL (NULL, sizes, types or strides that contradict each other), KV_EUNSUPPORTED (D*E no multiple of 16,
 * D > 256, unaligned rows, more than 65,535 sequences), KV_EHIP.
 */
KV_API kv_status kv_append(const kv_cache *cache, int32_t layer, const kv_batch *batch, const kv_rows *k,
                           const kv_rows *v, int32_t cache_dtype, float k_scale, float v_scale, void *stream);

/*
 * kv_attend -- out[row] = v_scale * sum over its tokens of softmax(s) * v, rounded once to q's type, and lse[row] = log
 * of the sum of exp(s), for every new row; query head h reads KV head h / (q->heads / H).  A row that sees no token
 * gets 0 and -infinity.  Sums, largest scores and lse are held in 32 bits.  The weights exp(s) meet V as two numbers of
 * q's type (the rounded weight and what it leaves) for sequences of up to 64 rows (new tokens times query heads) per KV
 * head, so that only the output's rounding shows.  For longer ones they are one number, rounded to nearest (off by up to
 * half a step of that type each), unless full_weights asks for two there as well.  What slots behind a sequence's last
 * token hold does not matter, but its own tokens' V are taken to be finite: 0 times an infinity of a token that a row
 * does not see reaches that row.  K of a token reaches the rows that see it and no others; where it is not finite, they
 * may become NaN.
 *   q, out:    [num_queries][query heads][D], same type; the cache's, or either 2-byte type for E4M3; rows of out do not
 *              overlap;
 *   lse:       DEVICE float[num_queries][query heads], or NULL;
 *   workspace: DEVICE, kv_attend_workspace's bytes (16-byte aligned; may be NULL for 0 bytes), the call's own until its
 *              work has completed: calls that may overlap, and graphs whose replays may, need one each.
 * Errors as kv_append; KV_EINVAL for a workspace that is too small; KV_EUNSUPPORTED also for more than 16,383 query heads,
 * scales whose product (or its quotient by softcap) leaves 1e-36 .. 1e36, and bounds of more rows than one launch takes.
 */
KV_API kv_status kv_attend(const kv_cache *cache, int32_t layer, const kv_batch *batch, const kv_attend_options *options,
                           const kv_rows *q, const kv_rows *out, float *lse, void *workspace, int64_t workspace_bytes,
                           void *stream);

/* Bytes of workspace that kv_attend needs for these arguments (host only; only the host's numbers count).  Negative:
 * the kv_status that kv_attend would return. */
KV_API int64_t kv_attend_workspace(const kv_cache *cache, const kv_batch *batch, const kv_attend_options *options,
                                   const kv_rows *q);

/*
 * kv_keep -- which tokens of each sequence (and KV head) a cache of `budget` tokens keeps.  A sequence of at most
 * `budget` tokens keeps all; a longer one its first `sinks`, its last `recent`, and the heaviest of the others, up to
 * `budget` in all; among equal weights the lower token is kept, and a NaN weighs less than any number.
 *   weights:      DEVICE float, row (b, h) of max_len elements at b*seq_stride + h*head_stride;
 *   lens:         DEVICE int32[num_seqs];
 *   keep:         DEVICE int32[num_seqs][heads][budget]: the kept tokens, ascending, then -1;
 *   kept_lens:    DEVICE int32[num_seqs]: min(lens[b], budget);
 *   kept_weights: DEVICE float[num_seqs][heads][budget]: their weights, then 0; or NULL.
 *   workspace:    DEVICE, kv_keep_workspace's bytes (4-byte aligned; may be NULL for 0 bytes), as kv_attend's.
 * heads: one row per KV head, or 1 for a choice that all heads share.  Errors: KV_EINVAL (NULL, sizes; sinks + recent
 * > budget; a workspace that is too small), KV_EUNSUPPORTED (more than 65,535 sequences, more than 2^31 - 2^20
 * tokens), KV_EHIP.
 */
KV_API kv_status kv_keep(const float *weights, int64_t seq_stride, int64_t head_stride, const int32_t *lens,
                         int32_t num_seqs, int32_t heads, int32_t max_len, int32_t budget, int32_t sinks,
                         int32_t recent, int32_t *keep, int32_t *kept_lens, float *kept_weights, void *workspace,
                         int64_t workspace_bytes, void *stream);

/* Bytes of workspace that kv_keep needs (host only; 0 unless a few long rows are cut).  Negative: a kv_status. */
KV_API int64_t kv_keep_workspace(int32_t num_seqs, int32_t heads, int32_t max_len, int32_t budget);

/*
 * kv_compact -- copy the kept tokens' K and V rows of layer `layer` into the pages of dst_tables: for j < kept_lens[b],
 * token keep[b][h][j] of source becomes token j of the destination, for KV head h (heads == 1: keep[b][0][j] for every
 * head).  Destination pages are distinct, and none of them is a source page of the call (precondition; otherwise the
 * result depends on the order of reads and writes): pages of a shared prefix stay as they are for their other users.
 * Every other byte of the cache is untouched.  From then on a kept token's place is its new slot: later calls count
 * causality, `window` and `slopes` in those, so distances to kept tokens shrink by what was left out between (for each
 * head by what that head left out).  A caller whose bias goes by the old distances has to carry it elsewhere, for
 * example in K, as rotated embeddings do.
 *   block_tables, dst_tables: DEVICE int32[num_seqs][stride], of which table_len and dst_len entries may be read.
 * Errors: KV_EINVAL (NULL, sizes; budget > dst_len * BS), KV_EUNSUPPORTED as kv_append, KV_EHIP.
 */
KV_API kv_status kv_compact(const kv_cache *cache, int32_t layer, int32_t num_seqs, const int32_t *block_tables,
                            int64_t table_stride, int32_t table_len, const int32_t *keep, int32_t heads,
                            int32_t budget, const int32_t *kept_lens, const int32_t *dst_tables, int64_t dst_stride,
                            int32_t dst_len, void *stream);

/* Device-side faults of these operators on the current device since the last clear (bitmask of KV_ASYNC_*; 0 if none),
 * meaningful after the caller has synchronised the streams it used; clear != 0 resets the word.  One word per device
 * and process.  Waits for the copy of that word; negative: a kv_status. */
KV_API int32_t kv_attend_async_error(int clear);

#ifdef __cplusplus
}
#endif

#endif /* KVX_ATTEND_H */
