/*
 * kvx_attend -- operators on a replica's paged KV cache (kv_cache of kvx.h), on AMD Instinct MI355X
 * (gfx950): what a replica computes on a cache that kv_load restored and kv_store will publish.
 *
 *   kv_append   the new tokens' K/V rows into the cache's pages (as they are, or as e4m3 with a scale);
 *               kv_append_scaled: as e4m3 with a scale for each page, K or V, and head
 *   kv_rotate   the new tokens' queries and keys normed for each head and rotated by their position; the keys, with
 *               the values, into the cache's pages
 *   kv_attend   attention of the new tokens over their sequence's cached tokens, from one new token per
 *               sequence to the tail of a prompt behind a restored prefix, and the weight that every
 *               cached token received
 *   kv_attend_pages  the same over pages with scales of their own, or over the pages alone that each new token chose
 *   kv_bounds   of each page the lowest and the highest K in every column
 *   kv_score    from these, what no token of a page can exceed with a new token's queries: a score to choose pages by
 *   kv_keep     from accumulated weights: the tokens that a sequence keeps under a budget (and from the scores of
 *               pages, the pages that a token attends over)
 *   kv_compact  the kept tokens' rows into fresh pages
 *
 * Conventions are kvx.h's: a plain C ABI, explicit HOST and DEVICE pointers, streams as void*, a kv_status from
 * every entry point (kv_last_error has the reason), nothing enqueued when an argument is refused.  Each call works on
 * one layer of the cache, on the current device, which must be the cache's, and only enqueues kernels on `stream`: it
 * allocates nothing, never blocks the host, keeps nothing between calls and may be captured into a graph.  All reads
 * and writes of a call follow earlier work on `stream` and precede later work there; calls on different streams are
 * ordered by the caller where they share a written buffer (a cache, an output or a workspace).  DEVICE arrays are read
 * and written until the call's work has completed there.  Outputs overlap neither inputs nor the workspace, unless
 * said.
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
#define KV_DTYPE_F32 4   /* norms' weights only */

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

/* The scales of an E4M3 cache's pages: a value is the stored e4m3 times 2^(e - 127), e the byte of its block, K (0) or
 * V (1), and head, at data + block*block_stride + kv*kv_stride + head; e is 1 to 254.  (Where kv_stride is padded to 16
 * bytes and block_stride is twice that, a layer's bytes are a kv_cache of their own with one token a block, which
 * kv_store and kv_load move by the same block tables, n / BS tokens rounded up: num_kv_heads 1, head_dim the padded
 * heads, elem_bytes 1, block_size 1, chunk_tokens C / BS.) */
typedef struct kv_page_scales {
    uint8_t *data;         /* DEVICE */
    int64_t block_stride;  /* bytes, >= kv_stride + heads */
    int64_t kv_stride;     /* bytes, >= heads */
} kv_page_scales;

/* The pages that each new token chose, for each KV head (heads == 1: the same for all): of row r and head h the first
 * counts[r] of the `budget` numbers at pages + r*token_stride + h*head_stride, each a place in its sequence's block
 * table, as kv_keep leaves them, but in any order.  A page that is named twice takes part twice. */
typedef struct kv_page_list {
    const int32_t *pages;  /* DEVICE */
    const int32_t *counts; /* DEVICE int32[num_queries] */
    int64_t token_stride;  /* elements, >= 0 */
    int64_t head_stride;
    int32_t heads;         /* the cache's KV heads, or 1 */
    int32_t budget;        /* most pages of a row, >= 1 */
} kv_page_list;

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
 * slopes[query head] * (p - t), with p the query's own token and t the cached one.  Token t takes part where t <= p
 * and, with window > 0, p - t < window.  Zero-initialised fields take the documented defaults. */
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
 * kv_append_scaled -- kv_append into an E4M3 cache whose pages have scales.  Of each page that a new token lies in, K
 * and V, and head, the scale is the smallest power of two with |x| <= 448 * scale for every finite x of the call's new
 * rows in it, and not smaller than it was where the page holds older tokens (of a page whose slot 0 is a new token's
 * nothing is older).  Where it grows, the older rows are rounded to it: e4m3(stored * old scale / new scale), which is
 * exact but for what leaves e4m3's normal numbers.  x is stored as e4m3(clamp(x / scale, -448, 448)), rounded to
 * nearest even; NaN stays NaN.  Every other byte of the cache and of the scales is untouched.  kv_compact does not move
 * scales.
 * Errors and preconditions as kv_append; KV_EINVAL also for strides of scales that overlap.
 */
KV_API kv_status kv_append_scaled(const kv_cache *cache, int32_t layer, const kv_batch *batch, const kv_rows *k,
                                  const kv_rows *v, const kv_page_scales *scales, void *stream);

/* Options of kv_rotate.  Zero-initialised fields take the documented defaults. */
typedef struct kv_rotate_options {
    int32_t cache_dtype;       /* KV_DTYPE_*: what the cache's elements are (required) */
    int32_t rotary_dim;        /* columns that are rotated, the first ones of a row: even, 0 to D */
    int32_t interleaved;       /* pairs of columns i: 0: (i, i + rotary_dim / 2); 1: (2i, 2i + 1) */
    int32_t weight_dtype;      /* of q_weight and k_weight: KV_DTYPE_F32, or the rows' type */
    const double *freqs;       /* DEVICE double[rotary_dim / 2]: radians per position of each pair */
    const int32_t *positions;  /* DEVICE int32[num_queries], or NULL: a token's place in its sequence */
    const void *q_weight;      /* DEVICE [D], or NULL: queries are not normed */
    const void *k_weight;      /* DEVICE [D], or NULL: keys are not normed */
    float eps;                 /* of the norms, >= 0 */
    float weight_offset;       /* added to the norms' weights */
    float magnitude;           /* factor of the rotated columns; 0 = 1 */
    float k_scale, v_scale;    /* 0 = 1; as in kv_append */
    int32_t reserved;          /* must be 0 */
    const kv_page_scales *scales;  /* HOST, or NULL; E4M3 caches: kv_append_scaled's; k_scale and v_scale are then 1 */
} kv_rotate_options;

/*
 * kv_rotate -- norm, rotate, and append.  Of each new token's row x of each head of q and k:
 *   y_d = x_d / sqrt(mean of x^2 + eps) * (weight_offset + weight_d)  (or x_d, without weights), and for each pair (a, b)
 *   of the first rotary_dim columns, with t = position * freqs[i]: (a cos t - b sin t, b cos t + a sin t) * magnitude.
 * A row is rounded once, at the end; sums are held in 32 bits (so a normed row's |x| stay under 1e18, and where eps is
 * 0 the largest over 1e-18), positions times frequencies in 64.  q's rows go to `out` (same type and heads; may be q
 * itself), k's rotated rows and v's as they are into layer `layer` of the cache, as kv_append, or with scales
 * kv_append_scaled, puts them there.  A row whose token has no place (before token 0) is rotated by its place or
 * position all the same; rows of no sequence are left as they were.
 * Errors and preconditions as kv_append; KV_EINVAL also for a rotary_dim that is odd or outside [0, D], a NULL freqs
 * with one, and numbers that are negative or not finite.
 */
KV_API kv_status kv_rotate(const kv_cache *cache, int32_t layer, const kv_batch *batch, const kv_rotate_options *options,
                           const kv_rows *q, const kv_rows *out, const kv_rows *k, const kv_rows *v, void *stream);

/*
 * kv_attend -- out[row] = v_scale * sum over its tokens of softmax(s) * v, rounded once to q's type, and lse[row] = log
 * of the sum of exp(s), for every new row; query head h reads KV head h / (q->heads / H).  A row that sees no token
 * gets 0 and -infinity.  Sums, largest scores and lse are held in 32 bits.  The weights exp(s) meet V as two numbers of
 * q's type (the rounded weight and what it leaves) for sequences of up to 64 rows (new tokens times query heads) per KV
 * head, so that only the output's rounding shows.  For longer ones they are one number, rounded to nearest (off by up
 * to half a step of that type each), unless full_weights asks for two there as well.  What slots behind a sequence's
 * last token hold does not matter, but its own tokens' V are taken to be finite: 0 times an infinity of a token that a
 * row does not see reaches that row.  K of a token reaches the rows that see it and no others; where it is not finite,
 * they may become NaN.
 *   q, out:    [num_queries][query heads][D], same type; the cache's, or either 2-byte type for E4M3; rows of out do not
 *              overlap;
 *   lse:       DEVICE float[num_queries][query heads], or NULL;
 *   workspace: DEVICE, kv_attend_workspace's bytes (16-byte aligned; may be NULL for 0 bytes), the call's own until its
 *              work has completed: calls that may overlap, and graphs whose replays may, need one each.
 * Errors as kv_append; KV_EINVAL for a workspace that is too small; KV_EUNSUPPORTED also for more than 16,383 query
 * heads, scales whose product (or its quotient by softcap) leaves 1e-36 .. 1e36, and bounds of more rows than one
 * launch takes.
 */
KV_API kv_status kv_attend(const kv_cache *cache, int32_t layer, const kv_batch *batch, const kv_attend_options *options,
                           const kv_rows *q, const kv_rows *out, float *lse, void *workspace, int64_t workspace_bytes,
                           void *stream);

/* Bytes of workspace that kv_attend needs for these arguments (host only; only the host's numbers count).  Negative:
 * the kv_status that kv_attend would return. */
KV_API int64_t kv_attend_workspace(const kv_cache *cache, const kv_batch *batch, const kv_attend_options *options,
                                   const kv_rows *q);

/*
 * kv_attend_pages -- kv_attend where an E4M3 cache's pages have scales (scales; options' k_scale and v_scale are then
 * 1), where each new token attends over the pages alone that it chose (list), or both; one of them must be given.
 * Token t of a chosen page takes part where t <= p and, with window > 0, p - t < window, and slopes count in p - t, as
 * in kv_attend; a row that chose nothing that it sees gets 0 and -infinity, and pages that a row sees no token of are
 * not looked up in its table.  Weights always meet V as two numbers, whatever the rows and full_weights, so that only
 * the output's rounding shows (with scales, and with a list in any E4M3 cache, in bfloat16).  With a list a V that is
 * not finite reaches no row that does not see it, and each row reads its pages for itself.  weights_in and weights_out
 * must be NULL.  Errors as kv_attend; KV_EINVAL also for a list that contradicts the cache, KV_EUNSUPPORTED for
 * weights_out, more than 2^31 - 1024 tokens in `budget` pages, and more rows than one launch takes.
 */
KV_API kv_status kv_attend_pages(const kv_cache *cache, int32_t layer, const kv_batch *batch,
                                 const kv_attend_options *options, const kv_page_scales *scales,
                                 const kv_page_list *list, const kv_rows *q, const kv_rows *out, float *lse,
                                 void *workspace, int64_t workspace_bytes, void *stream);

/* Bytes of workspace that kv_attend_pages needs, as kv_attend_workspace. */
KV_API int64_t kv_attend_pages_workspace(const kv_cache *cache, const kv_batch *batch, const kv_attend_options *options,
                                         const kv_page_scales *scales, const kv_page_list *list, const kv_rows *q);

/*
 * kv_bounds -- of each page of layer `layer` that a new token lies in, and each KV head, the lowest and the highest
 * stored K of every column over the page's tokens t < lens[b], new and older ones.  They go where `bounds`, a kv_cache
 * of the same heads, head_dim and elem_bytes with block_size 1 and at least as many blocks, has K and V of the same
 * block's one token, in the cache's own type (kv_store and kv_load move it as any cache, by the same tables).  Of an
 * E4M3 cache these are stored values; scales apply to them as to the page.  A NaN does not count; a column without a
 * number gets 0 twice. Bounds of other pages are untouched.  For a restored prefix all its tokens are new ones (lens[b]
 * of them).
 * Errors as kv_append; KV_EINVAL also for bounds that contradict the cache.
 */
KV_API kv_status kv_bounds(const kv_cache *cache, int32_t layer, const kv_batch *batch, int32_t cache_dtype,
                           const kv_cache *bounds, void *stream);

/* Options of kv_score. */
typedef struct kv_score_options {
    int32_t cache_dtype;  /* KV_DTYPE_*: what the bounds' elements are (required) */
    int32_t block_size;   /* tokens of a page of the cache that the bounds are of */
    float scale;          /* 0 = 1; e.g. kv_attend's scale times k_scale */
    int32_t reserved;     /* must be 0 */
    const kv_page_scales *scales;  /* HOST, or NULL: E4M3 pages' scales, of which K's are read */
    int64_t token_stride, head_stride;  /* elements between rows of scores */
} kv_score_options;

/*
 * kv_score -- for each new row r of token p, KV head h, and page j <= p / block_size of its sequence,
 *   scores[r*token_stride + h*head_stride + j] = scale * max over the query heads of h of sum_d max(q_d low_d, q_d high_d):
 * no token of the page has a larger scale * (q . k) with any of these heads.  Sums are held in 32 bits; where bounds
 * are not finite a score may be NaN.  A page whose block id is bad gets -infinity.  counts[r] = p / block_size + 1 (0
 * for a row before token 0): kv_keep's lens for num_queries "sequences" of pages.  Scores of pages from there on are
 * left as they were.
 *   bounds: kv_bounds's; batch: the sequences as in kv_attend, max_len in tokens, at most table_len * block_size;
 *   scores: DEVICE float, rows of (max_len + block_size - 1) / block_size elements that do not overlap;
 *   counts: DEVICE int32[num_queries], or NULL.
 * Errors as kv_attend.
 */
KV_API kv_status kv_score(const kv_cache *bounds, int32_t layer, const kv_batch *batch, const kv_score_options *options,
                          const kv_rows *q, float *scores, int32_t *counts, void *stream);

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
