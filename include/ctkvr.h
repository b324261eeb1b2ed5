/*
 * ctkvr.h -- C ABI of the MI355X (gfx950) implementation of CTkvr's data-parallel
 * hot path: the query-centroid inverted file built at prefill (Algorithm 1,
 * lines 1-4 of the paper) and the per-decode-step centroid-then-token retrieval
 * followed by sparse attention (Algorithm 2, lines 1-9).
 *
 * Notation (the paper's): b batch, h query heads, g KV heads, G = h/g, d head
 * dimension, s context length, C query centroids per head, C' probed centroids
 * (n_probe), rho keys per inverted list (list_len), rho' sparsity budget (top_k).
 * Query heads i*G .. (i+1)*G-1 share KV head i (Section 3.1.1, footnote on
 * grouped-query attention).
 *
 * Conventions
 *   - Every tensor pointer is a DEVICE pointer owned by the caller unless the
 *     comment says HOST.  The library never frees caller memory and keeps no
 *     reference to it after a call returns, except where stated.
 *   - Work is enqueued on the HIP stream passed as `hip_stream` (a hipStream_t
 *     cast to void*; NULL = the default stream).  ctkvr_decode_step does not
 *     synchronise and does not allocate.
 *   - Functions return CTKVR_OK (0) or a negative ctkvr_status; nothing is thrown
 *     across the boundary.  ctkvr_last_error() gives a thread-local message for
 *     the last non-OK return.  Argument errors are detected on the host before
 *     anything is launched.
 *   - The KV cache is paged: k_pages / v_pages are
 *     [num_pages][g][page_size][d] elements of `dtype`; token t of sequence i
 *     lives in page block_table[i*max_pages + t/page_size], slot t%page_size.
 *   - head_dim must be 128 and G one of 1, 2, 4, 8, else CTKVR_EUNSUPPORTED.
 *   - Selections break ties towards the lowest id and are reported in ascending
 *     id order.
 */
#ifndef CTKVR_H
#define CTKVR_H

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct ctkvr_index ctkvr_index;   /* opaque: centroids, their inverse norms, inverted lists, workspace */

typedef enum {
    CTKVR_OK = 0,
    CTKVR_EINVAL = -1,        /* bad argument (null pointer, C' > C, rho > s, h % g != 0, ...) */
    CTKVR_ENOMEM = -2,        /* device or host allocation failed */
    CTKVR_EHIP = -3,          /* a HIP runtime call failed */
    CTKVR_EUNSUPPORTED = -4   /* valid in the paper, not supported by this build (head_dim != 128, ...) */
} ctkvr_status;

typedef enum { CTKVR_F32 = 0, CTKVR_BF16 = 1 } ctkvr_dtype;

typedef enum {
    CTKVR_CENTROID_LAST_C = 0,   /* Algorithm 1 line 1: the last C prompt queries */
    CTKVR_CENTROID_KMEANS = 1    /* Lloyd iterations over the prompt queries replace line 1 only */
} ctkvr_centroid_mode;

typedef enum {
    CTKVR_BUILD_EXACT = 0,   /* list scores in the fixed fp32 arithmetic of the decode path (bit-reproducible) */
    CTKVR_BUILD_MFMA = 1     /* list scores on the matrix cores (bf16 inputs only); lists may differ from
                                EXACT only for keys whose score ties the rho-th within rounding */
} ctkvr_build_algo;

typedef struct {
    int32_t batch;           /* b */
    int32_t n_q_heads;       /* h */
    int32_t n_kv_heads;      /* g */
    int32_t head_dim;        /* d, must be 128 */
    int32_t page_size;       /* tokens per KV page (16 in the benchmark workloads) */
    int32_t dtype;           /* ctkvr_dtype of q, K, V and the centroid table */
    int32_t n_centroids;     /* C; 0 => per sequence C_i = ctx_len_i / centroid_div */
    int32_t centroid_div;    /* used when n_centroids == 0 */
    int32_t list_len;        /* rho  (Algorithm 1 line 4) */
    int32_t n_probe;         /* C'   (Algorithm 2 line 3) */
    int32_t top_k;           /* rho' (Algorithm 2 line 6) */
    float   sm_scale;        /* softmax scale applied to q.k; 0 => 1/sqrt(head_dim) */
    int32_t centroid_mode;   /* ctkvr_centroid_mode */
    int32_t kmeans_iters;    /* Lloyd iterations when centroid_mode == KMEANS */
    int32_t build_algo;      /* ctkvr_build_algo */
    int32_t n_init;          /* L_init: the first n_init keys stay with the attention (Algorithm 1 lines 5-6) */
    int32_t n_local;         /* L_local: so do the last n_local keys of the prompt; neither enters a list */
} ctkvr_params;

/*
 * Index construction at prefill (Algorithm 1, lines 1-4).
 *   q_prefill   post-RoPE prompt queries, [total_rows][h][d] of `dtype`, sequences
 *               concatenated; cu_seqlens (HOST, batch+1 entries) gives each
 *               sequence's row range.  With q_is_tail = 1 a sequence contributes
 *               only the queries of its last C_i prompt positions (all LAST_C needs);
 *               with q_is_tail = 0 it contributes all ctx_len_i of them.
 *   k_pages, block_table, max_pages   the paged key cache (see above).
 *   ctx_lens    HOST, [batch]: s of every sequence.  The index is built over keys
 *               0 .. s-1 and stays valid for decode steps over that frozen prefix.
 *   init_pos    KMEANS only, DEVICE int32 [batch][g][C]: prompt positions whose
 *               queries seed the centres (e.g. from k-means++ run by the caller).
 * For every sequence, KV head and centroid j the list holds the rho keys with the
 * largest max over the group's query heads of softmax_t(c_{h,j} . k_t * sm_scale)
 * taken over all s keys (lines 2-4), ascending; with n_init, n_local > 0 the rho keys are
 * chosen among keys n_init .. s - n_local - 1 only (the scores are unchanged).
 * On success *out_index owns device memory until ctkvr_free.  The call
 * synchronises the stream before returning.
 * Errors: EINVAL for null/inconsistent arguments (C_i < n_probe, rho > s_i - n_init - n_local, ...);
 * EUNSUPPORTED for head_dim != 128, G not in {1,2,4,8}, MFMA build with f32 data.
 */
int ctkvr_build_index(const ctkvr_params *p, const void *q_prefill, const int32_t *cu_seqlens, int32_t q_is_tail,
                      const void *k_pages, const int32_t *block_table, int32_t max_pages, const int32_t *ctx_lens,
                      const int32_t *init_pos, void *hip_stream, ctkvr_index **out_index);

/*
 * Wrap an index built elsewhere (Algorithm 1's outputs) so that decode steps can
 * run on it.  All pointers HOST: centroids [batch][h][C_max][d] of `dtype`
 * (C_max = max_i C_i; rows j >= C_i unused), lists int32 [batch][g][C_max][rho]
 * ascending key ids, ctx_lens [batch].  The data is copied; inverse centroid
 * norms are recomputed on the device.
 */
int ctkvr_index_load(const ctkvr_params *p, const int32_t *ctx_lens, const void *centroids, const int32_t *lists,
                     void *hip_stream, ctkvr_index **out_index);

/*
 * One decode step of retrieval + sparse attention for every sequence of the
 * batch (Algorithm 2, lines 1-9):
 *   lines 1-3  cosine of q_h to every centroid of head h, max over the group,
 *              top-C' centroids per KV head;
 *   line  4    union of their lists, deduplicated -> L recalled key ids;
 *   lines 5-6  max over the group of softmax(q . K^Recall * sm_scale) over the
 *              recalled keys, top-rho' key ids;
 *   lines 7-9  softmax(q . K^sparse * sm_scale) V^sparse per query head.
 *   q          [batch][h][d] post-RoPE, `dtype`.
 *   out        fp32 [batch][h][d].
 * Optional outputs (NULL to skip):
 *   out_lse    fp32 [batch][h]: natural-log sum of exp of the scaled logits over
 *              the selected keys (lets a caller merge a resident window later);
 *   out_sel    int32 [batch][g][rho'] selected key ids ascending, -1 padded when L < rho';
 *   out_ncand  int32 [batch][g]: L;
 *   out_probe  int32 [batch][g][C'] probed centroid ids ascending.
 * The KV cache must hold the same first ctx_len_i keys the index was built on.
 * The integers are the same in every call with the same arguments.  out and out_lse are too, except that in
 * a larger batch's one launch behind the scoring (CTKVR_TAIL = 2 below) a block whose bounded wait for its siblings'
 * words expires, as beside other work that holds the compute units, sums in another order: they may then differ in rounding.
 * Asynchronous on hip_stream; uses the index's workspace, so steps on one index
 * must not overlap.  Errors: EINVAL (null required pointer, max_pages too small).
 */
int ctkvr_decode_step(ctkvr_index *idx, const void *q, const void *k_pages, const void *v_pages,
                      const int32_t *block_table, int32_t max_pages, float *out, float *out_lse, int32_t *out_sel,
                      int32_t *out_ncand, int32_t *out_probe, void *hip_stream);

/*
 * The decode step with the resident window (Algorithm 2 lines 1-11; Section 3.2): as
 * ctkvr_decode_step, and in addition every query head attends over the first n_init keys and
 * over the keys from ctx_len_i - n_local to cur_lens[i] - 1, and the two attention outputs are
 * merged through their log-sum-exps (line 11), which equals attention over the union.
 *   cur_lens   DEVICE int32 [batch] or NULL: tokens of each sequence now in the KV cache,
 *              cur_lens[i] >= ctx_len_i.  The tokens decoded since the index was built belong
 *              to the local window; the caller appends their keys and values to the paged cache.
 *              NULL means cur_lens[i] = ctx_len_i.  Values are clamped to
 *              [ctx_len_i, max_pages * page_size].
 * The lists of an index built with n_init, n_local > 0 hold no window key, so nothing is
 * counted twice.  out_lse is the log-sum-exp over selected and window keys together.
 * ctkvr_decode_step on such an index is this call with cur_lens = NULL.
 * Errors: as ctkvr_decode_step.
 */
int ctkvr_decode_step_window(ctkvr_index *idx, const void *q, const void *k_pages, const void *v_pages,
                             const int32_t *block_table, int32_t max_pages, const int32_t *cur_lens, float *out,
                             float *out_lse, int32_t *out_sel, int32_t *out_ncand, int32_t *out_probe, void *hip_stream);

/*
 * ctkvr_decode_step for callers that cannot allocate device memory or tolerate a call that
 * does (code under HIP graph capture, tight serving loops, harnesses that forbid hipMalloc):
 * the same step with the same arguments, results and errors, but every intermediate buffer of
 * the step (cosines, recall bitmap, recalled ids and rows, logits, ranking keys and their
 * histogram, the selection's bitmap and list, the selected rows and logits) lives in a static
 * device array of the library, 36 MiB per GPU, instead of the workspace `idx` owns.  The call
 * allocates and frees nothing, on the host side of HIP or through it; the array's device
 * address is looked up on the first call on each device.
 *   - The step's buffers must fit 32 MiB of it (the rest is for the words that blocks of a launch hand to each other): about
 *       units * (l_stride * (16 + 4 G) + 4 C_max + s_max / 8 + top_k * (8 + 4 G) + 30 KiB)
 *     bytes, units = batch * g, plus, on geometries that allow the single-launch form (units at most
 *     the number of compute units), units * 32 * (4 top_k + 21 KiB) for its per-block slots (the 32K
 *     benchmark workload takes about 15 MiB).  Larger geometries return CTKVR_EUNSUPPORTED before
 *     anything is launched.
 *   - Every call on a GPU shares that GPU's array, whichever index it serves: calls that
 *     overlap on one GPU (different streams, different threads) race.  The call clears what a
 *     step expects to find zero, so it may follow a call for any other index.
 *   - ctkvr_centroid_update and ctkvr_index_last_candidates read the workspace `idx` owns: they
 *     follow ctkvr_decode_step, not this call.
 */
int ctkvr_decode_step_static(ctkvr_index *idx, const void *q, const void *k_pages, const void *v_pages,
                             const int32_t *block_table, int32_t max_pages, float *out, float *out_lse, int32_t *out_sel,
                             int32_t *out_ncand, int32_t *out_probe, void *hip_stream);

/*
 * Dynamic centroid update (Algorithm 2 line 12; Section 3.1.2, "Dynamic Centroid Update"),
 * to be called after ctkvr_decode_step with the same q, on the same stream, before the next
 * step: for every sequence and KV head the query vectors of the group's heads replace the
 * centroids of one slot of the index, and that slot's list becomes the rho keys with the
 * largest rerank score of the step (the quantity line 6 ranks by, over the recalled keys),
 * ties to the lowest id, ascending.  Slots are taken first in, first out: update number n
 * (counted from 0 since the build) writes slot n mod C_i, so the earliest prompt query goes
 * first.  With rho = rho' the list is the step's selection; otherwise the ranking is run
 * once more with budget rho.  Should fewer than rho keys have been recalled the last one is
 * repeated.  Asynchronous, allocates nothing, uses the index's workspace like a step.
 * Errors: EINVAL (null pointer; no decode step since the build or the last update).
 */
int ctkvr_centroid_update(ctkvr_index *idx, const void *q, void *hip_stream);

/* Release an index (NULL is allowed).  Synchronises the index's device first; where that is refused (a stream of it is being
 * captured) the index's memory is kept back until a later wait succeeds. */
void ctkvr_free(ctkvr_index *idx);

/* Thread-local description of the last non-OK return of this library. */
const char *ctkvr_last_error(void);

/* ---- the paged KV cache itself: append, dense attention, accumulated weights, eviction --------------- */
/*
 * What surrounds the index: filling the caller's pages with rotated keys, attending densely with the prompt's chunks and with
 * single tokens, and keeping a sequence within a budget of tokens by the attention that its keys have had.
 *
 * Tokens.  A call serves `batch` sequences with `total` new tokens, sequence after sequence: those of sequence b are cu_new[b] ..
 * cu_new[b + 1] - 1 (0, 1 or more; cu_new[0] = 0), and cur_lens[b] counts the tokens of b in the cache with the new ones among
 * them, so that new token i of n_b stands in slot (and, to the masks, at position) cur_lens[b] - n_b + i.  cu_new [batch + 1],
 * cur_lens [batch] and block_table [batch][max_pages] are DEVICE arrays: captured graphs stay valid as they change.
 * Outputs of tokens behind cu_new[batch] are left as they were.  A page id outside 0 .. num_pages - 1 (-1, say) is no page: nothing is
 * written there, and its keys are seen by no token.  Slots of cur_lens[b] beyond max_pages * page_size are no slots.
 *
 * Rows of q, k and v may be views of a wider array (a fused projection): *_stride is the distance from a token to the next in
 * elements, a token's heads are contiguous, and every row begins on a 16-byte boundary; so do pages and outputs.
 *
 * Each call is asynchronous on hip_stream, a stream of the device that was current when the handle was made (NULL: that device's default
 * stream; the calling thread's current device may be another), allocates nothing and can be captured into a HIP graph.
 * Attention (ctkvr_cache_attn and the calls of the next section that attend) uses the handle's workspace: two such calls on one handle must not overlap,
 * replays of graphs among them.
 * How a call is split goes by the mean of its tokens over the sequences and by the table's width: a prompt's chunk beside single tokens of other sequences is served
 * in one call, but faster in two, in each of which the other sequences have no new tokens.
 */
typedef struct ctkvr_cache ctkvr_cache;   /* opaque: geometry, rotary frequencies, workspace */

typedef struct {
    int32_t batch, n_q_heads, n_kv_heads;
    int32_t head_dim;            /* must be 128; n_q_heads / n_kv_heads one of 1, 2, 4, 8 */
    int32_t page_size;           /* a power of two up to 256 */
    int32_t dtype;               /* ctkvr_dtype of q, k, v, the pages and the attention's output */
    int32_t num_pages;           /* pages in k_pages and in v_pages */
    int32_t max_pages;           /* columns of the block table; max_pages * page_size at most 2^20 */
    int32_t max_new;             /* new tokens of a call, at most (over all sequences) */
    float   sm_scale;            /* factor of q.k, up to 1e15; 0 => 1/sqrt(head_dim) */
    float   softcap;             /* 0: none; else 1e-6 to 1e15: a score z becomes softcap * tanh(z / softcap) */
    double  rope_base;           /* frequency of pair i: rope_base^(-2 i / head_dim) */
    const double *rope_freq;     /* HOST [head_dim / 2] or NULL: these frequencies (radians per position) instead */
    const uint8_t *rope_axis;    /* HOST [head_dim / 2] or NULL (all 0): the axis, 0 to 2, that turns each pair */
} ctkvr_cache_params;

/* A handle on the current device; params' arrays are copied.  Clears words of its workspace (up to 73 MB of device memory) on hip_stream and synchronises it.
 * Errors: EINVAL, EUNSUPPORTED (as the index; a sequence of more than 2^20 tokens, a cache of 2^32 rows, more than 2^20 new tokens, 2^16
 * sequences or 2^10 heads, 2^22 or more KV heads of all sequences), ENOMEM. */
int ctkvr_cache_create(const ctkvr_cache_params *p, void *hip_stream, ctkvr_cache **out_cache);
/* Release a handle (NULL is allowed); synchronises its device first, as ctkvr_free does. */
void ctkvr_cache_free(ctkvr_cache *c);

/*
 * Rotate new queries and keys to their positions and write keys and values into their slots:
 *   x'_i = x_i cos a_i - x_{i+64} sin a_i,  x'_{i+64} = x_{i+64} cos a_i + x_i sin a_i,  a_i = position[axis_i] * frequency_i,
 * in fp32, rounded once to `dtype`; values are copied.  An angle is off by 2^-31 of a turn at any position (frequencies up to 2^32 radians), and by its
 * rounding to fp32 modulo a quarter of a turn.
 *   q, q_out   [total][h][128] (q_out contiguous; may be q where q is) or both NULL;  k, v  [total][g][128] or both NULL.
 *   positions  DEVICE int32 [axes][total], any values, for the axes that rope_axis names (text: the same on all), or NULL:
 *              the token's slot on every axis.  After an eviction slots are no positions any more.
 * No two sequences may write into one page's slot.  Errors: EINVAL.
 */
int ctkvr_cache_append(ctkvr_cache *c, const void *q, int64_t q_stride, const void *k, int64_t k_stride, const void *v, int64_t v_stride,
                       const int32_t *positions, const int32_t *cu_new, const int32_t *cur_lens, const int32_t *block_table, int32_t total,
                       void *q_out, void *k_pages, void *v_pages, void *hip_stream);

/*
 * Attention of the new tokens over the cache (which holds them already): per token and query head softmax(z) V over the keys it sees,
 *   z = cap(q . k * sm_scale) - slope_h * |pos - t|,
 * for key t of the token at pos:  first_key <= t < cur_lens[b]  and  (t <= pos or t < prefix_lens[b]).  pos and t are slots: in a cache that was
 * cut down the distance, first_key and prefix_lens count the tokens that are left, and those are others in each KV head.
 *   q           [total][h][128], rotated.
 *   slopes      DEVICE fp32 [h] or NULL: a bias by distance.
 *   prefix_lens DEVICE int32 [batch] or NULL: so many keys at the start are seen by every token, earlier ones too, from its first_key on.
 *   first_key   DEVICE int32 [total] or NULL: where the token's document begins (packed documents), or its window.
 *   out         [total][h][128] of `dtype`;  out_lse  fp32 [total][h] or NULL, natural log.
 * A token that sees no key, or none with a score above -infinity, gets zeros and -infinity.  What a token does not see does not touch its result,
 * infinities and NaN included.  Sums are fp32; with bf16 data the probabilities enter the product with V rounded to bf16.
 * The same call gives the same result, bit for bit.  Errors: EINVAL.
 */
int ctkvr_cache_attn(ctkvr_cache *c, const void *q, int64_t q_stride, const void *k_pages, const void *v_pages, const int32_t *cu_new,
                     const int32_t *cur_lens, const int32_t *block_table, int32_t total, const float *slopes, const int32_t *prefix_lens,
                     const int32_t *first_key, void *out, float *out_lse, void *hip_stream);

/*
 * The attention weight of every key of the batch under the new tokens:
 *   weights_out[b][kv][t] = decay * weights_in[b][kv][t] + sum over b's new tokens and the KV head's query heads of exp(z - lse)
 * with ctkvr_cache_attn's scores, masks and out_lse.  A key that the call's own tokens brought has no weight before it.
 *   lse          fp32 [total][h] of the attention (a row of -infinity adds nothing).
 *   weights_in   fp32 [batch][g][weights_stride] or NULL (zeros); weights_out likewise, may be weights_in.
 *                weights_stride >= max_pages * page_size; slots from cur_lens[b] on are left as they were.
 * With total = 0 the weights decay.  Sums are fp32, in an order of their own: the same result in every call.  Errors: EINVAL.
 */
int ctkvr_cache_weights(ctkvr_cache *c, const void *q, int64_t q_stride, const float *lse, const void *k_pages, const int32_t *cu_new,
                        const int32_t *cur_lens, const int32_t *block_table, int32_t total, const float *slopes, const int32_t *prefix_lens,
                        const int32_t *first_key, float decay, const float *weights_in, float *weights_out, int32_t weights_stride,
                        void *hip_stream);

/*
 * Cut every sequence longer than `budget` down to it: per sequence and KV head the first n_init and the last n_local tokens stay, and
 * of those in between the budget - n_init - n_local with the largest weights, ties to the lowest slot (-0 equals +0, NaN is below
 * -infinity).  The kept rows of K and V move to the front in place, in order: slot j then holds what slot out_ids[b][kv][j] held.
 *   weights_in  as ctkvr_cache_weights leaves them;  weights_out  the same shape or NULL, may be weights_in: the kept weights, moved alike.
 *   out_ids     int32 [batch][g][budget] ascending, -1 padded.
 *   out_lens    int32 [batch] or NULL: min(cur_lens[b], budget).  May be cur_lens, so that a captured step keeps one array of lengths (one
 *               more launch); an array that overlaps it otherwise is refused.
 * Pages that no kept token needs any more are the caller's again; slots from out_lens[b] on hold what they held before or moved rows.  A row whose
 * old or new page is no page is not moved.  Sequences must not share the pages.  Errors: EINVAL.
 */
int ctkvr_cache_evict(ctkvr_cache *c, const float *weights_in, int32_t weights_stride, const int32_t *cur_lens, const int32_t *block_table,
                      int32_t budget, int32_t n_init, int32_t n_local, void *k_pages, void *v_pages, float *weights_out, int32_t *out_ids,
                      int32_t *out_lens, void *hip_stream);

/* ---- the paged KV cache in 8 bits, in a window, with drafted tokens ------------------------------------ */
/*
 * Rows of 8 bits.  k_codes and v_codes [num_pages][g][page_size][128] hold a byte an element, k_scales and v_scales [num_pages][g][page_size] an fp32
 * scale a row: element i of a row is its code times its scale.  A row x is held as
 *   scale = max |x_i| / top,  code_i = x_i * top / max |x_i| to the nearest code, ties to even;  top = 127 (int8, -127 to 127) or 448 (e4m3),
 * computed in fp32: a value is off by half a step of its row at most, max |x_i| / 254, or in e4m3 by 2^-4 of itself (from max |x_i| * 2^-14.8 on; below by
 * max |x_i| * 2^-18.8).  A row that holds an infinity or NaN is NaN as a whole, with codes of 0 and a scale of NaN.  e4m3's codes for NaN are written by no
 * call; what they are read as is not said.
 * The calls below follow ctkvr_cache_*'s rules for tokens, rows, pages, streams, graphs and the workspace (which every attention uses), and take the
 * same handle, whose dtype is that of q, k, v, out and of plain rows.
 */
typedef enum { CTKVR_KV_PLAIN = 0, CTKVR_KV_INT8 = 1, CTKVR_KV_FP8 = 2 } ctkvr_kv_format;

/* ctkvr_cache_append into rows of 8 bits (format: INT8 or FP8).  Keys are rotated in fp32 and rounded once, to their codes; q and q_out may both be NULL, k and v
 * may not.  No two sequences may write into one page's slot.  Errors: EINVAL. */
int ctkvr_cache_quant_append(ctkvr_cache *c, const void *q, int64_t q_stride, const void *k, int64_t k_stride, const void *v, int64_t v_stride,
                             const int32_t *positions, const int32_t *cu_new, const int32_t *cur_lens, const int32_t *block_table, int32_t total,
                             void *q_out, int32_t format, void *k_codes, float *k_scales, void *v_codes, float *v_scales, void *hip_stream);

/*
 * Read rows of 8 bits back into plain pages, of which the index, the decode step, the weights and eviction read: token t of sequence b, first_tokens[b] <= t <
 * cur_lens[b], goes to slot t - first_tokens[b] of out_table's row b, code times scale in fp32, rounded once to `dtype`.
 *   first_tokens  DEVICE int32 [batch] or NULL: zeros (negative ones count as 0).
 *   out_table     DEVICE int32 [batch][out_max_pages], pages 0 .. out_num_pages - 1 of k_pages and v_pages [out_num_pages][g][page_size][128], of the handle's
 *                 page_size.  Rows from or to a page that is none are left out, and tokens beyond either table.  No two tokens may go to one slot.
 *   k_pages       or v_pages may be NULL: not read, nor its codes and scales.
 * Errors: EINVAL.
 */
int ctkvr_cache_quant_read(ctkvr_cache *c, int32_t format, const void *k_codes, const float *k_scales, const void *v_codes, const float *v_scales,
                           const int32_t *first_tokens, const int32_t *cur_lens, const int32_t *block_table, const int32_t *out_table, int32_t out_max_pages,
                           int32_t out_num_pages, void *k_pages, void *v_pages, void *hip_stream);

/*
 * ctkvr_cache_attn over rows of 8 bits (format: INT8 or FP8): the same scores, masks and results, on the values that the codes stand for.  Queries are not
 * rounded; their products with a row's codes, which the row's scale multiplies afterwards, are fp32 sums (finite for queries below 2^112, whatever the scales).  A probability
 * times its value's scale enters the product in fp16, with fp32 data as the sum of two such numbers, under a power of two of the row's own: it is off by 2^-11 of itself (2^-22)
 * or, if it is small, by 2^-35 of the largest magnitude of a scale that the row sees, or of 2^-80 if that is more.  Scales are finite, of either sign, or NaN for a row that is
 * NaN; scales and codes that no token sees may be anything.
 * Errors: EINVAL.
 */
int ctkvr_cache_quant_attn(ctkvr_cache *c, const void *q, int64_t q_stride, int32_t format, const void *k_codes, const float *k_scales, const void *v_codes,
                           const float *v_scales, const int32_t *cu_new, const int32_t *cur_lens, const int32_t *block_table, int32_t total,
                           const float *slopes, const int32_t *prefix_lens, const int32_t *first_key, void *out, float *out_lse, void *hip_stream);

/*
 * ctkvr_cache_attn in a sliding window beside the first tokens: the token at pos sees key t where
 *   t <= pos  and  (t > pos - window or t < n_sink),
 * over plain rows (format PLAIN, scales NULL) or rows of 8 bits (as in ctkvr_cache_quant_attn).  What it costs goes by the window, not by the cache.  Pages that lie before every
 * window of a sequence and behind its first n_sink tokens are not needed any more: their entries of the table may be -1, or pages of other sequences.
 *   window  1 or more (the token itself counts);  n_sink  0 or more.
 * Roundings and sums as there: over plain bf16 rows the probabilities enter the product with V rounded to bf16.  Errors: EINVAL.
 */
int ctkvr_cache_window_attn(ctkvr_cache *c, const void *q, int64_t q_stride, int32_t format, const void *k_pages, const float *k_scales, const void *v_pages,
                            const float *v_scales, const int32_t *cu_new, const int32_t *cur_lens, const int32_t *block_table, int32_t total, int32_t window,
                            int32_t n_sink, const float *slopes, void *out, float *out_lse, void *hip_stream);

/*
 * Attention of drafted tokens that branch: the new tokens of a sequence are a tree (or any order), each in a slot of its own, of which token i sees the
 * keys before the new tokens, from its first_key on, and those new tokens whose bits it has:
 *   tree_mask  DEVICE uint32 [total][mask_words]: bit j % 32 of word j / 32 of a token's row says that it sees the j-th new token of its sequence (itself
 *              only with its own bit; tokens beyond 32 * mask_words are not seen).
 *   first_key  DEVICE int32 [total] or NULL: it sees no key, new ones included, in an earlier slot.
 * Over plain rows (format PLAIN, scales NULL) or rows of 8 bits (as in ctkvr_cache_quant_attn).  The cache was appended to with the draft's own positions (a token's depth in its tree behind the
 * tokens before it); the tokens that are kept in the end go to their slots in order by another append, of their k and v, with cur_lens counting them alone.
 * A token that sees no key gets zeros and -infinity.  Roundings and sums as in ctkvr_cache_attn, over 8-bit rows as in ctkvr_cache_quant_attn.  Errors: EINVAL.
 */
int ctkvr_cache_tree_attn(ctkvr_cache *c, const void *q, int64_t q_stride, int32_t format, const void *k_pages, const float *k_scales, const void *v_pages,
                          const float *v_scales, const int32_t *cu_new, const int32_t *cur_lens, const int32_t *block_table, int32_t total,
                          const uint32_t *tree_mask, int32_t mask_words, const int32_t *first_key, void *out, float *out_lse, void *hip_stream);

/* ---- inspection (tests, tooling); each synchronises ----------------------- */
typedef struct {
    int32_t batch, n_q_heads, n_kv_heads, head_dim, dtype;
    int32_t c_max;           /* centroid rows allocated per head */
    int32_t list_len, n_probe, top_k;
    int32_t l_stride;        /* candidate slots per (sequence, KV head): max_i min(s_i, C' * rho) */
    int64_t index_bytes;     /* bytes of the inverted lists: b * g * C_max * rho * 4 */
    int64_t device_bytes;    /* everything the index holds on the device (kept memory it was given may be a quarter more than it needs) */
} ctkvr_index_info_t;

int ctkvr_index_info(const ctkvr_index *idx, ctkvr_index_info_t *out);
/* Copy out the inverted lists, int32 [batch][g][C_max][rho], to HOST memory. */
int ctkvr_index_lists(const ctkvr_index *idx, int32_t *dst_host);
/* Copy out the centroid table, [batch][h][C_max][d] of `dtype`, to HOST memory. */
int ctkvr_index_centroids(const ctkvr_index *idx, void *dst_host);
/* Recalled key ids of the last decode step, int32 [batch][g][l_stride] (first L valid), to HOST memory. */
int ctkvr_index_last_candidates(const ctkvr_index *idx, int32_t *dst_host);

/* ---- per-kernel timing (measurement aid) ----------------------------------- */
/* The decode step runs these kernels in order: 0 centroid cosine, 1 probe select + list
 * gather into a bitmap, 2 bitmap expansion into the recalled id list fused with key scoring,
 * 3 softmax denominators, 4 ranking keys + their histogram, 5 chip-wide pass over the
 * ranking keys (bitmap + deciding bucket's list), 6 rerank select, 7 sparse attention.  As a rule 3 to 7 are one
 * launch, timed as stage 7 (the others then read as the cost of an event pair), and where they are not (CTKVR_TAIL = 0 below)
 * 6 and 7 are for up to 64 (batch, KV head) pairs.  While timing is enabled a ninth, empty kernel follows (stage 8): its
 * figure is what a pair of events costs around a kernel that does nothing. */
#define CTKVR_N_STAGES 9
/* After this call every decode step on `idx` records a HIP event before its first
 * kernel and after each kernel, for up to max_steps steps (0 disables and frees
 * the events).  Recording adds work to the stream: use it for the breakdown, not
 * for the headline step time. */
int ctkvr_profile_enable(ctkvr_index *idx, int32_t max_steps);
/* Synchronises, writes ms_host[step][stage] (fp32, CTKVR_N_STAGES per step) for
 * the steps recorded since the last collect (at most capacity_steps), stores
 * their number in *n_steps and restarts recording at step 0. */
int ctkvr_profile_collect(ctkvr_index *idx, float *ms_host, int32_t capacity_steps, int32_t *n_steps);

/* ---- environment variables ------------------------------------------------------------- */
/* Read when an index is created (ctkvr_build_index, ctkvr_index_load); none changes a result beyond the outputs' rounding, all
 * exist so that each form of a launch can be measured and tested against the other:
 *   CTKVR_DECODE_PATH        = staged | fused | auto   default of ctkvr_index_set_decode_path
 *   CTKVR_DECODE_GROUPS      = n   sequences stepped as n forked groups (default 1)
 *   CTKVR_XCD_UNITS          = 0|1 the blocks of a (sequence, KV head) unit spread over the XCDs / all on one XCD in
 *                                  every kernel of a step (needs a multiple of 8 units; default: one XCD, except, for
 *                                  large batches, in the two bandwidth-bound launches)
 *   CTKVR_SCORE_BY_RANK      = 0|1 recalled ids split over a unit's blocks by id range / by rank
 *                                  (default: by rank for small batches)
 *   CTKVR_KEYCLASS           = 0|1 ranking-key histogram and classification as two launches / one
 *                                  (default: one for small batches)
 *   CTKVR_TAIL               = 0|1|2 what follows the scoring as separate launches / as one whose blocks all walk a unit's
 *                                  recalled keys / as one that shares those out over a unit's blocks (default: the second for small
 *                                  batches of up to 32768 candidate slots per unit, 65536 where a unit has an XCD of its own, else the
 *                                  third, or the first beyond a top_k of 8191 and for long contexts of more units than half the
 *                                  CUs; the first where CTKVR_KEYCLASS is set)
 *   CTKVR_TAIL_SPINS         = n   how often a block of those launches looks for its siblings' words before it does without them
 *                                  (0..256, default 256)
 *   CTKVR_SHARE_LATE         = w[:b]  (tests) in the third form, the wait that block b of every unit, or each block, gives up at once:
 *                                  0 for the sums, 1 the histograms, 2 the deciding bucket's keys, 3 the outputs
 *   CTKVR_FUSED_THREADS      = 256|1024  block size of the single-launch step
 *   CTKVR_BUILD_CANDIDATES   = 0|1 see ctkvr_index_build_route
 *   CTKVR_BUILD_CANDIDATES_REDO    (set: the candidate route also hands every chunk back; tests)
 *   CTKVR_BUILD_SCRATCH_CACHE = 0|1 see ctkvr_release_scratch (read whenever a block is given back) */

/* ---- how the matrix-core list build chose a unit's top-rho (Algorithm 1 line 4) ---------- */
/* CTKVR_BUILD_MFMA ranks either all s keys of a (KV head, centroid) unit (their 4-byte ranking keys
 * written once, read for a histogram and read again for the selection) or only the keys at or above
 * a per-unit threshold taken from a 1-in-16 sample of the positions (a few thousand candidates per
 * unit; taken when the batch has 60 million keys or more over all units, ten or more for each one
 * listed, or every sequence has more than 32768 tokens, 32 or more for each one listed, and the units 30 million keys or
 * the sequences 98304 tokens; when rho is 256..2730; and when the threshold leaves room for the spread of its sample, i.e. up to
 * 400 to 550 thousand tokens by rho).  The second route
 * yields exactly the same lists: a (sequence, KV head) pair in which a unit ends with fewer than rho
 * candidates, more than fit, or hundreds of candidates exactly equal to its rho-th key, is redone
 * by the first route.
 * The second route's scratch is 140 to 170 KB a unit, for at most 8192 units or four (sequence, KV head) pairs, whichever is more:
 * up to 1.4 GB, twice that where a pair has 4096 centroids; a build that hands pairs back takes 4 bytes a key of those of a chunk besides.
 * by_candidates_host: 1 if the index was built by the candidate route; chunks_redone_host: from how many
 * of its chunks of units it handed pairs back.  Both HOST, either may be NULL.  The environment variable
 * CTKVR_BUILD_CANDIDATES = 0 | 1, read at build time, forces the choice where the geometry allows it. */
int ctkvr_index_build_route(const ctkvr_index *idx, int32_t *by_candidates_host, int32_t *chunks_redone_host);

/* ---- device memory kept between indexes (Algorithm 1 runs once per prompt) ---------------- */
/* An index and the scratch of its build are one device allocation each.  Blocks that are no longer in use (the
 * scratch when a build returns, an index's memory when it is freed) are kept, at most 2 GiB per device, the oldest
 * given up first, and serve later builds and loads of about the same size (a block is at most twice what scratch needs and
 * five quarters of what an index needs), from any host thread and stream; they
 * are freed when an allocation of the library runs out of memory and by this call, which frees the current device's
 * idle blocks and the 8 MB of pinned host memory that copies of lists and centroids go through; an error if a build
 * is using scratch on that device.  Memory whose users could not be waited for (ctkvr_free while a stream is being captured)
 * is kept back and joins the idle blocks at the next build, load or call of this function that can wait for the device.
 * The environment variable
 * CTKVR_BUILD_SCRATCH_CACHE = 0, read when a block is given back, switches the keeping off. */
int ctkvr_release_scratch(void);

/* ---- how a decode step is launched ----------------------------------------- */
/* Algorithm 2 lines 1-9 run either as a sequence of launches (one per stage; any geometry) or as
 * ONE launch whose blocks walk the stages together, a fixed group of co-resident blocks per
 * (sequence, KV head) separated by barriers in device memory (batch * g at most the number of
 * compute units, and a shared-memory plan that fits).  Both give the same integers bit for bit;
 * outputs agree within rounding.  AUTO takes the staged launches, which measure faster on every
 * benchmark geometry of this part (an empty launch behind another costs 1.6 us in a graph, a
 * barrier among 32 blocks with what it has to wait for 1.5-2.5 us); FUSED is there to be measured.
 * The single launch needs all its blocks resident at once: two such steps (two indexes, two
 * streams) must not run on one GPU at the same time -- their waits are bounded, and an expired
 * wait is reported by ctkvr_index_check.  The environment variable CTKVR_DECODE_PATH = staged |
 * fused | auto sets the default of indexes created afterwards. */
typedef enum { CTKVR_PATH_AUTO = 0, CTKVR_PATH_STAGED = 1, CTKVR_PATH_FUSED = 2 } ctkvr_decode_path;
/* Errors: EINVAL (unknown path), EUNSUPPORTED (FUSED on a geometry that does not allow it). */
int ctkvr_index_set_decode_path(ctkvr_index *idx, int32_t path);
/* The path the next step will take: CTKVR_PATH_STAGED or CTKVR_PATH_FUSED (negative: error). */
int ctkvr_index_decode_path(const ctkvr_index *idx);
/* Synchronises the device and reports whether any single-launch step on `idx` gave up a wait
 * (CTKVR_EHIP; the index must then be freed) -- CTKVR_OK otherwise. */
int ctkvr_index_check(ctkvr_index *idx);
/* Measurement aid for the single launch: with enable != 0 the first block of the first unit
 * stamps the 100 MHz wall clock at kernel entry and after each of its phases (entries 0-7: when it
 * leaves the phase's barrier), when its own work of each phase is done (entries 8-13: when it
 * arrives at the barrier) and at points inside the phases (entries 16 and up; 0 = not stamped); the
 * call synchronises and copies the 64 entries of the last step to ticks_host (HOST, 64 values, may
 * be NULL). */
int ctkvr_profile_phases(ctkvr_index *idx, int32_t enable, long long *ticks_host);

/* Measurement aid: what a launch costs when the kernel does nothing.  Captures n_launches empty
 * kernels, one behind the other, in a HIP graph on a stream of its own, replays it once untimed and
 * once between two events, and stores the microseconds per launch in *us_per_launch_host (HOST).
 * Creates and destroys a stream, a graph and two events; synchronises that stream only. */
int ctkvr_measure_dispatch_floor(int32_t n_launches, float *us_per_launch_host, void *hip_stream);

/* Self-check of the fixed-point exponential that the softmax denominators are summed in (the
 * integer S of the score normalisation, Algorithm 1 line 2 and Algorithm 2 line 6): the library
 * holds it in two forms, one written out step by step after its definition and the straight-line
 * one its kernels use, which must agree bit for bit.  Evaluates both on the device for EVERY fp32 value in [-32, 0] (about
 * 1.1e9 inputs, -0 and +0 included), synchronises, and stores the number of inputs on which they
 * differ in *mismatches_host (HOST; 0 is the only acceptable value).  Allocates and frees 8 bytes
 * of device memory.  Returns a status code. */
int ctkvr_selftest_exp(uint64_t *mismatches_host, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* CTKVR_H */
