/*
 * stom_kv.h -- the paged key-value cache a model answers over, on NVIDIA B200
 * (sm_100a); part of libstom_oqm.so.
 *
 * After a retrieval (stom_oqm.h) the reconstructed groups, the question and
 * the tokens of the answer form the active cache of a stream.  These calls
 * keep such caches in PAGES that many sequences share: positions are rotated
 * into queries and keys (with their per-head norms) on the way to a page, one
 * new token per sequence attends over its pages, and pages are reserved,
 * shared between candidate answers, given back and moved together -- all from
 * arrays in device memory, so that a decode step can be captured in a CUDA
 * graph.
 *
 * Conventions are those of stom_oqm.h: device pointers unless marked "host",
 * structs read on the host, strides in elements with the channel axis
 * contiguous, caller-owned memory, work enqueued on `stream` without
 * synchronising, argument errors found before a launch (a call of no token or
 * no sequence does nothing, and its arrays may be NULL), and bits set in the
 * optional `dev_flags` word for what only the device can see.  Every buffer
 * lies on the device that is current at the call.  A workspace may be used by
 * one call at a time (calls on one stream, graphs replayed one after another);
 * nothing is kept in it from call to call.
 */
#ifndef STOM_KV_H
#define STOM_KV_H

#include "stom_oqm.h"

#ifdef __cplusplus
extern "C" {
#endif

/* further bits of dev_flags (STOM_FLAG_TIMEOUT: stom_kv_attend_tree gave up; its outputs are not to be used) */
#define STOM_FLAG_NO_PAGE 8u    /* stom_kv_reserve: too few free pages; the call changed nothing */
#define STOM_FLAG_BAD_VALUE 16u /* stom_sample_tokens: a NaN among a row's logits or settings */

/* How the channels of a rotated pair lie in a head. */
#define STOM_ROPE_HALF 0  /* channel i with channel i + rot_dim/2 */
#define STOM_ROPE_PAIRS 1 /* channel 2i with channel 2i + 1       */

/* Ways to reach positions beyond those trained on (stom_kv_frequencies). */
#define STOM_ROPE_PLAIN 0  /* f_i = theta^(-2i/rot_dim)                                                     */
#define STOM_ROPE_LINEAR 1 /* f_i / factor                                                                 */
#define STOM_ROPE_BASE 2   /* theta * factor^(rot_dim/(rot_dim-2)) in the place of theta                     */
#define STOM_ROPE_WAVES 3  /* pairs that turn more than `high` times over `trained` positions keep f_i, those
                              below `low` turns get f_i / factor, those between a linear mixture of the two */

/* Pages of keys and values.  Element (layer l, page p, token t, head h,
 * channel c) of either stands at l*stride_layer + p*stride_page +
 * t*stride_token + h*stride_head + c.  With stride_head = d and pages that
 * follow one another, a run of pages is one contiguous token axis, into which
 * stom_oqm_dequant_gather and stom_oqm_retrieve write directly. */
typedef struct stom_kv_pool {
    void *k;
    void *v;
    int32_t dtype;        /* STOM_BF16 | STOM_FP16                */
    int32_t n_layers;
    int32_t n_pages;
    int32_t page_tokens;  /* any number >= 1                      */
    int32_t n_kv_heads;
    int32_t head_dim;     /* 64, 128 or 256                       */
    int64_t stride_layer, stride_page, stride_token, stride_head;
} stom_kv_pool;

#define STOM_KV_MAX_SEQS 8192 /* rows that stom_kv_attend and stom_kv_reserve take */

/* The sequences that live in a pool.  Row i of `table` names, in order, the
 * ceil(len[i]/page_tokens) pages of sequence i; what stands behind them is not
 * read (but by stom_kv_append, if a slot lies there: with -1 in a new table's
 * entries such a token is skipped and flagged, which is what a step captured
 * in a graph needs if its stom_kv_reserve finds no page).  refs[p] counts the
 * rows that hold page p; 0 is a free page. */
typedef struct stom_kv_seqs {
    int32_t *table;       /* [n_seqs][table_stride], max_pages entries of a row are used */
    int32_t *len;         /* [n_seqs] tokens                                            */
    int32_t *refs;        /* [n_pages]; may be NULL for append and attend               */
    int32_t n_seqs;
    int32_t max_pages;
    int64_t table_stride;
} stom_kv_seqs;

/* Rotation: pair i of a token at position p is turned by p * freq[i] radians
 * and scaled by `magnitude`; channels from rot_dim on stay as they are. */
typedef struct stom_kv_rope {
    const double *freq;   /* device [rot_dim/2]; may be NULL if rot_dim == 0 */
    int32_t rot_dim;      /* a multiple of 16, 0..head_dim                   */
    int32_t layout;       /* STOM_ROPE_HALF | STOM_ROPE_PAIRS                */
    float magnitude;      /* 1 unless a scaling asks for another             */
} stom_kv_rope;

/* HOST helper: fills freq_host[rot_dim/2] (copy it to the device once).
 * `trained`, `low`, `high` are read by STOM_ROPE_WAVES only, `factor` by all
 * but STOM_ROPE_PLAIN.  Errors: INVALID_ARG, SHAPE, UNSUPPORTED. */
int32_t stom_kv_frequencies(int32_t rot_dim, double theta, int32_t scaling, double factor, double trained, double low,
                            double high, double *freq_host);

/* ---- rotary positions and per-head norms --------------------------------
 * For every token i < n_tokens and head h of q and of k:
 *     y = x * weight / sqrt(mean_c(x_c^2) + eps)     (if its weight is given)
 *     out = y turned to position pos[i]
 * in binary32 (angles in binary64, reduced before they are rounded), rounded
 * once to dtype.  q or k may be NULL (its head count is then ignored); an
 * output may be its input.  x (dtype: STOM_BF16 | STOM_FP16 | STOM_FP32):
 * element (i, h, c) at i*stride_token + h*stride_head + c.  Weights: binary32
 * [head_dim], 16-byte aligned.
 * Errors: INVALID_ARG, SHAPE, UNSUPPORTED, ALIGNMENT, CUDA. */
int32_t stom_kv_rotate(const stom_kv_rope *rope, int32_t dtype, int32_t head_dim, int32_t n_tokens, const int32_t *pos,
                       const void *q, int32_t n_q_heads, int64_t q_stride_token, int64_t q_stride_head,
                       void *q_out, int64_t q_out_stride_token, int64_t q_out_stride_head, const float *q_weight,
                       const void *k, int32_t n_k_heads, int64_t k_stride_token, int64_t k_stride_head,
                       void *k_out, int64_t k_out_stride_token, int64_t k_out_stride_head, const float *k_weight,
                       float eps, void *stream);

/* The same on the way into the cache: q goes to q_out (or stays away: q NULL),
 * k -- normed and turned -- and v -- as it is -- go to token slot[i] of
 * sequence seq[i] (seq NULL: sequence i, the decode step, with n_tokens <=
 * n_seqs) in layer `layer` of the pool.  All of pool->dtype.  A slot of -1
 * stores nothing (padding); a sequence out of range, a slot outside
 * [0, max_pages*page_tokens) or a page id outside [0, n_pages) is skipped and
 * sets STOM_FLAG_BAD_INDEX; q_out is written all the same.  len and refs are
 * not read: the pages have to be there (stom_kv_reserve) and a page written to
 * must not be shared.  No two tokens of a call may name the same slot.
 * Errors: INVALID_ARG, SHAPE, UNSUPPORTED, ALIGNMENT, CUDA. */
int32_t stom_kv_append(const stom_kv_pool *pool, const stom_kv_seqs *seqs, int32_t layer, const stom_kv_rope *rope,
                       int32_t n_tokens, const int32_t *pos, const int32_t *slot, const int32_t *seq,
                       const void *q, int32_t n_q_heads, int64_t q_stride_token, int64_t q_stride_head,
                       void *q_out, int64_t q_out_stride_token, int64_t q_out_stride_head, const float *q_weight,
                       const void *k, int64_t k_stride_token, int64_t k_stride_head, const float *k_weight,
                       const void *v, int64_t v_stride_token, int64_t v_stride_head,
                       float eps, uint32_t *dev_flags, void *stream);

/* ---- attention of one new token per sequence ------------------------------
 * For sequence i and query head h (kv head h / (n_q_heads/n_kv_heads)), over
 * the tokens t with max(0, len[i] - window) <= t < len[i] (window 0: all):
 *     x_t = softmax_scale * <q, K_t>,  softcap*tanh(x_t/softcap) if softcap > 0
 *     out = sum_t exp(x_t) V_t / sum_t exp(x_t),   lse = ln sum_t exp(x_t)
 * The sequence's own newest token is expected in the cache already.  An empty
 * sequence gives zeros and -inf.  A token whose page id is outside
 * [0, n_pages) counts as absent and sets STOM_FLAG_BAD_INDEX; so does what
 * len[i] has beyond max_pages*page_tokens.  What a page holds behind len[i] is
 * not read.  Products of 16-bit operands are summed in binary32; the softmax
 * weights enter the second product as a high and a low 16-bit part: off by
 * 2^-16 of themselves (bf16), or by 2^-22 of themselves or 2^-40 of the largest
 * weight of their 16 tokens, whichever is more (fp16).
 * q, out (pool->dtype): element (i, h, c) at i*stride_seq + h*stride_head + c.
 * lse: binary32 [n_seqs][n_q_heads], or NULL.
 * softmax_scale below 2e38 in magnitude; softcap 0, or below 2e38 with
 * softmax_scale / softcap a normal number of binary32 (or 0).
 * n_q_heads / n_kv_heads <= 64, n_seqs <= STOM_KV_MAX_SEQS, max_pages *
 * page_tokens < 2^31 - 32, and n_seqs * n_kv_heads * max_pages * page_tokens
 * below 2^34 (n_kv_heads counted twice where its query heads are more than 16,
 * or 8 at head_dim 256, and so on).  workspace: 16-byte aligned, of at least
 * stom_kv_attend_workspace_bytes() bytes; its contents do not matter.
 * Errors: INVALID_ARG, SHAPE, UNSUPPORTED, ALIGNMENT, WORKSPACE, CUDA. */
int64_t stom_kv_attend_workspace_bytes(const stom_kv_pool *pool, const stom_kv_seqs *seqs, int32_t n_q_heads);
int32_t stom_kv_attend(const stom_kv_pool *pool, const stom_kv_seqs *seqs, int32_t layer, int32_t n_q_heads,
                       const void *q, int64_t q_stride_seq, int64_t q_stride_head, float softmax_scale, float softcap,
                       int32_t window, void *out, int64_t out_stride_seq, int64_t out_stride_head, float *lse,
                       void *workspace, int64_t workspace_bytes, uint32_t *dev_flags, void *stream);

/* ---- attention of several new tokens per sequence -------------------------
 * The last n_i = first[i+1] - first[i] of the len[i] tokens of sequence i are
 * new: its NODES, rows first[i] .. first[i+1] - 1 of q, out, lse and parent.
 * parent[first[i] + j], below j, is the node that node j follows, or -1: it
 * follows the context, as a tree of drafted tokens may branch there too.  parent
 * NULL: node j follows node j - 1 (a question, or one draft).  Node j stands at
 * position (len[i] - n_i) + depth_j, where depth_j counts the nodes before it on
 * its path, and sees, for every query head as in stom_kv_attend, the tokens
 * before the nodes and the nodes of its path, itself among them; with a window,
 * those of them whose position is above its own minus `window`.
 * The nodes' keys and values are expected in the cache already, node j's at
 * slot (len[i] - n_i) + j (stom_kv_append with that slot and the position
 * above).
 * first: int32 [n_seqs + 1]; rows of no sequence are left as they were.  A
 * sequence whose first[i] .. first[i+1] do not lie in order within
 * 0 .. n_tokens, that has more nodes than tokens or, with parents, more than
 * STOM_KV_MAX_TREE, is skipped (its rows stay as they were) and sets
 * STOM_FLAG_BAD_INDEX; so does a parent outside -1 .. j - 1, which counts as -1,
 * and what stom_kv_attend flags.  A node that sees nothing (all of its pages
 * are none) gives zeros and -inf.
 * Keys and values of a token that a node does not see have no effect on it,
 * also where they are no finite numbers; a value that is none makes none of the
 * same channel of what sees it.  Products of 16-bit operands are
 * summed in binary32; a softmax weight enters the second product as a high and a
 * low part of the pool's type, as in stom_kv_attend: off by 2^-16 of itself (bf16),
 * or by 2^-22 of itself or the lesser of 2^-32 of the row's largest weight and
 * 2^-24 of the largest among the 127 tokens on either side (but for 2^-80 of the
 * row's), whichever is more (fp16).
 * q, out (pool->dtype): element (row, h, c) at row*stride_token +
 * h*stride_head + c.  lse: binary32 [n_tokens][n_q_heads], or NULL.  The
 * limits are those of stom_kv_attend for softmax_scale, softcap, heads and
 * n_seqs; max_pages * page_tokens < 2^31 - 256, n_tokens * n_q_heads < 2^31 - 128.
 * Errors as for stom_kv_attend. */
#define STOM_KV_MAX_TREE 256
int64_t stom_kv_attend_tree_workspace_bytes(const stom_kv_pool *pool, const stom_kv_seqs *seqs, int32_t n_tokens,
                                            int32_t n_q_heads);
int32_t stom_kv_attend_tree(const stom_kv_pool *pool, const stom_kv_seqs *seqs, int32_t layer, int32_t n_tokens,
                            const int32_t *first, const int32_t *parent, int32_t n_q_heads, const void *q,
                            int64_t q_stride_token, int64_t q_stride_head, float softmax_scale, float softcap,
                            int32_t window, void *out, int64_t out_stride_token, int64_t out_stride_head, float *lse,
                            void *workspace, int64_t workspace_bytes, uint32_t *dev_flags, void *stream);

/* ---- a drafted path is kept ------------------------------------------------
 * first, parent: as above.  draft[row] is the token that a node holds,
 * chosen[row] the one that was chosen to follow it (stom_sample_tokens of the
 * node's logits).  The path kept begins with node 0, whose token had been
 * chosen in the step before; node j is followed by the lowest node c > j with
 * parent j and draft[c] == chosen[j], until there is none (chosen[j] < 0: there
 * is none).  For every sequence with nodes:
 *     path[first[i] + k] = the path's k-th node, -1 behind its end;
 *     n_accepted[i] = its length;  next[i] = chosen of its last node;
 *     keys and values of its nodes, in all layers, move together to the slots
 *     behind the context; len[i] = (len[i] - n_i) + n_accepted[i]; pages that
 *     hold nothing any more are given back (as by stom_kv_free).
 * A sequence without nodes keeps what it has: n_accepted 0, next -1; so does one
 * that stom_kv_attend_tree would skip, or (without parents too) with more than
 * STOM_KV_MAX_TREE nodes or tokens than its row has, and sets
 * STOM_FLAG_BAD_INDEX.  Page ids outside [0, n_pages) are skipped and set it too,
 * and so does a parent outside -1 .. j - 1, which counts as -1.
 * Pages that nodes lie in must not be shared.  path, n_accepted and next may be
 * NULL.  Errors: INVALID_ARG, SHAPE, UNSUPPORTED, ALIGNMENT, CUDA. */
int32_t stom_kv_accept(const stom_kv_pool *pool, const stom_kv_seqs *seqs, int32_t n_tokens, const int32_t *first,
                       const int32_t *parent, const int32_t *draft, const int32_t *chosen, int32_t *path,
                       int32_t *n_accepted, int32_t *next, uint32_t *dev_flags, void *stream);

/* ---- pages: reserve, fork, free, compact -----------------------------------
 * All need seqs->refs and act on all layers.  Page ids outside [0, n_pages)
 * are skipped and set STOM_FLAG_BAD_INDEX.
 */

/* Sequence i grows to want[i] tokens (want[i] <= len[i]: it stays).  Pages are
 * taken lowest id first, rows in ascending order.  If the sequence's last page
 * is partly filled and other rows hold it too, the tokens in use are copied to
 * a page of its own; of several growing rows that share a page with nobody
 * else the last keeps it.  If there are not enough free pages for all rows,
 * nothing changes and STOM_FLAG_NO_PAGE is set.  A want[i] beyond
 * max_pages*page_tokens is skipped and sets STOM_FLAG_BAD_INDEX.
 * n_seqs <= STOM_KV_MAX_SEQS.  workspace: 16-byte aligned, of at least
 * stom_kv_pages_workspace_bytes() bytes.  Errors as for stom_kv_attend. */
int64_t stom_kv_pages_workspace_bytes(const stom_kv_pool *pool, const stom_kv_seqs *seqs);
int32_t stom_kv_reserve(const stom_kv_pool *pool, const stom_kv_seqs *seqs, const int32_t *want, void *workspace,
                        int64_t workspace_bytes, uint32_t *dev_flags, void *stream);

/* Every empty sequence i with parent[i] >= 0 becomes a sharer of all pages of
 * sequence parent[i] and takes its length (parent[i] == -1: not forked).
 * Nothing is copied until one of them grows.  Skipped, with
 * STOM_FLAG_BAD_INDEX: a parent out of range, a parent that is itself forked
 * in this call, a row i that is not empty. */
int32_t stom_kv_fork(const stom_kv_pool *pool, const stom_kv_seqs *seqs, const int32_t *parent, uint32_t *dev_flags,
                     void *stream);

/* Every sequence i with drop[i] != 0 gives its pages back: its row becomes -1,
 * its length 0. */
int32_t stom_kv_free(const stom_kv_pool *pool, const stom_kv_seqs *seqs, const int32_t *drop, uint32_t *dev_flags,
                     void *stream);

/* Moves the live pages to the front of the pool: with n live pages, the k-th
 * live page of id >= n goes to the k-th free page of id < n, whole.  table_out
 * [n_seqs][table_stride] gets the rows with their new ids (-1 behind the pages
 * of a row), refs_out [n_pages] the counts, *n_live the number n (n_live may
 * be NULL).  table_out and refs_out may be seqs->table and seqs->refs, or
 * separate arrays, in which case the old ones stay as they were. */
int32_t stom_kv_compact(const stom_kv_pool *pool, const stom_kv_seqs *seqs, int32_t *table_out, int32_t *refs_out,
                        int32_t *n_live, void *workspace, int64_t workspace_bytes, uint32_t *dev_flags, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* STOM_KV_H */
