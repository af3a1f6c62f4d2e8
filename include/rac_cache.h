/*
 * rac_cache.h - C ABI of the paged key-value cache and of attention over
 * drafted trees (MI355X, gfx950).
 *
 * The decode phase of a split model pays a network round trip per step.  With
 * speculative decoding one message carries a tree of drafted tokens, and the
 * accepted path of the tree is committed at once.  These entry points hold
 * what such a runtime (and the reference predictor, see
 * rac_predictor_tree_step) keeps per sequence: keys and values in pages that
 * sequences share, and the attention that reads them.
 *
 * The conventions of rac.h hold: device pointers, caller-owned memory, work
 * enqueued on `stream`, nothing allocated, kept or synchronized, argument
 * errors before any launch.  No kernel is captured state: every call can be
 * recorded in a HIP graph.  Sequence numbers, page numbers, lengths and row
 * ranges that lie in device memory are checked by the kernels: whatever they
 * hold, no access leaves the buffers.
 *
 * Memory
 *   pool    : [pages][layers][2][kv_heads][page_tokens][head_dim], keys then
 *             values, 16-byte aligned, contents of unused places unspecified
 *   table   : int32 [seqs][max_pages], the page of every page_tokens positions
 *             of a sequence; negative where there is none
 *   lengths : int32 [seqs], committed tokens
 *   refs    : int32 [pages], table entries that name the page; 0 = free
 * A new cache is a table of -1, lengths of 0 and refs of 0.  Entries of a
 * table beyond a sequence's pages are negative; a page appears at one place of
 * a sequence only.
 */
#ifndef RAC_CACHE_H
#define RAC_CACHE_H

#include "rac.h"

#ifdef __cplusplus
extern "C" {
#endif

enum {
    RAC_CACHE_BF16 = 0, /* queries, drafts, outputs and pages in bfloat16          */
    RAC_CACHE_FP16 = 1, /* the same in IEEE binary16                               */
    RAC_CACHE_FP8 = 2   /* pages in e4m3 (OCP, no infinities), the rest bfloat16   */
};

typedef struct {
    int32_t layers;      /* 1..1024                                                */
    int32_t kv_heads;    /* 1..1024                                                */
    int32_t head_dim;    /* multiple of 16, 16..256                                */
    int32_t page_tokens; /* power of two, 8..256                                   */
    int32_t pages;       /* 1..2^24                                                */
    int32_t seqs;        /* sequences (rows of the table), 1..4096                 */
    int32_t max_pages;   /* width of the table; max_pages * page_tokens <= 2^30    */
    int32_t type;        /* RAC_CACHE_*                                            */
    float k_scale;       /* RAC_CACHE_FP8: a key is k_scale times what is stored,  */
    float v_scale;       /* a value v_scale times (both > 0); else ignored         */
} rac_cache_config;

/* Host-only, pure.  Bytes of the pool, or 0 for a configuration outside the
 * ranges above. */
size_t rac_cache_pool_bytes(const rac_cache_config* cfg);

/* ---- Attention over a drafted tree --------------------------------------
 * Sequence s has L = lengths[s] committed tokens in its pages and n drafted
 * ones, rows draft_start[s] .. draft_start[s + 1] of k and v, not in the
 * cache; its queries are rows q_start[s] .. q_start[s + 1] of q.  Query row r
 * (the i-th of its sequence's m) sees
 *   - the committed positions 0 .. L - 1 that have a page, and
 *   - the drafted tokens j < n with bit j % 64 of mask[r][j / 64] set (an
 *     ancestor mask, itself included); without a mask the first n - m + i + 1
 *     drafted tokens (the queries are the last of the drafted, in order);
 * with a window w > 0 only the last w of these: of c drafted ones the last
 * min(c, w), and the committed positions from L - (w - c) on.
 *   out[r] = sum_j p_j v_j / sum_j p_j,  p_j = exp(scale q_r . k_j - max),
 *   lse[r] = max + ln(sum_j p_j)
 * for every query head, head h with key-value head h / (q_heads / kv_heads).
 * A row that sees nothing (or scores of -infinity only) gets zeros and an lse
 * of -infinity.  What a row does not see never reaches it, infinities and
 * NaNs included.  One drafted token a sequence and no mask is the ordinary
 * decode step, a chunk of a prompt and no mask its causal attention.
 *
 * Scores, maxima, sums and the accumulated output are fp32; the sum of the
 * weights takes them unrounded.  Before they meet the values the weights are
 * rounded to the 16-bit type of the queries (at most 2^-8 (bf16) or 2^-11 (fp16)
 * of each; fp16 weights below 2^-25 of the row's largest by at most 2^-36 of that
 * one); where a sequence has few rows a key-value head (max_rows * q_heads /
 * kv_heads <= 16, and up to 32 in some types) what the rounding left goes in as
 * well.  The output is rounded once.
 *
 * A call gives the same bits every time.  Which kernel runs, and how long
 * sequences are cut into parts, follows from the whole call (the configurations,
 * all lengths and row counts), so the last bits of a row may change with the
 * sequences beside it. */
typedef struct {
    int32_t q_heads;   /* a multiple of kv_heads, at most 64 times as many        */
    int32_t rows;      /* rows of q and out, 0..2^20; rows * q_heads below 2^26   */
    int32_t max_rows;  /* most query rows of a sequence; further ones are ignored */
    int32_t max_draft; /* most drafted tokens of a sequence; further ones unseen  */
    int32_t window;    /* 0: none                                                 */
    float scale;       /* 0: 1 / sqrt(head_dim)                                   */
} rac_tree_config;

typedef struct {
    const void* q;              /* [rows][q_heads][head_dim], rows q_stride apart  */
    const void* k;              /* [draft_rows][kv_heads][head_dim], rows          */
    const void* v;              /* kv_stride apart; both NULL: no drafted tokens   */
    const int32_t* q_start;     /* [seqs + 1]                                      */
    const int32_t* draft_start; /* [seqs + 1], NULL: q_start                       */
    const uint64_t* mask;       /* [rows][mask_words], or NULL                     */
    void* out;                  /* [rows][q_heads][head_dim], rows out_stride apart*/
    float* lse;                 /* [rows][q_heads], or NULL                        */
    int64_t q_stride, kv_stride, out_stride; /* elements, multiples of 8; kv_stride */
                                /* at most 2^25                                    */
    int32_t draft_rows;
    int32_t mask_words;         /* 0 without a mask                                */
} rac_tree_tensors;

/* Host-only, pure.  Bytes of the call's device scratch, or 0 for a
 * configuration outside the ranges above. */
size_t rac_tree_attention_workspace(const rac_cache_config* cfg, const rac_tree_config* tree);

/* Attention of layer `layer`.  q, k, v and out 16-byte aligned, mask 8-byte,
 * the int32 and fp32 arrays 4-byte, workspace 256-byte.  Rows of q outside
 * every sequence's range keep their out and lse.  RAC_ERR_INVALID, _ALIGN,
 * _UNSUPPORTED (2^26 or more rows * q_heads: split the call) and _CAPACITY
 * (workspace) before any launch. */
rac_status rac_tree_attention(const rac_cache_config* cfg, const rac_tree_config* tree, int32_t layer,
                              const void* pool, const int32_t* table, const int32_t* lengths,
                              const rac_tree_tensors* t, void* workspace, size_t workspace_bytes,
                              rac_stream_t stream);

/* ---- Pages ---------------------------------------------------------------- */

/* Sequence d becomes a view of positions [keep_from[d], keep_to[d]) of what
 * sequence parents[d] held before the call, for all sequences at once: forking
 * (several d with one parent), the reordering of beams, rollback (parents[d] =
 * d and a shorter keep_to), a bounded history (a keep_from: positions keep
 * their numbers, pages wholly before it are let go) and freeing (a parent
 * outside 0 .. seqs - 1).  Pages are shared, none is copied; refs follow.
 *   parents            : int32 [seqs]
 *   keep_from, keep_to : int32 [seqs], or NULL (0; the parent's length)
 * Positions before keep_from in a page that stays are still seen.  A keep_from
 * past the new length lets go of the last page too: the page that a later
 * commit takes for it has unspecified contents ahead of the appended tokens,
 * which the attention would see.
 * One kernel launch. */
rac_status rac_cache_fork(const rac_cache_config* cfg, const int32_t* parents, const int32_t* keep_from,
                          const int32_t* keep_to, int32_t* table, int32_t* lengths, int32_t* refs,
                          rac_stream_t stream);

/* Host-only, pure.  Bytes of rac_cache_commit's scratch, or 0. */
size_t rac_cache_commit_workspace(const rac_cache_config* cfg);

/* Appends the accepted drafted tokens of every sequence to it, in all layers.
 *   k, v        : [layers][draft_rows][kv_heads][head_dim] in the 16-bit type,
 *                 rows kv_stride and layers layer_stride elements apart
 *                 (multiples of 8), 16-byte aligned
 *   draft_start : int32 [seqs + 1], the rows of each sequence
 *   path        : int32 [seqs][max_path], the accepted tokens of a sequence in
 *                 order, relative to its first row; the first entry that names
 *                 none of them ends it.  NULL: all rows, at most max_path.
 *   committed   : int32 [seqs], receives how many tokens were appended
 * Sequences are served in order.  Each takes the lowest-numbered pages that
 * were free before the call, one for every page_tokens positions it newly
 * enters, and a last page that it shares is first copied (its committed tokens
 * only) and let go; a sequence whose demand exceeds what those before it left,
 * or whose tokens exceed the table, keeps its state, takes no page and has
 * committed = 0.
 * RAC_CACHE_FP8 stores x / k_scale (v_scale), clamped to +-448 and rounded to
 * nearest even; other types store the bits.  workspace 256-byte aligned.  Two
 * kernel launches. */
rac_status rac_cache_commit(const rac_cache_config* cfg, void* pool, int32_t* table, int32_t* lengths, int32_t* refs,
                            const void* k, const void* v, int64_t kv_stride, int64_t layer_stride, int32_t draft_rows,
                            const int32_t* draft_start, const int32_t* path, int32_t max_path, int32_t* committed,
                            void* workspace, size_t workspace_bytes, rac_stream_t stream);

/* Copies page src[i] of one pool to page dst[i] of another (or the same) of
 * the same configuration, all layers, i < n.  The dst differ from each other
 * and, within one pool, from every src; a pair with a number outside the pool
 * is skipped.  One kernel launch; RAC_ERR_UNSUPPORTED where it would take 2^24
 * pieces of 16 KiB or more (n times those of a page). */
rac_status rac_cache_copy(const rac_cache_config* cfg, const void* src_pool, const int32_t* src, void* dst_pool,
                          const int32_t* dst, int32_t n, rac_stream_t stream);

/* ---- A bounded cache: what a token is worth, and eviction ------------------
 * A cache that is full lets go of the tokens that received least attention.  The
 * caller keeps, for every sequence, sums of the attention weight that each position
 * received: one for all layers and heads (sets = 1), or one for every layer and
 * key-value head (sets = layers * kv_heads, number layer * kv_heads + head), whose
 * evictions may then choose different tokens:
 *   weight       : fp32 [seqs][sets][positions], positions = max_pages * page_tokens
 *   draft_weight : fp32 [sets][draft_rows], the drafted tokens'
 * A round is rac_tree_attention and rac_tree_weights for every layer, rac_cache_commit,
 * rac_cache_weights_commit, and rac_cache_evict.  rac_cache_fork knows nothing of
 * weights: those of a sequence are those of its parent, a copy of rows.  The predictor's step
 * below keeps its queries and lse to itself, so rac_tree_weights cannot follow it: its
 * cache is bounded by rac_cache_fork's keep_from. */

/* Adds to the sums of layer `layer` what the rows of rac_tree_attention's call give
 * to every key they see, with t, tree and cfg as there (t->v and t->out are not looked
 * at, t->lse is read: the call's own):
 *   weight[s][set][j] += sum_r sum_h exp(scale q_r,h . k_j - lse[r][h])
 * over the sequence's rows and the query heads of the set (those of key-value head
 * h, or all), for the committed positions j that have a page; in the same way
 * draft_weight for the drafted tokens (NULL: not wanted).  Sums of what no row sees,
 * positions without a page and rows outside every sequence are left as they are or get
 * 0 added.  A row whose lse is -infinity gives nothing.  Products of 16-bit numbers,
 * sums fp32.  A call gives the same bits every time; the order of a sum follows from
 * the whole call.  Every drafted row counts, also one that is later not accepted.
 *
 * Alignments as in rac_tree_attention, weights 4-byte.  RAC_ERR_INVALID (also sets
 * other than 1 or layers * kv_heads), _ALIGN, _UNSUPPORTED (as there, and seqs * sets *
 * positions of 2^36 and more) and _CAPACITY.  One kernel launch, two where a key-value
 * head may have 64 rows and more. */
size_t rac_tree_weights_workspace(const rac_cache_config* cfg, const rac_tree_config* tree);

rac_status rac_tree_weights(const rac_cache_config* cfg, const rac_tree_config* tree, int32_t layer, int32_t sets,
                            const void* pool, const int32_t* table, const int32_t* lengths, const rac_tree_tensors* t,
                            float* weight, float* draft_weight, void* workspace, size_t workspace_bytes,
                            rac_stream_t stream);

/* After rac_cache_commit: the sums of the committed[s] tokens at the end of every
 * sequence become those of the drafted rows they came from (draft_weight NULL: 0).
 * draft_start, path, max_path and draft_rows as given to the commit; lengths and
 * committed as it left them.  One kernel launch. */
rac_status rac_cache_weights_commit(const rac_cache_config* cfg, int32_t sets, const int32_t* lengths,
                                    const int32_t* committed, const int32_t* draft_start, const int32_t* path,
                                    int32_t max_path, const float* draft_weight, int32_t draft_rows, float* weight,
                                    rac_stream_t stream);

/* Every sequence s of more than keep[s] tokens (keep[s] >= 0) is cut to keep[s] of
 * them, in all layers.  Let c_0 < c_1 < .. < c_(m-1) be its positions that have a page (m of them,
 * the call's `places`) and n = keep[s] < m.  The last r = min(recent, n) places and the
 * first f = min(first, n - r) stay; of those between, the n - f - r of the largest weight,
 * ties to the lower place, a NaN below all numbers, for every set by itself.  Then
 *   - the last r places move, in order, to positions n - r .. n - 1,
 *   - of the others, those at a place below n - r are at that position, and
 *   - those above it take the positions that are still free, in ascending order both.
 * So most tokens stay where they are, and the last r keep their order; the attention
 * does not depend on the order of what it sees, but a `window` and a later keep_from or
 * keep_to count positions.  A sequence of no more places than keep[s] keeps its state.
 *   keep    : int32 [seqs], negative: the sequence is not asked
 *   evicted : int32 [seqs], receives m - n; 0 where the state was kept; -1 where it was
 *             for want of pages
 *   source  : int32 [seqs][sets][positions] or NULL, receives for every position below n
 *             of a cut sequence where its token was (rotary positions and ages move along)
 * weight moves along; the sums from n to the former length become 0.  A page that changes and
 * that other sequences or entries share is replaced by a free one, so what they hold
 * stays; sequences are served in order, each with the lowest-numbered pages that were
 * free before the call, and one whose demand exceeds what those before it left keeps its
 * state.  A sequence's pages that it shares with nobody are changed in place; pages past the
 * cut are let go.  No other byte of the pool changes.
 *
 * pool 16-byte aligned, workspace 256-byte, the others 4-byte.  Five kernel launches, ten where
 * workgroups share long sequences.  RAC_ERR_INVALID, _ALIGN, _UNSUPPORTED (seqs * sets * positions of 2^36 and more)
 * and _CAPACITY. */
typedef struct {
    int32_t sets;   /* 1, or layers * kv_heads                                      */
    int32_t first;  /* first places that stay, 0..2^30 (attention sinks)            */
    int32_t recent; /* last places that stay, 0..2^30                               */
} rac_evict_config;

/* Host-only, pure.  Bytes of the call's device scratch, or 0. */
size_t rac_cache_evict_workspace(const rac_cache_config* cfg, const rac_evict_config* evict);

rac_status rac_cache_evict(const rac_cache_config* cfg, const rac_evict_config* evict, void* pool, int32_t* table,
                           int32_t* lengths, int32_t* refs, float* weight, const int32_t* keep, int32_t* evicted,
                           int32_t* source, void* workspace, size_t workspace_bytes, rac_stream_t stream);

/* ---- The reference predictor over drafted trees ---------------------------
 * rac_predictor_step (rac.h) for sequences whose history lies in a paged cache
 * and whose inputs are nodes of drafted trees.  Sender and receiver run it
 * level by level: the states of a level are coded against the references that
 * their parents' reconstructions predict, and become the inputs of the next.
 * They hold the same references bit for bit if they make the same calls: a
 * reference's last bits follow from the whole call (see rac_tree_attention), so
 * a receiver must not batch other sequences with them than the sender does.
 * Row r is one input (the reconstruction of a node, or the last committed one):
 * its key and value go to row slot[r] of draft_k and draft_v, and it sees what
 * rac_tree_attention says for these drafted rows, mask, window (that of cfg) and
 * cache; every row should see its own.  The layers and their roundings are
 * those of rac_predictor_step, except that the turned queries are bf16 and that
 * rac_tree_attention rounds the weights as it says (the mean error of a
 * reference against the definition, which does neither, is 1.1 to 1.4 times that
 * of rac_predictor_step).  The accepted path's keys and values are committed with
 * rac_cache_commit.
 *   cfg       : batch sizes aside, the predictor; tree->rows <= cfg->max_batch
 *   cache     : one layer, kv_heads = cfg->heads, head_dim 64, not FP16
 *   tree      : q_heads = cfg->heads, window = cfg->window, scale 0
 *   h_prev    : bf16 [rows][hidden]           pos  : int32 [rows], the inputs' positions
 *   q_start   : int32 [seqs + 1], the rows of each sequence
 *   slot      : int32 [rows]; a row whose slot is none of the draft_rows stores nothing
 *   draft_k/v : bf16 [draft_rows][model]      draft_start : int32 [seqs + 1]
 *   ref_out   : bf16 [rows][hidden]           mask : as in rac_tree_tensors, or NULL
 * Alignments as in rac_predictor_step and rac_tree_attention; the workspace of
 * rac_predictor_tree_workspace() bytes, 256-byte aligned.  The launches of
 * rac_predictor_step and rac_tree_attention, the former's attention turning only. */
size_t rac_predictor_tree_workspace(const rac_predictor_config* cfg, const rac_cache_config* cache,
                                    const rac_tree_config* tree);

rac_status rac_predictor_tree_step(const rac_predictor_config* cfg, const rac_cache_config* cache,
                                   const rac_tree_config* tree, const void* weights, const void* pool,
                                   const int32_t* table, const int32_t* lengths, const int32_t* q_start,
                                   const int32_t* draft_start, const int32_t* slot, const int32_t* pos,
                                   const uint64_t* mask, int32_t mask_words, const void* h_prev, void* draft_k,
                                   void* draft_v, int32_t draft_rows, void* ref_out, void* workspace,
                                   size_t workspace_bytes, rac_stream_t stream);

#ifdef __cplusplus
}
#endif
#endif /* RAC_CACHE_H */
