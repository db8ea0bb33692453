/*
 * seq.h -- C ABI of the MI355X (gfx950) attention over token sequences (same library as na2d.h, whose dtype and status
 * codes are reused): softmax attention with causal order, a window, capped scores, a distance bias, a document mask and a
 * prefix mask, forward and backward; the rotation of queries and keys by their positions, with the norm of each head before it, forward and
 * backward; and, for serving, a cache of keys and values held in 8 bits, its append, reading it back, and attention over it.
 *
 * Conventions (as in na2d.h unless stated)
 * ----------------------------------------
 *  - All data pointers are DEVICE pointers owned by the caller.  The library never allocates, frees or synchronises; calls
 *    enqueue kernels (nothing else) on `stream`.  Outputs are fully overwritten.  Results are bitwise reproducible.
 *  - q, out, dout, dq: [B, heads, Lq, D]; k, v, dk, dv: [B, kv_heads, Lk, D] in the problem dtype, each with strides of its own
 *    (in elements) for batch, head and row; the D elements of a row are contiguous.  Pointers are 16-byte aligned and strides
 *    are multiples of 16 bytes; an input's may be 0, and no two rows of an output overlap.  Query head h reads key head h / (heads / kv_heads).
 *  - D in {32, 64, 128}; f32, f16, bf16.  Products, softmax statistics and sums are fp32; in the 16-bit types the weights, and
 *    in the backward pass their gradients, are rounded to the type where they enter a product.
 *  - fp16 has no step below 2^-24.  In out, a weight below 2^-14 of its row's largest loses digits, and one below 2^-25 of it counts as 0, as do a million of
 *    them.  The backward pass holds weights times 2^10, and their gradients on a scale that the largest |dout| and the largest sum |v| of the keys in reach (window and
 *    documents, to whole tiles) make, whatever the size of either: rows that are flat over their keys keep the type's digits up to about 2^20 keys, and one digit less for each power of two beyond.
 *  - Return value: NA2D_OK or a negative na2d_status; argument errors are detected on the host before any HIP call.
 *
 * Which keys a query sees
 * -----------------------
 *    Query i stands at position pos = i + Lk - Lq (the last query at the last key); distance = pos - j.  Key j is seen if
 *      near:    -window < distance < window (window 0: no limit), and with `causal` distance >= 0
 *      or       prefix[b, j] != 0
 *    and in both cases documents[b, pos] == documents[b, j] >= 0 where documents are given.  A negative document marks padding:
 *    such a token sees nothing and is seen by nobody, and its values in q, k, v, dout may be anything, NaN included.  All other values
 *    are expected to be finite.  A query that sees nothing gets out = 0, lse = -inf and gradients of 0.
 *    score = softcap * tanh(scale <q, k> / softcap) (softcap 0: scale <q, k>) - slopes[head] * |distance|
 */
#ifndef SEQ_H_
#define SEQ_H_

#include "na2d.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct {
    int64_t batch, head, row; /* in elements */
} seq_strides;

typedef struct {
    int32_t B, heads, kv_heads, Lq, Lk, D;
    int32_t dtype;  /* na2d_dtype */
    int32_t causal; /* 0 or 1 */
    int32_t window; /* 0: none */
    float scale;    /* finite, and so in fp32 times log2(e), with a cap times 2 log2(e) / softcap */
    float softcap;  /* 0: none; else finite, from 2^-20 on, and in the 16-bit types at most 4096; up to 1024, and in bf16 to 4096, scores are off by up to 2^-21 of it */
    seq_strides q, k, v, out;      /* forward and backward */
    seq_strides dout, dq, dk, dv;  /* backward */
} seq_problem;

/* Host only: NA2D_OK if the forward call accepts the problem (and, with backward != 0, the backward call).  heads must be a multiple of
 * kv_heads; one (batch, head) plane, strides included, stays below 2^31 bytes; Lq and Lk are at most 2^24. */
int seq_validate_problem(const seq_problem *p, int backward);

/* Bytes of workspace; 0 for an invalid problem.  `marked`: documents or prefix are given.  A call needs one only where this is not 0; no initialisation. */
size_t seq_attention_workspace_bytes(const seq_problem *p, int marked, int backward);

/* rest (nullable, 16-bit types; strides of out): what out's rounding took from it, in the type.  A backward call that is given it takes delta = <dout, out> from
 * their sum: where few keys carry a query's weight, out's rounding is otherwise as large a part of dS as dS's own.
 * slopes: fp32 [heads] or NULL.  documents: int32 [B, Lk] or NULL, contiguous; needs Lq <= Lk.  prefix: bytes [B, Lk] or NULL, contiguous.
 * lse (nullable): fp32 [B, heads, Lq], contiguous; the log-sum-exp of every query's scores. */
int seq_attention_fwd(const seq_problem *p, const void *q, const void *k, const void *v, const float *slopes, const int32_t *documents, const uint8_t *prefix,
                      void *out, float *lse, void *rest, void *workspace, size_t workspace_bytes, void *stream);

/* dq, dk, dv from the forward's inputs, its out, lse and (nullable) rest, and dout.  Nothing is added in an order that varies; dk and dv are the sums over the
 * query heads that share a key head. */
int seq_attention_bwd(const seq_problem *p, const void *q, const void *k, const void *v, const float *slopes, const int32_t *documents, const uint8_t *prefix,
                      const void *out, const float *lse, const void *rest, const void *dout, void *dq, void *dk, void *dv, void *workspace, size_t workspace_bytes,
                      void *stream);

/*
 * Rotation of head vectors by their tokens' positions, with the norm of each vector before it:
 *    y = x w / sqrt(mean of x^2 + eps)      (no weight: y = x)
 *    (z_a, z_b) = (y_a cos t - y_b sin t, y_b cos t + y_a sin t),  t = position * freqs[p] of pair p
 * Pair p is channels p and p + pairs, or if `interleaved` 2 p and 2 p + 1; channels from 2 pairs on are not rotated.  A token has a position on each axis (time, row,
 * column); the first sections[0] pairs turn by the first axis' position, the next sections[1] by the second's, and so on.  Angles are formed and reduced in 64 bits.
 */
typedef struct {
    int32_t pairs;        /* a multiple of 8, at most D / 2 */
    int32_t axes;         /* 1 to 4 */
    int32_t sections[4];  /* pairs of each axis, at least 1 each; their sum is pairs */
    int32_t interleaved;  /* 0 or 1 */
    int32_t weight_dtype; /* of the norms' weights and their gradients: the problem's dtype, or NA2D_F32 */
    float eps;            /* above 0 and finite; sums of squares are fp32 */
} seq_rotation;

typedef struct {
    int32_t B, heads, kv_heads, L, D; /* D in {16, 32, 64, 128}; kv_heads 0: queries only; B * L below 2^31 */
    int32_t dtype;
    seq_rotation rotation;
    int32_t shared;                   /* positions: 1: int32 [axes, L], of every batch item; 0: [B, axes, L]; contiguous */
    seq_strides q, k, q_out, k_out;   /* forward: inputs and outputs.  backward: the forward's inputs (read only where there is a weight), and the outputs' gradients */
    seq_strides dq, dk;               /* backward */
} seq_rotary_problem;

/* Host only. */
int seq_rotary_validate(const seq_rotary_problem *p, int backward);

/* q: [B, heads, L, D], k: [B, kv_heads, L, D] to q_out, k_out (other memory).  freqs: fp32 [pairs].  q_weight, k_weight: [D], each NULL for no norm. */
int seq_rotary_fwd(const seq_rotary_problem *p, const void *q, const void *k, const int32_t *positions, const float *freqs, const void *q_weight, const void *k_weight,
                   void *q_out, void *k_out, void *stream);

/* dq, dk and, of weights that are given, dq_weight, dk_weight [D] from the outputs' gradients dq_out, dk_out (strides p->q_out, p->k_out).  q, k may be NULL where their
 * weight is.  Sums are added in an order that does not vary. */
int seq_rotary_bwd(const seq_rotary_problem *p, const void *q, const void *k, const int32_t *positions, const float *freqs, const void *q_weight, const void *k_weight,
                   const void *dq_out, const void *dk_out, void *dq, void *dk, void *dq_weight, void *dk_weight, void *workspace, size_t workspace_bytes, void *stream);
size_t seq_rotary_bwd_workspace_bytes(const seq_rotary_problem *p);   /* for weights of both; needed only where there is one */

/*
 * The cache: pages of `page` consecutive tokens of one sequence, k_pages and v_pages int8 [pages, kv_heads, page, D], contiguous, with one fp32 scale
 * for each page and head, k_scales and v_scales [pages, kv_heads]; a value is the integer times the scale, of either
 * sign.  table: int32 [B, table_width]; position t of
 * sequence b lies in page table[b, t / page] at t % page.  lengths: int32 [B], tokens of each sequence.  Entries of the table whose positions a call
 * does not reach (behind the sequence, or before every query's window) may be anything, pages that nothing was ever written to included.  A page number outside [0, pages) is no page: nothing is written there, and nothing there is seen or
 * read; positions beyond table_width pages likewise.
 */
typedef struct {
    int32_t B, heads, kv_heads, D, page, pages, table_width;
    int32_t dtype; /* of the 16- or 32-bit tensors of the call */
    int32_t n;     /* new tokens of each sequence, or positions to read */
    int32_t window;
    float scale, softcap;
    seq_strides q, out; /* attention: queries and output.  append: the new keys and values.  gather: the keys and values read. */
} seq_cache_problem;

typedef enum { SEQ_CACHE_APPEND = 0, SEQ_CACHE_GATHER = 1, SEQ_CACHE_ATTENTION = 2 } seq_cache_call;

/* Host only.  page in {16, 32, 64, 128}; D in {32, 64, 128}; attention takes f16 and bf16, the others f32 too. */
int seq_cache_validate(const seq_cache_problem *p, int call);

/* Writes k, v [B, kv_heads, n, D] (strides p->q and p->out) at positions lengths[b] .. of every sequence; counts (nullable): int32 [B], how many of the n are
 * taken (at most n; 0 leaves the sequence alone).  A page's scale becomes the larger of the old one's magnitude and its new tokens' largest / 127; where that is another, the
 * tokens that the page held are rounded again, to nearest even, on the new scale (to 127 at most).  The first token of a page starts it afresh.  A NaN is
 * stored as 0, an infinity as the largest finite fp32 value (127 times the scale, which that rounding may make infinite again in fp32).  lengths is not changed.  A page must not be appended to twice in
 * one call (by two sequences, or through two entries of a table): which of the values it then holds is not defined. */
int seq_cache_append(const seq_cache_problem *p, const void *k, const void *v, const int32_t *table, const int32_t *lengths, const int32_t *counts,
                     int8_t *k_pages, int8_t *v_pages, float *k_scales, float *v_scales, void *stream);

/* The same of tokens picked out of k, v [B, kv_heads, given, D], with their keys normed and rotated on the way.  rows (nullable): int32 [B, n], the row of k and v that
 * is new token i; a row outside [0, given) is a token of zeros; NULL: the rows as they come, n of them.  r (nullable): how keys are rotated (pairs 0: not at all), with weight
 * (nullable) of a norm before that.  positions (nullable): int32 [axes, given] if `shared`, else [B, axes, given], of the given rows; NULL, with one axis: a token's place in its
 * sequence.  Rotated keys are rounded once, to the cache's 8 bits. */
int seq_cache_append_rows(const seq_cache_problem *p, const seq_rotation *r, int32_t given, const void *k, const void *v, const int32_t *rows, const int32_t *positions, int shared,
                          const float *freqs, const void *weight, const int32_t *table, const int32_t *lengths, const int32_t *counts, int8_t *k_pages, int8_t *v_pages,
                          float *k_scales, float *v_scales, void *stream);

/* k, v [B, kv_heads, n, D] (strides p->q and p->out): the values at positions first[b] .. first[b] + n - 1, 0 where the sequence has no token. */
int seq_cache_gather(const seq_cache_problem *p, const int8_t *k_pages, const int8_t *v_pages, const float *k_scales, const float *v_scales,
                     const int32_t *table, const int32_t *lengths, const int32_t *first, void *k, void *v, void *stream);

/* Attention of each sequence's last n tokens, q [B, heads, n, D], over its cache: the token at position lengths[b] - n + i sees positions
 * 0 .. lengths[b] - n + i, with `window` the nearest `window` of them.  Scores as above.  A query that sees nothing gives 0.  Weights are rounded to
 * fp16 where they enter a product; q enters it as fp16 on a power-of-two scale of its row (exact but for what is 2^-24 of the row's largest). */
int seq_cache_attention(const seq_cache_problem *p, const void *q, const int8_t *k_pages, const int8_t *v_pages, const float *k_scales,
                        const float *v_scales, const int32_t *table, const int32_t *lengths, const float *slopes, void *out, void *workspace,
                        size_t workspace_bytes, void *stream);
size_t seq_cache_attention_workspace_bytes(const seq_cache_problem *p);

/* Attention of a tree of n <= 64 drafted tokens, its nodes, over each sequence's cache, which does not hold them: q [B, heads, n, D]; k, v [B, kv_heads, n, D], the nodes'
 * own, in the problem dtype, with strides k_strides and v_strides.  parents: int32 [B, n]; a node's parent is a node before it, or -1: it follows the cache's last token.  Any
 * other value: no node (as padding), and neither is what descends from it; its q, k and v may be anything, and its row of out is 0.  A node stands at position lengths[b] +
 * its depth, and sees the cache, its ancestors and itself, all within `window` before it.  Scores as above.  Over the cache q and the
 * weights are rounded as in seq_cache_attention, but where a key head has more than 32 rows and the table holds work enough (rows times
 * tiles of 64 tokens of all sequences and key heads from 2^16 on) it is the weight times the size of its page's value scale that is held as fp16, on the power of two of the largest of those.  A value
 * scale of 2^-100 in size, or less, counts as 0 there; and of the tokens that a row sees one whose weight times scale (the nodes' own: 1) is not 0, but below 2^-126 of the largest such, is
 * left out of the row's sum.  Over the nodes weights are rounded to fp16, or in bf16 to a sum of two of them.  A node's k or v that is
 * infinite or no number reaches the rows that see the node, and no others.  The workspace is always needed. */
int seq_cache_tree_attention(const seq_cache_problem *p, const seq_strides *k_strides, const seq_strides *v_strides, const void *q, const void *k, const void *v, const int32_t *parents,
                             const int8_t *k_pages, const int8_t *v_pages, const float *k_scales, const float *v_scales, const int32_t *table, const int32_t *lengths, const float *slopes,
                             void *out, void *workspace, size_t workspace_bytes, void *stream);
size_t seq_cache_tree_attention_workspace_bytes(const seq_cache_problem *p);

/* Which drafted tokens a target accepts, and the token behind them.  tokens: int32 [B, n]; node 0 of a sequence is the token that its draft follows, the others are drafted.
 * logits: [B, n, V], the target's behind each node; rows' elements contiguous.  Of a row, p = softmax(logits / T), T = temperatures[b] (fp32 [B]; NULL: 1); T not above 0: all on the
 * largest logit, at its lowest index.  A logit of -infinity, or a NaN, is a token that is not chosen; an infinite one counts as the type's largest finite value.
 * A token is drawn from weights w by a number u: the lowest t with w_0 + .. + w_t > u (w_0 + .. + w_V-1), w_t > 0.  Everything from the logits on is in 64 bits.
 *
 * drafted 0: parents, int32 [B, n], makes the nodes a tree as seq_cache_tree_attention has it (NULL: a line).  At a node i a token is drawn from p_i by
 * uniforms[b, i] (fp32 [B, n]); if a child of it (the lowest) has this token the walk goes on there, else the token is the next one.
 * drafted 1: draft [B, n - 1, V], in the type of logits: the logits that tokens 1 .. n - 1 of a line were drawn from (parents NULL), q = softmax(draft / T).  Token x of node i + 1 is
 * accepted if uniforms[b, i] q_i(x) < p_i(x) (uniforms fp32 [B, n + 1]; T not above 0: if it is the largest logit's).  The first that is not, or whose number is no token (outside [0, V):
 * the end of a draft), ends the line; the next token is then drawn by uniforms[b, n], from max(p - q, 0) (from p where that is 0 throughout), at the end of the draft from p.
 * Numbers outside [0, 1) count as the nearest inside, a NaN as 0.
 *
 * path: int32 [B, n], the accepted nodes from node 0 on, then -1.  counts: int32 [B], how many there are (at least 1).  next: int32 [B], the next token; -1 from a row that gives none. */
typedef struct {
    int32_t B, n, V; /* n <= 64; V <= 2^24 */
    int32_t dtype;   /* of logits and draft */
    int32_t drafted; /* 1: with the draft's logits (draft is not read where n is 1) */
    int64_t batch, row, draft_batch, draft_row; /* strides in elements, 0 or more */
} seq_verify_problem;
int seq_verify_validate(const seq_verify_problem *p);
size_t seq_verify_workspace_bytes(const seq_verify_problem *p);
int seq_verify(const seq_verify_problem *p, const void *logits, const void *draft, const int32_t *tokens, const int32_t *parents, const float *uniforms, const float *temperatures,
               int32_t *path, int32_t *counts, int32_t *next, void *workspace, size_t workspace_bytes, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* SEQ_H_ */
