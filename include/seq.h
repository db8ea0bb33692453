/*
 * seq.h -- C ABI of the MI355X (gfx950) attention over token sequences (same library as na2d.h, whose dtype and status
 * codes are reused): softmax attention with causal order, a window, capped scores, a distance bias, a document mask and a
 * prefix mask, forward and backward; and, for serving, a cache of keys and values held in 8 bits, its append, reading it
 * back, and attention over it.
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
 * The cache: pages of `page` consecutive tokens of one sequence, k_pages and v_pages int8 [pages, kv_heads, page, D], contiguous, with one fp32 scale
 * for each page and head, k_scales and v_scales [pages, kv_heads]; a value is the integer times the scale.  table: int32 [B, table_width]; position t of
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
 * taken (at most n; 0 leaves the sequence alone).  A page's scale becomes the larger of the old one and its new tokens' largest magnitude / 127; where it grows, the
 * tokens that the page held are rounded again, to nearest even, on the new scale.  The first token of a page starts it afresh.  A NaN is
 * stored as 0, an infinity as the largest finite fp32 value.  lengths is not changed.  A page must not be appended to twice in
 * one call (by two sequences, or through two entries of a table): which of the values it then holds is not defined. */
int seq_cache_append(const seq_cache_problem *p, const void *k, const void *v, const int32_t *table, const int32_t *lengths, const int32_t *counts,
                     int8_t *k_pages, int8_t *v_pages, float *k_scales, float *v_scales, void *stream);

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

#ifdef __cplusplus
}
#endif
#endif /* SEQ_H_ */
