/*
 * dpo_ends.h -- the two ends of a pipeline and its residual stream, C ABI.
 *
 * The first stage's embedding and its gradient, the last stage's head with the log
 * probabilities of the tokens that follow and their gradient, and dropout where a
 * branch joins the stream: what a pipeline runs around the blocks of dpo.h ("The
 * feed-forward half of a pipeline stage"), with the same weights, dpo_read_weights's
 * stale ones, and the same gradient buffers.
 *
 * The rules are those of that part of dpo.h: no context; the caller owns every buffer,
 * workspace included, all device memory of the current device; matrices are row-major
 * with contiguous rows, ld their pitch in elements; outputs overlap neither inputs nor
 * one another, except where a call says so; nothing is allocated and the host is never
 * synchronized; two calls may share a workspace only on one stream; a call of zero
 * tokens or rows launches nothing, except that a gradient of weights that is not
 * accumulated is set to zero. Errors: a DPO_E* code, with the message of the calling
 * thread's last failure in dpo_last_error(NULL).
 *
 * Token ids. An id outside 0 .. vocab - 1 is no token but padding, whatever its value:
 * its embedding is a row of zeros, its log probability 0, and neither has a gradient.
 */
#ifndef DPO_ENDS_H
#define DPO_ENDS_H

#include "dpo.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Token t = r cols + c is element r ld + c: a block of a matrix of tokens, or a vector
 * (rows 1). */
typedef struct {
    const void *p;              /* int32 or int64 */
    int64_t rows, cols, ld;
    int bytes;                  /* of an id: 4 or 8 */
} dpo_ids;

/* out[t] = scale table[id_t], rounded once. */
typedef struct {
    dpo_ids ids;                /* rows x cols = tokens */
    const void *table;          /* table_dtype, vocab x dim */
    void *out;                  /* out_dtype, tokens x dim */
    int64_t vocab, dim;         /* both in [1, 2^31) */
    int64_t ld_table, ld_out;
    float scale;                /* finite */
    int table_dtype, out_dtype; /* DPO_F32 or DPO_BF16 */
} dpo_embed_args;

/* Returns DPO_OK, DPO_EINVAL, DPO_EALIGN (a pointer not aligned to its elements),
 * DPO_EDTYPE or DPO_ECUDA, as all calls here. */
int dpo_embed(const dpo_embed_args *args, void *cuda_stream);

/*
 * dtable[v] (+)= scale * sum over t with id_t = v of dy[t], in fp32, in an order that the
 * ids alone decide (ascending t in spans, then the spans' sums), rounded once for
 * DPO_EMBED_SPAN tokens; more tokens are added to dtable span after span. Written rows are all of
 * dtable's, or with accumulate those of the ids met.
 */
#define DPO_EMBED_SPAN 65536

typedef struct {
    const void *dy;             /* dtype, tokens x dim */
    dpo_ids ids;
    void *dtable;               /* grad_dtype, vocab x dim */
    int64_t vocab, dim;
    int64_t ld_dy, ld_dtable;
    float scale;
    int dtype, grad_dtype;
    int accumulate;             /* add to dtable instead of replacing it */
    void *workspace;            /* dpo_embed_workspace bytes, 256-byte aligned */
    int64_t workspace_bytes;
} dpo_embed_backward_args;

int dpo_embed_backward(const dpo_embed_backward_args *args, void *cuda_stream);
int dpo_embed_workspace(int64_t tokens, int64_t vocab, int64_t dim, int64_t *bytes);

/*
 * Dropout from a counter-based generator; no mask is stored:
 *   y = residual + (kept ? x / (1 - p') : 0)
 * p' = c / 65536, c = floor(65536 p + 1/2) < 65536. Element (row, col) is kept when its
 * 16 random bits are >= c: half col mod 2 (0: the low one) of word (col / 2) mod 4 of
 * Philox4x32-10 (Salmon, Moraes, Dror and Shaw, SC'11) on the counter
 * (col / 8, row's low word, row's high word, site) under the key seed. The mask depends on
 * (seed, site, row, col) alone; the backward pass is the same call on dy without a
 * residual. Dropped elements do not read as numbers: an infinity or NaN among them is
 * gone. y may be x or residual itself (same pointer and pitch).
 */
typedef struct {
    const void *x;              /* dtype, rows x cols */
    const void *residual;       /* dtype, or NULL: none */
    void *y;                    /* dtype */
    int64_t rows, cols;         /* below 2^31 */
    int64_t ld_x, ld_residual, ld_y;
    int dtype;
    uint32_t site;              /* which dropout of a step: masks of two sites are independent */
    uint64_t seed;
    const uint64_t *seed_source; /* device memory, or NULL: read in place of seed when the
                                    kernel runs, so that a captured call draws anew */
    double p;                   /* in [0, 1) */
} dpo_dropout_args;

int dpo_dropout(const dpo_dropout_args *args, void *cuda_stream);

/*
 * Log probabilities of given tokens. Per row of logits, with z = scale * logit in fp32,
 * m = max z, S = sum e^(z - m):
 *   logp = z_id - m - log S,  entropy = log S - sum e^(z - m) (z - m) / S,
 *   stats = (m, log S),
 *   top ids: those of the `top` largest z, descending, ties to the lowest id, NaN below
 *   all numbers; top logp: theirs.
 * Logits of -infinity are masked: probability 0, no part in sums. A row of nothing else,
 * or with a NaN or +infinity, has no distribution: logp, entropy and top logp are NaN.
 */
#define DPO_MAX_TOP 32

typedef struct {
    const void *logits;         /* dtype, rows x vocab */
    dpo_ids ids;                /* p NULL: none given (logp is then not written) */
    float *logp;                /* rows */
    float *entropy;             /* rows, or NULL */
    float *stats;               /* rows x 2 */
    float *top_logp;            /* rows x top */
    int64_t *top_ids;           /* rows x top */
    int64_t rows, vocab;        /* vocab in [1, 2^31) */
    int64_t ld_logits;
    float scale;                /* 1e-20 to 1e6 */
    int dtype;
    int top;                    /* 0 .. min(DPO_MAX_TOP, vocab) */
} dpo_logprobs_args;

int dpo_logprobs(const dpo_logprobs_args *args, void *cuda_stream);

/*
 * Its backward pass, with p = e^(z - m - log S), a = dlogp (0 for padding), b = dentropy:
 *   dlogits = scale (a (1[j = id] - p) - b p (log p + entropy))
 * A row with a = b = 0 gets zeros, whatever its logits. dlogits may be logits itself
 * (same pointer, pitch and type).
 */
typedef struct {
    const void *logits;
    dpo_ids ids;
    const float *stats;         /* the forward's */
    const float *entropy;       /* the forward's; needed with dentropy */
    const float *dlogp;         /* rows */
    const float *dentropy;      /* rows, or NULL: zeros */
    void *dlogits;              /* dtype */
    int64_t rows, vocab;
    int64_t ld_logits, ld_dlogits;
    float scale;
    int dtype;
} dpo_logprobs_backward_args;

int dpo_logprobs_backward(const dpo_logprobs_backward_args *args, void *cuda_stream);

/*
 * The head: the same from the stream and the head's weights,
 *   logits = x w^T  (bf16 operands, fp32 accumulation, not rounded),
 * and the gradients of both,
 *   G = dlogits in bf16 (the type of the products that read it),
 *   dx = G w,  dw (+)= G^T x.
 * Logits are never stored in full precision where `top` is 0. dim is a multiple of 8, vocab any;
 * pointers are 16-byte aligned and the pitches of x and dx multiples of 8.
 */
typedef struct {
    const void *x;              /* bf16, tokens x dim */
    const void *w;              /* bf16, vocab x dim, pitch dim */
    dpo_ids ids;                /* p NULL: none given (logp is then not written) */
    float *logp;                /* tokens */
    float *entropy;             /* tokens */
    float *stats;               /* tokens x 2, as dpo_logprobs's */
    float *top_logp;            /* tokens x top */
    int64_t *top_ids;
    void *kept;                 /* what the backward needs, or NULL: 256-byte aligned */
    int64_t tokens, dim, vocab;
    int64_t ld_x;
    float scale;                /* 1e-20 to 1e6 */
    int top;
    void *workspace;            /* 256-byte aligned */
    int64_t workspace_bytes;
} dpo_head_args;

int dpo_head(const dpo_head_args *args, void *cuda_stream);

typedef struct {
    const void *x, *w;
    dpo_ids ids;
    const void *kept;
    const float *logp, *entropy, *stats;   /* the forward's */
    const float *dlogp;         /* tokens */
    const float *dentropy;      /* tokens, or NULL: zeros */
    void *dx;                   /* bf16, tokens x dim, or NULL */
    void *dw;                   /* grad_dtype, vocab x dim, pitch dim */
    int64_t tokens, dim, vocab;
    int64_t ld_x, ld_dx;
    float scale;
    int grad_dtype;             /* DPO_F32 or DPO_BF16 */
    int accumulate;             /* add to dw instead of replacing it */
    void *workspace;
    int64_t workspace_bytes;
} dpo_head_backward_args;

int dpo_head_backward(const dpo_head_backward_args *args, void *cuda_stream);

/* Bytes of the forward's workspace (with or without kept, with such a top), of kept and of
 * the backward's workspace; each result may be NULL. */
int dpo_head_workspace(int64_t tokens, int64_t dim, int64_t vocab, int keep, int top,
                       int64_t *forward_bytes, int64_t *kept_bytes, int64_t *backward_bytes);

#ifdef __cplusplus
}
#endif
#endif /* DPO_ENDS_H */
