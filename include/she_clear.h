/*
 * she_clear.h - the clear side of split inference, part of the C ABI of the MI355X library (conventions of she.h).
 *
 * In split inference the projections whose weights a server shares among its clients are evaluated on ciphertexts
 * (she_shift_acc; Section 3.2 of arXiv 1906.00148), and the client runs what lies between a decryption and the next
 * encryption itself, on plain numbers: its own low-rank adapters beside such a projection, the norms and the rotation of
 * queries and keys, the places of new tokens in its cache, their attention over it, and the choice of the next token.  These calls
 * are that part for a decoder block and what a step of generation needs around it.
 *
 * Conventions beside those of she.h:
 *  - Every pointer inside an argument struct is a DEVICE pointer; the struct itself is read before the call returns.
 *  - Strides count elements; the last axis of every array is contiguous.  An array's rows may be views of a wider one.
 *  - The context's device (she_clear_device) has to be the current one (SHE_EINVAL).
 *  - A call enqueues its work on the context's stream and returns without waiting for it (like she_eval_gates_device).
 *    Arrays must stay valid until the stream has passed it.
 *  - Scratch belongs to the context and grows on demand, at least to twice its size; what it was before stays until she_free, so
 *    that captured graphs remain good.  A call that would have to allocate while its stream is captured is refused (SHE_ENOMEM):
 *    run it once before.  All calls of a context share the scratch: those on one stream are safe, and replays of a graph count as
 *    calls.
 *  - What the host can see is checked (SHE_EINVAL, SHE_ERANGE).  Ids in device arrays are checked by the kernels: one that is
 *    out of its range is left out, as each call says, never followed, and counted (she_clear_bad_ids).
 *  - Sums, softmax statistics and norms are held in 32 bits; results are rounded once, to nearest.  (Attention's weights are rounded to
 *    the type before, their sum is not, where requests have many rows, new tokens times the query heads of a key head, over many
 *    places.  Requests of up to 32 rows on average behind shared prefixes are not among them, nor single tokens of up to 8.)
 *  - No result depends on the order in which the GPU runs things: the same call gives the same bits.
 */
#ifndef SHE_CLEAR_H
#define SHE_CLEAR_H

#include "she.h"

#ifdef __cplusplus
extern "C" {
#endif

enum { SHE_BF16 = 0, SHE_F16 = 1, SHE_F32 = 2, SHE_I32 = 3, SHE_NO_BASE = -1 };   /* types of elements */

/* Low-rank adapters of many requests beside a shared projection:
 *   out[t][n] = base[t][n] + scale[a] * sum_{j < ranks[a]} up[a][j][n] * sum_k down[a][j][k] * x[t][k]
 * for the tokens t in [starts[s], starts[s+1]) of every segment s, a = which[s].  starts is ascending from 0 to `tokens`
 * (tokens outside every segment are not written).  which[s] = -1: no adapter, out = base; any other value outside
 * [0, adapters) likewise, and counted.  Both matrices lie rank-major, so that a rank's row is contiguous.
 * base: none, elements of `type`, SHE_F32, or SHE_I32: the projection's sums as decrypted, times step[n] (NULL: 1).  out may
 * be base itself where their elements are of one type. */
typedef struct {
    int32_t type;                        /* SHE_BF16 or SHE_F16: x, down, up, out */
    int32_t base_type;                   /* SHE_NO_BASE, `type`, SHE_F32 or SHE_I32 */
    uint32_t tokens, inputs, outputs;
    uint32_t adapters, rank, segments;   /* rank <= 512: the rows that every adapter has room for */
    const void *x;                       /* [tokens][inputs] */
    int64_t x_stride;
    const void *down;                    /* [adapters][rank][inputs] */
    int64_t down_adapter, down_rank;     /* strides of its first two axes */
    const void *up;                      /* [adapters][rank][outputs] */
    int64_t up_adapter, up_rank;
    const int32_t *starts;               /* [segments + 1] */
    const int32_t *which;                /* [segments] */
    const int32_t *ranks;                /* [adapters], each taken as at most `rank`; NULL: all have `rank` */
    const float *scale;                  /* [adapters] */
    const void *base;                    /* [tokens][outputs] */
    int64_t base_stride;
    const float *step;                   /* [outputs], with SHE_I32 */
    void *out;                           /* [tokens][outputs] */
    int64_t out_stride;
} she_adapters_args;
int she_adapters(she_ctx *ctx, const she_adapters_args *args);

/* Gradients of she_adapters for dy = d loss / d out:
 *   dx[t] = base[t] + scale[a] * sum_j (up[a][j] . dy[t]) * down[a][j]
 *   ddown[a][j] = scale[a] * sum_t (up[a][j] . dy[t]) * x[t],   dup[a][j] = scale[a] * sum_t (down[a][j] . x[t]) * dy[t]
 * over all tokens of all segments of adapter a.  base: the gradient that reaches x through the projection itself, of `type` or
 * SHE_F32, or none.  ddown and dup are written whole ([adapters][rank][..], contiguous): zeros where no token or rank leads. */
typedef struct {
    int32_t type, base_type;
    uint32_t tokens, inputs, outputs;
    uint32_t adapters, rank, segments;
    const void *dy;                      /* [tokens][outputs] */
    int64_t dy_stride;
    const void *x;
    int64_t x_stride;
    const void *down;
    int64_t down_adapter, down_rank;
    const void *up;
    int64_t up_adapter, up_rank;
    const int32_t *starts, *which, *ranks;
    const float *scale;
    const void *base;                    /* [tokens][inputs] */
    int64_t base_stride;
    void *dx;                            /* [tokens][inputs] */
    int64_t dx_stride;
    void *ddown, *dup;
} she_adapters_grad_args;
int she_adapters_grad(she_ctx *ctx, const she_adapters_grad_args *args);

/* Norms of queries and keys for each head, with the rotation of the position in the same pass.  For every head x[0..head) of q
 * and k:  n = x * w / sqrt(mean(x^2) + eps);  of its first `rot` elements the pairs (a, b), neighbours (interleaved) or `rot/2`
 * apart, become (a*c - b*s, b*c + a*s) with c, s = cos, sin[positions[t]][pair].  A token whose position is outside
 * [0, places) gets zeros, and is counted.
 * Without pages the keys go to k_out.  With pages (k_pages not NULL) keys and values go to place slots[t] of the cache, page
 * slots[t] / page_size, and k_out is not used; slots[t] = -1: the token is not stored; any other value outside
 * [0, pages * page_size) likewise, and counted (a token without a place in the rotation's table is not stored either).  No two
 * tokens of a call may name the same place.  q_out and k_out may be q and k. */
typedef struct {
    int32_t type;                        /* SHE_BF16 or SHE_F16 */
    int32_t interleaved;
    uint32_t tokens, q_heads, kv_heads;
    uint32_t head, rot;                  /* head <= 512, rot even, rot <= head */
    uint32_t places;
    float eps;
    const void *q, *k, *v;               /* [tokens][heads][head]; v only with pages */
    int64_t q_token, q_head, k_token, k_head, v_token, v_head;
    const float *wq, *wk;                /* [head]; NULL: ones */
    const float *cosines, *sines;        /* [places][rot / 2] */
    const int32_t *positions;            /* [tokens] */
    void *q_out, *k_out;
    int64_t q_out_token, q_out_head, k_out_token, k_out_head;
    void *k_pages, *v_pages;             /* [pages][page_size][kv_heads][head], strides shared by both */
    int64_t page_stride, slot_stride, page_head;
    uint32_t pages, page_size;
    const int64_t *slots;                /* [tokens] */
} she_qk_rotate_args;
int she_qk_rotate(she_ctx *ctx, const she_qk_rotate_args *args);

/* Gradients of she_qk_rotate (without pages) for dq_out, dk_out; q and k are its inputs.  dwq, dwk [head]: sums over all tokens
 * and heads.  Any of dwq, dwk may be NULL.  Tokens without a place get zeros and add nothing. */
typedef struct {
    int32_t type, interleaved;
    uint32_t tokens, q_heads, kv_heads;
    uint32_t head, rot;
    uint32_t places;
    float eps;
    const void *dq_out, *dk_out;
    int64_t dq_out_token, dq_out_head, dk_out_token, dk_out_head;
    const void *q, *k;
    int64_t q_token, q_head, k_token, k_head;
    const float *wq, *wk;
    const float *cosines, *sines;
    const int32_t *positions;
    void *dq, *dk;
    int64_t dq_token, dq_head, dk_token, dk_head;
    float *dwq, *dwk;
} she_qk_rotate_grad_args;
int she_qk_rotate_grad(she_ctx *ctx, const she_qk_rotate_grad_args *args);

/* Attention of each request's new tokens over its paged cache.  Request r has the new tokens [starts[r], starts[r+1]) of q and
 * lengths[r] places in the cache, the new tokens' own the last among them: new token i of n stands at p = lengths[r] - n + i and
 * attends to the places max(0, p - window + 1) .. p (window = 0: all from 0 on), place u of request r being slot u % page_size
 * of page table[r][u / page_size]:
 *   out = sum_u softmax_u(scale * q . k_u) v_u,  query head h reading key head h / (q_heads / kv_heads).
 * A token that attends to nothing gets zeros.  Places whose page id is outside [0, pages) are attended to by nobody, and counted
 * where a token's window has them (the pages that every window has passed may be gone); so are, uncounted, places that the table has
 * no column for.  What the slots of such places hold, of places beyond the length and
 * of places that a token does not attend to, infinities and NaN too, has no part in its result.  starts is ascending from 0 to
 * `tokens`.  At most 2^26 places (table_width * page_size). */
typedef struct {
    int32_t type;                        /* SHE_BF16 or SHE_F16 */
    uint32_t tokens, requests, q_heads, kv_heads;
    uint32_t head;                       /* a multiple of 8, at most 256 */
    uint32_t window;
    float scale;
    const void *q;                       /* [tokens][q_heads][head]; rows start on 16 bytes */
    int64_t q_token, q_head;
    const void *k_pages, *v_pages;       /* [pages][page_size][kv_heads][head], strides shared by both; rows start on 16 bytes */
    int64_t page_stride, slot_stride, page_head;
    uint32_t pages, page_size;
    const int32_t *table;                /* [requests][table_width] */
    int64_t table_stride;
    uint32_t table_width;
    const int32_t *starts;               /* [requests + 1] */
    const int32_t *lengths;              /* [requests] */
    void *out;                           /* [tokens][q_heads][head]; rows start on 16 bytes */
    int64_t out_token, out_head;
} she_attend_pages_args;
int she_attend_pages(she_ctx *ctx, const she_attend_pages_args *args);

/* Places in a paged cache for the new tokens of a step, worked out from the requests' lengths on the GPU: the starts, lengths,
 * positions, slots and table that she_qk_rotate and she_attend_pages read.  Request r has cached[r] places and gets news[r] more:
 *   starts[r+1] = min(starts[r] + news[r], tokens), starts[0] = 0;  lengths[r] = cached[r] + starts[r+1] - starts[r];
 * its columns of the table from ceil(cached[r] / page_size) up to ceil(lengths[r] / page_size), which it has not yet, get pages off
 * the list `free`, from its entry taken[0] on, request by request and column by column; taken_out[0] is the entry after the last.
 * Token starts[r] + i has place u = cached[r] + i: position before[r] + u and slot table[r][u / page_size] * page_size +
 * u % page_size.  A token gets slot -1, and is counted, where the list is at its end (that column gets -1, as it does from an id
 * outside [0, pages) in the list), where the page that its request has already is outside [0, pages), and where the table has no
 * column for it.  The tokens from starts[requests] on are the padding of a batch: position 0, slot -1, not counted.  Other columns are
 * left as they are.  Numbers below 0 in cached, news, taken and before count as 0, and positions end at 2^31 - 1.  lengths may be
 * cached, taken_out may be taken; no other two arrays, and no two rows of the table, may share memory. */
typedef struct {
    uint32_t requests, tokens;           /* tokens: the room in positions and slots */
    uint32_t pages, page_size, table_width, free_count;
    const int32_t *cached, *news;        /* [requests] */
    const int32_t *before;               /* [requests]: places before a request's own, as of a shared prefix; NULL: none */
    const int32_t *free;                 /* [free_count] */
    const int32_t *taken;                /* [1] */
    int32_t *table;                      /* [requests][table_width] */
    int64_t table_stride;
    int32_t *starts;                     /* [requests + 1] */
    int32_t *lengths;                    /* [requests] */
    int32_t *positions;                  /* [tokens] */
    int64_t *slots;                      /* [tokens] */
    int32_t *taken_out;                  /* [1] */
} she_plan_pages_args;
int she_plan_pages(she_ctx *ctx, const she_plan_pages_args *args);

/* she_attend_pages for requests that begin with the same text, whose places are in the cache once and are read once for all of
 * them.  The requests [prefix_requests[g], prefix_requests[g+1]) have the prefix g of prefix_lengths[g] places, place u being slot
 * u % page_size of page prefix_table[g][u / page_size]; prefix_requests is ascending, and requests outside all of it have no prefix.
 * lengths, starts and table are the requests' own places, which follow the prefix on pages of their own: new token i of n stands at
 * p = lengths[r] - n + i of them and attends to its own places 0 .. p and to the whole prefix; with a window, to the last `window`
 * of the row of both.  A token with p < 0 attends to nothing and gets zeros.  Page ids out of range, places without a column and
 * what lies in places that are not attended to: as in she_attend_pages.  At most 2^26 places of a prefix and of a request. */
typedef struct {
    int32_t type;                        /* SHE_BF16 or SHE_F16 */
    uint32_t tokens, requests, q_heads, kv_heads;
    uint32_t head;                       /* a multiple of 8, at most 256 */
    uint32_t window;
    float scale;
    const void *q;                       /* [tokens][q_heads][head]; rows start on 16 bytes */
    int64_t q_token, q_head;
    const void *k_pages, *v_pages;       /* [pages][page_size][kv_heads][head], strides shared by both; rows start on 16 bytes */
    int64_t page_stride, slot_stride, page_head;
    uint32_t pages, page_size;
    const int32_t *table;                /* [requests][table_width] */
    int64_t table_stride;
    uint32_t table_width;
    uint32_t prefixes, prefix_width;
    const int32_t *starts;               /* [requests + 1] */
    const int32_t *lengths;              /* [requests] */
    const int32_t *prefix_table;         /* [prefixes][prefix_width] */
    int64_t prefix_stride;
    const int32_t *prefix_requests;      /* [prefixes + 1] */
    const int32_t *prefix_lengths;       /* [prefixes] */
    void *out;                           /* [tokens][q_heads][head]; rows start on 16 bytes */
    int64_t out_token, out_head;
} she_attend_shared_args;
int she_attend_shared(she_ctx *ctx, const she_attend_shared_args *args);

/* The next token of every row of logits.  A logit is an element of `type`, or with SHE_I32 a projection's decrypted sum times step[i]
 * (NULL: 1), as a number of 32 bits; NaN counts as -infinity.  With x_i = logit_i / temperature, the weight of token i is
 * exp(x_i - max x).  Kept are the top_k largest (of equals the lower index first), of these the shortest head in that order whose
 * weight reaches top_p of theirs, and of these the tokens with a weight of at least min_p.  The token is the first, by index, at
 * which the running weight of the kept tokens exceeds uniform times their whole weight; probs is its share of that weight.
 * top_k < 1, top_p >= 1 or NaN, and min_p <= 0 or NaN keep all, and the likeliest token is kept in any case.  A temperature of 0 (or
 * below, or NaN) takes the largest logit of lowest index with probability 1, and so does +infinity, shared equally by all that have
 * it where the temperature is above 0.  A row without a logit above -infinity gets token -1, probability 0.  uniform is taken as at
 * least 0 (NaN too) and at most 1 - 2^-24.  Weights are held to 2^-44 of the largest, less than which is none, and their sums are exact;
 * but where temperature is all that a call sets and vocab is more than 8192, every 512 tokens' running weight is held to 2^-44 of the
 * row's largest, and each of theirs to 2^-44 of the largest among them: tokens of less than 2^-44.5 have some if others of the 512
 * have more.  tokens may be top_k, and probs may be uniform, temperature, top_p or min_p; neither shares memory with
 * anything else. */
typedef struct {
    int32_t type;                        /* SHE_BF16, SHE_F16, SHE_F32 or SHE_I32 */
    uint32_t rows, vocab;                /* vocab at most 2^20 */
    const void *logits;                  /* [rows][vocab] */
    int64_t row_stride;
    const float *step;                   /* [vocab], with SHE_I32 */
    const float *uniform;                /* [rows] */
    const float *temperature;            /* [rows]; NULL: 1 */
    const int32_t *top_k;                /* [rows]; NULL: all */
    const float *top_p;                  /* [rows]; NULL: 1 */
    const float *min_p;                  /* [rows]; NULL: 0 */
    int32_t *tokens;                     /* [rows] */
    float *probs;                        /* [rows]; may be NULL */
} she_sample_args;
int she_sample(she_ctx *ctx, const she_sample_args *args);

/* Ids out of range that the kernels of this context's clear calls have left out since the last reset (several for one id, where
 * several workgroups meet it).  Waits for the stream; refused while that is captured (SHE_EINVAL). */
int she_clear_bad_ids(she_ctx *ctx, uint64_t *count, int reset);

/* The HIP device that the context's arrays are on: the one that was current at she_keygen.  -1 for NULL. */
int she_clear_device(const she_ctx *ctx);

#ifdef __cplusplus
}
#endif
#endif /* SHE_CLEAR_H */
