/*
 * she_clear.h - the clear side of split inference, part of the C ABI of the MI355X library (conventions of she.h).
 *
 * In split inference the projections whose weights a server shares among its clients are evaluated on ciphertexts
 * (she_shift_acc; Section 3.2 of arXiv 1906.00148), and the client runs what lies between a decryption and the next
 * encryption itself, on plain numbers: its own low-rank adapters beside such a projection, the norms and the rotation of
 * queries and keys, and the attention of new tokens over its cache.  These calls are that part for a decoder block.
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
 *  - Sums, softmax statistics and norms are held in 32 bits; results are rounded once, to nearest.
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

/* Ids out of range that the kernels of this context's clear calls have left out since the last reset (several for one id, where
 * several workgroups meet it).  Waits for the stream; refused while that is captured (SHE_EINVAL). */
int she_clear_bad_ids(she_ctx *ctx, uint64_t *count, int reset);

/* The HIP device that the context's arrays are on: the one that was current at she_keygen.  -1 for NULL. */
int she_clear_device(const she_ctx *ctx);

#ifdef __cplusplus
}
#endif
#endif /* SHE_CLEAR_H */
