/*
 * kt operators -- the parts of a transformer block's training pass that make
 * the gradients which kt.h packs, reduces and applies: layer norm with its
 * backward pass, activation checkpoints in 8 bits with the weight gradient of
 * a linear layer from them, and attention with its backward pass.
 *
 * The conventions of kt.h hold: status codes, kt_last_error(), device pointers
 * owned by the caller, asynchronous calls on `stream`.  Beyond them:
 *  - The calls need no plan and keep nothing between calls: no allocation, no
 *    upload, no wait, no memory that has to start at zero.  Every one of them
 *    may be recorded into a HIP graph, without an eager call before it.
 *  - Scratch memory is the caller's: kt_*_workspace() says how many bytes a
 *    call needs (0: none, `ws` may be NULL), aligned to 16.  Its contents mean
 *    nothing before or after the call; calls on different streams need one each.
 *  - Weight gradients may be written where a bucket keeps them: any address
 *    that is a multiple of the element size will do.
 *  - Sums, softmax statistics and products are held in binary32; a result is
 *    rounded to bf16 once, to nearest-even.  bf16 attention rounds more on the
 *    way, as it says below.  Results depend on the arguments alone: no atomics,
 *    every sum has a fixed order.
 *  - A matrix [rows, cols] has adjacent columns and rows `ld` elements apart
 *    (ld >= cols).  Rows may be 0: then weight gradients are written as 0.
 *  - Outputs must not overlap inputs or each other, except where a call says so.
 */
#ifndef KT_OPS_H
#define KT_OPS_H

#include "kt.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ---- layer norm ---------------------------------------------------------------- */

#define KT_LAYERNORM_MAX_COLS 16384

/*
 * y = (x - mean) * rstd * gamma + beta for every row, with mean the row's mean
 * and rstd = 1 / sqrt(mean((x - mean)^2) + eps), both from the row itself in
 * two steps (no E[x^2] - mean^2).
 *
 *   dt          type of x and y;  pdt: type of gamma and beta.
 *   beta        may be NULL (no bias).
 *   mean, rstd  rows floats each, for the backward pass; both NULL: not wanted.
 *   y8, e8      both NULL, or the 8-bit checkpoint of y (as stored), written in
 *               the same pass: bit-identical to kt_act8_save(y).
 * y may be x itself (same ld).
 * Errors: KT_EINVAL (NULL, sizes, eps negative or not finite, overlap),
 * KT_EALIGN, KT_EUNSUPPORTED (cols > KT_LAYERNORM_MAX_COLS).
 */
KT_API kt_status kt_layernorm_fwd(kt_dtype dt, kt_dtype pdt, int64_t rows,
                                  int64_t cols, const void *x, int64_t ldx,
                                  const void *gamma, const void *beta, float eps,
                                  void *y, int64_t ldy, float *mean, float *rstd,
                                  int8_t *y8, uint8_t *e8, void *stream);

/*
 * The gradients of kt_layernorm_fwd from dy: with xh = (x - mean) * rstd and
 * t = gamma * dy,
 *   dx     = rstd * (t - mean(t) - xh * mean(t * xh))     (means over the row)
 *   dgamma = sum over rows of dy * xh,   dbeta = sum over rows of dy.
 * The input is x, or (x == NULL) its 8-bit checkpoint x8, e8; mean and rstd are
 * those that the forward pass left.
 *   dt          type of dy, x and dx;  pdt: type of gamma, dgamma and dbeta.
 *   dx          may be dy or x itself (same ld).
 *   dbeta       may be NULL.
 *   ws          kt_layernorm_bwd_workspace(rows, cols) bytes.
 * Errors as above; KT_EINVAL also for both or neither of x and x8, and for a
 * workspace that is too small.
 */
KT_API int64_t kt_layernorm_bwd_workspace(int64_t rows, int64_t cols);
KT_API kt_status kt_layernorm_bwd(kt_dtype dt, kt_dtype pdt, int64_t rows,
                                  int64_t cols, const void *dy, int64_t lddy,
                                  const void *x, int64_t ldx, const int8_t *x8,
                                  const uint8_t *e8, const void *gamma,
                                  const float *mean, const float *rstd, void *dx,
                                  int64_t lddx, void *dgamma, void *dbeta,
                                  void *ws, int64_t ws_bytes, void *stream);

/* ---- activation checkpoints in 8 bits ------------------------------------------- */

/*
 * A checkpoint of a matrix x [rows, cols] is
 *   q  rows x (32 * G) int8, G = ceil(cols / 32); columns past cols hold 0,
 *   e  rows x G bytes,
 * and stands for q * 2^(e - 127), one e for 32 neighbouring columns.  With a the
 * largest magnitude of the 32 and 2^E <= a < 2^(E+1):
 *   e = max(E - 6 + 127, 1),  q = rint(x * 2^(127 - e)) clamped to [-127, 127]
 * (ties to even).  The scale being a power of two, the one rounding is that of q:
 * at most half a step of 2^(e - 127), one step for a member that is clamped
 * (a >= 127.5 steps); every value that q stands for is exact in bf16.  A step is at
 * most a / 64 where a >= 2^-120; below that e stays 1 and a step 2^-126, and
 * members of up to half of it become 0.
 * A group with a member that is not finite has e = 255 and q = 0 and stands for
 * NaN throughout, so that an overflow is not hidden.
 * A checkpoint takes 1.03 bytes an element.
 */
KT_API kt_status kt_act8_save(kt_dtype dt, int64_t rows, int64_t cols,
                              const void *x, int64_t ldx, int8_t *q, uint8_t *e,
                              void *stream);
KT_API kt_status kt_act8_restore(kt_dtype dt, int64_t rows, int64_t cols,
                                 const int8_t *q, const uint8_t *e, void *y,
                                 int64_t ldy, void *stream);

/*
 * The weight gradient of a linear layer y = x W^T from the checkpoint of its
 * input: dw[o, i] = sum over t of dy[t, o] * x8[t, i].
 *   dt   type of dy [tokens, out];  gdt: type of dw [out, in].
 *   q, e the checkpoint of x [tokens, in].
 *   ws   kt_act8_weight_grad_workspace(...) bytes.
 * bf16 dy: products of bf16 pairs, exact, summed in binary32.  f32 dy: binary32
 * products and sums.  lddw >= in: dw may be a window of a larger matrix.  out
 * and in are at most 2^24, tokens at most 2^40.
 */
KT_API int64_t kt_act8_weight_grad_workspace(kt_dtype dt, int64_t tokens,
                                             int64_t out, int64_t in);
KT_API kt_status kt_act8_weight_grad(kt_dtype dt, kt_dtype gdt, int64_t tokens,
                                     int64_t out, int64_t in, const void *dy,
                                     int64_t lddy, const int8_t *q,
                                     const uint8_t *e, void *dw, int64_t lddw,
                                     void *ws, int64_t ws_bytes, void *stream);

/* ---- attention ------------------------------------------------------------------ */

#define KT_ATTENTION_MAX_DIM 128

/* A tensor [batch, tokens, heads, dim] with adjacent elements of a head; strides in elements, >= 0. */
typedef struct {
    void *data;
    int64_t batch, token, head;
} kt_heads;

/*
 * Sizes and mask shared by the forward and the backward pass.  KT_EUNSUPPORTED: dim over KT_ATTENTION_MAX_DIM, more than
 * 2^30 queries, keys or sequences, more than 2^16 heads, or 2^24 workgroups: batch * heads * ceil(nq / 128), and
 * in the backward pass batch * kv_heads * ceil(nk / 128).
 */
typedef struct {
    kt_dtype dt;                  /* type of all tensors but lse                         */
    int64_t batch, nq, nk;        /* sequences, queries and keys of each                 */
    int64_t heads, kv_heads;      /* kv_heads divides heads: query head h reads key head h / (heads / kv_heads) */
    int64_t dim;                  /* 1 .. KT_ATTENTION_MAX_DIM                           */
    float scale;                  /* of the scores; finite and > 0                       */
    int causal;                   /* query i sees keys j <= i + nk - nq only             */
    const int32_t *k_lens;        /* device, batch entries, or NULL: keys j >= k_lens[b] are not seen */
} kt_attention;

/*
 * Rounding in bf16: the probabilities are rounded to bf16 as an operand of the
 * product with v, and in the backward pass p and ds as operands of theirs; the
 * sum of the softmax takes them before that.  delta comes from o as it was stored.
 * So o stands 2.0e-3 from the formulas in norm and the gradients 2.4e-3; rounding
 * once at the end leaves 1.5e-3 and 1.8e-3 (normal inputs, 2048 and 8191 keys,
 * causal).  f32 has no rounding but that of its own arithmetic.
 *
 * o = softmax(scale * q k^T) v over the keys that a query sees, and lse, the
 * logarithm of the softmax's denominator [batch, heads, nq] in binary32.  A
 * query that sees no key gets o = 0 and lse = -inf whatever the keys hold.  Keys
 * at and past k_lens[b] are not read; a value k_lens[b] outside [0, nk] counts as the nearer end.
 * The causal mask gives a key no weight, and does not stop a NaN or infinity
 * in a v row from reaching earlier queries of the same tile (0 * inf).
 * lse may be NULL (no backward pass).
 */
KT_API kt_status kt_attention_fwd(const kt_attention *a, const kt_heads *q,
                                  const kt_heads *k, const kt_heads *v,
                                  const kt_heads *o, float *lse, void *stream);

/*
 * The gradients of q, k and v from that of o.  The probabilities are computed
 * again from q, k and lse: p = exp(scale * q k^T - lse); with
 * delta = rowsum(d_o * o) and ds = p * (d_o v^T - delta),
 *   dq = scale * ds k,  dk = scale * ds^T q,  dv = p^T d_o,
 * dk and dv summed over the query heads that share a key head.  Every element
 * of dq, dk and dv is written: 0 where a query sees no key, and for keys past
 * k_lens, whatever d_o, q and o hold.  As in the forward pass the causal mask
 * gives weight 0: a NaN or infinity in a query's row of q or d_o can reach dk or dv,
 * and one in a key's row dq, of what it is hidden from in the same tile.
 *   ws  kt_attention_bwd_workspace(a) bytes.
 */
KT_API int64_t kt_attention_bwd_workspace(const kt_attention *a);
KT_API kt_status kt_attention_bwd(const kt_attention *a, const kt_heads *d_o,
                                  const kt_heads *q, const kt_heads *k,
                                  const kt_heads *v, const kt_heads *o,
                                  const float *lse, const kt_heads *dq,
                                  const kt_heads *dk, const kt_heads *dv,
                                  void *ws, int64_t ws_bytes, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* KT_OPS_H */
