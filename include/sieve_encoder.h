/*
 * sieve_encoder.h -- C ABI of libsieve's encoder operators: what turns packed
 * documents into the unit rows that sieve_search takes, and the backward
 * passes that train it.
 *
 * The search of sieve.h starts from one unit-norm fp32 row per document.
 * These calls are the parts of a text encoder that are not plain matrix
 * products: layer norm, attention with a learned relative position bias, and
 * the pooling of a document's tokens into its unit row.  The paper takes the
 * rows as given, so it has no counterpart.
 *
 * Conventions are sieve.h's: device pointers of the current device, every
 * buffer the caller's, scratch from the caller's workspace (256-byte
 * aligned, sized by the *_workspace_size call), nothing allocated, nothing
 * printed, no abort; calls are asynchronous on `stream` and return
 * SIEVE_EINVAL before any device work for an argument they refuse, a pointer
 * that is not aligned to its elements among them.  The same
 * call on the same inputs gives the same bits: no sum depends on the order in
 * which blocks run.
 *
 * Packed documents.  The tokens of nseq documents (sequences) lie one after
 * the other, without padding, in arrays of `tokens` rows.  `offsets` (device
 * [nseq + 1] int32, nondecreasing, within [0, tokens]) holds where each
 * document starts and where the last ends; a document may have no token.
 * Rows outside [offsets[0], offsets[nseq]) belong to no document: they are
 * not read and their outputs are not written.  Offsets that break these
 * rules give undefined results; they are clamped into [0, tokens], so that
 * no access leaves the arrays.
 */
#ifndef SIEVE_ENCODER_H
#define SIEVE_ENCODER_H

#include "sieve.h"

#ifdef __cplusplus
extern "C" {
#endif

/* element types */
#define SIEVE_F32 0
#define SIEVE_F16 1
#define SIEVE_BF16 2

#define SIEVE_NORM_MAX_WIDTH 16384
#define SIEVE_ATTENTION_MAX_DIM 128
#define SIEVE_ATTENTION_MAX_BUCKETS 64
#define SIEVE_ATTENTION_MAX_REACH 256

/* Layer norm of every row of x:
 *   mu = mean(x), r = 1 / sqrt(mean((x - mu)^2) + eps), y = (x - mu) r w + b
 * with sums in fp32 over values held in registers (the variance is a second
 * pass over them, so a large mean costs no accuracy) and one rounding to the
 * output's type.
 *   x, y    device [rows][width] of `dtype`, rows `*_stride` elements apart
 *           (>= width), elements contiguous; y may be x
 *   weight  device [width] of `weight_dtype` (dtype, or SIEVE_F32)
 *   bias    the same, nullable
 *   mean, rstd  device [rows] fp32 out (nullable, both or none): what the
 *           backward pass needs
 * width 1..SIEVE_NORM_MAX_WIDTH, eps >= 0 and finite; rows = 0 does nothing. */
sieve_status sieve_layer_norm(const void *x, int64_t x_stride, const void *weight,
                              const void *bias, int64_t rows, int32_t width, int32_t dtype,
                              int32_t weight_dtype, float eps, void *y, int64_t y_stride,
                              float *mean, float *rstd, void *stream);

/* Its backward pass, from dy, the forward's input and its statistics: with
 * xh = (x - mu) r and g = dy w,
 *   dx = r (g - mean(g) - xh mean(g xh)),
 *   dweight = sum over rows of dy xh,  dbias = sum over rows of dy.
 *   dx       device [rows][width] of `dtype`, rows dx_stride elements apart;
 *            may be dy
 *   dweight  device [width] of weight_dtype out;  dbias the same, nullable
 * The sums over rows are fp32, in an order that depends on the sizes alone.
 * rows = 0 writes zeros to dweight and dbias. */
sieve_status sieve_layer_norm_backward_workspace_size(int64_t rows, int32_t width, size_t *bytes);
sieve_status sieve_layer_norm_backward(const void *dy, int64_t dy_stride, const void *x,
                                       int64_t x_stride, const void *weight, const float *mean,
                                       const float *rstd, int64_t rows, int32_t width,
                                       int32_t dtype, int32_t weight_dtype, void *dx,
                                       int64_t dx_stride, void *dweight, void *dbias, void *ws,
                                       size_t ws_bytes, void *stream);

/* Attention over packed documents.
 *   q        device [q_tokens][heads][head_dim] of `dtype` (SIEVE_F16 or
 *            SIEVE_BF16); k, v device [k_tokens][kv_heads][head_dim].  Tokens
 *            and heads lie `*_token_stride` and `*_head_stride` elements
 *            apart (multiples of 8, at least head_dim where the axis has more
 *            than one; base pointers 16-byte aligned), elements
 *            of a head contiguous, so they may be parts of one projection.
 *   heads    a multiple of kv_heads: query head h reads key head
 *            h / (heads / kv_heads)
 *   head_dim a multiple of 8, up to SIEVE_ATTENTION_MAX_DIM
 *   k_offsets  the documents of k and v.  The queries of document s are rows
 *            new_tokens * s .. new_tokens * (s + 1) - 1 of q where new_tokens
 *            > 0 (so q_tokens = nseq * new_tokens: the next tokens of
 *            growing documents), else rows q_offsets[s] .. q_offsets[s + 1] - 1
 *            (NULL: k_offsets, each document against itself)
 *   position the last query of a document stands at its last key: query i of
 *            Lq at place i + Lk - Lq.  causal = 1: a query sees the keys at
 *            its place and before; 0: all keys of its document
 *   table    device [num_buckets][heads] fp32 (nullable): the learned bias
 *   bucket_map  device [2 reach + 1] int32: the bucket of a key `distance`
 *            = key place - query place away, at index reach + distance, with
 *            the distance clamped to [-reach, reach]; entries outside
 *            [0, num_buckets) are clamped
 * The score of a query and a key it sees is s = scale q.k + table[bucket][h];
 * a score of -inf (a bias of -inf) hides the key.  Finite biases beyond
 * +-2.35e38 count as the type's largest or lowest.  Scores are fp32: beside a
 * bias of 1e9 the product vanishes, and keys of equal bias share their weight
 * evenly.
 *   out      device [q_tokens][heads][head_dim] of dtype, contiguous:
 *            sum of softmax(s) v
 *   lse      device [heads][q_tokens] fp32: log of the sum of exp(s)
 * A query that sees no key has out = 0 and lse = -inf.  Documents do not
 * affect each other, whatever their values; within one document a value that
 * is not finite may reach queries that do not see its token. */
typedef struct {
    int32_t dtype, heads, kv_heads, head_dim;
    int64_t nseq, q_tokens, k_tokens;
    int32_t new_tokens, causal;
    float scale;
    int32_t num_buckets, reach, reserved0;
    const int32_t *q_offsets, *k_offsets;
    const void *q, *k, *v;
    int64_t q_token_stride, q_head_stride, k_token_stride, k_head_stride, v_token_stride,
        v_head_stride;
    const float *table;
    const int32_t *bucket_map;
} sieve_attention_args;

sieve_status sieve_attention_workspace_size(const sieve_attention_args *a, size_t *bytes);
sieve_status sieve_attention(const sieve_attention_args *a, void *out, float *lse, void *ws,
                             size_t ws_bytes, void *stream);

/* Its backward pass: with p = exp(s - lse) recomputed from q and k,
 * dp = dout v^T, delta = sum over a query's keys of p dp, ds = p (dp - delta),
 *   dq = scale ds k,  dk = scale ds^T q,  dv = p^T dout  (dk and dv summed
 * over the heads that share a key head),
 *   dtable[b][h] = sum of ds over the pairs of bucket b.
 *   dout     device [q_tokens][heads][head_dim] of dtype, contiguous
 *   out, lse what sieve_attention wrote for the same arguments
 *   dq, dk, dv  device out, of dtype; tokens and heads `grad_strides` apart
 *            (token and head stride of dq, dk, dv in turn, with the same rules;
 *            bases 16-byte aligned)
 *   dtable   device [num_buckets][heads] fp32 out; required with a table
 * Every row of every document is written, with zeros where nothing reaches it. */
sieve_status sieve_attention_backward_workspace_size(const sieve_attention_args *a, size_t *bytes);
sieve_status sieve_attention_backward(const sieve_attention_args *a, const void *dout,
                                      const void *out, const float *lse, void *dq, void *dk,
                                      void *dv, const int64_t grad_strides[6], float *dtable,
                                      void *ws, size_t ws_bytes, void *stream);

/* The status word that the last sieve_attention or sieve_attention_backward
 * enqueued with workspace ws left there: 0, or SIEVE_ETIMEOUT where a bounded
 * wait inside a kernel gave up (its outputs are then undefined).  Copies the
 * word to *status (host) on `stream` and synchronizes `stream`. */
sieve_status sieve_encoder_status(const void *ws, size_t ws_bytes, int32_t *status, void *stream);

/* One unit row per document: m = the mean of its tokens' rows,
 * row = m / |m| (zeros where |m| is 0 or the document has no token).
 *   h      device [tokens][width] of dtype, tokens h_stride elements apart
 *   rows   device [nseq][width] fp32 out, contiguous: what sieve_search takes
 *   norms  device [nseq] fp32 out: |m|
 * width 1..SIEVE_NORM_MAX_WIDTH. */
sieve_status sieve_unit_pool_workspace_size(int64_t tokens, int64_t nseq, int32_t width,
                                            size_t *bytes);
sieve_status sieve_unit_pool(const void *h, int64_t h_stride, const int32_t *offsets,
                             int64_t tokens, int64_t nseq, int32_t width, int32_t dtype,
                             float *rows, float *norms, void *ws, size_t ws_bytes, void *stream);

/* Its backward pass: every token t of a document of L tokens gets
 *   dh_t = (g - (g.row) row) / (|m| L),  g the gradient of its row
 * (0 where |m| is 0).
 *   drows, rows  device [nseq][width] fp32, contiguous;  norms device [nseq]
 *   dh     device [tokens][width] of dtype out, tokens dh_stride apart */
sieve_status sieve_unit_pool_backward(const float *drows, const float *rows, const float *norms,
                                      const int32_t *offsets, int64_t tokens, int64_t nseq,
                                      int32_t width, int32_t dtype, void *dh, int64_t dh_stride,
                                      void *stream);

#ifdef __cplusplus
}
#endif

#endif /* SIEVE_ENCODER_H */
