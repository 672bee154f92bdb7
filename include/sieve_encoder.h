/*
 * sieve_encoder.h -- C ABI of libsieve's encoder operators: what turns packed
 * documents into the unit rows that sieve_search takes, and the backward
 * passes that train it.
 *
 * The search of sieve.h starts from one unit-norm fp32 row per document.
 * These calls are the parts of a text encoder that are not plain matrix
 * products: token embedding, layer norm, attention with a learned relative
 * position bias, the residual step between two blocks, the pooling of a
 * document's tokens into its unit row, and the cross entropy that an encoder
 * is trained with.  The paper takes the rows as given, so it has no
 * counterpart.
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
/* types of token ids and targets */
#define SIEVE_I32 3
#define SIEVE_I64 4

#define SIEVE_NORM_MAX_WIDTH 16384
#define SIEVE_ATTENTION_MAX_DIM 128
#define SIEVE_ATTENTION_MAX_BUCKETS 64
#define SIEVE_ATTENTION_MAX_REACH 256
#define SIEVE_EMBED_MAX_WIDTH 16384
#define SIEVE_EMBED_MAX_TOKENS (1 << 30)
#define SIEVE_EMBED_MAX_VOCAB (1 << 26)
#define SIEVE_RESIDUAL_NORM_MAX_WIDTH 8192
#define SIEVE_CROSS_ENTROPY_MAX_WIDTH 16384
#define SIEVE_CROSS_ENTROPY_MAX_ROWS (1 << 24)
#define SIEVE_CROSS_ENTROPY_MAX_CLASSES (1 << 24)

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

/* The status word that the last sieve_attention, sieve_cross_entropy or
 * backward pass of theirs enqueued with workspace ws left there: 0, or SIEVE_ETIMEOUT where a bounded
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

/* Token embedding: out[t] = scale table[ids[t]], rounded once.  An id outside
 * [0, vocab) has no row: zeros, and no gradient.
 *   ids    device [tokens], contiguous, of `id_type` (SIEVE_I32 or SIEVE_I64)
 *   table  device [vocab][width] of `table_dtype`, rows table_stride apart
 *          (>= width)
 *   out    device [tokens][width] of `dtype`, rows out_stride apart
 * Any of the three types for table and out.  width 1..SIEVE_EMBED_MAX_WIDTH,
 * tokens up to SIEVE_EMBED_MAX_TOKENS, vocab 1..SIEVE_EMBED_MAX_VOCAB; scale
 * finite.  tokens = 0 does nothing. */
sieve_status sieve_embed(const void *ids, int32_t id_type, int64_t tokens, const void *table,
                         int64_t table_stride, int64_t vocab, int32_t width, int32_t table_dtype,
                         float scale, void *out, int64_t out_stride, int32_t dtype, void *stream);

/* The gradient of its table: dtable[v] = scale * sum of dout[t] over the
 * tokens t with ids[t] = v, in fp32 and in an order that depends on the ids
 * alone (the tokens are sorted by id first, equal ids in the tokens' order).
 *   dout     device [tokens][width] of `dtype`, rows dout_stride apart
 *   dtable   device [vocab][width] of `table_dtype`, rows dtable_stride apart.
 *            accumulate = 0: every row is written, with zeros where no token
 *            has its id; 1: the sums are added to what is there and rows
 *            without a token stay as they are (a tied table's second gradient)
 */
sieve_status sieve_embed_backward_workspace_size(int64_t tokens, int64_t vocab, int32_t width,
                                                 size_t *bytes);
sieve_status sieve_embed_backward(const void *dout, int64_t dout_stride, const void *ids,
                                  int32_t id_type, int64_t tokens, int64_t vocab, int32_t width,
                                  int32_t dtype, float scale, void *dtable, int64_t dtable_stride,
                                  int32_t table_dtype, int32_t accumulate, void *ws,
                                  size_t ws_bytes, void *stream);

/* The residual step between two blocks of an encoder: the block's output y is
 * normed (post), gated and added to the scaled stream h, and the sum is normed
 * (pre) for the next block, in one pass:
 *   u = N(y; post_weight, post_bias), or y without post_weight
 *   stream = alpha h + gate u
 *   x = N(stream; weight, bias), from the sum before it is rounded
 * where N(v; w, b) = (v - mu) r w + b, mu = mean(v) and r = 1 / sqrt(mean((v -
 * mu)^2) + eps), or with rms = 1 mu = 0.
 *   h, y, stream, x  device [rows][width] of `dtype`, rows `*_stride` apart
 *            (>= width); stream may be h, x may be y
 *   weight, bias, post_weight, post_bias  device [width] of `weight_dtype`
 *            (dtype, or SIEVE_F32), nullable; a bias goes with its weight, and
 *            one of the weights is there.  Without weight there is no x.
 *   gate     gate_kind SIEVE_GATE_NONE: 1; _COLUMN: device [width] of
 *            weight_dtype; _ROW: device [rows][width] of dtype, gate_stride apart
 *   stats    device [4][rows] fp32: mu and r of the post norm, mu and r of the
 *            pre norm (0 and 1 where there is none): what the backward pass needs;
 *            nullable where there is none
 * width 1..SIEVE_RESIDUAL_NORM_MAX_WIDTH, eps >= 0 and finite, alpha finite. */
#define SIEVE_GATE_NONE 0
#define SIEVE_GATE_COLUMN 1
#define SIEVE_GATE_ROW 2
typedef struct {
    int64_t rows;
    int32_t width, dtype, weight_dtype, rms, gate_kind;
    float alpha, eps;
    int32_t reserved0;
    const void *h, *y, *gate;
    int64_t h_stride, y_stride, gate_stride;
    const void *weight, *bias, *post_weight, *post_bias;
} sieve_residual_norm_args;

sieve_status sieve_residual_norm(const sieve_residual_norm_args *a, void *stream_out,
                                 int64_t stream_stride, void *x, int64_t x_stride, float *stats,
                                 void *stream);

/* Its backward pass, from the gradients of both results (the sum is made again
 * from h and y, so it is not rounded here either):
 *   G = dstream + dN(dx; stream),  dh = alpha G,  dy = dN(gate G; y) or gate G,
 *   dgate = G u (summed over rows for a column gate),  and the weights'
 *   gradients summed over rows
 * with dN(d; v) = r (d w - mean(d w) - vh mean(d w vh)), vh = (v - mu) r, the
 * mean of d w left out with rms = 1.
 *   dstream  device [rows][width] of dtype, nullable where there is a weight
 *   dx       the same, required where there is a weight, else NULL
 *   dh, dy   device out, of dtype; dh may be dstream, dy may be dx
 *   dweight, dbias, dpost_weight, dpost_bias  device [width] of weight_dtype
 *            out, where the weight of that name is there
 *   dgate    like gate, out
 * The sums over rows are fp32, in an order that depends on the sizes alone;
 * rows = 0 writes zeros to them. */
typedef struct {
    const void *dstream, *dx;
    int64_t dstream_stride, dx_stride;
    const float *stats;
    void *dh, *dy, *dgate;
    int64_t dh_stride, dy_stride, dgate_stride;
    void *dweight, *dbias, *dpost_weight, *dpost_bias;
} sieve_residual_norm_grads;

sieve_status sieve_residual_norm_backward_workspace_size(int64_t rows, int32_t width, size_t *bytes);
sieve_status sieve_residual_norm_backward(const sieve_residual_norm_args *a,
                                          const sieve_residual_norm_grads *g, void *ws,
                                          size_t ws_bytes, void *stream);

/* Softmax cross entropy of rows against a table of classes, without keeping
 * the scores:
 *   z[r][v] = scale h[r].weight[v] + bias[v]
 *   lse[r] = log of the sum over v of exp(z[r][v]),
 *   loss[r] = lse[r] - z[r][targets[r]]
 * (as log1p of the other classes' sum against the target's, so that a small
 * loss keeps its digits).  A target outside [0, classes) means none: the row's
 * loss and lse are 0 and it gets and gives no gradient, whatever h holds there.
 * The rows with a target are found on the device and only they cost time.
 *   h        device [rows][width] of `dtype` (SIEVE_F16 or SIEVE_BF16), rows
 *            h_stride apart
 *   weight   device [classes][width] of dtype, rows weight_stride apart.
 *            width and strides are multiples of 8, bases 16-byte aligned.
 *   bias     device [classes] fp32, nullable; -inf hides a class
 *   targets  device [rows], contiguous, of `target_type`
 *   wait_limit  0, or the iteration limit of one device wait, the one for a tile's
 *            products: when it runs out the call's status word
 *            (sieve_encoder_status) is SIEVE_ETIMEOUT and its results are
 *            undefined.  Every wait gives up after two seconds.
 * A hidden target's loss is +inf.  Where every class is hidden lse is -inf.
 * width 8..SIEVE_CROSS_ENTROPY_MAX_WIDTH, up to SIEVE_CROSS_ENTROPY_MAX_ROWS
 * rows and 1..SIEVE_CROSS_ENTROPY_MAX_CLASSES classes, scale finite. */
typedef struct {
    int64_t rows, classes;
    int32_t width, dtype, target_type;
    float scale;
    const void *h, *weight;
    int64_t h_stride, weight_stride;
    const float *bias;
    const void *targets;
    int32_t wait_limit, reserved0;
} sieve_cross_entropy_args;

sieve_status sieve_cross_entropy_workspace_size(const sieve_cross_entropy_args *a, size_t *bytes);
sieve_status sieve_cross_entropy(const sieve_cross_entropy_args *a, float *loss, float *lse,
                                 void *ws, size_t ws_bytes, void *stream);

/* Its backward pass, for the gradient dloss of every row's loss: with
 * q = exp(z - lse) - [v = target] (exactly expm1(-loss) at the target; where
 * every class is hidden that is -1, and q is 0 elsewhere),
 *   dh[r] = dloss[r] scale sum over v of q weight[v],
 *   dweight[v] = scale sum over r of dloss[r] q h[r],
 *   dbias[v] = sum over r of dloss[r] q.
 * The scores are made anew in pieces of the classes; q (times the mantissa of
 * dloss, where the rows' dloss differ) is rounded once to dtype on its way into
 * both products.  The rest of dloss, a power of two, goes into a copy of h for
 * dweight: exact in bf16; in fp16 exact down to 2^-29 of the largest product
 * 2^e |h| of a call, and off by 2^-40 of that at most below.
 *   dloss    device [rows] fp32;  loss, lse what sieve_cross_entropy wrote
 *   dh       device [rows][width] of dtype out, rows dh_stride apart; nullable
 *   dweight  device [classes][width] of `dweight_dtype` (dtype or SIEVE_F32)
 *            out, rows dweight_stride apart; nullable.  accumulate = 1
 *            (SIEVE_F32 alone) adds to what is there.
 *   dbias    device [classes] fp32 out, nullable; without a bias there is none
 * Strides are multiples of 8, bases of dh and dweight 16-byte aligned.
 * Every call with the same arguments gives the same bits; dh's last ones may
 * depend on whether dweight is asked for (its sum is cut into other parts).
 * |dloss scale| stays below 2^127: its powers of two go into fp32 factors. */
typedef struct {
    const float *dloss, *loss, *lse;
    void *dh, *dweight;
    int64_t dh_stride, dweight_stride;
    int32_t dweight_dtype, accumulate;
    float *dbias;
} sieve_cross_entropy_grads;

sieve_status sieve_cross_entropy_backward_workspace_size(const sieve_cross_entropy_args *a,
                                                         size_t *bytes);
sieve_status sieve_cross_entropy_backward(const sieve_cross_entropy_args *a,
                                          const sieve_cross_entropy_grads *g, void *ws,
                                          size_t ws_bytes, void *stream);

#ifdef __cplusplus
}
#endif

#endif /* SIEVE_ENCODER_H */
