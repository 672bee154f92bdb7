// encoder_api.cu -- the C ABI of the encoder operators (declared in
// include/sieve_encoder.h): argument checks and workspace layout.
#include <cmath>

#include "encoder.cuh"

using namespace sieve;
using namespace sieve::enc;

namespace {

#define ENC_CUDA(call)                                          \
    do {                                                        \
        cudaError_t e_ = (call);                                \
        if (e_ != cudaSuccess) return record_cuda_error(e_);    \
    } while (0)

bool aligned_to(const void *p, size_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }
// fp32 and int32 arrays that are read or written element by element
template <typename... P>
bool aligned4(const P *...p) { return (aligned_to(p, 4) && ...); }

size_t type_bytes(int dtype) { return dtype == SIEVE_F32 ? 4 : 2; }
bool is_type(int dtype) { return dtype == SIEVE_F32 || dtype == SIEVE_F16 || dtype == SIEVE_BF16; }

sieve_status check_norm(int64_t rows, int32_t width, int32_t dtype, int32_t wtype) {
    if (rows < 0 || rows > INT32_MAX || width < 1 || width > SIEVE_NORM_MAX_WIDTH) return SIEVE_EINVAL;
    if (!is_type(dtype) || (wtype != dtype && wtype != SIEVE_F32)) return SIEVE_EINVAL;
    return SIEVE_OK;
}
// a row-strided matrix that a kernel reads or writes
bool bad_rows(const void *p, int64_t stride, int64_t rows, int32_t width, int32_t dtype) {
    return rows > 0 && (!p || stride < width || !aligned_to(p, type_bytes(dtype)));
}

sieve_status check_workspace(const void *ws, size_t have, size_t need) {
    if (have < need || (need && (!ws || !aligned_to(ws, 256)))) return SIEVE_EWORKSPACE;
    return SIEVE_OK;
}

// Whether the heads of an axis of `n` would overlap.  (A tensor map wants every
// stride to clear the axes below it.)
bool overlapping(int64_t n, int64_t stride, int32_t head_dim) { return n > 1 && stride < head_dim; }

sieve_status check_attention(const sieve_attention_args *a, bool pointers) {
    if (!a) return SIEVE_EINVAL;
    if (a->dtype != SIEVE_F16 && a->dtype != SIEVE_BF16) return SIEVE_EINVAL;
    if (a->heads < 1 || a->kv_heads < 1 || a->heads % a->kv_heads || a->heads > 65535) return SIEVE_EINVAL;
    if (a->head_dim < 8 || a->head_dim % 8 || a->head_dim > SIEVE_ATTENTION_MAX_DIM) return SIEVE_EINVAL;
    if (a->nseq < 0 || a->nseq > (1 << 26)) return SIEVE_EINVAL;
    if (a->q_tokens < 0 || a->k_tokens < 0 || a->q_tokens > INT32_MAX / 2 || a->k_tokens > INT32_MAX / 2)
        return SIEVE_EINVAL;
    if (a->nseq == 0 && (a->q_tokens || a->k_tokens)) return SIEVE_EINVAL;
    // one block takes one head of one tile
    if ((a->q_tokens / 8 + a->nseq) * a->heads > INT32_MAX || (a->k_tokens / 8 + a->nseq) * a->heads > INT32_MAX)
        return SIEVE_EINVAL;
    if (a->new_tokens < 0 || (a->causal != 0 && a->causal != 1)) return SIEVE_EINVAL;
    if (a->new_tokens > 0 && (a->q_offsets || (int64_t)a->new_tokens * a->nseq != a->q_tokens)) return SIEVE_EINVAL;
    if (a->new_tokens == 0 && !a->q_offsets && a->q_tokens != a->k_tokens) return SIEVE_EINVAL;
    if (!std::isfinite(a->scale)) return SIEVE_EINVAL;
    const bool biased = a->num_buckets != 0;
    if (biased && (a->num_buckets < 1 || a->num_buckets > SIEVE_ATTENTION_MAX_BUCKETS || a->reach < 0 ||
                   a->reach > SIEVE_ATTENTION_MAX_REACH))
        return SIEVE_EINVAL;
    if (!pointers) return SIEVE_OK;
    if (biased ? (!a->table || !a->bucket_map) : (a->table || a->bucket_map)) return SIEVE_EINVAL;
    if (a->nseq > 0 && !a->k_offsets) return SIEVE_EINVAL;
    if (!aligned4(a->q_offsets, a->k_offsets, a->table, a->bucket_map)) return SIEVE_EINVAL;
    const int64_t strides[6] = {a->q_token_stride, a->q_head_stride, a->k_token_stride,
                                a->k_head_stride,  a->v_token_stride, a->v_head_stride};
    for (int64_t s : strides)
        if (s < 0 || s % 8 || s >= (int64_t)1 << 38) return SIEVE_EINVAL;
    const int64_t counts[6] = {a->q_tokens, a->heads, a->k_tokens, a->kv_heads, a->k_tokens, a->kv_heads};
    for (int i = 0; i < 6; ++i)
        if (overlapping(counts[i], strides[i], a->head_dim)) return SIEVE_EINVAL;
    if (a->q_tokens > 0 && (!a->q || !aligned_to(a->q, 16))) return SIEVE_EINVAL;
    if (a->k_tokens > 0 && (!a->k || !a->v || !aligned_to(a->k, 16) || !aligned_to(a->v, 16))) return SIEVE_EINVAL;
    return SIEVE_OK;
}

// The arguments as the kernels take them, for sizes and launches alike: the
// queries' documents filled in, no reach (which nothing has checked) without a
// table.
sieve_attention_args resolved(const sieve_attention_args *a) {
    sieve_attention_args r = *a;
    if (!r.num_buckets) r.reach = 0;
    if (r.new_tokens == 0 && !r.q_offsets) r.q_offsets = r.k_offsets;
    return r;
}

// The status word of a call that launches no kernel to write it.
sieve_status nothing_to_do(void *ws, cudaStream_t st) {
    ENC_CUDA(cudaMemsetAsync(ws, 0, sizeof(EncCtl), st));
    return SIEVE_OK;
}

}  // namespace

extern "C" {

sieve_status sieve_layer_norm(const void *x, int64_t x_stride, const void *weight, const void *bias,
                              int64_t rows, int32_t width, int32_t dtype, int32_t weight_dtype, float eps,
                              void *y, int64_t y_stride, float *mean, float *rstd, void *stream) {
    sieve_status rc = check_norm(rows, width, dtype, weight_dtype);
    if (rc != SIEVE_OK) return rc;
    if (!(eps >= 0.f) || !std::isfinite(eps)) return SIEVE_EINVAL;
    if (bad_rows(x, x_stride, rows, width, dtype) || bad_rows(y, y_stride, rows, width, dtype)) return SIEVE_EINVAL;
    if (!weight || !aligned_to(weight, type_bytes(weight_dtype)) || !aligned_to(bias, type_bytes(weight_dtype)))
        return SIEVE_EINVAL;
    if (!mean != !rstd || !aligned4(mean, rstd)) return SIEVE_EINVAL;
    if ((rc = check_current_device()) != SIEVE_OK) return rc;
    if (rows == 0) return SIEVE_OK;
    NormArgs a = {};
    a.x = x;
    a.x_stride = x_stride;
    a.weight = weight;
    a.bias = bias;
    a.rows = rows;
    a.width = width;
    a.dtype = dtype;
    a.weight_dtype = weight_dtype;
    a.eps = eps;
    a.y = y;
    a.y_stride = y_stride;
    a.mean = mean;
    a.rstd = rstd;
    ENC_CUDA(launch_norm_forward(a, static_cast<cudaStream_t>(stream)));
    return SIEVE_OK;
}

sieve_status sieve_layer_norm_backward_workspace_size(int64_t rows, int32_t width, size_t *bytes) {
    if (!bytes) return SIEVE_EINVAL;
    sieve_status rc = check_norm(rows, width, SIEVE_F32, SIEVE_F32);
    if (rc != SIEVE_OK) return rc;
    *bytes = norm_backward_workspace_bytes(rows, width);
    return SIEVE_OK;
}

sieve_status sieve_layer_norm_backward(const void *dy, int64_t dy_stride, const void *x, int64_t x_stride,
                                       const void *weight, const float *mean, const float *rstd, int64_t rows,
                                       int32_t width, int32_t dtype, int32_t weight_dtype, void *dx,
                                       int64_t dx_stride, void *dweight, void *dbias, void *ws,
                                       size_t ws_bytes, void *stream) {
    sieve_status rc = check_norm(rows, width, dtype, weight_dtype);
    if (rc != SIEVE_OK) return rc;
    if (bad_rows(dy, dy_stride, rows, width, dtype) || bad_rows(x, x_stride, rows, width, dtype) ||
        bad_rows(dx, dx_stride, rows, width, dtype))
        return SIEVE_EINVAL;
    const size_t ws_type = type_bytes(weight_dtype);
    if (!weight || !dweight || !aligned_to(weight, ws_type) || !aligned_to(dweight, ws_type) ||
        !aligned_to(dbias, ws_type))
        return SIEVE_EINVAL;
    if ((rows > 0 && (!mean || !rstd)) || !aligned4(mean, rstd)) return SIEVE_EINVAL;
    if ((rc = check_workspace(ws, ws_bytes, norm_backward_workspace_bytes(rows, width))) != SIEVE_OK) return rc;
    if ((rc = check_current_device()) != SIEVE_OK) return rc;
    NormArgs a = {};
    a.dy = dy;
    a.dy_stride = dy_stride;
    a.x = x;
    a.x_stride = x_stride;
    a.weight = weight;
    a.mean_in = mean;
    a.rstd_in = rstd;
    a.rows = rows;
    a.width = width;
    a.dtype = dtype;
    a.weight_dtype = weight_dtype;
    a.dx = dx;
    a.dx_stride = dx_stride;
    a.dweight = dweight;
    a.dbias = dbias;
    a.partial = static_cast<float *>(ws);
    ENC_CUDA(launch_norm_backward(a, static_cast<cudaStream_t>(stream)));
    return SIEVE_OK;
}

sieve_status sieve_attention_workspace_size(const sieve_attention_args *a, size_t *bytes) {
    if (!bytes) return SIEVE_EINVAL;
    sieve_status rc = check_attention(a, false);
    if (rc != SIEVE_OK) return rc;
    *bytes = attention_workspace_bytes(resolved(a));
    return SIEVE_OK;
}

sieve_status sieve_attention(const sieve_attention_args *a, void *out, float *lse, void *ws, size_t ws_bytes,
                             void *stream) {
    sieve_status rc = check_attention(a, true);
    if (rc != SIEVE_OK) return rc;
    if (a->q_tokens > 0 && (!out || !lse || !aligned_to(out, 16) || !aligned4(lse))) return SIEVE_EINVAL;
    if ((rc = check_workspace(ws, ws_bytes, attention_workspace_bytes(resolved(a)))) != SIEVE_OK) return rc;
    if ((rc = check_current_device()) != SIEVE_OK) return rc;
    if (a->q_tokens == 0) return nothing_to_do(ws, static_cast<cudaStream_t>(stream));
    AttentionArgs p = {};
    p.a = resolved(a);
    p.out = out;
    p.lse = lse;
    return launch_attention_forward(p, ws, static_cast<cudaStream_t>(stream));
}

sieve_status sieve_attention_backward_workspace_size(const sieve_attention_args *a, size_t *bytes) {
    if (!bytes) return SIEVE_EINVAL;
    sieve_status rc = check_attention(a, false);
    if (rc != SIEVE_OK) return rc;
    *bytes = attention_backward_workspace_bytes(resolved(a));
    return SIEVE_OK;
}

sieve_status sieve_attention_backward(const sieve_attention_args *a, const void *dout, const void *out,
                                      const float *lse, void *dq, void *dk, void *dv,
                                      const int64_t grad_strides[6], float *dtable, void *ws, size_t ws_bytes,
                                      void *stream) {
    sieve_status rc = check_attention(a, true);
    if (rc != SIEVE_OK) return rc;
    if (!grad_strides) return SIEVE_EINVAL;
    const int64_t counts[6] = {a->q_tokens, a->heads, a->k_tokens, a->kv_heads, a->k_tokens, a->kv_heads};
    for (int i = 0; i < 6; ++i)
        if (grad_strides[i] < 0 || grad_strides[i] % 8 || overlapping(counts[i], grad_strides[i], a->head_dim))
            return SIEVE_EINVAL;
    if (a->q_tokens > 0 && (!dout || !out || !lse || !dq || !aligned_to(dout, 16) || !aligned_to(out, 16) ||
                            !aligned_to(dq, 16) || !aligned4(lse)))
        return SIEVE_EINVAL;
    if (a->k_tokens > 0 && (!dk || !dv || !aligned_to(dk, 16) || !aligned_to(dv, 16))) return SIEVE_EINVAL;
    if ((a->table && !dtable) || !aligned4(dtable)) return SIEVE_EINVAL;
    if ((rc = check_workspace(ws, ws_bytes, attention_backward_workspace_bytes(resolved(a)))) != SIEVE_OK) return rc;
    if ((rc = check_current_device()) != SIEVE_OK) return rc;
    if (a->q_tokens == 0 && a->k_tokens == 0)
        if ((rc = nothing_to_do(ws, static_cast<cudaStream_t>(stream))) != SIEVE_OK) return rc;
    AttentionArgs p = {};
    p.a = resolved(a);
    p.dout = dout;
    p.out_in = out;
    p.lse_in = lse;
    p.dq = dq;
    p.dk = dk;
    p.dv = dv;
    p.dq_ts = grad_strides[0];
    p.dq_hs = grad_strides[1];
    p.dk_ts = grad_strides[2];
    p.dk_hs = grad_strides[3];
    p.dv_ts = grad_strides[4];
    p.dv_hs = grad_strides[5];
    p.dtable = dtable;
    return launch_attention_backward(p, ws, static_cast<cudaStream_t>(stream));
}

sieve_status sieve_encoder_status(const void *ws, size_t ws_bytes, int32_t *status, void *stream) {
    if (!ws || !status || !aligned_to(ws, 256) || ws_bytes < kCtlBytes) return SIEVE_EINVAL;
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    ENC_CUDA(cudaMemcpyAsync(status, &static_cast<const EncCtl *>(ws)->status, sizeof(int32_t),
                             cudaMemcpyDeviceToHost, st));
    ENC_CUDA(cudaStreamSynchronize(st));
    return SIEVE_OK;
}

sieve_status sieve_unit_pool_workspace_size(int64_t tokens, int64_t nseq, int32_t width, size_t *bytes) {
    if (!bytes || tokens < 0 || tokens > INT32_MAX / 2 || nseq < 0 || nseq > (1 << 26) || width < 1 ||
        width > SIEVE_NORM_MAX_WIDTH)
        return SIEVE_EINVAL;
    *bytes = (size_t)round_up(doc_tiles(tokens, nseq, kPoolTile) * width * (int64_t)sizeof(float), 256);
    return SIEVE_OK;
}

static sieve_status check_pool(const int32_t *offsets, int64_t tokens, int64_t nseq, int32_t width, int32_t dtype,
                               const void *tok, int64_t stride, const float *r, const float *n) {
    size_t need;
    sieve_status rc = sieve_unit_pool_workspace_size(tokens, nseq, width, &need);
    if (rc != SIEVE_OK) return rc;
    if (!is_type(dtype) || (nseq == 0 && tokens > 0)) return SIEVE_EINVAL;
    if ((nseq > 0 && (!offsets || !r || !n)) || !aligned4(offsets, r, n)) return SIEVE_EINVAL;
    return bad_rows(tok, stride, tokens, width, dtype) ? SIEVE_EINVAL : SIEVE_OK;
}

sieve_status sieve_unit_pool(const void *h, int64_t h_stride, const int32_t *offsets, int64_t tokens,
                             int64_t nseq, int32_t width, int32_t dtype, float *rows, float *norms, void *ws,
                             size_t ws_bytes, void *stream) {
    sieve_status rc = check_pool(offsets, tokens, nseq, width, dtype, h, h_stride, rows, norms);
    if (rc != SIEVE_OK) return rc;
    size_t need;
    sieve_unit_pool_workspace_size(tokens, nseq, width, &need);
    if ((rc = check_workspace(ws, ws_bytes, need)) != SIEVE_OK) return rc;
    if ((rc = check_current_device()) != SIEVE_OK) return rc;
    if (nseq == 0) return SIEVE_OK;
    PoolArgs a = {};
    a.h = h;
    a.stride = h_stride;
    a.offsets = offsets;
    a.tokens = (int)tokens;
    a.nseq = nseq;
    a.width = width;
    a.dtype = dtype;
    a.rows = rows;
    a.norms = norms;
    a.partial = static_cast<float *>(ws);
    ENC_CUDA(launch_pool_forward(a, static_cast<cudaStream_t>(stream)));
    return SIEVE_OK;
}

sieve_status sieve_unit_pool_backward(const float *drows, const float *rows, const float *norms,
                                      const int32_t *offsets, int64_t tokens, int64_t nseq, int32_t width,
                                      int32_t dtype, void *dh, int64_t dh_stride, void *stream) {
    sieve_status rc = check_pool(offsets, tokens, nseq, width, dtype, dh, dh_stride, rows, norms);
    if (rc != SIEVE_OK) return rc;
    if ((nseq > 0 && !drows) || !aligned4(drows)) return SIEVE_EINVAL;
    if ((rc = check_current_device()) != SIEVE_OK) return rc;
    if (nseq == 0 || tokens == 0) return SIEVE_OK;
    PoolArgs a = {};
    a.dh = dh;
    a.stride = dh_stride;
    a.offsets = offsets;
    a.tokens = (int)tokens;
    a.nseq = nseq;
    a.width = width;
    a.dtype = dtype;
    a.drows = drows;
    a.rows_in = rows;
    a.norms_in = norms;
    ENC_CUDA(launch_pool_backward(a, static_cast<cudaStream_t>(stream)));
    return SIEVE_OK;
}

}  // extern "C"
