// blocks_api.cu -- the C ABI of the operators around an encoder's blocks
// (declared in include/sieve_encoder.h): argument checks and workspace layout.
#include <cmath>

#include "blocks.cuh"

using namespace sieve;
using namespace sieve::enc;

namespace {

#define BLOCKS_CUDA(call)                                       \
    do {                                                        \
        cudaError_t e_ = (call);                                \
        if (e_ != cudaSuccess) return record_cuda_error(e_);    \
    } while (0)

bool aligned_to(const void *p, size_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }
size_t type_bytes(int dtype) { return dtype == SIEVE_F32 ? 4 : 2; }
bool is_type(int dtype) { return dtype == SIEVE_F32 || dtype == SIEVE_F16 || dtype == SIEVE_BF16; }
bool is_id_type(int type) { return type == SIEVE_I32 || type == SIEVE_I64; }
constexpr int64_t kMaxStride = (int64_t)1 << 38;

// a row-strided matrix that a kernel reads or writes
bool bad_rows(const void *p, int64_t stride, int64_t rows, int64_t width, int32_t dtype) {
    return rows > 0 && (!p || (rows > 1 && stride < width) || stride >= kMaxStride || !aligned_to(p, type_bytes(dtype)));
}
// ids or targets
bool bad_ids(const void *p, int32_t type, int64_t n) {
    return !is_id_type(type) || (n > 0 && !p) || !aligned_to(p, type == SIEVE_I64 ? 8 : 4);
}
sieve_status check_workspace(const void *ws, size_t have, size_t need) {
    if (have < need || (need && (!ws || !aligned_to(ws, 256)))) return SIEVE_EWORKSPACE;
    return SIEVE_OK;
}

sieve_status check_embed(int64_t tokens, int64_t vocab, int32_t width) {
    if (tokens < 0 || tokens > SIEVE_EMBED_MAX_TOKENS || vocab < 1 || vocab > SIEVE_EMBED_MAX_VOCAB) return SIEVE_EINVAL;
    return width < 1 || width > SIEVE_EMBED_MAX_WIDTH ? SIEVE_EINVAL : SIEVE_OK;
}

sieve_status check_residual_sizes(int64_t rows, int32_t width) {
    return rows < 0 || rows > INT32_MAX || width < 1 || width > SIEVE_RESIDUAL_NORM_MAX_WIDTH ? SIEVE_EINVAL : SIEVE_OK;
}
sieve_status check_residual(const sieve_residual_norm_args *a) {
    if (!a) return SIEVE_EINVAL;
    const sieve_status rc = check_residual_sizes(a->rows, a->width);
    if (rc != SIEVE_OK) return rc;
    if (!is_type(a->dtype) || (a->weight_dtype != a->dtype && a->weight_dtype != SIEVE_F32)) return SIEVE_EINVAL;
    if ((a->rms != 0 && a->rms != 1) || !std::isfinite(a->alpha) || !(a->eps >= 0.f) || !std::isfinite(a->eps))
        return SIEVE_EINVAL;
    if ((!a->weight && !a->post_weight) || (a->bias && !a->weight) || (a->post_bias && !a->post_weight))
        return SIEVE_EINVAL;
    const size_t size = type_bytes(a->weight_dtype);
    for (const void *w : {a->weight, a->bias, a->post_weight, a->post_bias})
        if (!aligned_to(w, size)) return SIEVE_EINVAL;
    if (bad_rows(a->h, a->h_stride, a->rows, a->width, a->dtype) ||
        bad_rows(a->y, a->y_stride, a->rows, a->width, a->dtype))
        return SIEVE_EINVAL;
    switch (a->gate_kind) {
        case SIEVE_GATE_NONE: return a->gate ? SIEVE_EINVAL : SIEVE_OK;
        case SIEVE_GATE_COLUMN: return !a->gate || !aligned_to(a->gate, size) ? SIEVE_EINVAL : SIEVE_OK;
        case SIEVE_GATE_ROW:
            return bad_rows(a->gate, a->gate_stride, a->rows, a->width, a->dtype) ? SIEVE_EINVAL : SIEVE_OK;
        default: return SIEVE_EINVAL;
    }
}

// a matrix that tensor maps are made of
bool bad_tiles(const void *p, int64_t stride, int64_t rows, int64_t width) {
    return rows > 0 && (!p || !aligned_to(p, 16) || stride % 8 || (rows > 1 && stride < width) || stride < 0 ||
                        stride >= kMaxStride);
}
sieve_status check_cross_entropy(const sieve_cross_entropy_args *a, bool pointers) {
    if (!a) return SIEVE_EINVAL;
    if (a->dtype != SIEVE_F16 && a->dtype != SIEVE_BF16) return SIEVE_EINVAL;
    if (a->rows < 0 || a->rows > SIEVE_CROSS_ENTROPY_MAX_ROWS || a->classes < 1 ||
        a->classes > SIEVE_CROSS_ENTROPY_MAX_CLASSES)
        return SIEVE_EINVAL;
    if (a->width < 8 || a->width % 8 || a->width > SIEVE_CROSS_ENTROPY_MAX_WIDTH) return SIEVE_EINVAL;
    if (!is_id_type(a->target_type) || !std::isfinite(a->scale) || a->wait_limit < 0) return SIEVE_EINVAL;
    if (!pointers) return SIEVE_OK;
    if (bad_tiles(a->h, a->h_stride, a->rows, a->width) || bad_tiles(a->weight, a->weight_stride, a->classes, a->width))
        return SIEVE_EINVAL;
    return !aligned_to(a->bias, 4) || bad_ids(a->targets, a->target_type, a->rows) ? SIEVE_EINVAL : SIEVE_OK;
}

}  // namespace

extern "C" {

sieve_status sieve_embed(const void *ids, int32_t id_type, int64_t tokens, const void *table, int64_t table_stride,
                         int64_t vocab, int32_t width, int32_t table_dtype, float scale, void *out,
                         int64_t out_stride, int32_t dtype, void *stream) {
    sieve_status rc = check_embed(tokens, vocab, width);
    if (rc != SIEVE_OK) return rc;
    if (!is_type(dtype) || !is_type(table_dtype) || !std::isfinite(scale)) return SIEVE_EINVAL;
    if (bad_ids(ids, id_type, tokens) || bad_rows(table, table_stride, vocab, width, table_dtype) ||
        bad_rows(out, out_stride, tokens, width, dtype))
        return SIEVE_EINVAL;
    if ((rc = check_current_device()) != SIEVE_OK) return rc;
    if (tokens == 0) return SIEVE_OK;
    EmbedArgs a = {};
    a.ids = ids;
    a.id_type = id_type;
    a.tokens = (int)tokens;
    a.table = table;
    a.table_stride = table_stride;
    a.vocab = (int)vocab;
    a.width = width;
    a.table_dtype = table_dtype;
    a.scale = scale;
    a.out = out;
    a.out_stride = out_stride;
    a.dtype = dtype;
    BLOCKS_CUDA(launch_embed(a, static_cast<cudaStream_t>(stream)));
    return SIEVE_OK;
}

sieve_status sieve_embed_backward_workspace_size(int64_t tokens, int64_t vocab, int32_t width, size_t *bytes) {
    if (!bytes) return SIEVE_EINVAL;
    const sieve_status rc = check_embed(tokens, vocab, width);
    if (rc != SIEVE_OK) return rc;
    *bytes = embed_backward_workspace_bytes(tokens, vocab, width);
    return SIEVE_OK;
}

sieve_status sieve_embed_backward(const void *dout, int64_t dout_stride, const void *ids, int32_t id_type,
                                  int64_t tokens, int64_t vocab, int32_t width, int32_t dtype, float scale,
                                  void *dtable, int64_t dtable_stride, int32_t table_dtype, int32_t accumulate,
                                  void *ws, size_t ws_bytes, void *stream) {
    sieve_status rc = check_embed(tokens, vocab, width);
    if (rc != SIEVE_OK) return rc;
    if (!is_type(dtype) || !is_type(table_dtype) || !std::isfinite(scale) || (accumulate != 0 && accumulate != 1))
        return SIEVE_EINVAL;
    if (bad_ids(ids, id_type, tokens) || bad_rows(dout, dout_stride, tokens, width, dtype) ||
        bad_rows(dtable, dtable_stride, vocab, width, table_dtype))
        return SIEVE_EINVAL;
    if ((rc = check_workspace(ws, ws_bytes, embed_backward_workspace_bytes(tokens, vocab, width))) != SIEVE_OK) return rc;
    if ((rc = check_current_device()) != SIEVE_OK) return rc;
    EmbedArgs a = {};
    a.dout = dout;
    a.dout_stride = dout_stride;
    a.ids = ids;
    a.id_type = id_type;
    a.tokens = (int)tokens;
    a.vocab = (int)vocab;
    a.width = width;
    a.dtype = dtype;
    a.scale = scale;
    a.dtable = dtable;
    a.dtable_stride = dtable_stride;
    a.table_dtype = table_dtype;
    a.accumulate = accumulate;
    BLOCKS_CUDA(launch_embed_backward(a, ws, static_cast<cudaStream_t>(stream)));
    return SIEVE_OK;
}

sieve_status sieve_residual_norm(const sieve_residual_norm_args *a, void *stream_out, int64_t stream_stride, void *x,
                                 int64_t x_stride, float *stats, void *stream) {
    sieve_status rc = check_residual(a);
    if (rc != SIEVE_OK) return rc;
    if (bad_rows(stream_out, stream_stride, a->rows, a->width, a->dtype)) return SIEVE_EINVAL;
    if (a->weight ? bad_rows(x, x_stride, a->rows, a->width, a->dtype) : x != nullptr) return SIEVE_EINVAL;
    if (!aligned_to(stats, 4)) return SIEVE_EINVAL;
    if ((rc = check_current_device()) != SIEVE_OK) return rc;
    if (a->rows == 0) return SIEVE_OK;
    ResidualNormArgs p = {};
    p.a = *a;
    p.stream = stream_out;
    p.stream_stride = stream_stride;
    p.x = x;
    p.x_stride = x_stride;
    p.stats = stats;
    BLOCKS_CUDA(launch_residual_norm(p, static_cast<cudaStream_t>(stream)));
    return SIEVE_OK;
}

sieve_status sieve_residual_norm_backward_workspace_size(int64_t rows, int32_t width, size_t *bytes) {
    if (!bytes) return SIEVE_EINVAL;
    const sieve_status rc = check_residual_sizes(rows, width);
    if (rc != SIEVE_OK) return rc;
    *bytes = residual_norm_backward_workspace_bytes(rows, width);
    return SIEVE_OK;
}

sieve_status sieve_residual_norm_backward(const sieve_residual_norm_args *a, const sieve_residual_norm_grads *g,
                                          void *ws, size_t ws_bytes, void *stream) {
    sieve_status rc = check_residual(a);
    if (rc != SIEVE_OK) return rc;
    if (!g) return SIEVE_EINVAL;
    if (g->dstream || !a->weight)
        if (bad_rows(g->dstream, g->dstream_stride, a->rows, a->width, a->dtype)) return SIEVE_EINVAL;
    if (a->weight ? bad_rows(g->dx, g->dx_stride, a->rows, a->width, a->dtype) : g->dx != nullptr) return SIEVE_EINVAL;
    if (bad_rows(g->dh, g->dh_stride, a->rows, a->width, a->dtype) ||
        bad_rows(g->dy, g->dy_stride, a->rows, a->width, a->dtype))
        return SIEVE_EINVAL;
    if ((a->rows > 0 && !g->stats) || !aligned_to(g->stats, 4)) return SIEVE_EINVAL;
    const size_t size = type_bytes(a->weight_dtype);
    const void *weights[4] = {a->weight, a->bias, a->post_weight, a->post_bias};
    const void *grads[4] = {g->dweight, g->dbias, g->dpost_weight, g->dpost_bias};
    for (int i = 0; i < 4; ++i)
        if (!weights[i] != !grads[i] || !aligned_to(grads[i], size)) return SIEVE_EINVAL;
    if (a->gate_kind == SIEVE_GATE_ROW) {
        if (bad_rows(g->dgate, g->dgate_stride, a->rows, a->width, a->dtype)) return SIEVE_EINVAL;
    } else if (!g->dgate != (a->gate_kind == SIEVE_GATE_NONE) || !aligned_to(g->dgate, size)) {
        return SIEVE_EINVAL;
    }
    if ((rc = check_workspace(ws, ws_bytes, residual_norm_backward_workspace_bytes(a->rows, a->width))) != SIEVE_OK)
        return rc;
    if ((rc = check_current_device()) != SIEVE_OK) return rc;
    ResidualNormArgs p = {};
    p.a = *a;
    p.g = *g;
    p.partial = static_cast<float *>(ws);
    BLOCKS_CUDA(launch_residual_norm_backward(p, static_cast<cudaStream_t>(stream)));
    return SIEVE_OK;
}

sieve_status sieve_cross_entropy_workspace_size(const sieve_cross_entropy_args *a, size_t *bytes) {
    const sieve_status rc = check_cross_entropy(a, false);
    if (rc != SIEVE_OK || !bytes) return SIEVE_EINVAL;
    *bytes = cross_entropy_workspace_bytes(*a);
    return SIEVE_OK;
}

sieve_status sieve_cross_entropy(const sieve_cross_entropy_args *a, float *loss, float *lse, void *ws, size_t ws_bytes,
                                 void *stream) {
    sieve_status rc = check_cross_entropy(a, true);
    if (rc != SIEVE_OK) return rc;
    if ((a->rows > 0 && (!loss || !lse)) || !aligned_to(loss, 4) || !aligned_to(lse, 4)) return SIEVE_EINVAL;
    if ((rc = check_workspace(ws, ws_bytes, cross_entropy_workspace_bytes(*a))) != SIEVE_OK) return rc;
    if ((rc = check_current_device()) != SIEVE_OK) return rc;
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (a->rows == 0) {
        BLOCKS_CUDA(cudaMemsetAsync(ws, 0, kCtlBytes, st));
        return SIEVE_OK;
    }
    return launch_cross_entropy(*a, loss, lse, ws, st);
}

sieve_status sieve_cross_entropy_backward_workspace_size(const sieve_cross_entropy_args *a, size_t *bytes) {
    const sieve_status rc = check_cross_entropy(a, false);
    if (rc != SIEVE_OK || !bytes) return SIEVE_EINVAL;
    *bytes = cross_entropy_backward_workspace_bytes(*a);
    return SIEVE_OK;
}

sieve_status sieve_cross_entropy_backward(const sieve_cross_entropy_args *a, const sieve_cross_entropy_grads *g,
                                          void *ws, size_t ws_bytes, void *stream) {
    sieve_status rc = check_cross_entropy(a, true);
    if (rc != SIEVE_OK) return rc;
    if (!g) return SIEVE_EINVAL;
    if (a->rows > 0 && (!g->dloss || !g->loss || !g->lse)) return SIEVE_EINVAL;
    if (!aligned_to(g->dloss, 4) || !aligned_to(g->loss, 4) || !aligned_to(g->lse, 4) || !aligned_to(g->dbias, 4))
        return SIEVE_EINVAL;
    if (g->dh && bad_tiles(g->dh, g->dh_stride, a->rows, a->width)) return SIEVE_EINVAL;
    if (g->dbias && !a->bias) return SIEVE_EINVAL;
    if (g->dweight_dtype != a->dtype && g->dweight_dtype != SIEVE_F32) return SIEVE_EINVAL;
    if (g->accumulate != 0 && (g->accumulate != 1 || g->dweight_dtype != SIEVE_F32)) return SIEVE_EINVAL;
    if (g->dweight && bad_tiles(g->dweight, g->dweight_stride, a->classes, a->width)) return SIEVE_EINVAL;
    if ((rc = check_workspace(ws, ws_bytes, cross_entropy_backward_workspace_bytes(*a))) != SIEVE_OK) return rc;
    if ((rc = check_current_device()) != SIEVE_OK) return rc;
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (a->rows == 0) {
        const size_t size = type_bytes(g->dweight_dtype);
        BLOCKS_CUDA(cudaMemsetAsync(ws, 0, kCtlBytes, st));
        if (g->dweight && !g->accumulate) {
            const size_t row = a->width * size;
            BLOCKS_CUDA(cudaMemset2DAsync(g->dweight, a->classes > 1 ? g->dweight_stride * size : row, 0, row, a->classes, st));
        }
        if (g->dbias) BLOCKS_CUDA(cudaMemsetAsync(g->dbias, 0, a->classes * sizeof(float), st));
        return SIEVE_OK;
    }
    return launch_cross_entropy_backward(*a, *g, ws, st);
}

}  // extern "C"
