// blocks.cuh -- the operators around an encoder's blocks (embedding, residual
// norm, cross entropy): what their launchers take.
#pragma once

#include "encoder.cuh"

namespace sieve {
namespace enc {

// A type for a runtime element type.
template <typename T>
struct Type {
    using type = T;
};
template <typename F>
auto with_type(int dtype, F f) {
    if (dtype == SIEVE_F32) return f(Type<float>{});
    if (dtype == SIEVE_F16) return f(Type<__half>{});
    return f(Type<__nv_bfloat16>{});
}

// Id number i of an array of either type; -1 for one outside [0, n).
__device__ __forceinline__ int id_at(const void *ids, int id_type, int64_t i, int n) {
    if (id_type == SIEVE_I64) {
        const long long v = __ldg(static_cast<const long long *>(ids) + i);
        return v >= 0 && v < n ? (int)v : -1;
    }
    const int v = __ldg(static_cast<const int *>(ids) + i);
    return v >= 0 && v < n ? v : -1;
}

// two values of a word
template <typename T>
__device__ __forceinline__ float2 unpack2(uint32_t w);
template <>
__device__ __forceinline__ float2 unpack2<__half>(uint32_t w) { return __half22float2(*reinterpret_cast<const __half2 *>(&w)); }
template <>
__device__ __forceinline__ float2 unpack2<__nv_bfloat16>(uint32_t w) {
    return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
}

struct EmbedArgs {
    const void *ids, *table, *dout;
    void *out, *dtable;
    int64_t table_stride, out_stride, dout_stride, dtable_stride;
    int id_type, tokens, vocab, width, dtype, table_dtype, accumulate;
    float scale;
};
cudaError_t launch_embed(const EmbedArgs &a, cudaStream_t st);
cudaError_t launch_embed_backward(const EmbedArgs &a, void *ws, cudaStream_t st);
size_t embed_backward_workspace_bytes(int64_t tokens, int64_t vocab, int width);

struct ResidualNormArgs {
    sieve_residual_norm_args a;
    void *stream, *x;
    int64_t stream_stride, x_stride;
    float *stats;
    sieve_residual_norm_grads g;
    float *partial;   // [groups of threads][4][width]
    float inv_width, inv_width_rest;   // the backward launcher's: 1 / width, and what that was rounded by
};
cudaError_t launch_residual_norm(const ResidualNormArgs &p, cudaStream_t st);
cudaError_t launch_residual_norm_backward(const ResidualNormArgs &p, cudaStream_t st);
size_t residual_norm_backward_workspace_bytes(int64_t rows, int width);

size_t cross_entropy_workspace_bytes(const sieve_cross_entropy_args &a);
size_t cross_entropy_backward_workspace_bytes(const sieve_cross_entropy_args &a);
sieve_status launch_cross_entropy(const sieve_cross_entropy_args &a, float *loss, float *lse, void *ws,
                                  cudaStream_t st);
sieve_status launch_cross_entropy_backward(const sieve_cross_entropy_args &a, const sieve_cross_entropy_grads &g,
                                           void *ws, cudaStream_t st);

}  // namespace enc
}  // namespace sieve
