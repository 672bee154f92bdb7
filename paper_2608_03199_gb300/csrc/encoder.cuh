// encoder.cuh -- what the encoder operators share: element types, the
// documents of packed tokens, and the launchers behind include/sieve_encoder.h.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "common.cuh"
#include "sieve_encoder.h"

namespace sieve {

// api.cu: records the error for sieve_last_cuda_error; the sm_103 check
sieve_status record_cuda_error(cudaError_t e);
sieve_status check_current_device();

namespace enc {

// Control block at the start of an attention workspace.
struct EncCtl {
    int32_t status;   // 0 or a SIEVE_E* code of the last call
};
constexpr size_t kCtlBytes = 256;

template <typename T>
__device__ __forceinline__ float to_f32(T v);
template <>
__device__ __forceinline__ float to_f32<float>(float v) { return v; }
template <>
__device__ __forceinline__ float to_f32<__half>(__half v) { return __half2float(v); }
template <>
__device__ __forceinline__ float to_f32<__nv_bfloat16>(__nv_bfloat16 v) { return __bfloat162float(v); }

template <typename T>
__device__ __forceinline__ T from_f32(float v);
template <>
__device__ __forceinline__ float from_f32<float>(float v) { return v; }
template <>
__device__ __forceinline__ __half from_f32<__half>(float v) { return __float2half_rn(v); }
template <>
__device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

// two values rounded to 16 bits, the first in the low half
template <typename T>
__device__ __forceinline__ uint32_t pack2(float lo, float hi);
template <>
__device__ __forceinline__ uint32_t pack2<__half>(float lo, float hi) {
    const __half2 h = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t *>(&h);
}
template <>
__device__ __forceinline__ uint32_t pack2<__nv_bfloat16>(float lo, float hi) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t *>(&h);
}

// VEC consecutive elements to and from fp32; VEC > 1 moves them as one
// aligned access of 16 bytes, or two (loads of VEC * sizeof(T) = 32)
template <typename T, int VEC>
__device__ __forceinline__ void load_vec(const T *p, float (&v)[VEC]) {
    if constexpr (VEC == 1) {
        v[0] = to_f32<T>(*p);
    } else if constexpr (VEC * sizeof(T) == 16) {
        const uint4 raw = *reinterpret_cast<const uint4 *>(p);
        const T *e = reinterpret_cast<const T *>(&raw);
#pragma unroll
        for (int i = 0; i < VEC; ++i) v[i] = to_f32<T>(e[i]);
    } else {
        static_assert(VEC * sizeof(T) == 32, "");
        const uint4 r0 = reinterpret_cast<const uint4 *>(p)[0], r1 = reinterpret_cast<const uint4 *>(p)[1];
        const T *e0 = reinterpret_cast<const T *>(&r0), *e1 = reinterpret_cast<const T *>(&r1);
#pragma unroll
        for (int i = 0; i < VEC / 2; ++i) {
            v[i] = to_f32<T>(e0[i]);
            v[VEC / 2 + i] = to_f32<T>(e1[i]);
        }
    }
}
template <typename T, int VEC>
__device__ __forceinline__ void store_vec(T *p, const float (&v)[VEC]) {
    if constexpr (VEC == 1) {
        *p = from_f32<T>(v[0]);
    } else {
        static_assert(VEC * sizeof(T) == 16, "");
        uint4 raw;
        T *e = reinterpret_cast<T *>(&raw);
#pragma unroll
        for (int i = 0; i < VEC; ++i) e[i] = from_f32<T>(v[i]);
        *reinterpret_cast<uint4 *>(p) = raw;
    }
}

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}

// of the THREADS threads of a block; smem holds one float for each of its warps
template <int THREADS>
__device__ __forceinline__ float block_sum(float v, float *smem) {
    v = warp_sum(v);
    __syncthreads();
    if (lane_id() == 0) smem[threadIdx.x >> 5] = v;
    __syncthreads();
    v = 0.f;
#pragma unroll
    for (int w = 0; w < THREADS / 32; ++w) v += smem[w];
    return v;
}

__device__ __forceinline__ float warp_max(float v) {
#pragma unroll
    for (int o = 16; o; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, o));
    return v;
}

// The rows of document s among `tokens` packed rows, clamped into the array.
__device__ __forceinline__ void doc_range(const int32_t *__restrict__ off, int s, int tokens, int &first,
                                          int &len) {
    const int a = min(max(__ldg(off + s), 0), tokens);
    const int b = min(max(__ldg(off + s + 1), a), tokens);
    first = a;
    len = b - a;
}

// Tiles of `step` rows of packed documents, without a table: document s owns
// the tile numbers from off[s] / step + s up to those of document s + 1.  That
// is always room for its ceil(len / step) tiles (at most one number per
// document stays unused), so tokens / step + nseq numbers hold every tile, and
// a block finds its document by a search in the offsets.  A whole warp calls
// this (32 probes per level); returns the last document whose first number
// is at most t.
__host__ __device__ __forceinline__ int64_t doc_tiles(int64_t tokens, int64_t nseq, int step) {
    return tokens / step + nseq;
}
__device__ __forceinline__ int first_tile(const int32_t *__restrict__ off, int s, int tokens, int step) {
    return min(max(__ldg(off + s), 0), tokens) / step + s;
}
__device__ __forceinline__ int find_doc(const int32_t *__restrict__ off, int nseq, int tokens, int step, int t) {
    int lo = 0, n = nseq;   // the answer is in [lo, lo + n)
    const int lane = lane_id();
    while (n > 1) {
        const int stride = (n + 31) / 32;
        const int s = lo + lane * stride;
        const bool le = lane * stride < n && first_tile(off, s, tokens, step) <= t;
        // document lo always qualifies, so the highest set bit exists once
        // the offsets are nondecreasing; max() keeps broken ones in range
        const unsigned m = __ballot_sync(0xffffffffu, le);
        const int k = max(31 - __clz((int)m), 0);
        lo += k * stride;
        n = min(stride, n - k * stride);
    }
    return lo;
}
struct NormArgs {
    const void *x, *dy, *weight, *bias;
    void *y, *dx, *dweight, *dbias;
    float *mean, *rstd;
    const float *mean_in, *rstd_in;
    int64_t rows, x_stride, y_stride, dy_stride, dx_stride;
    int width, dtype, weight_dtype;
    float eps;
    float *partial;   // [blocks][2][width]
};
cudaError_t launch_norm_forward(const NormArgs &a, cudaStream_t st);
cudaError_t launch_norm_backward(const NormArgs &a, cudaStream_t st);
size_t norm_backward_workspace_bytes(int64_t rows, int width);

struct PoolArgs {
    const void *h;
    void *dh;
    const int32_t *offsets;
    const float *drows, *rows_in, *norms_in;
    float *rows, *norms, *partial;   // partial [tiles][width]
    int64_t stride, nseq;
    int tokens, width, dtype;
};
constexpr int kPoolTile = 256;   // tokens per block
cudaError_t launch_pool_forward(const PoolArgs &a, cudaStream_t st);
cudaError_t launch_pool_backward(const PoolArgs &a, cudaStream_t st);

struct AttentionArgs {
    sieve_attention_args a;
    void *out;
    float *lse;
    const void *dout;
    const void *out_in;
    const float *lse_in;
    void *dq, *dk, *dv;
    int64_t dq_ts, dq_hs, dk_ts, dk_hs, dv_ts, dv_hs;
    float *dtable;
    EncCtl *ctl;
};
size_t attention_workspace_bytes(const sieve_attention_args &a);
size_t attention_backward_workspace_bytes(const sieve_attention_args &a);
sieve_status launch_attention_forward(const AttentionArgs &p, void *ws, cudaStream_t st);
sieve_status launch_attention_backward(const AttentionArgs &p, void *ws, cudaStream_t st);

}  // namespace enc
}  // namespace sieve
