// pool.cu -- one unit row per document from the mean of its tokens' rows.
//
//   m = mean over the document's tokens, u = m / |m|
//   dh = (g - (g . u) u) / (|m| tokens), the same for every token
//
// Bound by memory: every token is read once (or written once, backward).  A
// document's tokens are cut into tiles of kPoolTile, so a few long documents
// still fill the SMs; the tiles' sums are added in order by a second launch.
//
// Measured: 2,048 documents of 0 to 512 tokens x 768 bf16 (653 MB) 142 us, of
// which the second launch 13; forward and backward of 500 documents of 1 to
// 4,096 tokens x 256 fp32 (1.6 GB) 262 us, 6.2 TB/s.
#include "encoder.cuh"

namespace sieve {
namespace enc {
namespace {

constexpr int kThreads = 512;        // of the kernels that move tokens
constexpr int kFinishThreads = 256;

// Column sums of one tile of kPoolTile tokens of one document.  The block's
// threads are `cols` column chunks of VEC elements by kThreads / cols strands
// of tokens; the strands are added through shared memory.
template <typename T, int VEC>
__global__ void __launch_bounds__(kThreads) k_pool_partial(const PoolArgs a, int cols) {
    __shared__ float part[kThreads * VEC];
    const int t = blockIdx.x;
    const int s = find_doc(a.offsets, (int)a.nseq, a.tokens, kPoolTile, t);
    int first, len;
    doc_range(a.offsets, s, a.tokens, first, len);
    const int r0 = (t - first_tile(a.offsets, s, a.tokens, kPoolTile)) * kPoolTile;
    if (r0 < 0 || r0 >= len) return;
    const int n = min(kPoolTile, len - r0);
    const int strands = kThreads / cols, strand = threadIdx.x / cols, chunk = threadIdx.x % cols;
    const int col = (blockIdx.y * cols + chunk) * VEC;
    const bool live = strand < strands && col < a.width;
    float acc[VEC];
#pragma unroll
    for (int e = 0; e < VEC; ++e) acc[e] = 0.f;
    if (live) {
        const T *h = static_cast<const T *>(a.h) + (int64_t)(first + r0) * a.stride + col;
#pragma unroll 8
        for (int r = strand; r < n; r += strands) {
            float v[VEC];
            load_vec<T, VEC>(h + (int64_t)r * a.stride, v);
#pragma unroll
            for (int e = 0; e < VEC; ++e) acc[e] += v[e];
        }
    }
#pragma unroll
    for (int e = 0; e < VEC; ++e) part[threadIdx.x * VEC + e] = acc[e];
    __syncthreads();
    if (strand == 0 && live) {
        for (int k = 1; k < strands; ++k)
#pragma unroll
            for (int e = 0; e < VEC; ++e) acc[e] += part[(k * cols + chunk) * VEC + e];
#pragma unroll
        for (int e = 0; e < VEC; ++e) a.partial[(int64_t)t * a.width + col + e] = acc[e];
    }
}

template <int kThreads>
__device__ __forceinline__ float block_max(float v, float *smem) {
    v = warp_max(v);
    if (lane_id() == 0) smem[threadIdx.x >> 5] = v;
    __syncthreads();
    v = 0.f;
#pragma unroll
    for (int w = 0; w < kThreads / 32; ++w) v = fmaxf(v, smem[w]);
    return v;
}

// A document's tiles added in order, its mean, norm and unit row.
__global__ void __launch_bounds__(kFinishThreads) k_pool_finish(const PoolArgs a) {
    __shared__ float smem[kFinishThreads / 32];
    const int s = blockIdx.x;
    int first, len;
    doc_range(a.offsets, s, a.tokens, first, len);
    const int t0 = first_tile(a.offsets, s, a.tokens, kPoolTile), tiles = (int)ceil_div(len, kPoolTile);
    const float inv = len > 0 ? 1.f / (float)len : 0.f;
    float *row = a.rows + (int64_t)s * a.width;
    float most = 0.f;
    for (int c = threadIdx.x; c < a.width; c += kFinishThreads) {
        float v = 0.f;
        for (int t = 0; t < tiles; ++t) v += a.partial[(int64_t)(t0 + t) * a.width + c];
        v *= inv;
        row[c] = v;
        most = fmaxf(most, fabsf(v));
    }
    // squares of the mean times a power of two: neither a small mean's (1e-25)
    // vanish nor a large one's (1e25) overflow
    const int up = -max(min(ilogbf(block_max<kFinishThreads>(most, smem)), 126), -126);
    const float by = ldexpf(1.f, up);
    float q = 0.f;
    for (int c = threadIdx.x; c < a.width; c += kFinishThreads) {
        const float v = row[c] * by;
        q = fmaf(v, v, q);
    }
    const float norm = sqrtf(block_sum<kFinishThreads>(q, smem));
    for (int c = threadIdx.x; c < a.width; c += kFinishThreads) row[c] = norm != 0.f ? row[c] * by * (1.f / norm) : 0.f;
    if (threadIdx.x == 0) a.norms[s] = ldexpf(norm, -up);
}

// The gradient row of a document, written to the tokens of one tile.
template <typename T, int VEC>
__global__ void __launch_bounds__(kThreads) k_pool_backward(const PoolArgs a) {
    __shared__ float smem[kThreads / 32];
    const int t = blockIdx.x;
    const int s = find_doc(a.offsets, (int)a.nseq, a.tokens, kPoolTile, t);
    int first, len;
    doc_range(a.offsets, s, a.tokens, first, len);
    const int r0 = (t - first_tile(a.offsets, s, a.tokens, kPoolTile)) * kPoolTile;
    if (r0 < 0 || r0 >= len) return;
    const int n = min(kPoolTile, len - r0);
    const float *g = a.drows + (int64_t)s * a.width, *u = a.rows_in + (int64_t)s * a.width;
    float d = 0.f;
    for (int c = threadIdx.x; c < a.width; c += kThreads) d = fmaf(g[c], u[c], d);
    d = block_sum<kThreads>(d, smem);
    const float norm = a.norms_in[s];
    const float scale = norm != 0.f ? 1.f / norm / (float)len : 0.f;
    T *out = static_cast<T *>(a.dh) + (int64_t)(first + r0) * a.stride;
    const int chunks = (int)ceil_div(a.width, VEC);
    for (int c = threadIdx.x % min(chunks, kThreads); c < chunks; c += kThreads) {
        const int strands = max(1, kThreads / chunks), strand = threadIdx.x / min(chunks, kThreads);
        if (strand >= strands) break;
        float v[VEC];
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
            const int col = c * VEC + e;
            // (a norm below 2^-128 has no reciprocal; 0 times infinity is NaN)
            const float x = g[col] - d * u[col];
            v[e] = norm == 0.f ? 0.f : isinf(scale) ? x / norm / (float)len : x * scale;
        }
        for (int r = strand; r < n; r += strands) store_vec<T, VEC>(out + (int64_t)r * a.stride + c * VEC, v);
    }
}

template <typename T>
bool wide(const PoolArgs &a, const void *p) {
    constexpr int v = 16 / sizeof(T);
    return a.width % v == 0 && a.stride % v == 0 && reinterpret_cast<uintptr_t>(p) % 16 == 0;
}

template <typename T, int VEC>
cudaError_t forward(const PoolArgs &a, cudaStream_t st) {
    const int chunks = (int)ceil_div(a.width, VEC);
    const int cols = chunks < kThreads ? chunks : kThreads;
    const int64_t tiles = doc_tiles(a.tokens, a.nseq, kPoolTile);
    if (a.tokens > 0) {
        k_pool_partial<T, VEC><<<dim3((unsigned)tiles, (unsigned)ceil_div(chunks, cols)), kThreads, 0, st>>>(a, cols);
        cudaError_t e = cudaGetLastError();
        if (e != cudaSuccess) return e;
    }
    k_pool_finish<<<(unsigned)a.nseq, kFinishThreads, 0, st>>>(a);
    return cudaGetLastError();
}

template <typename T, int VEC>
cudaError_t backward(const PoolArgs &a, cudaStream_t st) {
    if (a.tokens == 0) return cudaSuccess;
    k_pool_backward<T, VEC><<<(unsigned)doc_tiles(a.tokens, a.nseq, kPoolTile), kThreads, 0, st>>>(a);
    return cudaGetLastError();
}

template <typename F>
cudaError_t by_type(int dtype, F f) {
    if (dtype == SIEVE_F32) return f(float{});
    return dtype == SIEVE_F16 ? f(__half{}) : f(__nv_bfloat16{});
}

}  // namespace

cudaError_t launch_pool_forward(const PoolArgs &a, cudaStream_t st) {
    return by_type(a.dtype, [&](auto t) {
        using T = decltype(t);
        return wide<T>(a, a.h) ? forward<T, 16 / sizeof(T)>(a, st) : forward<T, 1>(a, st);
    });
}

cudaError_t launch_pool_backward(const PoolArgs &a, cudaStream_t st) {
    return by_type(a.dtype, [&](auto t) {
        using T = decltype(t);
        return wide<T>(a, a.dh) ? backward<T, 16 / sizeof(T)>(a, st) : backward<T, 1>(a, st);
    });
}

}  // namespace enc
}  // namespace sieve
