// norm.cu -- layer norm over the last axis, forward and backward.
#include "encoder.cuh"

namespace sieve {
namespace enc {
namespace {

// Sum of a value over a group of TPR threads (a warp, or the whole block).
template <int TPR>
__device__ __forceinline__ float group_sum(float v, float *smem) {
    v = warp_sum(v);
    if constexpr (TPR > 32) {
        __syncthreads();
        if (lane_id() == 0) smem[threadIdx.x >> 5] = v;
        __syncthreads();
        v = 0.f;
#pragma unroll
        for (int w = 0; w < TPR / 32; ++w) v += smem[w];
    }
    return v;
}

// One row per group of TPR threads, held in registers: NCH chunks of VEC
// elements a thread, chunk c of thread i at (c * TPR + i) * VEC.
template <typename T, typename W, int VEC, int TPR, int NCH>
__global__ void __launch_bounds__(TPR > 128 ? TPR : 128)
    k_norm_forward(const NormArgs a) {
    constexpr int kRows = TPR >= 128 ? 1 : 128 / TPR;
    __shared__ float smem[32];
    const int i = threadIdx.x % TPR;
    const int64_t row = (int64_t)blockIdx.x * kRows + threadIdx.x / TPR;
    if (TPR == 32 && row >= a.rows) return;
    const T *x = static_cast<const T *>(a.x) + row * a.x_stride;
    float v[NCH][VEC];
    float s = 0.f;
#pragma unroll
    for (int c = 0; c < NCH; ++c) {
        const int col = (c * TPR + i) * VEC;
        if (col < a.width) load_vec<T, VEC>(x + col, v[c]);
        else
#pragma unroll
            for (int e = 0; e < VEC; ++e) v[c][e] = 0.f;
#pragma unroll
        for (int e = 0; e < VEC; ++e) s += v[c][e];
    }
    const float mean = group_sum<TPR>(s, smem) / (float)a.width;
    float q = 0.f;
#pragma unroll
    for (int c = 0; c < NCH; ++c)
        if ((c * TPR + i) * VEC < a.width)
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                v[c][e] -= mean;
                q = fmaf(v[c][e], v[c][e], q);
            }
    const float rstd = 1.f / sqrtf(group_sum<TPR>(q, smem) / (float)a.width + a.eps);
    T *y = static_cast<T *>(a.y) + row * a.y_stride;
    const W *w = static_cast<const W *>(a.weight), *b = static_cast<const W *>(a.bias);
#pragma unroll
    for (int c = 0; c < NCH; ++c) {
        const int col = (c * TPR + i) * VEC;
        if (col >= a.width) continue;
        float wv[VEC], bv[VEC];
        load_vec<W, VEC>(w + col, wv);
        if (b) load_vec<W, VEC>(b + col, bv);
#pragma unroll
        for (int e = 0; e < VEC; ++e) v[c][e] = fmaf(v[c][e] * rstd, wv[e], b ? bv[e] : 0.f);
        store_vec<T, VEC>(y + col, v[c]);
    }
    if (a.mean && i == 0) {
        a.mean[row] = mean;
        a.rstd[row] = rstd;
    }
}

// Backward: a block of TPR threads walks its rows, R of them at a time, and
// keeps the column sums of dweight and dbias of its columns in registers;
// they go to partial[block][2][width] and k_norm_reduce adds the blocks up.
template <typename T, typename W, int VEC, int TPR, int NCH, int R>
__global__ void __launch_bounds__(TPR)
    k_norm_backward(const NormArgs a) {
    __shared__ float smem[2 * R][TPR / 32];
    const int i = threadIdx.x;
    const T *dy = static_cast<const T *>(a.dy), *x = static_cast<const T *>(a.x);
    T *dx = static_cast<T *>(a.dx);
    float wv[NCH][VEC], dw[NCH][VEC], db[NCH][VEC];
#pragma unroll
    for (int c = 0; c < NCH; ++c) {
        const int col = (c * TPR + i) * VEC;
        if (col < a.width) load_vec<W, VEC>(static_cast<const W *>(a.weight) + col, wv[c]);
#pragma unroll
        for (int e = 0; e < VEC; ++e) dw[c][e] = db[c][e] = 0.f;
    }
    const float inv_n = 1.f / (float)a.width;
    for (int64_t r0 = (int64_t)blockIdx.x * R; r0 < a.rows; r0 += (int64_t)gridDim.x * R) {
        float g[R][NCH][VEC], xh[R][NCH][VEC], rs[R], s1[R], s2[R];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int64_t row = r0 + r;
            const bool live = row < a.rows;
            const float mu = live ? __ldg(a.mean_in + row) : 0.f;
            rs[r] = live ? __ldg(a.rstd_in + row) : 0.f;
            s1[r] = s2[r] = 0.f;
#pragma unroll
            for (int c = 0; c < NCH; ++c) {
                const int col = (c * TPR + i) * VEC;
                if (live && col < a.width) {
                    load_vec<T, VEC>(dy + row * a.dy_stride + col, g[r][c]);
                    load_vec<T, VEC>(x + row * a.x_stride + col, xh[r][c]);
#pragma unroll
                    for (int e = 0; e < VEC; ++e) xh[r][c][e] = (xh[r][c][e] - mu) * rs[r];
                } else {
#pragma unroll
                    for (int e = 0; e < VEC; ++e) g[r][c][e] = xh[r][c][e] = 0.f;
                }
            }
        }
#pragma unroll
        for (int r = 0; r < R; ++r) {
#pragma unroll
            for (int c = 0; c < NCH; ++c)
                if ((c * TPR + i) * VEC < a.width)
#pragma unroll
                    for (int e = 0; e < VEC; ++e) {
                        const float d = g[r][c][e], u = xh[r][c][e];
                        dw[c][e] = fmaf(d, u, dw[c][e]);
                        db[c][e] += d;
                        const float gw = d * wv[c][e];
                        g[r][c][e] = gw;
                        s1[r] += gw;
                        s2[r] = fmaf(gw, u, s2[r]);
                    }
            s1[r] = warp_sum(s1[r]);
            s2[r] = warp_sum(s2[r]);
        }
        if constexpr (TPR > 32) {
            __syncthreads();
            if (lane_id() == 0)
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    smem[2 * r][i >> 5] = s1[r];
                    smem[2 * r + 1][i >> 5] = s2[r];
                }
            __syncthreads();
#pragma unroll
            for (int r = 0; r < R; ++r) {
                s1[r] = s2[r] = 0.f;
#pragma unroll
                for (int w = 0; w < TPR / 32; ++w) {
                    s1[r] += smem[2 * r][w];
                    s2[r] += smem[2 * r + 1][w];
                }
            }
        }
#pragma unroll
        for (int r = 0; r < R; ++r) {
            if (r0 + r >= a.rows) continue;
            const float m1 = s1[r] * inv_n, m2 = s2[r] * inv_n;
#pragma unroll
            for (int c = 0; c < NCH; ++c) {
                const int col = (c * TPR + i) * VEC;
                if (col >= a.width) continue;
                float o[VEC];
#pragma unroll
                for (int e = 0; e < VEC; ++e) o[e] = rs[r] * (g[r][c][e] - m1 - xh[r][c][e] * m2);
                store_vec<T, VEC>(dx + (r0 + r) * a.dx_stride + col, o);
            }
        }
    }
    float *pw = a.partial + (int64_t)blockIdx.x * 2 * a.width, *pb = pw + a.width;
#pragma unroll
    for (int c = 0; c < NCH; ++c) {
        const int col = (c * TPR + i) * VEC;
#pragma unroll
        for (int e = 0; e < VEC; ++e)
            if (col + e < a.width) {
                pw[col + e] = dw[c][e];
                pb[col + e] = db[c][e];
            }
    }
}

// dweight and dbias: the sum over blocks of their partial sums.  32 columns
// by 32 strands of blocks; each strand adds its blocks in order, the strands
// in order after that.
template <typename W>
__global__ void __launch_bounds__(1024) k_norm_reduce(const NormArgs a, int blocks) {
    __shared__ float part[32][33];
    const int lane = threadIdx.x & 31, strand = threadIdx.x >> 5;
    const int col = blockIdx.x * 32 + lane;
    const float *p = a.partial + (int64_t)blockIdx.y * a.width;
    float s = 0.f;
    if (col < a.width)
#pragma unroll 4
        for (int b = strand; b < blocks; b += 32) s += p[(int64_t)b * 2 * a.width + col];
    part[strand][lane] = s;
    __syncthreads();
    if (strand == 0 && col < a.width) {
        float t = 0.f;
#pragma unroll
        for (int k = 0; k < 32; ++k) t += part[k][lane];
        static_cast<W *>(blockIdx.y ? a.dbias : a.dweight)[col] = from_f32<W>(t);
    }
}

bool multiple(int64_t v, int m) { return v % m == 0; }
bool aligned(const void *p, size_t m) { return reinterpret_cast<uintptr_t>(p) % m == 0; }

// Whether rows can be moved 16 bytes at a time (weights of another type
// move the same number of elements).
template <typename T, typename W>
bool wide(const NormArgs &a) {
    constexpr int v = 16 / sizeof(T);
    return multiple(a.width, v) && multiple(a.x_stride, v) && multiple(a.y_stride, v) &&
           multiple(a.dy_stride, v) && multiple(a.dx_stride, v) && aligned(a.x, 16) && aligned(a.y, 16) &&
           aligned(a.dy, 16) && aligned(a.dx, 16) && aligned(a.weight, 16) && aligned(a.bias, 16);
}

template <typename T, typename W, int VEC, int TPR, int NCH>
cudaError_t forward_as(const NormArgs &a, cudaStream_t st) {
    constexpr int rows = TPR >= 128 ? 1 : 128 / TPR;
    k_norm_forward<T, W, VEC, TPR, NCH>
        <<<(unsigned)ceil_div(a.rows, rows), TPR > 128 ? TPR : 128, 0, st>>>(a);
    return cudaGetLastError();
}

template <typename T, typename W>
cudaError_t forward(const NormArgs &a, cudaStream_t st) {
    constexpr int V = 16 / sizeof(T);
    if (wide<T, W>(a)) {
        const int chunks = a.width / V;
        if (chunks <= 32) return forward_as<T, W, V, 32, 1>(a, st);
        if (chunks <= 64) return forward_as<T, W, V, 32, 2>(a, st);
        if (chunks <= 128) return forward_as<T, W, V, 32, 4>(a, st);
        if (chunks <= 512) return forward_as<T, W, V, 128, 4>(a, st);
        return forward_as<T, W, V, 512, V == 8 ? 4 : 8>(a, st);
    }
    if (a.width <= 256) return forward_as<T, W, 1, 32, 8>(a, st);
    if (a.width <= 2048) return forward_as<T, W, 1, 128, 16>(a, st);
    return forward_as<T, W, 1, 512, 32>(a, st);
}

template <typename T, typename W, int VEC, int TPR, int NCH, int R>
cudaError_t backward_as(const NormArgs &a, int blocks, cudaStream_t st) {
    k_norm_backward<T, W, VEC, TPR, NCH, R><<<blocks, TPR, 0, st>>>(a);
    return cudaGetLastError();
}

constexpr int kMaxBlocks = 152 * 4;

int backward_blocks(int64_t rows, int width) {
    (void)width;
    return (int)(rows < kMaxBlocks ? rows : kMaxBlocks);
}

template <typename T, typename W>
cudaError_t backward(const NormArgs &a, cudaStream_t st) {
    constexpr int V = 16 / sizeof(T);
    const int blocks = backward_blocks(a.rows, a.width);
    cudaError_t e = cudaSuccess;
    if (blocks > 0) {
        if (wide<T, W>(a)) {
            const int chunks = a.width / V;
            if (chunks <= 32) e = backward_as<T, W, V, 32, 1, 4>(a, blocks, st);
            else if (chunks <= 64) e = backward_as<T, W, V, 64, 1, 4>(a, blocks, st);
            else if (chunks <= 128) e = backward_as<T, W, V, 128, 1, 4>(a, blocks, st);
            else if (chunks <= 256) e = backward_as<T, W, V, 256, 1, 2>(a, blocks, st);
            else if (chunks <= 512) e = backward_as<T, W, V, 512, 1, 2>(a, blocks, st);
            else e = backward_as<T, W, V, 512, V == 8 ? 4 : 8, 1>(a, blocks, st);
        } else {
            if (a.width <= 128) e = backward_as<T, W, 1, 32, 4, 4>(a, blocks, st);
            else if (a.width <= 1024) e = backward_as<T, W, 1, 128, 8, 2>(a, blocks, st);
            else if (a.width <= 4096) e = backward_as<T, W, 1, 512, 8, 1>(a, blocks, st);
            else e = backward_as<T, W, 1, 1024, 16, 1>(a, blocks, st);
        }
        if (e != cudaSuccess) return e;
    }
    k_norm_reduce<W><<<dim3((unsigned)ceil_div(a.width, 32), a.dbias ? 2 : 1), 1024, 0, st>>>(a, blocks);
    return cudaGetLastError();
}

template <typename F>
cudaError_t by_type(int dtype, int wtype, F f) {
    if (dtype == SIEVE_F32) return f(float{}, float{});
    if (dtype == SIEVE_F16) return wtype == SIEVE_F32 ? f(__half{}, float{}) : f(__half{}, __half{});
    return wtype == SIEVE_F32 ? f(__nv_bfloat16{}, float{}) : f(__nv_bfloat16{}, __nv_bfloat16{});
}

}  // namespace

cudaError_t launch_norm_forward(const NormArgs &a, cudaStream_t st) {
    return by_type(a.dtype, a.weight_dtype,
                   [&](auto t, auto w) { return forward<decltype(t), decltype(w)>(a, st); });
}

cudaError_t launch_norm_backward(const NormArgs &a, cudaStream_t st) {
    return by_type(a.dtype, a.weight_dtype,
                   [&](auto t, auto w) { return backward<decltype(t), decltype(w)>(a, st); });
}

size_t norm_backward_workspace_bytes(int64_t rows, int width) {
    return (size_t)round_up((int64_t)backward_blocks(rows, width) * 2 * width * (int64_t)sizeof(float) + 256, 256);
}

}  // namespace enc
}  // namespace sieve
