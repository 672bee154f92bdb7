// norm.cu -- layer norm over the last axis, forward and backward.
//
//   forward   mu = mean(x), r = 1 / sqrt(mean((x - mu)^2) + eps), xh = (x - mu) r,
//             y = xh w + b
//   backward  g = dy w, dx = r (g - mean(g) - xh mean(g xh)),
//             dw = sum over rows of dy xh, db = sum over rows of dy
//
// Both are bound by memory: a row is read once into registers, where its sums
// and its outputs come from.  The column sums of dw and db stay in registers of
// the threads that walk the rows, one pair of partial rows a block, added in a
// fixed order by a second launch: no atomics, the same bits every time.
// Everything between the load and the store is fp32.
//
// Measured: forward 200,003 x 1024 bf16 (819 MB) 149 us, 5.5 TB/s; 100,003 x
// 768 bf16 forward 54 us (307 MB, 5.7 TB/s), backward 96 us (461 MB, 4.8 TB/s: a
// warp's next row is on its way while it works on this one, at two blocks an SM) and
// 4 us for the partial sums; odd widths, element by element: 20,011 x 1001 fp32
// forward 30 us (160 MB, 5.4 TB/s), backward 62 us (240 MB, 3.9 TB/s), bf16 29 and 59.
// (Figures of this file: device time of each launch, nothing in the L2 cache.)
#include <type_traits>

#include "encoder.cuh"

namespace sieve {
namespace enc {
namespace {

// Rows wider than 1,024, and wider than 384 that cannot move 16 bytes at a time:
// one row per block of TPR threads, held in registers: NCH chunks of VEC elements
// a thread, chunk c of thread i at (c * TPR + i) * VEC.
template <typename T, typename W, int VEC, int TPR, int NCH>
__global__ void __launch_bounds__(TPR)
    k_norm_forward(const NormArgs a) {
    __shared__ float smem[32];
    const int i = threadIdx.x;
    const int64_t row = blockIdx.x;
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
    const float mean = block_sum<TPR>(s, smem) / (float)a.width;
    float q = 0.f;
#pragma unroll
    for (int c = 0; c < NCH; ++c)
        if ((c * TPR + i) * VEC < a.width)
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                v[c][e] -= mean;
                q = fmaf(v[c][e], v[c][e], q);
            }
    const float rstd = 1.f / sqrtf(block_sum<TPR>(q, smem) / (float)a.width + a.eps);
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

// The backward pass of rows wider than 1,024 and of those that cannot move 16
// bytes at a time: a block of TPR threads walks its rows, R of them at a time (their
// loads go out together, and one meeting of the block serves all), and
// keeps the column sums of dweight and dbias of its columns in registers;
// they go to partial[block][2][width] and k_norm_reduce adds the blocks up.
// (20,011 x 1001 fp32, both passes: 99 us with two rows at a time and the next two
// on their way, at two blocks of 256 an SM, which is the grid, though the registers
// would let three; 115 with four rows and one block an SM; 132 with four and none on
// their way.)
template <typename T, typename W, int VEC, int TPR, int NCH, int R>
__global__ void __launch_bounds__(TPR, TPR <= 256 ? 768 / TPR : 1) k_norm_backward(const NormArgs a) {
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
    // Element by element the next rows are on their way while these are worked
    // on (wider pieces leave no registers for it).
    constexpr bool kAhead = VEC == 1 && TPR <= 256;
    using Rows = float[R][NCH][VEC];
    auto load = [&](int64_t r0, Rows &g, Rows &xh, float (&mu)[R], float (&rs)[R]) {
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int64_t row = r0 + r;
            const bool live = row < a.rows;
            // (places past the row or the rows read its last piece: all loads
            // go out before the first is used, with no branch between them)
            const int64_t at = live ? row : a.rows - 1;
            mu[r] = __ldg(a.mean_in + at);
            rs[r] = live ? __ldg(a.rstd_in + at) : 0.f;
#pragma unroll
            for (int c = 0; c < NCH; ++c) {
                const int col = min((c * TPR + i) * VEC, a.width - VEC);
                load_vec<T, VEC>(dy + at * a.dy_stride + col, g[r][c]);
                load_vec<T, VEC>(x + at * a.x_stride + col, xh[r][c]);
            }
        }
    };
    const int64_t first = (int64_t)blockIdx.x * R, step = (int64_t)gridDim.x * R;
    Rows next_g, next_x;
    float next_mu[R], next_rs[R];
    if (kAhead) load(first, next_g, next_x, next_mu, next_rs);
    for (int64_t r0 = first; r0 < a.rows; r0 += step) {
        Rows g, xh;
        float mu[R], rs[R], s1[R], s2[R];
        if (kAhead) {
#pragma unroll
            for (int r = 0; r < R; ++r) {
                mu[r] = next_mu[r];
                rs[r] = next_rs[r];
#pragma unroll
                for (int c = 0; c < NCH; ++c)
#pragma unroll
                    for (int e = 0; e < VEC; ++e) {
                        g[r][c][e] = next_g[r][c][e];
                        xh[r][c][e] = next_x[r][c][e];
                    }
            }
            if (r0 + step < a.rows) load(r0 + step, next_g, next_x, next_mu, next_rs);
        } else {
            load(r0, g, xh, mu, rs);
        }
#pragma unroll
        for (int r = 0; r < R; ++r) s1[r] = s2[r] = 0.f;
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int c = 0; c < NCH; ++c) {
                const bool live = r0 + r < a.rows && (c * TPR + i) * VEC < a.width;
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    g[r][c][e] = live ? g[r][c][e] : 0.f;
                    xh[r][c][e] = live ? (xh[r][c][e] - mu[r]) * rs[r] : 0.f;
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

// Rows up to 1,024 wide: a warp to a row, NCH chunks of VEC elements a lane,
// chunk c of lane i at (c * 32 + i) * VEC.
constexpr int kRowWarps = 8;

template <typename T, int VEC>
struct Raw {      // VEC elements as loaded
    static_assert(VEC == 1 || VEC * sizeof(T) == 16, "");
    uint4 v;
    __device__ __forceinline__ void load(const T *p) {
        if constexpr (VEC == 1) {
            if constexpr (sizeof(T) == 4) v.x = *reinterpret_cast<const uint32_t *>(p);
            else v.x = *reinterpret_cast<const uint16_t *>(p);
        } else {
            v = *reinterpret_cast<const uint4 *>(p);
        }
    }
    __device__ __forceinline__ void get(float (&x)[VEC]) const {
        const T *e = reinterpret_cast<const T *>(&v);
#pragma unroll
        for (int i = 0; i < VEC; ++i) x[i] = to_f32<T>(e[i]);
    }
};

// Forward: one row a warp.  (A warp that walks rows with the weights in its
// registers leaves too few warps to hide the loads: 2.5 times as long at 200K x
// 1024; the weights come from the L1 cache instead.)
template <typename T, typename W, int VEC, int NCH>
__global__ void __launch_bounds__(kRowWarps * 32) k_norm_forward_rows(const NormArgs a) {
    const int lane = lane_id();
    const int64_t row = (int64_t)blockIdx.x * kRowWarps + (threadIdx.x >> 5);
    if (row >= a.rows) return;
    const T *x = static_cast<const T *>(a.x) + row * a.x_stride;
    float v[NCH][VEC], s = 0.f, q = 0.f;
#pragma unroll
    for (int c = 0; c < NCH; ++c) {
        const int col = (c * 32 + lane) * VEC;
#pragma unroll
        for (int e = 0; e < VEC; ++e) v[c][e] = 0.f;
        if (col < a.width) load_vec<T, VEC>(x + col, v[c]);
#pragma unroll
        for (int e = 0; e < VEC; ++e) s += v[c][e];
    }
    const float inv_n = 1.f / (float)a.width, mean = warp_sum(s) * inv_n;
#pragma unroll
    for (int c = 0; c < NCH; ++c)
        if ((c * 32 + lane) * VEC < a.width)
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                v[c][e] -= mean;
                q = fmaf(v[c][e], v[c][e], q);
            }
    const float rstd = 1.f / sqrtf(fmaf(warp_sum(q), inv_n, a.eps));
    T *y = static_cast<T *>(a.y) + row * a.y_stride;
    const W *w = static_cast<const W *>(a.weight), *b = static_cast<const W *>(a.bias);
#pragma unroll
    for (int c = 0; c < NCH; ++c) {
        const int col = (c * 32 + lane) * VEC;
        if (col >= a.width) continue;
        float wv[VEC], bv[VEC];
        load_vec<W, VEC>(w + col, wv);
        if (b) load_vec<W, VEC>(b + col, bv);
#pragma unroll
        for (int e = 0; e < VEC; ++e) v[c][e] = fmaf(v[c][e] * rstd, wv[e], b ? bv[e] : 0.f);
        store_vec<T, VEC>(y + col, v[c]);
    }
    if (a.mean && lane == 0) {
        a.mean[row] = mean;
        a.rstd[row] = rstd;
    }
}

// Backward, moved 16 bytes at a time: a warp walks its rows, the next one's
// elements on their way while it works on this one, and needs no other warp
// until the end.
template <typename T, typename W, int VEC, int NCH>
__global__ void __launch_bounds__(kRowWarps * 32) k_norm_backward_rows(const NormArgs a) {
    __shared__ float part[kRowWarps][32 * VEC];
    const int lane = lane_id(), warp = threadIdx.x >> 5;
    const int64_t step = (int64_t)gridDim.x * kRowWarps;
    int64_t row = (int64_t)blockIdx.x * kRowWarps + warp;
    const T *dy = static_cast<const T *>(a.dy), *x = static_cast<const T *>(a.x);
    T *dx = static_cast<T *>(a.dx);
    float wv[NCH][VEC], dw[NCH][VEC], db[NCH][VEC], mu = 0.f, rs = 0.f;
    Raw<T, VEC> ny[NCH], nx[NCH];
#pragma unroll
    for (int c = 0; c < NCH; ++c) {
        const int col = (c * 32 + lane) * VEC;
#pragma unroll
        for (int e = 0; e < VEC; ++e) dw[c][e] = db[c][e] = 0.f;
        if (col < a.width) {
            load_vec<W, VEC>(static_cast<const W *>(a.weight) + col, wv[c]);
            if (row < a.rows) {
                ny[c].load(dy + row * a.dy_stride + col);
                nx[c].load(x + row * a.x_stride + col);
            }
        }
    }
    if (row < a.rows) {
        mu = __ldg(a.mean_in + row);
        rs = __ldg(a.rstd_in + row);
    }
    const float inv_n = 1.f / (float)a.width;
    for (; row < a.rows; row += step) {
        const bool more = row + step < a.rows;
        const float r = rs, m = mu;
        float g[NCH][VEC], u[NCH][VEC], s1 = 0.f, s2 = 0.f;
        if (more) {
            mu = __ldg(a.mean_in + row + step);
            rs = __ldg(a.rstd_in + row + step);
        }
#pragma unroll
        for (int c = 0; c < NCH; ++c) {
            const int col = (c * 32 + lane) * VEC;
            if (col >= a.width) continue;
            ny[c].get(g[c]);
            nx[c].get(u[c]);
            if (more) {
                ny[c].load(dy + (row + step) * a.dy_stride + col);
                nx[c].load(x + (row + step) * a.x_stride + col);
            }
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                const float d = g[c][e];
                u[c][e] = (u[c][e] - m) * r;
                dw[c][e] = fmaf(d, u[c][e], dw[c][e]);
                db[c][e] += d;
                g[c][e] = d * wv[c][e];
                s1 += g[c][e];
                s2 = fmaf(g[c][e], u[c][e], s2);
            }
        }
        const float m1 = warp_sum(s1) * inv_n, m2 = warp_sum(s2) * inv_n;
#pragma unroll
        for (int c = 0; c < NCH; ++c) {
            const int col = (c * 32 + lane) * VEC;
            if (col >= a.width) continue;
#pragma unroll
            for (int e = 0; e < VEC; ++e) g[c][e] = r * (g[c][e] - m1 - u[c][e] * m2);
            store_vec<T, VEC>(dx + row * a.dx_stride + col, g[c]);
        }
    }
    // the block's warps added up, in order
    float *out = a.partial + (int64_t)blockIdx.x * 2 * a.width;
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int c = 0; c < NCH; ++c) {
            __syncthreads();
#pragma unroll
            for (int e = 0; e < VEC; ++e) part[warp][lane * VEC + e] = k ? db[c][e] : dw[c][e];
            __syncthreads();
            for (int i = threadIdx.x; i < 32 * VEC; i += kRowWarps * 32) {
                const int col = c * 32 * VEC + i;
                if (col >= a.width) continue;
                float t = 0.f;
#pragma unroll
                for (int w = 0; w < kRowWarps; ++w) t += part[w][i];
                out[k * a.width + col] = t;
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
    k_norm_forward<T, W, VEC, TPR, NCH><<<(unsigned)a.rows, TPR, 0, st>>>(a);
    return cudaGetLastError();
}

constexpr int kMaxBlocks = 152 * 4;
// Widest row of the row-walking kernels.  (A warp to a row against a block: 200,003
// x 1024 bf16 forward 149 us, 309; 100,003 x 768 both passes 154, 394.)
constexpr int kRowsWidth = 1024;

template <typename T, typename W, int VEC, int NCH>
cudaError_t forward_rows(const NormArgs &a, cudaStream_t st) {
    k_norm_forward_rows<T, W, VEC, NCH><<<(unsigned)ceil_div(a.rows, kRowWarps), kRowWarps * 32, 0, st>>>(a);
    return cudaGetLastError();
}
template <typename T, typename W, int VEC, int NCH>
cudaError_t backward_rows(const NormArgs &a, int blocks, cudaStream_t st) {
    k_norm_backward_rows<T, W, VEC, NCH><<<blocks, kRowWarps * 32, 0, st>>>(a);
    return cudaGetLastError();
}
// chunks of a lane, rounded up to an instantiated number
template <int VEC, typename F>
cudaError_t by_chunks(int width, F f) {
    const int n = (int)ceil_div(width, 32 * VEC);
    if constexpr (VEC == 8) {
        if (n <= 1) return f(std::integral_constant<int, 1>{});
        if (n == 2) return f(std::integral_constant<int, 2>{});
        if (n == 3) return f(std::integral_constant<int, 3>{});
        return f(std::integral_constant<int, 4>{});
    } else {
        static_assert(VEC == 4, "");
        if (n <= 2) return f(std::integral_constant<int, 2>{});
        if (n <= 4) return f(std::integral_constant<int, 4>{});
        if (n <= 6) return f(std::integral_constant<int, 6>{});
        return f(std::integral_constant<int, 8>{});
    }
}

template <typename T, typename W>
cudaError_t forward(const NormArgs &a, cudaStream_t st) {
    constexpr int V = 16 / sizeof(T);
    if (a.width <= kRowsWidth) {
        if (wide<T, W>(a))
            return by_chunks<V>(a.width, [&](auto n) { return forward_rows<T, W, V, decltype(n)::value>(a, st); });
        // element by element: a warp to a row up to 12 a lane (fp32, 150,000 x 101
        // 37 us, 46 if compiled for 12; 60,000 x 301 29 us, 55 with a block); past
        // that a block with 8 a thread (20,011 x 1001 30 us, 44 with 32 a lane)
        if (a.width <= 128) return forward_rows<T, W, 1, 4>(a, st);
        if (a.width <= 384) return forward_rows<T, W, 1, 12>(a, st);
        return forward_as<T, W, 1, 128, 8>(a, st);
    }
    if (wide<T, W>(a)) {
        // (40,000 x 2048 bf16: 78 us, 259 with 512 threads)
        const int chunks = a.width / V;
        if (chunks <= 512) return forward_as<T, W, V, 128, 4>(a, st);
        return forward_as<T, W, V, 512, V == 8 ? 4 : 8>(a, st);
    }
    // (13,000 x 1501 fp32: 33 us, 221 with 512 threads)
    if (a.width <= 2048) return forward_as<T, W, 1, 128, 16>(a, st);
    return forward_as<T, W, 1, 512, 32>(a, st);
}

template <typename T, typename W, int VEC, int TPR, int NCH, int R>
cudaError_t backward_as(const NormArgs &a, int blocks, cudaStream_t st) {
    k_norm_backward<T, W, VEC, TPR, NCH, R><<<blocks, TPR, 0, st>>>(a);
    return cudaGetLastError();
}

// Blocks of either backward kernel: enough for the SMs, and few partial sums
// where there are few rows.
int backward_blocks(int64_t rows, int width) {
    const int64_t n = width <= kRowsWidth ? ceil_div(rows, kRowWarps) : rows;
    // rows of 513 to 1,024: their registers let two blocks share an SM, and more
    // blocks only make more partial sums (100,003 x 768 bf16, both passes: 157 us;
    // 162 with twice as many)
    const int64_t most = width > 512 && width <= kRowsWidth ? kMaxBlocks / 2 : kMaxBlocks;
    return (int)(n < most ? n : most);
}

template <typename T, typename W>
cudaError_t backward(const NormArgs &a, cudaStream_t st) {
    constexpr int V = 16 / sizeof(T);
    const int blocks = backward_blocks(a.rows, a.width);
    cudaError_t e = cudaSuccess;
    if (blocks > 0) {
        if (a.width <= kRowsWidth && wide<T, W>(a)) {
            e = by_chunks<V>(a.width, [&](auto n) { return backward_rows<T, W, V, decltype(n)::value>(a, blocks, st); });
        } else if (wide<T, W>(a)) {
            // (bf16: 40,000 x 2048 126 us, 229 with 512 threads; 20,000 x 4096 158,
            // 315 with 4 pieces a thread)
            const int chunks = a.width / V;
            if (chunks <= 256) e = backward_as<T, W, V, 256, 1, 2>(a, blocks, st);
            else if (chunks <= 512) e = backward_as<T, W, V, 512, 1, 2>(a, blocks, st);
            else e = backward_as<T, W, V, 512, V == 8 ? 4 : 8, 1>(a, blocks, st);
        } else {
            // the narrowest block that holds a row at 4 elements a thread, 8 from
            // 1,025 on (fp32, against the next wider one: 150,000 x 101 120 us, 163;
            // 60,000 x 301 74, 154; 20,011 x 1001 62, 183; 7,000 x 3001 86, 317)
            if (a.width <= 128) e = backward_as<T, W, 1, 32, 4, 2>(a, blocks, st);
            else if (a.width <= 512) e = backward_as<T, W, 1, 128, 4, 2>(a, blocks, st);
            else if (a.width <= 1024) e = backward_as<T, W, 1, 256, 4, 2>(a, blocks, st);
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
