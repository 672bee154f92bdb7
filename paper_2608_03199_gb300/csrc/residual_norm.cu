// residual_norm.cu -- the residual step between two blocks of an encoder,
// forward and backward:
//
//   forward   u = N1(y), stream = alpha h + gate u, x = N2(stream)
//   backward  G = dstream + dN2(dx), dh = alpha G, dgate = G u,
//             dy = dN1(gate G), and the sums over rows for the weights
//
// N(v) = (v - mu) r w + b with r = 1 / sqrt(mean((v - mu)^2) + eps), mu = mean(v)
// or 0 (rms); dN(d) = r (g - mean(g) - vh mean(g vh)) with g = d w, vh = (v - mu) r
// and mean(g) left out with rms.  Either norm may be absent.
//
// Both are bound by memory: a row is read once into registers and everything
// comes from there, in fp32, rounded once.  The backward pass makes the stream
// again from h and y, so it costs no other read than the stream would and the
// rounding of the stored stream does not enter.
//
// The sums over rows stay in registers of the threads that walk the rows, four
// of them for a column: A = dx xh2, B = dx, C = d uh, D = d, where uh is the
// normed y (y itself without a post norm) and d the gradient G, times the gate
// where every row has its own.  All weights' gradients follow from these after
// the rows: a column gate w is a common factor, dpost_weight = w C, dpost_bias = w D,
// dgate = post_weight C + post_bias D.
//
// Measured (device time).  Forward: 200,003 x 1,024 bf16, rms 269 us (1.64 GB, 6.1 TB/s);
// 100,003 x 768 bf16 with both biases 97 us (614 MB, 6.3 TB/s; 113 with values converted
// and worked on one by one).  Backward: 100,003 x 768 bf16 200 us (922 MB, 4.6 TB/s; 228 one by
// one) and 6 for the weights: a row's threads meet twice, and 128 registers a thread
// leave five blocks an SM to hide it.  Tried there, against 228: 112 registers and six blocks 333 us (spills), rows copied to shared memory three ahead 297,
// twice the threads with half the elements 358, two rows to a meeting 305.  Odd rows,
// element by element: 20,011 x 1,001 fp32 with a gate for each element forward 103 us
// (401 MB, 3.9 TB/s), backward 150 (641 MB, 4.3 TB/s).
#include <type_traits>

#include "attention.cuh"
#include "blocks.cuh"

namespace sieve {
namespace enc {
namespace {

template <typename T, int VEC>
struct Piece {      // VEC elements as loaded
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
    __device__ __forceinline__ void clear() { v = make_uint4(0, 0, 0, 0); }
    __device__ __forceinline__ float get(int i) const { return to_f32<T>(reinterpret_cast<const T *>(&v)[i]); }
};

// VEC values, two to an instruction where there are two: both passes are bound by
// the instructions that they issue as much as by memory (forward 71% of the issue slots,
// 43 instructions a value, value by value).
template <int VEC>
struct Vals {
    float v[VEC];
    template <typename F2, typename F1>
    static __device__ __forceinline__ Vals by(F2 two, F1 one) {
        Vals r;
        if constexpr (VEC == 1) {
            r.v[0] = one(0);
        } else {
#pragma unroll
            for (int e = 0; e < VEC; e += 2) {
                const float2 x = two(e);
                r.v[e] = x.x;
                r.v[e + 1] = x.y;
            }
        }
        return r;
    }
    __device__ __forceinline__ float2 two(int e) const { return make_float2(v[e], v[VEC == 1 ? 0 : e + 1]); }
    static __device__ __forceinline__ Vals all(float x) {
        Vals r;
#pragma unroll
        for (int e = 0; e < VEC; ++e) r.v[e] = x;
        return r;
    }
    template <typename T>
    static __device__ __forceinline__ Vals of(const Piece<T, VEC> &p) {
        Vals r;
        if constexpr (VEC > 1 && sizeof(T) == 2) {
            const uint32_t w[4] = {p.v.x, p.v.y, p.v.z, p.v.w};
#pragma unroll
            for (int e = 0; e < VEC; e += 2) {
                const float2 x = unpack2<T>(w[e / 2]);
                r.v[e] = x.x;
                r.v[e + 1] = x.y;
            }
        } else {
#pragma unroll
            for (int e = 0; e < VEC; ++e) r.v[e] = p.get(e);
        }
        return r;
    }
    template <typename W>
    static __device__ __forceinline__ Vals at(const W *p) {
        if constexpr (VEC * sizeof(W) == 16) {
            Piece<W, VEC> x;
            x.load(p);
            return of(x);
        } else {
            Vals r;
            load_vec<W, VEC>(p, r.v);
            return r;
        }
    }
    template <typename T>
    __device__ __forceinline__ void put(T *p) const {
        if constexpr (VEC == 8) *reinterpret_cast<uint4 *>(p) = pack8<T>(v);
        else store_vec<T, VEC>(p, v);
    }
    __device__ __forceinline__ float sum() const {
        if constexpr (VEC == 1) {
            return v[0];
        } else {
            float2 s = two(0);
#pragma unroll
            for (int e = 2; e < VEC; e += 2) s = add2(s, two(e));
            return s.x + s.y;
        }
    }
};
template <int VEC>
__device__ __forceinline__ Vals<VEC> operator*(const Vals<VEC> &a, const Vals<VEC> &b) {
    return Vals<VEC>::by([&](int e) { return mul2(a.two(e), b.two(e)); }, [&](int e) { return a.v[e] * b.v[e]; });
}
template <int VEC>
__device__ __forceinline__ Vals<VEC> operator+(const Vals<VEC> &a, const Vals<VEC> &b) {
    return Vals<VEC>::by([&](int e) { return add2(a.two(e), b.two(e)); }, [&](int e) { return a.v[e] + b.v[e]; });
}
template <int VEC>
__device__ __forceinline__ Vals<VEC> fma(const Vals<VEC> &a, const Vals<VEC> &b, const Vals<VEC> &c) {
    return Vals<VEC>::by([&](int e) { return fma2(a.two(e), b.two(e), c.two(e)); }, [&](int e) { return fmaf(a.v[e], b.v[e], c.v[e]); });
}

// sum over the TPR threads of a row: a warp, or the block
template <int TPR>
__device__ __forceinline__ float row_sum(float v, float *smem) {
    if constexpr (TPR == 32) return warp_sum(v);
    else return block_sum<TPR>(v, smem);
}

// Forward.  A row per warp (TPR = 32, eight rows a block) or per block of TPR
// threads; chunk c of thread i at (c * TPR + i) * VEC.  Up to 24 elements a lane fit
// 64 registers, so that four blocks share an SM (100,003 x 768 bf16: 113 us, 126 with
// three); 32 do not (200,003 x 1024: 269 us, 315 with spills).
template <typename T, typename W, int VEC, int TPR, int NCH>
__global__ void __launch_bounds__(TPR == 32 ? 256 : TPR, TPR == 32 ? (NCH * VEC <= 24 ? 4 : 3) : 1024 / TPR)
    k_residual_norm(const ResidualNormArgs p) {
    constexpr int kRows = TPR == 32 ? 8 : 1;
    __shared__ float smem[32];
    const sieve_residual_norm_args &a = p.a;
    const int i = TPR == 32 ? lane_id() : threadIdx.x;
    const int64_t row = (int64_t)blockIdx.x * kRows + (TPR == 32 ? threadIdx.x >> 5 : 0);
    if (row >= a.rows) return;
    const T *h = static_cast<const T *>(a.h) + row * a.h_stride, *y = static_cast<const T *>(a.y) + row * a.y_stride;
    const T *gate_row = static_cast<const T *>(a.gate) + row * a.gate_stride;
    const W *gate = static_cast<const W *>(a.gate);
    const W *w1 = static_cast<const W *>(a.post_weight), *b1 = static_cast<const W *>(a.post_bias);
    const W *w2 = static_cast<const W *>(a.weight), *b2 = static_cast<const W *>(a.bias);
    const int width = a.width;
    const float inv_n = 1.f / (float)width;
    using V = Vals<VEC>;
    auto column = [&](int c) { return (c * TPR + i) * VEC; };
    Piece<T, VEC> hp[NCH], yp[NCH];
    V v[NCH];
    float s = 0.f;
#pragma unroll
    for (int c = 0; c < NCH; ++c) {
        yp[c].clear();
        if (column(c) < width) {
            yp[c].load(y + column(c));
            hp[c].load(h + column(c));
        }
    }
#pragma unroll
    for (int c = 0; c < NCH; ++c) {
        v[c] = V::of(yp[c]);
        s += v[c].sum();
    }
    // mean and factor of v, which is centred; places past the row do not count (a mean times
    // the rounded 1 / width would be rounded twice, and rows far from zero pass that on)
    auto normed = [&](float sum, float &mean, float &r) {
        mean = a.rms ? 0.f : row_sum<TPR>(sum, smem) / (float)width;
        float q = 0.f;
#pragma unroll
        for (int c = 0; c < NCH; ++c) {
            v[c] = v[c] + V::all(-mean);
            if (column(c) < width) q += (v[c] * v[c]).sum();
        }
        r = 1.f / sqrtf(fmaf(row_sum<TPR>(q, smem), inv_n, a.eps));
    };
    // v times the factor and the weight, and the bias
    auto weighted = [&](const V &x, float r, const W *w, const W *b, int col) {
        const V z = x * V::all(r);
        return b ? fma(z, V::at(w + col), V::at(b + col)) : z * V::at(w + col);
    };
    float mean1 = 0.f, r1 = 1.f, mean2 = 0.f, r2 = 1.f;
    if (w1) normed(s, mean1, r1);
    s = 0.f;
    T *out = static_cast<T *>(p.stream) + row * p.stream_stride;
#pragma unroll
    for (int c = 0; c < NCH; ++c) {
        const int col = column(c);
        if (col >= width) continue;
        if (w1) v[c] = weighted(v[c], r1, w1, b1, col);
        if (a.gate_kind == SIEVE_GATE_ROW) v[c] = v[c] * V::at(gate_row + col);
        else if (a.gate_kind == SIEVE_GATE_COLUMN) v[c] = v[c] * V::at(gate + col);
        v[c] = fma(V::all(a.alpha), V::of(hp[c]), v[c]);
        s += v[c].sum();
        v[c].put(out + col);
    }
    if (w2) {
        normed(s, mean2, r2);
        T *x = static_cast<T *>(p.x) + row * p.x_stride;
#pragma unroll
        for (int c = 0; c < NCH; ++c)
            if (column(c) < width) weighted(v[c], r2, w2, b2, column(c)).put(x + column(c));
    }
    if (p.stats && i == 0) {
        p.stats[row] = mean1;
        p.stats[a.rows + row] = r1;
        p.stats[2 * a.rows + row] = mean2;
        p.stats[3 * a.rows + row] = r2;
    }
}

// Backward.  The TPR threads of a row (a warp, four rows a block; or a block)
// walk rows, and keep the four sums of their columns in registers, or in
// shared memory (kShared) where a thread holds too much; at the end they go to
// partial[group][4][width] and k_residual_reduce adds the groups up.
constexpr int kWarpRows = 4;
__host__ __device__ constexpr int groups_of(int tpr) { return tpr == 32 ? kWarpRows : 1; }
// Blocks that share an SM: 512 threads of 128 registers where a thread has 8
// elements of a row (576 of 112 spill: 100,003 x 768 bf16 333 us against 228), 768 of 80
// where it has 4.
__host__ __device__ constexpr int blocks_per_sm(int tpr, int elements) {
    const int threads = tpr == 32 ? 32 * kWarpRows : tpr;
    return threads >= 512 ? 1 : (elements == 8 ? 512 : 768) / threads;
}

template <typename T, typename W, int VEC, int TPR, int NCH, bool kShared>
__global__ void __launch_bounds__(TPR == 32 ? 32 * kWarpRows : TPR, blocks_per_sm(TPR, NCH * VEC))
    k_residual_norm_backward(const ResidualNormArgs p) {
    extern __shared__ float acc[];                 // kShared: [4][width]
    __shared__ float2 meet[2][32];
    // Rows of few columns, where the means take most of a gradient away: they are taken off
    // before dstream is added, or what either was rounded by stays.  (From some dozens on the
    // means are off by as much themselves, and the registers that keep dstream until then
    // cost 3% at 768 columns, 16% where elements move one by one.)
    constexpr bool kMeansFirst = TPR == 32;
    const sieve_residual_norm_args &a = p.a;
    const sieve_residual_norm_grads &g = p.g;
    const int i = TPR == 32 ? lane_id() : threadIdx.x;
    const int64_t group = (int64_t)blockIdx.x * groups_of(TPR) + (TPR == 32 ? threadIdx.x >> 5 : 0);
    const int64_t step = (int64_t)gridDim.x * groups_of(TPR);
    const T *h = static_cast<const T *>(a.h), *y = static_cast<const T *>(a.y);
    const T *dstream = static_cast<const T *>(g.dstream), *dx = static_cast<const T *>(g.dx);
    const T *gate_rows = a.gate_kind == SIEVE_GATE_ROW ? static_cast<const T *>(a.gate) : nullptr;
    const W *gate = a.gate_kind == SIEVE_GATE_COLUMN ? static_cast<const W *>(a.gate) : nullptr;
    const W *w1 = static_cast<const W *>(a.post_weight), *b1 = static_cast<const W *>(a.post_bias);
    const W *w2 = static_cast<const W *>(a.weight);
    const int width = a.width;
    // 1 / width in two parts: a sum times the rounded one alone is rounded twice, and a mean
    // that is off stays where it takes most of a value away.  From the arguments, or, where
    // elements move one by one, in registers (100,003 x 768 bf16 199 us, in registers 211;
    // 20,011 x 1,001 fp32 154 and 150; divisions 213 and 162).
    const float inv_n = VEC > 1 ? p.inv_width : 1.f / (float)width;
    const float inv_rest = VEC > 1 ? p.inv_width_rest : fmaf(-inv_n, (float)width, 1.f) * inv_n;
    auto mean = [&](float sum) { return fmaf(sum, inv_n, sum * inv_rest); };
    // this thread's columns: (c * TPR + i) * VEC.  Those past the row read its last
    // piece, so that no branch lies between loads, and count for nothing.
    auto column = [&](int c) { return (c * TPR + i) * VEC; };
    auto in = [&](int c) { return column(c) < width; };
    auto place = [&](int c) { return min(column(c), width - VEC); };
    using V = Vals<VEC>;
    V sum[kShared ? 1 : 4][NCH];
    if constexpr (kShared) {
        for (int c = i; c < 4 * width; c += TPR) acc[c] = 0.f;
        __syncthreads();
    } else {
#pragma unroll
        for (int k = 0; k < 4; ++k)
#pragma unroll
            for (int c = 0; c < NCH; ++c) sum[k][c] = V::all(0.f);
    }
    // a product, or a value, added to sum k
    auto add_product = [&](int k, int c, const V &x, const V &y) {
        if constexpr (kShared) {
            if (in(c))
#pragma unroll
                for (int e = 0; e < VEC; ++e) acc[k * width + column(c) + e] += x.v[e] * y.v[e];
        } else {
            sum[k][c] = fma(x, y, sum[k][c]);
        }
    };
    auto add = [&](int k, int c, const V &x) {
        if constexpr (kShared) {
            if (in(c))
#pragma unroll
                for (int e = 0; e < VEC; ++e) acc[k * width + column(c) + e] += x.v[e];
        } else {
            sum[k][c] = sum[k][c] + x;
        }
    };
    // two sums over the row's threads at once
    int turn = 0;
    auto both_sums = [&](float &s, float &t) {
        s = warp_sum(s);
        t = warp_sum(t);
        if constexpr (TPR > 32) {
            if (lane_id() == 0) meet[turn][threadIdx.x >> 5] = make_float2(s, t);
            __syncthreads();
            s = t = 0.f;
#pragma unroll
            for (int w = 0; w < TPR / 32; ++w) {
                s += meet[turn][w].x;
                t += meet[turn][w].y;
            }
            turn ^= 1;      // the next meeting's barrier lies between these reads and the next writes here
        }
    };
    // a row's elements, on their way while the row before is worked on
    Piece<T, VEC> nh[NCH], ny[NCH], ns[NCH], nx[NCH], ng[NCH];
    float n_stats[4] = {};
    auto load = [&](int64_t row) {
#pragma unroll
        for (int c = 0; c < NCH; ++c) {
            const int col = place(c);
            ny[c].load(y + row * a.y_stride + col);
            if (dstream) ns[c].load(dstream + row * g.dstream_stride + col);
            else ns[c].clear();
            if (w2) {
                nh[c].load(h + row * a.h_stride + col);
                nx[c].load(dx + row * g.dx_stride + col);
            }
            if (gate_rows) ng[c].load(gate_rows + row * a.gate_stride + col);
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) n_stats[k] = __ldg(g.stats + k * a.rows + row);
    };
    if (group < a.rows) load(group);
    for (int64_t row = group; row < a.rows; row += step) {
        V uh[NCH], sh[NCH], G[NCH];
        Piece<T, VEC> gr[NCH], gs[kMeansFirst ? NCH : 1];
        float s1 = 0.f, s2 = 0.f;
        const float mu1 = n_stats[0], r1 = n_stats[1], mu2 = n_stats[2], r2 = n_stats[3];
#pragma unroll
        for (int c = 0; c < NCH; ++c) {
            gr[c] = ng[c];
            uh[c] = (V::of(ny[c]) + V::all(-mu1)) * V::all(r1);
            if constexpr (kMeansFirst) gs[c] = ns[c];
            else G[c] = V::of(ns[c]);
            if (!w2) continue;
            // the stream again, then the gradient through its norm
            V u = uh[c];
            if (w1) {
                if (b1) u = fma(u, V::at(w1 + place(c)), V::at(b1 + place(c)));
                else u = u * V::at(w1 + place(c));
            }
            if (gate) u = u * V::at(gate + place(c));
            else if (gate_rows) u = u * V::of(gr[c]);
            sh[c] = (fma(V::all(a.alpha), V::of(nh[c]), u) + V::all(-mu2)) * V::all(r2);
            V d = in(c) ? V::of(nx[c]) : V::all(0.f);
            add_product(0, c, d, sh[c]);
            add(1, c, d);
            d = d * V::at(w2 + place(c));
            s1 += d.sum();
            s2 += (d * sh[c]).sum();
            G[c] = kMeansFirst ? d : fma(V::all(r2), d, G[c]);
        }
        if (row + step < a.rows) load(row + step);
        if (w2) {
            both_sums(s1, s2);
            const float f = kMeansFirst ? -1.f : -r2;
            const V m1 = V::all(a.rms ? 0.f : f * mean(s1)), m2 = V::all(f * mean(s2));
#pragma unroll
            for (int c = 0; c < NCH; ++c) {
                G[c] = G[c] + fma(sh[c], m2, m1);
                if constexpr (kMeansFirst) G[c] = fma(V::all(r2), G[c], V::of(gs[c]));
            }
        } else if constexpr (kMeansFirst) {
#pragma unroll
            for (int c = 0; c < NCH; ++c) G[c] = V::of(gs[c]);
        }
        T *dh = static_cast<T *>(g.dh) + row * g.dh_stride, *dy = static_cast<T *>(g.dy) + row * g.dy_stride;
        s1 = s2 = 0.f;
#pragma unroll
        for (int c = 0; c < NCH; ++c) {
            if (in(c)) (V::all(a.alpha) * G[c]).put(dh + column(c));
            if (gate_rows) {
                V u = uh[c];
                if (w1) u = b1 ? fma(u, V::at(w1 + place(c)), V::at(b1 + place(c))) : u * V::at(w1 + place(c));
                u = u * G[c];
                if (in(c)) u.put(static_cast<T *>(g.dgate) + row * g.dgate_stride + column(c));
                G[c] = G[c] * V::of(gr[c]);
            }
            add_product(2, c, G[c], uh[c]);
            add(3, c, G[c]);
            if (gate) G[c] = G[c] * V::at(gate + place(c));
            if (w1) {
                G[c] = in(c) ? G[c] * V::at(w1 + place(c)) : V::all(0.f);
                s1 += G[c].sum();
                s2 += (G[c] * uh[c]).sum();
            } else if (in(c)) {
                G[c].put(dy + column(c));
            }
        }
        if (w1) {
            both_sums(s1, s2);
            const V m1 = V::all(a.rms ? 0.f : -mean(s1)), m2 = V::all(-mean(s2));
#pragma unroll
            for (int c = 0; c < NCH; ++c)
                if (in(c)) (V::all(r1) * (G[c] + fma(uh[c], m2, m1))).put(dy + column(c));
        }
    }
    float *out = p.partial + group * 4 * width;
    if constexpr (kShared) {
        __syncthreads();
        for (int c = i; c < 4 * width; c += TPR) out[c] = acc[c];
    } else {
#pragma unroll
        for (int k = 0; k < 4; ++k)
#pragma unroll
            for (int c = 0; c < NCH; ++c)
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    const int col = (c * TPR + i) * VEC + e;
                    if (col < width) out[k * width + col] = sum[k][c].v[e];
                }
    }
}

// The weights' gradients from the groups' sums: 32 columns by 32 strands of
// groups; each strand adds its groups in order, the strands in order after that.
// blockIdx.y: the pre norm's, or the post norm's and the gate's.
template <typename W>
__global__ void __launch_bounds__(1024) k_residual_reduce(const ResidualNormArgs p, int groups) {
    __shared__ float part[2][32][33];
    const sieve_residual_norm_args &a = p.a;
    const int lane = threadIdx.x & 31, strand = threadIdx.x >> 5;
    const int col = blockIdx.x * 32 + lane;
    const float *in = p.partial + (int64_t)blockIdx.y * 2 * a.width;
    float s = 0.f, t = 0.f;
    if (col < a.width)
#pragma unroll 4
        for (int b = strand; b < groups; b += 32) {
            s += in[(int64_t)b * 4 * a.width + col];
            t += in[(int64_t)b * 4 * a.width + a.width + col];
        }
    part[0][strand][lane] = s;
    part[1][strand][lane] = t;
    __syncthreads();
    if (strand > 0 || col >= a.width) return;
    s = t = 0.f;
#pragma unroll
    for (int k = 0; k < 32; ++k) {
        s += part[0][k][lane];
        t += part[1][k][lane];
    }
    auto put = [&](void *to, float v) {
        if (to) static_cast<W *>(to)[col] = from_f32<W>(v);
    };
    if (blockIdx.y == 0) {
        put(p.g.dweight, s);
        put(p.g.dbias, t);
        return;
    }
    const float gate = a.gate_kind == SIEVE_GATE_COLUMN ? to_f32<W>(static_cast<const W *>(a.gate)[col]) : 1.f;
    const float w = a.post_weight ? to_f32<W>(static_cast<const W *>(a.post_weight)[col]) : 1.f;
    const float b = a.post_bias ? to_f32<W>(static_cast<const W *>(a.post_bias)[col]) : 0.f;
    put(p.g.dpost_weight, gate * s);
    put(p.g.dpost_bias, gate * t);
    if (a.gate_kind == SIEVE_GATE_COLUMN) put(p.g.dgate, fmaf(w, s, b * t));
}

bool aligned(const void *p, size_t m) { return reinterpret_cast<uintptr_t>(p) % m == 0; }
// Whether everything can be moved 16 bytes of a row at a time (weights of
// another type move the same number of elements).
template <typename T>
bool wide(const ResidualNormArgs &p) {
    constexpr int v = 16 / sizeof(T);
    const sieve_residual_norm_args &a = p.a;
    auto rows = [&](const void *q, int64_t stride) { return !q || (stride % v == 0 && aligned(q, 16)); };
    if (a.width % v) return false;
    for (const void *w : {a.weight, a.bias, a.post_weight, a.post_bias,
                          a.gate_kind == SIEVE_GATE_COLUMN ? a.gate : nullptr})
        if (!aligned(w, 16)) return false;
    const bool row_gate = a.gate_kind == SIEVE_GATE_ROW;
    return rows(a.h, a.h_stride) && rows(a.y, a.y_stride) && rows(row_gate ? a.gate : nullptr, a.gate_stride) &&
           rows(p.stream, p.stream_stride) && rows(p.x, p.x_stride) && rows(p.g.dstream, p.g.dstream_stride) &&
           rows(p.g.dx, p.g.dx_stride) && rows(p.g.dh, p.g.dh_stride) && rows(p.g.dy, p.g.dy_stride) &&
           rows(row_gate ? p.g.dgate : nullptr, p.g.dgate_stride);
}

template <typename T, typename W, int VEC, int TPR, int NCH>
cudaError_t forward_as(const ResidualNormArgs &p, cudaStream_t st) {
    constexpr int kRows = TPR == 32 ? 8 : 1;
    k_residual_norm<T, W, VEC, TPR, NCH><<<(unsigned)ceil_div(p.a.rows, kRows), TPR == 32 ? 256 : TPR, 0, st>>>(p);
    return cudaGetLastError();
}

template <typename T, typename W>
cudaError_t forward(const ResidualNormArgs &p, cudaStream_t st) {
    constexpr int V = 16 / sizeof(T);
    const int width = p.a.width;
    if (wide<T>(p)) {
        if (width <= 256) return forward_as<T, W, V, 32, 8 / V>(p, st);
        if (width <= 512) return forward_as<T, W, V, 32, 16 / V>(p, st);
        if (width <= 768) return forward_as<T, W, V, 32, 24 / V>(p, st);
        if (width <= 1024) return forward_as<T, W, V, 32, 32 / V>(p, st);
        if (width <= 2048) return forward_as<T, W, V, 128, 16 / V>(p, st);
        if (width <= 4096) return forward_as<T, W, V, 256, 16 / V>(p, st);
        return forward_as<T, W, V, 512, 16 / V>(p, st);
    }
    if (width <= 128) return forward_as<T, W, 1, 32, 4>(p, st);
    if (width <= 384) return forward_as<T, W, 1, 32, 12>(p, st);
    if (width <= 1024) return forward_as<T, W, 1, 128, 8>(p, st);
    if (width <= 2048) return forward_as<T, W, 1, 256, 8>(p, st);
    return forward_as<T, W, 1, 512, 16>(p, st);
}

// The backward pass' threads of a row and its blocks: 8 elements a thread where
// they move 16 bytes at a time, else 4 (one by one, 8 need more registers than
// there are), and 8 again past 4,096.
struct Plan {
    int tpr, elements, blocks, groups;
};
Plan plan(int64_t rows, int width, bool wide) {
    Plan p;
    p.elements = wide || width > 4096 ? 8 : 4;
    const int need = (width + p.elements - 1) / p.elements;
    p.tpr = need <= 32 ? 32 : need <= 64 ? 64 : need <= 96 ? 96 : need <= 128 ? 128 : need <= 256 ? 256 : need <= 512 ? 512 : 1024;
    const int64_t n = ceil_div(rows, groups_of(p.tpr)), most = 152 * blocks_per_sm(p.tpr, p.elements);
    p.blocks = (int)(n < most ? n : most);
    p.groups = p.blocks * groups_of(p.tpr);
    return p;
}

template <typename T, typename W, int VEC, int TPR, int ELEMENTS>
cudaError_t backward_as(const ResidualNormArgs &p, int blocks, cudaStream_t st) {
    constexpr bool kShared = TPR == 1024;
    auto kernel = k_residual_norm_backward<T, W, VEC, TPR, ELEMENTS / VEC, kShared>;
    size_t smem = 0;
    if (kShared) {
        cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                             4 * SIEVE_RESIDUAL_NORM_MAX_WIDTH * (int)sizeof(float));
        if (e != cudaSuccess) return e;
        smem = (size_t)4 * p.a.width * sizeof(float);
    }
    kernel<<<blocks, TPR == 32 ? 32 * kWarpRows : TPR, smem, st>>>(p);
    return cudaGetLastError();
}

template <typename T, typename W, int VEC, int ELEMENTS>
cudaError_t backward_by_width(const ResidualNormArgs &p, const Plan &q, cudaStream_t st) {
    switch (q.tpr) {
        case 32: return backward_as<T, W, VEC, 32, ELEMENTS>(p, q.blocks, st);
        case 64: return backward_as<T, W, VEC, 64, ELEMENTS>(p, q.blocks, st);
        case 96: return backward_as<T, W, VEC, 96, ELEMENTS>(p, q.blocks, st);
        case 128: return backward_as<T, W, VEC, 128, ELEMENTS>(p, q.blocks, st);
        case 256: return backward_as<T, W, VEC, 256, ELEMENTS>(p, q.blocks, st);
        case 512: return backward_as<T, W, VEC, 512, ELEMENTS>(p, q.blocks, st);
        default: return backward_as<T, W, VEC, 1024, ELEMENTS>(p, q.blocks, st);
    }
}

template <typename T, typename W>
cudaError_t backward(const ResidualNormArgs &p, cudaStream_t st) {
    const bool w = wide<T>(p);
    const Plan q = plan(p.a.rows, p.a.width, w);
    if (q.blocks > 0) {
        const cudaError_t e = w ? backward_by_width<T, W, 16 / sizeof(T), 8>(p, q, st)
                              : q.elements == 4 ? backward_by_width<T, W, 1, 4>(p, q, st)
                                                : backward_as<T, W, 1, 1024, 8>(p, q.blocks, st);
        if (e != cudaSuccess) return e;
    }
    const dim3 grid((unsigned)ceil_div(p.a.width, 32), 2);
    k_residual_reduce<W><<<grid, 1024, 0, st>>>(p, q.groups);
    return cudaGetLastError();
}

template <typename F>
cudaError_t by_type(int dtype, int wtype, F f) {
    if (dtype == SIEVE_F32) return f(float{}, float{});
    if (dtype == SIEVE_F16) return wtype == SIEVE_F32 ? f(__half{}, float{}) : f(__half{}, __half{});
    return wtype == SIEVE_F32 ? f(__nv_bfloat16{}, float{}) : f(__nv_bfloat16{}, __nv_bfloat16{});
}

}  // namespace

cudaError_t launch_residual_norm(const ResidualNormArgs &p, cudaStream_t st) {
    return by_type(p.a.dtype, p.a.weight_dtype,
                   [&](auto t, auto w) { return forward<decltype(t), decltype(w)>(p, st); });
}
cudaError_t launch_residual_norm_backward(const ResidualNormArgs &args, cudaStream_t st) {
    ResidualNormArgs p = args;
    const double inverse = 1.0 / p.a.width;
    p.inv_width = (float)inverse;
    p.inv_width_rest = (float)(inverse - p.inv_width);
    return by_type(p.a.dtype, p.a.weight_dtype,
                   [&](auto t, auto w) { return backward<decltype(t), decltype(w)>(p, st); });
}
size_t residual_norm_backward_workspace_bytes(int64_t rows, int width) {
    const int64_t a = plan(rows, width, true).groups, b = plan(rows, width, false).groups;
    return (size_t)round_up((a > b ? a : b) * 4 * width * (int64_t)sizeof(float) + 256, 256);
}

}  // namespace enc
}  // namespace sieve
