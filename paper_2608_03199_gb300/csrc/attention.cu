// attention.cu -- attention over packed documents with a relative position
// bias, backward: one warp per row, straight from the formulas.
#include "encoder.cuh"

namespace sieve {
namespace enc {
namespace {

constexpr int kWarps = 4;
constexpr int kMaxDim = SIEVE_ATTENTION_MAX_DIM;

struct Doc {
    int q0, nq, k0, nk;   // first rows and lengths
};
__device__ __forceinline__ Doc doc_at(const sieve_attention_args &a, int s) {
    Doc d;
    doc_range(a.k_offsets, s, (int)a.k_tokens, d.k0, d.nk);
    if (a.new_tokens > 0) {
        d.q0 = s * a.new_tokens;
        d.nq = a.new_tokens;
    } else {
        doc_range(a.q_offsets, s, (int)a.q_tokens, d.q0, d.nq);
    }
    return d;
}
__device__ __forceinline__ float bias_at(const sieve_attention_args &a, int dist, int head) {
    if (!a.table) return 0.f;
    const int b = __ldg(a.bucket_map + a.reach + min(max(dist, -a.reach), a.reach));
    return __ldg(a.table + min(max(b, 0), a.num_buckets - 1) * a.heads + head);
}

template <typename T>
__device__ __forceinline__ float dot_row(const float *q, const T *row, int d) {
    float s = 0.f;
    for (int c = 0; c < d; c += 8) {
        float v[8];
        load_vec<T, 8>(row + c, v);
#pragma unroll
        for (int e = 0; e < 8; ++e) s = fmaf(q[c + e], v[e], s);
    }
    return s;
}

// dq, delta and the table's gradient: a warp per query row and head.
template <typename T>
__global__ void __launch_bounds__(kWarps * 32) k_attend_dq(const AttentionArgs p) {
    __shared__ float qs[kWarps][kMaxDim], dos[kWarps][kMaxDim];
    const sieve_attention_args &a = p.a;
    if (blockIdx.x == 0 && threadIdx.x == 0) p.ctl->status = 0;
    const int warp = threadIdx.x >> 5, lane = lane_id();
    const int64_t w = (int64_t)blockIdx.x * kWarps + warp;
    if (w >= a.q_tokens * a.heads) return;
    const int t = (int)(w / a.heads), h = (int)(w % a.heads), hk = h / (a.heads / a.kv_heads);
    const int s = a.new_tokens > 0 ? t / a.new_tokens : doc_of_row(a.q_offsets, (int)a.nseq, t);
    const Doc doc = doc_at(a, s);
    const int i = t - doc.q0;
    if (i < 0 || i >= doc.nq) return;
    const int d = a.head_dim;
    const T *q = static_cast<const T *>(a.q) + t * a.q_token_stride + h * a.q_head_stride;
    const T *dout = static_cast<const T *>(p.dout) + w * d;
    for (int c = lane; c < d; c += 32) {
        qs[warp][c] = to_f32<T>(q[c]);
        dos[warp][c] = to_f32<T>(dout[c]);
    }
    __syncwarp();
    const int place = i + doc.nk - doc.nq;
    const int nk = a.causal ? min(doc.nk, place + 1) : doc.nk;
    const T *k = static_cast<const T *>(a.k) + doc.k0 * a.k_token_stride + hk * a.k_head_stride;
    const T *v = static_cast<const T *>(a.v) + doc.k0 * a.v_token_stride + hk * a.v_head_stride;
    const float lse = p.lse_in[(int64_t)h * a.q_tokens + t];
    float delta = 0.f, dq[kMaxDim / 32] = {}, row_sum[2] = {};   // buckets lane, lane + 32
    for (int pass = 0; pass < 2; ++pass) {
        float part = 0.f;
        for (int j0 = 0; j0 < nk; j0 += 32) {
            const int j = j0 + lane;
            float ds = 0.f;
            if (j < nk && lse > -INFINITY) {
                const float x =
                    fmaf(dot_row<T>(qs[warp], k + j * a.k_token_stride, d), a.scale, bias_at(a, j - place, h));
                const float pr = expf(x - lse), dp = dot_row<T>(dos[warp], v + j * a.v_token_stride, d);
                part = fmaf(pr, dp, part);
                ds = pr * (dp - delta);
            }
            if (pass == 0) continue;
            int b = -1;
            if (a.table && j < nk)
                b = min(max(a.bucket_map[a.reach + min(max(j - place, -a.reach), a.reach)], 0), a.num_buckets - 1);
            const int n = min(32, nk - j0);
            for (int jj = 0; jj < n; ++jj) {
                const float dj = __shfl_sync(0xffffffffu, ds, jj);
                const int bj = __shfl_sync(0xffffffffu, b, jj);
                if (bj == lane) row_sum[0] += dj;
                if (bj == lane + 32) row_sum[1] += dj;
#pragma unroll
                for (int c = 0; c < kMaxDim / 32; ++c)
                    if (c * 32 + lane < d)
                        dq[c] = fmaf(dj, to_f32<T>(k[(j0 + jj) * a.k_token_stride + c * 32 + lane]), dq[c]);
            }
        }
        if (pass == 0) delta = warp_sum(part);
    }
    T *o = static_cast<T *>(p.dq) + t * p.dq_ts + h * p.dq_hs;
#pragma unroll
    for (int c = 0; c < kMaxDim / 32; ++c)
        if (c * 32 + lane < d) o[c * 32 + lane] = from_f32<T>(dq[c] * a.scale);
    if (lane == 0) p.delta[(int64_t)h * a.q_tokens + t] = delta;
    if (a.table)
        for (int c = 0; c < 2; ++c)
            if (c * 32 + lane < a.num_buckets) p.row_sums[w * a.num_buckets + c * 32 + lane] = row_sum[c];
}

// The table's gradient: a block per bucket and head adds the rows' sums.
__global__ void __launch_bounds__(256) k_attend_dtable(const AttentionArgs p) {
    __shared__ float part[256];
    const sieve_attention_args &a = p.a;
    const int b = blockIdx.x, h = blockIdx.y, nb = a.num_buckets;
    const int32_t *off = a.new_tokens > 0 ? nullptr : a.q_offsets;
    const int lo = off ? min(max(off[0], 0), (int)a.q_tokens) : 0;
    const int hi = off ? min(max(off[a.nseq], lo), (int)a.q_tokens) : (int)a.q_tokens;
    float s = 0.f;
    for (int t = lo + threadIdx.x; t < hi; t += 256) s += p.row_sums[((int64_t)t * a.heads + h) * nb + b];
    part[threadIdx.x] = s;
    __syncthreads();
    if (threadIdx.x == 0) {
        s = 0.f;
        for (int i = 0; i < 256; ++i) s += part[i];
        p.dtable[b * a.heads + h] = s;
    }
}

// dk and dv: a warp per key row and key head.
template <typename T>
__global__ void __launch_bounds__(kWarps * 32) k_attend_dkv(const AttentionArgs p) {
    __shared__ float ks[kWarps][kMaxDim], vs[kWarps][kMaxDim];
    const sieve_attention_args &a = p.a;
    const int warp = threadIdx.x >> 5, lane = lane_id();
    const int64_t w = (int64_t)blockIdx.x * kWarps + warp;
    if (w >= a.k_tokens * a.kv_heads) return;
    const int t = (int)(w / a.kv_heads), hk = (int)(w % a.kv_heads), share = a.heads / a.kv_heads;
    const int s = doc_of_row(a.k_offsets, (int)a.nseq, t);
    const Doc doc = doc_at(a, s);
    const int j = t - doc.k0;
    if (j < 0 || j >= doc.nk) return;
    const int d = a.head_dim;
    const T *k = static_cast<const T *>(a.k) + t * a.k_token_stride + hk * a.k_head_stride;
    const T *v = static_cast<const T *>(a.v) + t * a.v_token_stride + hk * a.v_head_stride;
    for (int c = lane; c < d; c += 32) {
        ks[warp][c] = to_f32<T>(k[c]);
        vs[warp][c] = to_f32<T>(v[c]);
    }
    __syncwarp();
    float dk[kMaxDim / 32] = {}, dv[kMaxDim / 32] = {};
    const int shift = doc.nk - doc.nq;
    const int first = a.causal ? max(0, j - shift) : 0;   // the first query that sees this key
    for (int h = hk * share; h < (hk + 1) * share; ++h)
        for (int i0 = first; i0 < doc.nq; i0 += 32) {
            const int i = i0 + lane, row = doc.q0 + i;
            const T *q0 = static_cast<const T *>(a.q) + (doc.q0 + i0) * a.q_token_stride + h * a.q_head_stride;
            const T *do0 = static_cast<const T *>(p.dout) + ((int64_t)(doc.q0 + i0) * a.heads + h) * d;
            float pr = 0.f, ds = 0.f;
            if (i < doc.nq) {
                const float lse = p.lse_in[(int64_t)h * a.q_tokens + row];
                if (lse > -INFINITY) {
                    const float x = fmaf(dot_row<T>(ks[warp], q0 + lane * a.q_token_stride, d), a.scale,
                                         bias_at(a, j - i - shift, h));
                    pr = expf(x - lse);
                    ds = pr * (dot_row<T>(vs[warp], do0 + (int64_t)lane * a.heads * d, d) -
                               p.delta[(int64_t)h * a.q_tokens + row]);
                }
            }
            const int n = min(32, doc.nq - i0);
            for (int ii = 0; ii < n; ++ii) {
                const float pi = __shfl_sync(0xffffffffu, pr, ii), di = __shfl_sync(0xffffffffu, ds, ii);
#pragma unroll
                for (int c = 0; c < kMaxDim / 32; ++c)
                    if (c * 32 + lane < d) {
                        dv[c] = fmaf(pi, to_f32<T>(do0[(int64_t)ii * a.heads * d + c * 32 + lane]), dv[c]);
                        dk[c] = fmaf(di, to_f32<T>(q0[ii * a.q_token_stride + c * 32 + lane]), dk[c]);
                    }
            }
        }
    T *ok = static_cast<T *>(p.dk) + t * p.dk_ts + hk * p.dk_hs, *ov = static_cast<T *>(p.dv) + t * p.dv_ts + hk * p.dv_hs;
#pragma unroll
    for (int c = 0; c < kMaxDim / 32; ++c)
        if (c * 32 + lane < d) {
            ok[c * 32 + lane] = from_f32<T>(dk[c] * a.scale);
            ov[c * 32 + lane] = from_f32<T>(dv[c]);
        }
}

template <typename T>
cudaError_t backward(const AttentionArgs &p, cudaStream_t st) {
    cudaError_t e;
    if (p.a.q_tokens > 0) {
        k_attend_dq<T><<<(unsigned)ceil_div(p.a.q_tokens * p.a.heads, kWarps), kWarps * 32, 0, st>>>(p);
        if ((e = cudaGetLastError()) != cudaSuccess) return e;
    }
    if (p.a.table) {
        k_attend_dtable<<<dim3(p.a.num_buckets, p.a.heads), 256, 0, st>>>(p);
        if ((e = cudaGetLastError()) != cudaSuccess) return e;
    }
    if (p.a.k_tokens > 0) {
        k_attend_dkv<T><<<(unsigned)ceil_div(p.a.k_tokens * p.a.kv_heads, kWarps), kWarps * 32, 0, st>>>(p);
        e = cudaGetLastError();
        if (e != cudaSuccess) return e;
    }
    return cudaSuccess;
}

}  // namespace

size_t attention_backward_workspace_bytes(const sieve_attention_args &a) {
    // delta of every query row, and its sums of ds by bucket
    return kCtlBytes + (size_t)round_up((int64_t)a.heads * a.q_tokens * (1 + a.num_buckets) * (int64_t)sizeof(float), 256);
}

sieve_status launch_attention_backward(const AttentionArgs &p0, void *ws, cudaStream_t st) {
    AttentionArgs p = p0;
    p.ctl = static_cast<EncCtl *>(ws);
    p.delta = reinterpret_cast<float *>(static_cast<unsigned char *>(ws) + kCtlBytes);
    p.row_sums = p.delta + (int64_t)p.a.heads * p.a.q_tokens;
    const cudaError_t e = p.a.dtype == SIEVE_F16 ? backward<__half>(p, st) : backward<__nv_bfloat16>(p, st);
    return e == cudaSuccess ? SIEVE_OK : record_cuda_error(e);
}

}  // namespace enc
}  // namespace sieve
