// attention_fwd.cu -- attention over packed documents, forward.
//
// A block takes one tile of 128 queries of one head and walks the document's
// keys in tiles of 128:
//   S = Q K^T      tcgen05, both operands from shared memory, fp32 in tensor
//                  memory (a thread's lane is its query)
//   P = 2^(S c + bias - m), the running maximum m and sum l of a row in
//                  registers of its thread; P rounded to 16 bits into tensor
//                  memory
//   O += P V       tcgen05, P from tensor memory
// The maximum that P is taken against is raised only when a row's grows by
// more than 2^8 (its sum uses the same one, so the result is the same softmax;
// P stays below 2^8, exact in scale): then the thread rescales its row of O.
//
// Warps 0-3: softmax and epilogue; warp 4: TMA loads; warp 5: products.  Two
// blocks share an SM (256 tensor-memory columns each): one's products run
// under the other's softmax.
//
// Where every document has a few new queries against many keys, a block takes
// the rows of all heads that share a key head (up to 128) over one chunk of
// the keys, and k_attend_join adds the chunks up.
#include <cstring>

#include "attention.cuh"

namespace sieve {
namespace enc {
namespace {

constexpr int kSoftmaxWarps = 4;
constexpr int kThreads = (kSoftmaxWarps + 2) * 32;
constexpr int kBlocksPerSm = 2;
constexpr uint32_t kTmemCols = 256;
constexpr float kRaise = 8.f;
// Tiles of K and of V held at a time.  With one, the next K loads under the
// softmax of this one and the next V under the scores of the next: that is
// enough, and at 128 columns it lets two blocks share an SM.
__host__ __device__ constexpr int stages(int dp) { return dp == 64 ? 2 : 1; }

struct FwdArgs {
    AttentionArgs p;
    CUtensorMap q, k, v;
    int pack;            // heads of one key head in a tile (1: a tile is 128 queries of one head)
    int rows_per_doc;    // split: new_tokens * pack
    int chunk;           // split: keys per block
    int doc_tiles;       // new_tokens > 0, not split: tiles of a document
    int bias_stride;     // floats between the bias tables of packed heads
    float *part_o;       // split: [chunk number][head groups][rows][head_dim]
    float2 *part_ml;     // split: [chunk number][head groups][rows]: maximum (base 2), sum
};

template <typename T, int DP, bool BIAS, bool SPLIT>
__global__ void __launch_bounds__(kThreads, kBlocksPerSm) k_attend(const __grid_constant__ FwdArgs f) {
    constexpr int kB = DP / 64;                       // column blocks of a tile
    constexpr int kStages = stages(DP);
    constexpr uint32_t kTileBytes = kB * kBlockBytes;
    // tensor memory: S, P and O; with 64 columns of O the three fit side by
    // side and S of the next tile is computed while P is made, else P takes
    // the place of S
    constexpr bool kApart = DP == 64;
    constexpr uint32_t kPCol = kApart ? 128 : 0, kOCol = kApart ? 192 : 128;
    extern __shared__ unsigned char smem_raw[];
    __shared__ __align__(8) uint64_t q_full, k_full[kStages], k_empty[kStages], v_full[kStages], v_empty[kStages],
        s_full, s_free, p_full, o_full, drained;
    __shared__ uint32_t tmem_slot;
    __shared__ int s_abort;
    const sieve_attention_args &a = f.p.a;
    const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0), lane = lane_id();

    if (blockIdx.x == 0 && threadIdx.x == 0) f.p.ctl->status = 0;
    // ---- the block's work
    const int groups = a.heads / f.pack;               // tiles' heads
    const int t = blockIdx.x / groups, hg = blockIdx.x % groups;
    int s, k_first, k_end, row0, rows;                 // key range, first query of the tile, rows used
    Doc doc;
    if (SPLIT) {
        s = find_doc(a.k_offsets, (int)a.nseq, (int)a.k_tokens, f.chunk, t);
        doc = doc_at(a, s);
        k_first = (t - first_tile(a.k_offsets, s, (int)a.k_tokens, f.chunk)) * f.chunk;
        if (k_first < 0 || k_first >= doc.nk) return;
        k_end = min(doc.nk, k_first + f.chunk);
        row0 = 0;
        rows = f.rows_per_doc;
    } else {
        int tile;
        if (a.new_tokens > 0) {
            s = t / f.doc_tiles;
            tile = t % f.doc_tiles;
        } else {
            s = find_doc(a.q_offsets, (int)a.nseq, (int)a.q_tokens, kTile, t);
            tile = t - first_tile(a.q_offsets, s, (int)a.q_tokens, kTile);
        }
        doc = doc_at(a, s);
        const int tiles = (int)ceil_div(doc.nq, kTile);
        if (tile < 0 || tile >= tiles) return;
        row0 = (tiles - 1 - tile) * kTile;             // the tiles that see most keys first
        rows = min(kTile, doc.nq - row0);
        k_first = 0;
        k_end = doc.nk;
    }
    const int shift = doc.nk - doc.nq;                 // place of query 0
    if (a.causal) k_end = min(k_end, (SPLIT ? doc.nq : row0 + rows) + shift);
    const int n_tiles = k_end > k_first ? (k_end - k_first + kTile - 1) / kTile : 0;
    const int head0 = hg * f.pack, hk = head0 / (a.heads / a.kv_heads);

    unsigned char *base = reinterpret_cast<unsigned char *>(
        (reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~static_cast<uintptr_t>(1023));
    unsigned char *q_tile = base, *k_tiles = base + kTileBytes, *v_tiles = k_tiles + kStages * kTileBytes;
    float *bias = reinterpret_cast<float *>(v_tiles + kStages * kTileBytes);

    if (threadIdx.x == 0) {
        tc::mbar_init(&q_full, 1);
        for (int i = 0; i < kStages; ++i) {
            tc::mbar_init(&k_full[i], 1);
            tc::mbar_init(&k_empty[i], 1);
            tc::mbar_init(&v_full[i], 1);
            tc::mbar_init(&v_empty[i], 1);
        }
        tc::mbar_init(&s_full, 1);
        tc::mbar_init(&s_free, kSoftmaxWarps * 32);
        tc::mbar_init(&p_full, kSoftmaxWarps * 32);
        tc::mbar_init(&o_full, 1);
        tc::mbar_init(&drained, 1);
        s_abort = 0;
        tc::mbar_init_fence();
    }
    if (warp == 5) tc::tmem_alloc(&tmem_slot, kTmemCols);
    if (BIAS)
        for (int h = 0; h < f.pack; ++h)
            for (int i = threadIdx.x; i < bias_entries(a.reach); i += kThreads)
                bias[h * f.bias_stride + i] = a.table ? scaled_bias(a, i - a.reach - kPad, head0 + h) : 0.f;
    tc::fence_before_sync();
    __syncthreads();
    tc::fence_after_sync();
    const uint32_t tmem = __shfl_sync(0xffffffffu, tmem_slot, 0);
    const Waiter wait{&s_abort, &f.p.ctl->status};

    if (warp == 4) {
        // ---------------- loads ----------------
        const uint32_t lead = lane == 0;
        bool ok = n_tiles > 0;
        int k_issued = 0, v_issued = 0;
        if (lane == 0) {
            prefetch_map(&f.q);
            prefetch_map(&f.k);
            prefetch_map(&f.v);
        }
        if (ok) {
            tc::mbar_arrive_expect_tx(lead, &q_full, kB * 128u * (uint32_t)(f.pack * (kTile / f.pack)));
            for (int b = 0; b < kB; ++b)
                tma_load(lead, q_tile + b * kBlockBytes, &f.q, 64 * b, head0, doc.q0 + row0, &q_full);
        }
        for (int j = 0; ok && j < n_tiles; ++j) {
            const int st = j % kStages;
            const uint32_t ph = (uint32_t)(j / kStages) & 1u;
            const int row = doc.k0 + k_first + j * kTile;
            if (!(ok = wait.warp(&k_empty[st], ph ^ 1u))) break;
            tc::mbar_arrive_expect_tx(lead, &k_full[st], kTileBytes);
            for (int b = 0; b < kB; ++b)
                tma_load(lead, k_tiles + st * kTileBytes + b * kBlockBytes, &f.k, 64 * b, hk, row, &k_full[st]);
            k_issued = j + 1;
            if (!(ok = wait.warp(&v_empty[st], ph ^ 1u))) break;
            tc::mbar_arrive_expect_tx(lead, &v_full[st], kTileBytes);
            for (int b = 0; b < kB; ++b)
                tma_load(lead, v_tiles + st * kTileBytes + b * kBlockBytes, &f.v, 64 * b, hk, row, &v_full[st]);
            v_issued = j + 1;
        }
        if (!ok && n_tiles > 0) {
            // after an abort: the copies in flight land before the block ends
            auto landed = [&](uint64_t *bar, uint32_t parity) {
                for (uint32_t it = 0; it < kPolls; ++it)
                    if (tc::mbar_try_wait(bar, parity)) return;
            };
            landed(&q_full, 0);
            for (int j = max(0, k_issued - kStages); j < k_issued; ++j)
                landed(&k_full[j % kStages], (uint32_t)(j / kStages) & 1u);
            for (int j = max(0, v_issued - kStages); j < v_issued; ++j)
                landed(&v_full[j % kStages], (uint32_t)(j / kStages) & 1u);
        }
    } else if (warp == 5) {
        // ---------------- products ----------------
        const uint32_t lead = lane == 0;
        constexpr uint32_t id_s = idesc<T>(kTile, false), id_o = idesc<T>(DP, true);
        const uint32_t qa = tc::smem_u32(q_tile);
        bool ok = n_tiles > 0;
        auto score = [&](int j) {
            const int st = j % kStages;
            if (!wait.warp(&k_full[st], (uint32_t)(j / kStages) & 1u)) return false;
            tc::fence_after_sync();
            mma_kk<DP>(lead, tmem, qa, tc::smem_u32(k_tiles + st * kTileBytes), id_s);
            tc::mma_commit(lead, &k_empty[st]);
            tc::mma_commit(lead, &s_full);
            return true;
        };
        if (ok) ok = wait.warp(&q_full, 0) && score(0);
        for (int j = 0; ok && j < n_tiles; ++j) {
            const int st = j % kStages;
            if (kApart && j + 1 < n_tiles) {
                if (!(ok = wait.warp(&s_free, (uint32_t)j & 1u))) break;
                if (!(ok = score(j + 1))) break;
            }
            if (!(ok = wait.warp(&v_full[st], (uint32_t)(j / kStages) & 1u))) break;
            const int left = doc.nk - (k_first + j * kTile);     // keys of the document from this tile on
            if (left < kTile) clear_rows(v_tiles + st * kTileBytes, left, kB);
            if (!(ok = wait.warp(&p_full, (uint32_t)j & 1u))) break;
            tc::fence_after_sync();
            mma_tn(lead, tmem + kOCol, tmem + kPCol, tc::smem_u32(v_tiles + st * kTileBytes), id_o, j > 0);
            tc::mma_commit(lead, &v_empty[st]);
            tc::mma_commit(lead, &o_full);
            if (!kApart && j + 1 < n_tiles) ok = score(j + 1);
        }
        // every product issued ends before the block frees its memory (waited
        // for even after an abort, within the poll limit)
        tc::mma_commit(lead, &drained);
        for (uint32_t it = 0; it < kPolls; ++it)
            if (tc::mbar_try_wait(&drained, 0)) break;
        __syncwarp();
    } else {
        // ---------------- softmax and epilogue ----------------
        const int r = warp * 32 + lane;
        const bool live = r < rows;
        const int qi = row0 + (SPLIT ? r / f.pack : r);          // query of the document
        const int head = head0 + (SPLIT ? r % f.pack : 0);
        const int place = qi + shift;
        // keys that this row sees, counted from k_first
        const int seen = live ? (a.causal ? min(doc.nk, place + 1) : doc.nk) - k_first : 0;
        const float c = a.scale * kLog2e;
        const uint32_t lane_base = tmem + ((uint32_t)(warp * 32) << 16);
        // the warp's places, for the distances that a chunk of keys can have
        int place_lo = live ? place : INT32_MAX, place_hi = live ? place : INT32_MIN;
        if (BIAS) {
#pragma unroll
            for (int o = 16; o; o >>= 1) {
                place_lo = min(place_lo, __shfl_xor_sync(0xffffffffu, place_lo, o));
                place_hi = max(place_hi, __shfl_xor_sync(0xffffffffu, place_hi, o));
            }
        }
        const float *lut = bias + (SPLIT && live ? head - head0 : 0) * f.bias_stride + a.reach + kPad;
        const float bias_before = BIAS ? lut[-a.reach] : 0.f, bias_after = BIAS ? lut[a.reach] : 0.f;
        float m = -INFINITY, l = 0.f;
        bool ok = true;
        for (int j = 0; j < n_tiles; ++j) {
            if (!(ok = wait.warp(&s_full, (uint32_t)j & 1u))) break;
            tc::fence_after_sync();
            uint32_t raw[4][32];
#pragma unroll
            for (int i = 0; i < 4; ++i) tc::tmem_ld32_issue(lane_base + 32 * i, raw[i]);
#pragma unroll
            for (int i = 0; i < 4; ++i) tc::tmem_ld_wait(raw[i]);
            if (kApart) {
                tc::fence_before_sync();
                tc::mbar_arrive(&s_free);
            }
            float x[4][32];
            const int key0 = k_first + j * kTile;                // key of the document in column 0
            float top = -INFINITY;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (BIAS) {
                    const int d0 = key0 + 32 * i;                // distances d0 - place + 0 .. 31
                    if (d0 - place_hi >= a.reach) {
#pragma unroll
                        for (int e = 0; e < 32; ++e) x[i][e] = fmaf(__uint_as_float(raw[i][e]), c, bias_after);
                    } else if (d0 + 31 - place_lo <= -a.reach) {
#pragma unroll
                        for (int e = 0; e < 32; ++e) x[i][e] = fmaf(__uint_as_float(raw[i][e]), c, bias_before);
                    } else {
                        const float *at = lut + (live ? d0 - place : 0);
#pragma unroll
                        for (int e = 0; e < 32; ++e) x[i][e] = fmaf(__uint_as_float(raw[i][e]), c, at[e]);
                    }
                } else {
#pragma unroll
                    for (int e = 0; e < 32; ++e) x[i][e] = __uint_as_float(raw[i][e]) * c;
                }
            }
            const int vis = seen - j * kTile;                    // columns that this row sees
            if (!__all_sync(0xffffffffu, vis >= kTile)) {
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int e = 0; e < 32; ++e)
                        if (32 * i + e >= vis) x[i][e] = -INFINITY;
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) top = fmaxf(top, max_of_32(x[i]));
            const bool raise = top > m + kRaise || m == -INFINITY;
            if (j > 0) {
                // the last tile's product is done with P (and O) before they
                // are written
                if (!(ok = wait.warp(&o_full, (uint32_t)(j - 1) & 1u))) break;
                tc::fence_after_sync();
            }
            if (j == 0) {
                m = top;
            } else if (__any_sync(0xffffffffu, raise)) {
                const float old = m;
                if (raise) m = fmaxf(top, m);
                const float scale = raise && old != m ? exp2_approx(old - (m == -INFINITY ? 0.f : m)) : 1.f;
                l *= scale;
#pragma unroll
                for (int i = 0; i < DP / 32; ++i) {
                    float o[32];
                    tc::tmem_ld32(lane_base + kOCol + 32 * i, o);
                    uint32_t w[32];
#pragma unroll
                    for (int e = 0; e < 32; ++e) w[e] = __float_as_uint(o[e] * scale);
                    tmem_st32(lane_base + kOCol + 32 * i, w);
                }
            }
            const float sub = m == -INFINITY ? 0.f : m;
            float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                uint32_t w[32];
#pragma unroll
                for (int e = 0; e < 32; ++e) {
                    const float p0 = exp2_approx(x[2 * i + e / 16][2 * (e % 16)] - sub);
                    const float p1 = exp2_approx(x[2 * i + e / 16][2 * (e % 16) + 1] - sub);
                    sum[e & 3] += p0 + p1;
                    w[e] = pack2<T>(p0, p1);
                }
                tmem_st32(lane_base + kPCol + 32 * i, w);
            }
            l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
            tc::tmem_st_wait();
            tc::fence_before_sync();
            tc::mbar_arrive(&p_full);
        }
        if (ok && n_tiles > 0) ok = wait.warp(&o_full, (uint32_t)(n_tiles - 1) & 1u);
        if (ok) {
            tc::fence_after_sync();
            const int d = a.head_dim;
            if (SPLIT) {
                const int64_t at = ((int64_t)t * groups + hg) * f.rows_per_doc + r;
                if (live) f.part_ml[at] = make_float2(m, l);
#pragma unroll
                for (int i = 0; i < DP / 32; ++i) {
                    float o[32];
                    if (n_tiles > 0) tc::tmem_ld32(lane_base + kOCol + 32 * i, o);
                    if (live)
#pragma unroll
                        for (int e = 0; e < 32; e += 4)
                            if (32 * i + e < d)
                                *reinterpret_cast<float4 *>(f.part_o + at * d + 32 * i + e) =
                                    n_tiles > 0 ? make_float4(o[e], o[e + 1], o[e + 2], o[e + 3])
                                                : make_float4(0.f, 0.f, 0.f, 0.f);
                }
            } else {
                const float inv = 1.f / l;
                const bool none = n_tiles == 0 || l == 0.f;
                const int64_t row = doc.q0 + qi;
                T *out = static_cast<T *>(f.p.out) + (row * a.heads + head) * d;
                if (live) f.p.lse[(int64_t)head * a.q_tokens + row] = none ? -INFINITY : m * kLn2 + logf(l);
#pragma unroll
                for (int i = 0; i < DP / 32; ++i) {
                    float o[32];
                    if (n_tiles > 0) tc::tmem_ld32(lane_base + kOCol + 32 * i, o);
                    if (live)
#pragma unroll
                        for (int e = 0; e < 32; e += 8)
                            if (32 * i + e < d) {
                                float v[8];
#pragma unroll
                                for (int u = 0; u < 8; ++u) v[u] = none ? 0.f : o[e + u] * inv;
                                store_vec<T, 8>(out + 32 * i + e, v);
                            }
                }
            }
        }
    }
    tc::fence_before_sync();
    __syncthreads();
    if (warp == 5) {
        tc::fence_after_sync();
        tc::tmem_dealloc(tmem, kTmemCols);
    }
}

// The chunks of a document joined: a warp per query and head.
template <typename T>
__global__ void __launch_bounds__(128) k_attend_join(const __grid_constant__ FwdArgs f) {
    const sieve_attention_args &a = f.p.a;
    const int64_t w = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 5);
    if (w >= a.q_tokens * a.heads) return;
    const int lane = lane_id(), d = a.head_dim, groups = a.heads / f.pack;
    const int64_t row = w / a.heads;
    const int head = (int)(w % a.heads), s = (int)(row / a.new_tokens), qi = (int)(row % a.new_tokens);
    const Doc doc = doc_at(a, s);
    const int t0 = first_tile(a.k_offsets, s, (int)a.k_tokens, f.chunk), n = (int)ceil_div(doc.nk, f.chunk);
    const int r = qi * f.pack + head % f.pack;
    auto slot = [&](int i) { return ((int64_t)(t0 + i) * groups + head / f.pack) * f.rows_per_doc + r; };
    float top = -INFINITY;
    for (int i = lane; i < n; i += 32) top = fmaxf(top, f.part_ml[slot(i)].x);
#pragma unroll
    for (int o = 16; o; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
    const float base = top == -INFINITY ? 0.f : top;
    float l = 0.f, acc[4] = {0.f, 0.f, 0.f, 0.f};
    for (int i = 0; i < n; ++i) {
        const int64_t at = slot(i);
        const float2 ml = f.part_ml[at];
        const float e = exp2_approx(ml.x - base);
        l = fmaf(ml.y, e, l);
        if (4 * lane < d && ml.y != 0.f) {
            const float4 o = *reinterpret_cast<const float4 *>(f.part_o + at * d + 4 * lane);
            acc[0] = fmaf(o.x, e, acc[0]);
            acc[1] = fmaf(o.y, e, acc[1]);
            acc[2] = fmaf(o.z, e, acc[2]);
            acc[3] = fmaf(o.w, e, acc[3]);
        }
    }
    if (lane == 0) f.p.lse[(int64_t)head * a.q_tokens + row] = l == 0.f ? -INFINITY : top * kLn2 + logf(l);
    if (4 * lane < d) {
        const float inv = l == 0.f ? 0.f : 1.f / l;
        uint2 o;
        o.x = pack2<T>(acc[0] * inv, acc[1] * inv);
        o.y = pack2<T>(acc[2] * inv, acc[3] * inv);
        *reinterpret_cast<uint2 *>(static_cast<T *>(f.p.out) + w * d + 4 * lane) = o;
    }
}

// How a call runs: packed over chunks of keys where the queries of every
// document and of a key head's heads fit one tile together.
struct Shape {
    bool split;
    int pack, chunk;
    int64_t blocks, chunks;
    size_t smem;
};

constexpr int kMaxBiasBytes = 24 * 1024;

Shape shape_of(const sieve_attention_args &a) {
    Shape s = {};
    const int dp = a.head_dim <= 64 ? 64 : 128, share = a.heads / a.kv_heads;
    const int bias_bytes = a.num_buckets || a.scale < 0.f ? bias_entries(a.reach) * 4 : 0;
    s.pack = 1;
    if (a.new_tokens > 0 && a.new_tokens <= kTile) {
        s.split = true;
        for (int p = 1; p <= share; ++p)
            if (share % p == 0 && p * a.new_tokens <= kTile && p * bias_bytes <= kMaxBiasBytes) s.pack = p;
        // chunks: about two rounds of blocks, no fewer than two tiles each
        const int64_t want = a.k_tokens * (a.heads / s.pack) / (2 * 152 * kBlocksPerSm);
        s.chunk = (int)(round_up(want < 2 * kTile ? 2 * kTile : want, kTile));
        s.chunks = doc_tiles(a.k_tokens, a.nseq, s.chunk);
        s.blocks = s.chunks * (a.heads / s.pack);
    } else if (a.new_tokens > 0) {
        s.blocks = a.nseq * ceil_div(a.new_tokens, kTile) * a.heads;
    } else {
        s.blocks = doc_tiles(a.q_tokens, a.nseq, kTile) * a.heads;
    }
    s.smem = 1024 + (size_t)(1 + 2 * stages(dp)) * (dp / 64) * kBlockBytes + (size_t)s.pack * bias_bytes;
    return s;
}

size_t part_floats(const sieve_attention_args &a, const Shape &s) {
    return (size_t)s.blocks * a.new_tokens * s.pack;   // rows of all blocks
}

template <typename T, int DP, bool BIAS, bool SPLIT>
cudaError_t run(const FwdArgs &f, const Shape &s, cudaStream_t st) {
    auto kernel = k_attend<T, DP, BIAS, SPLIT>;
    cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)s.smem);
    if (e != cudaSuccess) return e;
    kernel<<<(unsigned)s.blocks, kThreads, s.smem, st>>>(f);
    if ((e = cudaGetLastError()) != cudaSuccess || !SPLIT) return e;
    k_attend_join<T><<<(unsigned)ceil_div(f.p.a.q_tokens * f.p.a.heads, 4), 128, 0, st>>>(f);
    return cudaGetLastError();
}

template <typename T, int DP>
cudaError_t by_shape(const FwdArgs &f, const Shape &s, cudaStream_t st) {
    // a negative scale turns the order of the raw scores around: the biased
    // form, which compares finished scores, takes it (with a bias of zero)
    const bool biased = f.p.a.num_buckets || f.p.a.scale < 0.f;
    if (s.split) return biased ? run<T, DP, true, true>(f, s, st) : run<T, DP, false, true>(f, s, st);
    return biased ? run<T, DP, true, false>(f, s, st) : run<T, DP, false, false>(f, s, st);
}

}  // namespace

size_t attention_workspace_bytes(const sieve_attention_args &a) {
    const Shape s = shape_of(a);
    if (!s.split) return kCtlBytes;
    return kCtlBytes + (size_t)round_up((int64_t)(part_floats(a, s) * (a.head_dim + 2) * sizeof(float)), 256);
}

sieve_status launch_attention_forward(const AttentionArgs &p, void *ws, cudaStream_t st) {
    const sieve_attention_args &a = p.a;
    const Shape s = shape_of(a);
    FwdArgs f;
    std::memset(&f, 0, sizeof f);
    f.p = p;
    f.p.ctl = static_cast<EncCtl *>(ws);
    f.pack = s.pack;
    f.rows_per_doc = a.new_tokens * s.pack;
    f.chunk = s.chunk;
    f.doc_tiles = a.new_tokens > 0 ? (int)ceil_div(a.new_tokens, kTile) : 0;
    f.bias_stride = bias_entries(a.reach);
    f.part_o = reinterpret_cast<float *>(static_cast<unsigned char *>(ws) + kCtlBytes);
    f.part_ml = reinterpret_cast<float2 *>(f.part_o + (s.split ? part_floats(a, s) * a.head_dim : 0));
    sieve_status rc = make_map(&f.q, a.dtype, a.q, a.head_dim, a.heads, a.q_tokens, a.q_token_stride,
                               a.q_head_stride, s.pack, kTile / s.pack);
    if (rc != SIEVE_OK) return rc;
    if (a.k_tokens > 0) {
        rc = make_map(&f.k, a.dtype, a.k, a.head_dim, a.kv_heads, a.k_tokens, a.k_token_stride, a.k_head_stride, 1,
                      kTile);
        if (rc == SIEVE_OK)
            rc = make_map(&f.v, a.dtype, a.v, a.head_dim, a.kv_heads, a.k_tokens, a.v_token_stride, a.v_head_stride,
                          1, kTile);
        if (rc != SIEVE_OK) return rc;
    }
    const bool wide = a.head_dim > 64;
    cudaError_t e;
    if (a.dtype == SIEVE_F16) e = wide ? by_shape<__half, 128>(f, s, st) : by_shape<__half, 64>(f, s, st);
    else e = wide ? by_shape<__nv_bfloat16, 128>(f, s, st) : by_shape<__nv_bfloat16, 64>(f, s, st);
    return e == cudaSuccess ? SIEVE_OK : record_cuda_error(e);
}

sieve_status make_map(CUtensorMap *map, int dtype, const void *base, int head_dim, int heads, int64_t tokens,
                      int64_t token_stride, int64_t head_stride, int box_heads, int box_tokens) {
    using Encode = CUresult (*)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *,
                                const cuuint64_t *, const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave,
                                CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
    static Encode encode = nullptr;   // the driver's function; the same whoever finds it first
    if (!encode) {
        void *fn = nullptr;
        cudaDriverEntryPointQueryResult found;
        const cudaError_t e =
            cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &fn, 12000, cudaEnableDefault, &found);
        if (e != cudaSuccess) return record_cuda_error(e);
        if (found != cudaDriverEntryPointSuccess || !fn) return SIEVE_EUNSUPPORTED;
        encode = reinterpret_cast<Encode>(fn);
    }
    const cuuint64_t dims[3] = {(cuuint64_t)head_dim, (cuuint64_t)heads, (cuuint64_t)tokens};
    // an axis of one element has no stride that matters
    const cuuint64_t strides[2] = {(cuuint64_t)(heads > 1 ? head_stride : head_dim) * 2,
                                   (cuuint64_t)(tokens > 1 ? token_stride : (int64_t)heads * head_dim) * 2};
    const cuuint32_t box[3] = {64, (cuuint32_t)box_heads, (cuuint32_t)box_tokens}, step[3] = {1, 1, 1};
    const CUresult r = encode(
        map, dtype == SIEVE_F16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3,
        const_cast<void *>(base), dims, strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE,
        CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return r == CUDA_SUCCESS ? SIEVE_OK : SIEVE_EINVAL;
}

}  // namespace enc
}  // namespace sieve
