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
// Warps 0-7 make P (two warps to the 32 lanes of a quarter, 64 columns each,
// so that a row's scores stay in registers); warp 8 loads and issues the
// products.  Two blocks share an SM (256 tensor-memory columns each): one's
// products run under the other's softmax.
//
// Where every document has a few new queries against many keys, a block takes
// the rows of all heads that share a key head (up to 128) over one chunk of
// the keys, and k_attend_join adds the chunks up.
#include <cstring>

#include "attention.cuh"

namespace sieve {
namespace enc {
namespace {

constexpr int kSoftmaxWarps = 8;
constexpr int kSoftmax = kSoftmaxWarps * 32;
constexpr int kThreads = kSoftmax + 32;
constexpr int kHalf = kTile / 2;
constexpr int kBlocksPerSm = 2;
constexpr uint32_t kTmemCols = 256;
constexpr float kRaise = 8.f;
// Tiles of K and of V held at a time.  With one, the next K loads under the
// softmax of this one and the next V under the scores of the next: that is
// enough, and at 128 columns it lets two blocks share an SM.
__host__ __device__ constexpr int stages(int dp) { return dp == 64 ? 2 : 1; }

// What the roles of a block need to know of its work.
struct Work {
    int q_row, rows, query0;      // first row of q, rows used, query of row 0
    int k_row, k_first, nk, n_tiles, shift;
};

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

template <bool SPLIT>
__device__ __forceinline__ Work find_work(const FwdArgs &f, int t) {
    const sieve_attention_args &a = f.p.a;
    Work w;
    w.n_tiles = -1;                                    // nothing to do
    int s, k_end;
    Doc doc;
    if (SPLIT) {
        s = find_doc(a.k_offsets, (int)a.nseq, (int)a.k_tokens, f.chunk, t);
        doc = doc_at(a, s);
        w.k_first = (t - first_tile(a.k_offsets, s, (int)a.k_tokens, f.chunk)) * f.chunk;
        if (w.k_first < 0 || w.k_first >= doc.nk) return w;
        k_end = min(doc.nk, w.k_first + f.chunk);
        w.query0 = 0;
        w.rows = f.rows_per_doc;
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
        if (tile < 0 || tile >= tiles) return w;
        w.query0 = (tiles - 1 - tile) * kTile;         // the tiles that see most keys first
        w.rows = min(kTile, doc.nq - w.query0);
        w.k_first = 0;
        k_end = doc.nk;
    }
    w.shift = doc.nk - doc.nq;                         // place of query 0
    w.nk = doc.nk;
    w.q_row = doc.q0 + w.query0;
    w.k_row = doc.k0 + w.k_first;
    if (a.causal) k_end = min(k_end, (SPLIT ? doc.nq : w.query0 + w.rows) + w.shift);
    w.n_tiles = k_end > w.k_first ? (k_end - w.k_first + kTile - 1) / kTile : 0;
    return w;
}

template <typename T, int DP, bool BIAS, bool SPLIT>
__global__ void __launch_bounds__(kThreads, kBlocksPerSm) k_attend(const __grid_constant__ FwdArgs f) {
    constexpr int kB = DP / 64;                       // column blocks of a tile
    constexpr int kStages = stages(DP);
    constexpr uint32_t kTileBytes = kB * kBlockBytes;
    // tensor memory: S, P and O; with 64 columns of O the three fit side by
    // side and S of the next tile is computed while P is made, else P takes
    // the place of S (each warp's half within its own columns)
    constexpr bool kApart = DP == 64;
    constexpr uint32_t kPCol = kApart ? 128 : 0, kPHalf = kApart ? 32 : 64, kOCol = kApart ? 192 : 128;
    extern __shared__ unsigned char smem_raw[];
    __shared__ __align__(8) uint64_t q_full, k_full[kStages], v_full[kStages], s_full, s_free, p_full, o_full, drained,
        pair_bar[4];
    __shared__ uint32_t tmem_slot;
    __shared__ int s_abort;
    __shared__ Work s_work;
    __shared__ float s_top[2][2][kTile];
    const sieve_attention_args &a = f.p.a;
    const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0), lane = lane_id();

    const int groups = a.heads / f.pack;               // a tile's heads
    const int t = blockIdx.x / groups, hg = blockIdx.x % groups;
    const int head0 = hg * f.pack, hk = head0 / (a.heads / a.kv_heads);
    unsigned char *base = reinterpret_cast<unsigned char *>(
        (reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~static_cast<uintptr_t>(1023));
    unsigned char *q_tile = base, *k_tiles = base + kTileBytes, *v_tiles = k_tiles + kStages * kTileBytes;
    float *bias = reinterpret_cast<float *>(v_tiles + kStages * kTileBytes);

    auto load_k = [&](const Work &w, int j) {
        const uint32_t lead = lane == 0;
        const int st = j % kStages;
        tc::mbar_arrive_expect_tx(lead, &k_full[st], kTileBytes);
        for (int b = 0; b < kB; ++b)
            tma_load(lead, k_tiles + st * kTileBytes + b * kBlockBytes, &f.k, 64 * b, hk, w.k_row + j * kTile, &k_full[st]);
    };
    auto load_v = [&](const Work &w, int j) {
        const uint32_t lead = lane == 0;
        const int st = j % kStages;
        tc::mbar_arrive_expect_tx(lead, &v_full[st], kTileBytes);
        for (int b = 0; b < kB; ++b)
            tma_load(lead, v_tiles + st * kTileBytes + b * kBlockBytes, &f.v, 64 * b, hk, w.k_row + j * kTile, &v_full[st]);
    };

    Work w;
    if (warp == kSoftmaxWarps) {
        // find the work and start its loads while the others set the block up
        if (lane == 0) {
            if (blockIdx.x == 0) f.p.ctl->status = 0;
            tc::mbar_init(&q_full, 1);
            for (int i = 0; i < kStages; ++i) {
                tc::mbar_init(&k_full[i], 1);
                tc::mbar_init(&v_full[i], 1);
            }
            tc::mbar_init(&s_full, 1);
            tc::mbar_init(&s_free, kSoftmax);
            tc::mbar_init(&p_full, kSoftmax);
            tc::mbar_init(&o_full, 1);
            tc::mbar_init(&drained, 1);
            for (int i = 0; i < 4; ++i) tc::mbar_init(&pair_bar[i], 64);
            s_abort = 0;
            tc::mbar_init_fence();
        }
        __syncwarp();
        w = find_work<SPLIT>(f, t);
        if (w.n_tiles > 0) {
            const uint32_t lead = lane == 0;
            tc::mbar_arrive_expect_tx(lead, &q_full, kB * 128u * (uint32_t)(f.pack * (kTile / f.pack)));
            for (int b = 0; b < kB; ++b) tma_load(lead, q_tile + b * kBlockBytes, &f.q, 64 * b, head0, w.q_row, &q_full);
            for (int j = 0; j < kStages && j < w.n_tiles; ++j) {
                load_k(w, j);
                load_v(w, j);
            }
        }
        if (lane == 0) s_work = w;
    } else {
        if (warp == 0) tc::tmem_alloc(&tmem_slot, kTmemCols);
        if (BIAS)
            for (int h = 0; h < f.pack; ++h)
                for (int i = threadIdx.x; i < bias_entries(a.reach); i += kSoftmax)
                    bias[h * f.bias_stride + i] = a.table ? scaled_bias(a, i - a.reach - kPad, head0 + h) : 0.f;
    }
    tc::fence_before_sync();
    __syncthreads();
    tc::fence_after_sync();
    const uint32_t tmem = __shfl_sync(0xffffffffu, tmem_slot, 0);
    const Waiter wait{&s_abort, &f.p.ctl->status};
    w = s_work;
    const int n_tiles = w.n_tiles;

    if (n_tiles < 0) {
        // a tile number that no document uses
    } else if (warp == kSoftmaxWarps) {
        // ---------------- loads and products ----------------
        const uint32_t lead = lane == 0;
        constexpr uint32_t id_s = idesc<T>(kTile, false), id_o = idesc<T>(DP, true);
        const uint32_t qa = tc::smem_u32(q_tile);
        int k_issued = min(kStages, n_tiles), v_issued = k_issued;
        bool ok = n_tiles > 0;
        auto score = [&](int j) {
            const int st = j % kStages;
            if (!wait.warp(&k_full[st], (uint32_t)(j / kStages) & 1u)) return false;
            tc::fence_after_sync();
            mma_kk<DP>(lead, tmem, qa, tc::smem_u32(k_tiles + st * kTileBytes), id_s);
            tc::mma_commit(lead, &s_full);
            return true;
        };
        if (ok) ok = wait.warp(&q_full, 0) && score(0);
        for (int j = 0; ok && j < n_tiles; ++j) {
            const int st = j % kStages;
            // the scores are in registers: so their product is done and its K
            // tile free
            if (!(ok = wait.warp(&s_free, (uint32_t)j & 1u))) break;
            if (j + kStages < n_tiles) {
                load_k(w, j + kStages);
                k_issued = j + kStages + 1;
            }
            if (kApart && j + 1 < n_tiles && !(ok = score(j + 1))) break;
            if (!(ok = wait.warp(&v_full[st], (uint32_t)(j / kStages) & 1u))) break;
            const int left = w.nk - (w.k_first + j * kTile);     // keys of the document from this tile on
            if (left < kTile) clear_rows(v_tiles + st * kTileBytes, left, kB);
            if (!(ok = wait.warp(&p_full, (uint32_t)j & 1u))) break;
            tc::fence_after_sync();
#pragma unroll
            for (int k = 0; k < kTile / 16; ++k)
                tc::mma_f16_ta(lead, tmem + kOCol, tmem + kPCol + (k / 4) * kPHalf + (k % 4) * 8,
                               desc_mn_sw128(tc::smem_u32(v_tiles + st * kTileBytes) + k * 2048, kBlockBytes), id_o,
                               j > 0 || k > 0);
            tc::mma_commit(lead, &o_full);
            if (!kApart && j + 1 < n_tiles && !(ok = score(j + 1))) break;
            // P of this tile was written after the product before it was
            // done, so with two stages that one's V tile is free; with one
            // stage this product has to end first
            if (kStages == 1 && j + 1 < n_tiles && !(ok = wait.warp(&o_full, (uint32_t)j & 1u))) break;
            if (j + 1 >= kStages && j + 1 < n_tiles) {
                load_v(w, j + 1);
                v_issued = j + 2;
            }
        }
        // every product issued ends before the block frees its memory, and
        // after an abort so does every copy (within the poll limit)
        auto landed = [&](uint64_t *bar, uint32_t parity) {
            for (uint32_t it = 0; it < kPolls; ++it)
                if (tc::mbar_try_wait(bar, parity)) return;
        };
        tc::mma_commit(lead, &drained);
        landed(&drained, 0);
        if (!ok && n_tiles > 0) {
            landed(&q_full, 0);
            for (int j = max(0, k_issued - kStages); j < k_issued; ++j)
                landed(&k_full[j % kStages], (uint32_t)(j / kStages) & 1u);
            for (int j = max(0, v_issued - kStages); j < v_issued; ++j)
                landed(&v_full[j % kStages], (uint32_t)(j / kStages) & 1u);
        }
        __syncwarp();
    } else {
        // ---------------- softmax and epilogue ----------------
        const int quarter = warp & 3, half = warp >> 2;
        const int r = quarter * 32 + lane;
        const bool live = r < w.rows;
        const int qi = w.query0 + (SPLIT ? r / f.pack : r);      // query of the document
        const int head = head0 + (SPLIT ? r % f.pack : 0);
        const int place = qi + w.shift;
        // keys that this row sees, counted from this half's first column
        const int seen = (live ? (a.causal ? min(w.nk, place + 1) : w.nk) - w.k_first : 0) - half * kHalf;
        const float c = a.scale * kLog2e;
        const uint32_t lane_base = tmem + ((uint32_t)(quarter * 32) << 16);
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
        float m = -INFINITY, l = 0.f;
        bool ok = true;
        for (int j = 0; j < n_tiles; ++j) {
            if (!(ok = wait.warp(&s_full, (uint32_t)j & 1u))) break;
            tc::fence_after_sync();
            float x[2][32];
            {
                uint32_t raw[2][32];
                tc::tmem_ld32_issue(lane_base + half * kHalf, raw[0]);
                tc::tmem_ld32_issue(lane_base + half * kHalf + 32, raw[1]);
                tc::tmem_ld_wait(raw[0]);
                tc::tmem_ld_wait(raw[1]);
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int e = 0; e < 32; ++e) x[i][e] = __uint_as_float(raw[i][e]);
            }
            tc::fence_before_sync();
            tc::mbar_arrive(&s_free);
            if (BIAS) {
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    // distances d0 - place + 0 .. 31
                    const int d0 = w.k_first + j * kTile + half * kHalf + 32 * i;
                    const bool after = d0 - place_hi >= a.reach, before = d0 + 31 - place_lo <= -a.reach;
                    if (after || before) {
                        const float b = lut[after ? a.reach : -a.reach];
#pragma unroll
                        for (int e = 0; e < 32; ++e) x[i][e] = fmaf(x[i][e], c, b);
                    } else {
                        const float *at = lut + (live ? d0 - place : 0);
#pragma unroll
                        for (int e = 0; e < 32; ++e) x[i][e] = fmaf(x[i][e], c, at[e]);
                    }
                }
            }
            const int vis = seen - j * kTile;                    // columns of the half that this row sees
            if (!__all_sync(0xffffffffu, vis >= kHalf)) {
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int e = 0; e < 32; ++e)
                        if (32 * i + e >= vis) x[i][e] = -INFINITY;
            }
            // the row's maximum over both halves (without a bias the scale is
            // not negative, so it can be applied after the comparison)
            float top = fmaxf(max_of_32(x[0]), max_of_32(x[1]));
            if (!BIAS) top *= c;
            s_top[j & 1][half][r] = top;
            tc::mbar_arrive(&pair_bar[quarter]);
            if (!(ok = wait.warp(&pair_bar[quarter], (uint32_t)j & 1u))) break;
            top = fmaxf(top, s_top[j & 1][half ^ 1][r]);
            if (j > 0) {
                // the last tile's product is done with P (and O) before they
                // are written
                if (!(ok = wait.warp(&o_full, (uint32_t)(j - 1) & 1u))) break;
                tc::fence_after_sync();
            }
            const bool raise = top > m + kRaise || m == -INFINITY;
            if (j == 0) {
                m = top;
            } else if (__any_sync(0xffffffffu, raise)) {
                const float old = m;
                if (raise) m = fmaxf(top, m);
                const float scale = raise && old != m ? exp2_approx(old - (m == -INFINITY ? 0.f : m)) : 1.f;
                l *= scale;
#pragma unroll
                for (int i = 0; i < DP / 32; ++i) {
                    uint32_t o[16];
                    tmem_ld16(lane_base + kOCol + half * (DP / 2) + 16 * i, o);
#pragma unroll
                    for (int e = 0; e < 16; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * scale);
                    tc::tmem_st16(lane_base + kOCol + half * (DP / 2) + 16 * i, o);
                }
            }
            const float sub = m == -INFINITY ? 0.f : m;
            float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                uint32_t pk[16];
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const float p0 = exp2_approx(BIAS ? x[i][2 * e] - sub : fmaf(x[i][2 * e], c, -sub));
                    const float p1 = exp2_approx(BIAS ? x[i][2 * e + 1] - sub : fmaf(x[i][2 * e + 1], c, -sub));
                    sum[2 * (e & 1)] += p0;
                    sum[2 * (e & 1) + 1] += p1;
                    pk[e] = pack2<T>(p0, p1);
                }
                tc::tmem_st16(lane_base + kPCol + half * kPHalf + 16 * i, pk);
            }
            l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
            tc::tmem_st_wait();
            tc::fence_before_sync();
            tc::mbar_arrive(&p_full);
        }
        // the row's sum over both halves
        if (ok) {
            s_top[n_tiles & 1][half][r] = l;
            tc::mbar_arrive(&pair_bar[quarter]);
            ok = wait.warp(&pair_bar[quarter], (uint32_t)n_tiles & 1u);
            l += s_top[n_tiles & 1][half ^ 1][r];
        }
        if (ok && n_tiles > 0) ok = wait.warp(&o_full, (uint32_t)(n_tiles - 1) & 1u);
        if (ok) {
            tc::fence_after_sync();
            const int d = a.head_dim;
            const bool none = n_tiles == 0 || l == 0.f;
            const float inv = SPLIT ? 1.f : 1.f / l;
            const int64_t at = ((int64_t)t * groups + hg) * f.rows_per_doc + r;         // split
            const int64_t row = w.q_row + r;                                            // not split
            if (live && half == 0) {
                if (SPLIT) f.part_ml[at] = make_float2(m, l);
                else f.p.lse[(int64_t)head * a.q_tokens + row] = none ? -INFINITY : m * kLn2 + logf(l);
            }
#pragma unroll
            for (int i = 0; i < DP / 64; ++i) {
                const int col = half * (DP / 2) + 32 * i;
                float o[32];
                if (n_tiles > 0) tc::tmem_ld32(lane_base + kOCol + col, o);
                if (!live) continue;
#pragma unroll
                for (int e = 0; e < 32; ++e) o[e] = none ? 0.f : o[e] * inv;
                if (SPLIT) {
#pragma unroll
                    for (int e = 0; e < 32; e += 4)
                        if (col + e < d)
                            *reinterpret_cast<float4 *>(f.part_o + at * d + col + e) =
                                make_float4(o[e], o[e + 1], o[e + 2], o[e + 3]);
                } else {
                    T *out = static_cast<T *>(f.p.out) + (row * a.heads + head) * d;
#pragma unroll
                    for (int e = 0; e < 32; e += 8)
                        if (col + e < d)
                            *reinterpret_cast<uint4 *>(out + col + e) =
                                make_uint4(pack2<T>(o[e], o[e + 1]), pack2<T>(o[e + 2], o[e + 3]),
                                           pack2<T>(o[e + 4], o[e + 5]), pack2<T>(o[e + 6], o[e + 7]));
                }
            }
        }
    }
    tc::fence_before_sync();
    __syncthreads();
    if (warp == 0) {
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
