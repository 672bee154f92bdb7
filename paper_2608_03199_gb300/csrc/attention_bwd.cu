// attention_bwd.cu -- attention over packed documents, backward.
//
// Two kernels recompute the probabilities tile by tile (128 x 128) from q, k
// and lse.  Each block owns its outputs, so nothing is added across blocks
// but the table's partial sums, and every sum has one order.
//
// k_attend_dq: a block per tile of queries and head, over the document's keys.
//   S = Q K^T, dP = dO V^T     a thread's lane is its query
//   dS = P (dP - delta), rounded to 16 bits into tensor memory
//   dQ += dS K
// It starts with delta = dO . O of its rows; O was rounded, so with a table it
// also sums dS along every row: that sum would be zero with the exact delta
// (the probabilities of a row add up to one), so delta plus the sum is the
// exact one, and the second kernel takes that.
//
// k_attend_dkv: a block per tile of keys and key head, over the heads that
// share it and their queries.
//   S^T = K Q^T, dP^T = V dO^T   a thread's lane is its key
//   dV += P^T dO, dK += dS^T Q   P^T and dS^T from tensor memory
// and the table's gradient: dS summed along diagonals (equal distances), in
// fp32, before any rounding.
//
// In both, warps 0-7 make P and dS (two warps to 32 lanes, 64 columns each),
// warp 8 loads, warp 9 issues the products: while the threads turn S into P
// the tensor cores work on dP and the product before, and the other way
// round.  A block takes all of tensor memory, so one runs per SM.
#include <cstring>

#include "attention.cuh"

namespace sieve {
namespace enc {
namespace {

constexpr int kWarps = 8;
constexpr int kCompute = kWarps * 32;
constexpr int kThreads = kCompute + 64;
constexpr int kHalf = kTile / 2;
constexpr int kScratch = 64;   // floats per warp for the diagonals of 32 x 32

// k_attend_dkv rounds P to 16 bits.  A long document's probabilities are small
// and fp16 has no bits below 2^-24, so it takes 2^14 P there (P <= 1 up to the
// rounding of lse), and dV is scaled back; dS = 2^14 P (2^-14 dP - 2^-14
// delta) costs no operation more.  dS itself stays as it is: its size is the
// caller's, and a factor could overflow what would not (fp16 gradients want a
// scaled loss).
template <typename T>
constexpr int kPShift = std::is_same_v<T, __half> ? 14 : 0;

struct BwdArgs {
    AttentionArgs p;
    CUtensorMap q, k, v, dout;
    float *stats;      // [q tile][head][2][128]: kPShift - lse in base 2, 2^-kPShift delta
    float *partial;    // [k tile][head][entries]: dS by distance
    int doc_tiles;     // new_tokens > 0: q tiles of a document
    int entries;       // bias_entries(reach)
};

// tiles of the walked operand pair held at a time
__host__ __device__ constexpr int stages(int dp) { return dp == 64 ? 3 : 2; }

__device__ __forceinline__ int first_q_tile(const BwdArgs &f, int s) {
    return f.p.a.new_tokens > 0 ? s * f.doc_tiles : first_tile(f.p.a.q_offsets, s, (int)f.p.a.q_tokens, kTile);
}

// The eight compute warps meet: bounded like every wait, so a warp that gave
// up leaves none behind.
struct Meeting {
    uint64_t *bar;
    uint32_t phase;
    __device__ __forceinline__ bool operator()(const Waiter &wait) {
        tc::mbar_arrive(bar);
        const bool ok = wait.warp(bar, phase);
        phase ^= 1u;
        return ok;
    }
};

template <typename T, int DP, bool BIAS>
__global__ void __launch_bounds__(kThreads, 1) k_attend_dq(const __grid_constant__ BwdArgs f) {
    constexpr int kB = DP / 64, kStages = stages(DP);
    constexpr uint32_t kTileBytes = kB * kBlockBytes;
    constexpr uint32_t kSCol = 0, kDpCol = 256, kDqCol = 384;   // S twice, dP (dS in its place), dQ
    extern __shared__ unsigned char smem_raw[];
    __shared__ __align__(8) uint64_t q_full, kv_full[kStages], kv_empty[kStages], s_full[2], s_free[2], dp_full,
        ds_full, meet_bar, done;
    __shared__ uint32_t tmem_slot;
    __shared__ int s_abort;
    __shared__ float s_row[2][kTile];
    const sieve_attention_args &a = f.p.a;
    const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0), lane = lane_id();
    if (blockIdx.x == 0 && threadIdx.x == 0) f.p.ctl->status = 0;

    const int t = blockIdx.x / a.heads, head = blockIdx.x % a.heads, hk = head / (a.heads / a.kv_heads);
    int s, tile;
    if (a.new_tokens > 0) {
        s = t / f.doc_tiles;
        tile = t % f.doc_tiles;
    } else {
        s = find_doc(a.q_offsets, (int)a.nseq, (int)a.q_tokens, kTile, t);
        tile = t - first_tile(a.q_offsets, s, (int)a.q_tokens, kTile);
    }
    const Doc doc = doc_at(a, s);
    const int tiles = (int)ceil_div(doc.nq, kTile);
    if (tile < 0 || tile >= tiles) return;
    tile = tiles - 1 - tile;                           // the tiles that see most keys first
    const int row0 = tile * kTile, rows = min(kTile, doc.nq - row0), shift = doc.nk - doc.nq;
    const int k_end = a.causal ? min(doc.nk, row0 + rows + shift) : doc.nk;
    const int n_tiles = k_end > 0 ? (k_end + kTile - 1) / kTile : 0;
    float *stats = f.stats + ((int64_t)(first_q_tile(f, s) + tile) * a.heads + head) * 2 * kTile;

    unsigned char *base = reinterpret_cast<unsigned char *>(
        (reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~static_cast<uintptr_t>(1023));
    unsigned char *q_tile = base, *do_tile = base + kTileBytes, *kv = do_tile + kTileBytes;
    float *bias = reinterpret_cast<float *>(kv + kStages * 2 * kTileBytes);

    if (threadIdx.x == 0) {
        tc::mbar_init(&q_full, 1);
        for (int i = 0; i < kStages; ++i) {
            tc::mbar_init(&kv_full[i], 1);
            tc::mbar_init(&kv_empty[i], 1);
        }
        for (int i = 0; i < 2; ++i) {
            tc::mbar_init(&s_full[i], 1);
            tc::mbar_init(&s_free[i], kCompute);
        }
        tc::mbar_init(&dp_full, 1);
        tc::mbar_init(&ds_full, kCompute);
        tc::mbar_init(&meet_bar, kCompute);
        tc::mbar_init(&done, 1);
        s_abort = 0;
        tc::mbar_init_fence();
    }
    if (warp == kWarps + 1) tc::tmem_alloc(&tmem_slot, 512);
    if (BIAS)
        fill_bias(bias, a, head, 1, threadIdx.x, kThreads);
    tc::fence_before_sync();
    __syncthreads();
    tc::fence_after_sync();
    const uint32_t tmem = __shfl_sync(0xffffffffu, tmem_slot, 0);
    const Waiter wait{&s_abort};

    if (warp == kWarps) {
        // ---------------- loads ----------------
        const uint32_t lead = lane == 0;
        bool ok = n_tiles > 0;
        int issued = 0;
        if (ok) {
            tc::mbar_arrive_expect_tx(lead, &q_full, 2 * kTileBytes);
            for (int b = 0; b < kB; ++b) {
                tma_load(lead, q_tile + b * kBlockBytes, &f.q, 64 * b, head, doc.q0 + row0, &q_full);
                tma_load(lead, do_tile + b * kBlockBytes, &f.dout, 64 * b, head, doc.q0 + row0, &q_full);
            }
        }
        for (int j = 0; ok && j < n_tiles; ++j) {
            const int st = j % kStages;
            if (!(ok = wait.warp(&kv_empty[st], ((uint32_t)(j / kStages) & 1u) ^ 1u))) break;
            tc::mbar_arrive_expect_tx(lead, &kv_full[st], 2 * kTileBytes);
            unsigned char *dst = kv + st * 2 * kTileBytes;
            for (int b = 0; b < kB; ++b) {
                tma_load(lead, dst + b * kBlockBytes, &f.k, 64 * b, hk, doc.k0 + j * kTile, &kv_full[st]);
                tma_load(lead, dst + kTileBytes + b * kBlockBytes, &f.v, 64 * b, hk, doc.k0 + j * kTile, &kv_full[st]);
            }
            issued = j + 1;
        }
        if (!ok && n_tiles > 0) {
            // after an abort: the copies in flight land before the block ends
            let_land(&q_full, 0);
            for (int j = max(0, issued - kStages); j < issued; ++j)
                let_land(&kv_full[j % kStages], (uint32_t)(j / kStages) & 1u);
        }
    } else if (warp == kWarps + 1) {
        // ---------------- products ----------------
        constexpr uint32_t id_s = idesc<T>(kTile, false), id_o = idesc<T>(DP, true);
        const uint64_t qa = desc_k(q_tile), doa = desc_k(do_tile);
        bool ok = n_tiles > 0;
        auto k_of = [&](int j) { return kv + (j % kStages) * 2 * kTileBytes; };
        auto loaded = [&](int j) {
            if (!wait.warp(&kv_full[j % kStages], (uint32_t)(j / kStages) & 1u)) return false;
            const int left = doc.nk - j * kTile;
            if (left < kTile) {
                clear_rows(k_of(j), left, kB);
                clear_rows(k_of(j) + kTileBytes, left, kB);
            }
            return true;
        };
        auto score = [&](int j) {
            if (elected()) {
                mma_kk<DP>(tmem + kSCol + (j & 1) * kTile, qa, desc_k(k_of(j)), id_s);
                commit(&s_full[j & 1]);
            }
            __syncwarp();
        };
        auto dprob = [&](int j) {
            if (elected()) {
                mma_kk<DP>(tmem + kDpCol, doa, desc_k(k_of(j) + kTileBytes), id_s);
                commit(&dp_full);
            }
            __syncwarp();
        };
        if (ok) ok = wait.warp(&q_full, 0) && loaded(0);
        if (ok) {
            tc::fence_after_sync();
            score(0);
            dprob(0);
        }
        for (int j = 0; ok && j < n_tiles; ++j) {
            if (j + 1 < n_tiles) {
                if (!(ok = loaded(j + 1))) break;
                // the buffer's scores before (j - 1) are in registers
                if (j > 0 && !(ok = wait.warp(&s_free[(j + 1) & 1], (uint32_t)((j - 1) / 2) & 1u))) break;
                tc::fence_after_sync();
                score(j + 1);
            }
            if (!(ok = wait.warp(&ds_full, (uint32_t)j & 1u))) break;
            tc::fence_after_sync();
            if (elected()) {
                mma_halves<kHalf>(tmem + kDqCol, tmem + kDpCol, desc_mn(k_of(j)), id_o, j > 0);
                commit(&kv_empty[j % kStages]);
            }
            __syncwarp();
            if (j + 1 < n_tiles) dprob(j + 1);
        }
        // every product issued ends before the block reads dQ or frees its
        // memory (waited for even after an abort, within the poll limit)
        if (elected()) commit(&done);
        __syncwarp();
        let_land(&done, 0);
        __syncwarp();
    } else {
        // ---------------- P, dS and dQ ----------------
        const int quarter = warp & 3, half = warp >> 2;
        const int r = quarter * 32 + lane;
        const bool live = r < rows;
        const int place = row0 + r + shift;
        const int seen = live ? (a.causal ? min(doc.nk, place + 1) : doc.nk) : 0;
        const int64_t row = doc.q0 + row0 + r;
        const int d = a.head_dim;
        const float c = a.scale * kLog2e;
        const uint32_t lane_base = tmem + ((uint32_t)(quarter * 32) << 16);
        // delta: each of a row's two threads adds one half of the products
        float part = 0.f, nl = -INFINITY;
        if (live) {
            const T *o = static_cast<const T *>(f.p.out_in) + (row * a.heads + head) * d;
            const T *g = static_cast<const T *>(f.p.dout) + (row * a.heads + head) * d;
            for (int i = half * 8; i < d; i += 16) {
                float x[8], y[8];
                load_vec<T, 8>(o + i, x);
                load_vec<T, 8>(g + i, y);
#pragma unroll
                for (int e = 0; e < 8; ++e) part = fmaf(x[e], y[e], part);
            }
            const float lse = f.p.lse_in[(int64_t)head * a.q_tokens + row];
            if (lse != -INFINITY) nl = -lse * kLog2e;
        }
        Meeting meet{&meet_bar, 0};
        s_row[half][r] = part;
        bool ok = meet(wait);
        const float delta = live ? s_row[0][r] + s_row[1][r] : 0.f;
        ok = ok && meet(wait);
        int place_lo = live ? place : INT32_MAX, place_hi = live ? place : INT32_MIN;
        if (BIAS) {
            place_lo = row0 + quarter * 32 + shift;
            place_hi = place_lo + 31;
        }
        const float bias_before = BIAS ? bias[bias_zero(a.reach) - a.reach] : 0.f;
        const float bias_after = BIAS ? bias[bias_zero(a.reach) + a.reach] : 0.f;
        float row_sum = 0.f;
        for (int j = 0; ok && j < n_tiles; ++j) {
            if (!(ok = wait.warp(&s_full[j & 1], (uint32_t)(j / 2) & 1u))) break;
            tc::fence_after_sync();
            float p[2][32];
            const uint32_t s_at = lane_base + kSCol + (j & 1) * kTile + half * kHalf;
            {
                uint32_t raw[2][32];
                tc::tmem_ld32_issue(s_at, raw[0]);
                tc::tmem_ld32_issue(s_at + 32, raw[1]);
                tc::tmem_ld_wait(raw[0]);
                tc::tmem_ld_wait(raw[1]);
                tc::fence_before_sync();
                tc::mbar_arrive(&s_free[j & 1]);
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const int d0 = j * kTile + half * kHalf + 32 * i;
                    if (!BIAS || d0 - place_hi >= a.reach || d0 + 31 - place_lo <= -a.reach) {
                        const float b = nl + (!BIAS ? 0.f : d0 - place_hi >= a.reach ? bias_after : bias_before);
#pragma unroll
                        for (int e = 0; e < 32; ++e) p[i][e] = exp2_approx(fmaf(__uint_as_float(raw[i][e]), c, b));
                    } else {
                        const float4 *at = bias_at(bias, a.reach, d0 - place);
#pragma unroll
                        for (int e = 0; e < 8; ++e) {
                            const float4 b = at[e];
                            p[i][4 * e + 0] = exp2_approx(fmaf(__uint_as_float(raw[i][4 * e + 0]), c, b.x + nl));
                            p[i][4 * e + 1] = exp2_approx(fmaf(__uint_as_float(raw[i][4 * e + 1]), c, b.y + nl));
                            p[i][4 * e + 2] = exp2_approx(fmaf(__uint_as_float(raw[i][4 * e + 2]), c, b.z + nl));
                            p[i][4 * e + 3] = exp2_approx(fmaf(__uint_as_float(raw[i][4 * e + 3]), c, b.w + nl));
                        }
                    }
                }
            }
            const int vis = seen - j * kTile - half * kHalf;
            if (!__all_sync(0xffffffffu, vis >= kHalf)) {
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int e = 0; e < 32; ++e)
                        if (32 * i + e >= vis) p[i][e] = 0.f;
            }
            if (!(ok = wait.warp(&dp_full, (uint32_t)j & 1u))) break;
            tc::fence_after_sync();
            const uint32_t dp_at = lane_base + kDpCol + half * kHalf;
            uint32_t w[32];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                float dp[32];
                tc::tmem_ld32(dp_at + 32 * i, dp);
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const float x0 = p[i][2 * e] * (dp[2 * e] - delta), x1 = p[i][2 * e + 1] * (dp[2 * e + 1] - delta);
                    if (BIAS) row_sum += x0 + x1;
                    w[16 * i + e] = pack2<T>(x0, x1);
                }
            }
            tmem_st32(dp_at, w);
            tc::tmem_st_wait();
            tc::fence_before_sync();
            tc::mbar_arrive(&ds_full);
        }
        if (ok && n_tiles > 0) ok = wait.warp(&done, 0);
        if (ok) {
            tc::fence_after_sync();
            T *out = static_cast<T *>(f.p.dq) + row * f.p.dq_ts + head * f.p.dq_hs;
#pragma unroll
            for (int i = 0; i < DP / 64; ++i) {
                const int col = half * (DP / 2) + 32 * i;
                float o[32];
                tc::tmem_ld32(lane_base + kDqCol + col, o);
                if (live)
#pragma unroll
                    for (int e = 0; e < 32; e += 8)
                        if (col + e < d) {
                            float v[8];
#pragma unroll
                            for (int u = 0; u < 8; ++u) v[u] = n_tiles > 0 && nl != -INFINITY ? o[e + u] * a.scale : 0.f;
                            store_vec<T, 8>(out + col + e, v);
                        }
            }
            s_row[half][r] = row_sum;
            if (meet(wait) && half == 0) {
                stats[r] = nl + (float)kPShift<T>;
                stats[kTile + r] = (delta + (BIAS && nl != -INFINITY ? s_row[0][r] + s_row[1][r] : 0.f)) *
                                   (1.f / (float)(1 << kPShift<T>));
            }
        }
    }
    tc::fence_before_sync();
    __syncthreads();
    if (threadIdx.x == 0 && s_abort) atomicExch(&f.p.ctl->status, SIEVE_ETIMEOUT);
    if (warp == kWarps + 1) {
        tc::fence_after_sync();
        tc::tmem_dealloc(tmem, 512);
    }
}

template <typename T, int DP, bool BIAS>
__global__ void __launch_bounds__(kThreads, 1) k_attend_dkv(const __grid_constant__ BwdArgs f) {
    constexpr int kB = DP / 64, kStages = stages(DP);
    constexpr uint32_t kTileBytes = kB * kBlockBytes;
    constexpr uint32_t kSCol = 0, kDpCol = 128, kDvCol = 256, kDkCol = 384;   // P in S's place, dS in dP's
    extern __shared__ unsigned char smem_raw[];
    __shared__ __align__(16) float s_stats[kStages][2][kTile];
    __shared__ __align__(8) uint64_t kv_full, q_full[kStages], q_empty[kStages], s_full, p_full, dp_full, ds_full,
        meet_bar, done;
    __shared__ uint32_t tmem_slot;
    __shared__ int s_abort;
    const sieve_attention_args &a = f.p.a;
    const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0), lane = lane_id();

    const int t = blockIdx.x / a.kv_heads, hk = blockIdx.x % a.kv_heads, share = a.heads / a.kv_heads;
    const int s = find_doc(a.k_offsets, (int)a.nseq, (int)a.k_tokens, kTile, t);
    const int tile = t - first_tile(a.k_offsets, s, (int)a.k_tokens, kTile);
    const Doc doc = doc_at(a, s);
    const int key0 = tile * kTile;
    if (tile < 0 || key0 >= doc.nk) {
        // a tile number that no document uses adds nothing to the table
        for (int e = threadIdx.x; e < share * f.entries; e += kThreads)
            f.partial[((int64_t)t * a.heads + hk * share) * f.entries + e] = 0.f;
        return;
    }
    const int rows = min(kTile, doc.nk - key0), shift = doc.nk - doc.nq;
    // the first tile of queries that sees any of these keys
    const int q_first = a.causal ? max(0, key0 - shift) / kTile : 0;
    const int q_tiles = max(0, (int)ceil_div(doc.nq, kTile) - q_first);
    const int n = q_tiles * share;                     // steps: heads, queries inside
    const int q_number = first_q_tile(f, s);

    unsigned char *base = reinterpret_cast<unsigned char *>(
        (reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~static_cast<uintptr_t>(1023));
    unsigned char *k_tile = base, *v_tile = base + kTileBytes, *qd = v_tile + kTileBytes;
    float *bias = reinterpret_cast<float *>(qd + kStages * 2 * kTileBytes);
    // the bias by minus the distance (columns run that way)
    constexpr int kCopies = DP == 64 ? 4 : 1;
    float *by_distance = bias + (BIAS ? bias_floats(a.reach, kCopies) : 0);   // [warps][entries]
    float *scratch = by_distance + kWarps * f.entries;         // [warps][kScratch]

    if (threadIdx.x == 0) {
        tc::mbar_init(&kv_full, 1);
        for (int i = 0; i < kStages; ++i) {
            tc::mbar_init(&q_full[i], 1);
            tc::mbar_init(&q_empty[i], 1);
        }
        tc::mbar_init(&s_full, 1);
        tc::mbar_init(&p_full, kCompute);
        tc::mbar_init(&dp_full, 1);
        tc::mbar_init(&ds_full, kCompute);
        tc::mbar_init(&meet_bar, kCompute);
        tc::mbar_init(&done, 1);
        s_abort = 0;
        tc::mbar_init_fence();
    }
    if (warp == kWarps + 1) tc::tmem_alloc(&tmem_slot, 512);
    tc::fence_before_sync();
    __syncthreads();
    tc::fence_after_sync();
    const uint32_t tmem = __shfl_sync(0xffffffffu, tmem_slot, 0);
    const Waiter wait{&s_abort};

    if (warp == kWarps) {
        // ---------------- loads ----------------
        const uint32_t lead = lane == 0;
        bool ok = n > 0;
        int issued = 0;
        if (ok) {
            tc::mbar_arrive_expect_tx(lead, &kv_full, 2 * kTileBytes);
            for (int b = 0; b < kB; ++b) {
                tma_load(lead, k_tile + b * kBlockBytes, &f.k, 64 * b, hk, doc.k0 + key0, &kv_full);
                tma_load(lead, v_tile + b * kBlockBytes, &f.v, 64 * b, hk, doc.k0 + key0, &kv_full);
            }
        }
        int g = 0, qt = q_first;
        for (int i = 0; ok && i < n; ++i) {
            const int st = i % kStages, head = hk * share + g, row = doc.q0 + qt * kTile;
            if (!(ok = wait.warp(&q_empty[st], ((uint32_t)(i / kStages) & 1u) ^ 1u))) break;
            tc::mbar_arrive_expect_tx(lead, &q_full[st], 2 * kTileBytes + 2 * kTile * 4);
            unsigned char *dst = qd + st * 2 * kTileBytes;
            for (int b = 0; b < kB; ++b) {
                tma_load(lead, dst + b * kBlockBytes, &f.q, 64 * b, head, row, &q_full[st]);
                tma_load(lead, dst + kTileBytes + b * kBlockBytes, &f.dout, 64 * b, head, row, &q_full[st]);
            }
            tc::bulk_g2s(lead, s_stats[st], f.stats + ((int64_t)(q_number + qt) * a.heads + head) * 2 * kTile,
                         2 * kTile * 4, &q_full[st]);
            issued = i + 1;
            if (++qt == q_first + q_tiles) {
                qt = q_first;
                ++g;
            }
        }
        if (!ok && n > 0) {
            // after an abort: the copies in flight land before the block ends
            let_land(&kv_full, 0);
            for (int i = max(0, issued - kStages); i < issued; ++i)
                let_land(&q_full[i % kStages], (uint32_t)(i / kStages) & 1u);
        }
    } else if (warp == kWarps + 1) {
        // ---------------- products ----------------
        constexpr uint32_t id_s = idesc<T>(kTile, false), id_o = idesc<T>(DP, true);
        const uint64_t ka = desc_k(k_tile), va = desc_k(v_tile);
        bool ok = n > 0;
        auto q_of = [&](int i) { return qd + (i % kStages) * 2 * kTileBytes; };
        int qt_loaded = q_first;
        auto loaded = [&](int i) {
            if (!wait.warp(&q_full[i % kStages], (uint32_t)(i / kStages) & 1u)) return false;
            const int left = doc.nq - qt_loaded * kTile;
            if (left < kTile) {
                clear_rows(q_of(i), left, kB);
                clear_rows(q_of(i) + kTileBytes, left, kB);
            }
            if (++qt_loaded == q_first + q_tiles) qt_loaded = q_first;
            return true;
        };
        auto score = [&](int i) {
            if (elected()) {
                mma_kk<DP>(tmem + kSCol, ka, desc_k(q_of(i)), id_s);
                commit(&s_full);
            }
            __syncwarp();
        };
        auto dprob = [&](int i) {
            if (elected()) {
                mma_kk<DP>(tmem + kDpCol, va, desc_k(q_of(i) + kTileBytes), id_s);
                commit(&dp_full);
            }
            __syncwarp();
        };
        if (ok) ok = wait.warp(&kv_full, 0) && loaded(0);
        if (ok) {
            tc::fence_after_sync();
            score(0);
            dprob(0);
        }
        for (int i = 0; ok && i < n; ++i) {
            if (!(ok = wait.warp(&p_full, (uint32_t)i & 1u))) break;
            tc::fence_after_sync();
            if (elected()) mma_halves<kHalf>(tmem + kDvCol, tmem + kSCol, desc_mn(q_of(i) + kTileBytes), id_o, i > 0);
            __syncwarp();
            if (i + 1 < n) {
                if (!(ok = loaded(i + 1))) break;
                tc::fence_after_sync();
                score(i + 1);
            }
            if (!(ok = wait.warp(&ds_full, (uint32_t)i & 1u))) break;
            tc::fence_after_sync();
            if (elected()) {
                mma_halves<kHalf>(tmem + kDkCol, tmem + kDpCol, desc_mn(q_of(i)), id_o, i > 0);
                commit(&q_empty[i % kStages]);
            }
            __syncwarp();
            if (i + 1 < n) dprob(i + 1);
        }
        // every product issued ends before the block reads dK and dV or frees
        // its memory (waited for even after an abort, within the poll limit)
        if (elected()) commit(&done);
        __syncwarp();
        let_land(&done, 0);
        __syncwarp();
    } else {
        // ---------------- P, dS, dK and dV ----------------
        const int quarter = warp & 3, half = warp >> 2;
        const int r = quarter * 32 + lane, key = key0 + r;
        const bool live = r < rows;
        const int d = a.head_dim;
        const float c = a.scale * kLog2e;
        const uint32_t lane_base = tmem + ((uint32_t)(quarter * 32) << 16);
        const int key_lo = key0 + quarter * 32;
        float *mine = by_distance + warp * f.entries, *line = scratch + warp * kScratch;
        const float not_first = lane == 0 ? 0.f : 1.f;
        constexpr float kDown = 1.f / (float)(1 << kPShift<T>);
        float far_before = 0.f, far_after = 0.f;
        Meeting meet{&meet_bar, 0};
        bool ok = true;
        int g = 0, qt = q_first;
        for (int i = 0; i < n; ++i) {
            const int head = hk * share + g, st = i % kStages;
            if (BIAS && qt == q_first) {
                // a new head: its bias, and its sums from zero
                if (!(ok = meet(wait))) break;
                fill_bias<kCopies>(bias, a, head, -1, threadIdx.x, kCompute);
                for (int e = lane; e < f.entries; e += 32) mine[e] = 0.f;
                far_before = far_after = 0.f;
                if (!(ok = meet(wait))) break;
            }
            const int place0 = qt * kTile + half * kHalf + shift;      // place of the half's first query
            if (!(ok = wait.warp(&q_full[st], (uint32_t)(i / kStages) & 1u))) break;   // the row statistics
            if (!(ok = wait.warp(&s_full, (uint32_t)i & 1u))) break;
            tc::fence_after_sync();
            float p[2][32];
            uint32_t w[32];
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                uint32_t raw[32];
                tc::tmem_ld32_issue(lane_base + kSCol + half * kHalf + 32 * q, raw);
                const float4 *nl = reinterpret_cast<const float4 *>(&s_stats[st][0][half * kHalf + 32 * q]);
                const int lo = key_lo - (place0 + 32 * q) - 31, hi = key_lo + 31 - (place0 + 32 * q);
                tc::tmem_ld_wait(raw);
                if (!BIAS || lo >= a.reach || hi <= -a.reach) {
                    const float b = !BIAS ? 0.f : bias[bias_zero(a.reach) + (lo >= a.reach ? -a.reach : a.reach)];
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const float4 x = nl[e];
                        p[q][4 * e + 0] = exp2_approx(fmaf(__uint_as_float(raw[4 * e + 0]), c, x.x + b));
                        p[q][4 * e + 1] = exp2_approx(fmaf(__uint_as_float(raw[4 * e + 1]), c, x.y + b));
                        p[q][4 * e + 2] = exp2_approx(fmaf(__uint_as_float(raw[4 * e + 2]), c, x.z + b));
                        p[q][4 * e + 3] = exp2_approx(fmaf(__uint_as_float(raw[4 * e + 3]), c, x.w + b));
                    }
                } else {
                    const int first = place0 + 32 * q - key;
                    const float4 *at = bias_at(bias, a.reach, first);
                    const float *one = bias + bias_zero(a.reach) + first;
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const float4 x = nl[e];
                        const float4 b = kCopies == 4 ? at[e] : make_float4(one[4 * e], one[4 * e + 1], one[4 * e + 2], one[4 * e + 3]);
                        p[q][4 * e + 0] = exp2_approx(fmaf(__uint_as_float(raw[4 * e + 0]), c, x.x + b.x));
                        p[q][4 * e + 1] = exp2_approx(fmaf(__uint_as_float(raw[4 * e + 1]), c, x.y + b.y));
                        p[q][4 * e + 2] = exp2_approx(fmaf(__uint_as_float(raw[4 * e + 2]), c, x.z + b.z));
                        p[q][4 * e + 3] = exp2_approx(fmaf(__uint_as_float(raw[4 * e + 3]), c, x.w + b.w));
                    }
                }
            }
            if (a.causal) {
                const int from = key - place0;                        // columns before it do not see this key
                if (!__all_sync(0xffffffffu, from <= 0)) {
#pragma unroll
                    for (int q = 0; q < 2; ++q)
#pragma unroll
                        for (int e = 0; e < 32; ++e)
                            if (32 * q + e < from) p[q][e] = 0.f;
                }
            }
#pragma unroll
            for (int q = 0; q < 2; ++q)
#pragma unroll
                for (int e = 0; e < 16; ++e) w[16 * q + e] = pack2<T>(p[q][2 * e], p[q][2 * e + 1]);
            tmem_st32(lane_base + kSCol + half * kHalf, w);
            tc::tmem_st_wait();
            tc::fence_before_sync();
            tc::mbar_arrive(&p_full);

            if (!(ok = wait.warp(&dp_full, (uint32_t)i & 1u))) break;
            tc::fence_after_sync();
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                float dp[32];
                tc::tmem_ld32(lane_base + kDpCol + half * kHalf + 32 * q, dp);
                const float4 *dl = reinterpret_cast<const float4 *>(&s_stats[st][1][half * kHalf + 32 * q]);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float4 x = dl[e];
                    p[q][4 * e + 0] *= fmaf(dp[4 * e + 0], kDown, -x.x);
                    p[q][4 * e + 1] *= fmaf(dp[4 * e + 1], kDown, -x.y);
                    p[q][4 * e + 2] *= fmaf(dp[4 * e + 2], kDown, -x.z);
                    p[q][4 * e + 3] *= fmaf(dp[4 * e + 3], kDown, -x.w);
                }
#pragma unroll
                for (int e = 0; e < 16; ++e) w[16 * q + e] = pack2<T>(p[q][2 * e], p[q][2 * e + 1]);
            }
            tmem_st32(lane_base + kDpCol + half * kHalf, w);
            tc::tmem_st_wait();
            tc::fence_before_sync();
            tc::mbar_arrive(&ds_full);

            if (BIAS) {
                // dS by distance, under the products.  A lane is a key, a step
                // to the next query lowers its distance by one: a sum that
                // moves up one lane with every step follows one distance, and
                // leaves complete at lane 31.
#pragma unroll
                for (int q = 0; q < 2; ++q) {
                    const int lo = key_lo - (place0 + 32 * q) - 31, hi = key_lo + 31 - (place0 + 32 * q);
                    if (!live)   // rows past the document's keys add nothing
#pragma unroll
                        for (int e = 0; e < 32; ++e) p[q][e] = 0.f;
                    if (lo >= a.reach || hi <= -a.reach) {
                        float x[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                        for (int e = 0; e < 32; ++e) x[e & 3] += p[q][e];
                        (lo >= a.reach ? far_after : far_before) += (x[0] + x[1]) + (x[2] + x[3]);
                    } else {
                        float acc = 0.f;
#pragma unroll
                        for (int e = 0; e < 32; ++e) {
                            if (e) acc = __shfl_up_sync(0xffffffffu, acc, 1);
                            acc = e ? fmaf(acc, not_first, p[q][e]) : p[q][e];
                            if (lane == 31) line[e] = acc;          // distance hi - e
                        }
                        if (lane < 31) line[62 - lane] = acc;       // lane's distance: hi - (62 - lane)
                        __syncwarp();
                        float *to = mine + a.reach + kPad + hi;
                        to[-lane] += line[lane];
                        if (lane < 31) to[-(lane + 32)] += line[lane + 32];
                        __syncwarp();
                    }
                }
                if (qt == q_first + q_tiles - 1) {
                    // the head's last step: add the warps up, in order
                    const float before = warp_sum(far_before), after = warp_sum(far_after);
                    if (lane == 0) {
                        mine[kPad] += before;
                        mine[kPad + 2 * a.reach] += after;
                    }
                    if (!(ok = meet(wait))) break;
                    float *out = f.partial + ((int64_t)t * a.heads + head) * f.entries;
                    for (int e = threadIdx.x; e < f.entries; e += kCompute) {
                        float x = 0.f;
#pragma unroll
                        for (int k = 0; k < kWarps; ++k) x += by_distance[k * f.entries + e];
                        out[e] = x;
                    }
                }
            }
            if (++qt == q_first + q_tiles) {
                qt = q_first;
                ++g;
            }
        }
        if (BIAS && n == 0)   // no query sees these keys
            for (int h = 0; h < share; ++h)
                for (int e = threadIdx.x; e < f.entries; e += kCompute)
                    f.partial[((int64_t)t * a.heads + hk * share + h) * f.entries + e] = 0.f;
        if (ok && n > 0) ok = wait.warp(&done, 0);
        if (ok) {
            tc::fence_after_sync();
            const int64_t row = doc.k0 + key;
            // one half of the warps writes dV, the other dK
            T *out = half ? static_cast<T *>(f.p.dk) + row * f.p.dk_ts + hk * f.p.dk_hs
                          : static_cast<T *>(f.p.dv) + row * f.p.dv_ts + hk * f.p.dv_hs;
            const float scale = half ? a.scale : kDown;
#pragma unroll
            for (int i = 0; i < DP / 32; ++i) {
                float o[32];
                tc::tmem_ld32(lane_base + (half ? kDkCol : kDvCol) + 32 * i, o);
                if (live)
#pragma unroll
                    for (int e = 0; e < 32; e += 8)
                        if (32 * i + e < d) {
                            float v[8];
#pragma unroll
                            for (int u = 0; u < 8; ++u) v[u] = n > 0 ? o[e + u] * scale : 0.f;
                            store_vec<T, 8>(out + 32 * i + e, v);
                        }
            }
        }
    }
    tc::fence_before_sync();
    __syncthreads();
    if (threadIdx.x == 0 && s_abort) atomicExch(&f.p.ctl->status, SIEVE_ETIMEOUT);
    if (warp == kWarps + 1) {
        tc::fence_after_sync();
        tc::tmem_dealloc(tmem, 512);
    }
}

// The table's gradient: the k tiles' sums by distance added up (in splits of
// consecutive tiles, then the splits), then the distances of each bucket.
constexpr int kReduceThreads = 512;
__global__ void __launch_bounds__(kReduceThreads) k_attend_dtable(const __grid_constant__ BwdArgs f, int64_t tiles,
                                                                  int splits, float *split_sums) {
    const int head = blockIdx.x, split = blockIdx.y;
    const int64_t per = ceil_div(tiles, splits), lo = split * per, hi = lo + per < tiles ? lo + per : tiles;
    for (int e = threadIdx.x; e < f.entries; e += kReduceThreads) {
        float x = 0.f;
#pragma unroll 8
        for (int64_t t = lo; t < hi; ++t) x += f.partial[(t * f.p.a.heads + head) * f.entries + e];
        split_sums[((int64_t)head * splits + split) * f.entries + e] = x;
    }
}
__global__ void __launch_bounds__(kReduceThreads) k_attend_buckets(const __grid_constant__ BwdArgs f, int splits,
                                                                   const float *split_sums) {
    extern __shared__ float sums[];   // [entries]
    const sieve_attention_args &a = f.p.a;
    const int head = blockIdx.x;
    for (int e = threadIdx.x; e < f.entries; e += kReduceThreads) {
        float x = 0.f;
#pragma unroll 4
        for (int k = 0; k < splits; ++k) x += split_sums[((int64_t)head * splits + k) * f.entries + e];
        sums[e] = x;
    }
    __syncthreads();
    // a warp per bucket, lanes over the distances
    for (int b = threadIdx.x >> 5; b < a.num_buckets; b += kReduceThreads / 32) {
        float x = 0.f;
        for (int e = (int)lane_id(); e < f.entries; e += 32) {
            const int dist = min(max(e - a.reach - kPad, -a.reach), a.reach);
            if (min(max(a.bucket_map[a.reach + dist], 0), a.num_buckets - 1) == b) x += sums[e];
        }
        x = warp_sum(x);
        if (lane_id() == 0) f.p.dtable[b * a.heads + head] = x;
    }
}

struct Layout {
    int64_t q_tiles, k_tiles;
    int entries, splits;
    size_t stats, partial, split_sums, total;   // byte offsets
};
Layout layout_of(const sieve_attention_args &a) {
    Layout l = {};
    l.q_tiles = a.new_tokens > 0 ? a.nseq * ceil_div(a.new_tokens, kTile) : doc_tiles(a.q_tokens, a.nseq, kTile);
    l.k_tiles = doc_tiles(a.k_tokens, a.nseq, kTile);
    l.entries = a.num_buckets ? bias_entries(a.reach) : 0;
    l.splits = (int)(l.k_tiles < 16 * 64 ? ceil_div(l.k_tiles, 16) : 64);
    l.stats = kCtlBytes;
    l.partial = l.stats + (size_t)l.q_tiles * a.heads * 2 * kTile * sizeof(float);
    l.split_sums = l.partial + (size_t)round_up(l.k_tiles * a.heads * l.entries * (int64_t)sizeof(float), 256);
    l.total = l.split_sums + (size_t)round_up((int64_t)a.heads * l.splits * l.entries * (int64_t)sizeof(float), 256);
    return l;
}

template <typename T, int DP, bool BIAS>
cudaError_t run(const BwdArgs &f, const Layout &l, unsigned char *ws, cudaStream_t st) {
    const sieve_attention_args &a = f.p.a;
    const size_t tiles = 1024 + (size_t)(2 + 2 * stages(DP)) * (DP / 64) * kBlockBytes;
    cudaError_t e;
    if (a.q_tokens > 0) {
        auto dq = k_attend_dq<T, DP, BIAS>;
        const size_t smem = tiles + (BIAS ? (size_t)bias_floats(a.reach) * 4 : 0);
        if ((e = cudaFuncSetAttribute(dq, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem)) != cudaSuccess) return e;
        dq<<<(unsigned)(l.q_tiles * a.heads), kThreads, smem, st>>>(f);
        if ((e = cudaGetLastError()) != cudaSuccess) return e;
    }
    if (a.k_tokens > 0) {
        auto dkv = k_attend_dkv<T, DP, BIAS>;
        const size_t smem = tiles + (BIAS ? (size_t)(bias_floats(a.reach, DP == 64 ? 4 : 1) + f.entries * kWarps + kWarps * kScratch) * 4 : 0);
        if ((e = cudaFuncSetAttribute(dkv, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem)) != cudaSuccess) return e;
        dkv<<<(unsigned)(l.k_tiles * a.kv_heads), kThreads, smem, st>>>(f);
        if ((e = cudaGetLastError()) != cudaSuccess) return e;
    }
    if (BIAS) {
        if (a.k_tokens == 0 || a.q_tokens == 0)
            return cudaMemsetAsync(f.p.dtable, 0, (size_t)a.num_buckets * a.heads * sizeof(float), st);
        float *sums = reinterpret_cast<float *>(ws + l.split_sums);
        k_attend_dtable<<<dim3(a.heads, l.splits), kReduceThreads, 0, st>>>(f, l.k_tiles, l.splits, sums);
        if ((e = cudaGetLastError()) != cudaSuccess) return e;
        k_attend_buckets<<<a.heads, kReduceThreads, f.entries * sizeof(float), st>>>(f, l.splits, sums);
        if ((e = cudaGetLastError()) != cudaSuccess) return e;
    }
    return cudaSuccess;
}

template <typename T, int DP>
cudaError_t by_bias(const BwdArgs &f, const Layout &l, unsigned char *ws, cudaStream_t st) {
    return f.p.a.num_buckets ? run<T, DP, true>(f, l, ws, st) : run<T, DP, false>(f, l, ws, st);
}

}  // namespace

size_t attention_backward_workspace_bytes(const sieve_attention_args &a) { return layout_of(a).total; }

sieve_status launch_attention_backward(const AttentionArgs &p, void *ws, cudaStream_t st) {
    const sieve_attention_args &a = p.a;
    const Layout l = layout_of(a);
    unsigned char *w = static_cast<unsigned char *>(ws);
    BwdArgs f;
    std::memset(&f, 0, sizeof f);
    f.p = p;
    f.p.ctl = static_cast<EncCtl *>(ws);
    f.stats = reinterpret_cast<float *>(w + l.stats);
    f.partial = reinterpret_cast<float *>(w + l.partial);
    f.doc_tiles = a.new_tokens > 0 ? (int)ceil_div(a.new_tokens, kTile) : 0;
    f.entries = l.entries;
    sieve_status rc = SIEVE_OK;
    if (a.q_tokens > 0) {
        rc = make_map(&f.q, a.dtype, a.q, a.head_dim, a.heads, a.q_tokens, a.q_token_stride, a.q_head_stride, 1, kTile);
        if (rc == SIEVE_OK)
            rc = make_map(&f.dout, a.dtype, p.dout, a.head_dim, a.heads, a.q_tokens, (int64_t)a.heads * a.head_dim,
                          a.head_dim, 1, kTile);
    }
    if (rc == SIEVE_OK && a.k_tokens > 0) {
        rc = make_map(&f.k, a.dtype, a.k, a.head_dim, a.kv_heads, a.k_tokens, a.k_token_stride, a.k_head_stride, 1, kTile);
        if (rc == SIEVE_OK)
            rc = make_map(&f.v, a.dtype, a.v, a.head_dim, a.kv_heads, a.k_tokens, a.v_token_stride, a.v_head_stride, 1,
                          kTile);
    }
    if (rc != SIEVE_OK) return rc;
    const bool wide = a.head_dim > 64;
    cudaError_t e;
    if (a.dtype == SIEVE_F16) e = wide ? by_bias<__half, 128>(f, l, w, st) : by_bias<__half, 64>(f, l, w, st);
    else e = wide ? by_bias<__nv_bfloat16, 128>(f, l, w, st) : by_bias<__nv_bfloat16, 64>(f, l, w, st);
    return e == cudaSuccess ? SIEVE_OK : record_cuda_error(e);
}

}  // namespace enc
}  // namespace sieve
