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
// k_attend_delta gives it delta = dO . O.  O was rounded, so with a table it
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
// Measured (bf16): 384 documents of 0 to 512 tokens,
// 12 heads of 64 with a bias: delta 55 us (249 MB, 4.5 TB/s), dq 351, dk and dv
// 444, the table's sums 19; at a reach of 256 dq 397, dk and dv 467.  fp16: the
// longest v 37 (124 MB), delta 76, dq 357, dk and dv 461.  A step of 128 x 128 pairs takes about 3.3K cycles
// there: 1.3K for P (an exponential and a bias read for each pair), 0.45K for dS,
// 0.9K for its sums by distance, the rest waits; its four products are 1.1K.
// Short documents pay for what a block's work costs once, 4K to 5K cycles.
// Without a bias, 3 documents of 3,001 to 8,192 tokens, 16 heads of 128 on 4 key
// heads: dq 420 us, dk and dv 610, 57% and 52% of the tensor pipe.  10,000 texts of 10
// to 60 tokens, 12 heads of 64, a tile to each: delta 412, dq 2,119, dk and dv 2,627.
//
// In both, 16 warps make P and dS, each for 32 lanes and 32 columns; one more
// loads, one more issues the products.  While the threads turn S into P
// the tensor cores work on dP and the product before, and the other way
// round.  A block takes all of tensor memory, so one runs per SM; when it is
// done it takes over a block that has not started, whose loads and first
// products run under its last sums and stores.
#include <cstring>

#include "attention.cuh"

namespace sieve {
namespace enc {
namespace {

constexpr int kSlots = 2;      // the work in hand and the next
// Steps of work that is short: the next is asked for, and looked for, while it runs.
// (dq and dkv with 0 / 4 / 16 / 64 here: 384 documents of up to 512 tokens 360, 442 /
// 351, 445 / 351, 445 / 351, 445 us; 64 of up to 2,048 442, 570 / 448, 580 / 434, 584 /
// 434, 583; 3 of up to 8,192 412, 599 / 415, 597 / 422, 614 / 465, 649.)
constexpr int kShort = 16;

// fp16 has no bits below 2^-24, and a long document's P and dS are small.  So
// k_attend_dkv takes 2^14 P (P <= 1 up to the rounding of lse) and scales dV
// back, and both kernels round dS times a power of two that its row (dq) or
// document (dk) cannot overflow with, and scale dQ and dK back.  The bound:
// |dS| <= |dP| + |delta| <= 2 |dout| |v| for the row's dout and the document's
// longest v (O is a mean of v), so the power is 2^14 over the next one above it.
// (Unscaled, dout of 1e-2 on 12,288 tokens left dq and dk off by 1.6e-3 of their
// norm, of 1e-3 by 1.6e-2; rounding the results alone takes 2.1e-4 and 1.1e-3.)
template <typename T>
constexpr int kPShift = std::is_same_v<T, __half> ? 14 : 0;
template <typename T>
constexpr bool kScaled = std::is_same_v<T, __half>;
__device__ __forceinline__ float power_for(float bound) {
    if (!(bound > 0.f) || isinf(bound)) return 1.f;
    const int e = (__float_as_int(bound) >> 23) - 126;      // bound < 2^e
    return __int_as_float((127 + min(14 - e, 100)) << 23);
}

struct BwdArgs {
    AttentionArgs p;
    CUtensorMap q, k, v, dout;
    float *stats;      // [q tile][head][stat_rows][128], see there
    float *partial;    // [k tile][head][entries]: dS by distance
    float *values;     // fp16: [k tile][key head]: the length of the longest v
    float *bounds;     // fp16: [q tile][head]: the largest bound of a row's dS
    int doc_tiles;     // new_tokens > 0: q tiles of a document
    int entries;       // bias_entries(reach)
    int q_numbers, k_numbers;   // tile numbers; blocks run over them head by head
};

// Tiles held at a time: of the operand pair a block walks, and of the pair it
// keeps (two: the next work's is loaded while this one's is in use).
constexpr int kWalked = 2;
__host__ __device__ constexpr int kept(int dp) { return dp == 64 ? 2 : 1; }

// Row statistics, 128 to a row: kPShift - lse in base 2; -2^-kPShift delta; in
// fp16 the power of two of its dS.  With a table two more, where the tile has a
// far query (see far_statistics): minus its largest score in base 2 and kPShift -
// log2 of the sum of the 2^(score - largest), zeros for the others.  A far query's
// first one is minus zero: its mark, which changes no sum.  The kernels hold the
// rows up to those two, which are read where they lie.
constexpr int kStats = 2;                                               // what k_attend_dkv holds
__host__ __device__ constexpr int held(bool scaled) { return kStats + (scaled ? 1 : 0); }   // k_attend_dq
__host__ __device__ constexpr int stat_rows(bool scaled, bool bias) { return held(scaled) + (bias ? 2 : 0); }
__device__ __forceinline__ bool is_far(float stat) { return __float_as_uint(stat) == 0x80000000u; }

// The threads that compute meet: bounded like every wait, so a warp that gave
// up leaves none behind.
struct Meeting {
    uint64_t *bar;
    uint32_t phase;
    __device__ __forceinline__ bool operator()(const Waiter &wait) {
        warp_arrive(bar);
        const bool ok = wait.warp(bar, phase);
        phase ^= 1u;
        return ok;
    }
};

// 16 warps compute: four groups of 32 columns (one thread's, read and written
// where they are), four warps to the 128 lanes.
constexpr int kWarps = 16, kGroups = kWarps / 4, kCols = kTile / kGroups;

// One block's work.
struct DqWork {
    int head, q_row, row0, nq, k_row, nk, n, stats;   // head < 0: no more; n: key tiles
};
struct DkvWork {
    int hk, k_row, key0, nk, q_row, nq, q_first, q_tiles, q_number, number;   // hk < 0: no more
    float power;                                                              // of dS
};

// A query all of whose keys have huge biases is far: beside 1e6 an lse in 32 bits
// leaves P off by a percent, beside 1e9 the log of the sum is lost in it and P of
// n keys would be 1 each, not 1 / n.  So its largest score and its sum are made
// anew, each for itself, from scores that are rounded as the forward pass rounds
// them; P = 2^((score - largest) - log2 sum) is exact at any size.  This takes a
// warp a pass over the query's keys without the tensor cores: 1.7 ms for one head
// of 12 that is all huge, on 384 documents of up to 512 tokens.  Biases that a
// model learns stay far below the limit.
constexpr float kFar = 256.f;      // of an lse (off by 2^-17 there) and of a bias in base 2
template <typename T>
__device__ __noinline__ bool far_statistics(const sieve_attention_args &a, const Doc &doc, int head, int qi, float &top,
                                            float &log2_sum) {
    const int lane = lane_id(), d = a.head_dim, place = qi + doc.nk - doc.nq;
    const int seen = a.causal ? min(doc.nk, place + 1) : doc.nk;
    // the largest bias of the keys seen: not huge, and the size is the scores' own
    const int lo = min(max(-place, -a.reach), a.reach), hi = min(max(seen - 1 - place, -a.reach), a.reach);
    float most = -INFINITY;
    for (int i = lo + lane; i <= hi; i += 32) most = fmaxf(most, scaled_bias(a, i, head));
#pragma unroll
    for (int o = 16; o; o >>= 1) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, o));
    if (seen <= 0 || !(fabsf(most) > kFar) || isinf(most)) return false;
    const T *q = static_cast<const T *>(a.q) + (int64_t)(doc.q0 + qi) * a.q_token_stride + head * a.q_head_stride;
    const T *k = static_cast<const T *>(a.k) + head / (a.heads / a.kv_heads) * a.k_head_stride;
    const float c = a.scale * kLog2e;
    float m = -INFINITY, l = 0.f;
    for (int j = lane; j < seen; j += 32) {
        const T *kj = k + (int64_t)(doc.k0 + j) * a.k_token_stride;
        float dot = 0.f;
        for (int i = 0; i < d; i += 8) {
            float x[8], y[8];
            load_vec<T, 8>(q + i, x);
            load_vec<T, 8>(kj + i, y);
#pragma unroll
            for (int e = 0; e < 8; ++e) dot = fmaf(x[e], y[e], dot);
        }
        const float x = fmaf(dot, c, scaled_bias(a, j - place, head));
        if (x == -INFINITY) continue;
        if (x > m) {
            l = fmaf(l, exp2f(m - x), 1.f);
            m = x;
        } else {
            l += exp2f(x - m);
        }
    }
    top = m;
#pragma unroll
    for (int o = 16; o; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
    l = warp_sum(m == -INFINITY ? l : l * exp2f(m - top));
    log2_sum = log2f(l);
    return true;
}

// fp16: the length of the longest v of every tile of keys and key head.
constexpr int kDeltaThreads = 256;
template <typename T, int kLanes>
__global__ void __launch_bounds__(kDeltaThreads) k_attend_values(const __grid_constant__ BwdArgs f) {
    const sieve_attention_args &a = f.p.a;
    __shared__ float s_most[kDeltaThreads / 32];
    const int t = blockIdx.x / a.kv_heads, head = blockIdx.x % a.kv_heads;
    const int s = find_doc(a.k_offsets, (int)a.nseq, (int)a.k_tokens, kTile, t);
    int first, len;
    doc_range(a.k_offsets, s, (int)a.k_tokens, first, len);
    const int r0 = (t - first_tile(a.k_offsets, s, (int)a.k_tokens, kTile)) * kTile;
    if (r0 < 0 || r0 >= len) return;
    const int rows = min(kTile, len - r0), piece = threadIdx.x % kLanes;
    const T *v = static_cast<const T *>(a.v) + (int64_t)(first + r0) * a.v_token_stride + head * a.v_head_stride + piece * 8;
    constexpr int kRows = kDeltaThreads / kLanes;
    float most = 0.f;
#pragma unroll
    for (int i = 0; i < kTile / kRows; ++i) {
        const int r = i * kRows + threadIdx.x / kLanes;
        float x[8], sum = 0.f;
        if (r < rows && piece * 8 < a.head_dim) {
            load_vec<T, 8>(v + (int64_t)r * a.v_token_stride, x);
#pragma unroll
            for (int e = 0; e < 8; ++e) sum = fmaf(x[e], x[e], sum);
        }
#pragma unroll
        for (int k = kLanes / 2; k; k >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, k);
        most = fmaxf(most, sum);
    }
    most = warp_max(most);
    if (lane_id() == 0) s_most[threadIdx.x >> 5] = most;
    __syncthreads();
    if (threadIdx.x >= 32) return;
    most = warp_max(threadIdx.x < kDeltaThreads / 32 ? s_most[threadIdx.x] : 0.f);
    if (threadIdx.x == 0) f.values[(int64_t)t * a.kv_heads + head] = sqrtf(most);
}

// delta = dO . O of every query, and -lse in base 2: a block per tile and head,
// 8 or 16 lanes to a row.  (Inside k_attend_dq, with a row to a thread, the same
// reads took 3K to 9K cycles of every block's time.)
template <typename T, int kLanes, bool BIAS>
__global__ void __launch_bounds__(kDeltaThreads, kScaled<T> ? 6 : 8) k_attend_delta(const __grid_constant__ BwdArgs f) {
    const sieve_attention_args &a = f.p.a;
    if (blockIdx.x == 0 && threadIdx.x == 0) f.p.ctl->status = 0;
    const int t = blockIdx.x / a.heads, head = blockIdx.x % a.heads;
    int s, tile;
    if (a.new_tokens > 0) {
        s = t / f.doc_tiles;
        tile = t % f.doc_tiles;
    } else {
        s = find_doc(a.q_offsets, (int)a.nseq, (int)a.q_tokens, kTile, t);
        tile = t - first_tile(a.q_offsets, s, (int)a.q_tokens, kTile);
    }
    const Doc doc = doc_at(a, s);
    if (tile < 0 || tile * kTile >= doc.nq) return;
    const int64_t row0 = doc.q0 + tile * kTile;
    const int rows = min(kTile, doc.nq - tile * kTile);
    constexpr int kHeld = held(kScaled<T>);
    float *stats = f.stats + ((int64_t)t * a.heads + head) * stat_rows(kScaled<T>, BIAS) * kTile;
    const int piece = threadIdx.x % kLanes, d = a.head_dim;
    const T *o = static_cast<const T *>(f.p.out_in) + (row0 * a.heads + head) * d + piece * 8;
    const T *g = static_cast<const T *>(f.p.dout) + (row0 * a.heads + head) * d + piece * 8;
    constexpr int kRows = kDeltaThreads / kLanes;
    uint32_t may_be_far = 0;      // of this thread's rows, one bit each
    // the document's longest v: its first tiles' are asked for here, and looked at
    // once the rows are in hand
    const int k_tiles = (doc.nk + kTile - 1) / kTile, lane = lane_id();
    const float *values = f.values + (int64_t)(doc.k0 / kTile + s) * a.kv_heads + head / (a.heads / a.kv_heads);
    float longest = kScaled<T> && lane < k_tiles ? values[(int64_t)lane * a.kv_heads] : 0.f, most = 0.f;
    float square[kScaled<T> ? kTile / kRows : 1];
#pragma unroll
    for (int i = 0; i < kTile / kRows; ++i) {
        const int r = i * kRows + threadIdx.x / kLanes;
        float x[8], y[8], part = 0.f, sum = 0.f;
        if (r < rows && piece * 8 < d) {
            load_vec<T, 8>(o + (int64_t)r * a.heads * d, x);
            load_vec<T, 8>(g + (int64_t)r * a.heads * d, y);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                part = fmaf(x[e], y[e], part);
                if (kScaled<T>) sum = fmaf(y[e], y[e], sum);
            }
        }
#pragma unroll
        for (int k = kLanes / 2; k; k >>= 1) {
            part += __shfl_xor_sync(0xffffffffu, part, k);
            if (kScaled<T>) sum += __shfl_xor_sync(0xffffffffu, sum, k);
        }
        if (kScaled<T>) square[i] = sum;
        if (piece == 0) {
            const float lse = r < rows ? f.p.lse_in[(int64_t)head * a.q_tokens + row0 + r] : -INFINITY;
            stats[r] = lse == -INFINITY ? -INFINITY : (float)kPShift<T> - lse * kLog2e + 0.f;   // (no minus zero)
            stats[kTile + r] = -part * (1.f / (float)(1 << kPShift<T>));
            if (BIAS && fabsf(lse) > kFar && !isinf(lse)) may_be_far |= 1u << i;
        }
    }
    if constexpr (kScaled<T>) {
        __shared__ float s_most[kDeltaThreads / 32];
        for (int i = lane + 32; i < k_tiles; i += 32) longest = fmaxf(longest, values[(int64_t)i * a.kv_heads]);
        longest = 2.f * warp_max(longest);
#pragma unroll
        for (int i = 0; i < kTile / kRows; ++i) {
            const float bound = sqrtf(square[i]) * longest;
            most = fmaxf(most, bound);
            if (piece == 0) stats[2 * kTile + i * kRows + threadIdx.x / kLanes] = power_for(bound);
        }
        most = warp_max(most);
        if (lane_id() == 0) s_most[threadIdx.x >> 5] = most;
        __syncthreads();
        if (threadIdx.x == 0) {
#pragma unroll
            for (int k = 1; k < kDeltaThreads / 32; ++k) most = fmaxf(most, s_most[k]);
            f.bounds[(int64_t)t * a.heads + head] = most;
        }
    }
    if (!BIAS || !__syncthreads_or(may_be_far)) return;
    stats[kHeld * kTile + threadIdx.x] = 0.f;
    static_assert(kDeltaThreads == 2 * kTile, "");
    __syncthreads();
#pragma unroll 1
    for (int n = 0; n < kTile / kRows * (32 / kLanes); ++n) {
        const int i = n / (32 / kLanes), from = n % (32 / kLanes) * kLanes;       // row of the warp, its first lane
        const int r = i * kRows + ((int)threadIdx.x / 32 * 32 + from) / kLanes;
        float top, log2_sum;
        if (!(__shfl_sync(0xffffffffu, may_be_far, from) >> i & 1u) ||
            !far_statistics<T>(a, doc, head, tile * kTile + r, top, log2_sum))
            continue;
        if (lane_id() == (uint32_t)from) {
            stats[r] = -0.f;
            stats[kHeld * kTile + r] = -top;
            stats[(kHeld + 1) * kTile + r] = (float)kPShift<T> - log2_sum;
        }
    }
}

template <typename T, int DP, bool BIAS>
__global__ void __launch_bounds__(18 * 32, 1) k_attend_dq(const __grid_constant__ BwdArgs f) {
    constexpr int kB = DP / 64, kKept = kept(DP);
    // K of a step is used twice, last after the next step's scores; V once
    constexpr int kKs = 3, kVs = DP == 64 ? 2 : 1;
    constexpr uint32_t kTileBytes = kB * kBlockBytes;
    constexpr uint32_t kSCol = 0, kDpCol = 128, kDqCol = 384;   // S, dP twice (dS in its place), dQ
    extern __shared__ unsigned char smem_raw[];
    __shared__ __align__(8) uint64_t q_full[kKept], q_empty[kKept], k_full[kKs], k_empty[kKs], v_full[kVs], v_empty[kVs], s_full, s_free,
        dp_full[2], ds_full[2], dq_full, done, work_full[kSlots], work_empty[kSlots], stat_full[kSlots], steal_bar;
    __shared__ __align__(16) uint4 s_answer;
    __shared__ uint32_t tmem_slot;
    __shared__ int s_abort;
    __shared__ DqWork s_work[kSlots];
    __shared__ float s_row[kSlots][kGroups][kTile];     // (a warp may be in the next work already)
    constexpr int kHeld = held(kScaled<T>), kStatRows = stat_rows(kScaled<T>, BIAS);
    __shared__ __align__(16) float s_stats[kSlots][kHeld][kTile];
    const sieve_attention_args &a = f.p.a;
    const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0), lane = lane_id();

    unsigned char *base = reinterpret_cast<unsigned char *>(
        (reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~static_cast<uintptr_t>(1023));
    unsigned char *qd = base, *k_tiles = qd + kKept * 2 * kTileBytes, *v_tiles = k_tiles + kKs * kTileBytes;   // qd: pairs
    float *bias = reinterpret_cast<float *>(v_tiles + kVs * kTileBytes);      // two heads' tables
    const int bias_set = BIAS ? bias_floats(a.reach) : 0;

    if (threadIdx.x == 0) {
        for (int i = 0; i < kKept; ++i) {
            tc::mbar_init(&q_full[i], 1);
            tc::mbar_init(&q_empty[i], 1);
        }
        for (int i = 0; i < kKs; ++i) {
            tc::mbar_init(&k_full[i], 1);
            tc::mbar_init(&k_empty[i], 1);
        }
        for (int i = 0; i < kVs; ++i) {
            tc::mbar_init(&v_full[i], 1);
            tc::mbar_init(&v_empty[i], 1);
        }
        for (int i = 0; i < 2; ++i) {
            tc::mbar_init(&dp_full[i], 1);
            tc::mbar_init(&ds_full[i], kWarps);
            tc::mbar_init(&work_full[i], 1);
            tc::mbar_init(&work_empty[i], kWarps + 1);
            tc::mbar_init(&stat_full[i], 1);
        }
        tc::mbar_init(&s_full, 1);
        tc::mbar_init(&s_free, kWarps);
        tc::mbar_init(&dq_full, 1);
        tc::mbar_init(&done, 1);
        tc::mbar_init(&steal_bar, 1);
        s_abort = 0;
        tc::mbar_init_fence();
    }
    if (warp == 0) tc::tmem_alloc(&tmem_slot, 512);
    tc::fence_before_sync();
    __syncthreads();
    tc::fence_after_sync();
    const uint32_t tmem = __shfl_sync(0xffffffffu, tmem_slot, 0);
    const Waiter wait{&s_abort};

    if (warp == kWarps + 1) {
        // ---------------- the work, one block's after another's, and its loads ----------------
        int block = blockIdx.x, item = 0, stats_issued = 0, kv_issued = 0, k_issued = 0, head0 = -1, head1 = -1;
        Blocks blocks{&s_answer, &steal_bar, 0, false};
        bool ok = true;
        // the next work that has steps (head < 0: none is left); false: a wait
        // gave up
        DocFinder find(a.q_offsets, a.nseq, a.q_tokens);
        auto fetch = [&](DqWork &w, bool own) {
            while (true) {
                if (!own && !blocks.next(wait, block)) return false;
                own = false;
                w.head = -1;
                if (block < 0) return true;
                const int head = block / f.q_numbers, t = block % f.q_numbers;
                int s, tile;
                Doc doc;
                if (a.new_tokens > 0) {
                    s = t / f.doc_tiles;
                    tile = t % f.doc_tiles;
                    doc = doc_at(a, s);
                } else {
                    find(t, s, doc.q0, doc.nq, tile);
                    keys_of(a, s, doc);
                }
                const int tiles = (doc.nq + kTile - 1) / kTile;
                if (tile < 0 || tile >= tiles) continue;
                const int number0 = t - tile;          // the document's first
                tile = tiles - 1 - tile;               // the tiles that see most keys first
                w.head = head;
                w.q_row = doc.q0;
                w.row0 = tile * kTile;
                w.nq = doc.nq;
                w.k_row = doc.k0;
                w.nk = doc.nk;
                const int last = min(doc.nq, w.row0 + kTile);
                const int end = a.causal ? min(doc.nk, last + doc.nk - doc.nq) : doc.nk;
                w.n = end > 0 ? (end + kTile - 1) / kTile : 0;
                w.stats = (number0 + tile) * a.heads + head;
                if (w.n > 0) {
                    if (w.n <= kShort) blocks.ask();
                    return true;
                }
                // no query of these sees a key
                const int pieces = a.head_dim / 8;
#pragma unroll 1
                for (int i = lane; i < (last - w.row0) * pieces; i += 32)
                    *reinterpret_cast<uint4 *>(static_cast<T *>(f.p.dq) + (int64_t)(doc.q0 + w.row0 + i / pieces) * f.p.dq_ts +
                                               head * f.p.dq_hs + i % pieces * 8) = make_uint4(0, 0, 0, 0);
            }
        };
        DqWork w;
        ok = fetch(w, true);
        while (ok && w.head >= 0) {
            const int slot = item % kSlots, qs = item % kKept, head = w.head, hk = head / (a.heads / a.kv_heads);
            if (item >= kSlots && !(ok = wait.warp(&work_empty[slot], (uint32_t)(item / kSlots - 1) & 1u))) break;
            // a slot has its own bias table, done with when the slot is
            if (BIAS && head != (slot ? head1 : head0)) {
                fill_bias(bias + slot * bias_set, a, head, 1, lane, 32);
                (slot ? head1 : head0) = head;
            }
            if (lane == 0) s_work[slot] = w;
            __syncwarp();
            if (lane == 0) tc::mbar_arrive(&work_full[slot]);
            // The row statistics complete on a barrier of their slot: every warp
            // has read them, and so passed it, before the slot is free again.
            // (q_full is no barrier for those warps: with one pair held the
            // products alone let the next pair in, and a warp that had not
            // looked yet would find its phase gone.)
            if (elected()) {
                expect(&stat_full[slot], kHeld * kTile * 4);
                tc::bulk_g2s(1u, s_stats[slot], f.stats + (int64_t)w.stats * kStatRows * kTile, kHeld * kTile * 4,
                             &stat_full[slot]);
            }
            __syncwarp();
            ++stats_issued;
            if (!(ok = wait.warp(&q_empty[qs], ((uint32_t)(item / kKept) & 1u) ^ 1u))) break;
            if (elected()) {
                expect(&q_full[qs], 2 * kTileBytes);
                for (int b = 0; b < kB; ++b) {
                    tma_load(qd + qs * 2 * kTileBytes + b * kBlockBytes, &f.q, 64 * b, head, w.q_row + w.row0, &q_full[qs]);
                    tma_load(qd + (qs * 2 + 1) * kTileBytes + b * kBlockBytes, &f.dout, 64 * b, head, w.q_row + w.row0,
                             &q_full[qs]);
                }
            }
            __syncwarp();
            ++item;
            // The next work is looked for while the first steps of this one
            // run.  Not so early for long work: others may be done sooner.
            DqWork then;
            const int when = w.n <= kShort ? min(w.n, 2) : w.n;
#pragma unroll 1
            for (int j = 0; j < w.n; ++j) {
                const int ks = kv_issued % kKs, vs = kv_issued % kVs, row = w.k_row + j * kTile;
                if (!(ok = wait.warp(&k_empty[ks], ((uint32_t)(kv_issued / kKs) & 1u) ^ 1u))) break;
                if (elected()) {
                    expect(&k_full[ks], kTileBytes);
                    for (int b = 0; b < kB; ++b)
                        tma_load(k_tiles + ks * kTileBytes + b * kBlockBytes, &f.k, 64 * b, hk, row, &k_full[ks]);
                }
                __syncwarp();
                k_issued = kv_issued + 1;
                if (!(ok = wait.warp(&v_empty[vs], ((uint32_t)(kv_issued / kVs) & 1u) ^ 1u))) break;
                if (elected()) {
                    expect(&v_full[vs], kTileBytes);
                    for (int b = 0; b < kB; ++b)
                        tma_load(v_tiles + vs * kTileBytes + b * kBlockBytes, &f.v, 64 * b, hk, row, &v_full[vs]);
                }
                __syncwarp();
                ++kv_issued;
                if (j + 1 == when && !(ok = fetch(then, false))) break;
            }
            if (!ok) break;
            w = then;
        }
        if (ok) {
            const int slot = item % kSlots;
            ok = item < kSlots || wait.warp(&work_empty[slot], (uint32_t)(item / kSlots - 1) & 1u);
            if (lane == 0) {
                s_work[slot].head = -1;
                tc::mbar_arrive(&work_full[slot]);
            }
        }
        if (!ok) {
            // after an abort: what is in flight lands before the block ends
            if (blocks.asking) let_land(&steal_bar, blocks.asked & 1u);
            for (int i = max(0, stats_issued - kSlots); i < stats_issued; ++i)
                let_land(&stat_full[i % kSlots], (uint32_t)(i / kSlots) & 1u);
            for (int i = max(0, item - kKept); i < item; ++i) let_land(&q_full[i % kKept], (uint32_t)(i / kKept) & 1u);
            for (int i = max(0, k_issued - kKs); i < k_issued; ++i) let_land(&k_full[i % kKs], (uint32_t)(i / kKs) & 1u);
            for (int i = max(0, kv_issued - kVs); i < kv_issued; ++i) let_land(&v_full[i % kVs], (uint32_t)(i / kVs) & 1u);
        }
        __syncwarp();
    } else if (warp == kWarps) {
        // ---------------- products ----------------
        constexpr uint32_t id_s = idesc<T>(kTile, false), id_o = idesc<T>(DP, true);
        constexpr uint32_t kPair = 2 * kTileBytes >> 4, kTileStep = kTileBytes >> 4;   // in a descriptor's units
        const uint64_t q0 = desc_k(qd), kk0 = desc_k(k_tiles), km0 = desc_mn(k_tiles), v0 = desc_k(v_tiles);
        uint32_t step = 0;
        bool ok = true;
        for (int item = 0; ok; ++item) {
            const int slot = item % kSlots;
            if (!(ok = wait.warp(&work_full[slot], (uint32_t)(item / kSlots) & 1u))) break;
            if (uniform(s_work[slot].head) < 0) break;
            const int n = uniform(s_work[slot].n), nk = uniform(s_work[slot].nk);
            const uint64_t qa = q0 + item % kKept * kPair;
            if (!(ok = wait.warp(&q_full[item % kKept], (uint32_t)(item / kKept) & 1u))) break;
            // round j: the scores of step j + 1 as soon as those of step j are
            // in registers; when dS of step j is there, dP of step j + 1, then
            // dQ of step j
#pragma unroll 1
            for (int j = -1; j < n; ++j) {
                const uint32_t i = step + (j < 0 ? 0u : 1u), ks = i % kKs, vs = i % kVs;
                const bool more = j + 1 < n;
                const int left = nk - (j + 1) * kTile;
                if (more) {
                    if (!(ok = wait.warp(&k_full[ks], (i / kKs) & 1u))) break;
                    // rows of another document: 0 x NaN in dS K
                    if (left < kTile) clear_rows(k_tiles + ks * kTileBytes, left, kB);
                    if (!(ok = wait.warp(&s_free, (i & 1u) ^ 1u))) break;
                    tc::fence_after_sync();
                    if (elected()) {
                        mma_kk<DP>(tmem + kSCol, qa, kk0 + ks * kTileStep, id_s);
                        commit(&s_full);
                    }
                    __syncwarp();
                }
                if (j >= 0 && !(ok = wait.warp(&ds_full[step & 1u], (step >> 1) & 1u))) break;
                if (more) {
                    if (!(ok = wait.warp(&v_full[vs], (i / kVs) & 1u))) break;
                    // and NaN in dP
                    if (left < kTile) clear_rows(v_tiles + vs * kTileBytes, left, kB);
                }
                tc::fence_after_sync();
                if (elected()) {
                    if (more) {
                        mma_kk<DP>(tmem + kDpCol + (i & 1u) * kTile, qa + kTileStep, v0 + vs * kTileStep, id_s);
                        commit(&dp_full[i & 1u]);
                        commit(&v_empty[vs]);
                        if (j + 2 == n) commit(&q_empty[item % kKept]);
                    }
                    if (j >= 0) {
                        mma_groups<kCols, kCols>(tmem + kDqCol, tmem + kDpCol + (step & 1u) * kTile,
                                                 km0 + step % kKs * kTileStep, id_o, j > 0);
                        commit(&k_empty[step % kKs]);
                        if (!more) commit(&dq_full);
                    }
                }
                __syncwarp();
                if (j >= 0) ++step;
            }
            if (ok && lane == 0) tc::mbar_arrive(&work_empty[slot]);
        }
        // every product issued ends before the block frees its memory (waited
        // for even after an abort, within the poll limit)
        if (elected()) commit(&done);
        __syncwarp();
        let_land(&done, 0);
        __syncwarp();
    } else {
        // ---------------- P, dS and dQ ----------------
        const int quarter = warp & 3, group = warp >> 2;
        const int r = quarter * 32 + lane, d = a.head_dim;
        const float c = a.scale * kLog2e;
        const uint32_t lane_base = tmem + ((uint32_t)(quarter * 32) << 16);
        uint32_t step = 0;
        bool ok = true;
#pragma unroll 1
        for (int item = 0; ok; ++item) {
            const int slot = item % kSlots;
            if (!(ok = wait.warp(&work_full[slot], (uint32_t)(item / kSlots) & 1u))) break;
            const DqWork &w = s_work[slot];
            if (w.head < 0) break;
            const bool live = w.row0 + r < w.nq, idle = w.row0 + quarter * 32 >= w.nq;
            const int place0 = w.row0 + quarter * 32 + w.nk - w.nq, place = place0 + lane;
            const int seen = (live ? (a.causal ? min(w.nk, place + 1) : w.nk) : 0) - group * kCols;
            const int64_t row = w.q_row + w.row0 + r;
            const float *table = bias + slot * bias_set;
            if (!(ok = wait.warp(&stat_full[slot], (uint32_t)(item / kSlots) & 1u))) break;
            const bool far = BIAS && is_far(s_stats[slot][0][r]), any_far = BIAS && __any_sync(0xffffffffu, far);
            const float nl = far ? 0.f : s_stats[slot][0][r] - (float)kPShift<T>;
            float *const stats = f.stats + (int64_t)w.stats * kStatRows * kTile + r;    // this row's
            const float power = kScaled<T> ? s_stats[slot][kHeld - 1][r] : 1.f;
            const float minus_delta = s_stats[slot][1][r] * (float)(1 << kPShift<T>);
            float2 sum2 = both(0.f);
#pragma unroll 1
            for (int j = 0; j < w.n; ++j, ++step) {
                if (!(ok = wait.warp(&s_full, step & 1u))) break;
                const uint32_t dp_at = lane_base + kDpCol + (step & 1u) * kTile + group * kCols;
                tc::fence_after_sync();
                const int vis = seen - j * kTile;                    // columns of the group that this row sees
                const bool all = __all_sync(0xffffffffu, vis >= kCols);
                const bool none = idle || (!all && __reduce_max_sync(0xffffffffu, vis) <= 0);
                uint32_t pk[kCols / 2];
                float2 x[kCols / 2];
                if (!none) {
                    uint32_t raw[32];
                    tc::tmem_ld32_issue(lane_base + kSCol + group * kCols, raw);
                    tc::tmem_ld_wait(raw);
#pragma unroll
                    for (int e = 0; e < 16; ++e) x[e] = make_float2(__uint_as_float(raw[2 * e]), __uint_as_float(raw[2 * e + 1]));
                }
                tc::fence_before_sync();
                warp_arrive(&s_free);
                if (!none) {
                    const int d0 = j * kTile + group * kCols;
                    const bool after = d0 - place0 - 31 >= a.reach, before = d0 + 31 - place0 <= -a.reach;
                    if (!BIAS || after || before) {
                        const float b = nl + (BIAS ? table[bias_zero(a.reach) + (after ? a.reach : -a.reach)] : 0.f);
#pragma unroll
                        for (int e = 0; e < 16; ++e) x[e] = fma2(x[e], both(c), both(b));
                    } else {
                        const float4 *at = bias_at(table, a.reach, d0 - place);
#pragma unroll
                        for (int e = 0; e < 8; ++e) {
                            const float4 b = at[e];
                            x[2 * e] = fma2(x[2 * e], both(c), add2(make_float2(b.x, b.y), both(nl)));
                            x[2 * e + 1] = fma2(x[2 * e + 1], both(c), add2(make_float2(b.z, b.w), both(nl)));
                        }
                    }
                    if (any_far) {
                        const float top = far ? stats[kHeld * kTile] : 0.f;
                        const float rest = far ? stats[(kHeld + 1) * kTile] - (float)kPShift<T> : 0.f;
#pragma unroll
                        for (int e = 0; e < 16; ++e) x[e] = add2(add2(x[e], both(top)), both(rest));
                    }
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        x[e].x = exp2_approx(x[e].x);
                        x[e].y = exp2_approx(x[e].y);
                    }
                    if (!all) {
#pragma unroll
                        for (int e = 0; e < 16; ++e) {
                            if (2 * e >= vis) x[e].x = 0.f;
                            if (2 * e + 1 >= vis) x[e].y = 0.f;
                        }
                    }
                }
                if (!(ok = wait.warp(&dp_full[step & 1u], (step >> 1) & 1u))) break;
                tc::fence_after_sync();
                if (!none) {
                    float dp[32];
                    tc::tmem_ld32(dp_at, dp);
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        x[e] = mul2(x[e], add2(make_float2(dp[2 * e], dp[2 * e + 1]), both(minus_delta)));
                        if (BIAS) sum2 = add2(sum2, x[e]);
                        const float2 y = kScaled<T> ? mul2(x[e], both(power)) : x[e];
                        pk[e] = pack2<T>(y.x, y.y);
                    }
                } else {
                    // no row of the warp sees these; the product reads them
#pragma unroll
                    for (int e = 0; e < 16; ++e) pk[e] = 0u;
                }
                tc::tmem_st16(dp_at, pk);
                tc::tmem_st_wait();
                if (BIAS && j == w.n - 1) s_row[slot][group][r] = sum2.x + sum2.y;
                tc::fence_before_sync();
                // (a warp may be a step ahead of another here: the scores of the
                // next step wait for all to have read this one's, not for dS)
                warp_arrive(&ds_full[step & 1u]);
            }
            if (!ok) break;
            // (every thread's sum of dS arrived with its last dS)
            if (!(ok = wait.warp(&ds_full[(step - 1) & 1u], ((step - 1) >> 1) & 1u) && wait.warp(&dq_full, (uint32_t)item & 1u))) break;
            tc::fence_after_sync();
            if (!idle) {
                constexpr int kOut = DP / kGroups;       // 16 or 32 columns of dQ
                const int col = group * kOut;
                uint4 c[kOut / 8];
                const float back = kScaled<T> ? a.scale / power : a.scale;
#pragma unroll
                for (int i = 0; i < kOut / 16; ++i) {
                    uint32_t o[16];
                    tmem_ld16(lane_base + kDqCol + col + 16 * i, o);
                    float v[16];
#pragma unroll
                    for (int e = 0; e < 16; ++e) v[e] = nl != -INFINITY ? __uint_as_float(o[e]) * back : 0.f;
                    c[2 * i] = pack8<T>(v);
                    c[2 * i + 1] = pack8<T>(v + 8);
                }
                store_rows(static_cast<T *>(f.p.dq) + (row - lane) * f.p.dq_ts + w.head * f.p.dq_hs + col, f.p.dq_ts,
                           w.nq - w.row0 - quarter * 32, d - col, c);
            }
            tc::fence_before_sync();
            if (BIAS && group == 0 && nl != -INFINITY) {
                // the exact delta, for k_attend_dkv
                float sum = 0.f;
#pragma unroll
                for (int k = 0; k < kGroups; ++k) sum += s_row[slot][k][r];
                stats[kTile] = (minus_delta - sum) * (1.f / (float)(1 << kPShift<T>));
            }
            __syncwarp();
            if (lane == 0) tc::mbar_arrive(&work_empty[slot]);
        }
    }
    tc::fence_before_sync();
    __syncthreads();
    if (threadIdx.x == 0 && s_abort) atomicExch(&f.p.ctl->status, SIEVE_ETIMEOUT);
    if (warp == 0) {
        tc::fence_after_sync();
        tc::tmem_dealloc(tmem, 512);
    }
}

// Sets of sums by distance: one for each group of columns and for its even and
// its odd quarters of keys.  The pieces (32 keys by 32 queries) that meet in a
// set lie a multiple of 64 distances apart, over all steps of a head, so the 63
// distances of a piece are its own: it stores its sums, and no order matters.
// Where there is room the sets are there twice, and the next head's are another
// than the ones being added up.
constexpr int kSums = 8;
__host__ __device__ constexpr int sum_sets(int dp) { return dp == 64 ? 2 : 1; }

template <typename T, int DP, bool BIAS>
__global__ void __launch_bounds__(18 * 32, 1) k_attend_dkv(const __grid_constant__ BwdArgs f) {
    constexpr int kCompute = kWarps * 32;
    static_assert(kSums == 2 * kGroups, "");
    constexpr int kB = DP / 64, kKept = kept(DP), kSumSets = sum_sets(DP);
    constexpr uint32_t kTileBytes = kB * kBlockBytes;
    constexpr uint32_t kSCol = 0, kDpCol = 128, kDvCol = 256, kDkCol = 384;   // P in S's place, dS in dP's
    extern __shared__ unsigned char smem_raw[];
    constexpr int kStatRows = stat_rows(kScaled<T>, BIAS);
    __shared__ __align__(16) float s_stats[kWalked][kStats][kTile];
    __shared__ __align__(8) uint64_t kv_full[kKept], kv_empty[kKept], q_full[kWalked], q_empty[kWalked], s_full, p_full,
        dp_full, ds_full, acc_full, meet_bar, done, work_full[kSlots], work_empty[kSlots], steal_bar;
    __shared__ __align__(16) uint4 s_answer;
    __shared__ uint32_t tmem_slot;
    __shared__ int s_abort;
    __shared__ DkvWork s_work[kSlots];
    __shared__ float s_far[kSumSets][kWarps][2];
    const sieve_attention_args &a = f.p.a;
    const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0), lane = lane_id();
    const int share = a.heads / a.kv_heads;

    unsigned char *base = reinterpret_cast<unsigned char *>(
        (reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~static_cast<uintptr_t>(1023));
    unsigned char *kv = base, *qd = kv + kKept * 2 * kTileBytes;      // pairs: K and V, Q and dO
    float *bias = reinterpret_cast<float *>(qd + kWalked * 2 * kTileBytes);
    // the bias by minus the distance (columns run that way)
    constexpr int kCopies = DP == 64 ? 4 : 1;
    float *by_distance = bias + (BIAS ? bias_floats(a.reach, kCopies) : 0);   // [kSumSets][kSums][entries]

    if (threadIdx.x == 0) {
        if (blockIdx.x == 0 && a.q_tokens == 0) f.p.ctl->status = 0;      // (else k_attend_delta did)
        for (int i = 0; i < kKept; ++i) {
            tc::mbar_init(&kv_full[i], 1);
            tc::mbar_init(&kv_empty[i], 1);
        }
        for (int i = 0; i < kWalked; ++i) {
            tc::mbar_init(&q_full[i], 1);
            tc::mbar_init(&q_empty[i], 1);
        }
        for (int i = 0; i < kSlots; ++i) {
            tc::mbar_init(&work_full[i], 1);
            tc::mbar_init(&work_empty[i], kWarps + 1);
        }
        tc::mbar_init(&s_full, 1);
        tc::mbar_init(&p_full, kWarps);
        tc::mbar_init(&dp_full, 1);
        tc::mbar_init(&ds_full, kWarps);
        tc::mbar_init(&acc_full, 1);
        tc::mbar_init(&meet_bar, kWarps);
        tc::mbar_init(&done, 1);
        tc::mbar_init(&steal_bar, 1);
        s_abort = 0;
        tc::mbar_init_fence();
    }
    if (warp == 0) tc::tmem_alloc(&tmem_slot, 512);
    tc::fence_before_sync();
    __syncthreads();
    tc::fence_after_sync();
    const uint32_t tmem = __shfl_sync(0xffffffffu, tmem_slot, 0);
    const Waiter wait{&s_abort};

    if (warp == kWarps + 1) {
        // ---------------- the work, one block's after another's, and its loads ----------------
        int block = blockIdx.x, item = 0, q_issued = 0;
        Blocks blocks{&s_answer, &steal_bar, 0, false};
        bool ok = true;
        // the next work that has steps (hk < 0: none is left); false: a wait
        // gave up
        DocFinder find(a.k_offsets, a.nseq, a.k_tokens);
        auto fetch = [&](DkvWork &w, bool own) {
            while (true) {
                if (!own && !blocks.next(wait, block)) return false;
                own = false;
                w.hk = -1;
                if (block < 0) return true;
                const int hk = block / f.k_numbers;
                w.number = block % f.k_numbers;
                int s, tile;
                Doc doc;
                find(w.number, s, doc.k0, doc.nk, tile);
                queries_of(a, s, doc);
                w.key0 = tile * kTile;
                const bool used = tile >= 0 && w.key0 < doc.nk;
                // the first tile of queries that sees any of these keys
                w.q_first = a.causal ? max(0, w.key0 - (doc.nk - doc.nq)) / kTile : 0;
                w.q_tiles = used ? max(0, (doc.nq + kTile - 1) / kTile - w.q_first) : 0;
                if (w.q_tiles > 0) {
                    w.hk = hk;
                    w.k_row = doc.k0;
                    w.nk = doc.nk;
                    w.q_row = doc.q0;
                    w.nq = doc.nq;
                    w.q_number = a.new_tokens > 0 ? s * f.doc_tiles : doc.q0 / kTile + s;
                    if (kScaled<T>) {
                        float most = 0.f;
                        for (int i = lane; i < w.q_tiles * share; i += 32)
                            most = fmaxf(most, f.bounds[(int64_t)(w.q_number + w.q_first + i / share) * a.heads + hk * share +
                                                        i % share]);
                        w.power = power_for(warp_max(most));
                    }
                    if (w.q_tiles * share <= kShort) blocks.ask();
                    return true;
                }
                // no query sees these keys, or no document uses the number:
                // nothing for the table, and zeros for the keys
#pragma unroll 1
                for (int e = lane; e < share * f.entries; e += 32)
                    f.partial[((int64_t)w.number * a.heads + hk * share) * f.entries + e] = 0.f;
                const int pieces = a.head_dim / 8;
#pragma unroll 1
                for (int i = lane; used && i < min(kTile, doc.nk - w.key0) * pieces; i += 32) {
                    const int64_t row = doc.k0 + w.key0 + i / pieces;
                    *reinterpret_cast<uint4 *>(static_cast<T *>(f.p.dk) + row * f.p.dk_ts + hk * f.p.dk_hs + i % pieces * 8) =
                        make_uint4(0, 0, 0, 0);
                    *reinterpret_cast<uint4 *>(static_cast<T *>(f.p.dv) + row * f.p.dv_ts + hk * f.p.dv_hs + i % pieces * 8) =
                        make_uint4(0, 0, 0, 0);
                }
            }
        };
        DkvWork w;
        ok = fetch(w, true);
        while (ok && w.hk >= 0) {
            const int slot = item % kSlots, ks = item % kKept;
            if (item >= kSlots && !(ok = wait.warp(&work_empty[slot], (uint32_t)(item / kSlots - 1) & 1u))) break;
            if (lane == 0) {
                s_work[slot] = w;
                tc::mbar_arrive(&work_full[slot]);
            }
            if (!(ok = wait.warp(&kv_empty[ks], ((uint32_t)(item / kKept) & 1u) ^ 1u))) break;
            if (elected()) {
                expect(&kv_full[ks], 2 * kTileBytes);
                for (int b = 0; b < kB; ++b) {
                    tma_load(kv + ks * 2 * kTileBytes + b * kBlockBytes, &f.k, 64 * b, w.hk, w.k_row + w.key0, &kv_full[ks]);
                    tma_load(kv + (ks * 2 + 1) * kTileBytes + b * kBlockBytes, &f.v, 64 * b, w.hk, w.k_row + w.key0, &kv_full[ks]);
                }
            }
            __syncwarp();
            ++item;
            // (the next work is looked for as in k_attend_dq)
            DkvWork then;
            const int n = w.q_tiles * share, when = n <= kShort ? min(n, 2) : n;
            int head = w.hk * share, qt = w.q_first;
#pragma unroll 1
            for (int i = 0; i < n; ++i) {
                const int st = q_issued % kWalked, row = w.q_row + qt * kTile;
                if (!(ok = wait.warp(&q_empty[st], ((uint32_t)(q_issued / kWalked) & 1u) ^ 1u))) break;
                if (elected()) {
                    expect(&q_full[st], 2 * kTileBytes + kStats * kTile * 4);
                    for (int b = 0; b < kB; ++b) {
                        tma_load(qd + st * 2 * kTileBytes + b * kBlockBytes, &f.q, 64 * b, head, row, &q_full[st]);
                        tma_load(qd + (st * 2 + 1) * kTileBytes + b * kBlockBytes, &f.dout, 64 * b, head, row, &q_full[st]);
                    }
                    tc::bulk_g2s(1u, s_stats[st], f.stats + ((int64_t)(w.q_number + qt) * a.heads + head) * kStatRows * kTile,
                                 kStats * kTile * 4, &q_full[st]);
                }
                __syncwarp();
                ++q_issued;
                if (++qt == w.q_first + w.q_tiles) {
                    qt = w.q_first;
                    ++head;
                }
                if (i + 1 == when && !(ok = fetch(then, false))) break;
            }
            if (!ok) break;
            w = then;
        }
        if (ok) {
            const int slot = item % kSlots;
            ok = item < kSlots || wait.warp(&work_empty[slot], (uint32_t)(item / kSlots - 1) & 1u);
            if (lane == 0) {
                s_work[slot].hk = -1;
                tc::mbar_arrive(&work_full[slot]);
            }
        }
        if (!ok) {
            // after an abort: what is in flight lands before the block ends
            if (blocks.asking) let_land(&steal_bar, blocks.asked & 1u);
            for (int i = max(0, item - kKept); i < item; ++i) let_land(&kv_full[i % kKept], (uint32_t)(i / kKept) & 1u);
            for (int i = max(0, q_issued - kWalked); i < q_issued; ++i)
                let_land(&q_full[i % kWalked], (uint32_t)(i / kWalked) & 1u);
        }
        __syncwarp();
    } else if (warp == kWarps) {
        // ---------------- products ----------------
        constexpr uint32_t id_s = idesc<T>(kTile, false), id_o = idesc<T>(DP, true);
        constexpr uint32_t kPair = 2 * kTileBytes >> 4, kSecond = kTileBytes >> 4;   // in a descriptor's units
        const uint64_t k0 = desc_k(kv), qk0 = desc_k(qd), qm0 = desc_mn(qd);
        uint32_t step = 0;
        bool ok = true;
        for (int item = 0; ok; ++item) {
            const int slot = item % kSlots;
            if (!(ok = wait.warp(&work_full[slot], (uint32_t)(item / kSlots) & 1u))) break;
            const DkvWork &w = s_work[slot];
            if (uniform(w.hk) < 0) break;
            const int q_tiles = uniform(w.q_tiles), n = q_tiles * share;
            const int left0 = uniform(w.nq - w.q_first * kTile);       // queries from the first tile on
            const uint64_t ka = k0 + item % kKept * kPair;
            if (!(ok = wait.warp(&kv_full[item % kKept], (uint32_t)(item / kKept) & 1u))) break;
            int left = left0, qt = 0;
            // round j: dV of step j, the scores of step j + 1, dK of step j,
            // dP of step j + 1
#pragma unroll 1
            for (int j = -1; j < n; ++j) {
                const bool more = j + 1 < n;
                const uint32_t i = step + (j < 0 ? 0u : 1u), st = i % kWalked, now = step % kWalked;
                if (j >= 0) {
                    if (!(ok = wait.warp(&p_full, step & 1u))) break;
                    tc::fence_after_sync();
                    if (elected())
                        mma_groups<kCols, kCols>(tmem + kDvCol, tmem + kSCol, qm0 + now * kPair + kSecond, id_o, j > 0);
                    __syncwarp();
                }
                if (more) {
                    if (!(ok = wait.warp(&q_full[st], (i / kWalked) & 1u))) break;
                    if (left < kTile) {
                        // rows of another document: their P and dS must be zeros
                        clear_rows(qd + st * 2 * kTileBytes, left, kB);
                        clear_rows(qd + (st * 2 + 1) * kTileBytes, left, kB);
                    }
                    left -= kTile;
                    if (++qt == q_tiles) {
                        qt = 0;
                        left = left0;
                    }
                    tc::fence_after_sync();
                    if (elected()) {
                        mma_kk<DP>(tmem + kSCol, ka, qk0 + st * kPair, id_s);
                        commit(&s_full);
                    }
                    __syncwarp();
                }
                if (j >= 0) {
                    if (!(ok = wait.warp(&ds_full, step & 1u))) break;
                    tc::fence_after_sync();
                    if (elected()) {
                        mma_groups<kCols, kCols>(tmem + kDkCol, tmem + kDpCol, qm0 + now * kPair, id_o, j > 0);
                        commit(&q_empty[now]);
                        if (!more) commit(&acc_full);
                    }
                    __syncwarp();
                    ++step;
                }
                if (more) {
                    if (elected()) {
                        mma_kk<DP>(tmem + kDpCol, ka + kSecond, qk0 + st * kPair + kSecond, id_s);
                        commit(&dp_full);
                        if (j + 2 == n) commit(&kv_empty[item % kKept]);
                    }
                    __syncwarp();
                }
            }
            if (ok && lane == 0) tc::mbar_arrive(&work_empty[slot]);
        }
        // every product issued ends before the block frees its memory (waited
        // for even after an abort, within the poll limit)
        if (elected()) commit(&done);
        __syncwarp();
        let_land(&done, 0);
        __syncwarp();
    } else {
        // ---------------- P, dS, dK and dV ----------------
        const int quarter = warp & 3, group = warp >> 2;
        const int r = quarter * 32 + lane, d = a.head_dim;
        const float c = a.scale * kLog2e;
        const uint32_t lane_base = tmem + ((uint32_t)(quarter * 32) << 16);
        // the group's sums of even or of odd quarters (see kSums)
        float *mine = by_distance + (2 * group + (quarter & 1)) * f.entries;
        const int set_size = kSums * f.entries;
        int set = 0;
        constexpr float kDown = 1.f / (float)(1 << kPShift<T>);
        Meeting meet{&meet_bar, 0};
        uint32_t step = 0;
        int head_in_table = -1;
        bool ok = true;
#pragma unroll 1
        for (int item = 0; ok; ++item) {
            const int slot = item % kSlots;
            if (!(ok = wait.warp(&work_full[slot], (uint32_t)(item / kSlots) & 1u))) break;
            const DkvWork &w = s_work[slot];
            if (w.hk < 0) break;
            const int key = w.key0 + r, key_lo = w.key0 + quarter * 32, shift = w.nk - w.nq;
            const bool live = key < w.nk, idle = key_lo >= w.nk;
#pragma unroll 1
            for (int g = 0; ok && g < share; ++g) {
                const int head = w.hk * share + g;
                float far_before = 0.f, far_after = 0.f;
                if (BIAS) {
                    // another head's bias (the last head's was last read before
                    // the warps met)
                    if (head != head_in_table) {
                        fill_bias<kCopies>(bias, a, head, -1, threadIdx.x, kCompute);
                        if (head_in_table < 0)
                            for (int e = threadIdx.x; e < kSumSets * set_size; e += kCompute) by_distance[e] = 0.f;
                        head_in_table = head;
                        if (!(ok = meet(wait))) break;
                    }
                }
#pragma unroll 1
                for (int qt = w.q_first; qt < w.q_first + w.q_tiles; ++qt, ++step) {
                    const uint32_t st = step % kWalked;
                    const int col0 = qt * kTile + group * kCols;              // the group's first query
                    const int place0 = col0 + shift;
                    // columns before `from` do not see this key, nor those
                    // past the document's queries
                    const int from = a.causal ? key - place0 : 0;
                    if (!(ok = wait.warp(&q_full[st], (step / kWalked) & 1u))) break;   // the row statistics
                    if (!(ok = wait.warp(&s_full, step & 1u))) break;
                    tc::fence_after_sync();
                    const bool none = idle || col0 >= w.nq || (a.causal && key_lo - place0 >= kCols);
                    float2 p[kCols / 2];
                    uint32_t pk[kCols / 2];
                    if (!none) {
                        uint32_t raw[32];
                        tc::tmem_ld32_issue(lane_base + kSCol + group * kCols, raw);
                        const float4 *nl = reinterpret_cast<const float4 *>(&s_stats[st][0][group * kCols]);
                        const int hi = key_lo + 31 - place0, lo = hi - 62;
                        const bool any_far =
                            BIAS && __any_sync(0xffffffffu, is_far(s_stats[st][0][group * kCols + lane]));
                        tc::tmem_ld_wait(raw);
                        if (!BIAS || lo >= a.reach || hi <= -a.reach) {
                            const float b =
                                !BIAS ? 0.f : bias[bias_zero(a.reach) + (lo >= a.reach ? -a.reach : a.reach)];
#pragma unroll
                            for (int e = 0; e < 8; ++e) {
                                const float4 x = nl[e];
                                float2 x0 = make_float2(x.x, x.y), x1 = make_float2(x.z, x.w);
                                if (BIAS) {
                                    x0 = add2(x0, both(b));
                                    x1 = add2(x1, both(b));
                                }
                                p[2 * e] = fma2(make_float2(__uint_as_float(raw[4 * e]), __uint_as_float(raw[4 * e + 1])), both(c), x0);
                                p[2 * e + 1] = fma2(make_float2(__uint_as_float(raw[4 * e + 2]), __uint_as_float(raw[4 * e + 3])), both(c), x1);
                            }
                        } else {
                            const int first = place0 - key;
                            const float4 *at = bias_at(bias, a.reach, first);
                            const float *one = bias + bias_zero(a.reach) + first;
#pragma unroll
                            for (int e = 0; e < 8; ++e) {
                                const float4 x = nl[e];
                                const float4 b = kCopies == 4 ? at[e] : make_float4(one[4 * e], one[4 * e + 1], one[4 * e + 2], one[4 * e + 3]);
                                p[2 * e] = fma2(make_float2(__uint_as_float(raw[4 * e]), __uint_as_float(raw[4 * e + 1])), both(c),
                                                   add2(make_float2(x.x, x.y), make_float2(b.x, b.y)));
                                p[2 * e + 1] = fma2(make_float2(__uint_as_float(raw[4 * e + 2]), __uint_as_float(raw[4 * e + 3])), both(c),
                                                       add2(make_float2(x.z, x.w), make_float2(b.z, b.w)));
                            }
                        }
                        if (any_far) {
                            const float *top = f.stats + held(kScaled<T>) * kTile + group * kCols + lane +
                                               ((int64_t)(w.q_number + qt) * a.heads + head) * kStatRows * kTile;
                            const float t = top[0], u = top[kTile];
#pragma unroll
                            for (int e = 0; e < 16; ++e) {
                                p[e].x = (p[e].x + __shfl_sync(0xffffffffu, t, 2 * e)) + __shfl_sync(0xffffffffu, u, 2 * e);
                                p[e].y = (p[e].y + __shfl_sync(0xffffffffu, t, 2 * e + 1)) + __shfl_sync(0xffffffffu, u, 2 * e + 1);
                            }
                        }
#pragma unroll
                        for (int e = 0; e < 16; ++e) {
                            p[e].x = exp2_approx(p[e].x);
                            p[e].y = exp2_approx(p[e].y);
                        }
                        if (a.causal && !__all_sync(0xffffffffu, from <= 0)) {
#pragma unroll
                            for (int e = 0; e < 16; ++e) {
                                if (2 * e < from) p[e].x = 0.f;
                                if (2 * e + 1 < from) p[e].y = 0.f;
                            }
                        }
#pragma unroll
                        for (int e = 0; e < 16; ++e) pk[e] = pack2<T>(p[e].x, p[e].y);
                    } else {
#pragma unroll
                        for (int e = 0; e < 16; ++e) pk[e] = 0u;
                    }
                    tc::tmem_st16(lane_base + kSCol + group * kCols, pk);
                    tc::tmem_st_wait();
                    tc::fence_before_sync();
                    warp_arrive(&p_full);

                    if (!(ok = wait.warp(&dp_full, step & 1u))) break;
                    tc::fence_after_sync();
                    if (!none) {
                        float dp[32];
                        tc::tmem_ld32(lane_base + kDpCol + group * kCols, dp);
                        const float4 *dl = reinterpret_cast<const float4 *>(&s_stats[st][1][group * kCols]);
#pragma unroll
                        for (int e = 0; e < 8; ++e) {
                            const float4 x = dl[e];
                            p[2 * e] = mul2(p[2 * e], fma2(make_float2(dp[4 * e], dp[4 * e + 1]), both(kDown), make_float2(x.x, x.y)));
                            p[2 * e + 1] =
                                mul2(p[2 * e + 1], fma2(make_float2(dp[4 * e + 2], dp[4 * e + 3]), both(kDown), make_float2(x.z, x.w)));
                        }
#pragma unroll
                        for (int e = 0; e < 16; ++e) {
                            const float2 y = kScaled<T> ? mul2(p[e], both(w.power)) : p[e];
                            pk[e] = pack2<T>(y.x, y.y);
                        }
                    }
                    tc::tmem_st16(lane_base + kDpCol + group * kCols, pk);   // (zeros where none)
                    tc::tmem_st_wait();
                    tc::fence_before_sync();
                    warp_arrive(&ds_full);

                    if (BIAS && !none) {
                        // dS by distance, under the products.  A lane is a key,
                        // column e a query e further: with every column turned by
                        // e lanes, lane l holds the elements of one distance, that
                        // of key l and the first query, and where the turn wrapped
                        // around those of the distance 32 less.  (One shuffle an
                        // element: 0.45K cycles a step less than a sum handed from
                        // lane to lane and stored by the last.)
                        const int hi = key_lo + 31 - place0, lo = hi - 62;
                        if (!live)   // rows past the document's keys add nothing
#pragma unroll
                            for (int e = 0; e < 16; ++e) p[e] = both(0.f);
                        if (lo >= a.reach || hi <= -a.reach) {
                            float2 x0 = p[0], x1 = p[1];
#pragma unroll
                            for (int e = 2; e < 16; e += 2) {
                                x0 = add2(x0, p[e]);
                                x1 = add2(x1, p[e + 1]);
                            }
                            x0 = add2(x0, x1);
                            (lo >= a.reach ? far_after : far_before) += x0.x + x0.y;
                        } else {
                            float up = 0.f, down = 0.f;
#pragma unroll
                            for (int e = 0; e < 32; ++e) {
                                const float v = __shfl_sync(0xffffffffu, e & 1 ? p[e / 2].y : p[e / 2].x, lane + e);
                                if (lane + e < 32) up += v;
                                else down += v;
                            }
                            float *to = mine + set * set_size + a.reach + kPad + hi - 31 + lane;
                            to[0] = up;
                            if (lane > 0) to[-32] = down;
                        }
                    }
                }
                if (BIAS && ok) {
                    // the head's sums: the warps' added up, in order
                    const float before = warp_sum(far_before), after = warp_sum(far_after);
                    if (lane == 0) {
                        s_far[set][warp][0] = before;
                        s_far[set][warp][1] = after;
                    }
                    if (!(ok = meet(wait))) break;
                    float *out = f.partial + ((int64_t)w.number * a.heads + head) * f.entries;
                    float *sums = by_distance + set * set_size;
                    for (int e = threadIdx.x; e < f.entries; e += kCompute) {
                        float x = 0.f;
#pragma unroll
                        for (int k = 0; k < kSums; ++k) {
                            x += sums[k * f.entries + e];
                            sums[k * f.entries + e] = 0.f;      // for a later head
                        }
                        if (e == kPad)
                            for (int k = 0; k < kWarps; ++k) x += s_far[set][k][0];
                        if (e == kPad + 2 * a.reach)
                            for (int k = 0; k < kWarps; ++k) x += s_far[set][k][1];
                        out[e] = x;
                    }
                    // (with two sets the next meeting keeps the order)
                    if (kSumSets == 1 && !(ok = meet(wait))) break;
                    set ^= kSumSets - 1;
                }
            }
            if (ok) ok = wait.warp(&acc_full, (uint32_t)item & 1u);
            if (!ok) break;
            tc::fence_after_sync();
            const int64_t row = w.k_row + key_lo;
            // the groups' shares: of dV first, then of dK
            constexpr int kOut = 2 * DP / kGroups;
            const bool is_k = group >= kGroups / 2;
            const int col0 = group % (kGroups / 2) * kOut;
            const int64_t stride = is_k ? f.p.dk_ts : f.p.dv_ts;
            T *out = is_k ? static_cast<T *>(f.p.dk) + row * stride + w.hk * f.p.dk_hs
                          : static_cast<T *>(f.p.dv) + row * stride + w.hk * f.p.dv_hs;
            const float scale = !is_k ? kDown : kScaled<T> ? a.scale / w.power : a.scale;
#pragma unroll
            for (int i = 0; i < kOut / 32 && !idle; ++i) {
                const int col = col0 + 32 * i;
                float v[32];
                tc::tmem_ld32(lane_base + (is_k ? kDkCol : kDvCol) + col, v);
#pragma unroll
                for (int e = 0; e < 32; ++e) v[e] *= scale;
                uint4 c[4] = {pack8<T>(v), pack8<T>(v + 8), pack8<T>(v + 16), pack8<T>(v + 24)};
                store_rows(out + col, stride, w.nk - key_lo, d - col, c);
            }
            tc::fence_before_sync();
            __syncwarp();
            if (lane == 0) tc::mbar_arrive(&work_empty[slot]);
        }
    }
    tc::fence_before_sync();
    __syncthreads();
    if (threadIdx.x == 0 && s_abort) atomicExch(&f.p.ctl->status, SIEVE_ETIMEOUT);
    if (warp == 0) {
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
    size_t stats, values, bounds, partial, split_sums, total;   // byte offsets
};
Layout layout_of(const sieve_attention_args &a) {
    Layout l = {};
    l.q_tiles = a.new_tokens > 0 ? a.nseq * ceil_div(a.new_tokens, kTile) : doc_tiles(a.q_tokens, a.nseq, kTile);
    l.k_tiles = doc_tiles(a.k_tokens, a.nseq, kTile);
    l.entries = a.num_buckets ? bias_entries(a.reach) : 0;
    l.splits = (int)(l.k_tiles < 16 * 64 ? ceil_div(l.k_tiles, 16) : 64);
    l.stats = kCtlBytes;
    const bool scaled = a.dtype == SIEVE_F16;
    auto floats = [](int64_t n) { return (size_t)round_up(n * (int64_t)sizeof(float), 256); };
    l.values = l.stats + floats(l.q_tiles * a.heads * stat_rows(scaled, a.num_buckets) * kTile);
    l.bounds = l.values + (scaled ? floats(l.k_tiles * a.kv_heads) : 0);
    l.partial = l.bounds + (scaled ? floats(l.q_tiles * a.heads) : 0);
    l.split_sums = l.partial + floats(l.k_tiles * a.heads * l.entries);
    l.total = l.split_sums + floats((int64_t)a.heads * l.splits * l.entries);
    return l;
}

template <int DP, bool BIAS>
size_t dq_smem(int reach) {
    return 1024 + (size_t)(2 * kept(DP) + 3 + (DP == 64 ? 2 : 1)) * (DP / 64) * kBlockBytes +
           (BIAS ? (size_t)2 * bias_floats(reach) * 4 : 0);
}
template <int DP, bool BIAS>
size_t dkv_smem(int reach) {
    return 1024 + (size_t)2 * (kWalked + kept(DP)) * (DP / 64) * kBlockBytes +
           (BIAS ? (size_t)(bias_floats(reach, DP == 64 ? 4 : 1) + sum_sets(DP) * kSums * bias_entries(reach)) * 4 : 0);
}

template <typename T, int DP, bool BIAS>
cudaError_t run(const BwdArgs &f, const Layout &l, unsigned char *ws, cudaStream_t st) {
    const sieve_attention_args &a = f.p.a;
    // (the kernels' limits are the process', so they are the most that any
    // call asks for: another host thread may launch at any moment)
    constexpr auto kLimit = cudaFuncAttributeMaxDynamicSharedMemorySize;
    constexpr int kMost = SIEVE_ATTENTION_MAX_REACH;
    cudaError_t e;
    if (a.q_tokens > 0) {
        if constexpr (kScaled<T>)
            if (a.k_tokens > 0) {
                k_attend_values<T, DP / 8><<<(unsigned)(l.k_tiles * a.kv_heads), kDeltaThreads, 0, st>>>(f);
                if ((e = cudaGetLastError()) != cudaSuccess) return e;
            }
        k_attend_delta<T, DP / 8, BIAS><<<(unsigned)(l.q_tiles * a.heads), kDeltaThreads, 0, st>>>(f);
        if ((e = cudaGetLastError()) != cudaSuccess) return e;
        auto dq = k_attend_dq<T, DP, BIAS>;
        if ((e = cudaFuncSetAttribute(dq, kLimit, (int)dq_smem<DP, BIAS>(kMost))) != cudaSuccess) return e;
        dq<<<(unsigned)(l.q_tiles * a.heads), 18 * 32, dq_smem<DP, BIAS>(a.reach), st>>>(f);
        if ((e = cudaGetLastError()) != cudaSuccess) return e;
    }
    if (a.k_tokens > 0) {
        auto dkv = k_attend_dkv<T, DP, BIAS>;
        if ((e = cudaFuncSetAttribute(dkv, kLimit, (int)dkv_smem<DP, BIAS>(kMost))) != cudaSuccess) return e;
        dkv<<<(unsigned)(l.k_tiles * a.kv_heads), 18 * 32, dkv_smem<DP, BIAS>(a.reach), st>>>(f);
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
    f.values = reinterpret_cast<float *>(w + l.values);
    f.bounds = reinterpret_cast<float *>(w + l.bounds);
    f.doc_tiles = a.new_tokens > 0 ? (int)ceil_div(a.new_tokens, kTile) : 0;
    f.entries = l.entries;
    f.q_numbers = (int)l.q_tiles;
    f.k_numbers = (int)l.k_tiles;
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
