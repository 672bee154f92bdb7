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
// P stays below 2^8, exact in scale): then the thread rescales its row of O.  In
// fp16 P is taken 2^7 times as large, sum and all: it stays below 2^15, and small
// weights keep their bits down to 2^-21 of the largest.
//
// Warps 0-7 make P (two warps to the 32 lanes of a quarter, 64 columns each,
// so that a row's scores stay in registers); warp 8 loads and issues the
// products; warp 9 finds the work and loads.  Two blocks share an SM (256
// tensor-memory columns each): one's products run under the other's softmax.
// A block that is done takes over one that has not started, found while it
// still worked, so its loads and products run on from document to document.
// (Blocks that each set up, worked and ended spent half of their time outside
// the steps on documents of a few tiles.)
//
// Measured (bf16): 4 documents of 6,001 to 8,192 tokens, causal, 16 heads of 128
// on 4 key heads: 705 us, 1.14 PFLOP/s, bound by the softmax between two products
// (two blocks an SM hide most of it).  512 documents of 0 to 512 tokens, 12 heads
// of 64 with a bias: 367 us (256 without); the products are a sixth of that, the rest
// is the softmax (an exponential and a bias read for each pair) and, for documents of a
// tile or two, what a block's work costs once.  One new token for each of 24
// documents of up to 32K tokens: 689 MB in 156 us, 4.4 TB/s with the join (8 us).
// Two blocks share an SM up to a reach of 130 or so; past that the bias tables leave
// room for one: 534 us on the 512 documents at a reach of 256.  A text of 10 to 60
// tokens has a tile to itself: 10,000 of them, 12 heads of 64, 1,266 us.
//
// Where every document has a few new queries against many keys, a block takes
// the rows of all heads that share a key head (up to 128) over one chunk of
// the keys, and k_attend_join adds the chunks up.
#include <cfloat>
#include <cstring>

#include "attention.cuh"

namespace sieve {
namespace enc {
namespace {

constexpr int kSoftmaxWarps = 8;
constexpr int kSoftmax = kSoftmaxWarps * 32;
constexpr int kThreads = kSoftmax + 64;
constexpr int kSlots = 2;     // the work in hand and the next
// Key tiles of work that is short: the next is asked for ahead of its end.  (With
// long work other blocks are done sooner: 4 documents of 6K to 8K tokens 677 us, 703
// with 64 here.  On short work it is worth little: never asking ahead, documents of
// 128 tokens 114 against 113 us, of 512 365 against 367.)
constexpr int kShort = 16;
constexpr int kHalf = kTile / 2;
constexpr uint32_t kTmemCols = 256;
constexpr int kBlocksPerSm = 2;
constexpr float kRaise = 8.f;
template <typename T>
constexpr float kUp = std::is_same_v<T, __half> ? 7.f : 0.f;
// Tiles of K and of V held at a time.  With one, the next K loads under the
// softmax of this one and the next V under the scores of the next: that is
// enough, and at 128 columns it lets two blocks share an SM.
// (Over chunks of keys too: one block with three tiles of K and two of V took
// half as long again as two blocks with one each.)
__host__ __device__ constexpr int stages(int dp) { return dp == 64 ? 2 : 1; }

// One block's work: a tile of queries of one document against the document's
// keys (or a chunk of them).
struct Work {
    int q_row, nq, query0;             // first row of q, queries, the tile's first query
    int k_row, k_first, nk, n;         // first row and key of the chunk, the document's keys; key tiles
    int group, number;                 // heads, tile or chunk number; group < 0: no more work
    int table;                         // which bias table
};

struct FwdArgs {
    AttentionArgs p;
    CUtensorMap q, k, v;
    int pack;            // heads of one key head in a tile (1: a tile is 128 queries of one head)
    int rows_per_doc;    // split: new_tokens * pack
    int chunk;           // split: keys per block
    int doc_tiles;       // new_tokens > 0, not split: tiles of a document
    int numbers;         // tile or chunk numbers; blocks run over them head by head
    float *part_o;       // split: [chunk number][head groups][rows][head_dim]
    float2 *part_ml;     // split: [chunk number][head groups][rows]: maximum (base 2), sum
};

// The log of a row's sum from its maximum in base 2 and its sum.  A bias at the
// end of the type's range stands there in base 2 as well (see scaled_bias), and
// so does its row's lse.
__device__ __forceinline__ float lse_of(float m, float l) {
    return fabsf(m) == FLT_MAX ? m : (m + log2_approx(l)) * kLn2;
}

// False where the block's number is one that no document uses.
template <bool SPLIT>
__device__ __forceinline__ bool find_work(const FwdArgs &f, DocFinder &find, int t, Work &w) {
    const sieve_attention_args &a = f.p.a;
    Doc doc;
    int k_end, last;                                   // of the tile's queries, the one that sees most
    if (SPLIT) {
        const int s = find_doc(a.k_offsets, (int)a.nseq, (int)a.k_tokens, f.chunk, t);
        doc = doc_at(a, s);
        w.k_first = (t - first_tile(a.k_offsets, s, (int)a.k_tokens, f.chunk)) * f.chunk;
        if (w.k_first < 0 || w.k_first >= doc.nk) return false;
        k_end = min(doc.nk, w.k_first + f.chunk);
        w.query0 = 0;
        last = doc.nq;
    } else {
        int s, tile;
        if (a.new_tokens > 0) {
            s = t / f.doc_tiles;
            tile = t % f.doc_tiles;
            doc = doc_at(a, s);
        } else {
            find(t, s, doc.q0, doc.nq, tile);
            keys_of(a, s, doc);
        }
        const int tiles = (doc.nq + kTile - 1) / kTile;
        if (tile < 0 || tile >= tiles) return false;
        w.query0 = (tiles - 1 - tile) * kTile;         // the tiles that see most keys first
        w.k_first = 0;
        k_end = doc.nk;
        last = min(doc.nq, w.query0 + kTile);
    }
    if (a.causal) k_end = min(k_end, last + doc.nk - doc.nq);
    w.n = k_end > w.k_first ? (k_end - w.k_first + kTile - 1) / kTile : 0;
    w.number = t;
    w.q_row = doc.q0;
    w.nq = doc.nq;
    w.k_row = doc.k0 + w.k_first;
    w.nk = doc.nk;
    return true;
}

template <typename T, int DP, bool BIAS, bool SPLIT>
__global__ void __launch_bounds__(kThreads, kBlocksPerSm) k_attend(const __grid_constant__ FwdArgs f) {
    constexpr int kB = DP / 64;                       // column blocks of a tile
    constexpr int kStages = stages(DP), kQStages = kStages;
    constexpr uint32_t kTileBytes = kB * kBlockBytes;
    // tensor memory: S, P and O; with 64 columns of O the three fit side by
    // side and S of the next tile is computed while P is made, else P takes
    // the place of S (each warp's half within its own columns)
    constexpr bool kApart = DP == 64;
    constexpr uint32_t kPCol = kApart ? 128 : 0, kPHalf = kApart ? 32 : 64, kOCol = kApart ? 192 : 128;
    extern __shared__ unsigned char smem_raw[];
    __shared__ __align__(8) uint64_t q_full[kQStages], k_full[kStages], v_full[kStages], s_full, s_free, p_full, o_full,
        drained, pair_bar[4], work_full[kSlots], work_empty[kSlots], steal_bar, q_empty[kQStages],
        k_empty[kStages], v_empty[kStages];
    __shared__ __align__(16) uint4 s_answer;
    __shared__ uint32_t tmem_slot;
    __shared__ int s_abort;
    __shared__ Work s_work[kSlots];
    __shared__ float s_top[2][2][kTile];
    const sieve_attention_args &a = f.p.a;
    const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0), lane = lane_id();
    const int share = a.heads / a.kv_heads;
    unsigned char *base = reinterpret_cast<unsigned char *>(
        (reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~static_cast<uintptr_t>(1023));
    unsigned char *q_tiles = base, *k_tiles = q_tiles + kQStages * kTileBytes, *v_tiles = k_tiles + kStages * kTileBytes;
    float *bias = reinterpret_cast<float *>(v_tiles + kStages * kTileBytes);   // two sets of `pack` tables
    constexpr int kCopies = SPLIT ? 1 : 4;     // (a chunk of many keys hardly meets the near ones)
    const int bias_set = BIAS ? f.pack * bias_floats(a.reach, kCopies) : 0;

    if (threadIdx.x == 0) {
        if (blockIdx.x == 0) f.p.ctl->status = 0;
        for (int i = 0; i < kQStages; ++i) {
            tc::mbar_init(&q_full[i], 1);
            tc::mbar_init(&q_empty[i], 1);
        }
        for (int i = 0; i < kStages; ++i) {
            tc::mbar_init(&k_empty[i], 1);
            tc::mbar_init(&k_full[i], 1);
            tc::mbar_init(&v_empty[i], 1);
            tc::mbar_init(&v_full[i], 1);
        }
        tc::mbar_init(&s_full, 1);
        tc::mbar_init(&s_free, kSoftmaxWarps);
        tc::mbar_init(&p_full, kSoftmaxWarps);
        tc::mbar_init(&o_full, 1);
        tc::mbar_init(&drained, 1);
        tc::mbar_init(&steal_bar, 1);
        for (int i = 0; i < 4; ++i) tc::mbar_init(&pair_bar[i], 2);
        for (int i = 0; i < kSlots; ++i) {
            tc::mbar_init(&work_full[i], 1);
            tc::mbar_init(&work_empty[i], kSoftmaxWarps + 1);
        }
        s_abort = 0;
        tc::mbar_init_fence();
    }
    if (warp == 0) tc::tmem_alloc(&tmem_slot, kTmemCols);
    tc::fence_before_sync();
    __syncthreads();
    tc::fence_after_sync();
    const uint32_t tmem = __shfl_sync(0xffffffffu, tmem_slot, 0);
    const Waiter wait{&s_abort};

    if (warp == kSoftmaxWarps + 1) {
        // ---------------- the work, one block's after another's, and its loads ----------------
        if (lane == 0) {
            prefetch_map(&f.q);
            if (a.k_tokens > 0) {     // (else there are no maps)
                prefetch_map(&f.k);
                prefetch_map(&f.v);
            }
        }
        int block = blockIdx.x, item = 0, set = 1, group_in_set = -1, q_issued = 0, k_issued = 0, v_issued = 0;
        Blocks blocks{&s_answer, &steal_bar, 0, false};
        DocFinder find(a.q_offsets, a.nseq, a.q_tokens);
        bool ok = true;
        while (ok && block >= 0) {
            Work w;
            w.group = block / f.numbers;
            const int head0 = w.group * f.pack, hk = head0 / share;
            const bool found = find_work<SPLIT>(f, find, block % f.numbers, w);
            if (found && w.n == 0) {
                // no query of these sees a key
                const int first = w.query0, last = min(w.nq, w.query0 + kTile);
                if (SPLIT) {
                    for (int r = lane; r < f.rows_per_doc; r += 32)
                        f.part_ml[((int64_t)w.number * (a.heads / f.pack) + w.group) * f.rows_per_doc + r] =
                            make_float2(-INFINITY, 0.f);
                } else {
                    for (int q = first + lane; q < last; q += 32)
                        f.p.lse[(int64_t)head0 * a.q_tokens + w.q_row + q] = -INFINITY;
                    for (int i = lane; i < (last - first) * (a.head_dim / 8); i += 32) {
                        const int64_t row = w.q_row + first + i / (a.head_dim / 8);
                        *reinterpret_cast<uint4 *>(static_cast<T *>(f.p.out) + (row * a.heads + head0) * a.head_dim +
                                                   i % (a.head_dim / 8) * 8) = make_uint4(0, 0, 0, 0);
                    }
                }
            } else if (found) {
                const int slot = item % kSlots;
                // the work before the last is done with its slot and its
                // bias tables
                if (item >= kSlots && !(ok = wait.warp(&work_empty[slot], (uint32_t)(item / kSlots - 1) & 1u))) break;
                if (BIAS && w.group != group_in_set) {
                    set ^= 1;
                    group_in_set = w.group;
                    for (int h = 0; h < f.pack; ++h)
                        fill_bias<kCopies>(bias + set * bias_set + h * bias_floats(a.reach, kCopies), a, head0 + h, 1,
                                           lane, 32);
                }
                w.table = set;
                if (lane == 0) s_work[slot] = w;
                __syncwarp();
                if (lane == 0) tc::mbar_arrive(&work_full[slot]);
                ++item;
                if (!SPLIT && w.n <= kShort) blocks.ask();
                const int qs = q_issued % kQStages;
                if (!(ok = wait.warp(&q_empty[qs], ((uint32_t)(q_issued / kQStages) & 1u) ^ 1u))) break;
                if (elected()) {
                    expect(&q_full[qs], kB * 128u * (uint32_t)(f.pack * (kTile / f.pack)));
                    for (int b = 0; b < kB; ++b)
                        tma_load(q_tiles + qs * kTileBytes + b * kBlockBytes, &f.q, 64 * b, head0, w.q_row + w.query0,
                                 &q_full[qs]);
                }
                __syncwarp();
                ++q_issued;
                // with two stages the values of a step are loaded after the
                // keys of the next: their place is free later
                constexpr int kBehind = kStages - 1;
#pragma unroll 1
                for (int j = 0; j < w.n + kBehind; ++j) {
                    if (j < w.n) {
                        const int st = k_issued % kStages;
                        if (!(ok = wait.warp(&k_empty[st], ((uint32_t)(k_issued / kStages) & 1u) ^ 1u))) break;
                        if (elected()) {
                            expect(&k_full[st], kTileBytes);
                            for (int b = 0; b < kB; ++b)
                                tma_load(k_tiles + st * kTileBytes + b * kBlockBytes, &f.k, 64 * b, hk, w.k_row + j * kTile,
                                         &k_full[st]);
                        }
                        __syncwarp();
                        ++k_issued;
                    }
                    if (j >= kBehind) {
                        const int st = v_issued % kStages;
                        if (!(ok = wait.warp(&v_empty[st], ((uint32_t)(v_issued / kStages) & 1u) ^ 1u))) break;
                        if (elected()) {
                            expect(&v_full[st], kTileBytes);
                            for (int b = 0; b < kB; ++b)
                                tma_load(v_tiles + st * kTileBytes + b * kBlockBytes, &f.v, 64 * b, hk,
                                         w.k_row + (j - kBehind) * kTile, &v_full[st]);
                        }
                        __syncwarp();
                        ++v_issued;
                    }
                }
                if (!ok) break;
            }
            ok = blocks.next(wait, block);
        }
        if (ok) {
            const int slot = item % kSlots;
            ok = item < kSlots || wait.warp(&work_empty[slot], (uint32_t)(item / kSlots - 1) & 1u);
            if (lane == 0) {
                s_work[slot].group = -1;
                tc::mbar_arrive(&work_full[slot]);
            }
        }
        if (!ok) {
            // after an abort: what is in flight lands before the block ends
            if (blocks.asking) let_land(&steal_bar, blocks.asked & 1u);
            for (int i = max(0, q_issued - kQStages); i < q_issued; ++i)
                let_land(&q_full[i % kQStages], (uint32_t)(i / kQStages) & 1u);
            for (int i = max(0, k_issued - kStages); i < k_issued; ++i)
                let_land(&k_full[i % kStages], (uint32_t)(i / kStages) & 1u);
            for (int i = max(0, v_issued - kStages); i < v_issued; ++i)
                let_land(&v_full[i % kStages], (uint32_t)(i / kStages) & 1u);
        }
        __syncwarp();
    } else if (warp == kSoftmaxWarps) {
        // ---------------- products ----------------
        constexpr uint32_t id_o = idesc<T>(DP, true), id_s = idesc<T>(kTile, false);
        const uint64_t q0 = desc_k(q_tiles), k0 = desc_k(k_tiles), v0 = desc_mn(v_tiles);
        uint32_t step = 0;
        bool ok = true;
        for (int item = 0; ok; ++item) {
            const int slot = item % kSlots;
            if (!(ok = wait.warp(&work_full[slot], (uint32_t)(item / kSlots) & 1u))) break;
            const Work &w = s_work[slot];
            if (uniform(w.group) < 0) break;
            const int n = uniform(w.n), keys = uniform(w.nk - w.k_first), qs = item % kQStages;
            if (!(ok = wait.warp(&q_full[qs], (uint32_t)(item / kQStages) & 1u))) break;
            // round j: the scores of step j + 1 and the product with P of step
            // j.  With P apart from S the scores come first (as soon as those
            // of step j are in registers), else P has their place until its
            // product.
#pragma unroll 1
            for (int j = -1; ok && j < n; ++j) {
                for (int part = 0; part < 2; ++part) {
                    if ((part == 0) == kApart) {
                        if (j + 1 == n) continue;
                        const uint32_t i = step + (j < 0 ? 0u : 1u), st = i % kStages;
                        if (kApart && j >= 0 && !(ok = wait.warp(&s_free, step & 1u))) break;
                        if (!(ok = wait.warp(&k_full[st], (i / kStages) & 1u))) break;
                        tc::fence_after_sync();
                        if (elected()) {
                            mma_kk<DP>(tmem, q0 + qs * (kTileBytes >> 4), k0 + st * (kTileBytes >> 4), id_s);
                            commit(&s_full);
                            commit(&k_empty[st]);
                            if (j + 2 == n) commit(&q_empty[qs]);
                        }
                        __syncwarp();
                    } else {
                        if (j < 0) continue;
                        const uint32_t st = step % kStages;
                        if (!(ok = wait.warp(&v_full[st], (step / kStages) & 1u))) break;
                        // rows of another document: 0 x NaN
                        if (keys - j * kTile < kTile) clear_rows(v_tiles + st * kTileBytes, keys - j * kTile, kB);
                        if (!(ok = wait.warp(&p_full, step & 1u))) break;
                        tc::fence_after_sync();
                        if (elected()) {
                            mma_groups<kHalf, kPHalf>(tmem + kOCol, tmem + kPCol, v0 + st * (kTileBytes >> 4), id_o, j > 0);
                            commit(&o_full);
                            commit(&v_empty[st]);
                        }
                        __syncwarp();
                    }
                }
                if (j >= 0) ++step;
            }
            if (ok && lane == 0) tc::mbar_arrive(&work_empty[slot]);
        }
        // every product issued ends before the block frees its memory (waited
        // for even after an abort, within the poll limit)
        if (elected()) commit(&drained);
        __syncwarp();
        let_land(&drained, 0);
        __syncwarp();
    } else {
        // ---------------- softmax and epilogue ----------------
        const int quarter = warp & 3, half = warp >> 2;
        const int r = quarter * 32 + lane;
        const float c = a.scale * kLog2e;
        const uint32_t lane_base = tmem + ((uint32_t)(quarter * 32) << 16);
        const uint32_t p_at = lane_base + kPCol + half * kPHalf;
        uint32_t step = 0, meets = 0;                  // steps and meetings of the two halves so far
        bool ok = true;
#pragma unroll 1
        for (int item = 0; ok; ++item) {
            if (!(ok = wait.warp(&work_full[item % kSlots], (uint32_t)(item / kSlots) & 1u))) break;
            const Work &w = s_work[item % kSlots];
            if (w.group < 0) break;
            const int head = w.group * f.pack + (SPLIT ? r % f.pack : 0);
            const float *table =
                bias + (BIAS ? w.table * bias_set + (SPLIT ? r % f.pack * bias_floats(a.reach, kCopies) : 0) : 0);
            const int n = w.n, qi = w.query0 + (SPLIT ? r / f.pack : r);     // query of the document
            const bool live = SPLIT ? r < f.rows_per_doc : qi < w.nq;
            // a warp without a live row only keeps the others company
            const bool idle = SPLIT ? quarter * 32 >= f.rows_per_doc : w.query0 + quarter * 32 >= w.nq;
            const int shift = w.nk - w.nq, place = qi + shift;
            // keys that this row sees, counted from this half's first column
            const int seen = (live ? (a.causal ? min(w.nk, place + 1) : w.nk) - w.k_first : 0) - half * kHalf;
            float m = -INFINITY, l = 0.f;
#pragma unroll 1
            for (int j = 0; j < n; ++j, ++step) {
                if (!(ok = wait.warp(&s_full, step & 1u))) break;
                tc::fence_after_sync();
                if (idle) {
                    warp_arrive(&s_free);
                    if (step > 0 && !(ok = wait.warp(&o_full, (step - 1) & 1u))) break;
                    warp_arrive(&p_full);
                    continue;
                }
                float2 x[2][16];
                {
                    uint32_t raw[2][32];
                    tc::tmem_ld32_issue(lane_base + half * kHalf, raw[0]);
                    tc::tmem_ld32_issue(lane_base + half * kHalf + 32, raw[1]);
                    tc::tmem_ld_wait(raw[0]);
                    tc::tmem_ld_wait(raw[1]);
#pragma unroll
                    for (int i = 0; i < 2; ++i)
#pragma unroll
                        for (int e = 0; e < 16; ++e)
                            x[i][e] = make_float2(__uint_as_float(raw[i][2 * e]), __uint_as_float(raw[i][2 * e + 1]));
                }
                tc::fence_before_sync();
                warp_arrive(&s_free);
                // columns of the half that this row sees; that any row of
                // the warp does
                const int vis = seen - j * kTile;
                const bool all = __all_sync(0xffffffffu, vis >= kHalf);
                const int vis_any = all ? kHalf : __reduce_max_sync(0xffffffffu, vis);
                if (BIAS) {
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        if (32 * i >= vis_any) continue;
                        // distances d0 - place + 0 .. 31; the warp's places
                        const int d0 = w.k_first + j * kTile + half * kHalf + 32 * i;
                        const int place_lo = w.query0 + (SPLIT ? quarter * 32 / f.pack : quarter * 32) + shift;
                        const int place_hi =
                            w.query0 + (SPLIT ? (quarter * 32 + 31) / f.pack : quarter * 32 + 31) + shift;
                        const bool after = d0 - place_hi >= a.reach, before = d0 + 31 - place_lo <= -a.reach;
                        if (after || before) {
                            const float b = table[bias_zero(a.reach) + (after ? a.reach : -a.reach)];
#pragma unroll
                            for (int e = 0; e < 16; ++e)
                                x[i][e] = fma2(x[i][e], make_float2(c, c), make_float2(b, b));
                        } else if (SPLIT) {
                            const float *b = table + bias_zero(a.reach) + d0 - place;
#pragma unroll
                            for (int e = 0; e < 16; ++e)
                                x[i][e] = fma2(x[i][e], make_float2(c, c), make_float2(b[2 * e], b[2 * e + 1]));
                        } else {
                            const float4 *b = bias_at(table, a.reach, d0 - place);
#pragma unroll
                            for (int e = 0; e < 8; ++e) {
                                const float4 v = b[e];
                                x[i][2 * e] = fma2(x[i][2 * e], make_float2(c, c), make_float2(v.x, v.y));
                                x[i][2 * e + 1] = fma2(x[i][2 * e + 1], make_float2(c, c), make_float2(v.z, v.w));
                            }
                        }
                    }
                }
                float t4[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    if (32 * i >= vis_any) continue;
                    if (!all && !__all_sync(0xffffffffu, vis >= 32 * i + 32)) {
#pragma unroll
                        for (int e = 0; e < 16; ++e) {
                            if (32 * i + 2 * e >= vis) x[i][e].x = -INFINITY;
                            if (32 * i + 2 * e + 1 >= vis) x[i][e].y = -INFINITY;
                        }
                    }
#pragma unroll
                    for (int e = 0; e < 16; ++e) t4[e & 3] = fmax3f(t4[e & 3], x[i][e].x, x[i][e].y);
                }
                float top = fmaxf(fmax3f(t4[0], t4[1], t4[2]), t4[3]);
                // the row's maximum over both halves (without a bias the
                // scale is above zero, so it can be applied after the
                // comparison)
                if (!BIAS) top *= c;
                s_top[meets & 1u][half][r] = top;
                warp_arrive(&pair_bar[quarter]);
                if (!(ok = wait.warp(&pair_bar[quarter], meets & 1u))) break;
                top = fmaxf(top, s_top[meets & 1u][half ^ 1][r]);
                ++meets;
                // the last step's product is done with P (and O) before
                // they are written
                if (step > 0 && !(ok = wait.warp(&o_full, (step - 1) & 1u))) break;
                tc::fence_after_sync();
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
                const float sub = m == -INFINITY ? 0.f : m - kUp<T>;
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    uint32_t pk[16];
                    if (32 * i >= vis_any) {
                        // no row of the warp sees these; the product may
                        // still read them
#pragma unroll
                        for (int e = 0; e < 16; ++e) pk[e] = 0u;
                    } else {
                        float2 s0 = make_float2(0.f, 0.f), s1 = s0;
#pragma unroll
                        for (int e = 0; e < 16; ++e) {
                            float2 y = BIAS ? add2(x[i][e], make_float2(-sub, -sub))
                                            : fma2(x[i][e], make_float2(c, c), make_float2(-sub, -sub));
                            y.x = exp2_approx(y.x);
                            y.y = exp2_approx(y.y);
                            if (e & 1) s1 = add2(s1, y);
                            else s0 = add2(s0, y);
                            pk[e] = pack2<T>(y.x, y.y);
                        }
                        s0 = add2(s0, s1);
                        l += s0.x + s0.y;
                    }
                    tc::tmem_st16(p_at + 16 * i, pk);
                }
                tc::tmem_st_wait();
                tc::fence_before_sync();
                warp_arrive(&p_full);
            }
            if (!ok) break;
            if (!idle) {
                // the row's sum over both halves, and the last product
                s_top[meets & 1u][half][r] = l;
                warp_arrive(&pair_bar[quarter]);
                if (!(ok = wait.warp(&pair_bar[quarter], meets & 1u))) break;
                l += s_top[meets & 1u][half ^ 1][r];
                ++meets;
                if (!(ok = wait.warp(&o_full, (step - 1) & 1u))) break;
                tc::fence_after_sync();
                const int d = a.head_dim;
                const bool none = l == 0.f;
                const float inv = SPLIT ? 1.f : rcp_approx(l);
                const int64_t at = ((int64_t)w.number * (a.heads / f.pack) + w.group) * f.rows_per_doc + r;   // split
                const int64_t row = w.q_row + qi;                                                             // not split
                if (live && half == 0) {
                    if (SPLIT) f.part_ml[at] = make_float2(m - kUp<T>, l);
                    else f.p.lse[(int64_t)head * a.q_tokens + row] = none ? -INFINITY : lse_of(m - kUp<T>, l);
                }
#pragma unroll
                for (int i = 0; i < DP / 64; ++i) {
                    const int col = half * (DP / 2) + 32 * i;
                    float o[32];
                    tc::tmem_ld32(lane_base + kOCol + col, o);
#pragma unroll
                    for (int e = 0; e < 32; ++e) o[e] = none ? 0.f : o[e] * inv;
                    if (SPLIT) {
#pragma unroll
                        for (int e = 0; e < 32; e += 4)
                            if (live && col + e < d)
                                *reinterpret_cast<float4 *>(f.part_o + at * d + col + e) =
                                    make_float4(o[e], o[e + 1], o[e + 2], o[e + 3]);
                    } else {
                        uint4 p[4] = {pack8<T>(o), pack8<T>(o + 8), pack8<T>(o + 16), pack8<T>(o + 24)};
                        store_rows(static_cast<T *>(f.p.out) + ((row - lane) * a.heads + head) * d + col,
                                   (int64_t)a.heads * d, w.nq - qi + lane, d - col, p);
                    }
                }
                tc::fence_before_sync();   // O is read before the next tile's first product
            }
            __syncwarp();
            if (ok && lane == 0) tc::mbar_arrive(&work_empty[item % kSlots]);
        }
    }
    tc::fence_before_sync();
    __syncthreads();
    if (threadIdx.x == 0 && s_abort) atomicExch(&f.p.ctl->status, SIEVE_ETIMEOUT);
    if (warp == 0) {
        tc::fence_after_sync();
        tc::tmem_dealloc(tmem, kTmemCols);
    }
}

// The chunks of a document joined: a warp per query and head.
template <typename T>
__global__ void __launch_bounds__(128) k_attend_join(const __grid_constant__ FwdArgs f) {
    const sieve_attention_args &a = f.p.a;
    const unsigned w = blockIdx.x * 4 + (threadIdx.x >> 5);     // query and head
    if (w >= (unsigned)a.q_tokens * a.heads) return;
    const int lane = lane_id(), d = a.head_dim, groups = a.heads / f.pack;
    const int row = w / a.heads, head = w % a.heads, s = row / a.new_tokens, qi = row % a.new_tokens;
    const Doc doc = doc_at(a, s);
    const int t0 = first_tile(a.k_offsets, s, (int)a.k_tokens, f.chunk), n = (doc.nk + f.chunk - 1) / f.chunk;
    const int r = qi * f.pack + head % f.pack;
    auto slot = [&](int i) { return ((int64_t)(t0 + i) * groups + head / f.pack) * f.rows_per_doc + r; };
    float top = -INFINITY;
    for (int i = lane; i < n; i += 32) top = fmaxf(top, f.part_ml[slot(i)].x);
#pragma unroll
    for (int o = 16; o; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
    const float base = top == -INFINITY ? 0.f : top;
    float l = 0.f, acc[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
    for (int i = 0; i < n; ++i) {
        const int64_t at = slot(i);
        const float2 ml = f.part_ml[at];
        float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
        if (4 * lane < d) o = *reinterpret_cast<const float4 *>(f.part_o + at * d + 4 * lane);
        const float e = exp2_approx(ml.x - base);
        l = fmaf(ml.y, e, l);
        if (ml.y == 0.f) continue;                 // (a chunk without visible keys has no sums)
        acc[0] = fmaf(o.x, e, acc[0]);
        acc[1] = fmaf(o.y, e, acc[1]);
        acc[2] = fmaf(o.z, e, acc[2]);
        acc[3] = fmaf(o.w, e, acc[3]);
    }
    if (lane == 0) f.p.lse[(int64_t)head * a.q_tokens + row] = l == 0.f ? -INFINITY : fabsf(top) == FLT_MAX ? top : top * kLn2 + logf(l);
    if (4 * lane < d) {
        const float inv = l == 0.f ? 0.f : 1.f / l;
        uint2 o;
        o.x = pack2<T>(acc[0] * inv, acc[1] * inv);
        o.y = pack2<T>(acc[2] * inv, acc[3] * inv);
        *reinterpret_cast<uint2 *>(static_cast<T *>(f.p.out) + (int64_t)w * d + 4 * lane) = o;
    }
}

// How a call runs: packed over chunks of keys where the queries of every
// document and of a key head's heads fit one tile together.
struct Shape {
    bool split;
    int pack, chunk, doc_tiles;
    int64_t blocks, chunks;
    size_t smem;
};

// Whether a call runs the kernels with a bias, if of zero.  Those compare and
// hide finished scores; the others compare raw ones, hide them with -inf and
// apply the scale after that, which takes a scale above zero (a negative one
// turns the order around, and -inf times zero is NaN).
bool runs_biased(const sieve_attention_args &a) { return a.num_buckets || !(a.scale > FLT_MIN); }

// bias tables of a block: what still lets two blocks share an SM
constexpr int kMaxBiasBytes = 14 * 1024;

// two sets of one head's tables
int bias_bytes_of(int reach, bool packed) { return 2 * 4 * bias_floats(reach, packed ? 1 : 4); }
size_t smem_bytes(int dp, int bias_bytes) {
    return 1024 + (size_t)(3 * stages(dp)) * (dp / 64) * kBlockBytes + (size_t)bias_bytes;
}
// The most that any call asks of an instance.
template <int DP, bool BIAS, bool SPLIT>
size_t most_smem() {
    const int one = BIAS ? bias_bytes_of(SIEVE_ATTENTION_MAX_REACH, SPLIT) : 0;
    return smem_bytes(DP, BIAS && SPLIT && one < kMaxBiasBytes ? kMaxBiasBytes : one);
}

Shape shape_of(const sieve_attention_args &a) {
    Shape s = {};
    const int dp = a.head_dim <= 64 ? 64 : 128, share = a.heads / a.kv_heads;
    const bool packed = a.new_tokens > 0 && a.new_tokens <= kTile;
    const int bias_bytes = runs_biased(a) ? bias_bytes_of(a.reach, packed) : 0;
    s.pack = 1;
    if (packed) {
        s.split = true;
        for (int p = 1; p <= share; ++p)
            if (share % p == 0 && p * a.new_tokens <= kTile && p * bias_bytes <= kMaxBiasBytes) s.pack = p;
        // as many heads of a key head to a block as their bias tables leave room
        // for: each block reads K and V once (8 heads on a key head at a reach of
        // 128, or 4 at 256, take two: 257 us where one takes 156)
        // chunks: about two rounds of blocks, no fewer than two tiles each.  (One
        // token, 1 / 2 / 4 rounds: 24 documents of up to 32K 176 / 164 / 168 us, 4 of
        // them 58 / 69 / 107, one 49 / 69 / 69, 300 of up to 1,000 100 / 100 / 98;
        // at least 1 / 2 / 4 tiles: 4 of up to 2,000 26 / 26 / 30, one of 32K 69 / 69 /
        // 49: where there are few documents it is the join that many chunks cost.)
        const int64_t want = a.k_tokens * (a.heads / s.pack) / (2 * 152 * kBlocksPerSm);
        s.chunk = (int)(round_up(want < 2 * kTile ? 2 * kTile : want, kTile));
        s.chunks = doc_tiles(a.k_tokens, a.nseq, s.chunk);
        s.blocks = s.chunks * (a.heads / s.pack);
    } else {
        // A block's work is one tile of queries.  (Up to four of a document
        // took a fortieth longer on 512 documents of 0 to 512 tokens and 12
        // heads of 64: the work is shared out less evenly.)
        s.doc_tiles = a.new_tokens > 0 ? (int)ceil_div(a.new_tokens, kTile) : 0;
        s.blocks = (a.new_tokens > 0 ? a.nseq * s.doc_tiles : doc_tiles(a.q_tokens, a.nseq, kTile)) * a.heads;
    }
    s.smem = smem_bytes(dp, s.pack * bias_bytes);
    return s;
}

size_t part_floats(const sieve_attention_args &a, const Shape &s) {
    return (size_t)s.blocks * a.new_tokens * s.pack;   // rows of all blocks
}

template <typename T, int DP, bool BIAS, bool SPLIT>
cudaError_t run(const FwdArgs &f, const Shape &s, cudaStream_t st) {
    auto kernel = k_attend<T, DP, BIAS, SPLIT>;
    // The limit is the process', the same whatever this call needs: another
    // host thread may launch between this line and the launch.
    cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                         (int)most_smem<DP, BIAS, SPLIT>());
    if (e != cudaSuccess) return e;
    kernel<<<(unsigned)s.blocks, kThreads, s.smem, st>>>(f);
    if ((e = cudaGetLastError()) != cudaSuccess || !SPLIT) return e;
    k_attend_join<T><<<(unsigned)ceil_div(f.p.a.q_tokens * f.p.a.heads, 4), 128, 0, st>>>(f);
    return cudaGetLastError();
}

template <typename T, int DP>
cudaError_t by_shape(const FwdArgs &f, const Shape &s, cudaStream_t st) {
    const bool biased = runs_biased(f.p.a);
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
    f.doc_tiles = s.doc_tiles;
    f.numbers = (int)(s.blocks / (a.heads / s.pack));
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

}  // namespace enc
}  // namespace sieve
