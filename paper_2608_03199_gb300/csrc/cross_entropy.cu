// cross_entropy.cu -- softmax cross entropy of rows against a table of classes,
// without keeping the scores, and its backward pass.
//
//   z = scale h W^T + b,  lse = log sum exp z,  loss = lse - z_t
//   q = exp(z - lse) - [v = t]
//   dh = dloss scale q W,  dW = scale (dloss q)^T h,  db = sum dloss q
//
// Four products of 2 rows classes width operations each: z in the forward pass;
// z again, dh and dW in the backward pass.  All run in one kernel,
// k_xent<MODE>: tiles of 256 x 256 of a pair of blocks on two SMs (each loads half
// of both operands by TMA into a ring of stages and keeps 128 rows of the result in
// tensor memory), tcgen05 products into one of two accumulators while eight warps
// of each block work on the other.
//   MODE 0  z tiles to a running maximum and sum per row; the target's score
//           is kept apart, so that loss = log1p(sum of the others against it)
//   MODE 1  z tiles to q, rounded to 16 bits, in a pool of panels
//   MODE 2  dh and dW from the pool
// The backward pass takes as many classes at a time as the pool holds (MODE 1,
// then MODE 2); dh is added up over these pieces in fp32.
//
// Rows without a target are left out: k_xent_rows makes the list of the others
// (and a copy of their h, unless every row has a target), and everything after it
// runs over that list, whose length only the device knows.
//
// The pool: panel j holds 64 classes of all listed rows, [rows padded to 256]
// [64], so its address needs no stride that depends on the list.  As operand of
// dh a panel is K-major, as operand of dW MN-major.
//
// With few rows (a list of up to kFine) a gradient's element is the sum of a few q, whose rounding
// no other evens out, and the products cost little beside the tables they read and
// write: there the pool holds what the rounding left off as well, in as many rows
// more, both products run over both, and scores are summed in shorter chunks.
//
// dloss differs from row to row, and dW needs it in the product.  Where all
// rows have the same one it is a factor at the end.  Else it is taken apart, m 2^e:
// q is rounded times m, h gets 2^e in a copy of its own, and so does dh at the end.
// In bf16 the copy is over the largest 2^e and exact.  In fp16 it is shifted so that the
// largest 2^e |h| of all rows is at the type's end: exact down to 2^-29 of that, and
// what is smaller is off by 2^-40 of it at most (over the largest 2^e, an h of 2^-4 in a
// row of 2^-20 had one bit left).  In fp16 q is taken 2^14 times as large as well, so that
// small probabilities keep their bits.
//
// The tensor cores cut a sum off at every step of 16 products instead of
// rounding it, which leaves a score of 2,048 products off by a few 1e-6 of itself, all to
// one side.  So a contraction runs in chunks (128 to 384 products of a score, 4,096 of
// a gradient) whose sums are added up in registers.
//
// A row's q add up to zero, its rounded q to some e.  Where the likely classes
// are much alike (rows of the same topic), q W is a difference of large numbers
// and e times what they have in common would show in dh.  So MODE 1 adds
// up what it rounded, and dh gets -e times the target's row of W at the end: a
// rounding error then counts with its class' distance from the target.
//
// Measured (device time).  8,192 rows x 131,072 classes x 1,024, bf16: MODE 0 1,050 us
// (2.09 PFLOP/s), MODE 1 604 for half of the classes (1.82), MODE 2 1,300 (1.69); over
// and over, the card's power limit leaves 1.56 PFLOP/s of the whole (the library's product
// 1.71).  What bounds them: shared memory, which a tile's products read and its copies
// write at full rate (64 + 64 bytes a cycle); in MODE 1 what the epilogue moves comes on
// top.  4,915 of 32,768 rows x 50,001 x 768 with a bias: 194, 248 and 483 us.  4,099 x 32,800
// x 256, fp16: 47, 63 and 115 us, the last bound by the pool's reads from memory (571 MB,
// 5.0 TB/s).  5 rows x 50,000 x 768: 24 us, 3.2 TB/s of the table.
#include <algorithm>
#include <atomic>
#include <cfloat>
#include <cmath>
#include <cstring>

#include "attention.cuh"
#include "blocks.cuh"
#include "tensor_map.cuh"

namespace sieve {
namespace enc {
namespace {

constexpr int kM = 256, kN = 256, kK = 64;            // a pair's tile, and the contraction of a stage
constexpr int kHalf = kM / 2;                         // rows of a block, and its columns of the second operand
constexpr int kBox = 64;                              // rows of a box of 128 bytes
constexpr uint32_t kBoxBytes = kBox * 128;
constexpr int kBoxes = kHalf / kBox;                  // of an operand in a block
constexpr uint32_t kStageBytes = 2 * kBoxes * kBoxBytes;
constexpr int kEpiWarps = 8;
constexpr int kFine = kM;                             // rows that are few
// rows of a panel of the pool
__host__ __device__ inline int64_t panel_rows(int64_t n) {
    const int64_t padded = (n + kM - 1) / kM * kM;
    return padded < 2 * kFine ? 2 * kFine : padded;
}
// Registers: 384 threads start with kRegisters each, 64,512 in all.  The eight warps that
// hold a tile's sums take 232, the four others (two of them idle) keep 40.
constexpr int kThreads = (kEpiWarps + 4) * 32, kRegisters = 168;
__device__ __forceinline__ void more_registers() { asm volatile("setmaxnreg.inc.sync.aligned.u32 232;"); }
__device__ __forceinline__ void fewer_registers() { asm volatile("setmaxnreg.dec.sync.aligned.u32 40;"); }
constexpr uint32_t kOutBytes = 32 * 128;              // a warp's rows on their way out
__host__ __device__ constexpr int stages(int mode) { return mode == 1 ? 4 : 6; }
__host__ __device__ constexpr int outs(int mode) { return mode == 0 ? 0 : mode == 1 ? 2 : 1; }   // buffers of a warp
__host__ __device__ constexpr uint32_t smem_bytes(int mode) {
    return 1024 + stages(mode) * kStageBytes + outs(mode) * kEpiWarps * kOutBytes;
}
constexpr uint32_t kTmemCols = 512;
constexpr int kGrid = 152, kPairs = kGrid / 2;        // one block an SM
constexpr int kMaxGroup = 16;                         // tiles of classes whose statistics one block keeps
constexpr int kMaxSlabs = 16;
constexpr int kRowTile = 256;                         // rows whose targets are counted together
constexpr int64_t kPoolBytes = (int64_t)1 << 30;

struct Ctl {
    int32_t status;
    int n;               // rows with a target
    int all;             // every row has one
    int same;            // all of them have the same dloss
    float factor;        // that dloss, or the power of two below the largest magnitude
};

struct XentArgs {
    CUtensorMap h, hc, hs, w, pool_in, pool_out, acc, dw;
    Ctl *ctl;
    const int *target;                    // of the list
    const float *lse, *at_target, *dloss, *part_of;   // of the list (q at the target; m, or 1)
    const float *bias;
    float *hit;                           // [rows] the target's score
    float2 *part;                         // [parts][rows of the list, padded] maximum and sum
    float *colsum;                        // [32 rows][classes]
    float *rest;                          // [halves of class tiles][rows of the list, padded] sums of rounded q
    int64_t pool_rows;
    int rows, classes, width;
    float scale, c;                       // c = scale log2(e)
    int want_dh, want_dw, want_db, dw_f32, accumulate, wait_limit;
};

template <typename T>
constexpr float kUp = std::is_same_v<T, __half> ? 16384.f : 1.f;

// two rounded values of a packed pair, added to two sums
template <typename T>
__device__ __forceinline__ float2 add_pair(float2 sum, uint32_t pair) {
    if constexpr (std::is_same_v<T, __half>)
        asm("{\n\t.reg .b16 lo, hi;\n\tmov.b32 {lo, hi}, %2;\n\tadd.f32.f16 %0, lo, %0;\n\tadd.f32.f16 %1, hi, %1;\n\t}"
            : "+f"(sum.x), "+f"(sum.y)
            : "r"(pair));
    else
        asm("{\n\t.reg .b16 lo, hi;\n\tmov.b32 {lo, hi}, %2;\n\tadd.f32.bf16 %0, lo, %0;\n\tadd.f32.bf16 %1, hi, %1;\n\t}"
            : "+f"(sum.x), "+f"(sum.y)
            : "r"(pair));
    return sum;
}

// classes of a piece, and how the forward pass groups its tiles
__host__ __device__ inline int64_t padded(int64_t n) { return (n < 1 ? 1 : n) + kM - 1 - ((n < 1 ? 1 : n) - 1) % kM; }
__host__ __device__ inline int piece_classes(int64_t n, int classes, int64_t pool_rows) {
    const int64_t most = pool_rows / panel_rows(n) / (kN / kK) * kN;
    const int64_t pieces = (classes + most - 1) / most, each = (classes + pieces - 1) / pieces;
    return (int)((each + kN - 1) / kN * kN);
}
__host__ __device__ inline int group_tiles(int64_t n, int classes) {
    const int64_t tiles = padded(n) / kM * ((classes + kN - 1) / kN), g = tiles / (8 * kPairs);
    return (int)(g < 1 ? 1 : g > kMaxGroup ? kMaxGroup : g);
}

// dh has few tiles and a long contraction: it is cut into `slabs`, each with
// sums of its own, so that no pair works longer on one than half of its share of
// the launch.
__host__ __device__ inline int dh_slabs(int64_t n, int classes, int width, int64_t pool_rows, bool dw) {
    const int64_t blocks = piece_classes(n, classes, pool_rows) / kK, across = (width + kN - 1) / kN;
    const int64_t tiles = padded(n) / kM * across, others = dw ? blocks / (kM / kK) * across * ((n + kK - 1) / kK) : 0;
    const int64_t share = (tiles * blocks + others) / kPairs / 2 + 1, slabs = (blocks + share - 1) / share;
    return (int)(slabs < kMaxSlabs ? slabs : kMaxSlabs);
}

// ---------------------------------------------------------------------------
constexpr int64_t kFewRows = 1 << 18;
constexpr int kManyBlocks = 8;                        // of a tile of rows where there are few

// The rows with a target.
struct RowArgs {
    const void *targets, *h;
    const float *dloss, *loss, *lse;      // backward
    float *loss_out, *lse_out;            // forward: zeros where there is no target
    void *dh;                             // backward: the same
    int64_t h_stride, dh_stride;
    int rows, classes, width, target_type;
    Ctl *ctl;
    int *count;                           // [blocks]
    uint32_t *top, *low;                  // [blocks] largest dloss, and its lowest, as ordered keys
    int *reach;                           // fp16: [blocks][SUB] largest exponent of 2^e |h|, or nullptr
    int least;                            // and what it counts as at least, so that the factor at the end stays normal
    int *row, *target;
    float *dloss_c, *at_target_c, *lse_c, *part_c, *whole_c;   // part_c whole_c = dloss
    void *hc, *hs;
};

// whole numbers in the order of the floats
__device__ __forceinline__ uint32_t ordered(float v) {
    const uint32_t b = __float_as_uint(v);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float unordered(uint32_t k) {
    return __uint_as_float(k & 0x80000000u ? k & 0x7fffffffu : ~k);
}

// m 2^e of a dloss, m from 1 to 2 (so that 2^e is finite).  A zero, or one that is not
// finite, stays whole: false, and its e is somebody else's choice.
__device__ __forceinline__ bool apart(float v, float &m, int &e) {
    m = 2.f * frexpf(v, &e);
    --e;
    if (v != 0.f && isfinite(v)) return true;
    m = v;
    return false;
}

// fp16, backward: how far 2^e |h| reaches in the rows of each of a tile's SUB blocks.
// Values that are not finite do not count.
constexpr int kNoReach = -1000;
template <int SUB>
__device__ __forceinline__ void find_reach(const RowArgs &a) {
    __shared__ int s_reach[kRowTile / 32];
    constexpr int kMine = kRowTile / SUB / (kRowTile / 32);        // rows of a warp
    const int lane = lane_id(), warp = threadIdx.x >> 5, chunks = a.width / 8;
    const int64_t first = ((int64_t)blockIdx.x * (kRowTile / 32) + warp) * kMine;
    int reach = kNoReach, mine = kNoReach;
    if (lane < kMine && first + lane < a.rows && id_at(a.targets, a.target_type, first + lane, a.classes) >= 0) {
        float m;
        int e;
        if (apart(a.dloss[first + lane], m, e)) mine = e;
    }
    // four rows at a time, a lane the exponent of its own columns
    for (int i = 0; i < kMine; i += 4) {
        int e[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) e[k] = __shfl_sync(0xffffffffu, mine, i + k);
        for (int c = lane; c < chunks; c += 32) {
            uint4 raw[4];
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (e[k] != kNoReach)
                    raw[k] = __ldg(reinterpret_cast<const uint4 *>(static_cast<const __half *>(a.h) + (first + i + k) * a.h_stride) + c);
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                if (e[k] == kNoReach) continue;
                uint32_t top = 0;
                for (const uint32_t w : {raw[k].x, raw[k].y, raw[k].z, raw[k].w})
                    for (const uint32_t x : {w & 0x7fffu, w >> 16 & 0x7fffu}) top = max(top, x < 0x7c00u ? x : 0u);
                const int e_h = (__float_as_int(__half2float(__ushort_as_half((unsigned short)top))) >> 23) - 127;
                if (top) reach = max(reach, e[k] + e_h);
            }
        }
    }
    reach = __reduce_max_sync(0xffffffffu, reach);
    if (lane == 0) s_reach[warp] = reach;
    __syncthreads();
    if (threadIdx.x) return;
    for (int w = 1; w < kRowTile / 32; ++w) reach = max(reach, s_reach[w]);
    a.reach[blockIdx.x] = reach;
}

// The rows of a tile that have a target, and their dloss.  With SUB blocks a tile,
// each looks how far its rows reach, and the first one counts.
template <int SUB>
__global__ void __launch_bounds__(kRowTile) k_xent_count(RowArgs a) {
    __shared__ uint32_t top[kRowTile / 32], low[kRowTile / 32];
    const int tile = SUB ? (int)blockIdx.x / (SUB ? SUB : 1) : (int)blockIdx.x;
    if constexpr (SUB > 0) {
        find_reach<SUB>(a);
        if (blockIdx.x % SUB) return;
    }
    const int64_t r = (int64_t)tile * kRowTile + threadIdx.x;
    const bool live = r < a.rows && id_at(a.targets, a.target_type, r, a.classes) >= 0;
    const int n = __syncthreads_count(live);
    if (threadIdx.x == 0) a.count[tile] = n;
    if (!a.dloss) return;
    const uint32_t k = live ? ordered(a.dloss[r]) : 0;
    const uint32_t t = __reduce_max_sync(0xffffffffu, k), l = __reduce_min_sync(0xffffffffu, live ? k : 0xffffffffu);
    if (lane_id() == 0) {
        top[threadIdx.x >> 5] = t;
        low[threadIdx.x >> 5] = l;
    }
    __syncthreads();
    if (threadIdx.x == 0) {
        uint32_t t2 = 0, l2 = 0xffffffffu;
        for (int w = 0; w < kRowTile / 32; ++w) {
            t2 = max(t2, top[w]);
            l2 = min(l2, low[w]);
        }
        a.top[tile] = t2;
        a.low[tile] = l2;
    }
}

// SUB blocks share a tile of rows, so that many blocks copy where there are few
// tiles (32,768 rows of 768, one in seven with a target, backward: 26 us with one).
// More than kFewRows rows have tiles enough, and every block reads all tiles' counts.
template <typename T, int SUB>
__global__ void __launch_bounds__(kRowTile) k_xent_rows(const RowArgs a) {
    constexpr int kWarps = kRowTile / 32;
    __shared__ int s_before[kWarps], s_all[kWarps], s_rank[kWarps], s_list[kRowTile];
    __shared__ uint32_t s_top[kWarps], s_low[kWarps];
    constexpr int kMine = kRowTile / SUB;            // rows of this block, from first on in its tile
    const int tile = (int)blockIdx.x / SUB, tiles = (int)gridDim.x / SUB, first = (int)blockIdx.x % SUB * kMine;
    const int tid = threadIdx.x, lane = lane_id(), warp = tid >> 5;
    int before = 0, all = 0;
    uint32_t top = 0, low = 0xffffffffu;
#pragma unroll 4
    for (int b = tid; tiles > 1 && b < tiles; b += kRowTile) {
        const int c = a.count[b];
        all += c;
        if (b < tile) before += c;
        if (a.dloss) {
            top = max(top, a.top[b]);
            low = min(low, a.low[b]);
        }
    }
    const int64_t r = (int64_t)tile * kRowTile + tid;
    const int t = r < a.rows ? id_at(a.targets, a.target_type, r, a.classes) : -1;
    if (tiles == 1) {            // one tile: nothing was counted before
        all = t >= 0;
        if (a.dloss && t >= 0) top = low = ordered(a.dloss[r]);
    }
    before = __reduce_add_sync(0xffffffffu, before);
    all = __reduce_add_sync(0xffffffffu, all);
    top = __reduce_max_sync(0xffffffffu, top);
    low = __reduce_min_sync(0xffffffffu, low);
    const unsigned live = __ballot_sync(0xffffffffu, t >= 0);
    if (lane == 0) {
        s_before[warp] = before;
        s_all[warp] = all;
        s_top[warp] = top;
        s_low[warp] = low;
        s_rank[warp] = __popc(live);
    }
    __syncthreads();
    before = all = 0;
    top = 0;
    low = 0xffffffffu;
    int rank = 0, here = 0;                          // before this thread's row in the block's, and of the block
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
        before += s_before[w];
        all += s_all[w];
        top = max(top, s_top[w]);
        low = min(low, s_low[w]);
        if (w * 32 < first) before += s_rank[w];
        else if (w * 32 < first + kMine) here += s_rank[w];
        if (w * 32 >= first && w < warp) rank += s_rank[w];
    }
    const bool mine = tid >= first && tid < first + kMine;
    rank += __popc(live & ((1u << lane) - 1));
    const bool every = all == a.rows, same = top == low;
    const float hi = unordered(top), lo = unordered(low);
    // what every 2^e is over in the copy of h; a dloss that stays whole has it for its e
    // (and its h stays whole too)
    const float largest = fmaxf(fabsf(hi), fabsf(lo));
    int e_all = 1;
    if (isfinite(largest)) frexpf(largest, &e_all);
    --e_all;
    if (a.reach && !same) {
        int reach = a.least;
        for (int b = tid; b < tiles * SUB; b += kRowTile) reach = max(reach, a.reach[b]);
        reach = __reduce_max_sync(0xffffffffu, reach);
        __syncthreads();
        if (lane == 0) s_rank[warp] = reach;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < kWarps; ++w) reach = max(reach, s_rank[w]);
        e_all = reach - 15;              // the largest 2^e |h| is below 2^16 in the copy
    }
    auto parts = [&](float v, int &e) {
        float m;
        if (!apart(v, m, e)) e = e_all;
        return m;
    };
    if (blockIdx.x == 0 && tid == 0) {
        a.ctl->status = 0;
        a.ctl->n = all;
        a.ctl->all = every;
        a.ctl->same = !a.dloss || same;
        a.ctl->factor = a.dloss && all > 0 ? (same ? hi : ldexpf(1.f, e_all)) : 0.f;
    }
    if (mine && t >= 0) {
        const int at = before + rank;
        s_list[rank] = tid;
        a.row[at] = (int)r;
        a.target[at] = t;
        if (a.dloss) {
            const float v = a.dloss[r];
            int e;
            const float m = parts(v, e);
            a.dloss_c[at] = v;
            a.part_c[at] = same ? 1.f : m;
            a.whole_c[at] = same ? v : ldexpf(1.f, e);
            a.at_target_c[at] = expm1f(-a.loss[r]);
            a.lse_c[at] = a.lse[r];
        }
    } else if (mine && r < a.rows && a.loss_out) {
        a.loss_out[r] = 0.f;
        a.lse_out[r] = 0.f;
    }
    __syncthreads();
    const T *h = static_cast<const T *>(a.h);
    const int chunks = a.width / 8;
    const bool scaled = a.dloss && a.hs && !same;
    if (!every || scaled) {
        T *hc = static_cast<T *>(a.hc), *hs = static_cast<T *>(a.hs);
        for (int i = warp; i < here; i += kWarps) {
            const int64_t from = (int64_t)tile * kRowTile + s_list[i], to = before + i;
            int e_row = e_all;
            if (scaled) parts(a.dloss[from], e_row);
            const float f = ldexpf(1.f, min(e_row - e_all, 39));     // (above that in fp16 where the row is all zeros)
#pragma unroll 4
            for (int c = lane; c < chunks; c += 32) {
                const uint4 raw = __ldg(reinterpret_cast<const uint4 *>(h + from * a.h_stride) + c);
                if (!every) reinterpret_cast<uint4 *>(hc + to * a.width)[c] = raw;
                if (scaled) {
                    const T *x = reinterpret_cast<const T *>(&raw);
                    float v[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[e] = f * to_f32<T>(x[e]);
                    reinterpret_cast<uint4 *>(hs + to * a.width)[c] = pack8<T>(v);
                }
            }
        }
        // the last tile's places past the list: zeros
        const int last = (int)min(padded(all), (int64_t)a.rows);
        for (int i = all + (int)blockIdx.x * kWarps + warp; i < last; i += (int)gridDim.x * kWarps)
            for (int c = lane; c < chunks; c += 32) {
                if (!every) reinterpret_cast<uint4 *>(hc + (int64_t)i * a.width)[c] = make_uint4(0, 0, 0, 0);
                if (scaled) reinterpret_cast<uint4 *>(hs + (int64_t)i * a.width)[c] = make_uint4(0, 0, 0, 0);
            }
    }
    if (a.dh && here < kMine)
        for (int i = warp; i < kMine; i += kWarps) {
            const int64_t row = (int64_t)tile * kRowTile + first + i;
            if (row >= a.rows || id_at(a.targets, a.target_type, row, a.classes) >= 0) continue;
            for (int c = lane; c < chunks; c += 32)
                reinterpret_cast<uint4 *>(static_cast<T *>(a.dh) + row * a.dh_stride)[c] = make_uint4(0, 0, 0, 0);
        }
}

// ---------------------------------------------------------------------------
// Instruction descriptor: fp32 accumulation, M = 256 over the pair, both operands
// T (fp16 is format 0, bf16 1), K- or MN-major.
template <typename T>
__device__ __forceinline__ uint32_t product(int N, bool a_mn, bool b_mn) {
    const uint32_t f = std::is_same_v<T, __half> ? 0u : 1u;
    return (1u << 4) | (f << 7) | (f << 10) | ((a_mn ? 1u : 0u) << 15) | ((b_mn ? 1u : 0u) << 16) |
           ((uint32_t)(N >> 3) << 17) | ((uint32_t)(kM >> 4) << 24);
}
// The instructions of a pair of blocks.  The first of the two issues the products;
// loads of both complete on its barriers, and its commits arrive on both blocks'.
__device__ __forceinline__ uint32_t pair_rank() {
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ uint32_t at_first(const void *p) {    // the same place in the first block's shared memory
    uint32_t a;
    asm volatile("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(a) : "r"(tc::smem_u32(p)));
    return a;
}
__device__ __forceinline__ void pair_sync() {
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ void pair_mma(uint32_t d_tmem, uint64_t a, uint64_t b, uint32_t id, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d_tmem),
        "l"(a), "l"(b), "r"(id), "r"(accumulate)
        : "memory");
}
__device__ __forceinline__ void pair_commit(uint64_t *bar) {
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(
                     tc::smem_u32(bar)),
                 "h"((uint16_t)3)
                 : "memory");
}
__device__ __forceinline__ void pair_alloc(uint32_t *slot, uint32_t cols) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(tc::smem_u32(slot)), "r"(cols)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
}
__device__ __forceinline__ void pair_dealloc(uint32_t tmem, uint32_t cols) {
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(cols) : "memory");
}
// One arrival of a warp whose lanes are all done, at a place in either block.  What
// it hands over is tensor memory, which the tcgen05 fences order; a release to
// the cluster would wait for every store of the warp besides (4,099 x 32,800 x 256
// forward: 75 us with it).
__device__ __forceinline__ void warp_arrive_at(uint32_t bar) {
    __syncwarp();
    if (lane_id() == 0) asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}
// Waits are bounded in time: one poll of an mbarrier may hold a thread back for as long as the
// hardware chooses, so a limit of polls alone says little (an arrival that never
// comes would look like a hang).  A wait gives up after kWaitNs, or once another role of
// the block has; every role then winds down and the block records SIEVE_ETIMEOUT.
constexpr uint32_t kWaitNs = 2000000000u;
__device__ __forceinline__ uint32_t now_ns() {        // wraps after 4.3 s
    uint32_t t;
    asm volatile("mov.u32 %0, %%globaltimer_lo;" : "=r"(t));
    return t;
}
struct PairWaiter {
    int *abort_flag;   // shared memory
    __device__ __forceinline__ bool operator()(uint64_t *bar, uint32_t parity, int limit) const {
        if (tc::mbar_test_wait(bar, parity)) return true;
        uint32_t start = 0;
#pragma unroll 1
        for (uint32_t it = 0; it < kPolls; ++it) {
            if (limit && it + 1 >= (uint32_t)limit) break;
            if (tc::mbar_try_wait(bar, parity)) return true;
            if ((it & 63u) != 63u) continue;
            if (*(volatile int *)abort_flag) break;
            if (it == 63u) start = now_ns();
            else if (now_ns() - start > kWaitNs) break;
        }
        *(volatile int *)abort_flag = 1;
        return false;
    }
    // the same for a whole warp in step, after `limit` polls at the latest (0: the usual limit)
    __device__ __forceinline__ bool warp(uint64_t *bar, uint32_t parity, int limit = 0) const {
        return __all_sync(0xffffffffu, (*this)(bar, parity, limit));
    }
};
// for products in flight, after an abort too
__device__ __forceinline__ void land(uint64_t *bar, uint32_t parity) {
    uint32_t start = 0;
#pragma unroll 1
    for (uint32_t it = 0; it < kPolls && !tc::mbar_try_wait(bar, parity); ++it) {
        if ((it & 63u) != 63u) continue;
        if (it == 63u) start = now_ns();
        else if (now_ns() - start > kWaitNs) break;
    }
}
// After an abort: ten milliseconds, in which the copies that nobody waits for any more land
// (a stage takes microseconds; whose barrier they complete on may never have expected them).
__device__ __forceinline__ void linger() {
    const uint32_t start = now_ns();
#pragma unroll 1
    for (int it = 0; it < 100000 && now_ns() - start < 10000000u; ++it) __nanosleep(1000);
}

// MN-major operand of boxes of 64 columns by 64 rows of the contraction axis
__device__ __forceinline__ uint64_t desc_boxes(const void *tile) {
    return (tc::desc_k_sw128(tc::smem_u32(tile)) & ~((uint64_t)0x3FFF << 16)) | (uint64_t)(kBoxBytes >> 4) << 16;
}

__device__ __forceinline__ void load_box(void *dst, const CUtensorMap *map, int x, int y, uint32_t bar) {
    asm volatile(
        "cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.cta_group::2 [%0], [%1, {%2, %3}], "
        "[%4];" ::"r"(tc::smem_u32(dst)),
        "l"(map), "r"(x), "r"(y), "r"(bar)
        : "memory");
}
__device__ __forceinline__ void store_box(const CUtensorMap *map, int x, int y, const void *src) {
    asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.tile.bulk_group [%0, {%1, %2}], [%3];" ::"l"(map), "r"(x),
                 "r"(y), "r"(tc::smem_u32(src))
                 : "memory");
}
__device__ __forceinline__ void add_box(const CUtensorMap *map, int x, int y, const void *src) {
    asm volatile("cp.reduce.async.bulk.tensor.2d.global.shared::cta.add.tile.bulk_group [%0, {%1, %2}], [%3];" ::"l"(map),
                 "r"(x), "r"(y), "r"(tc::smem_u32(src))
                 : "memory");
}
__device__ __forceinline__ void stores_issued() { asm volatile("cp.async.bulk.commit_group;" ::: "memory"); }
__device__ __forceinline__ void stores_read() { asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory"); }
__device__ __forceinline__ void one_store_read() { asm volatile("cp.async.bulk.wait_group.read 1;" ::: "memory"); }
__device__ __forceinline__ void stores_done() { asm volatile("cp.async.bulk.wait_group 0;" ::: "memory"); }

__device__ __forceinline__ float2 get(const float *p) { return make_float2(p[0], p[1]); }
__device__ __forceinline__ void put(float *p, float2 v) {
    p[0] = v.x;
    p[1] = v.y;
}

// One tile's work.
struct Tile {
    int m0, n0;          // first row and column of the result
    int n_boxes;         // of 64 columns, in each block
    int first, blocks;   // stages of the contraction axis
    int slab;            // MODE 2, dh: which sums
    int half;            // MODE 2: the stage from which on it runs over what the rounding left off
    bool dw;             // MODE 2: dW, else dh
};

// The tiles of a launch, in order: what every role walks.
template <int MODE>
struct Walk {
    int n, mp, panel, row_tiles, class_tiles, group, groups;
    bool fine;                                       // the pool holds q in two parts
    int v0, v1;                                      // classes of the piece
    int dh_tiles, d_tiles, dw_rows, total, width, slabs, slab_blocks;
    __device__ __forceinline__ Walk(const XentArgs &a, int piece) {
        n = a.ctl->n;
        mp = (int)padded(n);
        panel = (int)panel_rows(n);
        fine = n <= kFine;
        width = a.width;
        row_tiles = (n + kM - 1) / kM;
        d_tiles = (a.width + kN - 1) / kN;
        v0 = 0;
        v1 = a.classes;
        if (MODE != 0) {
            const int each = piece_classes(n, a.classes, a.pool_rows);
            v0 = (int)min((int64_t)piece * each, (int64_t)a.classes);
            v1 = (int)min((int64_t)v0 + each, (int64_t)a.classes);
        }
        class_tiles = (v1 - v0 + kN - 1) / kN;
        group = MODE == 0 ? group_tiles(n, a.classes) : 1;
        groups = (class_tiles + group - 1) / group;
        slabs = slab_blocks = 1;
        if (MODE == 2) {
            slabs = dh_slabs(n, a.classes, a.width, a.pool_rows, a.want_dw);
            slab_blocks = (piece_classes(n, a.classes, a.pool_rows) / kK + slabs - 1) / slabs;
        }
        dh_tiles = a.want_dh && v1 > v0 ? row_tiles * d_tiles * slabs : 0;
        dw_rows = a.want_dw ? (v1 - v0 + kM - 1) / kM : 0;
        total = MODE == 2 ? dh_tiles + dw_rows * d_tiles : row_tiles * groups;
    }
    // tiles of item i
    __device__ __forceinline__ int tiles(int i) const {
        return MODE == 0 ? min(group, class_tiles - i / row_tiles * group) : 1;
    }
    __device__ __forceinline__ Tile tile(int i, int k) const {
        Tile t;
        if (MODE != 2) {
            t.m0 = i % row_tiles * kM;
            t.n0 = v0 + (i / row_tiles * group + k) * kN;
            t.n_boxes = kBoxes;
            t.first = t.slab = 0;
            t.blocks = (width + kK - 1) / kK;
            t.dw = false;
            return t;
        }
        t.dw = i >= dh_tiles;
        if (t.dw) i -= dh_tiles;
        const int across = t.dw ? dw_rows : row_tiles;
        t.m0 = i % across * kM;
        i /= across;
        t.n0 = i % d_tiles * kN;
        t.slab = i / d_tiles;
        t.n_boxes = width - t.n0 > kN / 2 ? kBoxes : kBoxes / 2;
        t.first = t.slab * slab_blocks;
        t.blocks = t.dw ? (n + kK - 1) / kK : max(0, min(slab_blocks, (v1 - v0 + kK - 1) / kK - t.first));
        t.half = fine ? t.blocks : INT32_MAX;
        if (fine) t.blocks *= 2;
        return t;
    }
};

template <typename T, int MODE, bool BIAS>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kThreads, 1) k_xent(const __grid_constant__ XentArgs a, int piece) {
    constexpr int kStages = stages(MODE);
    extern __shared__ unsigned char smem_raw[];
    __shared__ __align__(8) uint64_t full[kStages], empty[kStages], d_full[2], d_empty[2], drained;
    __shared__ uint32_t tmem_slot;
    __shared__ int s_abort, s_chunk;
    __shared__ __align__(16) float s_bias[kEpiWarps][BIAS ? kN / 2 : 4];
    const Walk<MODE> walk(a, piece);
    if (walk.total == 0) return;
    const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0), lane = lane_id();
    unsigned char *base = reinterpret_cast<unsigned char *>(
        (reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~static_cast<uintptr_t>(1023));
    if (threadIdx.x == 0) {
        for (int s = 0; s < kStages; ++s) {
            tc::mbar_init(&full[s], 1);
            tc::mbar_init(&empty[s], 1);
        }
        for (int b = 0; b < 2; ++b) {
            tc::mbar_init(&d_full[b], 1);
            tc::mbar_init(&d_empty[b], 2 * kEpiWarps);
        }
        tc::mbar_init(&drained, 1);
        s_abort = 0;
        // Stages of a chunk.  Two where rows are few, or no pair has a second tile whose
        // products would wait (1,592 x 44 x 2,048: 15.8 and 20.0 us with two, four and six).  Else
        // four, and six in bf16 past 512 columns: two buffers then hold the next tile's products
        // for as long as this one's q take (4,915 x 50,001 with a bias, both passes over the
        // scores: 768 columns 512 us with four, 441 with six, 1,024 629 and 580, 2,048 1,123 and 1,070;
        // 512 364 and 365).  fp16 products have more bits to cut off: six left lse off by
        // 1.1e-6 of unit rows' at a scale of 20, four by 7e-7 (4,096 x 32,768 x 1,024: 358 us,
        // with six 334).  Read anew where it is used: the epilogue has no register for it.
        s_chunk = walk.fine || walk.total <= kPairs ? 2 : std::is_same_v<T, __half> || a.width <= 8 * kK ? 4 : 6;
        tc::mbar_init_fence();
    }
    __syncwarp();
    if (warp == 0) pair_alloc(&tmem_slot, kTmemCols);
    tc::fence_before_sync();
    __syncthreads();
    pair_sync();
    tc::fence_after_sync();
    const int rank = (int)pair_rank(), pair = blockIdx.x / 2, pairs = gridDim.x / 2;
    const uint32_t tmem = __shfl_sync(0xffffffffu, tmem_slot, 0);
    const PairWaiter wait{&s_abort};
    const bool all = a.ctl->all, same = a.ctl->same;
    auto chunk_of = [&] { return MODE == 2 ? 64 : *const_cast<const volatile int *>(&s_chunk); };

    if (warp == kEpiWarps) {
        // ---------------- loads ----------------
        fewer_registers();
        const CUtensorMap *rows = MODE == 2 && !same ? &a.hs : all ? &a.h : &a.hc;
        int s = 0;
        bool ok = true;
        for (int i = pair; ok && i < walk.total; i += pairs)
            for (int k = 0, nk = walk.tiles(i); ok && k < nk; ++k) {
                const Tile t = walk.tile(i, k);
#pragma unroll 1
                for (int b = 0; b < t.blocks; ++b, ++s) {
                    const int st = s % kStages;
                    if (!(ok = wait.warp(&empty[st], ((uint32_t)(s / kStages) & 1u) ^ 1u))) break;
                    if (elected()) {
                        unsigned char *pa = base + st * kStageBytes, *pb = pa + kBoxes * kBoxBytes;
                        const uint32_t bar = at_first(&full[st]);
                        if (rank == 0) expect(&full[st], 2 * (kBoxes + t.n_boxes) * kBoxBytes);
                        const int m = t.m0 + rank * kHalf, n = t.n0 + rank * t.n_boxes * kBox;
                        const int k0 = MODE == 2 && b >= t.half ? b - t.half : b, low = b == k0 ? 0 : walk.mp;
#pragma unroll
                        for (int j = 0; j < kBoxes; ++j) {
                            void *dst = pa + j * kBoxBytes;
                            if (MODE != 2) load_box(dst, rows, b * kK, m + j * kBox, bar);
                            else if (t.dw) load_box(dst, &a.pool_in, 0, (m / kBox + j) * walk.panel + low + k0 * kK, bar);
                            else load_box(dst, &a.pool_in, 0, (t.first + k0) * walk.panel + low + m + j * kBox, bar);
                        }
                        for (int j = 0; j < t.n_boxes; ++j) {
                            void *dst = pb + j * kBoxBytes;
                            if (MODE != 2) load_box(dst, &a.w, b * kK, n + j * kBox, bar);
                            else if (t.dw) load_box(dst, rows, n + j * kBox, k0 * kK, bar);
                            else load_box(dst, &a.w, n + j * kBox, walk.v0 + (t.first + k0) * kK, bar);
                        }
                    }
                    __syncwarp();
                }
            }
        // every release of a stage has arrived before this block leaves
        for (int j = max(0, s - kStages); ok && j < s; ++j) ok = wait.warp(&empty[j % kStages], (uint32_t)(j / kStages) & 1u);
        __syncwarp();
    } else if (warp == kEpiWarps + 1) {
        // ---------------- products ----------------
        fewer_registers();
        const int chunk = chunk_of();
        int s = 0, c = 0;
        bool ok = true;
        for (int i = pair; rank == 0 && ok && i < walk.total; i += pairs)
            for (int k = 0, nk = walk.tiles(i); ok && k < nk; ++k) {
                const Tile t = walk.tile(i, k);
                const bool a_mn = MODE == 2 && t.dw, b_mn = MODE == 2;
                const uint32_t id = product<T>(2 * t.n_boxes * kBox, a_mn, b_mn);
                const uint64_t step_a = a_mn ? 128 : 2, step_b = b_mn ? 128 : 2;
#pragma unroll 1
                for (int b = 0, in = 0; b < t.blocks; ++b, ++s) {
                    const int buf = c & 1;
                    const uint32_t d = tmem + buf * kN;
                    const bool first = in == 0, last = in + 1 == chunk || b + 1 == t.blocks;
                    if (first && !(ok = wait.warp(&d_empty[buf], ((uint32_t)(c >> 1) & 1u) ^ 1u))) break;
                    const int st = s % kStages;
                    if (!(ok = wait.warp(&full[st], (uint32_t)(s / kStages) & 1u))) break;
                    tc::fence_after_sync();
                    if (elected()) {
                        const unsigned char *pa = base + st * kStageBytes, *pb = pa + kBoxes * kBoxBytes;
                        const uint64_t da = a_mn ? desc_boxes(pa) : desc_k(pa), db = b_mn ? desc_boxes(pb) : desc_k(pb);
#pragma unroll
                        for (int x = 0; x < kK / 16; ++x)
                            pair_mma(d, da + x * step_a, db + x * step_b, id, !first || x > 0);
                        pair_commit(&empty[st]);
                        if (last) pair_commit(&d_full[buf]);
                    }
                    __syncwarp();
                    in = last ? 0 : in + 1;
                    if (last) ++c;
                }
            }
        // and every release of the results, the other block's too
        for (int j = max(0, c - 2); ok && j < c; ++j) ok = wait.warp(&d_empty[j & 1], (uint32_t)(j >> 1) & 1u);
        // every product issued ends before the blocks free their memory
        if (rank == 0) {
            if (elected()) pair_commit(&drained);
            __syncwarp();
            land(&drained, 0);
        }
        __syncwarp();
    } else if (warp > kEpiWarps) {
        fewer_registers();
    } else {
        // ---------------- what becomes of a tile ----------------
        more_registers();
        const int quarter = warp & 3, half = warp >> 2, r_warp = rank * kHalf + quarter * 32, r = r_warp + lane;
        const uint32_t released = at_first(&d_empty[0]);
        const uint32_t lanes = tmem + ((uint32_t)(quarter * 32) << 16);
        unsigned char *const outs_at = base + kStages * kStageBytes + warp * outs(MODE) * kOutBytes;
        unsigned char *out = outs_at;
        const float factor = MODE == 2 ? a.ctl->factor * a.scale / kUp<T> : 0.f;
        int c = 0;
        bool ok = true;
        for (int i = pair; ok && i < walk.total; i += pairs) {
            float top = -INFINITY, sum = 0.f, lse = INFINITY, dloss = 0.f, part = 0.f, q_target = 0.f;
            int target = -1, row = 0;
            bool live = false;
            if (MODE != 2) {
                row = walk.tile(i, 0).m0 + r;
                live = row < walk.n;
                if (live) target = a.target[row];
                if (MODE == 1 && live) {
                    lse = a.lse[row];
                    if (lse == -INFINITY) lse = INFINITY;       // every class hidden: no probabilities either
                    if (!BIAS) lse *= kLog2e;
                    dloss = a.dloss[row];
                    part = a.part_of[row] * kUp<T>;
                    q_target = a.at_target[row];
                }
            }
            for (int k = 0, nk = walk.tiles(i); ok && k < nk; ++k) {
                const Tile t = walk.tile(i, k);
                // this warp's columns of the tile
                const int col = t.n0 + half * (kN / 2);
                if (MODE != 2 && BIAS) {
                    __syncwarp();
#pragma unroll
                    for (int j = 0; j < kN / 2; j += 32)
                        s_bias[warp][j + lane] = col + j + lane < a.classes ? __ldg(a.bias + col + j + lane) : -INFINITY;
                    __syncwarp();
                }
                // The tile's sums: its chunks added up, each released as soon as it is
                // in registers, so that the next tile's products run under what follows.
                uint32_t acc[kN / 64][32];
                auto chunk = [&](bool first) {
                    if (!(ok = wait.warp(&d_full[c & 1], (uint32_t)(c >> 1) & 1u, a.wait_limit))) return;
                    tc::fence_after_sync();
                    const uint32_t from = lanes + (c & 1) * kN + half * (kN / 2);
                    if (first) {
#pragma unroll
                        for (int j = 0; j < kN / 64; ++j) tc::tmem_ld32_issue(from + 32 * j, acc[j]);
#pragma unroll
                        for (int j = 0; j < kN / 64; ++j) tc::tmem_ld_wait(acc[j]);
                    } else {
#pragma unroll
                        for (int j = 0; j < kN / 64; ++j) {
                            float x[32];
                            tc::tmem_ld32(from + 32 * j, x);
#pragma unroll
                            for (int e = 0; e < 32; e += 2) {
                                const float2 v = add2(get(x + e), make_float2(__uint_as_float(acc[j][e]), __uint_as_float(acc[j][e + 1])));
                                acc[j][e] = __float_as_uint(v.x);
                                acc[j][e + 1] = __float_as_uint(v.y);
                            }
                        }
                    }
                    tc::fence_before_sync();
                    warp_arrive_at(released + (c & 1) * 8);
                    ++c;
                };
                if (MODE != 2) {
                    chunk(true);
                } else {
#pragma unroll
                    for (int j = 0; j < kN / 64; ++j)
#pragma unroll
                        for (int e = 0; e < 32; ++e) acc[j][e] = 0u;
                }
#pragma unroll 1
                for (int b = MODE != 2 ? chunk_of() : 0; ok && b < t.blocks; b += chunk_of()) chunk(false);
                if (!ok) break;
                auto take = [&](int j, float (&x)[32]) {
#pragma unroll
                    for (int e = 0; e < 32; ++e) x[e] = __uint_as_float(acc[j / 32][e]);
                };
                const float *bias = s_bias[warp];
                // whether a row's target is among these columns, or the classes end there
                // (rows past the list: lse = inf, so their probabilities are zero)
                const int at0 = target >= 0 ? target - col : -1, left0 = a.classes - col;
                const bool hits = MODE == 0 && __any_sync(0xffffffffu, at0 >= 0 && at0 < kN / 2);
                const bool ends = MODE != 2 && left0 < kN / 2;
                if constexpr (MODE == 0) {
#pragma unroll
                    for (int j = 0; j < kN / 2; j += 32) {
                        float x[32];
                        take(j, x);
#pragma unroll
                        for (int e = 0; e < 32; e += 2)
                            put(x + e, BIAS ? fma2(get(x + e), both(a.scale), get(bias + j + e)) : mul2(get(x + e), both(a.c)));
                        if (!BIAS && ends)
#pragma unroll
                            for (int e = 0; e < 32; ++e) x[e] = j + e < left0 ? x[e] : -INFINITY;
                        const bool here = at0 >= j && at0 < j + 32;
                        if (hits && __any_sync(0xffffffffu, here)) {
                            float hit = 0.f;
#pragma unroll
                            for (int e = 0; e < 32; ++e)
                                if (j + e == at0) {
                                    hit = x[e];
                                    x[e] = -INFINITY;
                                }
                            if (here) a.hit[row] = hit;
                        }
                        const float high = fmaxf(top, max_of_32(x)), from = high == -INFINITY ? 0.f : high;
                        constexpr float unit = BIAS ? kLog2e : 1.f;
                        float2 s0 = make_float2(sum * exp2_approx((top - from) * unit), 0.f), s1 = make_float2(0.f, 0.f);
#pragma unroll
                        for (int e = 0; e < 32; e += 4) {
                            float2 u = add2(get(x + e), both(-from)), v = add2(get(x + e + 2), both(-from));
                            if (BIAS) {
                                u = mul2(u, both(unit));
                                v = mul2(v, both(unit));
                            }
                            s0 = add2(s0, make_float2(exp2_approx(u.x), exp2_approx(u.y)));
                            s1 = add2(s1, make_float2(exp2_approx(v.x), exp2_approx(v.y)));
                        }
                        s0 = add2(s0, s1);
                        sum = s0.x + s0.y;
                        top = high;
                    }
                } else if constexpr (MODE == 1) {
                    float2 rest = make_float2(0.f, 0.f);
                    auto columns = [&](auto second) {
                    constexpr bool pass = decltype(second)::value;
#pragma unroll
                    for (int j = 0; j < kN / 2; j += 64) {
                        uint32_t packed[32];
                        float2 some = make_float2(0.f, 0.f);      // of these columns
                        out = outs_at + j / 64 * kOutBytes;
                        one_store_read();      // the one from this buffer, but not the last
                        __syncwarp();
#pragma unroll
                        for (int jj = 0; jj < 64; jj += 32) {
                            float x[32];
                            take(j + jj, x);
#pragma unroll
                            for (int e = 0; e < 32; e += 2) {
                                float2 u;
                                if (BIAS)
                                    u = mul2(add2(fma2(get(x + e), both(a.scale), get(bias + j + jj + e)), both(-lse)), both(kLog2e));
                                else
                                    u = fma2(get(x + e), both(a.c), both(-lse));
                                x[e] = exp2_approx(u.x);
                                x[e + 1] = exp2_approx(u.y);
                            }
                            if (!BIAS && ends)      // (a bias ends in -inf)
#pragma unroll
                                for (int e = 0; e < 32; ++e) x[e] = j + jj + e < left0 ? x[e] : 0.f;
#pragma unroll
                            for (int e = 0; e < 32; e += 2) {
                                const float2 q = mul2(get(x + e), both(part));
                                packed[(jj + e) / 2] = pack2<T>(q.x, q.y);
                                if constexpr (pass) {
                                    const float2 is = add_pair<T>(make_float2(0.f, 0.f), packed[(jj + e) / 2]);
                                    packed[(jj + e) / 2] = pack2<T>(q.x - is.x, q.y - is.y);
                                }
                                some = add_pair<T>(some, packed[(jj + e) / 2]);
                            }
                            if (BIAS && !pass && a.want_db) {
                                // The columns' sums over the warp's rows, turned in the buffer that
                                // the packed values leave from later: a lane takes four columns of eight
                                // rows.  (In registers alone, 31 shuffles and twice as many selects.)
                                const float2 d = both(live ? dloss : 0.f);
#pragma unroll
                                for (int e = 0; e < 8; ++e) {
                                    const float2 u = mul2(get(x + 4 * e), d), v = mul2(get(x + 4 * e + 2), d);
                                    *reinterpret_cast<float4 *>(out + lane * 128 + ((e ^ (lane & 7)) << 4)) = make_float4(u.x, u.y, v.x, v.y);
                                }
                                if (at0 >= j + jj && at0 < j + jj + 32) {
                                    const int e = at0 - j - jj;
                                    *reinterpret_cast<float *>(out + lane * 128 + (((e >> 2) ^ (lane & 7)) << 4) + (e & 3) * 4) =
                                        q_target * dloss;
                                }
                                __syncwarp();
                                float2 u = make_float2(0.f, 0.f), v = u;
#pragma unroll
                                for (int k = 0; k < 8; ++k) {
                                    const float4 f = *reinterpret_cast<const float4 *>(out + ((lane & 24) + k) * 128 + (((lane & 7) ^ k) << 4));
                                    u = add2(u, make_float2(f.x, f.y));
                                    v = add2(v, make_float2(f.z, f.w));
                                }
#pragma unroll
                                for (int w = 8; w <= 16; w <<= 1) {
                                    u = add2(u, make_float2(__shfl_xor_sync(0xffffffffu, u.x, w), __shfl_xor_sync(0xffffffffu, u.y, w)));
                                    v = add2(v, make_float2(__shfl_xor_sync(0xffffffffu, v.x, w), __shfl_xor_sync(0xffffffffu, v.y, w)));
                                }
                                const int at = col + j + jj + 4 * (lane & 7) + (lane >> 3);
                                const float mine = lane & 16 ? (lane & 8 ? v.y : v.x) : (lane & 8 ? u.y : u.x);
                                if (at < a.classes) a.colsum[(int64_t)((t.m0 + r_warp) / 32) * a.classes + at] = mine;
                                __syncwarp();
                            }
                        }
#pragma unroll
                        for (int e = 0; e < 8; ++e)
                            *reinterpret_cast<uint4 *>(out + lane * 128 + ((e ^ (lane & 7)) << 4)) =
                                make_uint4(packed[4 * e], packed[4 * e + 1], packed[4 * e + 2], packed[4 * e + 3]);
                        // The target's goes to its place here: nearly every tile has some row's, and
                        // a choice at every element of it cost half as long again.  Such a
                        // row is added up anew: p near 1 must not leave its rounding in the sum.
                        if (at0 >= j && at0 < j + 64) {
                            const int e = at0 - j;
                            float q = q_target * part;
                            if (pass) q -= to_f32<T>(from_f32<T>(q));
                            reinterpret_cast<T *>(out + lane * 128 + (((e >> 3) ^ (lane & 7)) << 4))[e & 7] = from_f32<T>(q);
                            some = make_float2(0.f, 0.f);
#pragma unroll 1
                            for (int c8 = 0; c8 < 8; ++c8) {
                                const uint4 v = *reinterpret_cast<const uint4 *>(out + lane * 128 + (c8 << 4));
                                some = add_pair<T>(add_pair<T>(add_pair<T>(add_pair<T>(some, v.x), v.y), v.z), v.w);
                            }
                        }
                        rest = add2(rest, some);
                        tc::fence_proxy_async_smem();
                        __syncwarp();
                        if (lane == 0) {
                            store_box(&a.pool_out, 0, (col + j - walk.v0) / kK * walk.panel + (pass ? walk.mp : 0) + t.m0 + r_warp, out);
                            stores_issued();
                        }
                    }
                    };
                    columns(std::false_type{});
                    if (walk.fine) columns(std::true_type{});       // what the rounding left off
                    if (live) a.rest[(int64_t)(t.n0 / kN * 2 + half) * walk.mp + row] = rest.x + rest.y;
                } else {
                    const int columns = 2 * t.n_boxes * kBox;    // of the tile that exist
                    const int r0 = (t.dw ? walk.v0 : t.slab * walk.mp) + t.m0 + r_warp;
                    const bool some = t.dw ? r0 < walk.v1 : true;
                    const bool wide = !t.dw || a.dw_f32;         // fp32 results: 32 columns to a box, else 64
                    const bool adds = t.dw ? a.accumulate : piece > 0;
                    const float f = t.dw ? factor : 1.f;
                    // (dh: past the list's rows of the last tile nothing is read again)
#pragma unroll
                    for (int j = 0; j < kN / 2; j += 64) {
                        if (half * (kN / 2) + j >= columns) break;
                        const int x0 = t.n0 + half * (kN / 2) + j;
                        const CUtensorMap *map = t.dw ? &a.dw : &a.acc;
                        uint32_t packed[32];
#pragma unroll
                        for (int b = 0; b < 2; ++b) {
                            float x[32];
                            take(j + 32 * b, x);
#pragma unroll
                            for (int e = 0; e < 32; ++e) x[e] *= f;
                            if (wide) {
                                stores_read();
                                __syncwarp();
#pragma unroll
                                for (int e = 0; e < 8; ++e)
                                    *reinterpret_cast<float4 *>(out + lane * 128 + ((e ^ (lane & 7)) << 4)) =
                                        make_float4(x[4 * e], x[4 * e + 1], x[4 * e + 2], x[4 * e + 3]);
                                tc::fence_proxy_async_smem();
                                __syncwarp();
                                if (lane == 0 && some && x0 + 32 * b < a.width) {
                                    if (adds) add_box(map, x0 + 32 * b, r0, out);
                                    else store_box(map, x0 + 32 * b, r0, out);
                                    stores_issued();
                                }
                            } else {
#pragma unroll
                                for (int e = 0; e < 16; ++e) packed[16 * b + e] = pack2<T>(x[2 * e], x[2 * e + 1]);
                            }
                        }
                        if (!wide) {
                            stores_read();
                            __syncwarp();
#pragma unroll
                            for (int e = 0; e < 8; ++e)
                                *reinterpret_cast<uint4 *>(out + lane * 128 + ((e ^ (lane & 7)) << 4)) =
                                    make_uint4(packed[4 * e], packed[4 * e + 1], packed[4 * e + 2], packed[4 * e + 3]);
                            tc::fence_proxy_async_smem();
                            __syncwarp();
                            if (lane == 0 && some && x0 < a.width) {
                                store_box(map, x0, r0, out);
                                stores_issued();
                            }
                        }
                    }
                }
            }
            if (MODE == 0 && ok && live)
                a.part[(int64_t)(i / walk.row_tiles * 2 + half) * walk.mp + row] = make_float2(top, sum);
        }
        stores_done();
    }
    tc::fence_before_sync();
    __syncthreads();
    if (warp == kEpiWarps && *(volatile int *)&s_abort) linger();
    pair_sync();          // neither leaves while the other's copies, products or arrivals may reach it
    tc::fence_after_sync();
    if (warp == kEpiWarps + 1 && rank == 1) land(&drained, 0);      // the first block's last arrival here
    if (warp == 0) pair_dealloc(tmem, kTmemCols);
    if (threadIdx.x == 0 && s_abort) atomicExch(&a.ctl->status, SIEVE_ETIMEOUT);
}

// ---------------------------------------------------------------------------
// The parts of a row's statistics added up: 32 rows by 16 strands of parts.
struct JoinArgs {
    const Ctl *ctl;
    const int *row;
    const float *hit;
    const float2 *part;
    int classes, biased;
    float *loss, *lse;
};
constexpr int kStrands = 16;

__global__ void __launch_bounds__(32 * kStrands) k_xent_join(const JoinArgs a) {
    __shared__ float2 s_part[kStrands][32];
    const int lane = lane_id(), strand = threadIdx.x >> 5;
    const int n = a.ctl->n;
    const int group = group_tiles(n, a.classes), tiles = (a.classes + kN - 1) / kN;
    const int parts = (tiles + group - 1) / group * 2;
    const int64_t stride = padded(n);
    const float unit = a.biased ? kLog2e : 1.f;
    for (int64_t i0 = (int64_t)blockIdx.x * 32; i0 < n; i0 += (int64_t)gridDim.x * 32) {
        const int64_t i = i0 + lane;
        float m = -INFINITY, s = 0.f;
        // eight parts at a time against their common maximum
        auto merge = [&](const float2 (&p)[8]) {
            float high = m;
#pragma unroll
            for (int k = 0; k < 8; ++k) high = fmaxf(high, p[k].x);
            const float from = high == -INFINITY ? 0.f : high;
            s *= exp2_approx((m - from) * unit);
#pragma unroll
            for (int k = 0; k < 8; ++k) s += p[k].y * exp2_approx((p[k].x - from) * unit);
            m = high;
        };
        if (i < n)
            for (int p = strand; p < parts; p += 8 * kStrands) {
                float2 some[8];
#pragma unroll
                for (int k = 0; k < 8; ++k)
                    some[k] = p + k * kStrands < parts ? a.part[(p + k * kStrands) * stride + i] : make_float2(-INFINITY, 0.f);
                merge(some);
            }
        __syncthreads();
        s_part[strand][lane] = make_float2(m, s);
        __syncthreads();
        if (strand > 0 || i >= n) continue;
        m = -INFINITY;
        s = 0.f;
        for (int k0 = 0; k0 < kStrands; k0 += 8) {
            float2 some[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) some[k] = s_part[k0 + k][lane];
            merge(some);
        }
        // the others' sum s 2^m and the target's score, in base 2 (a bias: in base e)
        const float hit = a.hit[i], d = (m - hit) * unit;
        const float ln = a.biased ? 1.f : kLn2;               // to natural units
        float loss, lse;
        if (hit == -INFINITY) {                               // a hidden target
            loss = INFINITY;
            lse = m == -INFINITY ? -INFINITY : m * ln + logf(s);
        } else if (m <= hit) {
            loss = log1pf(s * exp2f(d));
            lse = hit * ln + loss;
        } else {
            const float more = logf(s + exp2f(-d));
            loss = (m - hit) * ln + more;
            lse = m * ln + more;
        }
        if (isnan(s) || isnan(hit)) loss = lse = NAN;
        const int64_t r = a.row[i];
        a.loss[r] = loss;
        a.lse[r] = lse;
    }
}

// dh from its slabs' sums: the list's rows to their places, 32 to a block, with
// what the rounded q of a row add up to taken off the target's.
struct DhArgs {
    const Ctl *ctl;
    const int *row, *target;
    const float *whole, *lse, *acc, *rest;
    const void *weight;
    void *dh;
    int64_t weight_stride, dh_stride, pool_rows;
    int classes, width, want_dw;
    float scale;
};
template <typename T>
__global__ void __launch_bounds__(32 * kStrands) k_xent_dh(const DhArgs a) {
    __shared__ float s_rest[kStrands][32];
    const int lane = lane_id(), strand = threadIdx.x >> 5, n = a.ctl->n, chunks = a.width / 8;
    const int64_t mp = padded(n);
    const int parts = (a.classes + kN - 1) / kN * 2;
    const int slabs = dh_slabs(n, a.classes, a.width, a.pool_rows, a.want_dw);
    for (int64_t i0 = (int64_t)blockIdx.x * 32; i0 < n; i0 += (int64_t)gridDim.x * 32) {
        float sum = 0.f;
        if (i0 + lane < n)
#pragma unroll 8
            for (int p = strand; p < parts; p += kStrands) sum += a.rest[p * mp + i0 + lane];
        __syncthreads();
        s_rest[strand][lane] = sum;
        __syncthreads();
        for (int k = strand; k < 32 && i0 + k < n; k += kStrands) {
            const int64_t i = i0 + k;
            float rest = 0.f;
            for (int p = 0; p < kStrands; ++p) rest -= s_rest[p][k];
            if (a.lse[i] == -INFINITY) rest = 0.f;        // every class hidden: the target's -1 is all that q holds
            const float f = a.whole[i] * a.scale / kUp<T>;
            const T *w = static_cast<const T *>(a.weight) + a.target[i] * a.weight_stride;
            T *out = static_cast<T *>(a.dh) + a.row[i] * a.dh_stride;
            for (int c = lane; c < chunks; c += 32) {
                float v[8];
                load_vec<T, 8>(w + 8 * c, v);
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] *= rest;
                for (int s = 0; s < slabs; ++s) {
                    const float4 *x = reinterpret_cast<const float4 *>(a.acc + (s * mp + i) * a.width) + 2 * c;
                    const float4 p = __ldcs(x), q = __ldcs(x + 1);
                    const float y[8] = {p.x, p.y, p.z, p.w, q.x, q.y, q.z, q.w};
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[e] += y[e];
                }
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] *= f;
                reinterpret_cast<uint4 *>(out)[c] = pack8<T>(v);
            }
        }
    }
}

// dbias from the column sums of every 32 rows: 32 columns by 8 strands.
__global__ void __launch_bounds__(256) k_xent_db(const Ctl *ctl, const float *colsum, int classes, float *db) {
    __shared__ float part[8][32];
    const int lane = lane_id(), strand = threadIdx.x >> 5, v = blockIdx.x * 32 + lane;
    const int sums = (ctl->n + kM - 1) / kM * (kM / 32);
    float s = 0.f;
    if (v < classes)
#pragma unroll 4
        for (int t = strand; t < sums; t += 8) s += colsum[(int64_t)t * classes + v];
    part[strand][lane] = s;
    __syncthreads();
    if (strand || v >= classes) return;
    for (int k = 1; k < 8; ++k) s += part[k][lane];
    db[v] = s;
}

// ---------------------------------------------------------------------------
struct Layout {
    size_t count, top, low, reach, row, target, dloss, at_target, lse, hc, hs, hit, part, part_of, whole, pool, acc, rest, colsum, bytes;
    int64_t pool_rows, acc_rows;
};
Layout layout(const sieve_cross_entropy_args &a, bool backward) {
    Layout l = {};
    size_t at = kCtlBytes;
    auto take = [&](int64_t bytes) {
        const size_t here = at;
        at += (size_t)round_up(bytes, 1024);
        return here;
    };
    const int64_t n = a.rows, np = padded(n), blocks = ceil_div(n, kRowTile);
    l.count = take(blocks * 4);
    l.row = take(n * 4);
    l.target = take(n * 4);
    l.hc = take(n * a.width * 2);
    if (!backward) {
        const int64_t row_tiles = np / kM, class_tiles = ceil_div(a.classes, kN);
        // (group_tiles: up to 16 tiles a part, and no fewer than 8 parts a pair before that)
        const int64_t whole = ceil_div(row_tiles * class_tiles, kMaxGroup), parts = (whole > 16 * kPairs ? whole : 16 * kPairs) + row_tiles;
        l.hit = take(n * 4);
        l.part = take((parts < row_tiles * class_tiles ? parts : row_tiles * class_tiles) * 2 * kM * 8);
    } else {
        l.top = take(blocks * 4);
        l.low = take(blocks * 4);
        if (a.dtype == SIEVE_F16) l.reach = take(blocks * (n <= kFewRows ? kManyBlocks : 1) * 4);
        l.dloss = take(n * 4);
        l.at_target = take(n * 4);
        l.lse = take(n * 4);
        l.part_of = take(n * 4);
        l.whole = take(n * 4);
        l.hs = take(n * a.width * 2);
        const int64_t needed = panel_rows(n) * (round_up(a.classes, kN) / kK), least = panel_rows(n) * (kN / kK), most = kPoolBytes / 128;
        l.pool_rows = needed < most ? needed : least > most ? least : most;
        l.pool = take(l.pool_rows * 128);
        // (dh_slabs: tiles times slabs stay below two shares for each pair, or there is one slab)
        const int64_t across = ceil_div(a.width, kN), some = 2 * kPairs / across + 1;
        const int64_t most_slabs = np / kM * kMaxSlabs < np / kM + some ? np / kM * kMaxSlabs : np / kM + some;
        l.acc_rows = most_slabs * kM;
        l.acc = take(l.acc_rows * a.width * 4);
        l.rest = take(ceil_div(a.classes, kN) * 2 * np * 4);
        if (a.bias) l.colsum = take(np / 32 * a.classes * 4);
    }
    l.bytes = at;
    return l;
}

template <typename T, int MODE, bool BIAS>
cudaError_t run(const XentArgs &a, int piece, cudaStream_t st) {
    auto kernel = k_xent<T, MODE, BIAS>;
    // The warps trade registers among each other, which takes all that kRegisters says: a
    // compiler that gives the kernel another number has built an image that cannot run.
    // (Asked once a kernel; an answer that is an error is not kept.)
    static std::atomic<int> registers{0};
    if (!registers) {
        cudaFuncAttributes f;
        const cudaError_t found = cudaFuncGetAttributes(&f, kernel);
        if (found != cudaSuccess) return found;
        registers = f.numRegs;
    }
    if (registers != kRegisters) return cudaErrorInvalidKernelImage;
    cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem_bytes(MODE));
    if (e != cudaSuccess) return e;
    kernel<<<kGrid, kThreads, smem_bytes(MODE), st>>>(a, piece);
    return cudaGetLastError();
}

struct Call {
    XentArgs x;
    RowArgs r;
    unsigned blocks;
};
sieve_status prepare(Call &c, const sieve_cross_entropy_args &a, const Layout &l, unsigned char *ws) {
    std::memset(&c, 0, sizeof c);
    XentArgs &x = c.x;
    x.ctl = reinterpret_cast<Ctl *>(ws);
    x.target = reinterpret_cast<int *>(ws + l.target);
    x.bias = a.bias;
    x.rows = (int)a.rows;
    x.classes = (int)a.classes;
    x.width = a.width;
    x.scale = a.scale;
    x.c = a.scale * kLog2e;
    x.wait_limit = a.wait_limit;
    RowArgs &r = c.r;
    r.targets = a.targets;
    r.h = a.h;
    r.h_stride = a.h_stride;
    r.rows = x.rows;
    r.classes = x.classes;
    r.width = a.width;
    r.target_type = a.target_type;
    r.ctl = x.ctl;
    r.count = reinterpret_cast<int *>(ws + l.count);
    r.row = reinterpret_cast<int *>(ws + l.row);
    r.target = reinterpret_cast<int *>(ws + l.target);
    r.hc = ws + l.hc;
    c.blocks = (unsigned)ceil_div(a.rows, kRowTile);
    sieve_status rc = make_matrix_map(&x.h, a.dtype, a.h, a.rows, a.width, a.h_stride, kBox);
    if (rc == SIEVE_OK) rc = make_matrix_map(&x.hc, a.dtype, ws + l.hc, a.rows, a.width, a.width, kBox);
    if (rc == SIEVE_OK) rc = make_matrix_map(&x.w, a.dtype, a.weight, a.classes, a.width, a.weight_stride, kBox);
    return rc;
}

template <typename T, int SUB>
cudaError_t list_rows_by(const Call &c, cudaStream_t st) {
    if (c.r.reach) {
        k_xent_count<SUB><<<c.blocks * SUB, kRowTile, 0, st>>>(c.r);
    } else if (c.blocks > 1) {
        k_xent_count<0><<<c.blocks, kRowTile, 0, st>>>(c.r);
    }
    k_xent_rows<T, SUB><<<c.blocks * SUB, kRowTile, 0, st>>>(c.r);
    return cudaGetLastError();
}
template <typename T>
cudaError_t list_rows(const Call &c, cudaStream_t st) {
    return c.x.rows <= kFewRows ? list_rows_by<T, kManyBlocks>(c, st) : list_rows_by<T, 1>(c, st);
}

template <typename T>
cudaError_t forward(const Call &c, const JoinArgs &j, cudaStream_t st) {
    cudaError_t e = list_rows<T>(c, st);
    if (e != cudaSuccess) return e;
    e = c.x.bias ? run<T, 0, true>(c.x, 0, st) : run<T, 0, false>(c.x, 0, st);
    if (e != cudaSuccess) return e;
    const int64_t blocks = ceil_div(c.x.rows, 32);
    k_xent_join<<<(unsigned)(blocks < 4096 ? blocks : 4096), 32 * kStrands, 0, st>>>(j);
    return cudaGetLastError();
}

template <typename T>
cudaError_t backward(const Call &c, const sieve_cross_entropy_grads &g, const DhArgs &d, int pieces, cudaStream_t st) {
    cudaError_t e = list_rows<T>(c, st);
    if (e != cudaSuccess) return e;
    for (int p = 0; p < pieces; ++p) {
        e = c.x.bias ? run<T, 1, true>(c.x, p, st) : run<T, 1, false>(c.x, p, st);
        if (e == cudaSuccess && (g.dh || g.dweight)) e = run<T, 2, false>(c.x, p, st);
        if (e != cudaSuccess) return e;
    }
    if (g.dh) {
        const int64_t blocks = ceil_div(c.x.rows, 32);
        k_xent_dh<T><<<(unsigned)(blocks < 4096 ? blocks : 4096), 32 * kStrands, 0, st>>>(d);
    }
    if (g.dbias) k_xent_db<<<(unsigned)ceil_div(c.x.classes, 32), 256, 0, st>>>(c.x.ctl, c.x.colsum, c.x.classes, g.dbias);
    return cudaGetLastError();
}

}  // namespace

size_t cross_entropy_workspace_bytes(const sieve_cross_entropy_args &a) { return layout(a, false).bytes; }
size_t cross_entropy_backward_workspace_bytes(const sieve_cross_entropy_args &a) { return layout(a, true).bytes; }

sieve_status launch_cross_entropy(const sieve_cross_entropy_args &a, float *loss, float *lse, void *ws,
                                  cudaStream_t st) {
    unsigned char *base = static_cast<unsigned char *>(ws);
    const Layout l = layout(a, false);
    Call c;
    const sieve_status rc = prepare(c, a, l, base);
    if (rc != SIEVE_OK) return rc;
    c.x.hit = reinterpret_cast<float *>(base + l.hit);
    c.x.part = reinterpret_cast<float2 *>(base + l.part);
    c.r.loss_out = loss;
    c.r.lse_out = lse;
    const JoinArgs j = {c.x.ctl, c.r.row, c.x.hit, c.x.part, c.x.classes, a.bias != nullptr, loss, lse};
    const cudaError_t e = a.dtype == SIEVE_F16 ? forward<__half>(c, j, st) : forward<__nv_bfloat16>(c, j, st);
    return e == cudaSuccess ? SIEVE_OK : record_cuda_error(e);
}

sieve_status launch_cross_entropy_backward(const sieve_cross_entropy_args &a, const sieve_cross_entropy_grads &g,
                                           void *ws, cudaStream_t st) {
    unsigned char *base = static_cast<unsigned char *>(ws);
    const Layout l = layout(a, true);
    Call c;
    sieve_status rc = prepare(c, a, l, base);
    if (rc != SIEVE_OK) return rc;
    c.x.lse = reinterpret_cast<float *>(base + l.lse);
    c.x.at_target = reinterpret_cast<float *>(base + l.at_target);
    c.x.dloss = reinterpret_cast<float *>(base + l.dloss);
    c.x.colsum = reinterpret_cast<float *>(base + l.colsum);
    c.x.rest = reinterpret_cast<float *>(base + l.rest);
    c.x.pool_rows = l.pool_rows;
    c.x.want_dh = g.dh != nullptr;
    c.x.want_dw = g.dweight != nullptr;
    c.x.want_db = g.dbias != nullptr;
    c.x.dw_f32 = g.dweight_dtype == SIEVE_F32;
    c.x.accumulate = g.accumulate;
    c.r.dloss = g.dloss;
    c.r.loss = g.loss;
    c.r.lse = g.lse;
    c.r.dh = g.dh;
    c.r.dh_stride = g.dh_stride;
    c.r.top = reinterpret_cast<uint32_t *>(base + l.top);
    c.r.low = reinterpret_cast<uint32_t *>(base + l.low);
    c.r.dloss_c = reinterpret_cast<float *>(base + l.dloss);
    c.r.at_target_c = reinterpret_cast<float *>(base + l.at_target);
    c.r.lse_c = reinterpret_cast<float *>(base + l.lse);
    c.r.part_c = reinterpret_cast<float *>(base + l.part_of);
    c.r.whole_c = reinterpret_cast<float *>(base + l.whole);
    c.x.part_of = c.r.part_c;
    if (g.dweight) {
        c.r.hs = base + l.hs;
        if (a.dtype == SIEVE_F16) c.r.reach = reinterpret_cast<int *>(base + l.reach);
        // (2^(least - 15), and that times the scale and over kUp, are normal)
        c.r.least = std::max(-97 - (a.scale == 0.f ? 0 : std::ilogb(a.scale)), -111);
    }
    rc = make_matrix_map(&c.x.hs, a.dtype, base + l.hs, a.rows, a.width, a.width, kBox);
    if (rc == SIEVE_OK) rc = make_matrix_map(&c.x.pool_in, a.dtype, base + l.pool, l.pool_rows, kK, kK, kBox);
    if (rc == SIEVE_OK) rc = make_matrix_map(&c.x.pool_out, a.dtype, base + l.pool, l.pool_rows, kK, kK, 32);
    if (rc == SIEVE_OK) rc = make_matrix_map(&c.x.acc, SIEVE_F32, base + l.acc, l.acc_rows, a.width, a.width, 32);
    if (rc == SIEVE_OK && g.dweight)
        rc = make_matrix_map(&c.x.dw, g.dweight_dtype, g.dweight, a.classes, a.width, g.dweight_stride, 32);
    if (rc != SIEVE_OK) return rc;
    const int each = piece_classes(a.rows, c.x.classes, l.pool_rows), pieces = (int)ceil_div(a.classes, each);
    const DhArgs d = {c.x.ctl, c.r.row, c.x.target, c.r.whole_c, c.r.lse_c, reinterpret_cast<const float *>(base + l.acc), c.x.rest, a.weight,
                      g.dh, a.weight_stride, g.dh_stride, l.pool_rows, c.x.classes, a.width, c.x.want_dw, a.scale};
    const cudaError_t e = a.dtype == SIEVE_F16 ? backward<__half>(c, g, d, pieces, st)
                                               : backward<__nv_bfloat16>(c, g, d, pieces, st);
    return e == cudaSuccess ? SIEVE_OK : record_cuda_error(e);
}

}  // namespace enc
}  // namespace sieve
