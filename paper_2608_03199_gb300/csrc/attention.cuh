// attention.cuh -- what the attention kernels share: the documents' rows,
// operand descriptors and tensor maps, the bias by distance, bounded waits.
//
// Operand tiles.  A tile of 128 rows (queries or keys) of one head is loaded
// by TMA as one or two column blocks of 64 elements: 128 rows of 128 bytes,
// 128-byte swizzle, 16 KB a block.  Columns past head_dim arrive as zeros, so
// every head_dim up to 64 runs as 64 and every one up to 128 as 128.  One tile
// serves two products: as a K-major operand its row is the contraction axis'
// vector (q k^T, dout v^T), as an MN-major operand its rows are the
// contraction axis (p v, ds k).
//
// Rows past a document's end belong to the next document and may hold
// anything.  Scores of such keys are replaced before they are used; where such
// rows are the contraction axis their probabilities are exact zeros, but
// 0 x NaN is NaN, so the warp that issues the products first clears those
// rows of the tile (the last of a document, in its idle time).
#pragma once

#include <cuda.h>

#include <type_traits>

#include "encoder.cuh"
#include "tcgen05.cuh"

namespace sieve {
namespace enc {

constexpr int kTile = 128;                    // rows of a tile
constexpr uint32_t kBlockBytes = kTile * 128;   // one 64-column block of a tile
constexpr uint32_t kPolls = 1u << 24;
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

// Instruction descriptor of kind::f16, fp32 accumulation, M = 128: both
// operands fp16 (format 0) or bf16 (format 1), B K-major or MN-major (bit 16).
template <typename T>
__host__ __device__ constexpr uint32_t idesc(int N, bool b_mn) {   // N a multiple of 16
    const uint32_t f = std::is_same_v<T, __half> ? 0u : 1u;
    return (1u << 4) | (f << 7) | (f << 10) | ((b_mn ? 1u : 0u) << 16) | ((uint32_t)(N >> 3) << 17) |
           ((uint32_t)(kTile >> 4) << 24);
}

// The products are issued by one elected thread of their warp, whole groups of
// them under one branch (measured 76 instructions for a group of 12 products
// and its wait; 175 with every instruction predicated on the lane).
__device__ __forceinline__ bool elected() {
    uint32_t p;
    asm volatile("{\n\t.reg .pred q;\n\telect.sync _|q, 0xffffffff;\n\tselp.u32 %0, 1, 0, q;\n\t}" : "=r"(p));
    return p != 0;
}
// Operand descriptors with 128-byte swizzle.  K-major: as in tcgen05.cuh.
// MN-major: the 64-element blocks of the M or N axis lie kBlockBytes apart
// (leading offset), groups of 8 rows of the contraction axis 1024 bytes apart.
__device__ __forceinline__ uint64_t desc_k(const void *tile) {      // K-major
    return tc::desc_k_sw128(tc::smem_u32(tile));
}
__device__ __forceinline__ uint64_t desc_mn(const void *tile) {     // MN-major
    return (tc::desc_k_sw128(tc::smem_u32(tile)) & ~((uint64_t)0x3FFF << 16)) | (uint64_t)(kBlockBytes >> 4) << 16;
}
constexpr uint32_t kBlockStep = kBlockBytes >> 4;                   // in a descriptor's units
__device__ __forceinline__ void mma_ss(uint32_t d_tmem, uint64_t a, uint64_t b, uint32_t id, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d_tmem),
        "l"(a), "l"(b), "r"(id), "r"(accumulate)
        : "memory");
}
__device__ __forceinline__ void mma_ts(uint32_t d_tmem, uint32_t a_tmem, uint64_t b, uint32_t id, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d_tmem),
        "r"(a_tmem), "l"(b), "r"(id), "r"(accumulate)
        : "memory");
}
__device__ __forceinline__ void commit(uint64_t *bar) { tc::mma_commit(1u, bar); }
// D = A B^T, both operands in shared memory and K-major: COLS contraction
// columns in blocks of 64, the blocks of A and B kBlockBytes apart.
template <int COLS>
__device__ __forceinline__ void mma_kk(uint32_t d_tmem, uint64_t a, uint64_t b, uint32_t id) {
#pragma unroll
    for (int k = 0; k < COLS / 16; ++k) {
        const uint64_t o = (k / 4) * kBlockStep + (k % 4) * 2;
        mma_ss(d_tmem, a + o, b + o, id, k > 0);
    }
}
// D (+)= A B with A (128 x 128, 16-bit pairs) in tensor memory, kept in groups
// of kCols columns: a group's pairs at the start of the kStride 32-bit columns
// of its own.  B a tile whose rows are the contraction axis.
template <int kCols, int kStride>
__device__ __forceinline__ void mma_groups(uint32_t d_tmem, uint32_t a_tmem, uint64_t b, uint32_t id,
                                           uint32_t accumulate) {
#pragma unroll
    for (int k = 0; k < kTile / 16; ++k)
        mma_ts(d_tmem, a_tmem + (16 * k / kCols) * kStride + (16 * k % kCols) / 2, b + k * 128, id,
               k > 0 ? 1u : accumulate);
}

// a value that is the same in the whole warp, made so for the compiler too:
// control flow that depends on it does not diverge
__device__ __forceinline__ int uniform(int x) { return __shfl_sync(0xffffffffu, x, 0); }

// one thread: a box of a map, and the bytes announced on `bar`
__device__ __forceinline__ void tma_load(void *dst, const CUtensorMap *map, int c, int h, int t, uint64_t *bar) {
    asm volatile(
        "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], "
        "[%5];" ::"r"(tc::smem_u32(dst)),
        "l"(map), "r"(c), "r"(h), "r"(t), "r"(tc::smem_u32(bar))
        : "memory");
}
__device__ __forceinline__ void expect(uint64_t *bar, uint32_t bytes) { tc::mbar_arrive_expect_tx(1u, bar, bytes); }
__device__ __forceinline__ void prefetch_map(const CUtensorMap *map) {
    asm volatile("prefetch.tensormap [%0];" ::"l"(map) : "memory");
}

// store 32 consecutive 32-bit columns of this thread's tensor-memory lane
__device__ __forceinline__ void tmem_st32(uint32_t taddr, const uint32_t (&r)[32]) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,"
        "%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31,%32};" ::"r"(taddr),
        "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]),
        "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]),
        "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]),
        "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31])
        : "memory");
}

// 16 consecutive 32-bit columns of this thread's tensor-memory lane
__device__ __forceinline__ void tmem_ld16(uint32_t taddr, uint32_t (&r)[16]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];\n\t"
        "tcgen05.wait::ld.sync.aligned;"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
          "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
        : "r"(taddr)
        : "memory");
}

__device__ __forceinline__ float exp2_approx(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// absolute error at most 2^-22 for x within (0.5, 2), relative elsewhere: the sum of
// 2^20 keys leaves an lse off by 2^-18 at most, and P of the backward pass by as much
__device__ __forceinline__ float log2_approx(float x) {
    float y;
    asm("lg2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float rcp_approx(float x) {    // relative error at most 2^-23
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// A bounded wait: gives up after the poll limit, or once another role of the
// block has; every role then winds down and the block records SIEVE_ETIMEOUT
// at its end.  (Kept short: it is inlined at every wait, and the kernels'
// instructions do not fit the first-level instruction caches.)
struct Waiter {
    int *abort_flag;   // shared memory
    __device__ __forceinline__ bool operator()(uint64_t *bar, uint32_t parity) const {
        if (tc::mbar_test_wait(bar, parity)) return true;
#pragma unroll 1
        for (uint32_t it = 0; it < kPolls; ++it) {
            if (tc::mbar_try_wait(bar, parity)) return true;
            if ((it & 255u) == 255u && *(volatile int *)abort_flag) break;
        }
        *(volatile int *)abort_flag = 1;
        return false;
    }
    // the same for a whole warp in step
    __device__ __forceinline__ bool warp(uint64_t *bar, uint32_t parity) const {
        return __all_sync(0xffffffffu, (*this)(bar, parity));
    }
};
// One arrival for a warp whose lanes are all done (an arrival of every lane is
// as many serialised operations on the barrier).
__device__ __forceinline__ void warp_arrive(uint64_t *bar) {
    __syncwarp();
    if (lane_id() == 0) tc::mbar_arrive(bar);
}
// the copies or products in flight after an abort
__device__ __forceinline__ void let_land(uint64_t *bar, uint32_t parity) {
#pragma unroll 1
    for (uint32_t it = 0; it < kPolls; ++it)
        if (tc::mbar_try_wait(bar, parity)) return;
}

// Work stealing between the blocks of one grid: a running block asks for the
// index of one that has not started and takes its place (the grid's hardware
// scheduler hands each index out once).  Asked by one thread; the answer
// arrives as 16 bytes in shared memory and completes on `bar`.
__device__ __forceinline__ void steal_block(uint32_t lead, uint4 *answer, uint64_t *bar) {
    tc::mbar_arrive_expect_tx(lead, bar, 16);
    asm volatile(
        "{\n\t.reg .pred q;\n\tsetp.ne.b32 q, %2, 0;\n\t"
        "@q clusterlaunchcontrol.try_cancel.async.shared::cta.mbarrier::complete_tx::bytes.b128 [%0], [%1];\n\t}" ::"r"(
            tc::smem_u32(answer)),
        "r"(tc::smem_u32(bar)), "r"(lead)
        : "memory");
}
// the stolen block's index, or -1 when none was left (then never ask again)
__device__ __forceinline__ int stolen_block(const uint4 *answer) {
    int x;
    asm volatile(
        "{\n\t.reg .b128 r;\n\t.reg .pred p;\n\t.reg .b32 x, y, z, w;\n\tld.shared.b128 r, [%1];\n\t"
        "clusterlaunchcontrol.query_cancel.is_canceled.pred.b128 p, r;\n\tmov.b32 %0, -1;\n\t"
        "@p clusterlaunchcontrol.query_cancel.get_first_ctaid.v4.b32.b128 {x, y, z, w}, r;\n\t"
        "@p mov.b32 %0, x;\n\t}"
        : "=r"(x)
        : "r"(tc::smem_u32(answer))
        : "memory");
    return x;
}

// The blocks of one grid, one after the other: this one's own, then what it
// takes over from blocks that have not started.
struct Blocks {
    uint4 *answer;
    uint64_t *bar;
    uint32_t asked;
    bool asking;
    // ask ahead (the answer is taken by next()): where the block at hand is
    // short, else another may have been free for the next one sooner
    __device__ __forceinline__ void ask() {
        if (elected()) steal_block(1u, answer, bar);
        __syncwarp();
        asking = true;
    }
    // the next block's index in `block`, or -1; false: the wait gave up
    __device__ __forceinline__ bool next(const Waiter &wait, int &block) {
        if (!asking) ask();
        if (!wait.warp(bar, asked & 1u)) return false;
        ++asked;
        asking = false;
        block = stolen_block(answer);
        tc::fence_proxy_async_smem();     // read before the next answer is written
        __syncwarp();
        return true;
    }
};

// two fp32 operations in one instruction
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
    float2 d;
    asm("{\n\t.reg .b64 a, b, d;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\t"
        "mul.rn.f32x2 d, a, b;\n\tmov.b64 {%0, %1}, d;\n\t}"
        : "=f"(d.x), "=f"(d.y)
        : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return d;
}
__device__ __forceinline__ float2 both(float x) { return make_float2(x, x); }
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
    float2 d;
    asm("{\n\t.reg .b64 a, b, c, d;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\tmov.b64 c, {%6, %7};\n\t"
        "fma.rn.f32x2 d, a, b, c;\n\tmov.b64 {%0, %1}, d;\n\t}"
        : "=f"(d.x), "=f"(d.y)
        : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
    return d;
}
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
    float2 d;
    asm("{\n\t.reg .b64 a, b, d;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\t"
        "add.rn.f32x2 d, a, b;\n\tmov.b64 {%0, %1}, d;\n\t}"
        : "=f"(d.x), "=f"(d.y)
        : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return d;
}

// A warp's rows to memory.  A thread holds N chunks (16 bytes) of its own row;
// turned among N neighbouring lanes, lane i of them holds chunk i of each of
// their rows, and one store of the warp writes 32 / N rows' N chunks side by
// side.  (Stored thread by thread, 16 bytes to each of 32 rows, 128 rows of dK
// and dV took 3.8K cycles of a block.)
template <int N>
__device__ __forceinline__ void turn_rows(uint4 (&c)[N]) {
#pragma unroll
    for (int b = 1; b < N; b <<= 1) {
        const bool up = lane_id() & b;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            if (i & b) continue;
            uint32_t *x = reinterpret_cast<uint32_t *>(&c[i]), *y = reinterpret_cast<uint32_t *>(&c[i | b]);
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                const uint32_t got = __shfl_xor_sync(0xffffffffu, up ? x[w] : y[w], b);
                if (up) x[w] = got;
                else y[w] = got;
            }
        }
    }
}
// `out`: the warp's first row, at this thread's first column; `rows` of the 32
// rows exist, `cols` columns from there on.
template <typename T, int N>
__device__ __forceinline__ void store_rows(T *out, int64_t stride, int rows, int cols, uint4 (&c)[N]) {
    turn_rows(c);
    const int at = (int)lane_id() % N, first = (int)lane_id() - at;
    if (8 * at >= cols) return;
#pragma unroll
    for (int i = 0; i < N; ++i)
        if (first + i < rows) *reinterpret_cast<uint4 *>(out + (first + i) * stride + 8 * at) = c[i];
}
template <typename T>
__device__ __forceinline__ uint4 pack8(const float *v) {
    return make_uint4(pack2<T>(v[0], v[1]), pack2<T>(v[2], v[3]), pack2<T>(v[4], v[5]), pack2<T>(v[6], v[7]));
}

struct Doc {
    int q0, nq, k0, nk;   // first rows and lengths
};
// the queries of document s, where its keys are known (most often they are the
// same rows)
__device__ __forceinline__ void queries_of(const sieve_attention_args &a, int s, Doc &d) {
    if (a.new_tokens > 0) {
        d.q0 = s * a.new_tokens;
        d.nq = a.new_tokens;
    } else if (a.q_offsets == a.k_offsets && a.q_tokens == a.k_tokens) {
        d.q0 = d.k0;
        d.nq = d.nk;
    } else {
        doc_range(a.q_offsets, s, (int)a.q_tokens, d.q0, d.nq);
    }
}
// and the other way round
__device__ __forceinline__ void keys_of(const sieve_attention_args &a, int s, Doc &d) {
    if (a.q_offsets == a.k_offsets && a.q_tokens == a.k_tokens) {
        d.k0 = d.q0;
        d.nk = d.nq;
    } else {
        doc_range(a.k_offsets, s, (int)a.k_tokens, d.k0, d.nk);
    }
}
__device__ __forceinline__ Doc doc_at(const sieve_attention_args &a, int s) {
    Doc d;
    doc_range(a.k_offsets, s, (int)a.k_tokens, d.k0, d.nk);
    queries_of(a, s, d);
    return d;
}

// The documents of rising tile numbers, for one warp (see find_doc): it keeps
// where every 32nd of 1,024 documents starts, so that most numbers take one
// dependent load, which brings the document's rows as well.  (A search from
// nothing and the rows after it are five, and a block's finder took 5K to 8K
// cycles for its next work.)
struct DocFinder {
    const int32_t *off;
    int nseq, tokens;
    int base, start;         // start: first number of document base + 32 * lane
    __device__ __forceinline__ DocFinder(const int32_t *offsets, int64_t n, int64_t t)
        : off(offsets), nseq((int)n), tokens((int)t), base(0), start(0x7fffffff) {}
    // number t: its document, the document's first row and length, which of the
    // document's tiles
    __device__ __forceinline__ void operator()(int t, int &doc, int &row, int &len, int &tile) {
        const int lane = lane_id();
        if (t < __shfl_sync(0xffffffffu, start, 0) || t >= __shfl_sync(0xffffffffu, start, 31)) {
            base = find_doc(off, nseq, tokens, kTile, t);
            start = base + 32 * lane < nseq ? first_tile(off, base + 32 * lane, tokens, kTile) : 0x7fffffff;
        }
        // (max(): broken offsets find something in range)
        const int from = base + 32 * max(31 - __clz((int)__ballot_sync(0xffffffffu, start <= t)), 0), d = from + lane;
        const int a = min(max(__ldg(off + min(d, nseq)), 0), tokens);
        const int b = min(max(__ldg(off + min(d + 1, nseq)), 0), tokens);
        const int first = a / kTile + d;
        const int k = max(31 - __clz((int)__ballot_sync(0xffffffffu, d < nseq && first <= t)), 0);
        doc = from + k;
        row = __shfl_sync(0xffffffffu, a, k);
        len = max(__shfl_sync(0xffffffffu, b, k) - row, 0);
        tile = t - __shfl_sync(0xffffffffu, first, k);
    }
};

// Clear the rows [first, end) of a tile of `blocks` column blocks (a warp).
__device__ __forceinline__ void clear_rows(unsigned char *tile, int first, int blocks, int end = kTile) {
#pragma unroll 1
    for (int b = 0; b < blocks; ++b)
#pragma unroll 1
        for (int c = first * 8 + (int)lane_id(); c < end * 8; c += 32)
            *reinterpret_cast<uint4 *>(tile + b * kBlockBytes + c * 16) = make_uint4(0, 0, 0, 0);
    tc::fence_proxy_async_smem();
    __syncwarp();
}

// The bias by distance of one head, times log2(e), for distances
// -reach - kPad .. reach + kPad: 32 rows by 32 columns that hold any distance
// inside (-reach, reach) hold none outside this range, so their lookups need
// no clamp.  Finite values stay finite: the type's lowest must not become
// -inf, which hides a key.  Beyond 2.35e38, where log2(e) leaves the type, they
// count as its lowest or largest.
//
// A thread needs 32 consecutive entries, from a start that falls by one from
// lane to lane.  So the table is kept four times, copy s shifted by s entries:
// whatever its start, a lane reads it from one of them in aligned vectors of
// four: 8 shared-memory instructions for 32 entries.  Copies lie 8 banks apart, and zero distance sits
// at an index of 3 mod 4: then the 8 lanes of a phase, whose tiles start at
// multiples of four, hit 32 different banks.
constexpr int kPad = 64;
__host__ __device__ __forceinline__ int bias_entries(int reach) { return 2 * (reach + kPad) + 1; }
__host__ __device__ __forceinline__ int bias_zero(int reach) { return (reach + kPad + 3) / 4 * 4 + 3; }
__host__ __device__ __forceinline__ int bias_stride(int reach) {   // floats from copy to copy: 8 mod 32
    return (bias_zero(reach) + reach + kPad + 4 + 31) / 32 * 32 + 8;
}
__host__ __device__ __forceinline__ int bias_floats(int reach, int copies = 4) { return copies * bias_stride(reach); }
__device__ __forceinline__ float scaled_bias(const sieve_attention_args &a, int dist, int head) {
    const int b = __ldg(a.bucket_map + a.reach + min(max(dist, -a.reach), a.reach));
    const float v = __ldg(a.table + min(max(b, 0), a.num_buckets - 1) * a.heads + head);
    const float w = v * kLog2e;
    return isinf(w) && !isinf(v) ? copysignf(3.402823466e38f, v) : w;
}

// fill the four copies (threads `tid` of `n`); sign = 1: entry i holds distance
// i - zero, -1: the distance zero - i
template <int kCopies = 4>
__device__ __forceinline__ void fill_bias(float *table, const sieve_attention_args &a, int head, int sign, int tid,
                                          int n) {
    const int stride = bias_stride(a.reach), zero = bias_zero(a.reach);
#pragma unroll 1
    for (int i = tid; i < stride; i += n) {
        const float v = a.table ? scaled_bias(a, sign * (i - zero), head) : 0.f;
#pragma unroll
        for (int s = 0; s < kCopies; ++s)
            if (i >= s) table[s * stride + i - s] = v;
    }
}
// the 32 entries from distance `first` on (in the table's direction)
__device__ __forceinline__ const float4 *bias_at(const float *table, int reach, int first) {
    const int i = bias_zero(reach) + first;
    return reinterpret_cast<const float4 *>(table + (i & 3) * bias_stride(reach) + (i & ~3));
}

// host: a map of [tokens][heads][head_dim], boxes of 64 columns x `box_heads`
// x `box_tokens`
sieve_status make_map(CUtensorMap *map, int dtype, const void *base, int head_dim, int heads, int64_t tokens,
                      int64_t token_stride, int64_t head_stride, int box_heads, int box_tokens);

}  // namespace enc
}  // namespace sieve
