// embed.cu -- token embedding and the gradient of its table.
//
//   forward   out[t] = scale table[id_t]; zeros for an id outside the table
//   backward  dtable[v] = scale * sum of dout[t] over the tokens with id_t = v
//
// Both are bound by memory.  The backward pass sorts the tokens by id (stable,
// so the sums have a fixed order), then walks the sorted list in pieces of
// kPiece tokens: a warp adds up the rows of one piece in registers and writes
// every id that lies wholly inside it.  An id that goes on into other pieces
// (a frequent word, the mask token) leaves one partial row a piece, which
// k_embed_join adds up in order.  So the sums' work is even whatever the ids are; what
// grows with a frequent id is its join, one row of every 64 tokens by a block for each 256
// columns.  Rows that no token has are found by the blocks that write their zeros
// (262,144 tokens of 64 columns, 64,000 ids: 104 us, with half of the tokens one id as
// well; 126 and 166 where such a block read all keys of its ids).
//
// Measured (device time).  Forward: 200,003 tokens of 1,024 columns from a table of 64,000
// in fp32 to bf16 99 us (587 MB of DRAM traffic, 5.9 TB/s).  Backward: 131,000 tokens of 768
// columns, bf16, 64,000 ids, one in eight the same: the sort 24 us (four launches), the
// sums 65 (398 MB, 6.1 TB/s), the join 19.
#include <type_traits>

#include "attention.cuh"
#include "blocks.cuh"

namespace sieve {
namespace enc {
namespace {

constexpr int kThreads = 256;

// VEC consecutive elements as loaded, 16 bytes at a time
template <typename T, int VEC>
struct Chunk {
    static constexpr int kWords = VEC * sizeof(T) >= 16 ? VEC * sizeof(T) / 16 : 1;
    static_assert(VEC == 1 || VEC * sizeof(T) % 16 == 0, "");
    uint4 w[kWords];
    __device__ __forceinline__ void load(const T *p) {
        if constexpr (VEC == 1) {
            if constexpr (sizeof(T) == 4) w[0].x = __ldg(reinterpret_cast<const unsigned int *>(p));
            else w[0].x = __ldg(reinterpret_cast<const unsigned short *>(p));
        } else {
#pragma unroll
            for (int i = 0; i < kWords; ++i) w[i] = __ldg(reinterpret_cast<const uint4 *>(p) + i);
        }
    }
    // values e and e + 1
    __device__ __forceinline__ float2 two(int e) const {
        static_assert(VEC > 1, "");
        const uint4 &q = w[e * sizeof(T) / 16];
        if constexpr (sizeof(T) == 4) return e % 4 ? make_float2(__uint_as_float(q.z), __uint_as_float(q.w)) : make_float2(__uint_as_float(q.x), __uint_as_float(q.y));
        else return unpack2<T>(e % 8 == 0 ? q.x : e % 8 == 2 ? q.y : e % 8 == 4 ? q.z : q.w);
    }
    __device__ __forceinline__ float one() const {
        if constexpr (sizeof(T) == 4) return __uint_as_float(w[0].x);
        else return to_f32<T>(__builtin_bit_cast(T, (unsigned short)w[0].x));
    }
};
template <typename T, int VEC>
__device__ __forceinline__ void put(T *p, const float (&v)[VEC]) {
    if constexpr (VEC == 1) {
        *p = from_f32<T>(v[0]);
    } else if constexpr (sizeof(T) == 2) {
        static_assert(VEC == 8, "");
        *reinterpret_cast<uint4 *>(p) = make_uint4(pack2<T>(v[0], v[1]), pack2<T>(v[2], v[3]), pack2<T>(v[4], v[5]), pack2<T>(v[6], v[7]));
    } else {
#pragma unroll
        for (int i = 0; i < VEC; i += 4) reinterpret_cast<float4 *>(p)[i / 4] = make_float4(v[i], v[i + 1], v[i + 2], v[i + 3]);
    }
}

// A block takes `tokens_per_block` tokens and its threads chunk after chunk of
// theirs, one at a time: many warps hide the two loads that depend on each other
// better than few with more of them in hand (200,003 tokens of 1024 columns, fp32 to
// bf16: 98 us, 125 with four chunks ahead, 169 with eight).
template <typename T, typename O, int VEC>
__global__ void __launch_bounds__(kThreads) k_embed(const EmbedArgs a, int tokens_per_block, int chunks) {
    const int64_t first = (int64_t)blockIdx.x * tokens_per_block;
    const int total = (int)min((int64_t)tokens_per_block, a.tokens - first) * chunks;
    const T *table = static_cast<const T *>(a.table);
    O *out = static_cast<O *>(a.out);
#pragma unroll 1
    for (int l = threadIdx.x; l < total; l += kThreads) {
        const int token = l / chunks, col = (l - token * chunks) * VEC;
        const int id = id_at(a.ids, a.id_type, first + token, a.vocab);
        float v[VEC] = {};
        if (id >= 0) {
            Chunk<T, VEC> x;
            x.load(table + id * a.table_stride + col);
            if constexpr (VEC == 1) {
                v[0] = a.scale * x.one();
            } else {
#pragma unroll
                for (int e = 0; e < VEC; e += 2) {
                    const float2 t = x.two(e);
                    v[e] = a.scale * t.x;
                    v[e + 1] = a.scale * t.y;
                }
            }
        }
        put<O, VEC>(out + (first + token) * a.out_stride + col, v);
    }
}

// Rows of single elements: a warp to a token, so that no element needs a division to
// find its place.
template <typename T, typename O>
__global__ void __launch_bounds__(kThreads) k_embed_odd(const EmbedArgs a) {
    const int lane = lane_id();
    const int64_t token = (int64_t)blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5);
    if (token >= a.tokens) return;
    const int id = id_at(a.ids, a.id_type, token, a.vocab);
    const T *row = static_cast<const T *>(a.table) + (id < 0 ? 0 : id) * a.table_stride;
    O *out = static_cast<O *>(a.out) + token * a.out_stride;
#pragma unroll 8
    for (int col = lane; col < a.width; col += 32) out[col] = from_f32<O>(id < 0 ? 0.f : a.scale * to_f32<T>(__ldg(row + col)));
}

// ---------------------------------------------------------------------------
// The sort: passes over digits of up to 9 bits, the lowest first.  The list is
// cut into `tiles` pieces of `per` tokens; k_sort_count counts every tile's
// digits, and k_sort_scatter finds from all counts where each of its digits
// starts and places its tokens in order.
constexpr int kSortThreads = 512;
constexpr int kSortItems = 4;
constexpr int kSortStep = kSortThreads * kSortItems;
constexpr int kSortWarps = kSortThreads / 32;
constexpr int kMaxDigits = 512;
constexpr int kMaxSortTiles = 304;     // two for each SM

struct Sort {
    int tokens, per, tiles, vocab;
    int shift, bits;                   // this pass' digit
    const int32_t *key_in, *val_in;    // nullptr in the first pass: the ids themselves
    int32_t *key_out, *val_out;
    int32_t *count;                    // [tiles][1 << bits]
    int32_t *joins;                    // number of ids to join, zeroed by the first pass
    const void *ids;
    int id_type;
};

// The token's key: its id, or vocab where it has none.
__device__ __forceinline__ int sort_key(const Sort &s, int i) {
    if (s.key_in) return s.key_in[i];
    const int id = id_at(s.ids, s.id_type, i, s.vocab);
    return id < 0 ? s.vocab : id;
}

__global__ void __launch_bounds__(kSortThreads) k_sort_count(const Sort s) {
    __shared__ int bins[kMaxDigits];
    const int n = 1 << s.bits;
    if (blockIdx.x == 0 && threadIdx.x == 0 && !s.key_in) *s.joins = 0;
    for (int i = threadIdx.x; i < n; i += kSortThreads) bins[i] = 0;
    __syncthreads();
    const int first = blockIdx.x * s.per, last = min(first + s.per, s.tokens);
#pragma unroll 4
    for (int i = first + threadIdx.x; i < last; i += kSortThreads)
        atomicAdd(&bins[(sort_key(s, i) >> s.shift) & (n - 1)], 1);
    __syncthreads();
    for (int i = threadIdx.x; i < n; i += kSortThreads) s.count[blockIdx.x * n + i] = bins[i];
}

__global__ void __launch_bounds__(kSortThreads) k_sort_scatter(const Sort s) {
    __shared__ int start[kMaxDigits];              // where the tile's next token of a digit goes
    __shared__ int of_warp[kSortWarps][kMaxDigits];
    __shared__ int sums[kSortWarps];
    const int n = 1 << s.bits, tid = threadIdx.x, lane = lane_id(), warp = tid >> 5;
    // digit tid: tokens of it in all tiles, and in the tiles before this one
    int all = 0, before = 0;
    if (tid < n) {
#pragma unroll 16
        for (int t = 0; t < s.tiles; ++t) {
            const int c = s.count[t * n + tid];
            all += c;
            before += t < (int)blockIdx.x ? c : 0;
        }
    }
    int scan = all;                                // exclusive sum over the digits
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int up = __shfl_up_sync(0xffffffffu, scan, o);
        if (lane >= o) scan += up;
    }
    if (lane == 31) sums[warp] = scan;
    __syncthreads();
    int base = scan - all + before;
    for (int w = 0; w < warp; ++w) base += sums[w];
    if (tid < n) start[tid] = base;
    const int first = blockIdx.x * s.per, last = min(first + s.per, s.tokens);
    for (int at = first; at < last; at += kSortStep) {
        for (int i = lane; i < n; i += 32) of_warp[warp][i] = 0;
        __syncwarp();
        int key[kSortItems], val[kSortItems], rank[kSortItems];
        const int mine = at + warp * 32 * kSortItems + lane;
#pragma unroll
        for (int k = 0; k < kSortItems; ++k) {
            const int i = mine + k * 32;
            key[k] = i < last ? sort_key(s, i) : -1;
            val[k] = i < last && s.key_in ? s.val_in[i] : i;
        }
        // the warp's tokens in order: how many of the same digit came before
#pragma unroll
        for (int k = 0; k < kSortItems; ++k) {
            const bool live = mine + k * 32 < last;
            const int d = live ? (key[k] >> s.shift) & (n - 1) : n;
            const unsigned same = __match_any_sync(0xffffffffu, d);
            if (live) rank[k] = of_warp[warp][d] + __popc(same & ((1u << lane) - 1));
            __syncwarp();
            if (live && lane == 31 - __clz((int)same)) of_warp[warp][d] += __popc(same);
            __syncwarp();
        }
        __syncthreads();
        // each warp's first place of a digit
        if (tid < n) {
            int p = start[tid];
#pragma unroll
            for (int w = 0; w < kSortWarps; ++w) {
                const int c = of_warp[w][tid];
                of_warp[w][tid] = p;
                p += c;
            }
            start[tid] = p;
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < kSortItems; ++k)
            if (mine + k * 32 < last) {
                const int to = of_warp[warp][(key[k] >> s.shift) & (n - 1)] + rank[k];
                s.key_out[to] = key[k];
                s.val_out[to] = val[k];
            }
        __syncthreads();
    }
}

// ---------------------------------------------------------------------------
constexpr int kPiece = 64;              // sorted tokens of a warp
constexpr int kPieceWarps = 4;
constexpr int kColumns = 256;           // columns of a warp, times NC: 8 a lane each
constexpr int kResidentWarps = 152 * 24;   // that the SMs hold at once
constexpr int kZeroRows = 32;           // table rows of a block that looks for empty ones
constexpr int kFewKeys = 4 * kPieceWarps * 32;   // of their tokens

struct Sums {
    EmbedArgs a;
    const int32_t *key, *val;           // sorted
    float *partial;                     // [pieces][2][width]: of an id that came from the piece before, of one that goes on
    int32_t *joins, *join_list;         // pieces where an id starts that goes on
    int pieces, slices, sum_blocks;
};

// Places of a lane's 8 NC columns in a slice: VEC together.
template <int VEC>
__device__ __forceinline__ int column(int lane, int e) {
    return (e / VEC * 32 + lane) * VEC + e % VEC;
}
template <typename T, int VEC, int NC>
struct Row {                            // a lane's columns of a row
    Chunk<T, VEC> c[8 * NC / VEC];
    __device__ __forceinline__ void load(const T *p, int lane, int left) {
#pragma unroll
        for (int i = 0; i < 8 * NC / VEC; ++i)
            if (column<VEC>(lane, i * VEC) < left) c[i].load(p + column<VEC>(lane, i * VEC));
    }
    // added to sums, where there are columns
    __device__ __forceinline__ void add_to(float (&sum)[8 * NC], int lane, int left) const {
#pragma unroll
        for (int i = 0; i < 8 * NC / VEC; ++i) {
            if (column<VEC>(lane, i * VEC) >= left) continue;
            if constexpr (VEC == 1) {
                sum[i] += c[i].one();
            } else {
#pragma unroll
                for (int e = 0; e < VEC; e += 2) {
                    const float2 s = add2(make_float2(sum[i * VEC + e], sum[i * VEC + e + 1]), c[i].two(e));
                    sum[i * VEC + e] = s.x;
                    sum[i * VEC + e + 1] = s.y;
                }
            }
        }
    }
};
// the finished sums of a table row
template <typename G, int VEC, int NC>
__device__ __forceinline__ void finish(const EmbedArgs &a, int id, int col0, int lane, const float (&sum)[8 * NC]) {
    G *to = static_cast<G *>(a.dtable) + id * a.dtable_stride + col0;
    const int left = a.width - col0;
#pragma unroll
    for (int i = 0; i < 8 * NC / VEC; ++i) {
        const int col = column<VEC>(lane, i * VEC);
        if (col >= left) continue;
        float v[VEC];
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
            v[e] = a.scale * sum[i * VEC + e];
            if (a.accumulate) v[e] += to_f32<G>(to[col + e]);
        }
        put<G, VEC>(to + col, v);
    }
}

// first place in the sorted keys whose key is at least v (a whole warp)
__device__ __forceinline__ int lower_bound(const int32_t *key, int n, int v) {
    int lo = 0, hi = n;                 // the answer is in [lo, hi]
    while (hi > lo) {
        const int step = (hi - lo + 31) / 32;
        const int i = lo + ((int)lane_id() + 1) * step - 1;
        // lanes whose stretch of `step` keys lies wholly below v
        const int below = __popc(__ballot_sync(0xffffffffu, i < hi && key[min(i, n - 1)] < v));
        const int from = lo + below * step;
        hi = min(hi, from + step - 1);
        lo = min(from, hi);
        if (step == 1) break;
    }
    return lo;
}

template <typename T, typename G, int VEC, int NC>
__global__ void __launch_bounds__(kPieceWarps * 32) k_embed_sums(const Sums s) {
    const EmbedArgs &a = s.a;
    const int lane = lane_id(), warp = threadIdx.x >> 5;
    if ((int)blockIdx.x >= s.sum_blocks) {
        // ---- the zeros of rows that no token has
        __shared__ int range[2];
        __shared__ int has[kZeroRows];
        const int v0 = ((int)blockIdx.x - s.sum_blocks) * kZeroRows, v1 = min(v0 + kZeroRows, a.vocab);
        if (threadIdx.x < kZeroRows) has[threadIdx.x] = 0;
        if (warp < 2) {
            const int p = lower_bound(s.key, a.tokens, warp ? v1 : v0);
            if (lane == 0) range[warp] = p;
        }
        __syncthreads();
        // Few keys of these ids are looked through.  More (a frequent word, the mask) would keep
        // this block on them for as long as they are many: every id is searched for.
        if (range[1] - range[0] <= kFewKeys) {
#pragma unroll 4
            for (int i = range[0] + threadIdx.x; i < range[1]; i += kPieceWarps * 32) has[s.key[i] - v0] = 1;
        } else if (threadIdx.x < kZeroRows) {
            int lo = range[0], hi = range[1];
            const int v = v0 + (int)threadIdx.x;
            while (lo < hi) {
                const int mid = lo + (hi - lo) / 2;
                if (s.key[mid] < v) lo = mid + 1;
                else hi = mid;
            }
            has[threadIdx.x] = lo < range[1] && s.key[lo] == v;
        }
        __syncthreads();
        float zero[VEC] = {};
        for (int v = v0 + warp; v < v1; v += kPieceWarps)
            if (!has[v - v0])
                for (int col = lane * VEC; col < a.width; col += 32 * VEC)
                    put<G, VEC>(static_cast<G *>(a.dtable) + v * a.dtable_stride + col, zero);
        return;
    }
    const int64_t work = (int64_t)blockIdx.x * kPieceWarps + warp;
    const int across = (s.slices + NC - 1) / NC;
    const int piece = (int)(work / across), col0 = (int)(work % across) * kColumns * NC;
    if (piece >= s.pieces) return;
    const int p0 = piece * kPiece, count = min(kPiece, a.tokens - p0), left = a.width - col0;
    int keys[2], vals[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int i = min(p0 + h * 32 + lane, a.tokens - 1);
        keys[h] = s.key[i];
        vals[h] = s.val[i];
    }
    const int prev = p0 > 0 ? s.key[p0 - 1] : -1, next = p0 + count < a.tokens ? s.key[p0 + count] : a.vocab;
    const T *dout = static_cast<const T *>(a.dout) + col0;
    constexpr int kAhead = NC == 1 ? 8 : 4;
    float sum[8 * NC] = {};
    int cur = __shfl_sync(0xffffffffu, keys[0], 0);
    // a whole id is written at once; what reaches into other pieces is kept
    auto flush = [&](int key, bool from_before, bool goes_on) {
        if (key >= a.vocab) return;
        if (!from_before && !goes_on) {
            finish<G, VEC, NC>(a, key, col0, lane, sum);
            return;
        }
        float *to = s.partial + ((int64_t)piece * 2 + (from_before ? 0 : 1)) * a.width + col0;
#pragma unroll
        for (int e = 0; e < 8 * NC; ++e)
            if (column<VEC>(lane, e) < left) to[column<VEC>(lane, e)] = sum[e];
        if (!from_before && col0 == 0 && lane == 0) s.join_list[atomicAdd(s.joins, 1)] = piece;
    };
    bool whole = true;                  // no id has ended in this piece yet
    for (int j0 = 0; j0 < count; j0 += kAhead) {
        Row<T, VEC, NC> x[kAhead];
        int key[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const int j = j0 + u;
            key[u] = __shfl_sync(0xffffffffu, j < 32 ? keys[0] : keys[1], j & 31);
            const int t = __shfl_sync(0xffffffffu, j < 32 ? vals[0] : vals[1], j & 31);
            if (j >= count) key[u] = -1;
            else if (key[u] < a.vocab) x[u].load(dout + t * a.dout_stride, lane, left);
        }
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            if (key[u] < 0) break;
            if (key[u] != cur) {
                flush(cur, whole && cur == prev, false);
                whole = false;
                cur = key[u];
#pragma unroll
                for (int e = 0; e < 8 * NC; ++e) sum[e] = 0.f;
            }
            if (cur < a.vocab) x[u].add_to(sum, lane, left);
        }
    }
    flush(cur, whole && cur == prev, cur == next);
}

// The ids that several pieces share: the partial row of the piece where the id
// starts, then of those that it goes on into.  Up to kShort of these are added by
// a warp for every kColumns columns; more (a very frequent id) by all strands of
// a block, each a stretch of the pieces in order, then the strands in order.
constexpr int kStrands = 16;
constexpr int kJoinThreads = kStrands * 32;
constexpr int kJoinBlocks = 152 * 4;
constexpr int kShort = 8;
template <typename G>
__global__ void __launch_bounds__(kJoinThreads) k_embed_join(const Sums s) {
    __shared__ float part[kStrands][kColumns];
    __shared__ int shared_end, found[kStrands], long_piece[kJoinThreads];
    const EmbedArgs &a = s.a;
    const int lane = lane_id(), warp = threadIdx.x >> 5;
    const int joins = *s.joins;
    auto write = [&](int id, int col, float v) {
        G *to = static_cast<G *>(a.dtable) + id * a.dtable_stride + col;
        v *= a.scale;
        if (a.accumulate) v += to_f32<G>(*to);
        *to = from_f32<G>(v);
    };
    // whether the id at the end of `piece` goes on into piece + n
    auto reaches = [&](int piece, int id, int n) {
        const int64_t p = (int64_t)(piece + n) * kPiece;
        return p < a.tokens && s.key[p] == id;
    };
    // the short ones: a warp for each and kColumns columns
    for (int64_t w = (int64_t)blockIdx.x * kStrands + warp; w < (int64_t)joins * s.slices; w += (int64_t)gridDim.x * kStrands) {
        const int piece = s.join_list[w / s.slices], col0 = (int)(w % s.slices) * kColumns, left = a.width - col0;
        const int id = s.key[piece * kPiece + kPiece - 1];
        const int n = __popc(__ballot_sync(0xffffffffu, lane <= kShort && reaches(piece, id, 1 + lane)));
        if (n > kShort) continue;
        const float *x = s.partial + (int64_t)piece * 2 * a.width + col0;
        float sum[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) sum[e] = x[a.width + min(e * 32 + lane, left - 1)];
#pragma unroll 4
        for (int p = 1; p <= n; ++p)
#pragma unroll
            for (int e = 0; e < 8; ++e) sum[e] += x[(int64_t)p * 2 * a.width + min(e * 32 + lane, left - 1)];
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (e * 32 + lane < left) write(id, col0 + e * 32 + lane, sum[e]);
    }
    // the long ones, by their number in the list: every block finds all of them and takes its share
    int64_t before = 0;
    for (int j0 = 0; j0 < joins; j0 += kJoinThreads) {
        const int j = j0 + (int)threadIdx.x, piece = j < joins ? s.join_list[j] : -1;
        const bool is_long = piece >= 0 && reaches(piece, s.key[piece * kPiece + kPiece - 1], 1 + kShort);
        const unsigned votes = __ballot_sync(0xffffffffu, is_long);
        __syncthreads();
        if (lane == 0) found[warp] = __popc(votes);
        __syncthreads();
        int rank = __popc(votes & ((1u << lane) - 1)), count = 0;
#pragma unroll
        for (int w = 0; w < kStrands; ++w) {
            rank += w < warp ? found[w] : 0;
            count += found[w];
        }
        if (is_long) long_piece[rank] = piece;
        __syncthreads();
        const int64_t first = before * s.slices, last = (before + count) * s.slices;
        before += count;
        for (int64_t w = first + (blockIdx.x + gridDim.x - first % gridDim.x) % gridDim.x; w < last; w += gridDim.x) {
            const int start = long_piece[(w - first) / s.slices], col0 = (int)((w - first) % s.slices) * kColumns;
            const int id = s.key[start * kPiece + kPiece - 1], left = a.width - col0;
            __syncthreads();
            if (warp == 0) {
                const int end = lower_bound(s.key, a.tokens, id + 1);   // past the id's last token
                if (lane == 0) shared_end = end;
            }
            __syncthreads();
            const int n = (shared_end - 1) / kPiece - start;
            const int each = (n + kStrands - 1) / kStrands;
            const int from = start + 1 + warp * each, to = min(from + each, start + 1 + n);
            float sum[8] = {};
            // (eight pieces' loads go out together: places past the row read its last element)
            for (int p = from; p < to; p += 8) {
                float v[8][8];
#pragma unroll
                for (int k = 0; k < 8; ++k)
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        v[k][e] = s.partial[(int64_t)min(p + k, to - 1) * 2 * a.width + col0 + min(e * 32 + lane, left - 1)];
#pragma unroll
                for (int k = 0; k < 8; ++k)
#pragma unroll
                    for (int e = 0; e < 8; ++e) sum[e] += p + k < to ? v[k][e] : 0.f;
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) part[warp][e * 32 + lane] = sum[e];
            __syncthreads();
            const int col = threadIdx.x;
            if (col < kColumns && col < left) {
                float v = s.partial[((int64_t)start * 2 + 1) * a.width + col0 + col];
#pragma unroll
                for (int k = 0; k < kStrands; ++k) v += part[k][col];
                write(id, col0 + col, v);
            }
        }
        __syncthreads();
    }
}

bool aligned(const void *p, size_t m) { return reinterpret_cast<uintptr_t>(p) % m == 0; }
// whether rows can be moved VEC elements (16 bytes or more) at a time
bool wide_rows(const void *p, int64_t stride, int width, int vec, size_t size) {
    return width % vec == 0 && stride * size % 16 == 0 && aligned(p, 16);
}

int key_bits(int64_t vocab) {            // of the numbers 0 .. vocab
    int b = 1;
    while (((int64_t)1 << b) <= vocab) ++b;
    return b;
}
struct SortShape {
    int passes, bits, per, tiles;
};
SortShape sort_shape(int64_t tokens, int64_t vocab) {
    SortShape s;
    const int all = key_bits(vocab);
    s.passes = (all + 8) / 9;
    s.bits = (all + s.passes - 1) / s.passes;
    const int64_t most = ceil_div(tokens, kMaxSortTiles);
    s.per = (int)round_up(most < 1 ? 1 : most, kSortStep);
    s.tiles = (int)ceil_div(tokens, s.per);
    return s;
}
// [tokens] keys and places twice, counts, [pieces] joins, their number, partial rows
struct Layout {
    size_t key[2], val[2], count, list, joins, partial, bytes;
};
Layout layout(int64_t tokens, int64_t vocab, int width) {
    const SortShape s = sort_shape(tokens, vocab);
    const int64_t pieces = ceil_div(tokens, kPiece);
    Layout l;
    size_t at = 0;
    auto take = [&](int64_t bytes) {
        const size_t here = at;
        at += (size_t)round_up(bytes, 256);
        return here;
    };
    for (int i = 0; i < 2; ++i) {
        l.key[i] = take(tokens * 4);
        l.val[i] = take(tokens * 4);
    }
    l.count = take((int64_t)s.tiles * (1 << s.bits) * 4);
    l.list = take(pieces * 4);
    l.joins = take(4);
    l.partial = take(pieces * 2 * width * 4);
    l.bytes = at;
    return l;
}

}  // namespace

cudaError_t launch_embed(const EmbedArgs &a, cudaStream_t st) {
    return with_type(a.table_dtype, [&](auto t) {
        using T = typename decltype(t)::type;
        return with_type(a.dtype, [&](auto o) {
            using O = typename decltype(o)::type;
            constexpr int V = sizeof(T) == 4 && sizeof(O) == 4 ? 4 : 8;
            const bool wide = wide_rows(a.table, a.table_stride, a.width, V, sizeof(T)) &&
                              wide_rows(a.out, a.out_stride, a.width, V, sizeof(O));
            const int chunks = wide ? a.width / V : a.width;
            const int per = chunks >= 1024 ? 1 : 1024 / chunks;
            const unsigned blocks = (unsigned)ceil_div(a.tokens, per);
            if (wide) k_embed<T, O, V><<<blocks, kThreads, 0, st>>>(a, per, chunks);
            else if (chunks < 32) k_embed<T, O, 1><<<blocks, kThreads, 0, st>>>(a, per, chunks);
            else k_embed_odd<T, O><<<(unsigned)ceil_div(a.tokens, kThreads / 32), kThreads, 0, st>>>(a);
            return cudaGetLastError();
        });
    });
}

cudaError_t launch_embed_backward(const EmbedArgs &a, void *ws, cudaStream_t st) {
    unsigned char *base = static_cast<unsigned char *>(ws);
    const Layout l = layout(a.tokens, a.vocab, a.width);
    const SortShape shape = sort_shape(a.tokens, a.vocab);
    auto ints = [&](size_t at) { return reinterpret_cast<int32_t *>(base + at); };
    Sort s = {};
    s.tokens = a.tokens;
    s.per = shape.per;
    s.tiles = shape.tiles;
    s.vocab = a.vocab;
    s.bits = shape.bits;
    s.count = ints(l.count);
    s.joins = ints(l.joins);
    s.ids = a.ids;
    s.id_type = a.id_type;
    for (int pass = 0; pass < shape.passes && a.tokens > 0; ++pass) {
        s.shift = pass * shape.bits;
        s.key_in = pass ? ints(l.key[(pass + 1) & 1]) : nullptr;
        s.val_in = pass ? ints(l.val[(pass + 1) & 1]) : nullptr;
        s.key_out = ints(l.key[pass & 1]);
        s.val_out = ints(l.val[pass & 1]);
        k_sort_count<<<s.tiles, kSortThreads, 0, st>>>(s);
        k_sort_scatter<<<s.tiles, kSortThreads, 0, st>>>(s);
        const cudaError_t e = cudaGetLastError();
        if (e != cudaSuccess) return e;
    }
    Sums u = {};
    u.a = a;
    u.key = ints(l.key[(shape.passes - 1) & 1]);
    u.val = ints(l.val[(shape.passes - 1) & 1]);
    u.partial = reinterpret_cast<float *>(base + l.partial);
    u.joins = s.joins;
    u.join_list = ints(l.list);
    u.pieces = (int)ceil_div(a.tokens, kPiece);
    u.slices = (int)ceil_div(a.width, kColumns);
    const int64_t zero_blocks = a.accumulate ? 0 : ceil_div(a.vocab, kZeroRows);
    return with_type(a.dtype, [&](auto t) {
        using T = typename decltype(t)::type;
        return with_type(a.table_dtype, [&](auto g) {
            using G = typename decltype(g)::type;
            constexpr int V = sizeof(T) == 4 && sizeof(G) == 4 ? 4 : 8;
            auto launch = [&](auto vec, auto nc) {
                constexpr int VEC = decltype(vec)::value, NC = decltype(nc)::value;
                u.sum_blocks = (int)ceil_div((int64_t)u.pieces * ceil_div(u.slices, NC), kPieceWarps);
                const unsigned blocks = (unsigned)(u.sum_blocks + zero_blocks);
                if (blocks) k_embed_sums<T, G, VEC, NC><<<blocks, kPieceWarps * 32, 0, st>>>(u);
            };
            using One = std::integral_constant<int, 1>;
            // 768 or 512 columns a warp instead of 256 where there are more warps than the SMs hold
            // at once: less work beside the sums for every token.  This kernel with 1, 2 and 3 times
            // 256, bf16, 64,000 ids: 131,000 tokens of 512 columns 52, 47 and 47 us, of 768 69, 78 and
            // 66; 60,000 of 1,024 71, 66 and 65, of 1,536 102, 100 and 96; below that number
            // 30,000 of 768 46, 52 and 57, 30,000 of 1,024 57, 61 and 63.  Odd rows move element by element.
            if (!wide_rows(a.dout, a.dout_stride, a.width, V, sizeof(T)) ||
                !wide_rows(a.dtable, a.dtable_stride, a.width, V, sizeof(G)))
                launch(One{}, One{});
            else if (u.slices == 1 || (int64_t)u.pieces * u.slices < kResidentWarps)
                launch(std::integral_constant<int, V>{}, One{});
            else if (u.slices % 3 == 0)
                launch(std::integral_constant<int, V>{}, std::integral_constant<int, 3>{});
            else
                launch(std::integral_constant<int, V>{}, std::integral_constant<int, 2>{});
            const cudaError_t e = cudaGetLastError();
            if (e != cudaSuccess || a.tokens <= kPiece) return e;
            k_embed_join<G><<<kJoinBlocks, kJoinThreads, 0, st>>>(u);
            return cudaGetLastError();
        });
    });
}

size_t embed_backward_workspace_bytes(int64_t tokens, int64_t vocab, int width) {
    return layout(tokens, vocab, width).bytes;
}

}  // namespace enc
}  // namespace sieve
