// Attention of a decode step: one query token a request over its pages, 16-bit or 4-bit, with an optional sliding window
// and sinks.  (The paper stops at the first token; this reads the pages that a composed prompt leaves behind.)
//   out = sum over visible keys of p v / l,  p = exp2(scale log2(e) q.k - m),  l = sum p,
// one pass over K and V with a running reference m; scores, l and the accumulators in fp32, p rounded to bf16 as an operand.
//
// Bound by memory: a key and value of a head are 512 bytes at head_dim 128 (4-bit: 144) for 4 D g flops.  The g <= 16 query heads
// of a KV head are the narrow side of mma.sync m16n8k16: keys are the 16 rows, queries the 8 (or twice 8) columns, so a
// score tile is S^T = K Q^T and the output O^T += V^T P^T.  (tcgen05 wants 128 rows of queries; there are at most 16.)
//
// Work: the visible keys of every (request, KV head), a pair, are cut into tiles of 16, in 4 bits of 32; the tiles of the whole batch, in order, are
// shared out evenly to the warps of one thread block an SM, whatever the lengths.  Which they are only the device knows (lengths
// are device data, so that a captured step can be replayed as they grow): every block sums the requests' tiles itself.  A warp
// goes through its stretch, pair after pair, by itself: it fills a ring of stages with cp.async, the next pair's tiles already on
// their way while it ends one, and writes the results of pairs that lie inside its stretch.  What it has of a pair that begins
// before or goes on behind its stretch is a part; at the end the block joins its warps' parts, and parts of pairs that
// leave the block go to the workspace, where the last block to arrive joins them, always in the order of the tiles.
// (Blocks that took pairs in turn, all their warps on one, and met at the end of each: 215 us where 64 requests of 200 to
// 16 384 tokens, 8 heads in 4 bits, then took 130 us, now 109 to 124 (boxes); a join in a kernel of its own: 4 us more for any batch.)
// A row that is not visible, past the end or on a page outside the pool is filled with zeros and never read, so what stands
// there does not matter.
#include <cmath>
#include <cstring>
#include <string>
#include <type_traits>

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include "decode.h"
#include "device_mem.cuh"
#include "launch.h"
#include "pair_chunk.cuh"
#include "plan.h"
#include "sm100_ptx.cuh"

namespace tessera {

int32_t api_set_error(int32_t code, const std::string &msg);

namespace {

constexpr float kValueUnit = 18446744073709551616.f;                 // 2^64: products of subnormal codes with scales near 1 come out near 2^-69
constexpr float kValueTop = 5192296858534827628530496329220096.f;    // 2^112: p (at most 2^8) times this is a bf16 number
constexpr int kMaxGroup = 16;

struct Args {
    const uint8_t *k, *v;
    const __nv_bfloat16 *q;
    __nv_bfloat16 *out;
    float *lse;
    const int32_t *table, *seq_len;
    int batch, max_pages, num_pool_pages, page_size, H_q, H_kv, g, window, n_sink;
    float scale_log2;
    uint32_t *ws_count;   // [grid] arrivals of the pair that begins in the block and goes on; 0 between calls
    float *ws_o;          // [2 grid][16][D] parts: block b's of a pair that began before it at 2 b, of one that goes on behind it at 2 b + 1
    float2 *ws_ml;        // [2 grid][16] reference (log2 units) and sum
};

// Shared memory: every warp's ring (a stage: the rows of a tile of K, of V and, 4-bit, their numbers) and its part of the pair that
// its stretch begins in; the part of the one it ends in goes into the ring.
template <int D, bool F4, int NQ> struct Geo {
    // (4-bit, 64 requests of up to 16 384 tokens, 8 heads: 12 warps of 168 registers 113 us, with a third stage 112 but a lone request
    // 12.0 -> 12.5; 16 of 128 115, 14 127; later, with the joins in less code, 12 warps 109 on that box, up to 124 on others.
    // Not folded: 5 queries a KV head 134, 8 137, 16, in 8 warps of 254 registers, 202; head_dim 64, half the bytes: 4 queries 83, 8 95, 16 154.  Two fifths of the instructions spread codes over operands; their pipe is busy 56 % of the time.)
    static constexpr int kWarps = F4 && NQ == 1 ? 12 : 8;
    static constexpr int kThreads = 32 * kWarps;
    static constexpr int kTile = F4 ? 32 : 16;                            // keys
    static constexpr int kRow = F4 ? D / 2 : 2 * D;                       // bytes of a row of K or V
    static constexpr int kStageBytes = 2 * kTile * (kRow + (F4 ? 8 : 0));
    static constexpr int kFew = F4 ? 24 : 30;                             // tiles that a block may have more for whole pairs (see stretch_of)
    static constexpr int kPart = 8 * NQ * (D + 4);                        // floats; rows 4 apart in banks: the lanes of a store spread over all
    static constexpr int kStages = F4 ? (NQ == 1 ? 2 : 4) * (128 / D) : (NQ == 1 ? 3 : 2) * (128 / D);
    static constexpr int kRing = kWarps * kStages * kStageBytes;
    static constexpr int kBytes = kRing + kWarps * kPart * 4;
    static_assert(kTile % kDecodeUnit == 0, "");
    static_assert(kStages * kStageBytes >= kPart * 4, "a part goes into a warp's ring");
};

__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float lg2(float x) {                      // 2^-22 off between 1/2 and 2, elsewhere an ulp or so
    float y;
    asm("lg2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float about_one_over(float x) {           // 1 ulp
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
// N bytes to shared memory; zeros in place of what is not there.
template <int N> __device__ __forceinline__ void cp_async(uint32_t dst, const void *src, bool there) {
    if constexpr (N == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(there ? 16 : 0) : "memory");
    else asm volatile("cp.async.ca.shared.global [%0], [%1], 8, %2;" ::"r"(dst), "l"(src), "r"(there ? 8 : 0) : "memory");
}
template <int N> __device__ __forceinline__ void cp_async(uint32_t dst, const void *src) {
    if constexpr (N == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
    else asm volatile("cp.async.ca.shared.global [%0], [%1], 8;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void cp_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void cp_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

__device__ __forceinline__ void ldmatrix_x4(uint32_t (&r)[4], uint32_t addr) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldmatrix_x4_trans(uint32_t (&r)[4], uint32_t addr) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ uint32_t transposed(uint32_t x) {
    uint32_t y;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}
// c (16 x 8) += a (16 x 16) b (16 x 8), bf16 operands, fp32 sums.
__device__ __forceinline__ void mma(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma_f16(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// A request's visible keys: k < len with k < sinks or k >= first; its tiles of T keys: the first `front` of the request's, then those
// from `front + skip` on, n in all.
struct Visible { int len, first, sinks, n, front, skip; };
template <int T>
__device__ __forceinline__ Visible visible(int len, const Args &a) {
    len = max(0, min(len, a.max_pages * a.page_size));
    const int all = (len + T - 1) / T;
    if (a.window == 0 || len <= a.window) return {len, 0, 0, all, 0, 0};
    const int first = len - a.window, sinks = min(a.n_sink, first), front = (sinks + T - 1) / T, skip = max(0, first / T - front);
    return {len, first, sinks, all - skip, front, skip};
}

// Of a stage: whether the tile is its pair's first and last.
constexpr uint32_t kFirst = 1, kLast = 2;

// A pair: its number (its first query's row is g times that), tiles of the batch before its first, its tiles (of a warp's part: < 0, there is none).
struct Pair { int pair, begin, tiles; };

// `all` tiles shared out to workers: worker i has those from all i / workers (rounded down) on.  At most 16 384 workers.
struct Shares {
    int workers, all;
    uint32_t whole, rest;
    float one;           // of a worker
    __device__ __forceinline__ Shares(int n, int tiles) : workers(n), all(tiles), whole((uint32_t)tiles / (uint32_t)n), rest((uint32_t)tiles - whole * (uint32_t)n), one(about_one_over((float)n)) {}
    __device__ __forceinline__ int first(int i) const {
        // rest i / workers, a quotient below 2^14 of a number below 2^28: by its reciprocal one off at most (an integer division takes 100
        // cycles, and a lone request waits for several in a row)
        const uint32_t n = rest * (uint32_t)i, q = (uint32_t)((float)n * one);
        const int left = (int)(n - q * (uint32_t)workers);
        return (int)(whole * (uint32_t)i + q) + (left >= workers) - (left < 0);
    }
    // The worker of tile x: the largest i with first(i) <= x.
    __device__ __forceinline__ int of(int x) const {
        int i = min(workers - 1, (int)((float)x * (float)workers / (float)all));           // (two too low or high at most)
        while (first(i) > x) --i;
        while (i + 1 < workers && first(i + 1) <= x) ++i;
        return i;
    }
};

// A warp's stretch of the batch's `all` tiles: [first, last), beginning in request r, before which lie `before` tiles.  Every warp sums the
// batch by itself, a stretch of the requests a lane: no waiting for others, and the lengths are in L1 after the first.
// As a rule all warps of the grid, `workers` of them, share the tiles evenly.  Where that makes no block's share much larger, blocks
// share the pairs instead, whole, and a block's warps their tiles: no parts leave a block then, and joining them takes 2 us.
// "Much": by more than `few` tiles, by the bound pairs a block x tiles of the longest pair.  (8 heads; whole for shared, us: one request
// of 300 tokens 6.1 for 6.6, of 600 7.6 for 6.7, 8 of 600 7.8 for 8.9, 64 of 300 13.0 for 14.5; 4-bit, one of 300 6.6 for 8.2, of 600
// 7.7 for 8.3, of 900 9.0 for 8.4, 8 of 600 8.0 for 8.9.)
struct Stretch { int first, last, all, workers, r, before; };
template <int T, int NW>
__device__ __forceinline__ Stretch stretch_of(const Args &a, int few) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x / 32, per = (a.batch + 31) / 32, r0 = lane * per, r1 = min(a.batch, r0 + per);
    auto tiles = [&](int r) { return visible<T>(a.seq_len[r], a).n; };
    int own = 0, some = 0, most = 0;                  // tiles, requests that have any, tiles of a head of the longest
#pragma unroll 2
    for (int r = r0; r < r1; ++r) {
        const int n = tiles(r);
        own += n * a.H_kv, some += n > 0, most = max(most, n);
    }
    int end = own, count = some;
#pragma unroll
    for (int o = 1; o < 32; o *= 2) {
        const int x = __shfl_up_sync(0xffffffffu, end, o), y = __shfl_up_sync(0xffffffffu, count, o);
        if (lane >= o) end += x, count += y;
    }
    most = __reduce_max_sync(0xffffffffu, most);
    // The request that has the x-th tile, respectively the x-th that has any, and the tiles before it: the lane whose stretch it is in walks.
    auto find = [&](int x, bool by_tile, int &r, int &before) {
        int passed = by_tile ? end - own : count - some;
        const bool mine = passed <= x && x < (by_tile ? end : count);
        r = r0, before = end - own;
        if (mine)
            for (;; ++r) {
                const int n = tiles(r) * a.H_kv, step = by_tile ? n : n > 0;
                if (x < passed + step) break;
                passed += step, before += n;
            }
        const int src = __ffs(__ballot_sync(0xffffffffu, mine)) - 1;
        r = __shfl_sync(0xffffffffu, r, src);
        before = __shfl_sync(0xffffffffu, before, src);
    };
    Stretch s;
    s.all = __shfl_sync(0xffffffffu, end, 31);
    const int grid = (int)gridDim.x, pairs = __shfl_sync(0xffffffffu, count, 31) * a.H_kv;
    const float a_block = about_one_over((float)grid);         // (a rule of thumb, the same for every warp)
    const bool whole = ceilf((float)pairs * a_block) * (float)most <= (float)few + (float)s.all * a_block;
    s.workers = min(grid * NW, s.all);
    s.first = s.last = s.all;
    s.r = s.before = 0;
    const int blocks = min(grid, pairs);
    if (whole ? (int)blockIdx.x >= blocks : (int)blockIdx.x * NW + warp >= s.workers) return s;       // (fewer tiles than warps: the first have one each)
    if (whole) {
        const Shares pair_shares(blocks, pairs);
        int first = 0, last = 0;
#pragma unroll 1                                           // (one copy of the search: see the note at the joins)
        for (int end = 0; end < 2; ++end) {
            const int pair = pairs <= grid ? (int)blockIdx.x : pair_shares.first((int)blockIdx.x + end);
            int r = 0, x = s.all, n = 0;
            if (pair < pairs) {
                const int nth = pair / a.H_kv;
                find(nth, false, r, x);
                n = tiles(r);
                s.r = r, s.before = x;
                x += (pair - nth * a.H_kv) * n;
            }
            (end ? last : first) = x;
            if (pairs <= grid) {
                last = first + n;
                break;
            }
        }
        const int mates = min(NW, last - first);
        const Shares shares(mates, last - first);
        s.first = warp < mates ? first + shares.first(warp) : last;
        s.last = warp < mates ? first + shares.first(warp + 1) : last;
        if (warp >= mates || pairs <= grid) return s;
    } else {
        const Shares shares(s.workers, s.all);
        s.first = shares.first((int)blockIdx.x * NW + warp);
        s.last = shares.first((int)blockIdx.x * NW + warp + 1);
    }
    find(s.first, true, s.r, s.before);
    return s;
}

// Requests without a key: zeros, and nothing for a sum.
template <int D, int NT, int T>
__device__ __forceinline__ void empty_requests(const Args &a) {
#pragma unroll 1
    for (int r = blockIdx.x; r < a.batch; r += gridDim.x)
        if (visible<T>(a.seq_len[r], a).n == 0) {
#pragma unroll 1
            for (int i = threadIdx.x; i < a.H_q * D / 8; i += NT) stg(reinterpret_cast<uint4 *>(a.out + (size_t)r * a.H_q * D) + i, make_uint4(0, 0, 0, 0));
            if (a.lse)
#pragma unroll 1
                for (int i = threadIdx.x; i < a.H_q; i += NT) a.lse[(size_t)r * a.H_q + i] = -INFINITY;
        }
}

// SMALL: pages of fewer tokens than a tile.  FOLD (4-bit, at most 4 queries a KV head): columns 4 to 7 hold the same queries as 0 to
// 3, and stand for the tile's second 16 keys where 0 to 3 stand for the first: a lane has half the scores to turn into weights, none
// of them of an empty column.  In the output they are the second half of head_dim (see the values' products).
template <int D, bool F4, int NQ, bool SMALL, bool FOLD>
__global__ void __launch_bounds__(Geo<D, F4, NQ>::kThreads, 1)
decode_attn_kernel(const __grid_constant__ Args a) {
    using G = Geo<D, F4, NQ>;
    constexpr int T = G::kTile, SUB = T / 16, NW = G::kWarps, NT = G::kThreads, CPR = G::kRow / 16, Q8 = 8 * NQ, KS = D / 16, RP = D + 4;
    constexpr int SC = FOLD ? 1 : SUB;                // sets of 16 keys that a lane has scores of
    static_assert(!FOLD || (F4 && NQ == 1 && SUB == 2), "");
    constexpr uint32_t kAllRows = T == 32 ? 0xffffffffu : 0xffffu;
    extern __shared__ __align__(128) uint8_t smem[];
    __shared__ uint2 s_stage[NW][G::kStages];         // rows that are there (bit i: row i) and flags
    __shared__ Pair s_pair[NW][G::kStages];           // of a stage that is its pair's first, or the warp's
    __shared__ float2 s_ml[NW][2][Q8];
    __shared__ Pair s_part[NW][2];                    // [0]: of a pair that began before the warp's stretch, [1]: of one that goes on behind it
    __shared__ int s_first[NW + 1], s_leaves[2], s_join[2][2], s_shared[2];
    const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32, quad = lane / 4, t = lane % 4;
    const int page_shift = __ffs(a.page_size) - 1;
    if (lane < 2) s_part[warp][lane] = {0, 0, -1};
    if (tid < 2) s_leaves[tid] = -1;
    grid_wait();
    grid_release();
    const Stretch mine = stretch_of<T, NW>(a, G::kFew);
    if (lane == 0) {                                  // (kept for the end)
        s_first[warp] = mine.first;
        s_shared[0] = mine.workers, s_shared[1] = mine.all;
        if (warp == NW - 1) s_first[NW] = mine.last;
    }
    const int my_tiles = mine.last - mine.first;
    const uint32_t smem0 = ptx::smem_u32(smem), ring = smem0 + warp * G::kStages * G::kStageBytes;
    float *part0 = reinterpret_cast<float *>(smem + G::kRing) + warp * G::kPart;

    if (my_tiles > 0) {
        // ---- the warp's fetching end: where the next tile to be sent for lies, and the page ids of the next kBatch tiles from jb on,
        // one a lane (SMALL: one a lane for every 8 rows)
        constexpr int GROUPS = T / 8, kBatch = SMALL ? 32 / GROUPS : 32;
        int r = mine.r, base = mine.before, sent = 0, h, j, jb, page_ids;
        Visible vis = visible<T>(a.seq_len[r], a);
        h = (mine.first - base) / vis.n;
        j = jb = (mine.first - base) - h * vis.n;
        auto tile_at = [&](int i) { return i < vis.front ? i : i + vis.skip; };
        auto load_pages = [&]() {
            const int i = jb + (SMALL ? lane / GROUPS : lane), key = tile_at(i) * T + (SMALL ? lane % GROUPS * 8 : 0);
            page_ids = i < vis.n && key < vis.len ? a.table[(size_t)r * a.max_pages + (key >> page_shift)] : -1;
        };
        load_pages();
        constexpr int RPT = 32 / CPR;              // rows a turn of 32 lanes
        const uint32_t head_bytes = F4 ? (uint32_t)a.page_size * (D / 2 + 8) : (uint32_t)G::kRow;
        const uint32_t row_bytes = F4 ? (uint32_t)G::kRow : a.H_kv * head_bytes, page_bytes = F4 ? a.H_kv * head_bytes : row_bytes << page_shift;
        const uint32_t numbers = (uint32_t)a.page_size * (D / 2);
        // A lane's own places: of its 16 bytes of a turn's rows (and its 8 of their numbers) in the keys of page 0, head h, and in a stage.  16-bit
        // chunks are turned by the row, as ldmatrix wants them; so are those of 4-bit values, of two rows (head_dim 64: four) alike,
        // so that 8 rows' lie in different banks.
        const uint32_t place = lane / CPR * row_bytes + lane % CPR * 16;
        const uint8_t *lane_k = a.k + (size_t)h * head_bytes + place;
        const ptrdiff_t to_v = a.v - a.k;
        const int32_t to_numbers = (int32_t)(numbers + lane * 8) - (int32_t)place;
        auto chunk_k = [&](int row) { return F4 ? lane % CPR : (lane % CPR) ^ (row & 7); };
        auto turned_v = [](int chunk, int row) { return chunk ^ (D == 128 ? (row >> 1) & 3 : (row >> 2) & 1); };
        auto chunk_v = [&](int row) { return F4 ? turned_v(lane % CPR, row) : chunk_k(row); };
        int run = 0;                               // tiles from j on that are neither first nor last of their pair and all there, pages apart
        uint32_t plain = 0;                        // stages that hold such a tile
        auto fetch = [&](int at) {
            if (sent < my_tiles) {
                const int key0 = tile_at(j) * T;
                auto in_pool = [&](int page) { return (uint32_t)page < (uint32_t)a.num_pool_pages; };
                // the page of row `row` (of any where a page holds the tile)
                auto page_of = [&](int row) { return __shfl_sync(0xffffffffu, page_ids, SMALL ? (j - jb) * GROUPS + row / 8 : j - jb); };
                const int page = page_of(lane & (T - 1));
                const uint32_t kb = ring + at * G::kStageBytes, vb = kb + T * G::kRow;
                uint32_t rows = kAllRows;
                if (!SMALL && run > 0 && in_pool(page)) {
                    plain |= 1u << at;
                } else {
                    plain &= ~(1u << at);
                    const int key = key0 + (lane & (T - 1));
                    rows = __ballot_sync(0xffffffffu, key < vis.len && (key < vis.sinks || key >= vis.first) && in_pool(page)) & kAllRows;
                    if (lane == 0) {
                        s_stage[warp][at] = make_uint2(rows, (j == 0 ? kFirst : 0u) | (j == vis.n - 1 ? kLast : 0u));
                        if (j == 0 || sent == 0) s_pair[warp][at] = {r * a.H_kv + h, base + h * vis.n, vis.n};
                    }
                }
                if (!SMALL && rows == kAllRows) {
                    const uint8_t *k = lane_k + (uint64_t)(uint32_t)page * page_bytes + (uint64_t)(uint32_t)(key0 & (a.page_size - 1)) * row_bytes;
                    const uint8_t *v = k + to_v;
#pragma unroll
                    for (int i = 0; i < T / RPT; ++i) {
                        const int row = i * RPT + lane / CPR;
                        cp_async<16>(kb + row * G::kRow + chunk_k(row) * 16, k + (size_t)(i * RPT) * row_bytes);
                        cp_async<16>(vb + row * G::kRow + chunk_v(row) * 16, v + (size_t)(i * RPT) * row_bytes);
                    }
                    if constexpr (F4) {                // (T = 32: a lane has a row's numbers)
                        // (the rows before the tile's have numbers of 8 bytes where their codes have kRow)
                        const ptrdiff_t back = to_numbers - (ptrdiff_t)(key0 & (a.page_size - 1)) * (G::kRow - 8);
                        cp_async<8>(vb + T * G::kRow + lane * 8, k + back);
                        cp_async<8>(vb + T * G::kRow + T * 8 + lane * 8, v + back);
                    }
                } else {
                    // (of a page that is not there nothing is read)
                    auto page_at = [&](int id) { return (uint64_t)(in_pool(id) ? (uint32_t)id : 0u) * page_bytes; };
                    const int within = key0 & (a.page_size - 1);
                    const uint8_t *k0 = lane_k + (SMALL ? 0 : page_at(page) + (uint64_t)(uint32_t)within * row_bytes);
#pragma unroll
                    for (int i = 0; i < T / RPT; ++i) {
                        const int row = i * RPT + lane / CPR;
                        const uint8_t *k = SMALL ? lane_k - place + page_at(page_of(row)) + (uint64_t)((key0 + row) & (a.page_size - 1)) * row_bytes + lane % CPR * 16
                                                 : k0 + (size_t)(i * RPT) * row_bytes;
                        cp_async<16>(kb + row * G::kRow + chunk_k(row) * 16, k, (rows >> row) & 1);
                        cp_async<16>(vb + row * G::kRow + chunk_v(row) * 16, k + to_v, (rows >> row) & 1);
                    }
                    if constexpr (F4) {
                        const uint8_t *k = lane_k - place + page_at(page) + numbers + (uint64_t)((key0 + lane) & (a.page_size - 1)) * 8;
                        cp_async<8>(vb + T * G::kRow + lane * 8, k, (rows >> lane) & 1);
                        cp_async<8>(vb + T * G::kRow + T * 8 + lane * 8, k + to_v, (rows >> lane) & 1);
                    }
                }
                ++sent, ++j;
                if (--run <= 0 && sent < my_tiles) {
                    if (j == vis.n) {
                        const bool same = jb == 0 && h + 1 < a.H_kv;          // the next head's pages are the ones at hand
                        j = jb = 0;
                        if (++h == a.H_kv) {
                            h = 0;
                            do {
                                base += vis.n * a.H_kv;
                                vis = visible<T>(a.seq_len[++r], a);
                            } while (vis.n == 0);
                        }
                        lane_k = a.k + (size_t)h * head_bytes + place;
                        if (!same) load_pages();
                    } else if (j - jb == kBatch) {
                        jb = j;
                        load_pages();
                    }
                    if (!SMALL && j > 0 && (j + 1 < vis.front || j > vis.front || vis.first == 0))
                        run = min(min(vis.n - 1, jb + kBatch), vis.first > 0 && j < vis.front ? vis.front - 1 : vis.n) - j;
                }
            }
            cp_commit();
        };

        // ---- the consuming end: one pair's queries, references, sums and accumulators at a time
        uint32_t qf[NQ][KS][2];          // Q^T as the MMA's second operand: column quad (+ 8) is a query
        float q_sum[NQ][2][2];           // 4-bit: sums of q over each half, of columns 2 t and 2 t + 1, in units of `unit`
        float unit[NQ][2];               // score times scale log2(e) per score sum: scale_log2, 4-bit: by column, for q's and the codes' scaling
        float m[NQ][2], l[NQ][2], off[NQ][2][2];         // off (4-bit): sums of p times a half's middle value
        constexpr int NA = FOLD ? D / 32 : D / 16;
        float acc[NQ][NA][4];            // 4-bit: times v_unit 2^-133, second half 2^-129 (FOLD: lanes of columns 4 to 7)
        float v_unit = kValueUnit, v_limit = kValueTop / kValueUnit;

        auto begin_pair = [&](int pair) {
#pragma unroll
            for (int n = 0; n < NQ; ++n) {
                const int col = n * 8 + (FOLD ? quad & 3 : quad);
                const bool there = col < a.g;
                const __nv_bfloat16 *q = a.q + ((size_t)pair * a.g + (there ? col : 0)) * D;
                if constexpr (F4) {
                    // A code in the last four bits of a half is the fp16 number c 2^-24 (16 c 2^-24 one nibble higher), so keys need no
                    // conversion where q is fp16: scaled by a power of two for its greatest element to lie below 2^14, the second
                    // half by another 1/16.  (Exact, but for elements 2^-26 of the greatest and less.)  The order is that in which a lane's codes
                    // come: elements 16 t + 4 w + {0, 2}, {1, 3} of each half.
                    uint2 x[2][KS / 2];
                    float top = 0.f, sum[2] = {0.f, 0.f};
#pragma unroll
                    for (int half = 0; half < 2; ++half)
#pragma unroll
                        for (int w = 0; w < KS / 2; ++w) {
                            x[half][w] = there ? *reinterpret_cast<const uint2 *>(q + half * (D / 2) + (D / 8) * t + 4 * w) : make_uint2(0, 0);
#pragma unroll
                            for (int i = 0; i < 4; ++i) {
                                const uint32_t v = i < 2 ? x[half][w].x : x[half][w].y;
                                const float f = __uint_as_float(i & 1 ? v & 0xffff0000u : v << 16);
                                top = fmaxf(top, fabsf(f));
                                sum[half] += f;
                            }
                        }
                    top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
                    top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
                    // 2^(13 - exponent of top), at most 2^100
                    const int up = min(13 + 127 - (int)(__float_as_uint(top) >> 23), 100);
                    const float scale = __uint_as_float((uint32_t)(127 + up) << 23);
#pragma unroll
                    for (int half = 0; half < 2; ++half)
#pragma unroll
                        for (int w = 0; w < KS / 2; ++w) {
                            float f[4];
#pragma unroll
                            for (int i = 0; i < 4; ++i) {
                                const uint32_t v = i < 2 ? x[half][w].x : x[half][w].y;
                                f[i] = __uint_as_float(i & 1 ? v & 0xffff0000u : v << 16) * scale * (half ? 0.0625f : 1.f);
                            }
                            const __half2 e = __floats2half2_rn(f[0], f[2]), o = __floats2half2_rn(f[1], f[3]);
                            qf[n][half * (KS / 2) + w][0] = *reinterpret_cast<const uint32_t *>(&e);
                            qf[n][half * (KS / 2) + w][1] = *reinterpret_cast<const uint32_t *>(&o);
                        }
                    const float mine = 16777216.f / scale;                // of column quad: score per sum
#pragma unroll
                    for (int e = 0; e < 2; ++e) unit[n][e] = a.scale_log2 * __shfl_sync(0xffffffffu, mine, 8 * t + 4 * e);     // column 2 t + e: lane 4 (2 t + e)
#pragma unroll
                    for (int half = 0; half < 2; ++half) {
                        float s = sum[half];
                        s += __shfl_xor_sync(0xffffffffu, s, 1);
                        s += __shfl_xor_sync(0xffffffffu, s, 2);
                        s *= scale * 5.9604644775390625e-8f;              // 2^-24
#pragma unroll
                        for (int e = 0; e < 2; ++e) q_sum[n][half][e] = __shfl_sync(0xffffffffu, s, 8 * t + 4 * e);
                    }
                } else {
#pragma unroll
                    for (int s = 0; s < KS; ++s)
#pragma unroll
                        for (int i = 0; i < 2; ++i) qf[n][s][i] = there ? *reinterpret_cast<const uint32_t *>(q + 16 * s + 8 * i + 2 * t) : 0u;
                    unit[n][0] = unit[n][1] = a.scale_log2;
                }
                v_unit = kValueUnit, v_limit = kValueTop / kValueUnit;
#pragma unroll
                for (int e = 0; e < 2; ++e) m[n][e] = -INFINITY, l[n][e] = off[n][0][e] = off[n][1][e] = 0.f;
#pragma unroll
                for (int d = 0; d < NA; ++d)
#pragma unroll
                    for (int e = 0; e < 4; ++e) acc[n][d][e] = 0.f;
            }
        };
        // Sums over the lanes of a column, and (4-bit) the middle values' share into the accumulators.
        auto sum_up = [&]() {
#pragma unroll
            for (int n = 0; n < NQ; ++n)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    auto column_sum = [](float x) {
                        x += __shfl_xor_sync(0xffffffffu, x, 4);
                        x += __shfl_xor_sync(0xffffffffu, x, 8);
                        x += __shfl_xor_sync(0xffffffffu, x, 16);
                        return FOLD ? x + __shfl_xor_sync(0xffffffffu, x, 2) : x;          // (columns c and c + 4: lanes t and t + 2)
                    };
                    l[n][e] = column_sum(l[n][e]);
                    if constexpr (F4) {
                        const float o[2] = {column_sum(off[n][0][e]), column_sum(off[n][1][e])};
                        const float back = kValueUnit / v_unit;
#pragma unroll
                        for (int d = 0; d < NA; ++d) {
                            const bool second = FOLD ? t >= 2 : d >= D / 32;
#pragma unroll
                            for (int i = 0; i < 2; ++i)          // 2^133 / v_unit, 2^129 / v_unit
                                acc[n][d][e + 2 * i] = fmaf(acc[n][d][e + 2 * i] * (second ? 3.6893488147419103e19f : 5.9029581035870565e20f), back, second ? o[1] : o[0]);
                        }
                    }
                }
        };
        // Element of head_dim that row quad (i = 0) or quad + 8 (i = 1) of accumulator d is.
        auto element = [&](int d, int i) {
            return F4 ? (FOLD ? t >> 1 : d / (D / 32)) * (D / 2) + d % (D / 32) * 16 + 2 * quad + i : 16 * d + 8 * i + quad;
        };
        // Query (of the KV head) whose column a lane's accumulators 0 and 2, respectively 1 and 3, are.
        auto column = [&](int n, int e) { return FOLD ? (2 * t + e) & 3 : n * 8 + 2 * t + e; };
        auto write_out = [&](int pair) {
            const size_t head0 = (size_t)pair * a.g;
#pragma unroll
            for (int n = 0; n < NQ; ++n) {
                float inv[2];
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const int col = column(n, e);
                    // (by the sum: the reference stays at -inf where all scores are NaN, too, and NaN is then the result)
                    inv[e] = l[n][e] == 0.f ? 0.f : about_one_over(l[n][e]);
                    if (a.lse && quad == 0 && col < a.g && (!FOLD || t < 2)) a.lse[head0 + col] = l[n][e] == 0.f ? -INFINITY : (m[n][e] + lg2(l[n][e])) * 0.6931471805599453f;
                }
                if constexpr (F4) {
                    // (accumulators e and e + 2 are neighbouring elements)
#pragma unroll
                    for (int e = 0; e < 2; ++e)
                        if (column(n, e) < a.g)
#pragma unroll
                            for (int d = 0; d < NA; ++d)
                                *reinterpret_cast<uint32_t *>(a.out + (head0 + column(n, e)) * D + element(d, 0)) = pack_bf16(acc[n][d][e] * inv[e], acc[n][d][e + 2] * inv[e]);
                } else {
                    // 8 x 8 blocks turned, so that a lane has two neighbouring elements of one query
                    const int col = n * 8 + quad;
#pragma unroll
                    for (int d = 0; d < D / 16; ++d)
#pragma unroll
                        for (int i = 0; i < 2; ++i) {
                            const uint32_t y = transposed(pack_bf16(acc[n][d][2 * i] * inv[0], acc[n][d][2 * i + 1] * inv[1]));
                            if (col < a.g) *reinterpret_cast<uint32_t *>(a.out + (head0 + col) * D + 16 * d + 8 * i + 2 * t) = y;
                        }
                }
            }
        };
        auto keep_part = [&](int which, float *to, const Pair &now) {
#pragma unroll
            for (int n = 0; n < NQ; ++n)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const int col = column(n, e);
                    if (quad == 0) s_ml[warp][which][col] = make_float2(m[n][e], l[n][e]);
#pragma unroll
                    for (int d = 0; d < NA; ++d) {
                        to[col * RP + element(d, 0)] = acc[n][d][e];
                        to[col * RP + element(d, 1)] = acc[n][d][e + 2];
                    }
                }
            if (lane == 0) s_part[warp][which] = now;
        };

        begin_pair(r * a.H_kv + h);           // (q comes in beside the page ids)
        bool begun_here = false;
        Pair now{};
        int at = 0;
        for (int s = 1 - G::kStages; s < my_tiles; ++s) {
            if (s >= 0) {
                cp_wait<G::kStages - 2>();
                __syncwarp();
            }
            fetch(s < 0 ? s + G::kStages - 1 : at == 0 ? G::kStages - 1 : at - 1);      // into the stage consumed in the last turn
            if (s < 0) continue;
            const uint2 stage = (plain >> at) & 1 ? make_uint2(kAllRows, 0u) : s_stage[warp][at];
            if (s == 0 || (stage.y & kFirst)) {
                now = s_pair[warp][at];
                begun_here = (stage.y & kFirst) != 0;
                if (s > 0) begin_pair(now.pair);
            }
            const uint32_t kb = ring + at * G::kStageBytes, vb = kb + T * G::kRow;
            const uint8_t *kp8 = smem + (kb - smem0), *vp8 = smem + (vb - smem0);
            auto key_row = [&](int u, int i) { return (FOLD ? t >> 1 : u) * 16 + quad + 8 * i; };      // of the tile, of a lane's scores 2 i and 2 i + 1
            float sc[SC][NQ][4];
            if constexpr (F4) {
                float part[SC][NQ][2][4];
#pragma unroll
                for (int sub = 0; sub < SUB; ++sub) {
                    float sum[NQ][2][4];
#pragma unroll
                    for (int n = 0; n < NQ; ++n)
#pragma unroll
                        for (int e = 0; e < 4; ++e) sum[n][0][e] = sum[n][1][e] = 0.f;
                    uint32_t w[2][D / 32];               // 16 (8) bytes of rows quad and quad + 8
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        const uint8_t *b = kp8 + (sub * 16 + quad + 8 * i) * G::kRow + (D / 8) * t;
                        if constexpr (D == 128) *reinterpret_cast<uint4 *>(w[i]) = *reinterpret_cast<const uint4 *>(b);
                        else *reinterpret_cast<uint2 *>(w[i]) = *reinterpret_cast<const uint2 *>(b);
                    }
#pragma unroll
                    for (int x = 0; x < D / 32; ++x) {
                        const uint32_t w0 = w[0][x], w1 = w[1][x], u0 = w0 >> 8, u1 = w1 >> 8;
                        const uint32_t lo[4] = {w0 & 0x000f000fu, w1 & 0x000f000fu, u0 & 0x000f000fu, u1 & 0x000f000fu};
                        const uint32_t hi[4] = {w0 & 0x00f000f0u, w1 & 0x00f000f0u, u0 & 0x00f000f0u, u1 & 0x00f000f0u};
#pragma unroll
                        for (int n = 0; n < NQ; ++n) {
                            mma_f16(sum[n][0], lo, qf[n][x][0], qf[n][x][1]);
                            mma_f16(sum[n][1], hi, qf[n][KS / 2 + x][0], qf[n][KS / 2 + x][1]);
                        }
                    }
#pragma unroll
                    for (int n = 0; n < NQ; ++n)
#pragma unroll
                        for (int half = 0; half < 2; ++half)
#pragma unroll
                            for (int e = 0; e < 4; ++e) part[FOLD ? 0 : sub][n][half][e] = FOLD && sub == 1 && t < 2 ? part[0][n][half][e] : sum[n][half][e];
                }
                // q.k = sum over the halves of s (q.c) + m sum q
#pragma unroll
                for (int u = 0; u < SC; ++u)
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        const uint2 pr = *reinterpret_cast<const uint2 *>(vp8 + T * G::kRow + key_row(u, i) * 8);
                        const float s0 = __uint_as_float(pr.x << 16), m0 = __uint_as_float(pr.x & 0xffff0000u), s1 = __uint_as_float(pr.y << 16), m1 = __uint_as_float(pr.y & 0xffff0000u);
#pragma unroll
                        for (int n = 0; n < NQ; ++n)
#pragma unroll
                            for (int e = 0; e < 2; ++e)
                                sc[u][n][2 * i + e] = fmaf(s0, part[u][n][0][2 * i + e], fmaf(m0, q_sum[n][0][e], fmaf(s1, part[u][n][1][2 * i + e], m1 * q_sum[n][1][e])));
                    }
            } else {
#pragma unroll
                for (int sub = 0; sub < SUB; ++sub) {
                    float odd[NQ][4];                    // (two chains of products)
#pragma unroll
                    for (int n = 0; n < NQ; ++n)
#pragma unroll
                        for (int e = 0; e < 4; ++e) sc[sub][n][e] = odd[n][e] = 0.f;
                    const int lr = sub * 16 + (lane & 15);            // lanes 0-15: rows, first 8 columns; 16-31: next 8
#pragma unroll
                    for (int ks = 0; ks < KS; ++ks) {
                        uint32_t f[4];
                        ldmatrix_x4(f, kb + lr * G::kRow + (((2 * ks + (lane >> 4)) ^ (lr & 7)) << 4));
#pragma unroll
                        for (int n = 0; n < NQ; ++n) mma(ks & 1 ? odd[n] : sc[sub][n], f, qf[n][ks][0], qf[n][ks][1]);
                    }
#pragma unroll
                    for (int n = 0; n < NQ; ++n)
#pragma unroll
                        for (int e = 0; e < 4; ++e) sc[sub][n][e] += odd[n][e];
                }
            }
            if (stage.x != kAllRows) {
#pragma unroll
                for (int u = 0; u < SC; ++u)
#pragma unroll
                    for (int n = 0; n < NQ; ++n)
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            if (!((stage.x >> key_row(u, e >> 1)) & 1)) sc[u][n][e] = a.scale_log2 < 0.f ? INFINITY : -INFINITY;
            }
            // Weights against the reference; that moves only where a score would go far above it (and at the first keys): then to the
            // columns' true maxima, the lanes of a column together.
            float p[SC][NQ][4];
            bool low = true;
            uint2 vpar[SC][2];                  // (4-bit) the values' numbers
            if constexpr (F4) {
#pragma unroll
                for (int u = 0; u < SC; ++u)
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        vpar[u][i] = *reinterpret_cast<const uint2 *>(vp8 + T * (G::kRow + 8) + key_row(u, i) * 8);
                        low = low && __uint_as_float(vpar[u][i].x << 16) <= v_limit && __uint_as_float(vpar[u][i].y << 16) <= v_limit;
                    }
            }
#pragma unroll
            for (int u = 0; u < SC; ++u)
#pragma unroll
                for (int n = 0; n < NQ; ++n)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        p[u][n][e] = fmaf(sc[u][n][e], unit[n][e & 1], -m[n][e & 1]);
                        low = low && p[u][n][e] <= 8.f;
                    }
            if (!__all_sync(0xffffffffu, low)) {
                if constexpr (F4) {
                    // The values' unit goes by the first scales of a pair, and changes where far larger ones come.
                    float top = 0.f;
#pragma unroll
                    for (int u = 0; u < SC; ++u)
#pragma unroll
                        for (int i = 0; i < 2; ++i) top = fmaxf(top, fmaxf(__uint_as_float(vpar[u][i].x << 16), __uint_as_float(vpar[u][i].y << 16)));
#pragma unroll
                    for (int o = 1; o < 32; o *= 2) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
                    const bool begins = __all_sync(0xffffffffu, m[0][0] == -INFINITY);
                    if ((top > v_limit || (begins && top > 0.f)) && top < INFINITY) {
                        // 2^(64 - exponent of top), where there is something already 2^(100 - exponent), at most 2^120
                        const float to = __uint_as_float((uint32_t)min((begins ? 64 : 100) + 254 - (int)(__float_as_uint(top) >> 23), 247) << 23);
                        const float f = to / v_unit;
                        v_unit = to, v_limit = kValueTop / to;
#pragma unroll
                        for (int n = 0; n < NQ; ++n)
#pragma unroll
                            for (int d = 0; d < NA; ++d)
#pragma unroll
                                for (int e = 0; e < 4; ++e) acc[n][d][e] *= f;
                    }
                }
#pragma unroll
                for (int n = 0; n < NQ; ++n)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        float top = -INFINITY;
#pragma unroll
                        for (int u = 0; u < SC; ++u) top = fmaxf(top, fmaxf(sc[u][n][e] * unit[n][e], sc[u][n][e + 2] * unit[n][e]));
                        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 4));
                        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 8));
                        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 16));
                        if (FOLD) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
                        const float mn = fmaxf(m[n][e], top), f = mn == -INFINITY ? 1.f : ex2(m[n][e] - mn), ref = mn == -INFINITY ? 0.f : mn;
                        m[n][e] = mn;
                        l[n][e] *= f;
                        off[n][0][e] *= f;
                        off[n][1][e] *= f;
#pragma unroll
                        for (int d = 0; d < NA; ++d) acc[n][d][e] *= f, acc[n][d][e + 2] *= f;
#pragma unroll
                        for (int u = 0; u < SC; ++u)
#pragma unroll
                            for (int i = 0; i < 2; ++i) p[u][n][e + 2 * i] = fmaf(sc[u][n][e + 2 * i], unit[n][e], -ref);
                    }
            }
            uint32_t other[2];                   // (FOLD) the weights of the lane 16 away: the other half's, of the other 16 keys
            uint32_t weight[NQ][2][2];           // (4-bit) the second operand of the values' products, by half and by rows quad and quad + 8
#pragma unroll
            for (int sub = 0; sub < SUB; ++sub) {
                if (!FOLD || sub == 0) {
#pragma unroll
                    for (int n = 0; n < NQ; ++n)
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            p[FOLD ? 0 : sub][n][e] = ex2(p[FOLD ? 0 : sub][n][e]);
                            l[n][e & 1] += p[FOLD ? 0 : sub][n][e];
                        }
                }
                if constexpr (F4) {
                    // sum p v = sum b (c - 8) + sum p (m + 8 s), half by half, with b = p s rounded to bf16 (in units of 1 / v_unit), the MMA's
                    // operand; a code in the last four bits of a half is the bf16 number c 2^-133 (16 c 2^-133 one nibble higher), a
                    // subnormal that needs no conversion.  The MMAs sum b c; -8 b of the lane's own keys joins p (m + 8 s), so that b's rounding
                    // counts for the distance from the middle alone.
                    const float eight = __uint_as_float((257u << 23) - __float_as_uint(v_unit));           // 8 / v_unit, a power of two
                    if (!FOLD || sub == 0) {
                        const int u = FOLD ? 0 : sub;
#pragma unroll
                        for (int i = 0; i < 2; ++i) {
                            const float vs[2] = {__uint_as_float(vpar[u][i].x << 16), __uint_as_float(vpar[u][i].y << 16)};
                            const float mid[2] = {fmaf(8.f, vs[0], __uint_as_float(vpar[u][i].x & 0xffff0000u)), fmaf(8.f, vs[1], __uint_as_float(vpar[u][i].y & 0xffff0000u))};
#pragma unroll
                            for (int half = 0; half < 2; ++half) {
                                const float su = vs[half] * v_unit;
#pragma unroll
                                for (int n = 0; n < NQ; ++n) {
                                    const uint32_t b = pack_bf16(p[u][n][2 * i] * su, p[u][n][2 * i + 1] * su);
                                    weight[n][half][i] = transposed(b);
#pragma unroll
                                    for (int e = 0; e < 2; ++e)
                                        off[n][half][e] = fmaf(p[u][n][2 * i + e], mid[half], fmaf(-eight, __uint_as_float(e ? b & 0xffff0000u : b << 16), off[n][half][e]));
                                }
                            }
                        }
                    }
                    // Without FOLD a product for each half.  FOLD: columns 0 to 3 are the first half of the 16 keys' values, 4 to 7 the second.  Bytes
                    // as they are, 16 c1 + c0, stand against the first half's weights; the second codes alone, 16 c1, against the second
                    // half's and, to take them off again, minus the first's.  (255 2^-133 is a bf16 number yet.)
                    uint32_t b[NQ][2][2];
#pragma unroll
                    for (int n = 0; n < NQ; ++n)
#pragma unroll
                        for (int i = 0; i < 2; ++i)
                            if constexpr (FOLD) {
                                if (sub == 0) other[i] = __shfl_xor_sync(0xffffffffu, quad < 4 ? weight[n][1][i] : weight[n][0][i], 16);
                                const uint32_t mine = sub == 0 ? (quad < 4 ? weight[n][0][i] : other[i]) : (quad < 4 ? other[i] : weight[n][1][i]);
                                b[n][0][i] = quad < 4 ? mine : 0u;
                                b[n][1][i] = quad < 4 ? mine ^ 0x80008000u : mine;
                            } else {
                                b[n][0][i] = weight[n][0][i], b[n][1][i] = weight[n][1][i];
                            }
                    // 8 x 8 blocks of pairs of bytes, turned: a lane has bytes 2 quad and 2 quad + 1 of 16 of the keys of operand rows 2 t and 2 t + 1
                    // (respectively 8 more), whose even and odd bytes are the products' rows quad and quad + 8.
                    const int row = sub * 16 + (lane & 15);
                    const uint32_t from = vb + row * G::kRow;
#pragma unroll
                    for (int c = 0; c < D / 32; c += 2) {
                        uint32_t w[4];
                        ldmatrix_x4_trans(w, from + turned_v(c + (lane >> 4), row) * 16);
#pragma unroll
                        for (int x = 0; x < 2; ++x) {
                            const uint32_t w0 = w[2 * x], w1 = w[2 * x + 1];
                            // (FOLD: the bytes, else the first half's codes; the odd ones a byte lower)
                            const uint32_t mask = FOLD ? 0x00ff00ffu : 0x000f000fu, u0 = FOLD ? __byte_perm(w0, 0, 0x4341) : w0 >> 8, u1 = FOLD ? __byte_perm(w1, 0, 0x4341) : w1 >> 8;
                            const uint32_t lo[4] = {w0 & mask, FOLD ? u0 : u0 & mask, w1 & mask, FOLD ? u1 : u1 & mask};
                            const uint32_t hi[4] = {w0 & 0x00f000f0u, u0 & 0x00f000f0u, w1 & 0x00f000f0u, u1 & 0x00f000f0u};
#pragma unroll
                            for (int n = 0; n < NQ; ++n) {
                                mma(acc[n][c + x], lo, b[n][0][0], b[n][0][1]);
                                mma(acc[n][(FOLD ? 0 : D / 32) + c + x], hi, b[n][1][0], b[n][1][1]);
                            }
                        }
                    }
                } else {
                    uint32_t b[NQ][2];
#pragma unroll
                    for (int n = 0; n < NQ; ++n)
#pragma unroll
                        for (int i = 0; i < 2; ++i) b[n][i] = transposed(pack_bf16(p[sub][n][2 * i], p[sub][n][2 * i + 1]));
                    const int lr = sub * 16 + (lane & 7) + ((lane >> 4) << 3), lc = (lane >> 3) & 1;      // blocks: keys 0-7 | 8-15 by lanes 0-15 | 16-31, columns alternating
#pragma unroll
                    for (int d = 0; d < D / 16; ++d) {
                        uint32_t f[4];
                        ldmatrix_x4_trans(f, vb + lr * G::kRow + (((2 * d + lc) ^ (lr & 7)) << 4));
#pragma unroll
                        for (int n = 0; n < NQ; ++n) mma(acc[n][d], f, b[n][0], b[n][1]);
                    }
                }
            }
            __syncwarp();                  // all lanes are through with the stage
            const bool ends = (stage.y & kLast) != 0;
            if (ends || s == my_tiles - 1) {
                sum_up();
                if (ends && begun_here) write_out(now.pair);
                else keep_part(begun_here, begun_here ? reinterpret_cast<float *>(smem + (ring - smem0)) : part0, now);     // (nothing is on its way into the ring any more)
            }
            at = at + 1 == G::kStages ? 0 : at + 1;
        }
        cp_wait<0>();
    }
    __syncthreads();

    // ---- the block's parts.  A chain is one pair's: a part at a stretch's end (c - 1 is the warp; or, c = 0, of a pair that began before
    // the block, at the first stretch's beginning), then the following warps' parts at their beginnings.
    const int first = s_first[0], last = s_first[NW];      // the block's tiles
    auto write_joined = [&](int pair, int col, int el, float top, float sum, const float4 &o) {
        const size_t head = (size_t)pair * a.g + col;
        const float inv = sum == 0.f ? 0.f : about_one_over(sum);
        *reinterpret_cast<uint2 *>(a.out + head * D + el) = make_uint2(pack_bf16(o.x * inv, o.y * inv), pack_bf16(o.z * inv, o.w * inv));
        if (a.lse && el == 0) a.lse[head] = sum == 0.f ? -INFINITY : (top + lg2(sum)) * 0.6931471805599453f;
    };
    // A thread takes four elements of a query; 16 threads side by side (a query's, or half of one's) share out the parts' references and
    // sums.  Little code, in rolled loops: what runs once costs what it takes to fetch.  (Written out part by part for every thread, pair
    // after pair, and with three copies of fetch(), the kernel had 85 KB of code for 49; a lone request of 5 312 tokens took 12.0 us, now
    // 9.0, 64 of 200 to 16 384 tokens in 4 bits 113, then 109.)
    const int per = a.g * (D / 4), sub16 = lane & 15;
    auto max16 = [](float x) {
#pragma unroll
        for (int o = 8; o > 0; o /= 2) x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, o));
        return x;
    };
    auto sum16 = [](float x) {
#pragma unroll
        for (int o = 8; o > 0; o /= 2) x += __shfl_xor_sync(0xffffffffu, x, o);
        return x;
    };
    auto add = [](float4 &o, const float4 &y, float f) { o.x = fmaf(y.x, f, o.x), o.y = fmaf(y.y, f, o.y), o.z = fmaf(y.z, f, o.z), o.w = fmaf(y.w, f, o.w); };
    static_assert(NW <= 16, "");
    const float *const beginnings = reinterpret_cast<const float *>(smem + G::kRing);
    int turn = 0;                                          // (chains one after the other, to different warps)
#pragma unroll 1
    for (uint32_t left = __ballot_sync(0xffffffffu, lane <= NW && s_part[max(min(lane, NW) - 1, 0)][lane == 0 ? 0 : 1].tiles >= 0); left; left &= left - 1) {
        const int c = __ffs(left) - 1, w0 = max(c - 1, 0), which = c == 0 ? 0 : 1;
        const Pair pt = s_part[w0][which];
        const int end = pt.begin + pt.tiles;
        const bool here = pt.begin >= first && end <= last;
        if (tid == 0 && !here) s_leaves[pt.begin >= first ? 1 : 0] = c;
        const bool has = sub16 < NW - w0 && (sub16 == 0 || s_first[w0 + sub16] < end);           // that warp has a part of it
        const int n = __popc(__ballot_sync(0xffffffffu, has)) / 2;
#pragma unroll 1
        for (int i0 = (warp >= turn ? warp - turn : warp - turn + NW) * 32; i0 < per; i0 += NT) {
            const uint32_t i = i0 + lane, col = i / (D / 4), el = i % (D / 4) * 4;          // (per is a multiple of 16: 16 threads are all there or none)
            const bool mine = i < (uint32_t)per;
            const float2 ml = mine && has ? s_ml[w0 + sub16][sub16 ? 0 : which][col] : make_float2(-INFINITY, 0.f);
            const float top = max16(ml.x), f = ex2(ml.x - (top == -INFINITY ? 0.f : top)), sum = sum16(ml.y * f);
            float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
            const float *y = which == 1 ? reinterpret_cast<const float *>(smem + w0 * G::kStages * G::kStageBytes) : beginnings + w0 * G::kPart;
#pragma unroll 2
            for (int w = 0; w < n; ++w) {
                const float fw = __shfl_sync(0xffffffffu, f, w, 16);
                if (mine) add(o, *reinterpret_cast<const float4 *>(y + col * RP + el), fw);
                y = beginnings + (w0 + w + 1) * G::kPart;
            }
            if (!mine) continue;
            if (here) {
                write_joined(pt.pair, col, el, top, sum, o);
            } else {
                const size_t slot = 2 * (size_t)blockIdx.x + (pt.begin >= first ? 1 : 0);
                __stcg(reinterpret_cast<float4 *>(a.ws_o + (slot * kMaxGroup + col) * D + el), o);
                if (el == 0) __stcg(a.ws_ml + slot * kMaxGroup + col, make_float2(top, sum));
            }
        }
        turn = min(turn + (per + 31) / 32, NW) % NW;
    }
    __syncthreads();
    // A pair that leaves the block (two at most: one that began before it, one that goes on behind it) has parts with the blocks b0 .. b1;
    // the last of them to arrive joins them, in their order.
    const bool leaves = s_leaves[0] >= 0 || s_leaves[1] >= 0;
    if (leaves && tid < 64 && lane == 0 && s_leaves[warp] >= 0) {
        const int c = s_leaves[warp];
        const Pair pt = s_part[max(c - 1, 0)][c == 0 ? 0 : 1];
        const Shares shares(s_shared[0], s_shared[1]);
        const int b0 = pt.begin >= first ? (int)blockIdx.x : shares.of(pt.begin) / NW;
        const int b1 = pt.begin + pt.tiles <= last ? (int)blockIdx.x : shares.of(pt.begin + pt.tiles - 1) / NW;
        uint32_t before;                               // (back to 0 with the last)
        asm volatile("atom.acq_rel.gpu.global.inc.u32 %0, [%1], %2;" : "=r"(before) : "l"(a.ws_count + b0), "r"((uint32_t)(b1 - b0)) : "memory");
        s_join[warp][0] = b0;
        s_join[warp][1] = before == (uint32_t)(b1 - b0) ? b1 - b0 + 1 : 0;
    }
    if (leaves) __syncthreads();
#pragma unroll 1
    for (int i0 = warp * 32; leaves && i0 < 2 * per; i0 += NT) {             // (both pairs at once)
        const uint32_t i = i0 + lane, which = i >= (uint32_t)per, it = i - which * per, col = it / (D / 4), el = it % (D / 4) * 4;
        const int c = i < 2u * per ? s_leaves[which] : -1, n_parts = c < 0 ? 0 : s_join[which][1];
        const int b0 = s_join[which][0];
        float top = -INFINITY, sum = 0.f;
        float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
        constexpr int kInFlight = 20;
#pragma unroll 1
        for (int p0 = 0; p0 < __reduce_max_sync(0xffffffffu, n_parts); p0 += kInFlight) {
            // part p's slot is 2 (b0 + p), of the first one more
            constexpr int kStep = 2 * kMaxGroup;
            const size_t row0 = (size_t)(b0 + p0) * kStep + col;
            const int first_too = p0 == 0 ? kMaxGroup : 0;
            float2 ml[2];
            float4 y[kInFlight];
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const int p = sub16 + 16 * u;
                ml[u] = p < kInFlight && p0 + p < n_parts ? __ldcg(a.ws_ml + row0 + p * kStep + (p == 0 ? first_too : 0)) : make_float2(-INFINITY, 0.f);
            }
            const float *from = a.ws_o + row0 * D + el;
#pragma unroll
            for (int p = 0; p < kInFlight; ++p) {
                y[p] = make_float4(0.f, 0.f, 0.f, 0.f);
                if (p0 + p < n_parts) y[p] = __ldcg(reinterpret_cast<const float4 *>(p == 0 ? from + first_too * D : from + p * (kStep * D)));
            }
            const float mx = fmaxf(top, max16(fmaxf(ml[0].x, ml[1].x))), ref = mx == -INFINITY ? 0.f : mx, f0 = ex2(top - ref);
            const float f[2] = {ex2(ml[0].x - ref), ex2(ml[1].x - ref)};
            sum = fmaf(sum, f0, sum16(fmaf(ml[0].y, f[0], ml[1].y * f[1])));
            o.x *= f0, o.y *= f0, o.z *= f0, o.w *= f0;
#pragma unroll
            for (int p = 0; p < kInFlight; ++p) add(o, y[p], __shfl_sync(0xffffffffu, f[p / 16], p % 16, 16));
            top = mx;
        }
        if (n_parts > 0) write_joined(s_part[max(c - 1, 0)][c == 0 ? 0 : 1].pair, col, el, top, sum, o);
    }
    empty_requests<D, NT, T>(a);
}

// Multiprocessors of the current device, 0 on failure.
int sm_count() {
    int dev = 0, n = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) {
        cudaGetLastError();
        return 0;
    }
    return n;
}
// Counters first: they keep their place whatever the head_dim.
constexpr size_t kCounterBytes = 4096;
size_t workspace_bytes(int sms, int D) { return kCounterBytes + (size_t)sms * 2 * kMaxGroup * (D * sizeof(float) + sizeof(float2)); }
bool misaligned(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15) != 0; }

template <int D, bool F4, int NQ, bool FOLD = false>
cudaError_t launch_decode(const Args &a, int sms, cudaStream_t st) {
    using G = Geo<D, F4, NQ>;
    auto kernel = a.page_size < G::kTile ? decode_attn_kernel<D, F4, NQ, true, FOLD> : decode_attn_kernel<D, F4, NQ, false, FOLD>;
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, G::kBytes);
    if (e != cudaSuccess) {
        cudaGetLastError();
        return e;
    }
    return launch_kernel(kernel, (unsigned)sms, G::kThreads, G::kBytes, st, true, a);
}

template <bool F4>
int32_t decode_attn(const tessera_model_cfg *cfg, const tessera_decode_desc *d, const void *k_pool, const void *v_pool, const void *q, void *out,
                    float *lse, void *workspace, int64_t bytes, void *stream) {
    std::string err;
    if (int32_t rc = check_decode(cfg, d, &err)) return api_set_error(rc, err);
    if (!std::isfinite(cfg->sm_scale)) return api_set_error(TESSERA_INVALID_ARG, "sm_scale must be finite");
    if (d->batch == 0) return TESSERA_OK;
    if (!k_pool || !v_pool || misaligned(k_pool) || misaligned(v_pool))
        return api_set_error(TESSERA_INVALID_ARG, "k_pool / v_pool must be non-null and 16-byte aligned");
    if (!q || !out || misaligned(q) || misaligned(out)) return api_set_error(TESSERA_INVALID_ARG, "q and out must be non-null and 16-byte aligned");
    const int D = cfg->head_dim, sms = sm_count();
    if (sms <= 0 || sms * sizeof(uint32_t) > kCounterBytes) return api_set_error(TESSERA_CUDA_ERROR, "no current device, or one of more than 1 024 multiprocessors");
    const size_t need = workspace_bytes(sms, D);
    if (!workspace || misaligned(workspace) || bytes < (int64_t)need)
        return api_set_error(TESSERA_INVALID_ARG, "workspace must be non-null, 16-byte aligned and of tessera_decode_workspace_bytes: " + std::to_string(need));
    char *ws = static_cast<char *>(workspace);
    const size_t o_ml = kCounterBytes + (size_t)sms * 2 * kMaxGroup * D * sizeof(float);
    const float scale = cfg->sm_scale != 0.f ? cfg->sm_scale : (float)(1.0 / std::sqrt((double)D));
    const int g = cfg->num_q_heads / cfg->num_kv_heads;
    const Args a{static_cast<const uint8_t *>(k_pool), static_cast<const uint8_t *>(v_pool), static_cast<const __nv_bfloat16 *>(q),
                 static_cast<__nv_bfloat16 *>(out), lse, d->block_table, d->seq_len, d->batch, d->max_pages, d->num_pool_pages, cfg->page_size,
                 cfg->num_q_heads, cfg->num_kv_heads, g, d->window, d->n_sink, scale * 1.4426950408889634f,
                 reinterpret_cast<uint32_t *>(ws), reinterpret_cast<float *>(ws + kCounterBytes), reinterpret_cast<float2 *>(ws + o_ml)};
    auto launch = D == 128 ? (F4 && g <= 4 ? launch_decode<128, F4, 1, F4> : g <= 8 ? launch_decode<128, F4, 1> : launch_decode<128, F4, 2>)
                           : (F4 && g <= 4 ? launch_decode<64, F4, 1, F4> : g <= 8 ? launch_decode<64, F4, 1> : launch_decode<64, F4, 2>);
    const cudaError_t e = launch(a, sms, static_cast<cudaStream_t>(stream));
    if (e != cudaSuccess) return api_set_error(TESSERA_CUDA_ERROR, std::string("decode attention launch: ") + cudaGetErrorName(e) + " (" + cudaGetErrorString(e) + ")");
    return TESSERA_OK;
}

}  // namespace
}  // namespace tessera

using namespace tessera;

extern "C" {

int32_t tessera_decode_workspace_bytes(const tessera_model_cfg *cfg, int64_t *bytes) {
    return guarded([&]() -> int32_t {
        if (!cfg || !bytes) return api_set_error(TESSERA_INVALID_ARG, "null cfg or bytes");
        *bytes = 0;
        if (cfg->head_dim != 64 && cfg->head_dim != 128) return api_set_error(TESSERA_UNSUPPORTED_SHAPE, "head_dim: only 64 and 128");
        const int sms = sm_count();
        if (sms <= 0) return api_set_error(TESSERA_CUDA_ERROR, "no current device");
        *bytes = (int64_t)workspace_bytes(sms, cfg->head_dim);
        return TESSERA_OK;
    });
}

int32_t tessera_decode_attn(const tessera_model_cfg *cfg, const tessera_decode_desc *desc, const void *k_pool, const void *v_pool, const void *q,
                            void *out, float *lse, void *workspace, int64_t workspace_bytes, void *stream) {
    return guarded([&] { return decode_attn<false>(cfg, desc, k_pool, v_pool, q, out, lse, workspace, workspace_bytes, stream); });
}

int32_t tessera_decode_attn_kv4(const tessera_model_cfg *cfg, const tessera_decode_desc *desc, const void *k_pool4, const void *v_pool4, const void *q,
                                void *out, float *lse, void *workspace, int64_t workspace_bytes, void *stream) {
    return guarded([&] { return decode_attn<true>(cfg, desc, k_pool4, v_pool4, q, out, lse, workspace, workspace_bytes, stream); });
}

}  // extern "C"
