// Attention of a decode step: one query token a request over its pages, 16-bit or 4-bit, with an optional sliding window
// and sinks.  (The paper stops at the first token; this reads the pages that a composed prompt leaves behind.)
//   out = sum over visible keys of p v / l,  p = exp2(scale log2(e) q.k - m),  l = sum p,
// one pass over K and V with a running reference m; scores, l and the accumulators in fp32, p rounded to bf16 as an operand.
//
// Bound by memory: a key and value of a head are 512 bytes at head_dim 128 (4-bit: 144) for 4 D g flops.  The g <= 16 query heads
// of a KV head are the narrow side of mma.sync m16n8k16: keys are the 16 rows, queries the 8 (or twice 8) columns, so a
// score tile is S^T = K Q^T and the output O^T += V^T P^T.  (tcgen05 wants 128 rows of queries; there are at most 16.)
//
// Work: the visible keys of every (request, KV head) are cut into units of 64; the units of the whole batch, in order, are
// shared out evenly to one thread block an SM, whatever the lengths.  Which they are only the device knows (lengths are
// device data, so that a captured step can be replayed as they grow): every block sums the requests' units itself.  A
// block's share may begin and end inside a pair; such parts go to the workspace and attn_join_kernel joins them, in order.
// Within a block, a warp takes stages of kStageKeys keys in turn, each through a ring of its own filled by cp.async, with its own
// m and l; warps meet only at the end of a pair's part.  A row that is not visible, past the end or on a page outside the pool is
// filled with zeros and never read, so what stands there does not matter.
#include <cmath>
#include <cstring>
#include <string>

#include <cuda_bf16.h>
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

constexpr int kUnit = kDecodeUnit;
constexpr int kMaxGroup = 16;

struct Args {
    const uint8_t *k, *v;
    const __nv_bfloat16 *q;
    __nv_bfloat16 *out;
    float *lse;
    const int32_t *table, *seq_len;
    int batch, max_pages, num_pool_pages, page_size, H_q, H_kv, g, window, n_sink;
    float scale_log2;
    float *ws_o;          // [2 grid][16][D] parts: block b's first part at 2 b if its pair began before, its last at 2 b + 1 if its pair goes on
    float2 *ws_ml;        // [2 grid][16] reference (log2 units) and sum
    int2 *ws_join;        // [grid] the pair that begins in block b and goes on, and how many blocks have a part of it; -1: none
};

// Shared memory of a stage: kStageKeys rows of K, of V and (4-bit) their numbers.
template <int D, bool F4, int NQ> struct Geo {
    static constexpr int kWarps = F4 && NQ == 1 ? 16 : 8;
    static constexpr int kThreads = 32 * kWarps;
    static constexpr int kStages = 3;
    static constexpr int kStageKeys = F4 || D == 64 ? 32 : 16;
    static constexpr int kRow = F4 ? D / 2 : 2 * D;                       // bytes of a row of K or V
    static constexpr int kStageBytes = 2 * kStageKeys * (kRow + (F4 ? 8 : 0));
    static constexpr int kRing = kWarps * kStages * kStageBytes;
};

__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
template <int N> __device__ __forceinline__ void cp_async(uint32_t dst, const void *src, bool there) {
    if constexpr (N == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(there ? 16 : 0) : "memory");
    else asm volatile("cp.async.ca.shared.global [%0], [%1], 8, %2;" ::"r"(dst), "l"(src), "r"(there ? 8 : 0) : "memory");
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
// Four-bit codes at bits 0-3 and 16-19 -> two bf16 numbers 128 + c: the code is the mantissa's last four bits.
__device__ __forceinline__ uint32_t codes_128(uint32_t w) {
    uint32_t r;
    asm("lop3.b32 %0, %1, 0x000f000f, 0x43004300, 0xea;" : "=r"(r) : "r"(w));     // (w & mask) | bits
    return r;
}
// ... -> c - 8, exact.
__device__ __forceinline__ uint32_t codes_centred(uint32_t w) {
    const uint32_t x = codes_128(w), mid = 0x43084308u;                            // 136
    const __nv_bfloat162 y = __hsub2(*reinterpret_cast<const __nv_bfloat162 *>(&x), *reinterpret_cast<const __nv_bfloat162 *>(&mid));
    return *reinterpret_cast<const uint32_t *>(&y);
}

// A request's visible keys: n of them, the first `sinks` at the front and the others `shift` further on.
struct Visible { int n, sinks, shift; };
__device__ __forceinline__ Visible visible(int len, const Args &a) {
    len = min(len, a.max_pages * a.page_size);
    if (len <= 0) return {0, 0, 0};
    if (a.window == 0 || len <= a.window) return {len, 0, 0};
    const int first = len - a.window, sinks = min(a.n_sink, first);
    return {sinks + a.window, sinks, first - sinks};
}
__device__ __forceinline__ int units_of(int len, const Args &a) { return (visible(len, a).n + kUnit - 1) / kUnit; }

// Where in the batch a unit lies: request, units of the requests before it.
struct Start { int request, before; };

// A block's share [x, y) of all z units, and where it starts.  (No more blocks than units take part, so that every block between
// a pair's first and last has a part of it.)  Sums run over the batch in chunks of a block's threads.
template <int NT>
__device__ __forceinline__ int3 share(const Args &a, Start *s_start, int *s_sum) {
    const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32;
    constexpr int W = NT / 32;
    auto scan = [&](int x, int &total) {              // inclusive prefix sum over the block's threads
#pragma unroll
        for (int o = 1; o < 32; o *= 2) {
            const int y = __shfl_up_sync(0xffffffffu, x, o);
            if (lane >= o) x += y;
        }
        __syncthreads();                              // (of an earlier use)
        if (lane == 31) s_sum[warp] = x;
        __syncthreads();
        int before = 0, all = 0;
#pragma unroll
        for (int w = 0; w < W; ++w) {
            const int n = s_sum[w];
            before += w < warp ? n : 0;
            all += n;
        }
        total = all;
        return x + before;
    };
    auto load = [&](int r) { return r < a.batch ? a.H_kv * units_of(a.seq_len[r], a) : 0; };
    int all = 0, chunk, own = load(tid), end = scan(own, chunk);
    all = chunk;
    for (int r0 = NT; r0 < a.batch; r0 += NT) {
        int n;
        scan(load(r0 + tid), n);
        all += n;
    }
    const int blocks = min((int)gridDim.x, all);
    if ((int)blockIdx.x >= blocks) return make_int3(0, 0, all);
    const int first = (int)((int64_t)all * blockIdx.x / blocks), last = (int)((int64_t)all * (blockIdx.x + 1) / blocks);
    int before = 0;
    for (int r0 = 0; r0 < a.batch; r0 += NT) {
        if (r0 > 0) {
            own = load(r0 + tid);
            end = scan(own, chunk);
        }
        if (before + end - own <= first && first < before + end) *s_start = {r0 + tid, before + end - own};
        before += chunk;
        if (before > first) break;
    }
    __syncthreads();
    return make_int3(first, last, all);
}

template <int D, bool F4, int NQ>
__global__ void __launch_bounds__(Geo<D, F4, NQ>::kThreads, 1)
decode_attn_kernel(const __grid_constant__ Args a) {
    using G = Geo<D, F4, NQ>;
    constexpr int SK = G::kStageKeys, NW = G::kWarps, NT = G::kThreads, CPR = G::kRow / 16, Q8 = 8 * NQ;
    extern __shared__ __align__(128) uint8_t smem[];
    __shared__ float2 s_ml[NW][Q8];
    __shared__ uint32_t s_valid[NW][G::kStages];
    __shared__ Start s_start;
    __shared__ int s_sum[NW];
    const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32, quad = lane / 4, t = lane % 4;
    const int page_shift = __ffs(a.page_size) - 1;
    grid_wait();
    grid_release();

    // requests without a key
    for (int r = blockIdx.x; r < a.batch; r += gridDim.x)
        if (visible(a.seq_len[r], a).n == 0) {
            for (int i = tid; i < a.H_q * D / 8; i += NT) stg(reinterpret_cast<uint4 *>(a.out + (size_t)r * a.H_q * D) + i, make_uint4(0, 0, 0, 0));
            if (a.lse)
                for (int i = tid; i < a.H_q; i += NT) a.lse[(size_t)r * a.H_q + i] = -INFINITY;
        }

    const int3 mine = share<NT>(a, &s_start, s_sum);
    if (tid == 0) a.ws_join[blockIdx.x] = make_int2(-1, -1);
    if (mine.x >= mine.y) return;
    int r = s_start.request, base = s_start.before;
    const uint32_t ring = ptx::smem_u32(smem) + warp * G::kStages * G::kStageBytes;

    for (int u = mine.x; u < mine.y;) {
        const Visible vis = visible(a.seq_len[r], a);
        const int nu = (vis.n + kUnit - 1) / kUnit;
        if (nu == 0 || u - base >= nu * a.H_kv) {          // on to the next request
            base += nu * a.H_kv;
            ++r;
            continue;
        }
        const int h = (u - base) / nu, j0 = (u - base) % nu, j1 = min(nu, j0 + mine.y - u);
        const int v0 = j0 * kUnit, v1 = min(vis.n, j1 * kUnit);            // visible keys of this part
        const int n_stages = (v1 - v0 + SK - 1) / SK, my_stages = n_stages > warp ? (n_stages - warp + NW - 1) / NW : 0;
        const int32_t *table = a.table + (size_t)r * a.max_pages;

        // slot of visible key v, -1 where there is none
        auto slot_of = [&](int v) {
            if (v >= v1) return -1;
            const int key = v < vis.sinks ? v : v + vis.shift;
            const int page = table[key >> page_shift];
            return page >= 0 && page < a.num_pool_pages ? (page << page_shift) + (key & (a.page_size - 1)) : -1;
        };
        auto stage_key = [&](int s) { return v0 + (warp + s * NW) * SK; };      // of the warp's s-th stage
        int next_slot = my_stages > 0 ? slot_of(stage_key(0) + lane % SK) : -1;
        auto fetch = [&](int s) {
            if (s < my_stages) {
                const int slot = next_slot, at = s % G::kStages;
                if (s + 1 < my_stages) next_slot = slot_of(stage_key(s + 1) + lane % SK);      // (its page id comes in while this stage is sent for)
                const uint32_t valid = __ballot_sync(0xffffffffu, slot >= 0);
                if (lane == 0) s_valid[warp][at] = valid;
                const uint32_t kb = ring + at * G::kStageBytes, vb = kb + SK * G::kRow;
#pragma unroll
                for (int i = 0; i < SK * CPR / 32; ++i) {
                    const int idx = i * 32 + lane, row = idx / CPR, c = idx % CPR;
                    const int sl = __shfl_sync(0xffffffffu, slot, row);
                    const bool there = sl >= 0;
                    const int s0 = there ? sl : 0;
                    if constexpr (F4) {
                        const size_t o = codes4_at<D>((size_t)(s0 >> page_shift), s0 & (a.page_size - 1), h, a.page_size, a.H_kv) + c * 16;
                        cp_async<16>(kb + row * G::kRow + c * 16, a.k + o, there);
                        // (the two 16-byte pieces of a 32-byte stretch stay side by side; rows 4-7 of 8 change places by halves, so that the
                        // four rows and eight columns that a warp's lanes ask for at once lie in different banks)
                        const int cv = D == 128 ? c ^ (((row >> 2) & 1) << 1) : c;
                        cp_async<16>(vb + row * G::kRow + cv * 16, a.v + o, there);
                    } else {
                        const size_t o = ((size_t)s0 * a.H_kv + h) * G::kRow + c * 16;
                        const int cs = c ^ (row & 7);
                        cp_async<16>(kb + row * G::kRow + cs * 16, a.k + o, there);
                        cp_async<16>(vb + row * G::kRow + cs * 16, a.v + o, there);
                    }
                }
                if constexpr (F4) {
                    const bool there = slot >= 0;
                    const int s0 = there ? slot : 0;
                    const size_t o = params4_at<D>((size_t)(s0 >> page_shift), s0 & (a.page_size - 1), h, a.page_size, a.H_kv);
                    cp_async<8>(vb + SK * G::kRow + lane * 8, a.k + o, there);
                    cp_async<8>(vb + SK * G::kRow + SK * 8 + lane * 8, a.v + o, there);
                }
            }
            cp_commit();
        };
#pragma unroll
        for (int s = 0; s < G::kStages - 1; ++s) fetch(s);

        // Q^T as the MMA's second operand: column quad (+ 8) is a query, rows go over head_dim - in natural order, respectively
        // in the order in which a lane's codes come (elements 16 t + 4 w + {0, 2}, {1, 3} of each half).
        constexpr int KS = D / 16;
        uint32_t qf[NQ][KS][2];
        float q_sum[NQ][2][2];           // 4-bit: sums of q over each half, of columns 2 t and 2 t + 1
#pragma unroll
        for (int n = 0; n < NQ; ++n) {
            const int col = n * 8 + quad;
            const bool there = col < a.g;
            const __nv_bfloat16 *q = a.q + ((size_t)r * a.H_q + h * a.g + (there ? col : 0)) * D;
            if constexpr (F4) {
                float sum[2] = {0.f, 0.f};
#pragma unroll
                for (int half = 0; half < 2; ++half)
#pragma unroll
                    for (int w = 0; w < KS / 2; ++w) {
                        const uint2 x = there ? *reinterpret_cast<const uint2 *>(q + half * (D / 2) + (D / 8) * t + 4 * w) : make_uint2(0, 0);
                        qf[n][half * (KS / 2) + w][0] = __byte_perm(x.x, x.y, 0x5410);
                        qf[n][half * (KS / 2) + w][1] = __byte_perm(x.x, x.y, 0x7632);
                        sum[half] += (__uint_as_float(x.x << 16) + __uint_as_float(x.x & 0xffff0000u)) + (__uint_as_float(x.y << 16) + __uint_as_float(x.y & 0xffff0000u));
                    }
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    float s = sum[half];
                    s += __shfl_xor_sync(0xffffffffu, s, 1);
                    s += __shfl_xor_sync(0xffffffffu, s, 2);
                    q_sum[n][half][0] = __shfl_sync(0xffffffffu, s, 8 * t);           // of column 2 t: lane 4 (2 t)
                    q_sum[n][half][1] = __shfl_sync(0xffffffffu, s, 8 * t + 4);
                }
            } else {
#pragma unroll
                for (int s = 0; s < KS; ++s)
#pragma unroll
                    for (int i = 0; i < 2; ++i) qf[n][s][i] = there ? *reinterpret_cast<const uint32_t *>(q + 16 * s + 8 * i + 2 * t) : 0u;
            }
        }

        float m[NQ][2], l[NQ][2], off[NQ][2][2];         // off (4-bit): sums of p times a half's middle value
        float acc[NQ][D / 16][4];
#pragma unroll
        for (int n = 0; n < NQ; ++n) {
#pragma unroll
            for (int e = 0; e < 2; ++e) m[n][e] = -INFINITY, l[n][e] = off[n][0][e] = off[n][1][e] = 0.f;
#pragma unroll
            for (int d = 0; d < D / 16; ++d)
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[n][d][e] = 0.f;
        }

        for (int s = 0; s < my_stages; ++s) {
            cp_wait<G::kStages - 2>();
            __syncwarp();
            fetch(s + G::kStages - 1);                    // into the stage consumed in the last turn
            const int at = s % G::kStages;
            const uint32_t valid = s_valid[warp][at];
            const uint32_t kb = ring + at * G::kStageBytes, vb = kb + SK * G::kRow;
#pragma unroll
            for (int sub = 0; sub < SK / 16; ++sub) {
                // rows of the score tile: natural keys of the 16, 4-bit: row i is key i ^ (i / 2 % 2) (see the bank note above)
                const int row0 = sub * 16 + (F4 ? quad ^ ((quad >> 1) & 1) : quad);
                float sc[NQ][4];
                float kp[2][4];
                if constexpr (F4) {
                    float part[NQ][2][4];
#pragma unroll
                    for (int n = 0; n < NQ; ++n)
#pragma unroll
                        for (int half = 0; half < 2; ++half)
#pragma unroll
                            for (int e = 0; e < 4; ++e) part[n][half][e] = -136.f * q_sum[n][half][e & 1];
                    uint32_t w[2][D / 32];               // 16 (8) bytes of rows row0 and row0 + 8
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        const uint8_t *p = smem + (kb - ptx::smem_u32(smem)) + (row0 + 8 * i) * G::kRow + (D / 8) * t;
                        if constexpr (D == 128) *reinterpret_cast<uint4 *>(w[i]) = *reinterpret_cast<const uint4 *>(p);
                        else *reinterpret_cast<uint2 *>(w[i]) = *reinterpret_cast<const uint2 *>(p);
                        const uint2 pr = *reinterpret_cast<const uint2 *>(smem + (vb - ptx::smem_u32(smem)) + SK * G::kRow + (row0 + 8 * i) * 8);
                        kp[i][0] = __uint_as_float(pr.x << 16);
                        kp[i][1] = fmaf(8.f, kp[i][0], __uint_as_float(pr.x & 0xffff0000u));
                        kp[i][2] = __uint_as_float(pr.y << 16);
                        kp[i][3] = fmaf(8.f, kp[i][2], __uint_as_float(pr.y & 0xffff0000u));
                    }
#pragma unroll
                    for (int x = 0; x < D / 32; ++x)
#pragma unroll
                        for (int half = 0; half < 2; ++half) {
                            const int sh = 4 * half;
                            const uint32_t f[4] = {codes_128(w[0][x] >> sh), codes_128(w[1][x] >> sh), codes_128(w[0][x] >> (sh + 8)), codes_128(w[1][x] >> (sh + 8))};
#pragma unroll
                            for (int n = 0; n < NQ; ++n) mma(part[n][half], f, qf[n][half * (KS / 2) + x][0], qf[n][half * (KS / 2) + x][1]);
                        }
                    // q.k = sum over the halves of s (q.(c - 8)) + (m + 8 s) sum q
#pragma unroll
                    for (int n = 0; n < NQ; ++n)
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const int i = e >> 1;
                            sc[n][e] = fmaf(kp[i][0], part[n][0][e], fmaf(kp[i][1], q_sum[n][0][e & 1], fmaf(kp[i][2], part[n][1][e], kp[i][3] * q_sum[n][1][e & 1])));
                        }
                } else {
#pragma unroll
                    for (int n = 0; n < NQ; ++n)
#pragma unroll
                        for (int e = 0; e < 4; ++e) sc[n][e] = 0.f;
                    const int lr = sub * 16 + (lane & 15);            // lanes 0-15: rows, first 8 columns; 16-31: next 8
#pragma unroll
                    for (int ks = 0; ks < KS; ++ks) {
                        uint32_t f[4];
                        ldmatrix_x4(f, kb + lr * G::kRow + (((2 * ks + (lane >> 4)) ^ (lr & 7)) << 4));
#pragma unroll
                        for (int n = 0; n < NQ; ++n) mma(sc[n], f, qf[n][ks][0], qf[n][ks][1]);
                    }
                }
                const bool here[2] = {((valid >> row0) & 1) != 0, ((valid >> (row0 + 8)) & 1) != 0};
                bool low = true;                      // every score is at most 2^8 above its column's reference
#pragma unroll
                for (int n = 0; n < NQ; ++n)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        sc[n][e] = here[e >> 1] ? sc[n][e] * a.scale_log2 : -INFINITY;
                        low = low && (sc[n][e] <= m[n][e & 1] + 8.f || sc[n][e] == -INFINITY);
                    }
                // The reference moves only where a score would go far above it (and at the first keys): then to the columns' true
                // maxima, the lanes of a column together.
                if (!__all_sync(0xffffffffu, low)) {
#pragma unroll
                    for (int n = 0; n < NQ; ++n)
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            float top = fmaxf(sc[n][e], sc[n][e + 2]);
                            top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 4));
                            top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 8));
                            top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 16));
                            const float mn = fmaxf(m[n][e], top), f = mn == -INFINITY ? 1.f : ex2(m[n][e] - mn);
                            m[n][e] = mn;
                            l[n][e] *= f;
                            off[n][0][e] *= f;
                            off[n][1][e] *= f;
#pragma unroll
                            for (int d = 0; d < D / 16; ++d) acc[n][d][e] *= f, acc[n][d][e + 2] *= f;
                        }
                }
                float p[NQ][4];
#pragma unroll
                for (int n = 0; n < NQ; ++n)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float ref = m[n][e & 1] == -INFINITY ? 0.f : m[n][e & 1];
                        p[n][e] = ex2(sc[n][e] - ref);
                        l[n][e & 1] += p[n][e];
                    }
                if constexpr (F4) {
                    float vp[2][4];
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        const uint2 pr = *reinterpret_cast<const uint2 *>(smem + (vb - ptx::smem_u32(smem)) + SK * G::kRow + SK * 8 + (row0 + 8 * i) * 8);
                        vp[i][0] = __uint_as_float(pr.x << 16);
                        vp[i][1] = fmaf(8.f, vp[i][0], __uint_as_float(pr.x & 0xffff0000u));
                        vp[i][2] = __uint_as_float(pr.y << 16);
                        vp[i][3] = fmaf(8.f, vp[i][2], __uint_as_float(pr.y & 0xffff0000u));
                    }
                    // sum p v = sum (p s) (c - 8) + sum p (m + 8 s), half by half: p s is the MMA's operand, rounded to bf16
                    uint32_t b[NQ][2][2];
#pragma unroll
                    for (int n = 0; n < NQ; ++n)
#pragma unroll
                        for (int half = 0; half < 2; ++half)
#pragma unroll
                            for (int i = 0; i < 2; ++i) {
                                b[n][half][i] = transposed(pack_bf16(p[n][2 * i] * vp[i][2 * half], p[n][2 * i + 1] * vp[i][2 * half]));
#pragma unroll
                                for (int e = 0; e < 2; ++e) off[n][half][e] = fmaf(p[n][2 * i + e], vp[i][2 * half + 1], off[n][half][e]);
                            }
                    // keys of operand rows 2 t, 2 t + 1, 2 t + 8, 2 t + 9, and of each the bytes whose elements this lane's rows of V^T are
                    uint32_t w[4][D / 64];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int op = 2 * t + (i & 1), row = sub * 16 + (i >> 1) * 8 + (op ^ ((op >> 1) & 1));
                        const uint8_t *p8 = smem + (vb - ptx::smem_u32(smem)) + row * G::kRow;
                        if constexpr (D == 128) *reinterpret_cast<uint2 *>(w[i]) = *reinterpret_cast<const uint2 *>(p8 + ((quad * 8) ^ (((row >> 2) & 1) << 5)));
                        else w[i][0] = *reinterpret_cast<const uint32_t *>(p8 + quad * 4);
                    }
#pragma unroll
                    for (int x = 0; x < D / 64; ++x)
#pragma unroll
                        for (int jp = 0; jp < 2; ++jp) {
                            uint32_t pr[2][2];                // byte 2 jp + j of two keys, keys 2 i and 2 i + 1
#pragma unroll
                            for (int j = 0; j < 2; ++j)
#pragma unroll
                                for (int i = 0; i < 2; ++i) pr[j][i] = __byte_perm(w[2 * i][x], w[2 * i + 1][x], 0x0400 + (2 * jp + j) * 0x0101 + 0x0000);
#pragma unroll
                            for (int half = 0; half < 2; ++half) {
                                const int sh = 4 * half;
                                const uint32_t f[4] = {codes_centred(pr[0][0] >> sh), codes_centred(pr[1][0] >> sh), codes_centred(pr[0][1] >> sh), codes_centred(pr[1][1] >> sh)};
#pragma unroll
                                for (int n = 0; n < NQ; ++n) mma(acc[n][(half * (D / 64) + x) * 2 + jp], f, b[n][half][0], b[n][half][1]);
                            }
                        }
                } else {
                    uint32_t b[NQ][2];
#pragma unroll
                    for (int n = 0; n < NQ; ++n)
#pragma unroll
                        for (int i = 0; i < 2; ++i) b[n][i] = transposed(pack_bf16(p[n][2 * i], p[n][2 * i + 1]));
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
        }

        // The warps' parts meet in shared memory (nothing is on its way into the ring any more).
        cp_wait<0>();
        __syncthreads();
        float *so = reinterpret_cast<float *>(smem) + warp * Q8 * D;
#pragma unroll
        for (int n = 0; n < NQ; ++n)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                auto column_sum = [](float x) {
                    x += __shfl_xor_sync(0xffffffffu, x, 4);
                    x += __shfl_xor_sync(0xffffffffu, x, 8);
                    return x + __shfl_xor_sync(0xffffffffu, x, 16);
                };
                const float sum = column_sum(l[n][e]);
                const float o0 = F4 ? column_sum(off[n][0][e]) : 0.f, o1 = F4 ? column_sum(off[n][1][e]) : 0.f;
                const int col = n * 8 + 2 * t + e;
                if (quad == 0) s_ml[warp][col] = make_float2(m[n][e], sum);
#pragma unroll
                for (int d = 0; d < D / 16; ++d)
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        // element of head_dim that row quad + 8 i of tile d is
                        int el = 16 * d + 8 * i + quad;
                        float y = acc[n][d][e + 2 * i];
                        if constexpr (F4) {
                            const int half = d / (D / 32), x = d / 2 % (D / 64), jp = d % 2;
                            el = half * (D / 2) + (D / 16) * quad + 4 * x + 2 * jp + i;
                            y += half ? o1 : o0;
                        }
                        so[col * D + el] = y;
                    }
            }
        __syncthreads();
        const bool whole = j0 == 0 && j1 == nu, begins = j0 == 0;
        const size_t slot = 2 * (size_t)blockIdx.x + (begins ? 1 : 0);
        for (int i = tid; i < a.g * (D / 4); i += NT) {
            const int col = i / (D / 4), el = i % (D / 4) * 4;
            float top = -INFINITY;
#pragma unroll
            for (int w = 0; w < NW; ++w) top = fmaxf(top, s_ml[w][col].x);
            const float ref = top == -INFINITY ? 0.f : top;
            float sum = 0.f;
            float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int w = 0; w < NW; ++w) {
                const float2 ml = s_ml[w][col];
                const float f = exp2f(ml.x - ref);
                const float4 y = *reinterpret_cast<const float4 *>(reinterpret_cast<const float *>(smem) + (w * Q8 + col) * D + el);
                sum = fmaf(ml.y, f, sum);
                o.x = fmaf(y.x, f, o.x), o.y = fmaf(y.y, f, o.y), o.z = fmaf(y.z, f, o.z), o.w = fmaf(y.w, f, o.w);
            }
            if (whole) {
                const float inv = top == -INFINITY ? 0.f : 1.f / sum;
                const size_t head = (size_t)r * a.H_q + h * a.g + col;
                *reinterpret_cast<uint2 *>(a.out + head * D + el) = make_uint2(pack_bf16(o.x * inv, o.y * inv), pack_bf16(o.z * inv, o.w * inv));
                if (a.lse && el == 0) a.lse[head] = top == -INFINITY ? -INFINITY : (top + log2f(sum)) * 0.6931471805599453f;
            } else {
                *reinterpret_cast<float4 *>(a.ws_o + (slot * kMaxGroup + col) * D + el) = o;
                if (el == 0) a.ws_ml[slot * kMaxGroup + col] = make_float2(top, sum);
            }
        }
        if (tid == 0 && begins && !whole) {
            // block b has the units from all b / blocks on (rounded down), so unit x is with block ((x + 1) blocks - 1) / all
            const int blocks = min((int)gridDim.x, mine.z);
            const int last = (int)((((int64_t)u + nu) * blocks - 1) / mine.z);
            a.ws_join[blockIdx.x] = make_int2(r * a.H_kv + h, last - (int)blockIdx.x + 1);
        }
        __syncthreads();                   // the ring is free for the next part
        u += j1 - j0;
    }
}

// Joins the parts of the pair that begins in block b and ends in another, in order: O = sum O_i 2^(m_i - m) / sum l_i 2^(m_i - m).
template <int D>
__global__ void __launch_bounds__(256)
attn_join_kernel(const __grid_constant__ Args a) {
    grid_wait();
    grid_release();
    const int b = blockIdx.x;
    const int2 join = a.ws_join[b];
    if (join.x < 0) return;
    const int r = join.x / a.H_kv, h = join.x % a.H_kv, n_parts = join.y;
    auto slot_of = [&](int i) { return i == 0 ? 2 * (size_t)b + 1 : 2 * (size_t)(b + i); };
    for (int i = threadIdx.x; i < a.g * (D / 4); i += 256) {
        const int col = i / (D / 4), el = i % (D / 4) * 4;
        float top = -INFINITY, sum = 0.f;
        float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
        constexpr int kBatch = 8;
        for (int p0 = 0; p0 < n_parts; p0 += kBatch) {
            float2 ml[kBatch];
            float4 y[kBatch];
#pragma unroll
            for (int p = 0; p < kBatch; ++p) {
                const bool there = p0 + p < n_parts;
                const size_t slot = slot_of(there ? p0 + p : 0);
                ml[p] = there ? __ldcg(a.ws_ml + slot * kMaxGroup + col) : make_float2(-INFINITY, 0.f);
                y[p] = __ldcg(reinterpret_cast<const float4 *>(a.ws_o + (slot * kMaxGroup + col) * D + el));
            }
            float m = top;
#pragma unroll
            for (int p = 0; p < kBatch; ++p) m = fmaxf(m, ml[p].x);
            const float ref = m == -INFINITY ? 0.f : m, f0 = exp2f(top - ref);
            sum *= f0;
            o.x *= f0, o.y *= f0, o.z *= f0, o.w *= f0;
#pragma unroll
            for (int p = 0; p < kBatch; ++p) {
                if (p0 + p >= n_parts) continue;
                const float f = exp2f(ml[p].x - ref);
                sum = fmaf(ml[p].y, f, sum);
                o.x = fmaf(y[p].x, f, o.x), o.y = fmaf(y[p].y, f, o.y), o.z = fmaf(y[p].z, f, o.z), o.w = fmaf(y[p].w, f, o.w);
            }
            top = m;
        }
        const float inv = top == -INFINITY ? 0.f : 1.f / sum;
        const size_t head = (size_t)r * a.H_q + h * a.g + col;
        *reinterpret_cast<uint2 *>(a.out + head * D + el) = make_uint2(pack_bf16(o.x * inv, o.y * inv), pack_bf16(o.z * inv, o.w * inv));
        if (a.lse && el == 0) a.lse[head] = top == -INFINITY ? -INFINITY : (top + log2f(sum)) * 0.6931471805599453f;
    }
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
size_t workspace_bytes(int sms, int D) {
    return (size_t)sms * (2 * kMaxGroup * (D * sizeof(float) + sizeof(float2)) + sizeof(int2));
}
bool misaligned(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15) != 0; }

template <int D, bool F4, int NQ>
cudaError_t launch_decode(const Args &a, int sms, cudaStream_t st) {
    using G = Geo<D, F4, NQ>;
    static_assert(G::kRing >= G::kWarps * 8 * NQ * D * 4, "the warps' parts meet in the ring");
    const cudaError_t e = cudaFuncSetAttribute(decode_attn_kernel<D, F4, NQ>, cudaFuncAttributeMaxDynamicSharedMemorySize, G::kRing);
    if (e != cudaSuccess) {
        cudaGetLastError();
        return e;
    }
    const cudaError_t f = launch_kernel(decode_attn_kernel<D, F4, NQ>, (unsigned)sms, G::kThreads, G::kRing, st, true, a);
    return f != cudaSuccess ? f : launch_kernel(attn_join_kernel<D>, (unsigned)sms, 256, 0, st, true, a);
}

template <bool F4>
int32_t decode_attn(const tessera_model_cfg *cfg, const tessera_decode_desc *d, const void *k_pool, const void *v_pool, const void *q, void *out,
                    float *lse, void *workspace, int64_t bytes, void *stream) {
    std::string err;
    if (int32_t rc = check_decode(cfg, d, &err)) return api_set_error(rc, err);
    if (d->batch == 0) return TESSERA_OK;
    if (!k_pool || !v_pool || misaligned(k_pool) || misaligned(v_pool))
        return api_set_error(TESSERA_INVALID_ARG, "k_pool / v_pool must be non-null and 16-byte aligned");
    if (!q || !out || misaligned(q) || misaligned(out)) return api_set_error(TESSERA_INVALID_ARG, "q and out must be non-null and 16-byte aligned");
    const int D = cfg->head_dim, sms = sm_count();
    if (sms <= 0) return api_set_error(TESSERA_CUDA_ERROR, "no current device");
    const size_t need = workspace_bytes(sms, D);
    if (!workspace || misaligned(workspace) || bytes < (int64_t)need)
        return api_set_error(TESSERA_INVALID_ARG, "workspace must be non-null, 16-byte aligned and of tessera_decode_workspace_bytes: " + std::to_string(need));
    char *ws = static_cast<char *>(workspace);
    const size_t o_ml = (size_t)sms * 2 * kMaxGroup * D * sizeof(float), o_join = o_ml + (size_t)sms * 2 * kMaxGroup * sizeof(float2);
    const float scale = cfg->sm_scale != 0.f ? cfg->sm_scale : (float)(1.0 / std::sqrt((double)D));
    const int g = cfg->num_q_heads / cfg->num_kv_heads;
    const Args a{static_cast<const uint8_t *>(k_pool), static_cast<const uint8_t *>(v_pool), static_cast<const __nv_bfloat16 *>(q),
                 static_cast<__nv_bfloat16 *>(out), lse, d->block_table, d->seq_len, d->batch, d->max_pages, d->num_pool_pages, cfg->page_size,
                 cfg->num_q_heads, cfg->num_kv_heads, g, d->window, d->n_sink, scale * 1.4426950408889634f,
                 reinterpret_cast<float *>(ws), reinterpret_cast<float2 *>(ws + o_ml), reinterpret_cast<int2 *>(ws + o_join)};
    auto launch = D == 128 ? (g <= 8 ? launch_decode<128, F4, 1> : launch_decode<128, F4, 2>) : (g <= 8 ? launch_decode<64, F4, 1> : launch_decode<64, F4, 2>);
    const cudaError_t e = launch(a, sms, static_cast<cudaStream_t>(stream));
    if (e != cudaSuccess) return api_set_error(TESSERA_CUDA_ERROR, std::string("decode attention launch: ") + cudaGetErrorName(e) + " (" + cudaGetErrorString(e) + ")");
    return TESSERA_OK;
}

}  // namespace
}  // namespace tessera

using namespace tessera;

extern "C" {

int32_t tessera_decode_workspace_bytes(const tessera_model_cfg *cfg, int64_t *bytes) {
    if (!cfg || !bytes) return api_set_error(TESSERA_INVALID_ARG, "null cfg or bytes");
    *bytes = 0;
    if (cfg->head_dim != 64 && cfg->head_dim != 128) return api_set_error(TESSERA_UNSUPPORTED_SHAPE, "head_dim: only 64 and 128");
    const int sms = sm_count();
    if (sms <= 0) return api_set_error(TESSERA_CUDA_ERROR, "no current device");
    *bytes = (int64_t)workspace_bytes(sms, cfg->head_dim);
    return TESSERA_OK;
}

int32_t tessera_decode_attn(const tessera_model_cfg *cfg, const tessera_decode_desc *desc, const void *k_pool, const void *v_pool, const void *q,
                            void *out, float *lse, void *workspace, int64_t workspace_bytes, void *stream) {
    return decode_attn<false>(cfg, desc, k_pool, v_pool, q, out, lse, workspace, workspace_bytes, stream);
}

int32_t tessera_decode_attn_kv4(const tessera_model_cfg *cfg, const tessera_decode_desc *desc, const void *k_pool4, const void *v_pool4, const void *q,
                                void *out, float *lse, void *workspace, int64_t workspace_bytes, void *stream) {
    return decode_attn<true>(cfg, desc, k_pool4, v_pool4, q, out, lse, workspace, workspace_bytes, stream);
}

}  // extern "C"
