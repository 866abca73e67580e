// Fresh rows of layers that normalise q and k per head: norm, rotation and the writes to the pages in one pass, for a
// plan's recompute rows (Sec. 5.3 "Completing prefill") and for the one new token of every request of a decode step.
//   y = w x / sqrt(mean over the head of x^2 + eps),  y' = R(position) y,  one round-to-nearest-even to bf16
// in fp32 throughout (angle, cosine and sine in fp64).  The paper's models normalise nothing per head; with null weights this
// is the arithmetic of tessera_extend_write.
//
// A thread holds 8 elements of a head and the 8 that lie D/2 later, so rotary pairs need no exchange and the sum of squares
// is three shuffles (two at head_dim 64) among the head's neighbouring threads.  HBM-bound: every row is read and written once.
// 59 816 rows of 64 + 2 x 8 heads (2.45 GB): 409 to 431 us (boxes) = 5 990 to 5 680 GB/s, 92 to 87 % of a copy, with two tasks in flight
// a thread and three blocks an SM (on the box of the 409 four tasks and two blocks took 450, two and four 408 with spills, more blocks
// 770 to 950).  A decode step's write is latency: 2.4 us for 8 requests.
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

namespace tessera {

int32_t api_set_error(int32_t code, const std::string &msg);

namespace {

// tessera_fresh_rows as the kernels take it: row strides in 16-byte chunks.
struct Fresh {
    const uint4 *q, *k, *v;
    uint4 *q_out;
    int64_t q_row, k_row, v_row;
    const uint4 *q_weight, *k_weight;
    float eps;
};

// One head's chunk pair: normalised (when w is not null) in fp32.  All threads of the head call it together.
template <int D>
__device__ __forceinline__ void norm_chunks(float (&lo)[8], float (&hi)[8], const uint4 *w, int c, float eps) {
    if (!w) return;
    float ss = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) ss = fmaf(lo[i], lo[i], fmaf(hi[i], hi[i], ss));
    const float r = rsqrtf(HeadLanes<D>::sum(ss) * (1.f / D) + eps);
    float wl[8], wh[8];
    unpack_bf16x8(ldg_plain(w + c), wl);
    unpack_bf16x8(ldg_plain(w + c + D / 16), wh);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        lo[i] = lo[i] * r * wl[i];
        hi[i] = hi[i] * r * wh[i];
    }
}

// A block owns kRowsPerBlock recompute rows, kThreadsPerRow threads each.  A thread keeps one chunk index c, so the eight
// (cos, sin) of its pairs stay in registers for all heads of its row, and it has kFlight heads' loads in flight.
constexpr int kRowsPerBlock = 4, kThreadsPerRow = 64, kFlight = 2;
template <int D, bool INTERLEAVED>
__global__ void __launch_bounds__(kRowsPerBlock *kThreadsPerRow, 3)
extend_norm_kernel(Fresh f, uint4 *k_pool, uint4 *v_pool, uint4 *k_cache, uint4 *v_cache, const int32_t *__restrict__ q_pos,
                   const int32_t *__restrict__ fresh_dst, const int32_t *__restrict__ retain_dst, const double *__restrict__ inv_freq,
                   int n_q, int H_q, int H_kv) {
    constexpr int CPH = D / 16, HALF = D / 16, HEADS = kThreadsPerRow / CPH;
    __shared__ float2 s_cs[kRowsPerBlock][D / 2];
    const int r = threadIdx.x / kThreadsPerRow, i64 = threadIdx.x % kThreadsPerRow;
    const int c = i64 % CPH, h0 = i64 / CPH;
    const int64_t j = (int64_t)blockIdx.x * kRowsPerBlock + r;
    const bool row = j < n_q;
    if (row && i64 < D / 2) {
        double sn, cs;
        sincos((double)q_pos[j] * inv_freq[i64], &sn, &cs);
        s_cs[r][i64] = make_float2((float)cs, (float)sn);
    }
    const int64_t dst = row ? fresh_dst[j] : 0, keep = row && retain_dst ? retain_dst[j] : -1;
    grid_wait();
    grid_release();
    __syncthreads();
    if (!row) return;
    float2 cs[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) cs[i] = s_cs[r][cs_entry<D, INTERLEAVED>(c, i)];

    for (int h = h0; f.q && h < H_q; h += kFlight * HEADS) {
        uint4 lo[kFlight], hi[kFlight];
#pragma unroll
        for (int u = 0; u < kFlight; ++u)
            if (h + u * HEADS < H_q) {
                const uint4 *p = f.q + j * f.q_row + (h + u * HEADS) * (D / 8) + c;
                lo[u] = ldg_stream(p);
                hi[u] = ldg_stream(p + HALF);
            }
#pragma unroll
        for (int u = 0; u < kFlight; ++u)
            if (h + u * HEADS < H_q) {
                float a[8], b[8];
                unpack_bf16x8(lo[u], a);
                unpack_bf16x8(hi[u], b);
                norm_chunks<D>(a, b, f.q_weight, c, f.eps);
                rotate_f<INTERLEAVED>(a, b, cs);
                uint4 *o = f.q_out + (j * H_q + h + u * HEADS) * (D / 8) + c;
                stg(o, pack_bf16x8(a));
                stg(o + HALF, pack_bf16x8(b));
            }
    }
    for (int h = h0; h < H_kv; h += HEADS) {
        const uint4 *pk = f.k + j * f.k_row + h * (D / 8) + c, *pv = f.v + j * f.v_row + h * (D / 8) + c;
        const uint4 klo = ldg_stream(pk), khi = ldg_stream(pk + HALF), vlo = ldg_stream(pv), vhi = ldg_stream(pv + HALF);
        const size_t o = (size_t)(dst * H_kv + h) * (D / 8) + c, ko = (size_t)(keep * H_kv + h) * (D / 8) + c;
        stg(v_pool + o, vlo);
        stg(v_pool + o + HALF, vhi);
        float a[8], b[8];
        unpack_bf16x8(klo, a);
        unpack_bf16x8(khi, b);
        norm_chunks<D>(a, b, f.k_weight, c, f.eps);
        if (keep >= 0) {                       // the cache keeps the key as it is before rotation
            stg(k_cache + ko, pack_bf16x8(a));
            stg(k_cache + ko + HALF, pack_bf16x8(b));
            stg(v_cache + ko, vlo);
            stg(v_cache + ko + HALF, vhi);
        }
        rotate_f<INTERLEAVED>(a, b, cs);
        stg(k_pool + o, pack_bf16x8(a));
        stg(k_pool + o + HALF, pack_bf16x8(b));
    }
}

// A decode step's new tokens: request r = blockIdx.x has its token at position seq_len[r] - 1; the blocks of blockIdx.y share its
// heads out, one chunk pair a thread, so that the latency of a small batch is one chain: length, page and angles; row; store.
// FOUR: the pools are 4-bit ones; what they keep is the row a 16-bit pool would, quantised.
constexpr int kStepThreads = 256;
struct StepTables {
    const int32_t *table, *seq_len;
    int max_pages, num_pool_pages, page_size, H_q, H_kv;
    double inv_freq[64];
};
template <int D, bool INTERLEAVED, bool FOUR>
__global__ void __launch_bounds__(kStepThreads)
decode_write_kernel(Fresh f, void *k_pool, void *v_pool, const __grid_constant__ StepTables s) {
    constexpr int CPH = D / 16, HALF = D / 16;
    __shared__ float2 s_cs[D / 2];
    const int tid = threadIdx.x, c = tid % CPH;
    const int64_t r = blockIdx.x;
    const int head = blockIdx.y * (kStepThreads / CPH) + tid / CPH;
    const bool is_q = head < s.H_q, mine = is_q ? f.q != nullptr : head < s.H_q + s.H_kv;
    grid_wait();
    grid_release();
    uint4 lo, hi, vlo, vhi;                       // (loaded before the chain of length, page and angles has come in)
    if (mine) {
        const uint4 *p = is_q ? f.q + r * f.q_row + head * (D / 8) + c : f.k + r * f.k_row + (head - s.H_q) * (D / 8) + c;
        lo = ldg_stream(p);
        hi = ldg_stream(p + HALF);
        if (!is_q) {
            const uint4 *pv = f.v + r * f.v_row + (head - s.H_q) * (D / 8) + c;
            vlo = ldg_stream(pv);
            vhi = ldg_stream(pv + HALF);
        }
    }
    const int pos = s.seq_len[r] - 1, col = pos / s.page_size;
    if (pos < 0 || col >= s.max_pages) return;                                   // (the same for the whole block)
    const int page = s.table[r * s.max_pages + col], off = pos - col * s.page_size;
    if (tid < D / 2) {
        double sn, cs;
        sincos((double)pos * s.inv_freq[tid], &sn, &cs);
        s_cs[tid] = make_float2((float)cs, (float)sn);
    }
    __syncthreads();
    if (page < 0 || page >= s.num_pool_pages || !mine) return;                   // (the same for the threads of a head)
    float2 cs[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) cs[i] = s_cs[cs_entry<D, INTERLEAVED>(c, i)];
    float a[8], b[8];
    unpack_bf16x8(lo, a);
    unpack_bf16x8(hi, b);
    norm_chunks<D>(a, b, is_q ? f.q_weight : f.k_weight, c, f.eps);
    rotate_f<INTERLEAVED>(a, b, cs);
    lo = pack_bf16x8(a);
    hi = pack_bf16x8(b);
    if (is_q) {
        uint4 *o = f.q_out + (r * s.H_q + head) * (D / 8) + c;
        stg(o, lo);
        stg(o + HALF, hi);
        return;
    }
    const int h = head - s.H_q;
    if constexpr (!FOUR) {
        const size_t o = (((size_t)page * s.page_size + off) * s.H_kv + h) * (D / 8) + c;
        uint4 *kp = static_cast<uint4 *>(k_pool), *vp = static_cast<uint4 *>(v_pool);
        stg(kp + o, lo);
        stg(kp + o + HALF, hi);
        stg(vp + o, vlo);
        stg(vp + o + HALF, vhi);
    } else {
        const size_t co = codes4_at<D>(page, off, h, s.page_size, s.H_kv), po = params4_at<D>(page, off, h, s.page_size, s.H_kv);
#pragma unroll
        for (int which = 0; which < 2; ++which) {
            uint2 codes, numbers;
            quantise4<D>(which ? vlo : lo, which ? vhi : hi, codes, numbers);
            uint8_t *pool = static_cast<uint8_t *>(which ? v_pool : k_pool);
            *reinterpret_cast<uint2 *>(pool + co + c * 8) = codes;
            if (c == 0) *reinterpret_cast<uint2 *>(pool + po) = numbers;
        }
    }
}

bool misaligned(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15) != 0; }

// Checks the description of n rows and fills in the kernels' form of it.
int32_t check_rows(const tessera_fresh_rows *rows, int64_t n, int H_q, int H_kv, int D, Fresh *f) {
    if (!rows) return api_set_error(TESSERA_INVALID_ARG, "null rows");
    if (!rows->k || !rows->v || (rows->q && !rows->q_out)) return api_set_error(TESSERA_INVALID_ARG, "k, v and (with q) q_out must be non-null");
    for (const void *p : {rows->q, rows->k, rows->v, (const void *)rows->q_out, rows->q_weight, rows->k_weight})
        if (misaligned(p)) return api_set_error(TESSERA_INVALID_ARG, "q, k, v, q_out and the weights must be 16-byte aligned");
    if (!(rows->eps >= 0.f) || std::isinf(rows->eps)) return api_set_error(TESSERA_INVALID_ARG, "eps must be finite and not negative");
    const int64_t q_least = (int64_t)H_q * D, kv_least = (int64_t)H_kv * D;
    const int64_t q_row = rows->q_row ? rows->q_row : q_least, k_row = rows->k_row ? rows->k_row : kv_least, v_row = rows->v_row ? rows->v_row : kv_least;
    if (q_row < q_least || k_row < kv_least || v_row < kv_least || q_row % 8 || k_row % 8 || v_row % 8)
        return api_set_error(TESSERA_INVALID_ARG, "row strides must be multiples of 8 elements and at least a row");
    if (rows->q && rows->q_out == rows->q && q_row != q_least)
        return api_set_error(TESSERA_INVALID_ARG, "q_out may be q itself only where q's rows lie side by side");
    // (blocks read their rows when they get to them: one that lies under another's result would be read after it)
    const uintptr_t to = reinterpret_cast<uintptr_t>(rows->q_out), to_end = to + (uintptr_t)(n * q_least) * 2;
    const void *const from[3] = {rows->q_out == rows->q ? nullptr : rows->q, rows->k, rows->v};
    const int64_t stride[3] = {q_row, k_row, v_row}, least[3] = {q_least, kv_least, kv_least};
    for (int i = 0; rows->q && i < 3; ++i) {
        const uintptr_t at = reinterpret_cast<uintptr_t>(from[i]);
        if (at && at < to_end && to < at + (uintptr_t)((n - 1) * stride[i] + least[i]) * 2)
            return api_set_error(TESSERA_INVALID_ARG, "q_out overlaps rows that are read");
    }
    *f = {static_cast<const uint4 *>(rows->q), static_cast<const uint4 *>(rows->k), static_cast<const uint4 *>(rows->v), static_cast<uint4 *>(rows->q_out),
          q_row / 8, k_row / 8, v_row / 8, static_cast<const uint4 *>(rows->q_weight), static_cast<const uint4 *>(rows->k_weight), rows->eps};
    return TESSERA_OK;
}

int32_t launched(cudaError_t e, const char *what) {
    if (e == cudaSuccess) return TESSERA_OK;
    return api_set_error(TESSERA_CUDA_ERROR, std::string(what) + ": " + cudaGetErrorName(e) + " (" + cudaGetErrorString(e) + ")");
}

template <bool FOUR>
int32_t decode_write(const tessera_model_cfg *cfg, const tessera_decode_desc *d, void *k_pool, void *v_pool, const tessera_fresh_rows *rows, void *stream) {
    std::string err;
    if (int32_t rc = check_decode(cfg, d, &err)) return api_set_error(rc, err);
    if (cfg->rope_pairing != 0 && cfg->rope_pairing != 1) return api_set_error(TESSERA_UNSUPPORTED_SHAPE, "rope_pairing: 0 (half-split pairs) or 1 (interleaved pairs)");
    if (!cfg->inv_freq && !(cfg->rope_theta > 0.0)) return api_set_error(TESSERA_INVALID_ARG, "rope_theta must be positive");
    if (d->batch == 0) return TESSERA_OK;
    if (!k_pool || !v_pool || misaligned(k_pool) || misaligned(v_pool))
        return api_set_error(TESSERA_INVALID_ARG, "k_pool / v_pool must be non-null and 16-byte aligned");
    const int D = cfg->head_dim;
    Fresh f;
    if (int32_t rc = check_rows(rows, d->batch, cfg->num_q_heads, cfg->num_kv_heads, D, &f)) return rc;
    StepTables s{d->block_table, d->seq_len, d->max_pages, d->num_pool_pages, cfg->page_size, cfg->num_q_heads, cfg->num_kv_heads, {}};
    for (int m = 0; m < D / 2; ++m) s.inv_freq[m] = cfg->inv_freq ? cfg->inv_freq[m] : std::pow(cfg->rope_theta, -2.0 * m / D);
    const int heads = kStepThreads / (D / 16);
    const dim3 grid((unsigned)d->batch, (unsigned)((cfg->num_q_heads + cfg->num_kv_heads + heads - 1) / heads));
    const bool il = cfg->rope_pairing == 1;
    auto kernel = D == 128 ? (il ? decode_write_kernel<128, true, FOUR> : decode_write_kernel<128, false, FOUR>)
                           : (il ? decode_write_kernel<64, true, FOUR> : decode_write_kernel<64, false, FOUR>);
    return launched(launch_grid(kernel, grid, kStepThreads, 0, static_cast<cudaStream_t>(stream), true, f, k_pool, v_pool, s), "launch of the decode write");
}

int32_t extend_write_norm(const tessera_plan *pl, void *k_pool, void *v_pool, const tessera_fresh_rows *rows, void *k_cache, void *v_cache, void *stream) {
    if (!pl) return api_set_error(TESSERA_INVALID_ARG, "null plan");
    if (pl->host_only) return api_set_error(TESSERA_INVALID_ARG, "plan was created with TESSERA_PLAN_HOST_ONLY");
    if (!on_plan_device(pl)) return api_set_error(TESSERA_INVALID_ARG, "the current device is not the plan's");
    if (pl->n_q == 0) return TESSERA_OK;
    if (!k_pool || !v_pool || misaligned(k_pool) || misaligned(v_pool))
        return api_set_error(TESSERA_INVALID_ARG, "k_pool / v_pool must be non-null and 16-byte aligned");
    if (misaligned(k_cache) || misaligned(v_cache)) return api_set_error(TESSERA_INVALID_ARG, "k_cache / v_cache must be 16-byte aligned");
    if (pl->retained_tokens > 0 && (!k_cache || !v_cache))
        return api_set_error(TESSERA_INVALID_ARG, "the plan captures units: k_cache and v_cache must be non-null");
    if (pl->retained_tokens > 0 && pl->retain_pool_pages == 0 && (k_cache != k_pool || v_cache != v_pool))
        return api_set_error(TESSERA_INVALID_ARG, "the plan's cache pages are pages of the destination pool: pass k_pool / v_pool as k_cache / v_cache");
    const int D = pl->cfg.head_dim, Hq = pl->cfg.num_q_heads, H = pl->cfg.num_kv_heads;
    Fresh f;
    if (int32_t rc = check_rows(rows, pl->n_q, Hq, H, D, &f)) return rc;
    const DeviceTables &d = pl->dev;
    const bool il = pl->cfg.rope_pairing == 1;
    auto kernel = D == 128 ? (il ? extend_norm_kernel<128, true> : extend_norm_kernel<128, false>) : (il ? extend_norm_kernel<64, true> : extend_norm_kernel<64, false>);
    return launched(launch_kernel(kernel, (unsigned)((pl->n_q + kRowsPerBlock - 1) / kRowsPerBlock), kRowsPerBlock * kThreadsPerRow, 0,
                                  static_cast<cudaStream_t>(stream), pl->chained, f, static_cast<uint4 *>(k_pool), static_cast<uint4 *>(v_pool),
                                  static_cast<uint4 *>(k_cache), static_cast<uint4 *>(v_cache), d.q_pos, d.fresh_dst,
                                  pl->retained_tokens > 0 ? d.retain_dst : nullptr, d.inv_freq, (int)pl->n_q, Hq, H),
                    "launch of the normalising write");
}

}  // namespace

int32_t check_decode(const tessera_model_cfg *cfg, const tessera_decode_desc *d, std::string *err) {
    auto fail = [&](int32_t code, const char *msg) { *err = msg; return code; };
    if (!cfg || !d) return fail(TESSERA_INVALID_ARG, "null cfg or desc");
    const int Hq = cfg->num_q_heads, H = cfg->num_kv_heads, B = cfg->page_size;
    if (Hq <= 0 || H <= 0 || Hq % H != 0) return fail(TESSERA_UNSUPPORTED_SHAPE, "num_q_heads must be a positive multiple of num_kv_heads");
    if (H > 4096) return fail(TESSERA_UNSUPPORTED_SHAPE, "more than 4 096 KV heads");
    if (Hq / H > 16) return fail(TESSERA_UNSUPPORTED_SHAPE, "group size H_q/H_kv above 16");
    if (cfg->head_dim != 64 && cfg->head_dim != 128) return fail(TESSERA_UNSUPPORTED_SHAPE, "head_dim: only 64 and 128");
    if (B < 8 || B > 128 || (B & (B - 1)) != 0) return fail(TESSERA_UNSUPPORTED_SHAPE, "page_size: a power of two in 8..128");
    if (d->batch < 0 || d->max_pages < 0 || d->num_pool_pages < 0 || d->window < 0 || d->n_sink < 0)
        return fail(TESSERA_INVALID_ARG, "negative batch, max_pages, num_pool_pages, window or n_sink");
    if (d->batch > 0 && (!d->seq_len || (!d->block_table && d->max_pages > 0))) return fail(TESSERA_INVALID_ARG, "null seq_len or block_table");
    if ((int64_t)d->num_pool_pages * B > INT32_MAX) return fail(TESSERA_UNSUPPORTED_SHAPE, "pool has more than 2^31 slots");
    if ((int64_t)d->max_pages * B > (1 << 30)) return fail(TESSERA_UNSUPPORTED_SHAPE, "a block table of more than 2^30 tokens a request");
    // (tiles a request, divided out: the product of all three passes 64 bits)
    if (d->batch > 0 && (int64_t)d->max_pages * B / kDecodeUnit + 1 > INT32_MAX / ((int64_t)d->batch * H)) return fail(TESSERA_UNSUPPORTED_SHAPE, "block tables of more than 2^31 tiles of 16 keys");
    return TESSERA_OK;
}

}  // namespace tessera

using namespace tessera;

extern "C" {

int32_t tessera_extend_write_norm(const tessera_plan *pl, void *k_pool, void *v_pool, const tessera_fresh_rows *rows, void *k_cache,
                                  void *v_cache, void *stream) {
    return guarded([&] { return extend_write_norm(pl, k_pool, v_pool, rows, k_cache, v_cache, stream); });
}

int32_t tessera_decode_write(const tessera_model_cfg *cfg, const tessera_decode_desc *desc, void *k_pool, void *v_pool,
                             const tessera_fresh_rows *rows, void *stream) {
    return guarded([&] { return decode_write<false>(cfg, desc, k_pool, v_pool, rows, stream); });
}

int32_t tessera_decode_write_kv4(const tessera_model_cfg *cfg, const tessera_decode_desc *desc, void *k_pool4, void *v_pool4,
                                 const tessera_fresh_rows *rows, void *stream) {
    return guarded([&] { return decode_write<true>(cfg, desc, k_pool4, v_pool4, rows, stream); });
}

}  // extern "C"
