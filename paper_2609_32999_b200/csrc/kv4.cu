// Cached units stored in 4 bits (format: pair_chunk.cuh; the paper's system keeps 16-bit K/V, Sec. 8, and has no
// counterpart).  A row of a head takes D / 2 + 8 bytes in place of 2 D.  Both directions are driven by a plan's copy list and
// shift table, as those of the 8-bit tier:
//   retain : 16-bit pages -> 4-bit pages (keys rotated by the plan's shifts, rounded to bf16, then quantised)
//   expand : 4-bit pages -> the request's 16-bit pages (keys rotated on the way)
// A task is a pair-chunk of a row: a thread holds bytes 8 c .. 8 c + 7 of the codes, i.e. elements 8 c .. and their partners
// D / 2 later, on the 4-bit side one 8-byte access.  Bound by HBM on the 16-bit side.
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <string>

#include "device_mem.cuh"
#include "launch.h"
#include "pair_chunk.cuh"
#include "plan.h"

namespace tessera {

int32_t api_set_error(int32_t code, const std::string &msg);

namespace {

constexpr int kThreads = 256;

// One thread block per GatherItem.
template <int D, bool TO_4BIT, bool ROTATE, bool INTERLEAVED>
__global__ void __launch_bounds__(kThreads)
kv4_kernel(const uint8_t *__restrict__ k_src, const uint8_t *__restrict__ v_src, uint8_t *__restrict__ k_dst, uint8_t *__restrict__ v_dst,
           const int32_t *__restrict__ g_src, const int32_t *__restrict__ g_dst, const GatherItem *__restrict__ items,
           const float2 *__restrict__ rope, int H_kv, int page_size) {
    constexpr int CPH = D / 16, HALF = D / 16;
    __shared__ float2 s_rope[kGatherItemTokens * (D / 2)];
    __shared__ int32_t s_src[kGatherItemTokens], s_dst[kGatherItemTokens];

    const int tid = threadIdx.x;
    const GatherItem it = items[blockIdx.x];
    const int n_rows = ROTATE ? (it.row_step ? it.count : 1) : 0;
    const int first_row = it.row_step < 0 ? it.row0 - (it.count - 1) : it.row0;
    for (int i = tid; i < n_rows * (D / 2); i += kThreads) s_rope[i] = rope[(size_t)first_row * (D / 2) + i];
    if (tid < it.count) {
        s_dst[tid] = g_dst[it.begin + tid];
        s_src[tid] = g_src[it.begin + tid];
    }
    grid_wait();
    grid_release();
    __syncthreads();

    // Tasks go over the item's tokens first: four heads' worth of neighbouring threads are four tokens of one head, whose codes (256
    // bytes) and numbers (32) lie side by side.
    const int page_shift = __ffs(page_size) - 1;
    const int tasks_per_head = it.count * CPH, n_tasks = H_kv * tasks_per_head;
    const int c = tid % CPH;             // kThreads and tasks_per_head are multiples of CPH: a head's threads stay together
    float2 cr[8];
    if (ROTATE && it.row_step == 0)
#pragma unroll
        for (int i = 0; i < 8; ++i) cr[i] = s_rope[cs_entry<D, INTERLEAVED>(c, i)];
    constexpr int U = TO_4BIT ? 1 : 2;   // tasks in flight per thread
    for (int t0 = tid; t0 < n_tasks; t0 += U * kThreads) {
        uint4 w[U][4];                   // 16-bit: K and V, both chunks; 4-bit: x, y of [0] K's codes and numbers, of [1] V's
        int tok[U], head[U];
        bool ok[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int t = t0 + u * kThreads;
            ok[u] = t < n_tasks;
            if (!ok[u]) continue;
            head[u] = t / tasks_per_head;
            tok[u] = (t - head[u] * tasks_per_head) / CPH;
            const int src = s_src[tok[u]];
            if constexpr (TO_4BIT) {
                const size_t o = ((size_t)src * H_kv + head[u]) * (D / 8) + c;
                const uint4 *k = reinterpret_cast<const uint4 *>(k_src) + o, *v = reinterpret_cast<const uint4 *>(v_src) + o;
                w[u][0] = ldg_stream(k);
                w[u][1] = ldg_stream(k + HALF);
                w[u][2] = ldg_stream(v);
                w[u][3] = ldg_stream(v + HALF);
            } else {
                const int off = src & (page_size - 1);
                const size_t co = codes4_at<D>(src >> page_shift, off, head[u], page_size, H_kv) + c * 8;
                const size_t po = params4_at<D>(src >> page_shift, off, head[u], page_size, H_kv);
                const uint2 kc = ldg_pieces(reinterpret_cast<const uint2 *>(k_src + co)), kp = ldg_pieces(reinterpret_cast<const uint2 *>(k_src + po));
                const uint2 vc = ldg_pieces(reinterpret_cast<const uint2 *>(v_src + co)), vp = ldg_pieces(reinterpret_cast<const uint2 *>(v_src + po));
                w[u][0] = make_uint4(kc.x, kc.y, kp.x, kp.y);
                w[u][1] = make_uint4(vc.x, vc.y, vp.x, vp.y);
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (!ok[u]) continue;
            const int dst = s_dst[tok[u]];
            if (ROTATE && it.row_step != 0) {
                const int sr = it.row_step < 0 ? it.count - 1 - tok[u] : tok[u];
#pragma unroll
                for (int i = 0; i < 8; ++i) cr[i] = s_rope[sr * (D / 2) + cs_entry<D, INTERLEAVED>(c, i)];
            }
            float lo[8], hi[8];
            if constexpr (TO_4BIT) {
                const int off = dst & (page_size - 1);
                const size_t co = codes4_at<D>(dst >> page_shift, off, head[u], page_size, H_kv) + c * 8;
                const size_t po = params4_at<D>(dst >> page_shift, off, head[u], page_size, H_kv);
                if (ROTATE) {
                    unpack_bf16x8(w[u][0], lo);
                    unpack_bf16x8(w[u][1], hi);
                    rotate_f<INTERLEAVED>(lo, hi, cr);
                    w[u][0] = pack_bf16x8(lo);                    // what a 16-bit row would hold
                    w[u][1] = pack_bf16x8(hi);
                }
#pragma unroll
                for (int which = 0; which < 2; ++which) {
                    uint2 codes, numbers;
                    quantise4<D>(w[u][2 * which], w[u][2 * which + 1], codes, numbers);
                    uint8_t *pool = which ? v_dst : k_dst;
                    *reinterpret_cast<uint2 *>(pool + co) = codes;
                    if (c == 0) *reinterpret_cast<uint2 *>(pool + po) = numbers;
                }
            } else {
                const size_t o = ((size_t)dst * H_kv + head[u]) * (D / 8) + c;
#pragma unroll
                for (int which = 0; which < 2; ++which) {
                    unpack4(make_uint2(w[u][which].x, w[u][which].y), make_uint2(w[u][which].z, w[u][which].w), lo, hi);
                    if (ROTATE && which == 0) rotate_f<INTERLEAVED>(lo, hi, cr);
                    uint4 *pool = reinterpret_cast<uint4 *>(which ? v_dst : k_dst) + o;
                    stg(pool, pack_bf16x8(lo));
                    stg(pool + HALF, pack_bf16x8(hi));
                }
            }
        }
    }
}

template <int D, bool TO_4BIT>
cudaError_t launch_kv4(const tessera_plan *pl, const void *k_src, const void *v_src, void *k_dst, void *v_dst, bool rotate, cudaStream_t st) {
    const DeviceTables &d = pl->dev;
    const bool il = pl->cfg.rope_pairing == 1;
    auto kernel = rotate ? (il ? kv4_kernel<D, TO_4BIT, true, true> : kv4_kernel<D, TO_4BIT, true, false>) : kv4_kernel<D, TO_4BIT, false, false>;
    return launch_kernel(kernel, (unsigned)pl->items.size(), kThreads, 0, st, pl->chained, static_cast<const uint8_t *>(k_src),
                         static_cast<const uint8_t *>(v_src), static_cast<uint8_t *>(k_dst), static_cast<uint8_t *>(v_dst), d.g_src, d.g_dst, d.items,
                         d.rope, pl->cfg.num_kv_heads, pl->cfg.page_size);
}

template <bool TO_4BIT>
int32_t call_kv4(const tessera_plan *pl, const void *k_src, const void *v_src, void *k_dst, void *v_dst, uint32_t flags, void *stream) {
    if (!pl) return api_set_error(TESSERA_INVALID_ARG, "null plan");
    if (pl->host_only) return api_set_error(TESSERA_INVALID_ARG, "plan was created with TESSERA_PLAN_HOST_ONLY");
    if (flags & ~uint32_t(TESSERA_FUSE_ROPE)) return api_set_error(TESSERA_INVALID_ARG, "unknown compose flag");
    if (pl->num_source_pages <= 0)
        return api_set_error(TESSERA_INVALID_ARG, "the plan was created without a separate source pool (desc.num_source_pages)");
    for (const void *p : {k_src, v_src, (const void *)k_dst, (const void *)v_dst})
        if (!p || (reinterpret_cast<uintptr_t>(p) & 15) != 0)
            return api_set_error(TESSERA_INVALID_ARG, "source and destination pools must be non-null and 16-byte aligned");
    if (pl->items.empty()) return TESSERA_OK;
    const bool rotate = (flags & TESSERA_FUSE_ROPE) != 0;
    const cudaError_t e = (pl->cfg.head_dim == 128 ? launch_kv4<128, TO_4BIT> : launch_kv4<64, TO_4BIT>)(pl, k_src, v_src, k_dst, v_dst, rotate,
                                                                                                         static_cast<cudaStream_t>(stream));
    if (e != cudaSuccess) return api_set_error(TESSERA_CUDA_ERROR, std::string("4-bit tier launch: ") + cudaGetErrorName(e) + " (" + cudaGetErrorString(e) + ")");
    return TESSERA_OK;
}

}  // namespace
}  // namespace tessera

using namespace tessera;

extern "C" {

int32_t tessera_kv_retain_kv4(const tessera_plan *plan, const void *k_src, const void *v_src, void *k_dst4, void *v_dst4, uint32_t flags, void *stream) {
    return call_kv4<true>(plan, k_src, v_src, k_dst4, v_dst4, flags, stream);
}

int32_t tessera_kv_compose_from_kv4(const tessera_plan *plan, const void *k_src4, const void *v_src4, void *k_pool, void *v_pool, uint32_t flags, void *stream) {
    return call_kv4<false>(plan, k_src4, v_src4, k_pool, v_pool, flags, stream);
}

}  // extern "C"
