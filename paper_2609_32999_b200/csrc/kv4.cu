// Cached units stored in 4 bits (format: pair_chunk.cuh; the paper's system keeps 16-bit K/V, Sec. 8, and has no
// counterpart).  A row of a head takes D / 2 + 8 bytes in place of 2 D.  Both directions are driven by a plan's copy list and
// shift table, as those of the 8-bit tier:
//   retain : 16-bit pages -> 4-bit pages (keys rotated by the plan's shifts, rounded to bf16, then quantised)
//   expand : 4-bit pages -> the request's 16-bit pages (keys rotated on the way)
// A task is a pair-chunk of a row: a thread holds bytes 8 c .. 8 c + 7 of the codes, i.e. elements 8 c .. and their partners
// D / 2 later, on the 4-bit side one 8-byte access.
// 73 268 rows of 8 heads of 128 (384 MB read and written a direction, 59 us at the rate of a copy): retain 68 to 77 us, whose extremes,
// quotients and roundings fill 72 % of the issue slots, 81 to 89 with keys rotated (see kAhead); expand 72, waiting for its loads (slots, then
// codes), 68 without rotation.  Four blocks an SM with two heads under way a thread; three with four heads 75 us, four with one 89 (expand).
// At 64 registers expand with rotation spills 12 bytes, retain with interleaved pairs 4.
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <string>

#include "decode.h"
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
__global__ void __launch_bounds__(kThreads, 4)
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

    // A thread keeps its token and its chunk pair and goes through the heads: slots, places and (cos, sin) are worked out once, and four
    // groups of neighbouring threads are four tokens of one head, whose codes (256 bytes) and numbers (32) lie side by side.
    // Items of fewer tokens have several heads under way at once.
    const int slots = it.count > 16 ? 32 : it.count > 8 ? 16 : 8;
    const int c = tid % CPH, tok = tid / CPH % slots, page_shift = __ffs(page_size) - 1;
    if (tok >= it.count) return;         // (the threads of a head together)
    float2 cr[8];
    if (ROTATE) {
        const float2 *row = s_rope + (it.row_step == 0 ? 0 : it.row_step < 0 ? it.count - 1 - tok : tok) * (D / 2);
#pragma unroll
        for (int i = 0; i < 8; ++i) cr[i] = row[cs_entry<D, INTERLEAVED>(c, i)];
    }
    const int src = s_src[tok], dst = s_dst[tok], wide = TO_4BIT ? src : dst, narrow = TO_4BIT ? dst : src;
    const int h0 = tid / CPH / slots, step = kThreads / CPH / slots;
    const size_t head4 = (size_t)page_size * (D / 2 + 8);
    const size_t o16 = ((size_t)wide * H_kv + h0) * (D / 8) + c;
    const size_t oc = codes4_at<D>(narrow >> page_shift, narrow & (page_size - 1), h0, page_size, H_kv) + c * 8;
    const size_t on = params4_at<D>(narrow >> page_shift, narrow & (page_size - 1), h0, page_size, H_kv);
    if constexpr (TO_4BIT) {
        const uint4 *k = reinterpret_cast<const uint4 *>(k_src) + o16, *v = reinterpret_cast<const uint4 *>(v_src) + o16;
        uint8_t *kd = k_dst + oc, *vd = v_dst + oc, *kn = k_dst + on, *vn = v_dst + on;
        // The next head is on its way while one is worked on, but for keys that are rotated as well (72 000 rows, with the quotients one at a
        // time as they then were: 79.5 -> 74.8 us, rotated 90.7 -> 93.8, for want of registers).
        constexpr bool kAhead = !ROTATE;
        uint4 klo, khi, vlo, vhi, next[4];
        auto load = [&](uint4 &a, uint4 &b, uint4 &x, uint4 &y) { a = ldg_stream(k), b = ldg_stream(k + HALF), x = ldg_stream(v), y = ldg_stream(v + HALF); };
        if (kAhead && h0 < H_kv) load(next[0], next[1], next[2], next[3]);
        for (int h = h0; h < H_kv; h += step) {
            if (kAhead) klo = next[0], khi = next[1], vlo = next[2], vhi = next[3];
            else load(klo, khi, vlo, vhi);
            k += step * (D / 8), v += step * (D / 8);
            if (kAhead && h + step < H_kv) load(next[0], next[1], next[2], next[3]);
            if (ROTATE) {
                float lo[8], hi[8];
                unpack_bf16x8(klo, lo);
                unpack_bf16x8(khi, hi);
                rotate_f<INTERLEAVED>(lo, hi, cr);
                klo = pack_bf16x8(lo);                    // what a 16-bit row would hold
                khi = pack_bf16x8(hi);
            }
            uint2 codes, numbers;
            quantise4<D>(klo, khi, codes, numbers);
            *reinterpret_cast<uint2 *>(kd) = codes;
            if (c == 0) *reinterpret_cast<uint2 *>(kn) = numbers;
            quantise4<D>(vlo, vhi, codes, numbers);
            *reinterpret_cast<uint2 *>(vd) = codes;
            if (c == 0) *reinterpret_cast<uint2 *>(vn) = numbers;
            kd += step * head4, vd += step * head4, kn += step * head4, vn += step * head4;
        }
    } else {
        const uint8_t *kc = k_src + oc, *vc = v_src + oc, *kn = k_src + on, *vn = v_src + on;
        uint4 *kd = reinterpret_cast<uint4 *>(k_dst) + o16, *vd = reinterpret_cast<uint4 *>(v_dst) + o16;
        constexpr int U = 2;             // heads in flight
        for (int h = h0; h < H_kv; h += U * step) {
            uint2 w[U][4];
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (h + u * step < H_kv) {
                    w[u][0] = ldg_pieces(reinterpret_cast<const uint2 *>(kc + u * step * head4));
                    w[u][1] = ldg_pieces(reinterpret_cast<const uint2 *>(kn + u * step * head4));
                    w[u][2] = ldg_pieces(reinterpret_cast<const uint2 *>(vc + u * step * head4));
                    w[u][3] = ldg_pieces(reinterpret_cast<const uint2 *>(vn + u * step * head4));
                }
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (h + u * step < H_kv) {
                    float lo[8], hi[8];
                    unpack4(w[u][0], w[u][1], lo, hi);
                    if (ROTATE) rotate_f<INTERLEAVED>(lo, hi, cr);
                    stg(kd, pack_bf16x8(lo));
                    stg(kd + HALF, pack_bf16x8(hi));
                    unpack4(w[u][2], w[u][3], lo, hi);
                    stg(vd, pack_bf16x8(lo));
                    stg(vd + HALF, pack_bf16x8(hi));
                    kd += step * (D / 8), vd += step * (D / 8);
                }
            kc += U * step * head4, vc += U * step * head4, kn += U * step * head4, vn += U * step * head4;
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
    if (!on_plan_device(pl)) return api_set_error(TESSERA_INVALID_ARG, "the current device is not the plan's");
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
    return guarded([&] { return call_kv4<true>(plan, k_src, v_src, k_dst4, v_dst4, flags, stream); });
}

int32_t tessera_kv_compose_from_kv4(const tessera_plan *plan, const void *k_src4, const void *v_src4, void *k_pool, void *v_pool, uint32_t flags, void *stream) {
    return guarded([&] { return call_kv4<false>(plan, k_src4, v_src4, k_pool, v_pool, flags, stream); });
}

}  // extern "C"
