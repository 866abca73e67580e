// What the kernels that move head rows share: a thread holds 8 elements of a head and the 8 that lie D/2 elements
// later, so both halves of every rotary pair (half-split or interleaved) sit in one thread.
#pragma once
#include <cstdint>

#include <cuda_bf16.h>
#include <cuda_runtime.h>

namespace tessera {

__device__ __forceinline__ void unpack_bf16x8(const uint4 &v, float (&f)[8]) {
    const uint32_t *w = reinterpret_cast<const uint32_t *>(&v);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        f[2 * i] = __uint_as_float(w[i] << 16);
        f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
}
__device__ __forceinline__ uint4 pack_bf16x8(const float (&f)[8]) {
    uint4 v;
    uint32_t *w = reinterpret_cast<uint32_t *>(&v);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        __nv_bfloat162 p = __floats2bfloat162_rn(f[2 * i], f[2 * i + 1]);
        w[i] = *reinterpret_cast<uint32_t *>(&p);
    }
    return v;
}

// x' = x cos - y sin, y' = y cos + x sin in fp32, the arithmetic of the 16-bit gather; a table entry
// that is exactly (1, 0) leaves the pair untouched (signed zeros and infinities survive a zero shift).
__device__ __forceinline__ void rotate_pair_f(float &x, float &y, const float2 c) {
    const bool identity = c.x == 1.f && c.y == 0.f;
    const float a = fmaf(-y, c.y, x * c.x), b = fmaf(x, c.y, y * c.x);
    x = identity ? x : a;
    y = identity ? y : b;
}
template <bool INTERLEAVED>
__device__ __forceinline__ void rotate_f(float (&lo)[8], float (&hi)[8], const float2 *cs) {
    if (INTERLEAVED) {
        // lo holds pairs (0,1) (2,3) .. with cs[0..3]; hi the chunk D/2 elements later with cs[4..7]
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            rotate_pair_f(lo[2 * i], lo[2 * i + 1], cs[i]);
            rotate_pair_f(hi[2 * i], hi[2 * i + 1], cs[4 + i]);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) rotate_pair_f(lo[i], hi[i], cs[i]);
    }
}
// Index (within a D/2-entry cos/sin row) of entry i of the 8 that a thread with chunk index c needs.
template <int D, bool INTERLEAVED>
__device__ __forceinline__ int cs_entry(int c, int i) {
    return INTERLEAVED ? (i < 4 ? 4 * c + i : 4 * c + D / 4 + (i - 4)) : c * 8 + i;
}

// The D/16 neighbouring threads that hold a head: all of them take part together.
template <int D>
struct HeadLanes {
    static constexpr int kN = D / 16;
    __device__ static uint32_t mask() { return (kN == 32 ? ~0u : ((1u << kN) - 1)) << ((threadIdx.x & 31) & ~(kN - 1)); }
    __device__ static float sum(float v) {
#pragma unroll
        for (int o = kN / 2; o > 0; o /= 2) v += __shfl_xor_sync(mask(), v, o);
        return v;
    }
    // (the largest of both arguments over the head's threads; NaN is lost, see quantise4)
    __device__ static float max(float v) {
#pragma unroll
        for (int o = kN / 2; o > 0; o /= 2) v = fmaxf(v, __shfl_xor_sync(mask(), v, o));
        return v;
    }
};

// ---- 4-bit rows.  A half of a head (D/2 elements) is kept as the least value m (a bf16 number, as the elements are), a
// scale s = bf16_rne((M - m) / 15) with M the greatest, and codes c = the nearest integer to (x - m) / s, ties to even, at
// most 15; it stands for s c + m.  s is 0, and so are the codes, where it would be below 2^-126.  A half that holds a NaN or an
// infinity, or whose range is above fp32's, is kept as s = m = NaN.

// Scale and least value of a half whose elements the head's threads hold, 8 each.
template <int D>
__device__ __forceinline__ void range4(const float (&x)[8], float &scale, float &least) {
    float lo = x[0], hi = x[0], bad = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        lo = fminf(lo, x[i]);
        hi = fmaxf(hi, x[i]);
        bad = fmaf(x[i], 0.f, bad);            // NaN where an element is NaN or infinite, 0 otherwise
    }
    hi = HeadLanes<D>::max(hi);
    lo = -HeadLanes<D>::max(-lo);
    const float range = __fsub_rn(hi, lo) + HeadLanes<D>::sum(bad);
    const bool fine = range <= 3.402823466e38f;
    const float s = __bfloat162float(__float2bfloat16_rn(__fdiv_rn(range, 15.f)));
    least = fine ? lo : __int_as_float(0x7fc00000);
    scale = fine ? (s < 1.17549435e-38f ? 0.f : s) : least;
}
// Codes of 8 elements, 0 where there is no scale.  The quotient's integer is corrected where its rounding could have moved it
// across a border: c s is exact, so x - m - c s tells on which side of half a step the element lies.
__device__ __forceinline__ void codes4(const float (&x)[8], float scale, float least, uint32_t (&c)[8]) {
    const bool some = scale > 0.f;
    const float inv = some ? __frcp_rn(scale) : 0.f, half = 0.5f * scale;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float d = __fsub_rn(x[i], least);
        float n = rintf(d * inv);
        const float rest = fmaf(-n, scale, d);
        const bool odd = (__float2int_rn(n) & 1) != 0;
        if (rest > half || (rest == half && odd)) n += 1.f;
        if (rest < -half || (rest == -half && odd)) n -= 1.f;
        c[i] = some ? (uint32_t)fminf(fmaxf(n, 0.f), 15.f) : 0u;
    }
}
// 8 bytes of a row of codes: low four bits the elements of the first half, high four those D/2 later.
__device__ __forceinline__ uint2 pack4(const uint32_t (&lo)[8], const uint32_t (&hi)[8]) {
    uint32_t w[2];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        w[k] = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) w[k] |= (lo[4 * k + i] | hi[4 * k + i] << 4) << (8 * i);
    }
    return make_uint2(w[0], w[1]);
}
// Scale and least value of both halves as the pool holds them: (s0, m0, s1, m1), bf16.
__device__ __forceinline__ uint2 pack_params4(float s0, float m0, float s1, float m1) {
    const __nv_bfloat162 a = __floats2bfloat162_rn(s0, m0), b = __floats2bfloat162_rn(s1, m1);
    return make_uint2(*reinterpret_cast<const uint32_t *>(&a), *reinterpret_cast<const uint32_t *>(&b));
}
__device__ __forceinline__ void unpack4(const uint2 &w, const uint2 &p, float (&lo)[8], float (&hi)[8]) {
    const float s0 = __uint_as_float(p.x << 16), m0 = __uint_as_float(p.x & 0xffff0000u);
    const float s1 = __uint_as_float(p.y << 16), m1 = __uint_as_float(p.y & 0xffff0000u);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint32_t b = ((i < 4 ? w.x : w.y) >> (8 * (i & 3))) & 0xffu;
        lo[i] = fmaf((float)(b & 15u), s0, m0);
        hi[i] = fmaf((float)(b >> 4), s1, m1);
    }
}
// Where a token's row lies in a 4-bit pool [pages][H_kv][page_size * (D/2 + 8)]: its codes and its four numbers.
template <int D>
__device__ __forceinline__ size_t codes4_at(size_t page, int off, int head, int page_size, int H_kv) {
    return (page * H_kv + head) * (size_t)(page_size * (D / 2 + 8)) + (size_t)off * (D / 2);
}
template <int D>
__device__ __forceinline__ size_t params4_at(size_t page, int off, int head, int page_size, int H_kv) {
    return (page * H_kv + head) * (size_t)(page_size * (D / 2 + 8)) + (size_t)page_size * (D / 2) + (size_t)off * 8;
}

}  // namespace tessera
