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
};

// ---- 4-bit rows.  A half of a head (D/2 elements) is kept as the least value m (a bf16 number, as the elements are), a
// scale s = bf16_rne((M - m) / 15) with M the greatest, and codes c = the nearest integer to (x - m) / s, ties to even; it stands
// for s c + m.  (s is within 2^-8 of (M - m) / 15, so no quotient reaches 15.5.)  s is 0, and so are the codes, where it would be
// below 2^-100 (so that no rest of a quotient is subnormal).  A half that holds a NaN or an infinity, or whose range is above fp32's, is kept as s = m = NaN.

// a / b from an approximate reciprocal of b by Markstein's correction (IBM J. Res. Dev. 34, 1990): the rest a - q b is exact, so
// q + rest inv is the rounded quotient, and the quotient itself where that is a number (half way between integers, say).
__device__ __forceinline__ float quotient(float a, float b, float inv) {
    const float q = __fmul_rn(a, inv);
    return fmaf(fmaf(-q, b, a), inv, q);
}

// Scales and least values of both halves of a head, whose elements the head's threads hold, 8 of each half as they were loaded.
// (Comparisons in pairs of bf16: the extremes are elements.)
template <int D>
__device__ __forceinline__ void ranges4(const uint4 &lo, const uint4 &hi, float (&scale)[2], float (&least)[2]) {
    auto pairs = [](uint32_t x) { return *reinterpret_cast<const __nv_bfloat162 *>(&x); };
    auto bits = [](__nv_bfloat162 x) { return *reinterpret_cast<const uint32_t *>(&x); };
    const __nv_bfloat162 top0 = __hmax2_nan(__hmax2_nan(pairs(lo.x), pairs(lo.y)), __hmax2_nan(pairs(lo.z), pairs(lo.w)));
    const __nv_bfloat162 top1 = __hmax2_nan(__hmax2_nan(pairs(hi.x), pairs(hi.y)), __hmax2_nan(pairs(hi.z), pairs(hi.w)));
    const __nv_bfloat162 low0 = __hmin2_nan(__hmin2_nan(pairs(lo.x), pairs(lo.y)), __hmin2_nan(pairs(lo.z), pairs(lo.w)));
    const __nv_bfloat162 low1 = __hmin2_nan(__hmin2_nan(pairs(hi.x), pairs(hi.y)), __hmin2_nan(pairs(hi.z), pairs(hi.w)));
    // (first half, second half) from here on
    uint32_t top = bits(__hmax2_nan(pairs(__byte_perm(bits(top0), bits(top1), 0x5410)), pairs(__byte_perm(bits(top0), bits(top1), 0x7632))));
    uint32_t low = bits(__hmin2_nan(pairs(__byte_perm(bits(low0), bits(low1), 0x5410)), pairs(__byte_perm(bits(low0), bits(low1), 0x7632))));
#pragma unroll
    for (int o = HeadLanes<D>::kN / 2; o > 0; o /= 2) {
        top = bits(__hmax2_nan(pairs(top), pairs(__shfl_xor_sync(HeadLanes<D>::mask(), top, o))));
        low = bits(__hmin2_nan(pairs(low), pairs(__shfl_xor_sync(HeadLanes<D>::mask(), low, o))));
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const float m = __uint_as_float(h ? low & 0xffff0000u : low << 16);
        const float range = __fsub_rn(__uint_as_float(h ? top & 0xffff0000u : top << 16), m);
        const bool fine = range <= 3.402823466e38f;             // (of infinities: NaN or infinite)
        const float s = __bfloat162float(__float2bfloat16_rn(quotient(range, 15.f, 1.f / 15.f)));
        least[h] = fine ? m : __int_as_float(0x7fc00000);
        scale[h] = fine ? (s < 7.8886091e-31f ? 0.f : s) : least[h];
    }
}
// Two numbers in one register pair, for the instructions that take both at once.
__device__ __forceinline__ uint64_t two(float x, float y) {
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(x), "f"(y));
    return r;
}
__device__ __forceinline__ uint64_t fma_two(uint64_t a, uint64_t b, uint64_t c) {
    uint64_t r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ uint64_t mul_two(uint64_t a, uint64_t b) {
    uint64_t r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ uint64_t add_two(uint64_t a, uint64_t b) {
    uint64_t r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
// Codes of 8 elements as the low bytes of eight numbers: the quotient of x - m and s as above, and adding 1.5 2^23 rounds it to an
// integer, ties to even.  (Of a scale of 0 or NaN: anything.)  72 000 rows of 8 heads stored: one element an instruction 74.4 us, two 68.4.
__device__ __forceinline__ void codes4(const float (&x)[8], float scale, float least, uint32_t (&c)[8]) {
    float inv;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(inv) : "f"(scale));
    const uint64_t inv2 = two(inv, inv), minus_s = two(-scale, -scale), minus_m = two(-least, -least), magic = two(12582912.f, 12582912.f);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint64_t d = add_two(two(x[2 * i], x[2 * i + 1]), minus_m), q = mul_two(d, inv2);
        const uint64_t n = add_two(fma_two(fma_two(q, minus_s, d), inv2, q), magic);
        asm("mov.b64 {%0, %1}, %2;" : "=r"(c[2 * i]), "=r"(c[2 * i + 1]) : "l"(n));
    }
}
// 8 bytes of a row of codes: low four bits the elements of the first half, high four those D/2 later.  some: which halves have codes.
__device__ __forceinline__ uint2 pack4(const uint32_t (&lo)[8], const uint32_t (&hi)[8], bool some_lo, bool some_hi) {
    const uint32_t on_lo = some_lo ? 0x0f0f0f0fu : 0u, on_hi = some_hi ? 0x0f0f0f0fu : 0u;
    auto bytes = [](const uint32_t *c) { return __byte_perm(__byte_perm(c[0], c[1], 0x0040), __byte_perm(c[2], c[3], 0x0040), 0x5410); };
    return make_uint2((bytes(hi) & on_hi) * 16u + (bytes(lo) & on_lo), (bytes(hi + 4) & on_hi) * 16u + (bytes(lo + 4) & on_lo));
}
// Scale and least value of both halves as the pool holds them: (s0, m0, s1, m1), bf16.
__device__ __forceinline__ uint2 pack_params4(float s0, float m0, float s1, float m1) {
    const __nv_bfloat162 a = __floats2bfloat162_rn(s0, m0), b = __floats2bfloat162_rn(s1, m1);
    return make_uint2(*reinterpret_cast<const uint32_t *>(&a), *reinterpret_cast<const uint32_t *>(&b));
}
// A thread's 8 bytes of codes of a head's chunk pair, and the head's numbers.
template <int D>
__device__ __forceinline__ void quantise4(const uint4 &lo, const uint4 &hi, uint2 &codes, uint2 &numbers) {
    float s[2], m[2], f[8];
    uint32_t c0[8], c1[8];
    ranges4<D>(lo, hi, s, m);
    unpack_bf16x8(lo, f);
    codes4(f, s[0], m[0], c0);
    unpack_bf16x8(hi, f);
    codes4(f, s[1], m[1], c1);
    codes = pack4(c0, c1, s[0] > 0.f, s[1] > 0.f);
    numbers = pack_params4(s[0], m[0], s[1], m[1]);
}
// A code becomes a number as the last byte of 2^23's mantissa.
__device__ __forceinline__ void unpack4(const uint2 &w, const uint2 &p, float (&lo)[8], float (&hi)[8]) {
    const float s0 = __uint_as_float(p.x << 16), m0 = __uint_as_float(p.x & 0xffff0000u);
    const float s1 = __uint_as_float(p.y << 16), m1 = __uint_as_float(p.y & 0xffff0000u);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint32_t b = i < 4 ? w.x : w.y;
        lo[i] = fmaf(__uint_as_float(__byte_perm(b & 0x0f0f0f0fu, 0x4b000000u, 0x7650 + (i & 3))) - 8388608.f, s0, m0);
        hi[i] = fmaf(__uint_as_float(__byte_perm((b >> 4) & 0x0f0f0f0fu, 0x4b000000u, 0x7650 + (i & 3))) - 8388608.f, s1, m1);
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
