// Pieces of the epilogues of the CTA-pair GEMMs (gemm_fp8_pair.cu, gemm_fp4_pair.cu):
// two fp32 values in a 64-bit register, GELU and SiLU of two values, and 16-byte pieces of a
// slab's row.
#pragma once

#include "dit_kernels.cuh"

namespace wdc {

__device__ __forceinline__ uint64_t pack64(uint32_t lo, uint32_t hi) {
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "r"(lo), "r"(hi));
    return r;
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
    uint64_t r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
    uint64_t r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ uint64_t twice(float v) { return pack64(__float_as_uint(v), __float_as_uint(v)); }
__device__ __forceinline__ float2 unpack64(uint64_t v) {
    float2 r;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(v));
    return r;
}

// gelu_tanh_f of two values with one reciprocal for both: 1 / a = b / (a b).  The
// epilogue's exponentials and reciprocals (16 a clock) are what a GELU costs.  The
// exponent is cut off at 60, so that a b is finite; beyond it (x < -7) the result,
// below 2^-60 |x|, is 0, as gelu_tanh_f's is from 2^-126 on.  PAIRED: the exponents by
// instructions for two values, the same bits (17776 x 12288 x 3072 with bf16 results 595
// -> 570 us; with fp32 results, whose slabs hold half the columns, 1350 rows 62 -> 69).
template <bool PAIRED>
__device__ __forceinline__ void gelu_pair(float& x, float& y) {
    const float k0 = 0.7978845608028654f, k1 = 0.044715f, m2log2e = -2.0f * 1.4426950408889634f;
    float u, v, a, b, r;
    if constexpr (PAIRED) {
        const uint64_t p = pack64(__float_as_uint(x), __float_as_uint(y));
        const float2 e = unpack64(mul2(twice(k0 * m2log2e), fma2(mul2(mul2(twice(k1), p), p), p, p)));
        u = e.x;
        v = e.y;
    } else {
        u = k0 * m2log2e * fmaf(k1 * x * x, x, x);
        v = k0 * m2log2e * fmaf(k1 * y * y, y, y);
    }
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(a) : "f"(fminf(u, 60.f)));
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(b) : "f"(fminf(v, 60.f)));
    a += 1.0f;
    b += 1.0f;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(a * b));
    x *= u > 60.f ? 0.f : r * b;
    y *= v > 60.f ? 0.f : r * a;
}

// A 16-byte piece of a slab's row.
__device__ __forceinline__ void load_piece(const float* p, float (&v)[4]) {
    const float4 a = *reinterpret_cast<const float4*>(p);
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
}
__device__ __forceinline__ void load_piece(const __nv_bfloat16* p, float (&v)[8]) {
    const uint4 u = *reinterpret_cast<const uint4*>(p);
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[2 * i] = __uint_as_float(w[i] << 16);
        v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
}
__device__ __forceinline__ void store_piece(float* p, const float (&v)[4]) {
    *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
}
__device__ __forceinline__ void store_piece(__nv_bfloat16* p, const float (&v)[8]) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const __nv_bfloat162 h = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
        w[i] = *reinterpret_cast<const uint32_t*>(&h);
    }
    *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
}

// v / (1 + exp(-v)) of two values, with one reciprocal as there; below -41 (2^-60 |x|) 0.
__device__ __forceinline__ void silu_pair(float& x, float& y) {
    const float mlog2e = -1.4426950408889634f;
    const float u = x * mlog2e, v = y * mlog2e;
    float a, b, r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(a) : "f"(fminf(u, 60.f)));
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(b) : "f"(fminf(v, 60.f)));
    a += 1.0f;
    b += 1.0f;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(a * b));
    x *= u > 60.f ? 0.f : r * b;
    y *= v > 60.f ? 0.f : r * a;
}

}  // namespace wdc
