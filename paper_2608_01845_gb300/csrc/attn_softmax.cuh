// Pieces of the tensor-core attentions' softmax: exponentials of score pairs
// straight into fp16 probability words.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <cstdint>

namespace wdc {

__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// Three-input maximum (one instruction for two comparisons).
__device__ __forceinline__ float fmax3(float a, float b, float c) {
    float d;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
    return d;
}

__device__ __forceinline__ uint32_t pack2(float a, float b) {
    __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<uint32_t*>(&h);
}

// Two f32 values as one paired-fp32 operand (lo = a, hi = b).
__device__ __forceinline__ uint64_t pair(float a, float b) {
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
    return r;
}

// Two softmax numerators: x pair (fma.f32x2) -> f16x2 -> ex2.approx.f16x2
// (one SFU instruction for both) = the P word; the pair is added into an
// f16x2 partial sum.
__device__ __forceinline__ uint32_t exp2_pair_h(float s0, float s1, uint64_t scale2, uint64_t nm2, uint32_t& acc) {
    uint32_t p;
    asm("{\n .reg .b64 x;\n .reg .f32 a, b;\n .reg .b32 h;\n"
        " mov.b64 x, {%2, %3};\n"
        " fma.rn.f32x2 x, x, %4, %5;\n"
        " mov.b64 {a, b}, x;\n"
        " cvt.rn.f16x2.f32 h, b, a;\n"
        " ex2.approx.f16x2 %0, h;\n"
        " add.rn.f16x2 %1, %1, %0;\n}"
        : "=r"(p), "+r"(acc)
        : "f"(s0), "f"(s1), "l"(scale2), "l"(nm2));
    return p;
}

// The same with the pair added into two fp32 sums.  x is rounded to fp16 before the
// exponential, which moves a probability by 2^-9 ln 2 of itself where |x| < 8, 2^-8 ln 2
// up to 16: less than the bf16 result's own rounding, in numerator and sum alike.  In
// fp32 there is an exponential for each: a step of two tiles of 128 keys (32768 of them,
// 16 a clock) would take that unit 1.0 us, all the time that the step has at d = 64.
__device__ __forceinline__ uint32_t exp2_pair_f(float s0, float s1, uint64_t scale2, uint64_t nm2, float& lo, float& hi) {
    uint32_t p;
    asm("{\n .reg .b64 x;\n .reg .f32 a, b;\n .reg .b32 h;\n .reg .b16 l, u;\n"
        " mov.b64 x, {%3, %4};\n"
        " fma.rn.f32x2 x, x, %5, %6;\n"
        " mov.b64 {a, b}, x;\n"
        " cvt.rn.f16x2.f32 h, b, a;\n"
        " ex2.approx.f16x2 %0, h;\n"
        " mov.b32 {l, u}, %0;\n"
        " add.rn.f32.f16 %1, l, %1;\n"
        " add.rn.f32.f16 %2, u, %2;\n}"
        : "=r"(p), "+f"(lo), "+f"(hi)
        : "f"(s0), "f"(s1), "l"(scale2), "l"(nm2));
    return p;
}

__device__ __forceinline__ float half2_sum(uint32_t v) {
    __half2 h = *reinterpret_cast<__half2*>(&v);
    return __low2float(h) + __high2float(h);
}

}  // namespace wdc
