// What the kernels that write 8 and 4 bits share (quant_fp8.cu, quant_fp4.cu,
// add_norm.cu): 16-byte loads of a row, maxima, and the conversions.
#pragma once

#include <cuda_fp8.h>

#include "dit_kernels.cuh"

namespace wdc {

constexpr float kE4m3Max = 448.0f;

// Maximum that keeps a NaN (fmaxf drops it).
__device__ __forceinline__ float max_nan(float a, float b) {
    float d;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(d) : "f"(a), "f"(b));
    return d;
}

// Four quotients to e4m3, to nearest even; beyond 448 saturated, NaN kept.
__device__ __forceinline__ uint32_t e4m3x4(float a, float b, float c, float d) {
    uint32_t r;
    asm("{\n .reg .b16 lo, hi;\n cvt.rn.satfinite.e4m3x2.f32 lo, %2, %1;\n cvt.rn.satfinite.e4m3x2.f32 hi, %4, %3;\n"
        " mov.b32 %0, {lo, hi};\n}"
        : "=r"(r)
        : "f"(a), "f"(b), "f"(c), "f"(d));
    return r;
}

// A lane's 8 elements as they lie in memory, and in fp32.
template <typename T> struct Raw8;
template <> struct Raw8<float> { float4 a, b; };
template <> struct Raw8<__nv_bfloat16> { uint4 a; };
__device__ __forceinline__ void load_raw(const float* p, Raw8<float>& r) {
    r.a = reinterpret_cast<const float4*>(p)[0];
    r.b = reinterpret_cast<const float4*>(p)[1];
}
// The same, and a store, in one instruction where the address is a multiple of 32 bytes
// (`wide`): two of 16 bytes, 32 apart from lane to lane, pass through L1 in twice as many
// cycles.
__device__ __forceinline__ void load_raw(const float* p, Raw8<float>& r, bool wide) {
    if (wide)
        asm volatile("ld.global.v8.f32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                     : "=f"(r.a.x), "=f"(r.a.y), "=f"(r.a.z), "=f"(r.a.w), "=f"(r.b.x), "=f"(r.b.y), "=f"(r.b.z), "=f"(r.b.w)
                     : "l"(p));
    else
        load_raw(p, r);
}
// Rows that are read once leave L1 to what is read again.
__device__ __forceinline__ void load_once(const float* p, Raw8<float>& r, bool wide) {
    if (wide)
        asm volatile("ld.global.L1::no_allocate.v8.f32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                     : "=f"(r.a.x), "=f"(r.a.y), "=f"(r.a.z), "=f"(r.a.w), "=f"(r.b.x), "=f"(r.b.y), "=f"(r.b.z), "=f"(r.b.w)
                     : "l"(p));
    else
        load_raw(p, r);
}
__device__ __forceinline__ void load_once(const __nv_bfloat16* p, Raw8<__nv_bfloat16>& r, bool) {
    asm volatile("ld.global.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];"
                 : "=r"(r.a.x), "=r"(r.a.y), "=r"(r.a.z), "=r"(r.a.w)
                 : "l"(p));
}
__device__ __forceinline__ bool is_wide(const void* p) { return ((uintptr_t)p & 31) == 0; }
__device__ __forceinline__ void load_raw(const __nv_bfloat16* p, Raw8<__nv_bfloat16>& r, bool = true) {
    r.a = *reinterpret_cast<const uint4*>(p);
}
__device__ __forceinline__ void widen8(const Raw8<float>& r, float (&v)[8]) {
    v[0] = r.a.x; v[1] = r.a.y; v[2] = r.a.z; v[3] = r.a.w;
    v[4] = r.b.x; v[5] = r.b.y; v[6] = r.b.z; v[7] = r.b.w;
}
__device__ __forceinline__ void widen8(const Raw8<__nv_bfloat16>& r, float (&v)[8]) {
    const uint32_t w[4] = {r.a.x, r.a.y, r.a.z, r.a.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[2 * i] = __uint_as_float(w[i] << 16);
        v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
}
template <typename T> __device__ __forceinline__ void load8(const T* p, float (&v)[8], bool wide = false) {
    Raw8<T> r;
    load_raw(p, r, wide);
    widen8(r, v);
}

// The largest of three magnitudes, NaN kept.
__device__ __forceinline__ float max_abs(float a, float b, float c) {
    float d;
    asm("max.NaN.abs.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
    return d;
}
__device__ __forceinline__ float absmax8(const float (&v)[8]) {
    return max_abs(max_abs(max_abs(v[0], v[1], v[2]), v[3], v[4]), max_abs(v[5], v[6], v[7]), 0.f);
}

// The eight quotients by a scale outside the range of store8's shorter way.
static __device__ __noinline__ uint2 quotients(float4 a, float4 b, float s) {
    return make_uint2(e4m3x4(a.x / s, a.y / s, a.z / s, a.w / s), e4m3x4(b.x / s, b.y / s, b.z / s, b.w / s));
}

// The eight quotients by s, in e4m3.  With r the correctly rounded reciprocal of s,
// t = x r corrected once by its remainder, t + (x - t s) r, is the correctly rounded
// quotient (Markstein, "Computation of elementary functions on the IBM RISC
// System/6000 processor", 1990) as long as nothing underflows that matters.  Three
// instructions an element and little code: eight divisions a lane were what the
// kernel waited for, and their code what a short call fetched (1576 x 3072 bf16 8.2
// us, now 4.2).
__device__ __forceinline__ void store8(uint8_t* q, const float (&v)[8], float s) {
    uint2 w;
    const float by = s == 0.f ? 1.f : s;           // a block of zeros (or one so small that its scale is)
    if (by >= 0x1p-100f && by < INFINITY) {
        const float r = 1.0f / by;
        float y[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float t = v[i] * r;
            y[i] = fmaf(fmaf(-t, by, v[i]), r, t);
        }
        w = make_uint2(e4m3x4(y[0], y[1], y[2], y[3]), e4m3x4(y[4], y[5], y[6], y[7]));
    } else {
        w = quotients(make_float4(v[0], v[1], v[2], v[3]), make_float4(v[4], v[5], v[6], v[7]), s);
    }
    *reinterpret_cast<uint2*>(q) = w;
}

// Blocks of a kernel that the device holds at a time.
template <class K>
int resident_blocks(const Ctx* c, K kernel, int threads) {
    int n = 0;
    if (cudaOccupancyMaxActiveBlocksPerMultiprocessor(&n, kernel, threads, 0) != cudaSuccess || n < 1) {
        cudaGetLastError();
        n = 1;
    }
    return n * c->num_sms;
}

// ---------------------------------------------------------------- four bits
// Scales of 16 columns lie in pieces of 512 bytes, for 128 rows and 64 columns each:
// byte (row % 32) * 16 + (row / 32 % 4) * 4 + (column / 16) % 4, the order in which
// the tensor core takes them.  A word holds the four scales of a row's 64 columns.
constexpr int kPiece4 = 512, kPieceCols4 = 64;
// The widest matrix of the e2m1 operators (as kMaxWidth8).
constexpr int kMaxWidth4 = 0x7fffffff - 511;
constexpr int kMaxRows4 = 0x7fffffff - 127;        // rounded up to 128 rows still an int
constexpr float kRow4 = 1.0f / 2688;     // a row's scale of its largest magnitude: 6 (e2m1) * 448 (e4m3) steps

__device__ __forceinline__ size_t piece_word4(int row, int piece, int pieces) {
    return ((size_t)(row >> 7) * pieces + piece) * (kPiece4 / 4) + (row & 31) * 4 + (row >> 5 & 3);
}

// A row's scale from its largest magnitude: 0 where that is below 2^-100 (no
// intermediate below is then subnormal), NaN where it is infinite or NaN.
__device__ __forceinline__ float row_scale4(float top) {
    return !(top < INFINITY) ? __int_as_float(0x7fffffff) : (top < 0x1p-100f ? 0.f : top * kRow4);
}

// Eight values to e2m1, the first in the low bits; to nearest even, beyond 6 saturated.
__device__ __forceinline__ uint32_t e2m1x8(const float (&y)[8]) {
    uint32_t r;
    asm("{\n .reg .b8 a, b, c, d;\n"
        " cvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\n cvt.rn.satfinite.e2m1x2.f32 b, %4, %3;\n"
        " cvt.rn.satfinite.e2m1x2.f32 c, %6, %5;\n cvt.rn.satfinite.e2m1x2.f32 d, %8, %7;\n"
        " mov.b32 %0, {a, b, c, d};\n}"
        : "=r"(r)
        : "f"(y[0]), "f"(y[1]), "f"(y[2]), "f"(y[3]), "f"(y[4]), "f"(y[5]), "f"(y[6]), "f"(y[7]));
    return r;
}

// Their values.
__device__ __forceinline__ void e2m1_values(uint32_t q, float (&v)[8]) {
    uint32_t h[4];
    asm("{\n .reg .b8 a, b, c, d;\n mov.b32 {a, b, c, d}, %4;\n"
        " cvt.rn.f16x2.e2m1x2 %0, a;\n cvt.rn.f16x2.e2m1x2 %1, b;\n"
        " cvt.rn.f16x2.e2m1x2 %2, c;\n cvt.rn.f16x2.e2m1x2 %3, d;\n}"
        : "=r"(h[0]), "=r"(h[1]), "=r"(h[2]), "=r"(h[3])
        : "r"(q));
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&h[i]));
        v[2 * i] = f.x;
        v[2 * i + 1] = f.y;
    }
}

// A lane's 8 elements, rounded to the model's type.
__device__ __forceinline__ void put8(float* p, const float (&v)[8], bool wide = false) {
    if (wide) {
        asm volatile("st.global.v8.f32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "f"(v[0]), "f"(v[1]), "f"(v[2]),
                     "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7])
                     : "memory");
        return;
    }
    reinterpret_cast<float4*>(p)[0] = make_float4(v[0], v[1], v[2], v[3]);
    reinterpret_cast<float4*>(p)[1] = make_float4(v[4], v[5], v[6], v[7]);
}
__device__ __forceinline__ void put8(__nv_bfloat16* p, const float (&v)[8], bool = true) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const __nv_bfloat162 h = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
        w[i] = *reinterpret_cast<const uint32_t*>(&h);
    }
    *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
}

// A row's scale, 6 times it and the reciprocal of that.
struct Row4 {
    float row, six, by_six;
    bool live;                                     // neither 0 nor NaN
    __device__ __forceinline__ explicit Row4(float top)
        : row(row_scale4(top)), six(6.f * row), by_six(1.0f / six), live(row > 0.f) {}
};

// IEEE's quotient of a and a row's six: by its reciprocal and remainder (Markstein, see
// store8) as long as nothing that matters underflows; out of line below that.
static __device__ __noinline__ float small_quotient(float a, float six) { return a / six; }

// A lane's 8 neighbouring columns of a row (two lanes a scale, eight a word of
// scales) to codes and scales; `top`: their largest magnitude.  The whole warp calls it;
// lanes past the row's end (!in) hold zeros; `word` is looked at in every eighth lane.
__device__ __forceinline__ void store_fp4(const float (&v)[8], float top, const Row4& r, bool in, uint32_t* codes, uint32_t* word) {
    top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
    const float t = top * r.by_six;
    float quotient = fmaf(fmaf(-t, r.six, top), r.by_six, t);
    if (r.six < 0x1p-80f) quotient = small_quotient(top, r.six);       // (the row's, so the warp's)
    uint32_t s;
    float scale;
    asm("{\n .reg .b16 p, h;\n .reg .b32 w;\n cvt.rn.satfinite.e4m3x2.f32 p, %3, %2;\n cvt.rn.f16x2.e4m3x2 w, p;\n"
        " mov.b32 {h, _}, w;\n cvt.f32.f16 %1, h;\n cvt.u32.u16 %0, p;\n}"
        : "=r"(s), "=f"(scale)
        : "f"(r.live ? quotient : 0.f), "f"(0.f));
    const float step = scale * r.row;
    const float by = step > 0.f ? 1.0f / step : 0.f;
    float y[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = v[i] * by;
    const uint32_t q = e2m1x8(y);
    if (in) *codes = r.live ? q : 0u;              // (a NaN's or infinity's row)
    s |= __shfl_down_sync(0xffffffffu, s, 2) << 8;
    s |= __shfl_down_sync(0xffffffffu, s, 4) << 16;
    if (in && (threadIdx.x & 7) == 0) *word = s;
}

}  // namespace wdc
