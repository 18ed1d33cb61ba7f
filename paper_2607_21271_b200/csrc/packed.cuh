// Packed float arithmetic and the special-function operations as single instructions.
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

namespace eql {

// Two floats as one operand of a packed operation (sm_100's f32x2 forms): one issue slot instead of two, of which kernels that move memory
// and compute a little run out before anything else.  Each half is rounded as by the plain operation.
__device__ __forceinline__ float2 pair(float v) { return make_float2(v, v); }
#define EQL_PACKED(name, op)                                                                                                     \
    __device__ __forceinline__ float2 name(float2 a, float2 b) {                                                                 \
        float2 d;                                                                                                                \
        asm(op ".rn.f32x2 %0, %1, %2;" : "=l"(reinterpret_cast<uint64_t&>(d)) : "l"(reinterpret_cast<uint64_t&>(a)), "l"(reinterpret_cast<uint64_t&>(b))); \
        return d;                                                                                                                \
    }
EQL_PACKED(add2, "add")
EQL_PACKED(mul2, "mul")
#undef EQL_PACKED
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
    float2 d;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(reinterpret_cast<uint64_t&>(d)) : "l"(reinterpret_cast<uint64_t&>(a)), "l"(reinterpret_cast<uint64_t&>(b)),
        "l"(reinterpret_cast<uint64_t&>(c)));
    return d;
}
__device__ __forceinline__ float2 sub2(float2 a, float2 b) { return fma2(b, pair(-1.0f), a); }

// The special-function unit's exponential and reciprocal, good to 2^-22; subnormals count as zero.
__device__ __forceinline__ float exp2_fast(float v) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
    return r;
}
__device__ __forceinline__ float reciprocal(float v) {
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
    return r;
}
// The larger one, NaN where either is.
__device__ __forceinline__ float fmax_nan(float a, float b) {
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ float2 exp2_fast(float2 v) { return make_float2(exp2_fast(v.x), exp2_fast(v.y)); }
__device__ __forceinline__ float2 reciprocal(float2 v) { return make_float2(reciprocal(v.x), reciprocal(v.y)); }

}  // namespace eql
