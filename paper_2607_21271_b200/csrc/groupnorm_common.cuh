// Group norm with an activation: what its kernels share - vectors of 16 bytes as floats, the merging of partial statistics, the
// activations and their slopes.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <climits>
#include <type_traits>

#include "eql_internal.h"
#include "ptx_sm100.cuh"

namespace eql {

// One norm, as the kernels see it.  A vector is 16 bytes: 8 elements of a 16-bit type, 4 of float.
struct NormShape {
    int T, C, groups, act;
    int D, width;             // elements of a row, and of a group's part of it
    int vectors;              // 16-byte vectors of a row
    int64_t B, S;
    float eps;
};

// Small units (groupnorm_warp.cu): a unit is one instance's part of one group.
struct WarpNorm {
    bool supported;
    int vectors, unit;        // 16-byte vectors of a row of the unit, and of the unit
    int lanes, each;          // lanes a unit has, vectors a lane (rounded up to what kernels exist for)
    int groups, instances;    // units that a CTA holds at a time: so many groups of so many instances
    int group_blocks, ctas;   // CTAs that cover all groups, and how many such sets there are
    int sums, shared_bytes;
};
constexpr int kWarpNormShared = 66 * 1024;        // 256 lanes x 4 vectors x 8 sums x 8 bytes, and some
WarpNorm warp_norm_plan(const NormShape& s, eql_dtype_t dtype, bool backward);
cudaError_t launch_warp_norm(const NormShape& s, const WarpNorm& w, eql_dtype_t dtype, const void* x, const void* gamma, const void* beta,
                             const int32_t* lengths, void* y, float* stats, cudaStream_t stream);
// parts: float2 [ctas][C], the CTAs' sums of dz and dz * xh
cudaError_t launch_warp_gradient(const NormShape& s, const WarpNorm& w, eql_dtype_t dtype, const void* x, const void* dy, const void* gamma,
                                 const void* beta, const int32_t* lengths, const float* stats, void* dx, float* parts, cudaStream_t stream);

template <typename F>
cudaError_t dispatch_act(int act, F&& f) {
    if (act == EQL_ACT_GELU) return f(std::integral_constant<int, EQL_ACT_GELU>{});
    if (act == EQL_ACT_SILU) return f(std::integral_constant<int, EQL_ACT_SILU>{});
    return f(std::integral_constant<int, EQL_ACT_NONE>{});
}
template <typename F>
cudaError_t dispatch_io(int dtype, F&& f) {
    if (dtype == EQL_FP16) return f(__half{});
    if (dtype == EQL_BF16) return f(__nv_bfloat16{});
    return f(float{});
}

template <typename IO> struct NormIo;
template <> struct NormIo<float> {
    static constexpr int kVec = 4;
    static __device__ __forceinline__ void widen(const uint4& u, float* f) {
        f[0] = __uint_as_float(u.x); f[1] = __uint_as_float(u.y); f[2] = __uint_as_float(u.z); f[3] = __uint_as_float(u.w);
    }
    static __device__ __forceinline__ uint4 narrow(const float* f) {
        return make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
    }
    static __device__ __forceinline__ float one(const float* p, int i) { return p[i]; }
};
template <> struct NormIo<__half> {
    static constexpr int kVec = 8;
    static __device__ __forceinline__ void widen(const uint4& u, float* f) {
        const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 p = __half22float2(*reinterpret_cast<const __half2*>(&w[i]));
            f[2 * i] = p.x; f[2 * i + 1] = p.y;
        }
    }
    static __device__ __forceinline__ uint4 narrow(const float* f) {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const __half2 h = __floats2half2_rn(f[2 * i], f[2 * i + 1]);
            w[i] = *reinterpret_cast<const uint32_t*>(&h);
        }
        return make_uint4(w[0], w[1], w[2], w[3]);
    }
    static __device__ __forceinline__ float one(const __half* p, int i) { return __half2float(p[i]); }
};
template <> struct NormIo<__nv_bfloat16> {
    static constexpr int kVec = 8;
    static __device__ __forceinline__ void widen(const uint4& u, float* f) {
        const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            f[2 * i] = __uint_as_float(w[i] << 16);
            f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
        }
    }
    static __device__ __forceinline__ uint4 narrow(const float* f) {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const __nv_bfloat162 h = __floats2bfloat162_rn(f[2 * i], f[2 * i + 1]);
            w[i] = *reinterpret_cast<const uint32_t*>(&h);
        }
        return make_uint4(w[0], w[1], w[2], w[3]);
    }
    static __device__ __forceinline__ float one(const __nv_bfloat16* p, int i) { return __bfloat162float(p[i]); }
};

// Mean and sum of squared distances from it, of n values; merged pairwise (Chan, Golub and LeVeque 1979), which loses nothing where
// the mean is far larger than the spread.
struct Moments {
    float n, mean, m2;
};
__device__ __forceinline__ Moments merge(const Moments& a, const Moments& b) {
    const float n = a.n + b.n;
    if (!(b.n > 0.0f)) return a;
    if (!(a.n > 0.0f)) return b;
    const float d = b.mean - a.mean, share = __fdividef(b.n, n);
    return Moments{n, fmaf(d, share, a.mean), a.m2 + b.m2 + d * d * a.n * share};
}
__device__ __forceinline__ Moments warp_merge(Moments v) {
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) {
        const Moments o{__shfl_down_sync(0xffffffffu, v.n, d), __shfl_down_sync(0xffffffffu, v.mean, d), __shfl_down_sync(0xffffffffu, v.m2, d)};
        v = merge(v, o);
    }
    return v;                 // lane 0's
}
// The running form (Welford 1962) for columns of V values, row after row: a fourth operation an element, and unlike with sums behind a
// fixed pivot it does not matter how far the first value lies from the rest.
template <int V>
struct RunningMoments {
    float rows = 0.0f, mean[V] = {}, m2[V] = {};
    __device__ __forceinline__ void add(const float* f) {
        rows += 1.0f;
        const float share = __fdividef(1.0f, rows);
#pragma unroll
        for (int j = 0; j < V; ++j) {
            const float d = f[j] - mean[j];
            mean[j] = fmaf(d, share, mean[j]);
            m2[j] = fmaf(d, f[j] - mean[j], m2[j]);
        }
    }
};
__device__ __forceinline__ float rstd_of(const Moments& v, float eps) { return 1.0f / sqrtf((v.n > 0.0f ? v.m2 / v.n : 0.0f) + eps); }

__device__ __forceinline__ int64_t positions_of(const int32_t* lengths, int64_t b, int64_t S) {
    if (!lengths) return S;
    const int64_t n = lengths[b];
    return n < 0 ? 0 : n > S ? S : n;
}

template <int ACT> __device__ __forceinline__ float activate(float z) {
    if (ACT == EQL_ACT_GELU) return 0.5f * z * (1.0f + erff(z * 0.70710678118654752440f));
    if (ACT == EQL_ACT_SILU) return __fdividef(z, 1.0f + __expf(-z));
    return z;
}
template <int ACT> __device__ __forceinline__ float slope(float z) {
    if (ACT == EQL_ACT_GELU)
        return 0.5f * (1.0f + erff(z * 0.70710678118654752440f)) + z * 0.39894228040143267794f * __expf(-0.5f * z * z);
    if (ACT == EQL_ACT_SILU) {
        const float p = __fdividef(1.0f, 1.0f + __expf(-z));
        return p * fmaf(z, 1.0f - p, 1.0f);
    }
    return 1.0f;
}

}  // namespace eql
