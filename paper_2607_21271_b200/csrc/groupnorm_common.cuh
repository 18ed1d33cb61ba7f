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
#include "packed.cuh"
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
constexpr int kWarpNormShared = 32 * 1024;        // 256 lanes x 2 vectors (128 x 4) x 8 sums x 8 bytes
WarpNorm warp_norm_plan(const NormShape& s, eql_dtype_t dtype, bool backward);
cudaError_t launch_warp_norm(const NormShape& s, const WarpNorm& w, eql_dtype_t dtype, const void* x, const void* gamma, const void* beta,
                             const int32_t* lengths, void* y, float* stats, cudaStream_t stream);
// parts: float2 [ctas][C], the CTAs' sums of dz and dz * xh
cudaError_t launch_warp_gradient(const NormShape& s, const WarpNorm& w, eql_dtype_t dtype, const void* x, const void* dy, const void* gamma,
                                 const void* beta, const int32_t* lengths, const float* stats, void* dx, float* parts, cudaStream_t stream);

// Units resident in shared memory (groupnorm_resident.cu): a unit is one instance's part of a block of groups.
// e / d for e below 2^16 and d up to 2^16, by a reciprocal: ceil(2^32 / d).
struct Divisor {
    unsigned d, inverse;
    __host__ __device__ Divisor() : d(1), inverse(0) {}
    __host__ __device__ explicit Divisor(unsigned by) : d(by), inverse(by > 1 ? 0xffffffffu / by + 1 : 0) {}
    __device__ __forceinline__ unsigned operator()(unsigned e) const { return d > 1 ? __umulhi(e, inverse) : e; }
};
// The same for all e and d of 32 bits: ceil(2^64 / d).
struct WideDivisor {
    unsigned d;
    unsigned long long inverse;
    __host__ __device__ WideDivisor() : d(1), inverse(0) {}
    __host__ __device__ explicit WideDivisor(unsigned by) : d(by), inverse(by > 1 ? ~0ull / by + 1 : 0) {}
    __device__ __forceinline__ unsigned operator()(unsigned e) const { return d > 1 ? (unsigned)__umul64hi(e, inverse) : e; }
};
struct ResidentNorm {
    bool supported;
    int groups, blocks;       // groups of a block, blocks of a row
    int cluster, threads;     // CTAs of a unit, threads of a CTA
    int instances;            // instances that are worked on side by side
    int64_t rows;             // rows of a CTA
    int form;                 // N of the kernels that are launched (see Runs), by which everything a thread puts side by side is laid out
    int run, sums, share;     // backward: neighbouring elements summed up in a thread, sums of a vector, lanes that add up a channel
    int slot_bytes, side_offset, shared_bytes;
    Divisor tuple, width, entry, runs;        // T; elements of a group; entries of a group in a row (its vectors, or elements); runs of a tuple
    Divisor columns, lanes;   // of a full block
    WideDivisor by_cluster, by_blocks;
};
constexpr int kResidentShared = 220 * 1024;
ResidentNorm resident_norm_plan(const NormShape& s, eql_dtype_t dtype, bool backward);
cudaError_t launch_resident_norm(const NormShape& s, const ResidentNorm& r, eql_dtype_t dtype, const void* x, const void* gamma, const void* beta,
                                 const int32_t* lengths, void* y, float* stats, cudaStream_t stream);
// parts: float2 [instances * cluster][C], the CTAs' sums of dz and dz * xh
cudaError_t launch_resident_gradient(const NormShape& s, const ResidentNorm& r, eql_dtype_t dtype, const void* x, const void* dy, const void* gamma,
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

// A vector of 16 bytes as pairs of floats.
template <typename IO> struct NormIo;
template <> struct NormIo<float> {
    static constexpr int kVec = 4;
    static __device__ __forceinline__ void widen(const uint4& u, float2* f) {
        f[0] = make_float2(__uint_as_float(u.x), __uint_as_float(u.y));
        f[1] = make_float2(__uint_as_float(u.z), __uint_as_float(u.w));
    }
    static __device__ __forceinline__ uint4 narrow(const float2* f) {
        return make_uint4(__float_as_uint(f[0].x), __float_as_uint(f[0].y), __float_as_uint(f[1].x), __float_as_uint(f[1].y));
    }
    static __device__ __forceinline__ float one(const float* p, int i) { return p[i]; }
};
template <> struct NormIo<__half> {
    static constexpr int kVec = 8;
    static __device__ __forceinline__ void widen(const uint4& u, float2* f) {
        const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) f[i] = __half22float2(*reinterpret_cast<const __half2*>(&w[i]));
    }
    static __device__ __forceinline__ uint4 narrow(const float2* f) {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const __half2 h = __floats2half2_rn(f[i].x, f[i].y);
            w[i] = *reinterpret_cast<const uint32_t*>(&h);
        }
        return make_uint4(w[0], w[1], w[2], w[3]);
    }
    static __device__ __forceinline__ float one(const __half* p, int i) { return __half2float(p[i]); }
};
template <> struct NormIo<__nv_bfloat16> {
    static constexpr int kVec = 8;
    static __device__ __forceinline__ void widen(const uint4& u, float2* f) {
        const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) f[i] = make_float2(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xffff0000u));
    }
    static __device__ __forceinline__ uint4 narrow(const float2* f) {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const __nv_bfloat162 h = __floats2bfloat162_rn(f[i].x, f[i].y);
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
// The running form (Welford 1962) for columns of 2 P values, row after row: a fourth operation an element, and unlike with sums behind a
// fixed pivot it does not matter how far the first value lies from the rest.
template <int P>
struct RunningMoments {
    float rows = 0.0f;
    float2 mean[P] = {}, m2[P] = {};
    __device__ __forceinline__ void add(const float2* f) {
        rows += 1.0f;
        const float2 share = pair(reciprocal(rows));
#pragma unroll
        for (int j = 0; j < P; ++j) {
            const float2 d = sub2(f[j], mean[j]);
            mean[j] = fma2(d, share, mean[j]);
            m2[j] = fma2(d, sub2(f[j], mean[j]), m2[j]);
        }
    }
};
__device__ __forceinline__ float rstd_of(const Moments& v, float eps) { return rsqrtf((v.n > 0.0f ? __fdividef(v.m2, v.n) : 0.0f) + eps); }

// Entries of a vector of P pairs in N runs: one a run, or each element for itself.
constexpr int entries_of(int N, int P) { return N < P ? N : 2 * P; }
// What belongs to the elements of a vector in N equal runs: channels and groups begin where runs do.  N = 1 where the vector is of one
// channel, 2 where it is of two of half its length each, all pairs otherwise (and then each element for itself).
template <int N, int P>
struct Runs {
    float2 v[N];
    __device__ __forceinline__ const float2& of(int pair_index) const { return v[pair_index * N / P]; }
    __device__ __forceinline__ float2& of(int pair_index) { return v[pair_index * N / P]; }
    __device__ __forceinline__ void set(int entry, float value) {         // entry of kEntries
        if (N < P) v[entry] = pair(value);
        else (&v[entry / 2].x)[entry % 2] = value;
    }
    static constexpr int kEntries = entries_of(N, P), kLength = 2 * P / kEntries;      // (an entry's elements)
    // set(entry, its channel), and the same for groups, for the vector whose first element is element `at` of the channel or group `first`
    template <typename Set>
    static __device__ __forceinline__ void each(int first, int at, int length, Set&& set) {
#pragma unroll
        for (int e = 0; e < kEntries; ++e) {
            set(e, first);
            at += kLength;
            if (at >= length) { at -= length; ++first; }
        }
    }
};
// The N above for tuples of T elements, and the neighbouring elements of a vector that are of one channel (whatever the vector).
constexpr int runs_of(int T, int V) { return T % V == 0 ? 1 : T % (V / 2) == 0 ? 2 : V / 2; }
constexpr int run_length(int T, int V) { return T % V == 0 ? V : T % (V / 2) == 0 ? V / 2 : V % T == 0 ? T : 1; }

__device__ __forceinline__ int64_t positions_of(const int32_t* lengths, int64_t b, int64_t S) {
    if (!lengths) return S;
    const int64_t n = lengths[b];
    return n < 0 ? 0 : n > S ? S : n;
}


__device__ __forceinline__ float2 minus_abs(float2 v) { return make_float2(-fabsf(v.x), -fabsf(v.y)); }

// 1 / (1 + exp(-z)), good to 2^-22.  TOGETHER: by one reciprocal of the pair's product, which the two values then turn into each other's, so
// that the special-function unit has a quarter less to do; z is held at -41.5 from below for it, so that the product stays a float's (for
// the caller too: what the sigmoid is multiplied by must not grow on), and a NaN of one reaches the other, so it is for pairs of one
// channel.  (128 x 197 x 768 bfloat16 with SiLU, forward and backward: 59.3 -> 58.1 us.  GELU, whose polynomial keeps the multiplying
// units as busy, does not gain: 128 x 3136 x 384 490 -> 494.)
template <bool TOGETHER> __device__ __forceinline__ float2 sigmoid(float2& z) {
    if (TOGETHER) z = make_float2(fmax_nan(z.x, -41.5f), fmax_nan(z.y, -41.5f));
    const float2 d = add2(exp2_fast(mul2(z, pair(-1.44269504088896341f))), pair(1.0f));
    if (!TOGETHER) return reciprocal(d);
    return mul2(pair(reciprocal(d.x * d.y)), make_float2(d.y, d.x));
}
// Phi(-|z|) = erfc(|z| / sqrt 2) / 2 by the rational approximation 7.1.26 of Abramowitz and Stegun (error of erfc at most 1.5e-7, a float's
// at 1; falling with exp(-z^2 / 2) in the tail).  `density`: phi(z) = exp(-z^2 / 2) / sqrt(2 pi), its constant part of the exponent, and
// the polynomial's coefficients (halves of theirs) divided by it.
__device__ __forceinline__ float2 tail_of_normal(float2 z, float2* density) {
    constexpr float kPerDensity = 0.5f * 2.50662827463100050242f;
    const float2 t = reciprocal(fma2(minus_abs(z), pair(-0.3275911f * 0.70710678118654752f), pair(1.0f)));
    *density = exp2_fast(fma2(mul2(z, z), pair(-0.72134752044448170f), pair(-1.32574806473615915f)));
    float2 p = fma2(t, pair(kPerDensity * 1.061405429f), pair(kPerDensity * -1.453152027f));
    p = fma2(p, t, pair(kPerDensity * 1.421413741f));
    p = fma2(p, t, pair(kPerDensity * -0.284496736f));
    p = fma2(p, t, pair(kPerDensity * 0.254829592f));
    return mul2(mul2(p, t), *density);
}

// TOGETHER: the pair is of one channel.
template <int ACT, bool TOGETHER> __device__ __forceinline__ float2 activate(float2 z) {
    if (ACT == EQL_ACT_GELU) {                                // z Phi(z) = max(z, 0) - |z| Phi(-|z|)
        float2 density;
        const float2 q = tail_of_normal(z, &density);
        return fma2(minus_abs(z), q, make_float2(fmaxf(z.x, 0.0f), fmaxf(z.y, 0.0f)));
    }
    if (ACT == EQL_ACT_SILU) {
        const float2 p = sigmoid<TOGETHER>(z);
        return mul2(z, p);
    }
    return z;
}
template <int ACT, bool TOGETHER> __device__ __forceinline__ float2 slope(float2 z) {
    if (ACT == EQL_ACT_GELU) {                                // Phi(z) + z phi(z)
        float2 density;
        const float2 h = sub2(pair(0.5f), tail_of_normal(z, &density));
        const float2 cdf = add2(make_float2(copysignf(h.x, z.x), copysignf(h.y, z.y)), pair(0.5f));
        return fma2(z, density, cdf);
    }
    if (ACT == EQL_ACT_SILU) {
        const float2 p = sigmoid<TOGETHER>(z);
        return mul2(p, fma2(z, sub2(pair(1.0f), p), pair(1.0f)));
    }
    return pair(1.0f);
}

}  // namespace eql
